// C entry points of answering models: appends to a paged cache, attention over it, sampling.  Every argument that lies on the host is checked before anything
// is launched; arrays on the device are checked by the kernels.
#include <hip/hip_runtime.h>

#include <cmath>
#include <vector>

#include "answer.hpp"
#include "api_jobs.hpp"
#include "salus.h"

using namespace salus;

namespace {

const char *const kHeads = "Hq must be a positive multiple of Hkv, at most 4096, D 32, 64, 96, 128, 192 or 256";
const char *const kPages = "pages have a power of two of tokens from 32 to 1024, a cache fewer than 2^31 pages and at least one, a page table fewer than 2^31 entries and at least one a sequence";
const char *const kRows = "M and n_seqs must be positive, M Hq + 32 n_seqs Hkv below 2^31";

bool heads_ok(uint32_t Hq, uint32_t Hkv, uint32_t D)
{
    return Hkv != 0 && Hq != 0 && Hq <= 4096 && Hq % Hkv == 0 && (D == 32 || D == 64 || D == 96 || D == 128 || D == 192 || D == 256);
}
bool below_2_31(uint64_t v) { return v < 1ull << 31; }
bool page_ok(uint32_t page) { return page >= 32 && page <= 1024 && (page & (page - 1)) == 0; }
bool seqs_ok(uint32_t M, uint32_t n_seqs, uint32_t Hq, uint32_t Hkv)
{
    return rows_ok(M) && n_seqs != 0 && below_2_31((uint64_t)M * Hq + 32ull * n_seqs * Hkv);
}

template <typename Desc>
const char *cache_wrong(const Desc &d)
{
    if (!heads_ok(d.Hq, d.Hkv, d.D)) return kHeads;
    if (!page_ok(d.page) || d.n_pages == 0 || !below_2_31(d.n_pages) || d.max_pages == 0 || !below_2_31((uint64_t)d.max_pages * d.n_seqs)) return kPages;
    if (!seqs_ok(d.M, d.n_seqs, d.Hq, d.Hkv)) return kRows;
    return nullptr;
}

// The arrays of a job's sequences: ranges of its lane, and what the kernels need of them.
template <typename Desc>
Sequences sequences(const Desc &d, const Placed &at, Ranges &lane)
{
    lane.read(d.starts_off, 4 * ((uint64_t)d.n_seqs + 1));
    lane.read(d.lens_off, 4ull * d.n_seqs);
    lane.read(d.table_off, 4ull * d.n_seqs * d.max_pages);
    return {(const int32_t *)(at.lane + d.starts_off), (const int32_t *)(at.lane + d.lens_off), (const int32_t *)(at.lane + d.table_off),
            d.n_seqs, d.M, d.max_pages, d.n_pages, d.Hq, d.Hkv, d.D, (uint32_t)__builtin_ctz(d.page)};
}

int32_t append(salus_pool_t *pool, const salus_append_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<AppendProblem> problems;
    problems.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_append_desc &d, const Placed &at) -> const char * {
        if (const char *wrong = cache_wrong(d)) return wrong;
        if (d.rotary % 2 || d.rotary > d.D) return "rotary must be even and at most D";
        if (d.layout != SALUS_ROTARY_HALF && d.layout != SALUS_ROTARY_INTERLEAVED) return "bad rotary layout";
        if (!std::isfinite(d.magnitude)) return "magnitude must be finite";
        if ((d.rotary == 0) != (d.freq_off == SALUS_ABSENT)) return "frequencies are given exactly if something is rotated";
        const uint64_t M = d.M, cache = salus_cache_bytes(d.n_pages, d.Hkv, d.page, d.D);
        Ranges persist(at.P), lane(at.lane_size);
        persist.write(d.k_off, cache);
        persist.write(d.v_off, cache);
        if (d.rotary) persist.read(d.freq_off, 4ull * d.rotary);
        lane.read(d.x_off, M * (d.Hq + 2ull * d.Hkv) * d.D * 2);
        lane.write(d.q_off, M * d.Hq * d.D * 2);
        const Sequences seq = sequences(d, at, lane);
        if (persist.outside()) return kCache;
        if (lane.outside()) return kLane;
        if (persist.overlap() || lane.overlap()) return kOverlap;
        problems.push_back({seq, at.lane + d.x_off, at.lane + d.q_off, at.persist + d.k_off, at.persist + d.v_off,
                            (const double *)at_or_null(at.persist, d.freq_off), d.rotary, d.layout == SALUS_ROTARY_INTERLEAVED, d.magnitude, 0});
        return nullptr;
    });
    if (rc) return rc;
    return launched(pool, launch_append(problems.data(), n, stream, launch_counter(pool)));
}

int32_t attention(salus_pool_t *pool, const salus_attention_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<AttentionProblem> problems;
    problems.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_attention_desc &d, const Placed &at) -> const char * {
        if (const char *wrong = cache_wrong(d)) return wrong;
        if (d.max_len == 0 || d.max_len > (uint64_t)d.max_pages * d.page || d.max_len >= 1u << 30) return "max_len must be positive, below 2^30 and at most max_pages * page";
        const float scale = d.scale * 1.4426950408889634f;       // of powers of two
        if (!(d.scale > 0.0f) || !std::isfinite(scale)) return "scale must be positive, and finite times log2(e)";
        const uint64_t M = d.M, cache = salus_cache_bytes(d.n_pages, d.Hkv, d.page, d.D),
                       // what this call uses, which may be less than the room that the host function wants for it and all smaller ones
                       work = up256(4 * attention_work_floats(d.M, d.Hq, d.D, attention_parts(d.M, d.n_seqs, d.Hq, d.Hkv, d.D, d.max_len, 0)));
        Ranges persist(at.P), lane(at.lane_size);
        persist.read(d.k_off, cache);
        persist.read(d.v_off, cache);
        lane.read(d.q_off, M * d.Hq * d.D * 2);
        lane.write(d.y_off, M * d.Hq * d.D * 2);
        if (work) lane.write(d.work_off, work);
        const Sequences seq = sequences(d, at, lane);
        if (persist.outside()) return kCache;
        if (lane.outside()) return kLane;
        if (lane.overlap()) return kOverlap;
        const AttentionParts parts = attention_parts(d.M, d.n_seqs, d.Hq, d.Hkv, d.D, d.max_len, d.window);
        problems.push_back({seq, at.lane + d.q_off, at.persist + d.k_off, at.persist + d.v_off, at.lane + d.y_off,
                            work ? (float *)(at.lane + d.work_off) : nullptr, d.max_len, d.window, scale, parts.part, parts.parts, parts.columns});
        return nullptr;
    });
    if (rc) return rc;
    return launched(pool, launch_attention(problems.data(), n, stream, launch_counter(pool)));
}

constexpr uint32_t kMostLogits = 1u << 19;

int32_t sample(salus_pool_t *pool, const salus_sample_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<SampleProblem> problems;
    problems.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_sample_desc &d, const Placed &at) -> const char * {
        if (!rows_ok(d.M)) return "M must be positive and below 2^31";
        if (d.V == 0 || d.V > kMostLogits || d.ld % 8 || d.ld < d.V) return "V must be 1 - 2^19, ld a multiple of 8 and at least V";
        if (d.dtype != SALUS_F32 && d.dtype != SALUS_BF16) return "bad dtype";
        const uint64_t M = d.M, size = d.dtype == SALUS_BF16 ? 2 : 4;
        Ranges lane(at.lane_size);
        lane.read(d.logits_off, M * d.ld * size);
        lane.read(d.params_off, 16 * M);
        lane.read(d.u_off, 4 * M);
        lane.write(d.tokens_off, 4 * M);
        lane.write(d.work_off, salus_sample_work_bytes(d.M, d.V));
        if (lane.outside()) return kLane;
        if (lane.overlap()) return kOverlap;
        problems.push_back({at.lane + d.logits_off, (const uint32_t *)(at.lane + d.params_off), (const float *)(at.lane + d.u_off),
                            (int32_t *)(at.lane + d.tokens_off), at.lane + d.work_off, d.M, d.V, d.ld, d.dtype == SALUS_BF16});
        return nullptr;
    });
    if (rc) return rc;
    return launched(pool, launch_sample(problems.data(), n, stream, launch_counter(pool)));
}

}  // namespace

extern "C" {

uint64_t salus_cache_bytes(uint32_t n_pages, uint32_t Hkv, uint32_t page, uint32_t D)
{
    if (!heads_ok(Hkv, Hkv, D) || !page_ok(page) || !below_2_31(n_pages)) return 0;
    return 2ull * n_pages * Hkv * page * D;
}

int32_t salus_rotary_frequencies(double *out, uint32_t rotary, double base, int32_t scaling, double factor, double trained, double slow, double fast)
{
    if (!out || rotary == 0 || rotary % 2 || rotary > 256 || !std::isfinite(base) || !(base > 1) || !std::isfinite(factor) || !(factor >= 1)) return SALUS_EINVAL;
    if (scaling < SALUS_ROTARY_PLAIN || scaling > SALUS_ROTARY_PARTS) return SALUS_EINVAL;
    if (scaling == SALUS_ROTARY_PARTS && !(std::isfinite(trained) && trained > 0 && slow >= 0 && fast > slow && std::isfinite(fast))) return SALUS_EINVAL;
    if (scaling == SALUS_ROTARY_BASE && rotary > 2) base *= std::pow(factor, rotary / (rotary - 2.0));
    for (uint32_t j = 0; j < rotary / 2; ++j) {
        double f = std::pow(base, -2.0 * j / rotary);
        if (scaling == SALUS_ROTARY_LINEAR) f /= factor;
        if (scaling == SALUS_ROTARY_PARTS) {
            const double turns = trained * f / 6.283185307179586, r = std::fmin(std::fmax((turns - slow) / (fast - slow), 0.0), 1.0);
            f = r * f + (1 - r) * f / factor;
        }
        out[j] = f;
    }
    return SALUS_OK;
}

int32_t salus_grouped_append(salus_pool_t *pool, const salus_append_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return append(pool, descs, n, (hipStream_t)stream); });
}

uint64_t salus_attention_work_bytes(uint32_t M, uint32_t n_seqs, uint32_t Hq, uint32_t Hkv, uint32_t D, uint32_t max_len)
{
    if (!heads_ok(Hq, Hkv, D) || !seqs_ok(M, n_seqs, Hq, Hkv) || max_len == 0 || max_len >= 1u << 30) return 0;
    return up256(4 * attention_room_floats(M, Hq, Hkv, D, max_len));
}

int32_t salus_grouped_attention(salus_pool_t *pool, const salus_attention_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return attention(pool, descs, n, (hipStream_t)stream); });
}

uint64_t salus_sample_work_bytes(uint32_t M, uint32_t V)
{
    if (!rows_ok(M) || V == 0 || V > kMostLogits) return 0;
    return up256(sample_work_bytes(M, V));
}

int32_t salus_grouped_sample(salus_pool_t *pool, const salus_sample_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return sample(pool, descs, n, (hipStream_t)stream); });
}

}  // extern "C"
