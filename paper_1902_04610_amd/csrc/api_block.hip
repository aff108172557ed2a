// C entry points of the transformer blocks: gated feed-forward blocks, dense layers with bias and residual, gradient clipping.
// Every argument is checked before anything is launched.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>
#include <vector>

#include "api.hpp"
#include "block.hpp"
#include "salus.h"

using namespace salus;

namespace {

uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }

// The ranges of one job's call inside its lane (or its persistent block): what is wrong with them, or null.
class Ranges {
public:
    explicit Ranges(uint64_t size) : size_(size) {}
    void read(uint64_t off, uint64_t len) { add(off, len, false); }
    void write(uint64_t off, uint64_t len) { add(off, len, true); }
    bool outside() const { return outside_; }
    // Does a written range meet another one?  Sorted by their beginnings, a range meets an earlier one if it begins before the largest
    // end among them; only the two largest ends, of any range and of a written one, are needed.
    bool overlap()
    {
        if (!std::is_sorted(r_.begin(), r_.end(), before)) std::sort(r_.begin(), r_.end(), before);
        uint64_t end = 0, written = 0;
        for (const Range &r : r_) {
            if (r.off < written || (r.written && r.off < end)) return true;
            end = std::max(end, r.off + r.len);
            if (r.written) written = std::max(written, r.off + r.len);
        }
        return false;
    }

private:
    struct Range { uint64_t off, len; bool written; };
    static bool before(const Range &a, const Range &b) { return a.off < b.off; }
    void add(uint64_t off, uint64_t len, bool written)
    {
        if (off % 16 || off > size_ || len > size_ - off) outside_ = true;
        else r_.push_back({off, len, written});
    }
    uint64_t size_;
    bool outside_ = false;
    std::vector<Range> r_;
};

// A call's body, if there is anything to do and to do it with.  Nothing is thrown across the C boundary.
template <typename Desc, typename F>
int32_t guarded(salus_pool_t *pool, const Desc *descs, uint32_t n, F body)
{
    if (!pool) return SALUS_EINVAL;
    if (n == 0) return SALUS_OK;
    try {
        if (!descs) return pool_error(pool, SALUS_EINVAL, "null descriptor array");
        if (!has_device(pool)) return pool_error(pool, SALUS_EINVAL, "pool has no device memory");
        return body();
    } catch (const std::bad_alloc &) {
        return SALUS_ENOMEM;
    }
}

bool width_ok(uint64_t w) { return w != 0 && w % 8 == 0 && w < kTiledMaxWidth; }
bool rows_ok(uint32_t m) { return m != 0 && m < 1u << 31; }
bool act_ok(int32_t act) { return act >= SALUS_ACT_NONE && act <= SALUS_ACT_SILU; }

const char *const kWidths = "K, F and N must be positive multiples of 8 below 2^22 (2 F as well), M positive and below 2^31";
const char *const kAct = "bad activation";
const char *const kWeights = "weights outside the persistent block";
const char *const kLane = "buffer outside the job's lane";
const char *const kOverlap = "a buffer that is written overlaps another one";

template <typename Desc, typename Place>
int32_t for_jobs(salus_pool_t *pool, const Desc *descs, uint32_t n, Place place)
{
    std::vector<int32_t> lanes_used;
    lanes_used.reserve(n);
    for (uint32_t i = 0; i < n; ++i) {
        Placed at;
        if (int32_t rc = place_job(pool, descs[i].job, lanes_used, &at)) return rc;
        if (const char *wrong = place(descs[i], at)) return pool_error(pool, SALUS_EINVAL, wrong);
    }
    return SALUS_OK;
}

int32_t launched(salus_pool_t *pool, hipError_t e)
{
    return e == hipSuccess ? SALUS_OK : pool_error(pool, SALUS_EHIP, hipGetErrorString(e));
}

char *at_or_null(char *base, uint64_t off) { return off == SALUS_ABSENT ? nullptr : base + off; }

int32_t gated_forward(salus_pool_t *pool, const salus_gated_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<BlockProblem> in, out;
    in.reserve(n);
    out.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_gated_desc &d, const Placed &at) -> const char * {
        if (!rows_ok(d.M) || !width_ok(d.K) || !width_ok(2ull * d.F) || !width_ok(d.F) || !width_ok(d.N)) return kWidths;
        if (!act_ok(d.act)) return kAct;
        const uint64_t M = d.M;
        Ranges weights(at.P), lane(at.lane_size);
        weights.read(d.w_in_off, 4ull * d.K * d.F);
        weights.read(d.w_out_off, 2ull * d.F * d.N);
        if (weights.outside()) return kWeights;
        lane.read(d.x_off, M * d.K * 2);
        lane.write(d.y_off, M * d.N * 2);
        lane.write(d.h_off, M * d.F * 2);
        if (d.r_off != SALUS_ABSENT && d.r_off != d.y_off) lane.read(d.r_off, M * d.N * 2);
        if (d.gu_off != SALUS_ABSENT) lane.write(d.gu_off, M * d.F * 8);
        if (lane.outside()) return kLane;
        if (lane.overlap()) return kOverlap;
        const uint32_t flags = kOutBf16 | (d.gu_off != SALUS_ABSENT ? kReadAgain : 0u);
        in.push_back({at.persist + d.w_in_off, at.lane + d.x_off, at.lane + d.h_off, nullptr, (float *)at_or_null(at.lane, d.gu_off), nullptr,
                      d.M, d.K, d.F, (uint32_t)d.act | flags});
        out.push_back({at.persist + d.w_out_off, at.lane + d.h_off, at.lane + d.y_off, at_or_null(at.lane, d.r_off), nullptr, nullptr, d.M, d.F, d.N,
                       (uint32_t)SALUS_ACT_NONE | flags});
        return nullptr;
    });
    if (rc) return rc;
    const bool cached = weights_cached(pool);
    hipError_t e = launch_block_gated(in.data(), n, cached, stream, launch_counter(pool));
    if (e == hipSuccess) e = launch_block_dense(out.data(), n, cached, stream, launch_counter(pool));
    return launched(pool, e);
}

int32_t gated_backward(salus_pool_t *pool, const salus_gated_grad_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<BlockProblem> gate, input;
    std::vector<WeightGradProblem> weight;
    gate.reserve(n);
    input.reserve(n);
    weight.reserve(2 * n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_gated_grad_desc &d, const Placed &at) -> const char * {
        if (!rows_ok(d.M) || !width_ok(d.K) || !width_ok(2ull * d.F) || !width_ok(d.F) || !width_ok(d.N)) return kWidths;
        if (!act_ok(d.act)) return kAct;
        const uint64_t M = d.M;
        Ranges weights(at.P), lane(at.lane_size);
        weights.read(d.w_in_off, 4ull * d.K * d.F);
        weights.read(d.w_out_off, 2ull * d.F * d.N);
        if (weights.outside()) return kWeights;
        lane.read(d.x_off, M * d.K * 2);
        lane.read(d.h_off, M * d.F * 2);
        lane.read(d.gu_off, M * d.F * 8);
        lane.read(d.dy_off, M * d.N * 2);
        if (d.dx_off != SALUS_ABSENT) lane.write(d.dx_off, M * d.K * 2);
        lane.write(d.dw_in_off, 4ull * d.K * d.F);
        lane.write(d.dw_out_off, 2ull * d.F * d.N);
        lane.write(d.work_off, salus_gated_grad_work_bytes(d.M, d.F));
        if (lane.outside()) return kLane;
        if (lane.overlap()) return kOverlap;
        char *dgu = at.lane + d.work_off, *dy = at.lane + d.dy_off;
        gate.push_back({at.persist + d.w_out_off, dy, dgu, nullptr, (float *)(at.lane + d.gu_off), nullptr, d.M, d.N, d.F, (uint32_t)d.act | kOutBf16});
        if (d.dx_off != SALUS_ABSENT)
            input.push_back({at.persist + d.w_in_off, dgu, at.lane + d.dx_off, nullptr, nullptr, nullptr, d.M, 2 * d.F, d.K, kOutBf16});
        weight.push_back({at.lane + d.x_off, dgu, at.lane + d.dw_in_off, d.M, d.K, 2 * d.F});
        weight.push_back({at.lane + d.h_off, dy, at.lane + d.dw_out_off, d.M, d.F, d.N});
        return nullptr;
    });
    if (rc) return rc;
    const bool cached = weights_cached(pool);
    uint64_t *count = launch_counter(pool);
    hipError_t e = launch_block_gate_grad(gate.data(), n, cached, stream, count);
    if (e == hipSuccess)
        e = launch_gradients(input.data(), (uint32_t)input.size(), weight.data(), (uint32_t)weight.size(), nullptr, 0, cached, stream, count);
    return launched(pool, e);
}

int32_t dense_forward(salus_pool_t *pool, const salus_dense_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<BlockProblem> problems;
    problems.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_dense_desc &d, const Placed &at) -> const char * {
        if (!rows_ok(d.M) || !width_ok(d.K) || !width_ok(d.N)) return kWidths;
        if (!act_ok(d.act)) return kAct;
        if (d.y_dtype != SALUS_F32 && d.y_dtype != SALUS_BF16) return "bad dtype";
        const uint64_t M = d.M;
        Ranges weights(at.P), lane(at.lane_size);
        weights.read(d.w_off, 2ull * d.K * d.N);
        if (d.b_off != SALUS_ABSENT) weights.read(d.b_off, 2ull * d.N);
        if (weights.outside()) return kWeights;
        lane.read(d.x_off, M * d.K * 2);
        lane.write(d.y_off, M * d.N * (d.y_dtype == SALUS_BF16 ? 2 : 4));
        if (d.r_off != SALUS_ABSENT && (d.r_off != d.y_off || d.y_dtype != SALUS_BF16)) lane.read(d.r_off, M * d.N * 2);
        if (d.z_off != SALUS_ABSENT) lane.write(d.z_off, M * d.N * 4);
        if (lane.outside()) return kLane;
        if (lane.overlap()) return kOverlap;
        problems.push_back({at.persist + d.w_off, at.lane + d.x_off, at.lane + d.y_off, at_or_null(at.lane, d.r_off), (float *)at_or_null(at.lane, d.z_off),
                            at_or_null(at.persist, d.b_off), d.M, d.K, d.N, (uint32_t)d.act | (d.y_dtype == SALUS_BF16 ? kOutBf16 : 0u) | (d.z_off != SALUS_ABSENT ? kReadAgain : 0u)});
        return nullptr;
    });
    if (rc) return rc;
    return launched(pool, launch_block_dense(problems.data(), n, weights_cached(pool), stream, launch_counter(pool)));
}

int32_t dense_backward(salus_pool_t *pool, const salus_dense_grad_desc *descs, uint32_t n, hipStream_t stream)
{
    std::vector<SlopeProblem> slope;
    std::vector<BlockProblem> input;
    std::vector<WeightGradProblem> weight;
    slope.reserve(n);
    input.reserve(n);
    weight.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_dense_grad_desc &d, const Placed &at) -> const char * {
        if (!rows_ok(d.M) || !width_ok(d.K) || !width_ok(d.N)) return kWidths;
        if (!act_ok(d.act)) return kAct;
        const bool linear = d.act == SALUS_ACT_NONE;
        if (linear != (d.z_off == SALUS_ABSENT)) return "z is given exactly if there is an activation";
        const uint64_t M = d.M;
        Ranges weights(at.P), lane(at.lane_size);
        weights.read(d.w_off, 2ull * d.K * d.N);
        if (weights.outside()) return kWeights;
        lane.read(d.x_off, M * d.K * 2);
        if (!linear) lane.read(d.z_off, M * d.N * 4);
        lane.read(d.dy_off, M * d.N * 2);
        if (d.dx_off != SALUS_ABSENT) lane.write(d.dx_off, M * d.K * 2);
        lane.write(d.dw_off, 2ull * d.K * d.N);
        if (d.db_off != SALUS_ABSENT) lane.write(d.db_off, 4ull * d.N);
        lane.write(d.work_off, salus_dense_grad_work_bytes(d.M, d.N));
        if (lane.outside()) return kLane;
        if (lane.overlap()) return kOverlap;
        char *dy = at.lane + d.dy_off, *work = at.lane + d.work_off, *dz = linear ? dy : work;      // dZ of a linear layer is dY
        slope.push_back({dy, linear ? nullptr : (const float *)(at.lane + d.z_off), linear ? nullptr : work, (float *)(work + up256(M * d.N * 2)),
                         (float *)at_or_null(at.lane, d.db_off), d.M, d.N, (uint32_t)d.act});
        if (d.dx_off != SALUS_ABSENT)
            input.push_back({at.persist + d.w_off, dz, at.lane + d.dx_off, nullptr, nullptr, nullptr, d.M, d.N, d.K, kOutBf16});
        weight.push_back({at.lane + d.x_off, dz, at.lane + d.dw_off, d.M, d.K, d.N});
        return nullptr;
    });
    if (rc) return rc;
    uint64_t *count = launch_counter(pool);
    hipError_t e = launch_block_slope(slope.data(), n, stream, count);
    slope.erase(std::remove_if(slope.begin(), slope.end(), [](const SlopeProblem &q) { return !q.db || q.M <= kSlopeRows; }), slope.end());
    if (e == hipSuccess)
        e = launch_gradients(input.data(), (uint32_t)input.size(), weight.data(), n, slope.data(), (uint32_t)slope.size(), weights_cached(pool), stream, count);
    return launched(pool, e);
}

constexpr uint64_t kClipMaxCount = 1ull << 48;

int32_t clip(salus_pool_t *pool, const salus_clip_desc *descs, uint32_t n, bool sgd, hipStream_t stream)
{
    std::vector<ClipJob> jobs;
    std::vector<std::vector<ClipTensor>> tensors;
    jobs.reserve(n);
    tensors.reserve(n);
    const int32_t rc = for_jobs(pool, descs, n, [&](const salus_clip_desc &d, const Placed &at) -> const char * {
        if (d.n_tensors == 0 || !d.tensors) return "empty job descriptor";
        if (!(d.max_norm > 0.0f)) return "max_norm must be positive";
        Ranges weights(at.P), lane(at.lane_size);
        std::vector<ClipTensor> list;
        list.reserve(d.n_tensors);
        for (uint32_t i = 0; i < d.n_tensors; ++i) {
            const salus_clip_tensor &t = d.tensors[i];
            if (t.count == 0 || t.count >= kClipMaxCount) return "a tensor has at least one element and fewer than 2^48";
            if (t.dtype != SALUS_F32 && t.dtype != SALUS_BF16) return "bad dtype";
            lane.write(t.g_off, t.count * (t.dtype == SALUS_BF16 ? 2 : 4));
            if (sgd) {
                weights.write(t.wm_off, t.count * 4);
                weights.write(t.wb_off, t.count * 2);
            }
            list.push_back({at.lane + t.g_off, sgd ? (float *)(at.persist + t.wm_off) : nullptr, sgd ? at.persist + t.wb_off : nullptr, t.count,
                            t.dtype == SALUS_BF16});
        }
        lane.write(d.norm_off, 4);
        lane.write(d.work_off, salus_clip_work_bytes(d.tensors, d.n_tensors));
        if (weights.outside()) return kWeights;
        if (lane.outside()) return kLane;
        if (lane.overlap() || weights.overlap()) return kOverlap;
        tensors.push_back(std::move(list));
        jobs.push_back({tensors.back().data(), d.n_tensors, d.max_norm, d.lr, (float *)(at.lane + d.norm_off), (double *)(at.lane + d.work_off)});
        return nullptr;
    });
    if (rc) return rc;
    return launched(pool, launch_clip(jobs.data(), n, sgd, stream, launch_counter(pool)));
}

}  // namespace

extern "C" {

int32_t salus_grouped_gated_forward(salus_pool_t *pool, const salus_gated_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return gated_forward(pool, descs, n, (hipStream_t)stream); });
}

uint64_t salus_gated_grad_work_bytes(uint32_t M, uint32_t F) { return up256((uint64_t)M * F * 4); }      // [dG dU]

int32_t salus_grouped_gated_backward(salus_pool_t *pool, const salus_gated_grad_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return gated_backward(pool, descs, n, (hipStream_t)stream); });
}

int32_t salus_grouped_dense_forward(salus_pool_t *pool, const salus_dense_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return dense_forward(pool, descs, n, (hipStream_t)stream); });
}

// dZ, then the column sums of its blocks of rows
uint64_t salus_dense_grad_work_bytes(uint32_t M, uint32_t N)
{
    return up256((uint64_t)M * N * 2) + up256(((uint64_t)M + kSlopeRows - 1) / kSlopeRows * N * 4);
}

int32_t salus_grouped_dense_backward(salus_pool_t *pool, const salus_dense_grad_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return dense_backward(pool, descs, n, (hipStream_t)stream); });
}

uint64_t salus_clip_work_bytes(const salus_clip_tensor *tensors, uint32_t n_tensors)
{
    if (!tensors) return 0;
    return 8 * clip_sums(n_tensors, [&](uint32_t i) { return tensors[i].count; });
}

int32_t salus_grouped_clip(salus_pool_t *pool, const salus_clip_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return clip(pool, descs, n, false, (hipStream_t)stream); });
}

int32_t salus_grouped_clip_sgd(salus_pool_t *pool, const salus_clip_desc *descs, uint32_t n, void *stream)
{
    return guarded(pool, descs, n, [&] { return clip(pool, descs, n, true, (hipStream_t)stream); });
}

}  // extern "C"
