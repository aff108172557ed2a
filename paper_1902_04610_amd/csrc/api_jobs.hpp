// Pieces of the packed entry points: the ranges of a call's buffers, and a call over the jobs of a round.  Every argument is checked before anything is launched.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>
#include <vector>

#include "api.hpp"

namespace salus {

inline uint64_t up256(uint64_t v) { return (v + 255) & ~(uint64_t)255; }

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

inline bool rows_ok(uint32_t m) { return m != 0 && m < 1u << 31; }

const char *const kWeights = "weights outside the persistent block";
const char *const kCache = "cache or frequencies outside the persistent block";
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

inline int32_t launched(salus_pool_t *pool, hipError_t e)
{
    return e == hipSuccess ? SALUS_OK : pool_error(pool, SALUS_EHIP, hipGetErrorString(e));
}

inline char *at_or_null(char *base, uint64_t off) { return off == SALUS_ABSENT ? nullptr : base + off; }

}  // namespace salus
