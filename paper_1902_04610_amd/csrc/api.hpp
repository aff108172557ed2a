// What the entry points of other files need of a pool (implemented in api.hip).
#pragma once
#include <cstdint>
#include <vector>

#include "salus.h"

namespace salus {

struct Placed {
    char *persist, *lane;        // device addresses of the job's persistent block and of its lane
    uint64_t P, lane_size;
};
// Where a job of a packed call lies; an error if it is not resident, in transit, or in a lane that is already used (lanes_used
// grows by its lane).
int32_t place_job(salus_pool_t *pool, int32_t job, std::vector<int32_t> &lanes_used, Placed *out);
int32_t pool_error(salus_pool_t *pool, int32_t code, const char *message);      // sets salus_last_error, returns code
bool has_device(const salus_pool_t *pool);
bool weights_cached(const salus_pool_t *pool);      // `cached` of the launchers
uint64_t *launch_counter(salus_pool_t *pool);

}  // namespace salus
