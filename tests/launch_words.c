/* Preloaded in front of launch_recorder.c: writes down the first four words of what each kernel is given by value. */
#define _GNU_SOURCE
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>

typedef struct { uint32_t x, y, z; } dim3;

static char log_[1 << 20];
static size_t used;

const char *words_take(void)          /* a line per launch since the last call */
{
    static char out[sizeof log_];
    snprintf(out, sizeof out, "%s", log_);
    used = 0;
    log_[0] = 0;
    return out;
}

int hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t shared, void *stream)
{
    static int (*next)(const void *, dim3, dim3, void **, size_t, void *);
    const uint32_t *w = (const uint32_t *)args[0];
    if (!next) next = (int (*)(const void *, dim3, dim3, void **, size_t, void *))dlsym(RTLD_NEXT, "hipLaunchKernel");
    if (used + 64 < sizeof log_) used += (size_t)snprintf(log_ + used, sizeof log_ - used, "%u %u %u %u\n", w[0], w[1], w[2], w[3]);
    return next(fn, grid, block, args, shared, stream);
}
