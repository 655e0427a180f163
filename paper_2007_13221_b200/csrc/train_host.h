// train_host.h - what the translation units of libcser.so share on the host (defined in cser.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>
#include "cser.h"

// Sets the thread's cser_last_error() and returns `code`.
__attribute__((visibility("hidden"))) int cser_internal_fail(int code, const char *fmt, ...)
    __attribute__((format(printf, 2, 3)));
// CSER_OK if p is memory of the current device.
__attribute__((visibility("hidden"))) int cser_internal_check_ptr(const void *p, const char *what);

// Returns from the calling function with the error of a CUDA call that failed.
#define TRY(expr)                                                                                              \
    do {                                                                                                       \
        cudaError_t _e = (expr);                                                                               \
        if (_e != cudaSuccess)                                                                                 \
            return cser_internal_fail(_e == cudaErrorMemoryAllocation ? CSER_ERR_NOMEM : CSER_ERR_CUDA, "%s: %s", #expr, \
                                      cudaGetErrorString(_e));                                                 \
    } while (0)

static inline long long up(long long v, long long to) { return (v + to - 1) / to * to; }

// A word of mapped pinned memory, 0, for kernels to report a wait that ran out in: its host and its device address.  From a page that
// the process keeps (pinning one per handle took 2 ms of a handle's 2.8).
__attribute__((visibility("hidden"))) cudaError_t cser_internal_take_word(unsigned **host, unsigned **device);
__attribute__((visibility("hidden"))) void cser_internal_give_word(unsigned *host);
