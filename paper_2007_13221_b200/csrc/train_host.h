// train_host.h - what the translation units of libcser.so share on the host (defined in cser.cu).
#pragma once
#include <stdint.h>
#include "cser.h"

// Sets the thread's cser_last_error() and returns `code`.
__attribute__((visibility("hidden"))) int cser_internal_fail(int code, const char *fmt, ...)
    __attribute__((format(printf, 2, 3)));
// CSER_OK if p is memory of the current device.
__attribute__((visibility("hidden"))) int cser_internal_check_ptr(const void *p, const char *what);
