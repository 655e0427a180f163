// The rules by which the layers' launches are cut, for Python: compiled for the host alone.
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <numeric>

namespace {
#include "layer_arrays.h"
#include "layer_plan.h"
}

// What plan_resident makes of these sizes, with `preset` in the place of the shared memory before the call; 0 if it refuses.
extern "C" int plan_norm(const int64_t *sizes, int v, int two, uint64_t preset, uint64_t *shared, Resident *r) {
    const NormSizes k{(int)sizes[0], sizes[1], sizes[2], sizes[3], sizes[4], sizes[5], sizes[6] != 0};
    size_t bytes = (size_t)preset;
    const bool found = plan_resident(k, v, two != 0, *r, bytes);
    *shared = bytes;
    return found;
}

// Floats a worker of a dropout's workspace, and of its sums for one call.
extern "C" int64_t drop_sums(int64_t max_rows, int64_t cols, int n, int v) { return sums_of(max_rows, cols, n, v); }
extern "C" int64_t drop_used(int64_t rows, int64_t cols, int n, int v, int dense) {
    const Walk k = walk_of(rows, cols, n, v, dense && walked_as_one(rows, cols, v), true);
    return k.chunks == 1 && k.width == cols ? 0 : k.chunks * k.width;
}

// Whether a written array shares memory with another; each is {place, run, three times size and stride}, in elements of 2 bytes.
extern "C" int arrays_share(const int64_t *a, const int64_t *b, int *is_same) {
    auto of = [](const int64_t *v) {
        const Axis axes[3] = {{v[2], v[3]}, {v[4], v[5]}, {v[6], v[7]}};
        return array_of(reinterpret_cast<const void *>((uintptr_t)(4096 + 2 * v[0])), v[1], axes, 2);
    };
    *is_same = same(of(a), of(b));
    return shares(of(a), of(b));
}
