// The rules by which the layers' launches are cut, for Python: compiled for the host alone.
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <numeric>

namespace {
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
