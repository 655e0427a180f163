// layer_arrays.h - whether two arrays of a call share memory.  Plain C++ that needs no GPU, so that it can be checked against every element on
// the host; included by layers.cuh inside its unnamed namespace.
#pragma once

struct Axis { int64_t size, stride; };

// Runs of contiguous bytes with up to three axes around them, the widest first.  Axes that reach nothing new are left out.
struct Array {
    __int128 at = 0, run = 0;
    int axes = 0;
    struct { __int128 size, stride; } axis[3];

    __int128 reach(int from = 0) const {
        __int128 span = run;
        for (int k = from; k < axes; ++k) span += (axis[k].size - 1) * axis[k].stride;
        return span;
    }
};
// An array of `run` contiguous elements of `size` bytes with these axes around them, strides in elements and not negative.
template <int N> Array array_of(const void *data, int64_t run, const Axis (&given)[N], int size) {
    static_assert(N <= 3, "");
    Array a;
    a.at = (uintptr_t)data, a.run = (__int128)run * size;
    for (const Axis &g : given) {
        if (g.size <= 1 || g.stride == 0) continue;
        int k = a.axes++;
        for (; k > 0 && a.axis[k - 1].stride < (__int128)g.stride * size; --k) a.axis[k] = a.axis[k - 1];
        a.axis[k] = {g.size, (__int128)g.stride * size};
    }
    return a;
}

inline bool alike(const Array &a, const Array &b) {
    if (a.run != b.run || a.axes != b.axes) return false;
    for (int k = 0; k < a.axes; ++k)
        if (a.axis[k].size != b.axis[k].size || a.axis[k].stride != b.axis[k].stride) return false;
    return true;
}
inline bool same(const Array &a, const Array &b) { return a.at == b.at && alike(a, b); }
// Whether it is one stretch of memory without gaps.
inline bool dense(const Array &a) {
    for (int k = 0; k < a.axes; ++k)
        if (a.axis[k].stride > a.reach(k + 1)) return false;
    return true;
}
// Whether some of what the axes from k on reach, beginning at `at`, lies in low .. high - 1.
inline bool within(const Array &a, int k, __int128 at, __int128 low, __int128 high) {
    const __int128 end = at + a.reach(k);
    if (end <= low || at >= high) return false;
    if (k == a.axes || at >= low || end <= high) return true;              // (its first and its last byte exist)
    const __int128 stride = a.axis[k].stride, inner = a.reach(k + 1);
    __int128 i = low - at < inner ? 0 : (low - at - inner) / stride + 1;
    for (int tries = 0; tries < 4 && i < a.axis[k].size && at + i * stride < high; ++i, ++tries)        // two, unless steps lie on one another
        if (within(a, k + 1, at + i * stride, low, high)) return true;
    return false;
}
// Whether elements of arrays that are alike and `ahead` bytes apart coincide: whether steps of the axes, each fewer than its size either way, come
// that near.  Each axis steps over all that is inside it, so two numbers of steps are possible at most.
inline bool meets(const Array &a, int k, __int128 ahead) {
    if (k == a.axes) return ahead < a.run && ahead > -a.run;
    const __int128 stride = a.axis[k].stride, most = a.axis[k].size - 1;
    const __int128 near = ahead >= 0 ? ahead / stride : -((-ahead + stride - 1) / stride);              // rounded down
    for (__int128 d = near; d <= near + 1; ++d)
        if (d <= most && d >= -most && meets(a, k + 1, ahead - d * stride)) return true;
    return false;
}
// Whether `written`, whose elements lie apart, shares memory with another array.  Exact where the two are alike or one has no gaps; of
// others, whose gaps may hold each other, it says no.
inline bool shares(const Array &written, const Array &other) {
    if (written.at + written.reach() <= other.at || other.at + other.reach() <= written.at) return false;
    if (alike(written, other)) return meets(written, 0, other.at - written.at);
    if (dense(other)) return within(written, 0, written.at, other.at, other.at + other.reach());
    return dense(written) && within(other, 0, other.at, written.at, written.at + written.reach());
}
