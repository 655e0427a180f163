// layers.cuh - host side of the layers between the models' products (include/cser_layers.h); included by cser.cu.
//
// Launches are cut by the rules of layer_plan.h, arrays told apart by layer_arrays.h.  Kernels: drop_kernels.cuh (dropout), norm_resident.cuh and norm_kernels.cuh (group norm), layer_common.cuh (what both use).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cser_layers.h"

namespace {
namespace layers {

#include "layer_arrays.h"
#include "layer_plan.h"
#include "layer_common.cuh"
#include "drop_kernels.cuh"
#include "norm_kernels.cuh"
#include "norm_resident.cuh"

int size_of(int type) { return type == CSER_TYPE_F32 ? 4 : 2; }
bool aligned(const void *p, int to) { return (uintptr_t)p % to == 0; }

int check_device(int device) {
    int dev = -1;
    TRY(cudaGetDevice(&dev));
    if (dev != device) return fail(CSER_ERR_INVALID, "handle belongs to device %d, current device is %d", device, dev);
    return CSER_OK;
}

// fp32 parameters or their gradients: [n][count], `stride` from one worker to the next.
int check_params(const float *p, int64_t stride, int64_t least, int n, const char *what) {
    if (int rc = check_device_ptr(p, what)) return rc;
    if (!aligned(p, 4)) return fail(CSER_ERR_INVALID, "%s: a pointer is not aligned to its element type", what);
    if (n > 1 && stride < least) return fail(CSER_ERR_INVALID, "%s: stride from worker to worker is less than %lld", what, (long long)least);
    return CSER_OK;
}

// An array whose innermost `run` elements are contiguous, with these axes around them.  What is written must not lie on itself: from the
// closest axis to the widest, each has to step over all that is inside.
template <int N> int check_array(const void *data, int type, int64_t run, const Axis (&given)[N], bool written, const char *what) {
    if (int rc = check_device_ptr(data, what)) return rc;
    if (!aligned(data, size_of(type))) return fail(CSER_ERR_INVALID, "%s: a pointer is not aligned to its element type", what);
    Axis axes[N];
    for (int i = 0; i < N; ++i) {
        axes[i] = given[i];
        if (axes[i].stride < 0) return fail(CSER_ERR_INVALID, "%s: strides must not be negative", what);
    }
    std::sort(axes, axes + N, [](const Axis &a, const Axis &b) { return a.stride < b.stride; });
    __int128 span = run;
    for (const Axis &a : axes)
        if (a.size > 1) {
            if (written && a.stride < span) return fail(CSER_ERR_INVALID, "%s: its strides make elements share memory", what);
            span += (__int128)(a.size - 1) * a.stride;
        }
    return span <= (1ll << 60) ? CSER_OK : fail(CSER_ERR_INVALID, "%s: its strides are too large", what);
}

// What a call writes shares no memory with its other arrays, but a result may take the place of an input: all of it.
struct Given {
    const char *name;
    Array array;
    bool written, replaces;                            // replaces: a result, or an input that one may replace
};
template <int N> int check_apart(const Given (&all)[N], const char *what) {
    for (const Given &w : all)
        for (const Given &o : all)
            if (w.written && w.array.at && o.array.at && &w != &o && shares(w.array, o.array) && !(w.replaces && o.replaces && same(w.array, o.array)))
                return fail(CSER_ERR_INVALID, "%s: %s and %s share memory", what, w.name, o.name);
    return CSER_OK;
}
Array params_of(const float *p, int64_t stride, int64_t count, int n) {
    const Axis axes[1] = {{n, stride}};
    return p ? array_of(p, count, axes, 4) : Array();
}

int check_step_at(const uint64_t *p) {
    if (!p) return CSER_OK;
    if (int rc = check_device_ptr(p, "step_at")) return rc;
    return aligned(p, 8) ? CSER_OK : fail(CSER_ERR_INVALID, "step_at: a pointer is not aligned to its element type");
}

Draw draw_of(double p, uint64_t seed, uint32_t site, int first_worker, uint64_t step, const uint64_t *step_at) {
    Draw d;
    d.k0 = (uint32_t)seed, d.k1 = (uint32_t)(seed >> 32), d.c3 = site * 4096u + (uint32_t)first_worker;
    d.threshold = (uint32_t)floor(p * 4294967296.0), d.factor = (float)(1.0 / (1.0 - p));
    d.step = step, d.step_at = reinterpret_cast<const unsigned long long *>(step_at);
    return d;
}

// A launch that may be set up while the kernel before it ends; `cluster` blocks form one.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned block, size_t shared, unsigned cluster, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid, cfg.blockDim = dim3(block), cfg.dynamicSmemBytes = shared, cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization, at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

int launch_row_sums(const RowSums &s, long long n, int planes, int64_t &launches, cudaStream_t st) {
    TRY(launch(sum_rows_kernel, dim3((unsigned)ceil_div(s.cols, 32), (unsigned)n, (unsigned)planes), s.rows > 64 ? 1024 : 256, 0, 1, st, s));
    launches++;
    return CSER_OK;
}

// Zeros where there is nothing to sum.
int clear_params(float *p, int64_t stride, int64_t count, int n, cudaStream_t st) {
    if (!p) return CSER_OK;
    for (int w = 0; w < n; ++w) TRY(cudaMemsetAsync(p + w * stride, 0, (size_t)count * 4, st));
    return CSER_OK;
}

}  // namespace layers
}  // namespace

// ------------------------------------------------------------------ dropout
struct cser_drop {
    int n = 0, type = 0, device = 0, first_worker = 0;
    int64_t max_rows = 0, cols = 0, launches = 0;
    double p = 0.0;
    uint64_t seed = 0;
    uint32_t site = 0;
    float *part = nullptr;                             // sums of chunks of rows
};

namespace {
namespace layers {

int check_rows(const cser_rows *a, const cser_drop *h, int64_t rows, bool written, const char *what) {
    const Axis axes[2] = {{rows, a->row_stride}, {h->n, a->worker_stride}};
    return check_array(a->data, h->type, h->cols, axes, written, what);
}
Array rows_of(const cser_rows *a, const cser_drop *h, int64_t rows) {
    if (!a) return Array();
    const Axis axes[2] = {{rows, a->row_stride}, {h->n, a->worker_stride}};
    return array_of(a->data, h->cols, axes, size_of(h->type));
}

template <typename T, int MODE, bool SHIFTED> cudaError_t drop_rows_launch(const DropArgs<T> &a, unsigned grid, bool sums, cudaStream_t st) {
    const auto kernel = sums ? drop_rows_kernel<T, MODE, SHIFTED, kSums>
                             : a.r ? drop_rows_kernel<T, MODE, SHIFTED, kResidual> : drop_rows_kernel<T, MODE, SHIFTED, kForward>;
    return launch(kernel, dim3(grid), 256, 0, 1, st, a);
}

template <typename T>
int drop_launch(cser_drop *h, int64_t rows, const Draw &draw, const cser_rows *x, const float *bias, int64_t bias_stride,
                const cser_rows *residual, const cser_rows *y, float *dbias, int64_t dbias_stride, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    DropArgs<T> a{};
    a.rows = rows, a.cols = h->cols, a.draw = draw, a.bias = bias, a.bias_worker = bias_stride;
    a.ahead = (int)((uintptr_t)x->data % 16 / sizeof(T)), a.ahead_worker = h->n == 1 ? 0 : (int)(x->worker_stride % V);
    bool dense = true, plain = h->cols % V == 0;
    auto take = [&](const cser_rows *r) {
        const int at = (int)((uintptr_t)r->data % 16 / sizeof(T)), more = h->n == 1 ? 0 : (int)(r->worker_stride % V);
        dense = dense && (rows == 1 || r->row_stride == h->cols) && at == a.ahead && more == a.ahead_worker;
        plain = plain && at == 0 && more == 0 && (rows == 1 || r->row_stride % V == 0);
    };
    a.x = static_cast<const T *>(x->data), a.x_row = x->row_stride, a.x_worker = x->worker_stride;
    take(x);
    if (residual) a.r = static_cast<const T *>(residual->data), a.r_row = residual->row_stride, a.r_worker = residual->worker_stride, take(residual);
    if (y) a.y = static_cast<T *>(y->data), a.y_row = y->row_stride, a.y_worker = y->worker_stride, take(y);
    const bool shifted = a.ahead || a.ahead_worker;
    if (dense && !bias && !dbias) {
        const long long blocks = ceil_div(rows * h->cols + V - 1, 256 * V * kFlat);
        const dim3 grid((unsigned)blocks, (unsigned)h->n);
        const auto kernel = shifted ? (a.r ? drop_flat_kernel<T, true, true> : drop_flat_kernel<T, true, false>)
                                    : (a.r ? drop_flat_kernel<T, false, true> : drop_flat_kernel<T, false, false>);
        TRY(launch(kernel, grid, 256, 0, 1, st, a));
        h->launches++;
        return CSER_OK;
    }
    dense = dense && !(plain && h->cols >= 32 * V) && walked_as_one(rows, h->cols, V);         // wide rows of whole vectors: the simpler walk
    const Walk k = walk_of(rows, h->cols, h->n, V, dense, dbias);
    a.width = k.width, a.chunk_rows = k.chunk_rows, a.tx = k.tx, a.log_rows = 8 - (int)std::log2(k.tx);
    a.walked = dense ? ceil_div(rows * h->cols, k.width) : rows, a.last_row = rows * h->cols - (a.walked - 1) * k.width;
    a.col_blocks = k.col_blocks, a.chunks = k.chunks;
    const long long blocks = (long long)k.col_blocks * k.chunks * h->n;
    if (blocks > kMostBlocks) return fail(CSER_ERR_INVALID, "dropout: too many elements");
    const bool direct = k.chunks == 1 && k.width == h->cols;
    if (dbias) a.part = direct ? dbias : h->part, a.part_worker = direct ? dbias_stride : k.chunks * k.width;
    TRY((dense && shifted ? drop_rows_launch<T, kDense, true>(a, (unsigned)blocks, dbias, st)
         : dense          ? drop_rows_launch<T, kDense, false>(a, (unsigned)blocks, dbias, st)
         : plain          ? drop_rows_launch<T, kPlain, false>(a, (unsigned)blocks, dbias, st)
                          : drop_rows_launch<T, kOdd, true>(a, (unsigned)blocks, dbias, st)));
    h->launches++;
    if (!dbias || direct) return CSER_OK;
    RowSums s{};
    s.part = h->part, s.out[0] = dbias, s.out_stride[0] = dbias_stride, s.rows = k.chunks * (k.width / h->cols), s.cols = h->cols;
    return launch_row_sums(s, h->n, 1, h->launches, st);
}

int drop_call(cser_drop *h, int64_t rows, uint64_t step, const uint64_t *step_at, const cser_rows *x, const float *bias, int64_t bias_stride,
              const cser_rows *residual, const cser_rows *y, float *dbias, int64_t dbias_stride, cudaStream_t st) {
    const Draw d = draw_of(h->p, h->seed, h->site, h->first_worker, step, step_at);
    if (h->type == CSER_TYPE_F32) return drop_launch<float>(h, rows, d, x, bias, bias_stride, residual, y, dbias, dbias_stride, st);
    if (h->type == CSER_TYPE_BF16) return drop_launch<__nv_bfloat16>(h, rows, d, x, bias, bias_stride, residual, y, dbias, dbias_stride, st);
    return drop_launch<__half>(h, rows, d, x, bias, bias_stride, residual, y, dbias, dbias_stride, st);
}

}  // namespace layers
}  // namespace

extern "C" {

cser_drop_handle cser_drop_create(int32_t n_workers, int64_t max_rows, int64_t cols, double p, uint64_t seed, uint32_t site,
                                  int32_t first_worker, int32_t type) {
    auto bad = [](int code, const char *what) { fail(code, "cser_drop_create: %s", what); return nullptr; };
    if (n_workers < 1 || first_worker < 0 || n_workers > 4096 || first_worker > 4096 - n_workers)
        return bad(CSER_ERR_INVALID, "n_workers must be positive, first_worker not negative and their sum at most 4096");
    if (max_rows < 1 || cols < 1 || max_rows > (1ll << 34) / cols)
        return bad(CSER_ERR_INVALID, "max_rows and cols must be positive and their product at most 2^34");
    if (!(p >= 0.0 && p < 1.0) || floor(p * 4294967296.0) >= 4294967296.0) return bad(CSER_ERR_INVALID, "p must be in [0, 1)");
    if (site < 1 || site >= (1u << 20)) return bad(CSER_ERR_INVALID, "site must be in 1..2^20-1");
    if (type != CSER_TYPE_F32 && type != CSER_TYPE_BF16 && type != CSER_TYPE_F16)
        return bad(CSER_ERR_INVALID, "type must be CSER_TYPE_F32, CSER_TYPE_BF16 or CSER_TYPE_F16");
    cser_drop *h = new (std::nothrow) cser_drop;
    if (!h) return bad(CSER_ERR_NOMEM, "host allocation failed");
    h->n = n_workers, h->max_rows = max_rows, h->cols = cols, h->p = p, h->seed = seed, h->site = site, h->first_worker = first_worker,
    h->type = type;
    const long long sums = layers::sums_of(max_rows, cols, n_workers, 16 / layers::size_of(type));
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaMalloc(&h->part, (size_t)(n_workers * sums) * 4);
    if (e != cudaSuccess) {
        fail(e == cudaErrorMemoryAllocation ? CSER_ERR_NOMEM : CSER_ERR_CUDA, "cser_drop_create: %s", cudaGetErrorString(e));
        delete h;
        return nullptr;
    }
    return h;
}

int cser_drop_apply(cser_drop_handle h, int64_t rows, uint64_t step, const uint64_t *step_at, const cser_rows *x,
                    const float *bias, int64_t bias_stride, const cser_rows *residual, const cser_rows *y, void *stream) {
    using namespace layers;
    if (!h) return fail(CSER_ERR_INVALID, "cser_drop_apply: NULL handle");
    if (!x || !y) return fail(CSER_ERR_INVALID, "cser_drop_apply: NULL array");
    if (int rc = check_device(h->device)) return rc;
    if (rows < 0 || rows > h->max_rows) return fail(CSER_ERR_INVALID, "cser_drop_apply: rows must be in 0..%lld", (long long)h->max_rows);
    if (rows == 0) return CSER_OK;
    if (int rc = check_rows(x, h, rows, false, "cser_drop_apply: x")) return rc;
    if (residual)
        if (int rc = check_rows(residual, h, rows, false, "cser_drop_apply: residual")) return rc;
    if (int rc = check_rows(y, h, rows, true, "cser_drop_apply: y")) return rc;
    if (bias)
        if (int rc = check_params(bias, bias_stride, 0, h->n, "cser_drop_apply: bias")) return rc;
    if (int rc = check_step_at(step_at)) return rc;
    const Given all[] = {{"y", rows_of(y, h, rows), true, true},
                         {"x", rows_of(x, h, rows), false, true},
                         {"residual", rows_of(residual, h, rows), false, true},
                         {"bias", params_of(bias, bias_stride, h->cols, h->n), false, false}};
    if (int rc = check_apart(all, "cser_drop_apply")) return rc;
    return drop_call(h, rows, step, step_at, x, bias, bias_stride, residual, y, nullptr, 0, (cudaStream_t)stream);
}

int cser_drop_grad(cser_drop_handle h, int64_t rows, uint64_t step, const uint64_t *step_at, const cser_rows *dy,
                   const cser_rows *dx, float *dbias, int64_t dbias_stride, void *stream) {
    using namespace layers;
    if (!h) return fail(CSER_ERR_INVALID, "cser_drop_grad: NULL handle");
    if (!dy) return fail(CSER_ERR_INVALID, "cser_drop_grad: NULL array");
    if (int rc = check_device(h->device)) return rc;
    if (rows < 0 || rows > h->max_rows) return fail(CSER_ERR_INVALID, "cser_drop_grad: rows must be in 0..%lld", (long long)h->max_rows);
    if (dbias)
        if (int rc = check_params(dbias, dbias_stride, h->cols, h->n, "cser_drop_grad: dbias")) return rc;
    if (rows == 0) return clear_params(dbias, dbias_stride, h->cols, h->n, (cudaStream_t)stream);
    if (!dx && !dbias) return CSER_OK;
    if (int rc = check_rows(dy, h, rows, false, "cser_drop_grad: dy")) return rc;
    if (dx)
        if (int rc = check_rows(dx, h, rows, true, "cser_drop_grad: dx")) return rc;
    if (int rc = check_step_at(step_at)) return rc;
    const Given all[] = {{"dx", rows_of(dx, h, rows), true, true},
                         {"dy", rows_of(dy, h, rows), false, true},
                         {"dbias", params_of(dbias, dbias_stride, h->cols, h->n), true, false}};
    if (int rc = check_apart(all, "cser_drop_grad")) return rc;
    return drop_call(h, rows, step, step_at, dy, nullptr, 0, nullptr, dx, dbias, dbias_stride, (cudaStream_t)stream);
}

void cser_drop_destroy(cser_drop_handle h) {
    if (!h) return;
    if (h->part) cudaFree(h->part);
    delete h;
}

int64_t cser_drop_launch_count(cser_drop_handle h) { return h ? h->launches : 0; }

}  // extern "C"

// ------------------------------------------------------------------ group norm
struct cser_norm {
    int n = 0, type = 0, device = 0, act = 0;
    int64_t max_samples = 0, channels = 0, groups = 0, launches = 0;
    float eps = 0.f;
    bool drop = false;
    cser_drop dropout;                                 // a copy: p, seed, site and first worker
    float *part = nullptr;                             // two planes of channels' sums
    float2 *group_sums = nullptr;
    long long plane = 0;
    struct Fit {                                       // clusters that the GPU holds at a time
        const void *kernel = nullptr;
        int log_cluster = 0, log_block = 0, clusters = 0;
        size_t shared = 0;
    } fits[4];
    unsigned next_fit = 0;
};

namespace {
namespace layers {

int check_pixels(const cser_pixels *a, const cser_norm *h, const cser_norm_inputs *in, bool written, const char *what) {
    const Axis axes[3] = {{in->pixels, a->pixel_stride}, {in->samples, a->sample_stride}, {h->n, a->worker_stride}};
    return check_array(a->data, h->type, h->channels, axes, written, what);
}

Array pixels_of(const cser_pixels *a, const cser_norm *h, const cser_norm_inputs *in) {
    if (!a) return Array();
    const Axis axes[3] = {{in->pixels, a->pixel_stride}, {in->samples, a->sample_stride}, {h->n, a->worker_stride}};
    return array_of(a->data, h->channels, axes, size_of(h->type));
}
Array stats_of(const float *stats, const cser_norm *h, const cser_norm_inputs *in) {
    return params_of(stats, 0, 2 * h->n * in->samples * h->groups, 1);
}

// Elements that one load or store can take from an array: the largest power of two up to 16 bytes' worth that all of its starts allow.
int vector_of(const cser_norm *h, const cser_norm_inputs *in, const cser_pixels *a) {
    const int size = size_of(h->type);
    int v = 16 / size;
    auto fits = [&](long long stride, long long times) { return times <= 1 || stride % v == 0; };
    while (v > 1 && !(h->channels % v == 0 && (uintptr_t)a->data % (v * size) == 0 && fits(a->pixel_stride, in->pixels) &&
                      fits(a->sample_stride, in->samples) && fits(a->worker_stride, h->n)))
        v /= 2;
    return v;
}

NormSizes sizes_of(const cser_norm *h, const cser_norm_inputs *in) {
    return {size_of(h->type), h->n, in->samples, in->pixels, h->channels, h->groups, h->drop};
}
View view_of(const cser_pixels *a) { return {(long long)a->pixel_stride, (long long)a->sample_stride, (long long)a->worker_stride}; }

template <typename T> NormArgs<T> norm_args(const cser_norm *h, const cser_norm_inputs *in, float *stats) {
    NormArgs<T> a{};
    a.x = static_cast<const T *>(in->x.data), a.xs = view_of(&in->x);
    a.weight = in->weight, a.bias = in->bias, a.weight_worker = in->weight_stride, a.bias_worker = in->bias_stride;
    a.stats = stats, a.group_sums = h->group_sums, a.part = h->part, a.plane = h->plane;
    a.n = h->n, a.samples = (int)in->samples, a.channels = (int)h->channels, a.groups = (int)h->groups;
    a.per_group = (int)(h->channels / h->groups), a.act = h->act, a.pixels = in->pixels, a.eps = h->eps;
    if (h->drop) a.draw = draw_of(h->dropout.p, h->dropout.seed, h->dropout.site, h->dropout.first_worker, in->step, in->step_at);
    return a;
}

// Cuts the pixels of a sample into chunks for blocks of 256 threads; false if the grid is too large.
template <typename T> bool cut(NormArgs<T> &a, int v, bool sums, unsigned &grid) {
    column_blocks(a.channels, v, a.tx, a.col_blocks);
    const long long others = (long long)a.n * a.samples * a.col_blocks;
    const long long most = ceil_div(a.pixels, 4 * (256 / a.tx)), want = sums ? ceil_div(kBusy / 2, (long long)a.n * a.samples) : ceil_div(kBusy, others);
    const long long chunks = most < want ? most : want;
    a.chunk_pixels = ceil_div(a.pixels, chunks);
    a.chunks = (int)ceil_div(a.pixels, a.chunk_pixels);
    grid = (unsigned)(others * a.chunks);
    return others * a.chunks <= kMostBlocks;
}

// Threads that join the parts of a group: eight parts each, if that many are.
template <typename T> unsigned join_threads(const NormArgs<T> &a) {
    unsigned k = 32;
    while (k < 1024 && k * 8ll < (long long)a.chunks * a.per_group) k *= 2;
    return k;
}

// Calls f with the kernel's vector length as a constant.
template <typename T, typename F> int with_vector(int v, F f) {
    if (sizeof(T) == 2 && v == 8) return f(std::integral_constant<int, 16 / sizeof(T)>());
    if (v == 4) return f(std::integral_constant<int, 4>());
    return v == 2 ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 1>());
}

// The call's launch: as many clusters as the GPU holds at a time, or as there are units.  How many it holds is asked once for a kernel and a
// shape, and the kernel allowed its shared memory then (for all kernels when a handle is made, loading them took 40 ms of a process).
template <typename T>
int resident_launch(cser_norm *h, void (*kernel)(NormArgs<T>, Resident), const NormArgs<T> &a, const Resident &r, size_t shared, cudaStream_t st) {
    cser_norm::Fit *fit = nullptr;
    for (auto &f : h->fits)
        if (f.kernel == (const void *)kernel && f.log_cluster == r.log_cluster && f.log_block == r.log_block && f.shared == shared) fit = &f;
    if (!fit) {
        fit = &h->fits[h->next_fit++ % 4];
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(1u << r.log_cluster), cfg.blockDim = dim3(1u << r.log_block), cfg.dynamicSmemBytes = shared;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 1u << r.log_cluster, at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at, cfg.numAttrs = 1;
        fit->kernel = nullptr;
        TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared));
        TRY(cudaOccupancyMaxActiveClusters(&fit->clusters, kernel, &cfg));
        fit->kernel = (const void *)kernel, fit->log_cluster = r.log_cluster, fit->log_block = r.log_block, fit->shared = shared;
    }
    const uint32_t clusters = std::min<uint32_t>(r.units, std::max(fit->clusters, 1));
    TRY(launch(kernel, dim3(clusters << r.log_cluster), 1u << r.log_block, shared, 1u << r.log_cluster, st, a, r));
    h->launches++;
    return CSER_OK;
}

template <typename T> int norm_apply(cser_norm *h, const cser_norm_inputs *in, const cser_pixels *y, float *stats, cudaStream_t st) {
    NormArgs<T> a = norm_args<T>(h, in, stats);
    a.y = static_cast<T *>(y->data), a.ys = view_of(y);
    const int v = std::min(vector_of(h, in, &in->x), vector_of(h, in, y));
    return with_vector<T>(v, [&](auto vector) -> int {
        constexpr int V = decltype(vector)::value;
        unsigned grid;
        if constexpr (V * sizeof(T) >= 4) {
            Resident r;
            size_t shared;
            if (plan_resident(sizes_of(h, in), V, false, r, shared)) {
                return resident_launch<T>(h, h->drop ? norm_resident_kernel<T, V, true> : norm_resident_kernel<T, V, false>, a, r, shared, st);
            }
        }
        if (!cut(a, V, true, grid)) return fail(CSER_ERR_INVALID, "cser_norm_apply: too many elements");
        TRY(launch(h->drop ? norm_moments_kernel<T, V, true> : norm_moments_kernel<T, V, false>, dim3(grid), 256, 0, 1, st, a));
        TRY(launch(norm_join_moments_kernel<T>, dim3((unsigned)(a.n * a.samples * a.groups)), join_threads(a), 0, 1, st, a));
        if (!cut(a, V, false, grid)) return fail(CSER_ERR_INVALID, "cser_norm_apply: too many elements");
        TRY(launch(h->drop ? norm_apply_kernel<T, V, true> : norm_apply_kernel<T, V, false>, dim3(grid), 256, 0, 1, st, a));
        h->launches += 3;
        return CSER_OK;
    });
}

template <typename T>
int norm_grad(cser_norm *h, const cser_norm_inputs *in, const float *stats, const cser_pixels *dy, const cser_pixels *dx, float *dweight,
              int64_t dweight_stride, float *dbias, int64_t dbias_stride, cudaStream_t st) {
    NormArgs<T> a = norm_args<T>(h, in, const_cast<float *>(stats));
    a.dy = static_cast<const T *>(dy->data), a.dys = view_of(dy);
    int v = std::min(vector_of(h, in, &in->x), vector_of(h, in, dy));
    if (dx) a.y = static_cast<T *>(dx->data), a.ys = view_of(dx), v = std::min(v, vector_of(h, in, dx));
    return with_vector<T>(v, [&](auto vector) -> int {
        constexpr int V = decltype(vector)::value;
        unsigned grid;
        bool done = false, direct = false;
        if constexpr (V * sizeof(T) >= 4) {
            Resident r;
            size_t shared;
            if (plan_resident(sizes_of(h, in), V, true, r, shared)) {
                // A worker's only sample's sums are its gradients; those of several are added up behind.
                a.chunks = 1, done = true, direct = a.samples == 1;
                a.sums[0] = direct ? dbias : h->part, a.sums_sample[0] = direct ? dbias_stride : a.channels;
                a.sums[1] = direct ? dweight : h->part + h->plane, a.sums_sample[1] = direct ? dweight_stride : a.channels;
                if (!dbias && !dweight) a.sums[0] = a.sums[1] = nullptr;
                if (int rc = resident_launch<T>(h, h->drop ? norm_grad_resident_kernel<T, V, true> : norm_grad_resident_kernel<T, V, false>, a, r, shared, st))
                    return rc;
            }
        }
        if (!done) {
            if (!cut(a, V, true, grid)) return fail(CSER_ERR_INVALID, "cser_norm_grad: too many elements");
            TRY(launch(h->drop ? norm_grad_sums_kernel<T, V, true> : norm_grad_sums_kernel<T, V, false>, dim3(grid), 256, 0, 1, st, a));
            h->launches++;
        }
        if ((dweight || dbias) && !direct) {
            RowSums s{};
            s.part = a.part, s.plane = a.plane, s.rows = (long long)a.samples * a.chunks, s.cols = a.channels;
            s.out[0] = dbias, s.out_stride[0] = dbias_stride, s.out[1] = dweight, s.out_stride[1] = dweight_stride;
            if (int rc = launch_row_sums(s, a.n, 2, h->launches, st)) return rc;
        }
        if (!dx || done) return CSER_OK;
        TRY(launch(norm_join_sums_kernel<T>, dim3((unsigned)(a.n * a.samples * a.groups)), join_threads(a), 0, 1, st, a));
        if (!cut(a, V, false, grid)) return fail(CSER_ERR_INVALID, "cser_norm_grad: too many elements");
        TRY(launch(h->drop ? norm_grad_apply_kernel<T, V, true> : norm_grad_apply_kernel<T, V, false>, dim3(grid), 256, 0, 1, st, a));
        h->launches += 2;
        return CSER_OK;
    });
}

// Checks that both calls make; *empty: nothing to compute.
int check_norm(const cser_norm *h, const cser_norm_inputs *in, const char *what, bool *empty) {
    if (!h) return fail(CSER_ERR_INVALID, "%s: NULL handle", what);
    if (!in) return fail(CSER_ERR_INVALID, "%s: NULL inputs", what);
    if (int rc = check_device(h->device)) return rc;
    if (in->samples < 0 || in->samples > h->max_samples)
        return fail(CSER_ERR_INVALID, "%s: samples must be in 0..%lld", what, (long long)h->max_samples);
    if (in->pixels < 0 || in->pixels > 0x7fffffff) return fail(CSER_ERR_INVALID, "%s: pixels must be in 0..2^31-1", what);
    *empty = in->samples == 0 || in->pixels == 0;
    if (*empty) return CSER_OK;
    if (h->drop && in->pixels > (1ll << 34) / h->channels / in->samples)
        return fail(CSER_ERR_INVALID, "%s: with a dropout samples * pixels * channels must be at most 2^34", what);
    if (int rc = check_pixels(&in->x, h, in, false, "x")) return rc;
    if (in->weight)
        if (int rc = check_params(in->weight, in->weight_stride, 0, h->n, "weight")) return rc;
    if (in->bias)
        if (int rc = check_params(in->bias, in->bias_stride, 0, h->n, "bias")) return rc;
    return h->drop ? check_step_at(in->step_at) : CSER_OK;
}

int check_stats(const float *stats) {
    if (int rc = check_device_ptr(stats, "stats")) return rc;
    return aligned(stats, 4) ? CSER_OK : fail(CSER_ERR_INVALID, "stats: a pointer is not aligned to its element type");
}

}  // namespace layers
}  // namespace

extern "C" {

cser_norm_handle cser_norm_create(int32_t n_workers, int64_t max_samples, int64_t channels, int64_t groups, int32_t act, float eps,
                                  int32_t type, cser_drop_handle drop) {
    auto bad = [](int code, const char *what) { fail(code, "cser_norm_create: %s", what); return nullptr; };
    if (n_workers < 1 || n_workers > 4096 || max_samples < 1 || max_samples > (1 << 24) / n_workers)
        return bad(CSER_ERR_INVALID, "n_workers must be in 1..4096, max_samples positive and their product at most 2^24");
    if (channels < 1 || channels > 65536 || groups < 1 || channels % groups)
        return bad(CSER_ERR_INVALID, "channels must be in 1..65536 and a multiple of groups");
    if ((long long)n_workers * max_samples > 0x7fffffff / groups)
        return bad(CSER_ERR_INVALID, "n_workers * max_samples * groups must be below 2^31");
    if (act != CSER_ACT_NONE && act != CSER_ACT_RELU && act != CSER_ACT_SILU)
        return bad(CSER_ERR_INVALID, "act must be CSER_ACT_NONE, CSER_ACT_RELU or CSER_ACT_SILU");
    if (!(eps >= 0.f) || !isfinite(eps)) return bad(CSER_ERR_INVALID, "eps must be finite and not negative");
    if (type != CSER_TYPE_F32 && type != CSER_TYPE_BF16 && type != CSER_TYPE_F16)
        return bad(CSER_ERR_INVALID, "type must be CSER_TYPE_F32, CSER_TYPE_BF16 or CSER_TYPE_F16");
    if (drop && (drop->n != n_workers || drop->cols != channels || drop->type != type))
        return bad(CSER_ERR_INVALID, "the dropout must be for the same workers, channels and type");
    cser_norm *h = new (std::nothrow) cser_norm;
    if (!h) return bad(CSER_ERR_NOMEM, "host allocation failed");
    h->n = n_workers, h->max_samples = max_samples, h->channels = channels, h->groups = groups, h->act = act, h->eps = eps, h->type = type;
    if (drop) h->drop = true, h->dropout = *drop, h->dropout.part = nullptr;
    const long long all = (long long)n_workers * max_samples;
    h->plane = (all + layers::kBusy) * channels;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaMalloc(&h->part, (size_t)h->plane * 2 * 4);
    if (e == cudaSuccess) e = cudaMalloc(&h->group_sums, (size_t)(all * groups) * sizeof(float2));
    if (e != cudaSuccess) {
        fail(e == cudaErrorMemoryAllocation ? CSER_ERR_NOMEM : CSER_ERR_CUDA, "cser_norm_create: %s", cudaGetErrorString(e));
        cser_norm_destroy(h);
        return nullptr;
    }
    return h;
}

int cser_norm_apply(cser_norm_handle h, const cser_norm_inputs *in, const cser_pixels *y, float *stats, void *stream) {
    using namespace layers;
    bool empty;
    cudaStream_t st = (cudaStream_t)stream;
    if (int rc = check_norm(h, in, "cser_norm_apply", &empty)) return rc;
    if (in->samples == 0) return CSER_OK;
    if (int rc = check_stats(stats)) return rc;
    if (empty) {
        TRY(cudaMemsetAsync(stats, 0, (size_t)(2 * h->n * in->samples * h->groups) * 4, st));
        return CSER_OK;
    }
    if (!y) return fail(CSER_ERR_INVALID, "cser_norm_apply: NULL array");
    if (int rc = check_pixels(y, h, in, true, "cser_norm_apply: y")) return rc;
    const Given all[] = {{"y", pixels_of(y, h, in), true, true},
                         {"x", pixels_of(&in->x, h, in), false, true},
                         {"stats", stats_of(stats, h, in), true, false},
                         {"weight", params_of(in->weight, in->weight_stride, h->channels, h->n), false, false},
                         {"bias", params_of(in->bias, in->bias_stride, h->channels, h->n), false, false}};
    if (int rc = check_apart(all, "cser_norm_apply")) return rc;
    if (h->type == CSER_TYPE_F32) return norm_apply<float>(h, in, y, stats, st);
    return h->type == CSER_TYPE_BF16 ? norm_apply<__nv_bfloat16>(h, in, y, stats, st) : norm_apply<__half>(h, in, y, stats, st);
}

int cser_norm_grad(cser_norm_handle h, const cser_norm_inputs *in, const float *stats, const cser_pixels *dy, const cser_pixels *dx,
                   float *dweight, int64_t dweight_stride, float *dbias, int64_t dbias_stride, void *stream) {
    using namespace layers;
    bool empty;
    cudaStream_t st = (cudaStream_t)stream;
    if (int rc = check_norm(h, in, "cser_norm_grad", &empty)) return rc;
    if (dweight)
        if (int rc = check_params(dweight, dweight_stride, h->channels, h->n, "cser_norm_grad: dweight")) return rc;
    if (dbias)
        if (int rc = check_params(dbias, dbias_stride, h->channels, h->n, "cser_norm_grad: dbias")) return rc;
    if (empty) {
        if (int rc = clear_params(dweight, dweight_stride, h->channels, h->n, st)) return rc;
        return clear_params(dbias, dbias_stride, h->channels, h->n, st);
    }
    if (!dx && !dweight && !dbias) return CSER_OK;
    if (int rc = check_stats(stats)) return rc;
    if (!dy) return fail(CSER_ERR_INVALID, "cser_norm_grad: NULL array");
    if (int rc = check_pixels(dy, h, in, false, "cser_norm_grad: dy")) return rc;
    if (dx)
        if (int rc = check_pixels(dx, h, in, true, "cser_norm_grad: dx")) return rc;
    const Given all[] = {{"dx", pixels_of(dx, h, in), true, true},
                         {"x", pixels_of(&in->x, h, in), false, true},
                         {"dy", pixels_of(dy, h, in), false, true},
                         {"stats", stats_of(stats, h, in), false, false},
                         {"weight", params_of(in->weight, in->weight_stride, h->channels, h->n), false, false},
                         {"bias", params_of(in->bias, in->bias_stride, h->channels, h->n), false, false},
                         {"dweight", params_of(dweight, dweight_stride, h->channels, h->n), true, false},
                         {"dbias", params_of(dbias, dbias_stride, h->channels, h->n), true, false}};
    if (int rc = check_apart(all, "cser_norm_grad")) return rc;
    if (h->type == CSER_TYPE_F32) return norm_grad<float>(h, in, stats, dy, dx, dweight, dweight_stride, dbias, dbias_stride, st);
    return h->type == CSER_TYPE_BF16 ? norm_grad<__nv_bfloat16>(h, in, stats, dy, dx, dweight, dweight_stride, dbias, dbias_stride, st)
                                     : norm_grad<__half>(h, in, stats, dy, dx, dweight, dweight_stride, dbias, dbias_stride, st);
}

void cser_norm_destroy(cser_norm_handle h) {
    if (!h) return;
    if (h->part) cudaFree(h->part);
    if (h->group_sums) cudaFree(h->group_sums);
    delete h;
}

int64_t cser_norm_launch_count(cser_norm_handle h) { return h ? h->launches : 0; }

}  // extern "C"
