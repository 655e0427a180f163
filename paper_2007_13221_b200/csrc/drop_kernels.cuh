// drop_kernels.cuh - dropout with its mask drawn on the spot, forward and gradient.
// Device code; included by layers.cuh inside its unnamed namespace.
//
//   y = residual + keep * (x + bias) / (1 - p),   dx = keep * dy / (1 - p),   dbias = sum over rows of dx
//
// A draw is one Philox call for four elements: its number is the element's place in the worker's array, so a thread draws what it needs
// wherever it stands and nothing is stored.  Bound: memory; a call's 20 wide multiplies and 40 xors for 16 bytes in and
// out of 16-bit elements are about half of what the SMs issue in the time of the traffic.
#pragma once

template <typename T> struct DropArgs {
    const T *x, *r;                                    // r: residual, or null
    T *y;                                              // or null (sums alone)
    const float *bias;                                 // or null
    float *part;                                       // column sums of each chunk of rows, or null
    long long x_row, x_worker, r_row, r_worker, y_row, y_worker, bias_worker;
    long long rows, cols, part_worker;                 // part_worker: from one worker's sums to the next
    int tx, col_blocks, chunks;
    long long chunk_rows;
    int ahead;                                         // elements between a 16-byte boundary and a worker's first element (flat)
    Draw draw;
};

// One rounding with a residual, and the same in every kernel: results do not depend on strides or alignment.
__device__ __forceinline__ float dropped_out(float v, bool keep, float factor, bool add, float residual) {
    if (add) return keep ? fmaf(v, factor, residual) : residual;
    return keep ? v * factor : 0.f;
}

// Arrays that are dense for each worker and all begin at the same distance from a 16-byte boundary: one thread a 16-byte vector of the
// worker's array, whatever its rows.  SHIFTED: that distance is not 0, so vectors start in the middle of draws and the first and
// the last are partial.  Grid (vectors / 256, workers).
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(256) drop_flat_kernel(DropArgs<T> a) {
    constexpr int V = 16 / sizeof(T);
    const long long count = a.rows * a.cols;
    const int w = blockIdx.y;
    const long long e = ((long long)blockIdx.x * 256 + threadIdx.x) * V - (SHIFTED ? a.ahead : 0);
    if (e >= count) return;
    const T *x = a.x + w * a.x_worker + e, *r = a.r ? a.r + w * a.r_worker + e : nullptr;
    T *y = a.y + w * a.y_worker + e;
    const bool whole = e >= 0 && e + V <= count;
    Vec<T, V> vx, vr;
    if (whole) {
        vx = Vec<T, V>(x);
        if (r) vr = Vec<T, V>(r);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j >= 0 && e + j < count) {
                vx.at[j] = x[j];
                if (r) vr.at[j] = r[j];
            }
    }
    const uint32_t keep = keep_bits<V, !SHIFTED>(a.draw, step_of(a.draw), a.draw.c3 + w, e);
    float f[V];
    vx.floats(f);
    if (a.bias) {
        const float *b = a.bias + w * a.bias_worker;
        long long c = e < 0 ? 0 : count <= 0xffffffffll && a.cols <= 0xffffffffll ? (uint32_t)e % (uint32_t)a.cols : e % a.cols;
        if (e < 0) c = (a.cols - (-e) % a.cols) % a.cols;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (whole || (e + j >= 0 && e + j < count)) f[j] += b[c];
            if (++c == a.cols) c = 0;
        }
    }
    float g[V];
    if (r) vr.floats(g);
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = dropped_out(f[j], keep >> j & 1, a.draw.factor, r != nullptr, g[j]);
    Vec<T, V> out;
    out.round(f);
    if (whole) {
        out.to(y);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j >= 0 && e + j < count) y[j] = out.at[j];
    }
}

// Any strides, and sums over rows: a thread keeps V neighbouring columns and walks down the rows of its chunk.  VECTOR: every row of
// every array begins on a 16-byte boundary and holds whole vectors.  256 threads are tx columns of vectors (a power of two up to 32) x
// 256 / tx rows.  Grid: column blocks x chunks x workers, flattened.
template <typename T, bool VECTOR, bool SUMS>
__global__ void __launch_bounds__(256) drop_rows_kernel(DropArgs<T> a) {
    constexpr int V = 16 / sizeof(T);
    const int col_block = blockIdx.x % a.col_blocks, rest = blockIdx.x / a.col_blocks, chunk = rest % a.chunks, w = rest / a.chunks;
    const int tx = threadIdx.x & (a.tx - 1), ty = threadIdx.x / a.tx, step_rows = 256 / a.tx;
    const long long c = ((long long)col_block * a.tx + tx) * V;
    const int here = c >= a.cols ? 0 : a.cols - c < V ? (int)(a.cols - c) : V;
    const long long first = chunk * a.chunk_rows, last = first + a.chunk_rows < a.rows ? first + a.chunk_rows : a.rows;
    const unsigned long long step = step_of(a.draw);
    const uint32_t c3 = a.draw.c3 + w;
    float b[V], sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        b[j] = a.bias && j < here ? a.bias[w * a.bias_worker + c + j] : 0.f;
        sum[j] = 0.f;
    }
    if (here)
        for (long long row = first + ty; row < last; row += step_rows) {
            const T *x = a.x + w * a.x_worker + row * a.x_row + c, *r = a.r ? a.r + w * a.r_worker + row * a.r_row + c : nullptr;
            T *y = a.y ? a.y + w * a.y_worker + row * a.y_row + c : nullptr;
            Vec<T, V> vx, vr;
            if (VECTOR) {
                vx = Vec<T, V>(x);
                if (r) vr = Vec<T, V>(r);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j < here) {
                        vx.at[j] = x[j];
                        if (r) vr.at[j] = r[j];
                    }
            }
            const uint32_t keep = keep_bits<V, VECTOR>(a.draw, step, c3, row * a.cols + c);
            float f[V], g[V];
            vx.floats(f);
            if (r) vr.floats(g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool k = keep >> j & 1 && j < here;
                const float v = f[j] + b[j];
                if (SUMS) sum[j] += k ? v * a.draw.factor : 0.f;
                f[j] = dropped_out(v, k, a.draw.factor, r != nullptr, g[j]);
            }
            if (!y) continue;
            Vec<T, V> out;
            out.round(f);
            if (VECTOR) {
                out.to(y);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j < here) y[j] = out.at[j];
            }
        }
    if (!SUMS) return;
    // Rows of a warp first, then the eight warps.
    __shared__ float sums[8][32 * V];
    for (int o = a.tx; o < 32; o <<= 1)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += __shfl_xor_sync(~0u, sum[j], o);
    if ((threadIdx.x & 31) < a.tx)
#pragma unroll
        for (int j = 0; j < V; ++j) sums[threadIdx.x >> 5][tx * V + j] = sum[j];
    __syncthreads();
    const long long col = (long long)col_block * a.tx * V + threadIdx.x;
    if (threadIdx.x < a.tx * V && col < a.cols) {
        float s = sums[0][threadIdx.x];
#pragma unroll
        for (int k = 1; k < 8; ++k) s += sums[k][threadIdx.x];
        a.part[w * a.part_worker + chunk * a.cols + col] = s;
    }
}
