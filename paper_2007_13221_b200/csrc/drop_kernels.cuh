// drop_kernels.cuh - dropout with its mask drawn on the spot, forward and gradient.
// Device code; included by layers.cuh inside its unnamed namespace.
//
//   y = residual + keep * (x + bias) / (1 - p),   dx = keep * dy / (1 - p),   dbias = sum over rows of dx
//
// A call of the generator makes four draws: its number is the element's place in the worker's array, so a thread draws what it needs
// wherever it stands and nothing is stored.  Bound: memory, with the generator close behind for 16-bit elements (a call's 18 wide
// multiplies occupy their pipe for four cycles each: eight elements take 144 of the 176 cycles that an SM's quarter has for them
// at the copy rate), so nothing is drawn twice that a neighbour has and what all calls share is made once a thread.
#pragma once

template <typename T> struct DropArgs {
    const T *x, *r;                                    // r: residual, or null
    T *y;                                              // or null (sums alone)
    const float *bias;                                 // or null
    float *part;                                       // column sums of each chunk of rows, or null
    long long x_row, x_worker, r_row, r_worker, y_row, y_worker, bias_worker;
    long long rows, cols, part_worker;                 // part_worker: from one worker's sums to the next
    long long width;                                   // elements of a row as it is walked
    long long chunk_rows;
    int tx, col_blocks, chunks;
    int ahead, ahead_worker;                           // elements between a 16-byte boundary and the first worker's first element; more for each worker
    Draw draw;
};

// One rounding with a residual, and the same in every kernel: results do not depend on strides or alignment.
__device__ __forceinline__ float dropped_out(float v, bool keep, float factor, bool add, float residual) {
    if (add) return keep ? fmaf(v, factor, residual) : residual;
    return keep ? v * factor : 0.f;
}

// V elements of which those from `first` up to, not with, `end` exist.
template <typename T, int V> __device__ __forceinline__ void load_some(Vec<T, V> &v, const T *p, long long first, long long end) {
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j >= first && j < end) v.at[j] = p[j];
}
template <typename T, int V> __device__ __forceinline__ void store_some(const Vec<T, V> &v, T *p, long long first, long long end) {
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j >= first && j < end) p[j] = v.at[j];
}

// Arrays that are dense for each worker and lie alike: all at the same distance from a 16-byte boundary.  Without bias and sums
// columns do not matter: a warp takes kFlat * 32 vectors of the worker's array, 32 at a time.  SHIFTED: for some worker that distance is not
// 0, so vectors start in the middle of four draws; what a lane lacks is its neighbour's, or, for the last lane, the first's of the 32
// vectors behind, which are drawn first.  Grid (vectors / (256 kFlat), workers).
constexpr int kFlat = 4;
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(256) drop_flat_kernel(DropArgs<T> a) {
    constexpr int V = 16 / sizeof(T);
    const long long count = a.rows * a.cols;
    const int w = blockIdx.y, lane = threadIdx.x & 31;
    const int ahead = SHIFTED ? (a.ahead + w * a.ahead_worker) % V : 0;
    const long long e0 = (((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * (kFlat * 32) + lane) * V - ahead;
    if (e0 - lane * V >= count) return;                // the whole warp
    const T *x = a.x + w * a.x_worker + e0, *r = a.r ? a.r + w * a.r_worker + e0 : nullptr;
    T *y = a.y + w * a.y_worker + e0;
    Vec<T, V> vx[kFlat], vr[kFlat];
#pragma unroll
    for (int u = 0; u < kFlat; ++u) {
        const long long e = e0 + u * 32 * V;
        if (e >= 0 && e + V <= count) {
            vx[u] = Vec<T, V>(x + u * 32 * V);
            if (r) vr[u] = Vec<T, V>(r + u * 32 * V);
        } else {
            load_some<T, V>(vx[u], x + u * 32 * V, -e, count - e);
            if (r) load_some<T, V>(vr[u], r + u * 32 * V, -e, count - e);
        }
    }
    const Words words(a.draw, w);
    uint32_t next[3];                                  // the first draws of the 32 vectors behind
    if (SHIFTED) {
        uint32_t four[4];
        words.four(four, (uint32_t)((e0 + (kFlat * 32 - lane) * V) >> 2));
        next[0] = four[0], next[1] = four[1], next[2] = four[2];
    }
#pragma unroll
    for (int u = kFlat - 1; u >= 0; --u) {
        const long long e = e0 + u * 32 * V;
        uint32_t d[V + 3];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) words.four(d + 4 * k, (uint32_t)(e >> 2) + k);
        if (SHIFTED) {
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                const uint32_t neighbour = __shfl_down_sync(~0u, d[j], 1), first = __shfl_sync(~0u, d[j], 0);
                d[V + j] = lane == 31 ? next[j] : neighbour;
                next[j] = first;
            }
            shift_words(d, (uint32_t)e & 3);
        }
        float f[V], g[V];
        vx[u].floats(f);
        if (r) vr[u].floats(g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = dropped_out(f[j], d[j] >= a.draw.threshold, a.draw.factor, r != nullptr, g[j]);
        vx[u].round(f);
        if (e >= 0 && e + V <= count)
            vx[u].to(y + u * 32 * V);
        else
            store_some<T, V>(vx[u], y + u * 32 * V, -e, count - e);
    }
}

// With a bias or sums over rows, and for any strides: a thread keeps V neighbouring columns and walks down the rows of its chunk.  256
// threads are tx columns of vectors (a power of two up to 32) x 256 / tx rows.  Grid: column blocks x chunks x workers, flattened.
//   DENSE  arrays as the flat kernel takes them, walked as rows of `width` elements, so many rows of theirs that vectors end with them (and
//          fill a block), whatever the columns; `ahead` elements of the first row do not exist, and the last can be short.
//          Sums are of all `width` columns; those of one column are added up with the chunks.
//   PLAIN  rows that begin on 16-byte boundaries and hold whole vectors (width = cols).
//   ODD    any rows, element by element.
enum DropRows { kDense, kPlain, kOdd };
template <typename T, int MODE, bool SHIFTED, bool SUMS>
__global__ void __launch_bounds__(256) drop_rows_kernel(DropArgs<T> a) {
    constexpr int V = 16 / sizeof(T);
    const int col_block = blockIdx.x % a.col_blocks, rest = blockIdx.x / a.col_blocks, chunk = rest % a.chunks, w = rest / a.chunks;
    const int tx = threadIdx.x & (a.tx - 1), ty = threadIdx.x / a.tx, step_rows = 256 / a.tx;
    const long long count = a.rows * a.cols;
    const int ahead = MODE == kDense && SHIFTED ? (a.ahead + w * a.ahead_worker) % V : 0;
    const long long c = ((long long)col_block * a.tx + tx) * V;                    // of the row as it is walked
    const long long walked = MODE == kDense ? (count + ahead + a.width - 1) / a.width : a.rows;
    const long long first = chunk * a.chunk_rows, last = first + a.chunk_rows < walked ? first + a.chunk_rows : walked;
    const bool in = c < a.width;
    const Words words(a.draw, w);
    float b[V], sum[V];
    long long col = c - ahead;
    if (MODE == kDense && a.bias) {                                                // width is a multiple of cols
        col = col < 0 ? col + a.width : col;
        col = a.width <= 0xffffffffll ? (uint32_t)col % (uint32_t)a.cols : col % a.cols;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        b[j] = sum[j] = 0.f;
        if (a.bias && in && col < a.cols) b[j] = a.bias[w * a.bias_worker + col];
        if (++col == a.cols && MODE == kDense) col = 0;
    }
    if (in)
        for (long long row = first + ty; row < last; row += step_rows) {
            const long long e = MODE == kDense ? row * a.width + c - ahead : row * a.cols + c;
            const T *x, *r = nullptr;
            T *y = nullptr;
            if (MODE == kDense) {
                x = a.x + w * a.x_worker + e;
                if (a.r) r = a.r + w * a.r_worker + e;
                if (a.y) y = a.y + w * a.y_worker + e;
            } else {
                x = a.x + w * a.x_worker + row * a.x_row + c;
                if (a.r) r = a.r + w * a.r_worker + row * a.r_row + c;
                if (a.y) y = a.y + w * a.y_worker + row * a.y_row + c;
            }
            const long long begin = MODE == kDense ? -e : 0, end = MODE == kDense ? count - e : a.cols - c;
            const bool whole = MODE == kPlain || (MODE == kDense && begin <= 0 && end >= V);
            Vec<T, V> vx, vr;
            if (whole) {
                vx = Vec<T, V>(x);
                if (r) vr = Vec<T, V>(r);
            } else {
                load_some<T, V>(vx, x, begin, end);
                if (r) load_some<T, V>(vr, r, begin, end);
            }
            const Drawn<V, !SHIFTED> d(words, e);
            float f[V], g[V];
            vx.floats(f);
            if (r) vr.floats(g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool keep = d.w[j] >= a.draw.threshold && (whole || (j >= begin && j < end));
                const float v = f[j] + b[j];
                if (SUMS) sum[j] += keep ? v * a.draw.factor : 0.f;
                f[j] = dropped_out(v, keep, a.draw.factor, r != nullptr, g[j]);
            }
            if (!y) continue;
            vx.round(f);
            if (whole)
                vx.to(y);
            else
                store_some<T, V>(vx, y, begin, end);
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
    const long long k = (long long)col_block * a.tx * V + threadIdx.x;
    if (threadIdx.x < a.tx * V && k < a.width) {
        float s = sums[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 8; ++i) s += sums[i][threadIdx.x];
        const long long at = k < ahead ? k - ahead + a.width : k - ahead;
        a.part[w * a.part_worker + chunk * a.width + at] = s;
    }
}
