// drop_kernels.cuh - dropout with its mask drawn on the spot, forward and gradient.
// Device code; included by layers.cuh inside its unnamed namespace.
//
//   y = residual + keep * (x + bias) / (1 - p),   dx = keep * dy / (1 - p),   dbias = sum over rows of dx
//
// A call of the generator makes four draws: its number is the element's place in the worker's array, so a thread draws what it needs
// wherever it stands and nothing is stored.  Bound: memory for 32-bit elements (8 x 4096 x 1024 with bias and residual 6.7 TB/s), the generator for
// 16-bit ones: of the 176 cycles that an SM's quarter has for eight of them at the copy rate, two calls' wide multiplies occupy their pipe
// for 140 (four cycles each) and all instructions about 140 slots, and the two overlap to 225 (8 x 8192 x 4096 5.2 TB/s, 206 us; floor 164).  So what
// all calls share is made once a thread (the round that differs in one word, the first product, which grows by addition from call to call:
// 379 -> 206 us together with whole vectors), and nothing is drawn twice that a neighbour has.  Tried: products from the FP64 pipe (106 cycles a
// call for 88), high and low halves apart (90).
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
    long long walked, last_row;                        // such rows, and elements of the last, with nothing ahead
    int tx, log_rows, col_blocks, chunks;              // log_rows: of 256 / tx
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

constexpr int kFlat = 4;

// The kFlat * 32 vectors of a warp, from its lane's element e0 on.  CHECKED: some of their elements may not exist.
template <typename T, bool SHIFTED, bool RESIDUAL, bool CHECKED>
__device__ __forceinline__ void drop_flat_warp(const DropArgs<T> &a, int w, int lane, long long e0, long long count) {
    constexpr int V = 16 / sizeof(T);
    const T *x = a.x + w * a.x_worker + e0, *r = RESIDUAL ? a.r + w * a.r_worker + e0 : nullptr;
    T *y = a.y + w * a.y_worker + e0;
    Vec<T, V> vx[kFlat], vr[kFlat];
    auto whole = [&](int u) { return !CHECKED || (e0 + u * 32 * V >= 0 && e0 + (u * 32 + 1) * V <= count); };
#pragma unroll
    for (int u = 0; u < kFlat; ++u) {
        const long long e = e0 + u * 32 * V;
        if (whole(u)) {
            vx[u] = Vec<T, V>(x + u * 32 * V);
            if (RESIDUAL) vr[u] = Vec<T, V>(r + u * 32 * V);
        } else {
            load_some<T, V>(vx[u], x + u * 32 * V, -e, count - e);
            if (RESIDUAL) load_some<T, V>(vr[u], r + u * 32 * V, -e, count - e);
        }
    }
    const Words words(a.draw, w);
    const uint64_t call = Words::call(e0 >> 2);
    const uint32_t by = (uint32_t)e0 & 3;
    uint32_t next[3];                                  // the first draws of the 32 vectors behind
    if (SHIFTED) {
        uint32_t four[4];
        words.four(four, call + (uint64_t)((kFlat * 32 - lane) * (V / 4)) * Words::kCall);
        next[0] = four[0], next[1] = four[1], next[2] = four[2];
    }
#pragma unroll
    for (int u = kFlat - 1; u >= 0; --u) {
        uint32_t d[V + 3];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) words.four(d + 4 * k, call + (u * 8 * V + k) * Words::kCall);
        if (SHIFTED) {
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                const uint32_t neighbour = __shfl_down_sync(~0u, d[j], 1), first = __shfl_sync(~0u, d[j], 0);
                d[V + j] = lane == 31 ? next[j] : neighbour;
                next[j] = first;
            }
            shift_words(d, by);
        }
        float f[V], g[V];
        vx[u].floats(f);
        if (RESIDUAL) vr[u].floats(g);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = dropped_out(f[j], d[j] >= a.draw.threshold, a.draw.factor, RESIDUAL, RESIDUAL ? g[j] : 0.f);
        vx[u].round(f);
        if (whole(u))
            vx[u].to(y + u * 32 * V);
        else
            store_some<T, V>(vx[u], y + u * 32 * V, -(e0 + u * 32 * V), count - (e0 + u * 32 * V));
    }
}

// Arrays that are dense for each worker and lie alike: all at the same distance from a 16-byte boundary.  Without bias and sums
// columns do not matter: a warp takes kFlat * 32 vectors of the worker's array, 32 at a time.  SHIFTED: for some worker that distance is not
// 0, so vectors start in the middle of four draws; what a lane lacks is its neighbour's, or, for the last lane, the first's of the 32
// vectors behind, which are drawn first.  Grid (vectors / (256 kFlat), workers).
template <typename T, bool SHIFTED, bool RESIDUAL>
__global__ void __launch_bounds__(256) drop_flat_kernel(DropArgs<T> a) {
    constexpr int V = 16 / sizeof(T);
    after_previous();
    let_next();
    const long long count = a.rows * a.cols;
    const int w = blockIdx.y, lane = threadIdx.x & 31;
    const int ahead = SHIFTED ? (a.ahead + w * a.ahead_worker) % V : 0;
    const long long first = (long long)blockIdx.x * (256 * kFlat * V) - ahead;          // of the block
    const long long e0 = first + ((threadIdx.x >> 5) * (kFlat * 32) + lane) * V;
    if (first >= 0 && first + 256 * kFlat * V <= count)
        drop_flat_warp<T, SHIFTED, RESIDUAL, false>(a, w, lane, e0, count);
    else if (e0 - lane * V < count)                    // the whole warp
        drop_flat_warp<T, SHIFTED, RESIDUAL, true>(a, w, lane, e0, count);
}

// With a bias or sums over rows, and for any strides: a thread keeps V neighbouring columns and walks down the rows of its chunk.  256
// threads are tx columns of vectors (a power of two up to 32) x 256 / tx rows.  Grid: column blocks x chunks x workers, flattened.
//   DENSE  arrays as the flat kernel takes them, walked as rows of `width` elements, so many rows of theirs that vectors end with them (and
//          fill a block), whatever the columns; `ahead` elements of the first row do not exist, and the last can be short.
//          Sums are of all `width` columns; those of one column are added up with the chunks.
//   PLAIN  rows that begin on 16-byte boundaries and hold whole vectors (width = cols).
//   ODD    any rows, element by element.
enum DropRows { kDense, kPlain, kOdd };
enum DropKind { kSums, kForward, kResidual };       // the gradient with sums; the forward pass without and with a residual
template <typename T, int MODE, bool SHIFTED, int KIND>
__global__ void __launch_bounds__(256, 4) drop_rows_kernel(DropArgs<T> a) {
    constexpr int V = 16 / sizeof(T);
    constexpr bool SUMS = KIND == kSums, residual = KIND == kResidual;
    after_previous();
    let_next();
    const int col_block = blockIdx.x % a.col_blocks, rest = blockIdx.x / a.col_blocks, chunk = rest % a.chunks, w = rest / a.chunks;
    const int tx = threadIdx.x & (a.tx - 1), step_rows = 1 << a.log_rows, ty = threadIdx.x >> (8 - a.log_rows);
    const long long count = a.rows * a.cols;
    const int ahead = MODE == kDense && SHIFTED ? (a.ahead + w * a.ahead_worker) % V : 0;
    const long long c = ((long long)col_block * a.tx + tx) * V;                    // of the row as it is walked
    const long long walked = a.walked + (MODE == kDense && a.last_row + ahead > a.width);
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
        if (!SUMS && a.bias && in && col < a.cols) b[j] = a.bias[w * a.bias_worker + col];
        if (++col == a.cols && MODE == kDense) col = 0;
    }
    if (in && first + ty < last) {
        // Places of the thread's first row, and how far its next is.
        const long long row0 = first + ty, e_row = MODE == kDense ? a.width : a.cols, e = row0 * e_row + c - ahead;
        const long long x_step = (MODE == kDense ? a.width : a.x_row) << a.log_rows, r_step = (MODE == kDense ? a.width : a.r_row) << a.log_rows,
                        y_step = (MODE == kDense ? a.width : a.y_row) << a.log_rows, e_step = e_row << a.log_rows;
        const bool store = !SUMS || a.y;
        uint64_t call = Words::call(e >> 2);
        const uint64_t call_step = Words::call(e_step >> 2);                               // (not odd: rows are whole fours)
        const uint32_t by = (uint32_t)e & 3;
        const T *x = a.x + w * a.x_worker + (e - (MODE == kDense ? 0 : row0 * (e_row - a.x_row))), *r = nullptr;
        T *y = nullptr;
        if (residual) r = a.r + w * a.r_worker + (e - (MODE == kDense ? 0 : row0 * (e_row - a.r_row)));
        if (store) y = a.y + w * a.y_worker + (e - (MODE == kDense ? 0 : row0 * (e_row - a.y_row)));
        const int steps = (int)((last - row0 + step_rows - 1) >> a.log_rows);

        auto finish = [&](Vec<T, V> &vx, const Vec<T, V> &vr, const Drawn<V, !SHIFTED> &d) {
            float f[V], g[V];
            vx.floats(f);
            if (residual) vr.floats(g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                f[j] = dropped_out(SUMS ? f[j] : f[j] + b[j], d.w[j] >= a.draw.threshold, a.draw.factor, residual, residual ? g[j] : 0.f);
                if (SUMS) sum[j] += f[j];
            }
            vx.round(f);
        };
        auto next = [&](int rows) {
            x += rows * x_step, call += rows * call_step;
            if (residual) r += rows * r_step;
            if (store) y += rows * y_step;
        };
        // A row of which some elements may not exist, or that begins anywhere.
        auto some = [&](int i) {
            const long long at = e + i * e_step, begin = MODE == kDense ? -at : 0, end = MODE == kDense ? count - at : a.cols - c;
            Vec<T, V> vx, vr;
#pragma unroll
            for (int j = 0; j < V; ++j) vx.at[j] = vr.at[j] = from_float<T>(0.f);
            load_some<T, V>(vx, x, begin, end);
            if (residual) load_some<T, V>(vr, r, begin, end);
            finish(vx, vr, Drawn<V, !SHIFTED>(words, at));
            if (store) store_some<T, V>(vx, y, begin, end);
            next(1);
        };
        int i = 0;
        if (MODE == kOdd) {
            for (; i < steps; ++i) some(i);
        } else {
            // Of the dense rows only the first and the last can be short.
            const bool short_last = MODE == kDense && row0 + ((long long)(steps - 1) << a.log_rows) == walked - 1;
            const int whole = short_last ? steps - 1 : steps;
            if (MODE == kDense && row0 == 0 && whole) some(i++);
            // Rows whose loads are under way together (8 x 4096 x 1024: two for all 32-bit rows with a bias 47 us for 42, four for 16-bit ones
            // with a residual 38 for 35).
            constexpr int U = residual || V == 8 ? 2 : 4;
            for (; i + U <= whole; i += U) {
                Vec<T, V> vx[U], vr[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    vx[u] = Vec<T, V>(x + u * x_step);
                    if (residual) vr[u] = Vec<T, V>(r + u * r_step);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    finish(vx[u], vr[u], Drawn<V, !SHIFTED>(words, call + u * call_step, by));
                    if (store) vx[u].to(y + u * y_step);
                }
                next(U);
            }
            for (; i < whole; ++i) {
                Vec<T, V> vx(x), vr;
                if (residual) vr = Vec<T, V>(r);
                finish(vx, vr, Drawn<V, !SHIFTED>(words, call, by));
                if (store) vx.to(y);
                next(1);
            }
            if (i < steps) some(i);
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
    const long long k = (long long)col_block * a.tx * V + threadIdx.x;
    if (threadIdx.x < a.tx * V && k < a.width) {
        float s = sums[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 8; ++i) s += sums[i][threadIdx.x];
        const long long at = k < ahead ? k - ahead + a.width : k - ahead;
        a.part[w * a.part_worker + chunk * a.width + at] = s;
    }
}
