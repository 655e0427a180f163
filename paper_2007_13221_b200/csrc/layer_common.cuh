// layer_common.cuh - what the layers' kernels share: vectors of elements, draws of the dropout, sums over rows.
// Device code; included by layers.cuh inside its unnamed namespace.
#pragma once

// Every kernel is set up while the one before it in the stream ends, and touches no memory before that end.
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The next kernel may be set up from here on.
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ------------------------------------------------------------------ elements
template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef uint4 type; };
template <> struct Raw<8> { typedef uint2 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float(float v) { return v; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }

// V elements as one load or store; V * sizeof(T) bytes, aligned to that.
template <typename T, int V> struct Vec {
    typedef typename Raw<V * sizeof(T)>::type raw;
    union {
        raw bits;
        T at[V];
    };
    __device__ __forceinline__ Vec() {}
    __device__ __forceinline__ explicit Vec(const T *p) : bits(*reinterpret_cast<const raw *>(p)) {}
    __device__ __forceinline__ void to(T *p) const { *reinterpret_cast<raw *>(p) = bits; }
    __device__ __forceinline__ void floats(float (&f)[V]) const {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = to_float(at[j]);
    }
    __device__ __forceinline__ void round(const float (&f)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) at[j] = from_float<T>(f[j]);
    }
};
template <> __device__ __forceinline__ void Vec<__nv_bfloat16, 8>::floats(float (&f)[8]) const {
    const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(w[j] << 16), f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16, 8>::round(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t *>(&two);
    }
    bits = make_uint4(w[0], w[1], w[2], w[3]);
}
template <> __device__ __forceinline__ void Vec<__half, 8>::round(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2 two = __floats2half2_rn(f[2 * j], f[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t *>(&two);
    }
    bits = make_uint4(w[0], w[1], w[2], w[3]);
}

// Two floats that one instruction works on: half the issue slots of the layers whose arithmetic would otherwise bound them.
struct F2 {
    float x, y;
};
__device__ __forceinline__ unsigned long long bits_of(F2 a) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
    return r;
}
__device__ __forceinline__ F2 pair_of(unsigned long long r) {
    F2 a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(r));
    return a;
}
__device__ __forceinline__ F2 two(float v) { return {v, v}; }
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits_of(a)), "l"(bits_of(b)));
    return pair_of(r);
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits_of(a)), "l"(bits_of(b)));
    return pair_of(r);
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits_of(a)), "l"(bits_of(b)), "l"(bits_of(c)));
    return pair_of(r);
}
__device__ __forceinline__ F2 operator-(F2 a, F2 b) { return fma2(b, two(-1.f), a); }

// V elements as pairs; of a single one the other half is 0.
template <int V> constexpr int kPairs = (V + 1) / 2;
template <typename T, int V> __device__ __forceinline__ void pairs_of(const Vec<T, V> &v, F2 (&p)[kPairs<V>]) {
    float f[V];
    v.floats(f);
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) p[j] = {f[2 * j], 2 * j + 1 < V ? f[(2 * j + 1) % V] : 0.f};
}
template <typename T, int V> __device__ __forceinline__ void round_pairs(Vec<T, V> &v, const F2 (&p)[kPairs<V>]) {
    float f[V];
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = j & 1 ? p[j / 2].y : p[j / 2].x;
    v.round(f);
}

// ------------------------------------------------------------------ draws
struct Draw {
    uint32_t k0 = 0, k1 = 0, c3 = 0, threshold = 0;    // c3: of the first worker
    float factor = 1.f;                                // 1 / (1 - p)
    unsigned long long step = 0;
    const unsigned long long *step_at = nullptr;
};

// A worker's generator.  Of a call's four counter words only the first differs from call to call, so the first round's second product and
// the second round's first are the same for all: they are made once a thread.
struct Words {
    uint32_t k0, k1, a, b, c, d;

    __device__ __forceinline__ Words(const Draw &g, int worker) : k0(g.k0), k1(g.k1) {
        const unsigned long long step = g.step_at ? g.step + *g.step_at : g.step;
        const uint64_t p = (uint64_t)0xCD9E8D57u * (uint32_t)(step >> 32);
        const uint64_t q = (uint64_t)0xD2511F53u * ((uint32_t)(p >> 32) ^ (uint32_t)step ^ k0);
        a = (g.c3 + worker) ^ k1;
        b = (uint32_t)p ^ (k0 + 0x9E3779B9u);
        c = (uint32_t)(q >> 32) ^ (k1 + 0xBB67AE85u);
        d = (uint32_t)q;
    }

    // The first round's first product, of the call number itself: from call to call it grows by kCall, so it is multiplied out once.
    static constexpr uint64_t kCall = 0xD2511F53u;
    __device__ __forceinline__ static uint64_t call(long long number) { return kCall * (uint64_t)number; }

    // The draws of the call with this product.
    __device__ __forceinline__ void four(uint32_t *w, uint64_t p) const {
        const uint64_t q = (uint64_t)0xCD9E8D57u * ((uint32_t)(p >> 32) ^ a);
        uint32_t c0 = (uint32_t)(q >> 32) ^ b, c1 = (uint32_t)q, c2 = (uint32_t)p ^ c, c3 = d;
        philox4x32_rounds<8>(c0, c1, c2, c3, k0 + 2 * 0x9E3779B9u, k1 + 2 * 0xBB67AE85u);
        w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
    }
};

// w[j] <- w[j + by], by in 0..3.
template <int N> __device__ __forceinline__ void shift_words(uint32_t (&w)[N], uint32_t by) {
    if (by & 1) {
#pragma unroll
        for (int j = 0; j + 1 < N; ++j) w[j] = w[j + 1];
    }
    if (by & 2) {
#pragma unroll
        for (int j = 0; j + 2 < N; ++j) w[j] = w[j + 2];
    }
}

// The draws of the V elements from element e of a worker's array on.  ALIGNED: e is a multiple of 4, as V is.  Otherwise a call more,
// and the words are shifted into place.
template <int V, bool ALIGNED> struct Drawn {
    static constexpr int kCalls = ALIGNED ? V / 4 : (V + 2) / 4 + 1;
    uint32_t w[kCalls * 4];
    __device__ __forceinline__ Drawn(const Words &words, uint64_t call, uint32_t by) {
#pragma unroll
        for (int k = 0; k < kCalls; ++k) words.four(w + 4 * k, call + k * Words::kCall);
        if (!ALIGNED) shift_words(w, by);
    }
    __device__ __forceinline__ Drawn(const Words &words, long long e) : Drawn(words, Words::call(e >> 2), (uint32_t)e & 3) {}
};

// ------------------------------------------------------------------ sums over rows
// out[k][i][c] = sum over r of part[k][i][r][c]: a block's warps take every so many rows each, and their sums are added in order.  Grid
// (ceil(cols / 32), n, planes): a warp reads 32 columns of a row.
struct RowSums {
    const float *part;
    float *out[2];
    long long out_stride[2];
    long long rows, cols, plane;                       // plane: elements from one plane of parts to the next
};
__global__ void __launch_bounds__(1024) sum_rows_kernel(RowSums a) {
    __shared__ float sums[32][32];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float *out = a.out[blockIdx.z];
    if (!out) return;
    const float *p = a.part + blockIdx.z * a.plane + (long long)blockIdx.y * a.rows * a.cols + c;
    float s = 0.f;
    if (c < a.cols) {
        constexpr int U = 8;                           // rows whose loads are under way together
        long long r = warp;
        for (; r + (U - 1) * warps < a.rows; r += U * warps) {
            float v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = p[(r + u * warps) * a.cols];
#pragma unroll
            for (int u = 0; u < U; ++u) s += v[u];
        }
#pragma unroll 4
        for (; r < a.rows; r += warps) s += p[r * a.cols];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < a.cols) {
        for (int k = 1; k < warps; ++k) s += sums[k][lane];
        out[blockIdx.y * a.out_stride[blockIdx.z] + c] = s;
    }
}
