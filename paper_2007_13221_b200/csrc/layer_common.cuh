// layer_common.cuh - what the layers' kernels share: vectors of elements, draws of the dropout, sums over rows.
// Device code; included by layers.cuh inside its unnamed namespace.
#pragma once

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

// ------------------------------------------------------------------ draws
struct Draw {
    uint32_t k0 = 0, k1 = 0, c3 = 0, threshold = 0;    // c3: of the first worker
    float factor = 1.f;                                // 1 / (1 - p)
    unsigned long long step = 0;
    const unsigned long long *step_at = nullptr;
};

__device__ __forceinline__ unsigned long long step_of(const Draw &d) { return d.step_at ? d.step + *d.step_at : d.step; }

// Keep bits of the V elements from element e of a worker's array on, bit j for e + j.  V a multiple of 4 with e too: V / 4 draws.
// Otherwise one draw more, and the words are shifted into place.
template <int V, bool ALIGNED>
__device__ __forceinline__ uint32_t keep_bits(const Draw &d, unsigned long long step, uint32_t c3, long long e) {
    constexpr int kDraws = ALIGNED ? V / 4 : (V + 2) / 4 + 1;
    uint32_t w[kDraws * 4];
    const uint32_t q = (uint32_t)(e >> 2);
#pragma unroll
    for (int k = 0; k < kDraws; ++k) {
        uint32_t four[4];
        philox4x32_10(four, d.k0, d.k1, q + k, (uint32_t)step, (uint32_t)(step >> 32), c3);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[k * 4 + j] = four[j];
    }
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < kDraws * 4; ++j) bits |= (w[j] >= d.threshold ? 1u : 0u) << j;
    return ALIGNED ? bits : bits >> ((uint32_t)e & 3);
}

// ------------------------------------------------------------------ sums over rows
// out[k][i][c] = sum over r of part[k][i][r][c], in an order of its own for each (k, i, c): 32 lanes of rows each take every 32nd, and
// their sums are added in order.  Grid (ceil(cols / 32), n, planes), 1024 threads: a warp reads 32 columns of a row.
struct RowSums {
    const float *part;
    float *out[2];
    long long out_stride[2];
    long long rows, cols, plane;                       // plane: elements from one plane of parts to the next
};
__global__ void __launch_bounds__(1024) sum_rows_kernel(RowSums a) {
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float *out = a.out[blockIdx.z];
    if (!out) return;
    const float *p = a.part + blockIdx.z * a.plane + (long long)blockIdx.y * a.rows * a.cols;
    float s = 0.f;
    if (c < a.cols) {
        long long r = warp;
        for (; r + 96 < a.rows; r += 128) {
            const float v0 = p[r * a.cols + c], v1 = p[(r + 32) * a.cols + c], v2 = p[(r + 64) * a.cols + c], v3 = p[(r + 96) * a.cols + c];
            s = ((s + v0) + v1) + (v2 + v3);
        }
        for (; r < a.rows; r += 32) s += p[r * a.cols + c];
    }
    sums[warp][lane] = s;
    __syncthreads();
    s = sums[lane][warp];                              // warp now stands for the column
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    const long long col = (long long)blockIdx.x * 32 + warp;
    if (lane == 0 && col < a.cols) out[blockIdx.y * a.out_stride[blockIdx.z] + col] = s;
}
