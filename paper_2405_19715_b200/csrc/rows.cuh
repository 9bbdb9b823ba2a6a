// Pieces shared by the kernels that take whole vocabulary rows through registers (top_logits.cu, beam.cu,
// distill.cu): rows of any alignment as a grid of 16-byte vectors, order-preserving keys, softmax terms, and the
// split of a row over the CTAs of a thread-block cluster.
#pragma once

#include <cuda_fp16.h>

#include "row_ops.h"
#include "verify_cluster.cuh"

namespace rw {

using sd::f2;

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int NV = 8;                          // 16-byte vectors a thread holds: 32 registers
constexpr int TILE = THREADS * NV;             // vectors of a row that a CTA holds at a time (64 KB)
constexpr int MAX_CLUSTER = 8;

template <typename T> struct Row;
template <> struct Row<float> {
    static constexpr int N = 4, KEY_BITS = 32;   // elements per vector; leading key bits that tell two values apart
    static __device__ __forceinline__ float wide(float v) { return v; }
    static __device__ __forceinline__ uint32_t bits(float v) { return __float_as_uint(v); }
    static __device__ __forceinline__ uint32_t neg_inf() { return 0xff800000u; }
};
template <> struct Row<__nv_bfloat16> {
    static constexpr int N = 8, KEY_BITS = 16;
    static __device__ __forceinline__ float wide(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ uint32_t bits(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
    static __device__ __forceinline__ uint32_t neg_inf() { return 0xff80ff80u; }
};
template <> struct Row<__half> {
    static constexpr int N = 8, KEY_BITS = 19;   // fp16 widened to fp32: sign, 8 exponent bits, 10 of the mantissa
    static __device__ __forceinline__ float wide(__half v) { return __half2float(v); }
    static __device__ __forceinline__ uint32_t bits(__half v) { return __half_as_ushort(v); }
    static __device__ __forceinline__ uint32_t neg_inf() { return 0xfc00fc00u; }
};

// The elements of a vector as fp32, two to a packed register pair; widening is exact.
__device__ __forceinline__ void pairs(const uint4& r, f2 (&x)[2], float) { sd::to_pairs(r, x, 0.f); }
__device__ __forceinline__ void pairs(const uint4& r, f2 (&x)[4], __nv_bfloat16 t) { sd::to_pairs(r, x, t); }
__device__ __forceinline__ f2 half_pair(uint32_t w) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return sd::pack2(v.x, v.y);
}
__device__ __forceinline__ void pairs(const uint4& r, f2 (&x)[4], __half) {
    x[0] = half_pair(r.x); x[1] = half_pair(r.y); x[2] = half_pair(r.z); x[3] = half_pair(r.w);
}
template <typename T>
__device__ __forceinline__ void widen(const uint4& r, float (&x)[Row<T>::N]) {
    f2 p[Row<T>::N / 2];
    pairs(r, p, T());
#pragma unroll
    for (int q = 0; q < Row<T>::N / 2; ++q) sd::unpack2(p[q], x[2 * q], x[2 * q + 1]);
}

// Largest element of a vector; NaN if it holds one.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float vec_max(const uint4& r, float) {
    return max_nan(max_nan(__uint_as_float(r.x), __uint_as_float(r.y)), max_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
}
__device__ __forceinline__ float vec_max(const uint4& r, __nv_bfloat16) {
    uint32_t a, b, m;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(r.x), "r"(r.y));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(r.z), "r"(r.w));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}
__device__ __forceinline__ float vec_max(const uint4& r, __half) {
    uint32_t a, b, m;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(a) : "r"(r.x), "r"(r.y));
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(b) : "r"(r.z), "r"(r.w));
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return max_nan(v.x, v.y);
}

// Keys: larger value <-> larger key, NaN below everything, -0 and +0 alike; with the token in the low word a
// larger key also means the lower of two tokens that tie.
__device__ __forceinline__ uint32_t value_key(float x) {
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
    return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key);
}
__device__ __forceinline__ unsigned long long full_key(float x, int token) {
    return ((unsigned long long)value_key(x) << 32) | (uint32_t)~token;
}
__device__ __forceinline__ int key_token(unsigned long long key) { return (int)~(uint32_t)key; }

// A row as vectors on 16-byte boundaries: vector j holds elements [j*N - shift, j*N - shift + N).  Only vectors
// that lie inside the row are read as such; the elements of the first and last one are read singly, so nothing
// outside the row is touched whatever its alignment.
template <typename T>
__device__ __forceinline__ int row_shift(const T* row) { return (int)(reinterpret_cast<uintptr_t>(row) % 16) / (int)sizeof(T); }
template <typename T>
__device__ __forceinline__ int row_vectors(int shift, int V) { return (shift + V + Row<T>::N - 1) / Row<T>::N; }

template <typename T>
__device__ __noinline__ uint4 load_edge(const T* row, int e0, int V) {
    constexpr int N = Row<T>::N, PER = 4 / sizeof(T);
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        w[q] = Row<T>::neg_inf();
#pragma unroll
        for (int h = 0; h < PER; ++h) {
            const int e = e0 + q * PER + h;
            if (e >= 0 && e < V) {
                const uint32_t b = Row<T>::bits(row[e]);
                if constexpr (PER == 1) w[q] = b;
                else w[q] = h ? ((w[q] & 0xffffu) | (b << 16)) : ((w[q] & 0xffff0000u) | b);
            }
        }
    }
    (void)N;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ uint4 load_vec(const T* row, int shift, int V, int j) {
    constexpr int N = Row<T>::N;
    const int e0 = j * N - shift;
    if (e0 >= 0 && e0 + N <= V) return __ldcg(reinterpret_cast<const uint4*>(row + e0));
    return load_edge<T>(row, e0, V);
}
// This thread's share of tile t0: vectors t0 + i*THREADS + tid below v1; -inf where there is none.
template <typename T>
__device__ __forceinline__ void load_tile(const T* row, int shift, int V, int t0, int v1, int tid, uint4 (&r)[NV]) {
    const uint32_t w = Row<T>::neg_inf();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t0 + i * THREADS + tid;
        r[i] = j < v1 ? load_vec<T>(row, shift, V, j) : make_uint4(w, w, w, w);
    }
}

// 2^((x - m) * log2(e)/T).  x - m is formed before scaling: rows masked with the type's lowest value neither overflow
// nor turn into NaN.
__device__ __forceinline__ f2 term2(f2 x, f2 neg_m, f2 hi, f2 lo) {
    const f2 d = sd::add2(x, neg_m);
    return sd::ex2_2(sd::fma2(d, lo, sd::mul2(d, hi)));
}
// Sum of a vector's terms; fp32 is enough for the eight terms of a vector and the eight vectors of a thread, the
// sums of threads are added in 64 bits.
template <int NP>
__device__ __forceinline__ f2 terms(const f2 (&x)[NP], f2 neg_m, f2 hi, f2 lo) {
    if constexpr (NP == 4)
        return sd::add2(sd::add2(term2(x[0], neg_m, hi, lo), term2(x[1], neg_m, hi, lo)),
                        sd::add2(term2(x[2], neg_m, hi, lo), term2(x[3], neg_m, hi, lo)));
    else
        return sd::add2(term2(x[0], neg_m, hi, lo), term2(x[1], neg_m, hi, lo));
}
__device__ __forceinline__ float fold2(f2 a) {
    float x, y;
    sd::unpack2(a, x, y);
    return x + y;
}
__device__ __forceinline__ float term(float x, float m, Scale c) {
    const float d = x - m;
    return sd::ex2(fmaf(d, c.lo, d * c.hi));
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ double rescale(float from, float to, double c) {   // factor that moves a sum to another reference
    return from == to ? 1.0 : exp2(((double)from - (double)to) * c);
}
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ double cl_ld_f64(const double* p, uint32_t rank) { return sd::cl_ld_f64(sd::cl_map(p, rank)); }
__device__ __forceinline__ float cl_ld_f32(const float* p, uint32_t rank) { return sd::cl_ld_f32(sd::cl_map(p, rank)); }
__device__ __forceinline__ int cl_ld_s32(const int* p, uint32_t rank) { return sd::cl_ld_s32(sd::cl_map(p, rank)); }
__device__ __forceinline__ unsigned long long cl_ld_u64(const unsigned long long* p, uint32_t rank) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(sd::cl_map(p, rank)) : "memory");
    return v;
}

// Largest of the non-NaN lane values.
__device__ __forceinline__ float warp_max(float v) { return sd::warp_max(v); }

// CTAs per row.  A row that does not fit one CTA's registers is spread over a cluster; with few rows more CTAs
// share a row, down to 2 KB each, as long as every one of them can have an SM of its own.
inline int cluster_size(long long rows, int nvec, int sm_count) {
    int C = 1;
    while (C < MAX_CLUSTER && C * TILE < nvec) C *= 2;
    while (C < MAX_CLUSTER && rows * C * 2 <= sm_count && nvec >= 256 * C) C *= 2;
    return C;
}

template <typename P>
inline cudaError_t launch(void (*kernel)(P), const P& p, long long rows, int C, size_t smem, cudaStream_t s) {
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * C));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeClusterDimension;
    a[0].val.clusterDim.x = C;
    a[0].val.clusterDim.y = 1;
    a[0].val.clusterDim.z = 1;
    cfg.attrs = a;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace rw
