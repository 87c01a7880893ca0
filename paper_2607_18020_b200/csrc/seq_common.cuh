// What the sequence operators (causal convolution, selective scan) and the orthogonalised update
// share: element types, wide loads with a scalar form, the gate functions, launch helpers.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "../../include/fpde.h"
#include "fpde_common.cuh"
#include "fpde_internal.h"

namespace fpde {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N elements of type T moved by one load or store of N * sizeof(T) bytes (at most 16).
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
    return *reinterpret_cast<const Pack<T, N>*>(p);
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const float (&v)[N]) {
    Pack<T, N> k;
#pragma unroll
    for (int i = 0; i < N; ++i) k.v[i] = from_f32<T>(v[i]);
    *reinterpret_cast<Pack<T, N>*>(p) = k;
}

__device__ __forceinline__ float exp2_f32(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float reciprocal_f32(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
constexpr float LOG2_E = 1.4426950408889634f;

// exp(-v) may overflow to infinity: the quotient is then 0, which is the limit.
__device__ __forceinline__ float sigmoid_f32(float v) { return reciprocal_f32(1.f + exp2_f32(-LOG2_E * v)); }
// log(1 + exp(v)) = max(v, 0) + log(1 + e), e = exp(-|v|) in (0, 1]; log(1 + e) / e is a polynomial of
// degree 8 fitted to the relative error on [0, 1] (3e-8), so small results keep their digits.  The product
// with log2(e) is carried in two parts: its rounding alone would cost |v| 2^-24 of the result.
__device__ __forceinline__ float softplus_f32(float v) {
    const float a = fmaxf(-fabsf(v), -150.f), hi = a * LOG2_E;      // exp(-150) is 0
    const float lo = fmaf(a, 1.925963033e-8f, fmaf(a, LOG2_E, -hi));
    float e = exp2_f32(hi);
    e = fmaf(e, lo * 0.6931471806f, e);
    float p = 0.00523267686f;
    p = fmaf(p, e, -0.029505169f);
    p = fmaf(p, e, 0.0782258362f);
    p = fmaf(p, e, -0.136632353f);
    p = fmaf(p, e, 0.191060022f);
    p = fmaf(p, e, -0.248429805f);
    p = fmaf(p, e, 0.333190978f);
    p = fmaf(p, e, -0.499994934f);
    p = fmaf(p, e, 0.99999994f);
    return fmaf(e, p, v < 0.f ? 0.f : v);      // a NaN stays
}

// Pairs of fp32 values in one 64-bit register: one instruction for two multiplications or fused adds.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
__device__ __forceinline__ float sum2(uint64_t p) {
    float lo, hi;
    unpair(p, lo, hi);
    return lo + hi;
}

__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// softplus_f32 and sigmoid_f32 of two values.
__device__ __forceinline__ uint64_t softplus_pair(uint64_t v) {
    float x, y, nx, ny;
    unpair(v, x, y);
    const uint64_t a = pair(fmaxf(-fabsf(x), -150.f), fmaxf(-fabsf(y), -150.f));
    const uint64_t neg = mul2(a, both(-LOG2_E));
    const uint64_t lo = fma2(a, both(1.925963033e-8f), fma2(a, both(LOG2_E), neg));
    unpair(neg, nx, ny);
    uint64_t e = pair(exp2_f32(-nx), exp2_f32(-ny));
    e = fma2(e, mul2(lo, both(0.6931471806f)), e);
    uint64_t p = both(0.00523267686f);
    p = fma2(p, e, both(-0.029505169f));
    p = fma2(p, e, both(0.0782258362f));
    p = fma2(p, e, both(-0.136632353f));
    p = fma2(p, e, both(0.191060022f));
    p = fma2(p, e, both(-0.248429805f));
    p = fma2(p, e, both(0.333190978f));
    p = fma2(p, e, both(-0.499994934f));
    p = fma2(p, e, both(0.99999994f));
    return fma2(e, p, pair(max_nan(x, 0.f), max_nan(y, 0.f)));
}
__device__ __forceinline__ uint64_t sigmoid_pair(uint64_t v) {
    float x, y;
    unpair(mul2(v, both(-LOG2_E)), x, y);
    unpair(add2(pair(exp2_f32(x), exp2_f32(y)), both(1.f)), x, y);
    return pair(reciprocal_f32(x), reciprocal_f32(y));
}

// One value, or a pair of them, in the same code.
template <int N> struct Lanes;
template <> struct Lanes<1> { using V = float; };
template <> struct Lanes<2> { using V = uint64_t; };
__device__ __forceinline__ float fma_v(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ uint64_t fma_v(uint64_t a, uint64_t b, uint64_t c) { return fma2(a, b, c); }
__device__ __forceinline__ float mul_v(float a, float b) { return a * b; }
__device__ __forceinline__ uint64_t mul_v(uint64_t a, uint64_t b) { return mul2(a, b); }
__device__ __forceinline__ float add_v(float a, float b) { return a + b; }
__device__ __forceinline__ uint64_t add_v(uint64_t a, uint64_t b) { return add2(a, b); }
__device__ __forceinline__ float sigmoid_v(float v) { return sigmoid_f32(v); }
__device__ __forceinline__ uint64_t sigmoid_v(uint64_t v) { return sigmoid_pair(v); }
template <typename V> __device__ __forceinline__ V all_v(float v);
template <> __device__ __forceinline__ float all_v<float>(float v) { return v; }
template <> __device__ __forceinline__ uint64_t all_v<uint64_t>(float v) { return both(v); }
__device__ __forceinline__ float of_array(const float (&v)[1]) { return v[0]; }
__device__ __forceinline__ uint64_t of_array(const float (&v)[2]) { return pair(v[0], v[1]); }
__device__ __forceinline__ void to_array(float (&v)[1], float a) { v[0] = a; }
__device__ __forceinline__ void to_array(float (&v)[2], uint64_t a) { unpair(a, v[0], v[1]); }

// The same for the one or two channels of a thread.
template <int N>
__device__ __forceinline__ void softplus_of(float (&v)[N]) {
    if constexpr (N == 2) unpair(softplus_pair(pair(v[0], v[1])), v[0], v[1]);
    else v[0] = softplus_f32(v[0]);
}
template <int N>
__device__ __forceinline__ void sigmoid_of(float (&out)[N], const float (&v)[N]) {
    if constexpr (N == 2) unpair(sigmoid_pair(pair(v[0], v[1])), out[0], out[1]);
    else out[0] = sigmoid_f32(v[0]);
}
template <typename T, int N>
__device__ __forceinline__ void widen(float (&out)[N], const Pack<T, N>& k) {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = to_f32<T>(k.v[i]);
}

template <typename T, int N>
__device__ __forceinline__ typename Lanes<N>::V widen_v(const Pack<T, N>& k) {
    float v[N];
    widen<T, N>(v, k);
    return of_array(v);
}
template <typename T, int N>
__device__ __forceinline__ void store_v(T* p, typename Lanes<N>::V a) {
    float v[N];
    to_array(v, a);
    store_pack<T, N>(p, v);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Sizes whose product is at most 2^48: strides can be zero, so an input of any extents can be handed in, and workspaces,
// grids and offsets of at most 2^12 times the product still fit 64 bits.
inline bool product_fits(int64_t a, int64_t b, int64_t c) {
    const auto at_least_1 = [](int64_t v) { return (unsigned __int128)(v > 0 ? v : 1); };
    const unsigned __int128 most = (unsigned __int128)1 << 48, ab = at_least_1(a) * at_least_1(b);
    return ab <= most && ab * at_least_1(c) <= most;
}
inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline size_t dtype_bytes(int dtype) { return dtype == FPDE_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == FPDE_F32 || dtype == FPDE_BF16 || dtype == FPDE_F16; }

// Allows a kernel its dynamic shared memory, once per device: `done` is the kernel's own mask of devices.
template <typename K>
inline cudaError_t allow_smem(K* kernel, size_t bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Can rows of this array be read in packs of n elements?
inline bool packs(const void* p, int64_t batch_stride, int64_t node_stride, size_t elem, int n) {
    return aligned(p, elem * n) && batch_stride % n == 0 && node_stride % n == 0;
}

}  // namespace fpde
