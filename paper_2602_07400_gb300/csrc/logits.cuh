// Shared by the kernels over rows of logits (top.cu, distill.cu, sample.cu):
// element types, the order of logits, reductions over a block, and the
// selection of a row's largest by count or by mass.
#pragma once

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>
#include <cmath>

#include "common.cuh"

namespace bitlogic {

constexpr int kMaxClasses = 1 << 20;   // classes of a row
constexpr int kMaxTop = 256;           // entries of a record

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
#define BITLOGIC_NEG_INF (-HUGE_VALF)

__device__ __forceinline__ float logit_value(float x) { return x; }
__device__ __forceinline__ float logit_value(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float logit_value(__half x) { return __half2float(x); }
// counts: the lowest int stands for a masked class
__device__ __forceinline__ float logit_value(int x) { return x == INT_MIN ? BITLOGIC_NEG_INF : (float)x; }

template <typename T> __device__ __forceinline__ T logit_of(float x);
template <> __device__ __forceinline__ float logit_of<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 logit_of<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half logit_of<__half>(float x) { return __float2half_rn(x); }

// 2^y by the exponential unit (y <= 0 here; 0 below -126).  exp2f returns the
// same bits on the range that counts, [-64, 0], checked for every float there.
__device__ __forceinline__ float exp2_unit(float y) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    return r;
}

// The order of logits as unsigned numbers: larger logits have larger keys,
// -0 and 0 the same.  NaN has key 0; -inf and NaN do not rank (ranks()).
__device__ __forceinline__ uint32_t logit_key(float z) {
    const uint32_t u = __float_as_uint(z + 0.0f);
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return (z != z) ? 0u : k;
}
constexpr uint32_t kKeyNegInf = 0x007fffffu;
__device__ __forceinline__ bool ranks(uint32_t key) { return key > kKeyNegInf; }

// A draw's weight: whole multiples of 2^-40 of the largest logit's weight, so
// that sums of weights are exact in any order (2^20 classes: below 2^61).
__device__ __forceinline__ unsigned long long draw_weight(float e) {
    return (unsigned long long)__float2ll_rn(e * 1099511627776.0f);
}

// floor(total * x) with x in [0, 1] held to 24 bits
__device__ __forceinline__ unsigned long long share_of(unsigned long long total, float x) {
    const unsigned long long x24 = (unsigned long long)(x * 16777216.0f);
    return (((total >> 32) * x24) << 8) + (((total & 0xffffffffull) * x24) >> 24);
}

template <typename T> __device__ __forceinline__ T shuffle_xor(T v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }

template <typename T> __device__ __forceinline__ T warp_add(T v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += shuffle_xor(v, o);
    return v;
}
__device__ __forceinline__ float warp_largest(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, shuffle_xor(v, o));
    return v;
}

// Reductions over a block of `warps` warps; every thread gets the result.
// `buf` holds one value per warp and may be used again after the call.
template <typename T> __device__ __forceinline__ T block_add(T v, T* buf, int warps) {
    v = warp_add(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    T t = 0;
    for (int i = 0; i < warps; ++i) t += buf[i];
    return t;
}
__device__ __forceinline__ float block_largest(float v, float* buf, int warps) {
    v = warp_largest(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = buf[0];
    for (int i = 1; i < warps; ++i) t = fmaxf(t, buf[i]);
    return t;
}

// Cut of an order: the classes whose key is above `key`, and the first `ties`
// (by class) of those whose key equals it.
struct Cut {
    uint32_t key;
    unsigned long long ties;
};

struct SelectScratch {
    unsigned long long bins[256];
    unsigned long long above;
    uint32_t prefix;
};

// Over keys key_at(v) with amounts amount_at(v, key), v < V: the largest key t
// whose classes of key >= t amount to at least `want` (0 < want <= all), and
// the amount of the keys above t, by 8 bits of the key at a time.  Called by
// the whole block.
template <typename KeyAt, typename AmountAt>
__device__ uint32_t select_key(KeyAt key_at, AmountAt amount_at, int V, unsigned long long want, SelectScratch* sc,
                               unsigned long long* above_out) {
    uint32_t prefix = 0;
    unsigned long long above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += blockDim.x) sc->bins[i] = 0;
        __syncthreads();
        for (int v = threadIdx.x; v < V; v += blockDim.x) {
            const uint32_t k = key_at(v);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) {
                const unsigned long long a = amount_at(v, k);
                if (a) atomicAdd(&sc->bins[(k >> shift) & 255u], a);
            }
        }
        __syncthreads();
        if (threadIdx.x < 32) {   // lane l: bins 255 - 8 l down to 248 - 8 l
            const int lane = threadIdx.x;
            unsigned long long own = 0;
            for (int i = 0; i < 8; ++i) own += sc->bins[255 - 8 * lane - i];
            unsigned long long upto = own;
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long t = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += t;
            }
            const unsigned m = __ballot_sync(0xffffffffu, above + upto >= want);
            const int first = m ? __ffs(m) - 1 : 31;
            if (lane == first) {
                unsigned long long a = above + upto - own;
                int d = 255 - 8 * lane;
                const int last = d - 7;
                while (d > last && a + sc->bins[d] < want) a += sc->bins[d--];
                sc->above = a;
                sc->prefix = prefix | ((uint32_t)d << shift);
            }
        }
        __syncthreads();
        prefix = sc->prefix;
        above = sc->above;
    }
    *above_out = above;
    return prefix;
}

// What a row kernel needs of a dtype known at run time.
template <typename F>
inline int with_logit_type(int dtype, bool whole, F f) {
    switch (dtype) {
        case BITLOGIC_F32: return f((const float*)nullptr);
        case BITLOGIC_BF16: return f((const __nv_bfloat16*)nullptr);
        case BITLOGIC_F16: return f((const __half*)nullptr);
        case BITLOGIC_I32: if (whole) return f((const int*)nullptr); return BITLOGIC_ERR_DTYPE;
        default: return BITLOGIC_ERR_DTYPE;
    }
}

inline int logit_bytes(int dtype) { return dtype == BITLOGIC_F32 || dtype == BITLOGIC_I32 ? 4 : 2; }

// Whether a temperature is positive and finite, and so is its inverse times
// log2(e), the slope of a row's powers.
inline bool temperature_ok(float temperature) { return temperature > 0.f && isfinite(temperature) && isfinite(kLog2E / temperature); }

// Checks of a matrix of logits that the three operators share.
inline int check_logits(const void* X, int dtype, bool whole, int64_t T, int32_t V, int64_t ld) {
    if (dtype < BITLOGIC_F32 || dtype > BITLOGIC_I32 || (dtype == BITLOGIC_I32 && !whole)) return BITLOGIC_ERR_DTYPE;
    if (T < 0 || T > 0x7fffffffLL / 8 || V < 1 || V > kMaxClasses || ld < V || ld > (1LL << 40)) return BITLOGIC_ERR_SHAPE;
    if (T > 0 && !X) return BITLOGIC_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(X) % logit_bytes(dtype)) return BITLOGIC_ERR_ALIGN;
    return BITLOGIC_OK;
}

}  // namespace bitlogic
