// Eight consecutive values of a row, as the row operators on activations
// (dropout.cu, norm.cu) move them: 16 bytes of a 16-bit type, 32 of fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "packed.cuh"

namespace bitlogic {

// The loads do not go through the read-only path: an output may be the input.
// load_once and store_once mark what L2 need not keep.
template <typename T> struct Eight;

template <> struct Eight<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const uint4*>(p);
        b = *reinterpret_cast<const uint4*>(p + 4);
    }
    __device__ __forceinline__ void load_once(const float* p) {
        a = __ldcs(reinterpret_cast<const uint4*>(p));
        b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<uint4*>(p) = a;
        *reinterpret_cast<uint4*>(p + 4) = b;
    }
    __device__ __forceinline__ void store_once(float* p) const {
        __stcs(reinterpret_cast<uint4*>(p), a);
        __stcs(reinterpret_cast<uint4*>(p) + 1, b);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
        v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        a = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        b = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = a; }
    __device__ __forceinline__ void store_once(__nv_bfloat16* p) const { __stcs(reinterpret_cast<uint4*>(p), a); }
    static __device__ __forceinline__ void two(uint32_t u, float& x, float& y) {
        x = __uint_as_float(u << 16);
        y = __uint_as_float(u & 0xffff0000u);
    }
    static __device__ __forceinline__ uint32_t pair(float x, float y) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        two(a.x, v[0], v[1]);
        two(a.y, v[2], v[3]);
        two(a.z, v[4], v[5]);
        two(a.w, v[6], v[7]);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        a = make_uint4(pair(v[0], v[1]), pair(v[2], v[3]), pair(v[4], v[5]), pair(v[6], v[7]));
    }
};
template <> struct Eight<__half> {
    uint4 a;
    __device__ __forceinline__ void load(const __half* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_once(const __half* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void store(__half* p) const { *reinterpret_cast<uint4*>(p) = a; }
    __device__ __forceinline__ void store_once(__half* p) const { __stcs(reinterpret_cast<uint4*>(p), a); }
    static __device__ __forceinline__ void two(uint32_t u, float& x, float& y) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
        x = f.x;
        y = f.y;
    }
    static __device__ __forceinline__ uint32_t pair(float x, float y) {
        const __half2 p = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        two(a.x, v[0], v[1]);
        two(a.y, v[2], v[3]);
        two(a.z, v[4], v[5]);
        two(a.w, v[6], v[7]);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        a = make_uint4(pair(v[0], v[1]), pair(v[2], v[3]), pair(v[4], v[5]), pair(v[6], v[7]));
    }
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Eight by vector, or the first n of them by element (the others 0).
template <typename T>
__device__ __forceinline__ void load_eight(const T* p, int n, bool vec, float (&v)[8]) {
    if (vec && n >= 8) {
        Eight<T> e;
        e.load(p);
        e.get(v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store_eight(T* p, int n, bool vec, const float (&v)[8]) {
    if (vec && n >= 8) {
        Eight<T> e;
        e.set(v);
        e.store(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}

// Eight values as four pairs, for packed arithmetic.
template <typename T>
__device__ __forceinline__ void pairs_of(const Eight<T>& e, f32x2 (&z)[4]) {
    float v[8];
    e.get(v);
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = pack2(v[2 * i], v[2 * i + 1]);
}
template <typename T>
__device__ __forceinline__ Eight<T> eight_of(const f32x2 (&z)[4]) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(z[i], v[2 * i], v[2 * i + 1]);
    Eight<T> e;
    e.set(v);
    return e;
}
__device__ __forceinline__ f32x2 twice(float v) { return pack2(v, v); }

inline int row_type_bytes(int dtype) { return dtype == BITLOGIC_F32 ? 4 : 2; }

// f(pointer of the type) for the three types of activations.
template <typename F>
inline int with_row_type(int dtype, F f) {
    switch (dtype) {
        case BITLOGIC_F32: return f((const float*)nullptr);
        case BITLOGIC_BF16: return f((const __nv_bfloat16*)nullptr);
        case BITLOGIC_F16: return f((const __half*)nullptr);
        default: return BITLOGIC_ERR_DTYPE;
    }
}

// Whether rows of `bytes`-byte values at p, `ld` values apart, all start on 16
// bytes (a single row: its start alone).
inline bool rows_aligned16(const void* p, int64_t ld, int64_t rows, int bytes) {
    return aligned16(p) && (rows <= 1 || (ld * bytes) % 16 == 0);
}

}  // namespace bitlogic
