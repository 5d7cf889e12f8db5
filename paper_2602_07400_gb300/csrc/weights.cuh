// Sums of whole-number weights, shared by the kernels that draw a class
// (sample.cu, verify.cu).
#pragma once

#include "packed.cuh"

namespace bitlogic {

// Sums of weights w = rint(2^40 e), 0 <= e <= 1, of at most 1024 of them, in
// fp32 and 32-bit integer operations: 16 + e rounds e to a multiple of 2^-19,
// the remainder is exact, and 1.5 2^23 + 2^40 remainder rounds it to a whole
// number as rint does; so w = 2^21 high + low with the offsets of the two
// floats' bits taken off, in arithmetic modulo 2^32.
struct WeightSum {
    uint32_t high = 0, low = 0;
    __device__ __forceinline__ void add(f32x2 e) {
        const f32x2 c16 = pack2(16.0f, 16.0f), scale = pack2(1099511627776.0f, 1099511627776.0f),
                    whole = pack2(12582912.0f, 12582912.0f);
        const f32x2 t = add2(e, c16), r = sub2(e, sub2(t, c16)), u = fma2(r, scale, whole);
        float a, b;
        unpack2(t, a, b);
        high += __float_as_uint(a) + __float_as_uint(b) - 2u * 0x41800000u;
        unpack2(u, a, b);
        low += __float_as_uint(a) + __float_as_uint(b) - 2u * 0x4b400000u;
    }
    __device__ __forceinline__ unsigned long long total() const {
        return ((unsigned long long)high << 21) + (unsigned long long)(long long)(int)low;
    }
    // the sum over a warp (of at most 1024 weights), in every lane
    __device__ __forceinline__ unsigned long long warp_total() const {
        WeightSum s;
        s.high = __reduce_add_sync(0xffffffffu, high);
        s.low = __reduce_add_sync(0xffffffffu, low);
        return s.total();
    }
};

}  // namespace bitlogic
