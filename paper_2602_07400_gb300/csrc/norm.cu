// Rows divided by their root mean square, with the addition of a residual before
// it and an output in 8 bits with scales behind it (include/bitlogic.h).
//
//   h = x + residual,  y_j = h_j w_j / sqrt(mean_j h_j^2 + eps)
//   scale = max |y| / 448 (e4m3) or / 127 (codes), of a row or of a group of its
//   columns;  out = e4m3(y / scale) or 128 + rint(y / scale)
//
// Bound by reading and writing every value once: a block (or, where rows are
// short, a warp) holds a row in its registers between its reductions, while the
// next row comes into shared memory.  Sums are fp32, in a fixed order.  32768 rows
// of 8192 bf16 columns with a residual to e4m3: 295 us, 1.88 GB at 94% of the
// measured HBM rate; a block per row without the row ahead took 698, and 362 before
// the arithmetic went by pairs.  16384 such rows with a scale per 128 columns: 169
// us, and 201 with the groups' scales found among the stores.  Rows that do not lie
// on 16 bytes go by element, a warp's lanes side by side (16384 x 8191: bf16 316 us,
// fp32 333; 688 and 878 with eight neighbouring columns to a thread).  One row of
// 8192 columns: 3.4 us, latency.
#include <cuda_fp8.h>

#include "norm_rows.cuh"

namespace bitlogic {
namespace {

struct NormOut {
    void* out;           // uint8 or e4m3 bytes
    long long ldo;
    float* scale;        // [T][groups], or NULL with a fixed scale
    int groups, group;   // columns of a group (a power of two, 16 to 256), 0: the row
    float fixed;         // > 0: the scale
    float most;          // 448 or 127
    bool codes;
};

// The largest |y| below which a row or group counts as zeros, so that neither
// the scale nor its inverse leaves fp32.
constexpr float kLeast = 7.8886091e-31f;   // 2^-100

__device__ __forceinline__ float inverse_scale(float big, float most) { return big < kLeast ? 0.f : most / big; }

// The larger of |a| and |b|; NaN where either is.
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

__device__ __forceinline__ uint2 to_bytes(const f32x2 (&y)[4], float inv, bool codes) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(mul2(y[i], twice(inv)), q[2 * i], q[2 * i + 1]);
    uint2 r;
    if (codes) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = __float2int_rn(fminf(fmaxf(q[i] != q[i] ? 0.f : q[i], -127.f), 127.f)) + 128;
            w[i >> 2] |= (uint32_t)c << (8 * (i & 3));
        }
        r = make_uint2(w[0], w[1]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(q[2 * i], q[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        r = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
    return r;
}

template <typename T, int kVec, bool kWarp, int kThreads, Way kWay>
__global__ void __launch_bounds__(kThreads, resident_by_registers(kThreads, kVec, kWarp))
norm_bytes_kernel(const T* x, long long ldx, const T* residual, long long ldr, T* total, long long ldt, Weight weight,
                  long long rows, int d, float eps, bool vec, bool vec_out, NormOut o) {
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ float sums[2][32], again_sums[32];
    __shared__ uint32_t tops[2][32];
    dependent_kernel_start();
    const Walk<kWarp> walk;
    auto xs = [&](int turn) { return Slots<T, kVec>(raw, turn); };
    auto rs = [&](int turn) { return Slots<T, kVec>(raw, 2 + turn); };
    auto ask = [&](long long row, int turn) {
        if (row < rows) {
            xs(turn).ask(x + row * ldx, walk, d);
            if (residual) rs(turn).ask(residual + row * ldr, walk, d);
        }
        cp_async_commit();
    };
    const float per = 1.0f / (float)d;
    if (kWay == kAhead) ask(walk.first, 0);
    int turn = 0;
    for (long long row = walk.first; row < rows; row += walk.step, turn ^= 1) {
        if (kWay == kAhead) {
            ask(row + walk.step, turn ^ 1);
            cp_async_wait<1>();
        }
        f32x2 h[kVec][4], square = twice(0.f);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.template start<kWay>(i);
            if (kWay == kAhead && c >= d) {
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = twice(0.f);
                continue;
            }
            f32x2 r[4];
            if (kWay == kAhead) xs(turn).get(i, h[i]);
            else read_pairs<kWay>(x + row * ldx + c, d - c, vec, h[i]);
            if (residual) {
                if (kWay == kAhead) rs(turn).get(i, r);
                else read_pairs<kWay>(residual + row * ldr + c, d - c, vec, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = add2(h[i][e], r[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) square = fma2(h[i][e], h[i][e], square);
        }
        const float sum = row_add<kWarp>(sum_of(square), sums[turn]);
        const float rstd = row_rstd(sum, per, eps, [&](float by) {
            f32x2 s = twice(0.f);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x2 v = mul2(h[i][e], twice(by));
                    s = fma2(v, v, s);
                }
            if (!kWarp) __syncthreads();
            return row_add<kWarp>(sum_of(s), again_sums);
        });
        if (total) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const int c = walk.template start<kWay>(i);
                if (kWay != kAhead) write_pairs<kWay>(total + row * ldt + c, d - c, vec, h[i]);
                else if (c < d) eight_of<T>(h[i]).store(total + row * ldt + c);
            }
        }
        float tops_of[kVec], top = 0.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.template start<kWay>(i);
            f32x2 w[4];
            if (weight.w) weight_pairs<T, kWay>(weight, c, d - c, w);
            tops_of[i] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                h[i][e] = mul2(h[i][e], twice(rstd));
                if (weight.w) h[i][e] = mul2(h[i][e], w[e]);
                float a, b;
                unpack2(h[i][e], a, b);
                if (c < d) tops_of[i] = larger(larger(a, b), tops_of[i]);
            }
            top = larger(top, tops_of[i]);
        }
        float inv[kVec];
        if (kWay == kSpread || o.fixed > 0.f || o.group == 0) {
            float one;
            if (o.fixed > 0.f) {
                one = 1.0f / o.fixed;
            } else {
                const float big = __uint_as_float(row_largest<kWarp>(__float_as_uint(top), tops[turn]));
                one = inverse_scale(big, o.most);
                if (walk.t == 0) o.scale[row] = big < kLeast ? 0.f : big / o.most;
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) inv[i] = one;
        } else {
            // a group is held by 2 to 32 neighbouring lanes
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const int c = walk.column(i);
                uint32_t t = __float_as_uint(tops_of[i]);
                for (int lanes = o.group >> 4; lanes > 0; lanes >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, lanes));
                const float big = __uint_as_float(t);
                inv[i] = inverse_scale(big, o.most);
                if (c < d && (c & (o.group - 1)) == 0) o.scale[row * o.groups + (c >> (31 - __clz(o.group)))] = big < kLeast ? 0.f : big / o.most;
            }
        }
        unsigned char* out = static_cast<unsigned char*>(o.out) + row * o.ldo;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.template start<kWay>(i);
            const uint2 b = to_bytes(h[i], inv[i], o.codes);
            if (kWay != kSpread && vec_out && c + 8 <= d) {
                *reinterpret_cast<uint2*>(out + c) = b;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (const int at = c + (kWay == kSpread ? 32 * e : e); at < d) out[at] = (unsigned char)((e < 4 ? b.x : b.y) >> (8 * (e & 3)));
            }
        }
    }
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

extern "C" int bitlogic_norm_bytes(const void* X, int32_t dtype, int64_t T, int32_t d, int64_t ldx, const void* residual,
                                   int64_t ldr, void* total, int64_t ldt, const void* weight, int32_t weight_dtype, float eps,
                                   int32_t form, void* out, int64_t ldo, float* scale, int32_t group, float fixed_scale,
                                   cudaStream_t stream) {
    if (dtype != BITLOGIC_F32 && dtype != BITLOGIC_BF16 && dtype != BITLOGIC_F16) return BITLOGIC_ERR_DTYPE;
    if (form != BITLOGIC_CODES && form != BITLOGIC_E4M3) return BITLOGIC_ERR_DTYPE;
    if (weight && weight_dtype != dtype && weight_dtype != BITLOGIC_F32) return BITLOGIC_ERR_DTYPE;
    if (T < 0 || T > 0x7fffffffLL || d < 1 || d > kMaxCols) return BITLOGIC_ERR_SHAPE;
    if (group != 0 && (group < 16 || group > 256 || (group & (group - 1)))) return BITLOGIC_ERR_SHAPE;
    if (!stride_ok(X, ldx, T, d) || !stride_ok(residual, ldr, T, d) || !stride_ok(total, ldt, T, d) || !stride_ok(out, ldo, T, d))
        return BITLOGIC_ERR_SHAPE;
    if (!(eps > 0.f) || !std::isfinite(eps) || !(fixed_scale >= 0.f) || !std::isfinite(fixed_scale) ||
        (fixed_scale > 0.f && !std::isfinite(1.0f / fixed_scale)))
        return BITLOGIC_ERR_HYPER;
    if (T == 0) return BITLOGIC_OK;
    if (!X || !out || (fixed_scale == 0.f && !scale)) return BITLOGIC_ERR_NULL;
    const int size = row_type_bytes(dtype);
    if (misaligned(X, size) || misaligned(residual, size) || misaligned(total, size) || misaligned(scale, 4) ||
        (weight && misaligned(weight, row_type_bytes(weight_dtype))))
        return BITLOGIC_ERR_ALIGN;
    const bool vec_in = rows_aligned16(X, ldx, T, size) && (!residual || rows_aligned16(residual, ldr, T, size)) &&
                        (!total || rows_aligned16(total, ldt, T, size));
    const bool vec_out = reinterpret_cast<uintptr_t>(out) % 8 == 0 && (T <= 1 || ldo % 8 == 0), vec_w = aligned16(weight);
    const NormOut o = {out, ldo, scale, group ? (d + group - 1) / group : 1, group, fixed_scale, form == BITLOGIC_CODES ? 127.f : 448.f,
                       form == BITLOGIC_CODES};
    const Weight wt = {weight, weight && weight_dtype == BITLOGIC_F32, vec_w};
    const RowShape s = row_shape(T, d);
    return with_row_type(dtype, [&](auto* type) {
        using V = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
        return with_shape(s, [&](auto vec, auto warp, auto most) {
            constexpr int kVec = decltype(vec)::value, kThreads = decltype(most)::value;
            constexpr bool kWarp = decltype(warp)::value;
            const int resident = resident_by_registers(s.threads, kVec, kWarp);
            const size_t slots = Slots<V, kVec>::bytes(residual ? 4 : 2, s.threads);
            const bool ahead = vec_in && d % 8 == 0 && slots <= kMostShared && row_blocks(T, s) > sm_count();
            // rows off 16 bytes, where no group of columns has to stay with its lanes
            const bool spread = !vec_in && (group == 0 || fixed_scale > 0.f);
            auto kern = ahead    ? norm_bytes_kernel<V, kVec, kWarp, kThreads, kAhead>
                        : spread ? norm_bytes_kernel<V, kVec, kWarp, kThreads, kSpread>
                                 : norm_bytes_kernel<V, kVec, kWarp, kThreads, kDirect>;
            const size_t smem = ahead ? slots : 0;
            if (allow_shared(kern, smem, kMostShared) != cudaSuccess) return (int)BITLOGIC_ERR_CUDA;
            return done(launch_dependent(kern, (unsigned)resident_blocks(s, resident, smem, T), (unsigned)s.threads, smem, stream,
                                         static_cast<const V*>(X), (long long)ldx, static_cast<const V*>(residual), (long long)ldr,
                                         static_cast<V*>(total), (long long)ldt, wt, (long long)T, (int)d, eps, vec_in, vec_out, o));
        });
    });
}
