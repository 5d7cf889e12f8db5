// Rows divided by their root mean square, with the addition of a residual before
// it and an output in 8 bits with scales behind it, and the gradient.
//
//   h = x + residual,  y_j = h_j w_j / sqrt(mean_j h_j^2 + eps)
//   scale = max |y| / 448 (e4m3) or / 127 (codes), of a row or of a group of its
//   columns;  out = e4m3(y / scale) or 128 + rint(y / scale)
//
// The gradient passes the rounding to 8 bits as if it were not there:
//   g = dy w,  xh = h rstd,  dh = rstd (g - xh mean(g xh)),  dw = sum_rows dy xh
//
// Both are bound by reading and writing every value once: a block (or, where
// rows are short, a warp) per row holds the row in its registers between its
// reductions.  Sums are fp32, in a fixed order.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include <cuda_fp8.h>

#include "rows8.cuh"

namespace bitlogic {
namespace {

constexpr int kMaxCols = 32768;   // 1024 threads of four vectors of eight
constexpr int kNormPartials = 1024;

__device__ __forceinline__ float norm_warp_add(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The sum over a row's threads (blockDim.x of them); every thread gets it.
// `buf`: 32 floats, free again after the next barrier of the block.
__device__ __forceinline__ float row_add(float v, float* buf) {
    v = norm_warp_add(v);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return norm_warp_add(lane < warps ? buf[lane] : 0.f);
}
// The largest of |v| by its bits, which NaN and infinity lead.
__device__ __forceinline__ uint32_t row_largest(uint32_t v, uint32_t* buf) {
    v = __reduce_max_sync(0xffffffffu, v);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return __reduce_max_sync(0xffffffffu, lane < warps ? buf[lane] : 0u);
}

__device__ __forceinline__ float reciprocal_root(float mean_square) { return 1.0f / sqrtf(mean_square); }

// 1 / sqrt(mean h^2 + eps) from the sum of squares; where that passed fp32, from
// the squares of 2^-96 h, which `again` sums.
template <typename Again>
__device__ __forceinline__ float row_rstd(float sum, int d, float eps, Again again) {
    if (!isinf(sum)) return reciprocal_root(sum / (float)d + eps);
    constexpr float kBy = 1.262177448e-29f;   // 2^-96
    return reciprocal_root(again(kBy) / (float)d) * kBy;
}

struct NormOut {
    void* out;           // uint8 or e4m3 bytes
    long long ldo;
    float* scale;        // [T][groups], or NULL with a fixed scale
    int groups, group;   // columns of a group (a power of two, 16 to 256), 0: the row
    float fixed;         // > 0: the scale
    float most;          // 448 or 127
};

// The largest |y| below which a row or group counts as zeros, so that neither
// the scale nor its inverse leaves fp32.
constexpr float kLeast = 7.8886091e-31f;   // 2^-100

__device__ __forceinline__ float inverse_scale(float big, float most) { return big < kLeast ? 0.f : most / big; }

template <bool kCodes>
__device__ __forceinline__ uint2 to_bytes(const float (&y)[8], float inv, float most) {
    uint2 r;
    if (kCodes) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = y[i] * inv;
            const int c = __float2int_rn(fminf(fmaxf(q != q ? 0.f : q, -127.f), 127.f)) + 128;
            w[i >> 2] |= (uint32_t)c << (8 * (i & 3));
        }
        r = make_uint2(w[0], w[1]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[2 * i] * inv, y[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        r = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
    return r;
}

// A row per block of 32 to 1024 threads: thread t holds the vectors of eight
// columns t, t + threads, ... (kVec of them).
template <typename T, typename W, int kVec, bool kCodes>
__global__ void __launch_bounds__(1024)
norm_bytes_kernel(const T* x, long long ldx, const T* residual, long long ldr, T* total, long long ldt, const W* __restrict__ weight,
                  int d, float eps, bool vec_in, bool vec_w, bool vec_out, NormOut o) {
    __shared__ float sums[32], again_sums[32];
    __shared__ uint32_t tops[32];
    dependent_kernel_start();
    const long long row = blockIdx.x;
    const int tid = threadIdx.x, threads = blockDim.x;
    const T* xr = x + row * ldx;
    float h[kVec][8];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = 8 * (i * threads + tid);
        load_eight(xr + c, d - c, vec_in, h[i]);
    }
    if (residual) {
        const T* rr = residual + row * ldr;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = 8 * (i * threads + tid);
            float r[8];
            load_eight(rr + c, d - c, vec_in, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] += r[e];
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(h[i][e], h[i][e], sum);
    sum = row_add(sum, sums);
    const float rstd = row_rstd(sum, d, eps, [&](float by) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(h[i][e] * by, h[i][e] * by, s);
        return row_add(s, again_sums);
    });
    if (total) {
        T* tr = total + row * ldt;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = 8 * (i * threads + tid);
            store_eight(tr + c, d - c, vec_in, h[i]);
        }
    }
    uint32_t top = 0u, group_top[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = 8 * (i * threads + tid);
        float w[8];
        if (weight) load_eight(weight + c, d - c, vec_w, w);
        group_top[i] = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[i][e] = h[i][e] * rstd;
            if (weight && c + e < d) h[i][e] *= w[e];
            group_top[i] = max(group_top[i], __float_as_uint(h[i][e]) & 0x7fffffffu);
        }
        top = max(top, group_top[i]);
    }
    float inv = 0.f;
    if (o.fixed > 0.f) {
        inv = 1.0f / o.fixed;
    } else if (o.group == 0) {
        const float big = __uint_as_float(row_largest(top, tops));
        inv = inverse_scale(big, o.most);
        if (tid == 0) o.scale[row] = big < kLeast ? 0.f : big / o.most;
    }
    unsigned char* out = static_cast<unsigned char*>(o.out) + row * o.ldo;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = 8 * (i * threads + tid);
        if (o.fixed <= 0.f && o.group != 0) {
            // a group is held by 2 to 32 neighbouring lanes
            uint32_t t = group_top[i];
            for (int lanes = o.group >> 4; lanes > 0; lanes >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, lanes));
            const float big = __uint_as_float(t);
            inv = inverse_scale(big, o.most);
            if (c < d && c % o.group == 0) o.scale[row * o.groups + c / o.group] = big < kLeast ? 0.f : big / o.most;
        }
        const uint2 b = to_bytes<kCodes>(h[i], inv, o.most);
        if (vec_out && c + 8 <= d) {
            *reinterpret_cast<uint2*>(out + c) = b;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < d) out[c + e] = (unsigned char)((e < 4 ? b.x : b.y) >> (8 * (e & 3)));
        }
    }
}

// The gradient: blocks that walk over the rows, their columns' part of dw in
// registers until the end, then in `partial` [blocks][d].
template <typename T, typename W, int kVec>
__global__ void __launch_bounds__(1024)
norm_backward_kernel(const T* dy, long long ldy, const T* h, long long ldh, const W* __restrict__ weight, const T* dres, long long lds,
                     T* dx, long long ldx, float* __restrict__ partial, long long rows, int d, float eps, bool vec, bool vec_w) {
    __shared__ float sums[2][2][32], again_sums[32];
    dependent_kernel_start();
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    float w[kVec][8], dw[kVec][8];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = 8 * (i * threads + tid);
        if (weight) load_eight(weight + c, d - c, vec_w, w[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!weight) w[i][e] = 1.f;
            dw[i][e] = 0.f;
        }
    }
    int turn = 0;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        float a[kVec][8], g[kVec][8];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = 8 * (i * threads + tid);
            load_eight(h + row * ldh + c, d - c, vec, a[i]);
            load_eight(dy + row * ldy + c, d - c, vec, g[i]);
        }
        float square = 0.f, along = 0.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                square = fmaf(a[i][e], a[i][e], square);
                along = fmaf(a[i][e] * w[i][e], g[i][e], along);
            }
        // two sums with one barrier; the buffers of a row are free when the next
        // row's barrier is passed
        square = norm_warp_add(square);
        along = norm_warp_add(along);
        if (warps > 1) {
            if (lane == 0) {
                sums[turn][0][warp] = square;
                sums[turn][1][warp] = along;
            }
            __syncthreads();
            square = norm_warp_add(lane < warps ? sums[turn][0][lane] : 0.f);
            along = norm_warp_add(lane < warps ? sums[turn][1][lane] : 0.f);
        }
        const float rstd = row_rstd(square, d, eps, [&](float by) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < kVec; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fmaf(a[i][e] * by, a[i][e] * by, s);
            __syncthreads();
            return row_add(s, again_sums);
        });
        // xh mean(g xh) = h (rstd^2 mean(g h))
        const float back = along * rstd / (float)d * rstd;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = 8 * (i * threads + tid);
            float v[8];
            if (dres) load_eight(dres + row * lds + c, d - c, vec, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[i][e] = fmaf(g[i][e], a[i][e] * rstd, dw[i][e]);
                const float q = (g[i][e] * w[i][e] - a[i][e] * back) * rstd;
                v[e] = dres ? q + v[e] : q;
            }
            store_eight(dx + row * ldx + c, d - c, vec, v);
        }
    }
    if (partial) {
        float* p = partial + (long long)blockIdx.x * d;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = 8 * (i * threads + tid);
            store_eight(p + c, d - c, d % 8 == 0, dw[i]);
        }
    }
}

// dw[c] = sum of the partials, 32 columns by 8 strided runs of rows per block,
// the runs joined in order.
__global__ void __launch_bounds__(256)
norm_weight_kernel(const float* __restrict__ partial, int blocks, int d, float* __restrict__ dweight) {
    __shared__ float part[8][33];
    dependent_kernel_start();
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < d)
        for (int b = run; b < blocks; b += 8) s += partial[(long long)b * d + c];
    part[run][lane] = s;
    __syncthreads();
    if (run == 0 && c < d) {
        for (int r = 1; r < 8; ++r) s += part[r][lane];
        dweight[c] = s;
    }
}

// dw of no rows
__global__ void norm_zero_kernel(float* __restrict__ dweight, int d) {
    dependent_kernel_start();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < d) dweight[c] = 0.f;
}

// Threads of a row: a vector each, up to 1024 threads; then more vectors.
struct RowShape {
    int threads, vec;
};
inline RowShape row_shape(int d) {
    const int vectors = (d + 7) / 8;
    RowShape s = {32 * ((vectors + 31) / 32), 1};
    while (s.threads > 1024) {
        s.vec *= 2;
        s.threads = 32 * ((vectors + 32 * s.vec - 1) / (32 * s.vec));
    }
    return s;
}

template <typename F>
inline int with_vec(int vec, F f) {
    if (vec == 1) return f(std::integral_constant<int, 1>());
    if (vec == 2) return f(std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 4>());
}

inline int done(cudaError_t e) { return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA; }

inline bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes != 0; }

// Row strides of the [T][d] matrices of a call.
inline bool stride_ok(const void* p, int64_t ld, int64_t T, int d) {
    return !p || T <= 1 || (ld >= d && ld <= (1LL << 40) / T);
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
    const NormOut o = {out, ldo, scale, group ? (d + group - 1) / group : 1, group, fixed_scale, form == BITLOGIC_CODES ? 127.f : 448.f};
    const RowShape s = row_shape(d);
    return with_row_type(dtype, [&](auto* type) {
        using V = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
        auto go = [&](auto* wtype) {
            using W = std::remove_const_t<std::remove_pointer_t<decltype(wtype)>>;
            return with_vec(s.vec, [&](auto vec) {
                auto kern = form == BITLOGIC_CODES ? norm_bytes_kernel<V, W, decltype(vec)::value, true>
                                                   : norm_bytes_kernel<V, W, decltype(vec)::value, false>;
                return done(launch_dependent(kern, (unsigned)T, (unsigned)s.threads, 0, stream, static_cast<const V*>(X), (long long)ldx,
                                             static_cast<const V*>(residual), (long long)ldr, static_cast<V*>(total), (long long)ldt,
                                             static_cast<const W*>(weight), (int)d, eps, vec_in, vec_w, vec_out, o));
            });
        };
        return weight && weight_dtype == BITLOGIC_F32 ? go((const float*)nullptr) : go((const V*)nullptr);
    });
}

extern "C" size_t bitlogic_norm_backward_workspace(int64_t T, int32_t d) {
    if (T < 1 || d < 1 || d > kMaxCols) return 0;
    return (size_t)(T < kNormPartials ? T : kNormPartials) * (size_t)d * 4;
}

extern "C" int bitlogic_norm_backward(const void* dY, int32_t dtype, int64_t T, int32_t d, int64_t ldy, const void* H, int64_t ldh,
                                      const void* weight, int32_t weight_dtype, const void* residual_grad, int64_t ldr, float eps,
                                      void* dX, int64_t ldx, float* dweight, void* workspace, size_t workspace_bytes,
                                      cudaStream_t stream) {
    if (dtype != BITLOGIC_F32 && dtype != BITLOGIC_BF16 && dtype != BITLOGIC_F16) return BITLOGIC_ERR_DTYPE;
    if (weight && weight_dtype != dtype && weight_dtype != BITLOGIC_F32) return BITLOGIC_ERR_DTYPE;
    if (T < 0 || T > 0x7fffffffLL || d < 1 || d > kMaxCols) return BITLOGIC_ERR_SHAPE;
    if (!stride_ok(dY, ldy, T, d) || !stride_ok(H, ldh, T, d) || !stride_ok(residual_grad, ldr, T, d) || !stride_ok(dX, ldx, T, d))
        return BITLOGIC_ERR_SHAPE;
    if (!(eps > 0.f) || !std::isfinite(eps)) return BITLOGIC_ERR_HYPER;
    if (misaligned(dweight, 4)) return BITLOGIC_ERR_ALIGN;
    if (T == 0) {
        if (!dweight) return BITLOGIC_OK;
        return done(launch_dependent(norm_zero_kernel, (unsigned)((d + 255) / 256), 256, 0, stream, dweight, (int)d));
    }
    if (!dY || !H || !dX || (dweight && !workspace)) return BITLOGIC_ERR_NULL;
    const int size = row_type_bytes(dtype);
    if (misaligned(dY, size) || misaligned(H, size) || misaligned(dX, size) || misaligned(residual_grad, size) ||
        (weight && misaligned(weight, row_type_bytes(weight_dtype))) || (dweight && misaligned(workspace, 16)))
        return BITLOGIC_ERR_ALIGN;
    if (dweight && workspace_bytes < bitlogic_norm_backward_workspace(T, d)) return BITLOGIC_ERR_WORKSPACE;
    const bool vec = rows_aligned16(dY, ldy, T, size) && rows_aligned16(H, ldh, T, size) && rows_aligned16(dX, ldx, T, size) &&
                     (!residual_grad || rows_aligned16(residual_grad, ldr, T, size));
    const bool vec_w = aligned16(weight);
    const RowShape s = row_shape(d);
    const long long most = std::min<long long>(kNormPartials, (long long)sm_count() * std::max(1, 2048 / s.threads));
    const unsigned blocks = (unsigned)std::min<long long>(T, most);
    float* partial = dweight ? static_cast<float*>(workspace) : nullptr;
    const int st = with_row_type(dtype, [&](auto* type) {
        using V = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
        auto go = [&](auto* wtype) {
            using W = std::remove_const_t<std::remove_pointer_t<decltype(wtype)>>;
            return with_vec(s.vec, [&](auto n) {
                return done(launch_dependent(norm_backward_kernel<V, W, decltype(n)::value>, blocks, (unsigned)s.threads, 0, stream,
                                             static_cast<const V*>(dY), (long long)ldy, static_cast<const V*>(H), (long long)ldh,
                                             static_cast<const W*>(weight), static_cast<const V*>(residual_grad), (long long)ldr,
                                             static_cast<V*>(dX), (long long)ldx, partial, (long long)T, (int)d, eps, vec, vec_w));
            });
        };
        return weight && weight_dtype == BITLOGIC_F32 ? go((const float*)nullptr) : go((const V*)nullptr);
    });
    if (st != BITLOGIC_OK || !dweight) return st;
    return done(launch_dependent(norm_weight_kernel, (unsigned)((d + 31) / 32), 256, 0, stream, (const float*)partial, (int)blocks,
                                 (int)d, dweight));
}
