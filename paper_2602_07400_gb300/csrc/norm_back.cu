// The gradient of the norm of rows (norm.cu), the rounding to 8 bits passed as if
// it were not there:
//
//   g = dy w,  xh = h rstd,  dx = rstd (g - xh mean(g xh)) + dres,  dw = sum_rows dy xh
//
// Bound by reading and writing every value once: persistent blocks (or, where rows
// are short, warps) read a row's values twice from shared memory, into which the
// next row comes meanwhile, and keep their columns' part of dw in registers until
// the end.  Sums are fp32, in a fixed order; where one passes fp32 both are formed
// again of numbers brought nearer (sums_again).  16384 rows of 8192 bf16 columns with
// a residual's gradient: 160 us, 1.07 GB at 99% of the measured HBM rate; 286 with a
// block's rows read as they are wanted, 217 with rows ahead, 195 with two sums reduced
// at once.  Rows off 16 bytes go by element, a warp's lanes side by side: 509 x 1001
// fp32 6.3 us, latency of two kernels, and 16384 x 8191 bf16 340 (10 and 625 with
// eight neighbouring columns to a thread).
#include <cfloat>

#include "norm_rows.cuh"

namespace bitlogic {
namespace {

constexpr int kNormPartials = 1024;   // rows of partial sums of dw, at most
constexpr float k2m96 = 0x1p-96f, k2m72 = 0x1p-72f;

// The two sums of a row again where fp32 does not hold them, of numbers brought
// nearer: the squares of 2^-96 h, and h and g by 2^-72 each, which leaves the largest
// term of a sum past 2^128 above 2^-31.  Rare, so not unrolled.
template <typename T>
__device__ __forceinline__ float2 sums_again(const T* h, const T* dy, Weight weight, int t, int threads, int d) {
    float squares = 0.f, along = 0.f;
#pragma unroll 1
    for (int c = t; c < d; c += threads) {
        const float a = to_f32(h[c]);
        float g = to_f32(dy[c]);
        if (weight.w) g *= weight.wide ? static_cast<const float*>(weight.w)[c] : to_f32(static_cast<const T*>(weight.w)[c]);
        squares = fmaf(a * k2m96, a * k2m96, squares);
        along = fmaf(a * k2m72, g * k2m72, along);
    }
    return make_float2(squares, along);
}

// dw goes to `partial` [blocks][d], a block's warps joined in order where each has
// rows.
template <typename T, int kVec, bool kWarp, int kThreads, Way kWay>
__global__ void __launch_bounds__(kThreads, resident_by_registers(kThreads, kVec, kWarp))
norm_backward_kernel(const T* dy, long long ldy, const T* h, long long ldh, Weight weight, const T* dres, long long lds,
                     T* dx, long long ldx, float* __restrict__ partial, long long rows, int d, float eps, bool vec) {
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ float sums[2][64], again_sums[64];
    dependent_kernel_start();
    const Walk<kWarp> walk;
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    auto as = [&](int turn) { return Slots<T, kVec>(raw, turn); };
    auto gs = [&](int turn) { return Slots<T, kVec>(raw, 2 + turn); };
    auto ask = [&](long long row, int turn) {
        if (row < rows) {
            as(turn).ask(h + row * ldh, walk, d);
            gs(turn).ask(dy + row * ldy, walk, d);
        }
        cp_async_commit();
    };
    const float per = 1.0f / (float)d;
    f32x2 dw[kVec][4];
#pragma unroll
    for (int i = 0; i < kVec; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[i][e] = twice(0.f);
    const WeightSlots<T, kVec> ws = {raw + Slots<T, kVec>::place(4), weight.wide};
    if (kWay == kAhead && weight.w) ws.fill(weight, walk, d);
    if (kWay == kAhead) ask(walk.first, 0);
    int turn = 0;
    for (long long row = walk.first; row < rows; row += walk.step, turn ^= 1) {
        Eight<T> extra[kVec];   // of dres, wanted at the row's end
        if (kWay == kAhead) {
            ask(row + walk.step, turn ^ 1);
            if (dres) {
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (walk.column(i) < d) extra[i].load(dres + row * lds + walk.column(i));
            }
            cp_async_wait<1>();
        }
        // of vector i: h and dy
        auto values = [&](int i, int c, f32x2 (&a)[4], f32x2 (&g)[4]) {
            if (kWay == kAhead) {
                as(turn).get(i, a);
                gs(turn).get(i, g);
            } else {
                read_pairs<kWay>(h + row * ldh + c, d - c, vec, a);
                read_pairs<kWay>(dy + row * ldy + c, d - c, vec, g);
            }
        };
        f32x2 squares = twice(0.f), alongs = twice(0.f);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.template start<kWay>(i);
            if (kWay == kAhead && c >= d) continue;
            f32x2 a[4], g[4], w[4];
            values(i, c, a, g);
            if (weight.w) {
                if (kWay == kAhead) ws.get(i, w);
                else weight_pairs<T, kWay>(weight, c, d - c, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = mul2(g[e], w[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                squares = fma2(a[e], a[e], squares);
                alongs = fma2(a[e], g[e], alongs);
            }
        }
        // two sums with one barrier; the buffers of a row are free when the next
        // row's barrier is passed
        float square = sum_of(squares), along = sum_of(alongs);
        row_add_two<kWarp>(square, along, sums[turn]);
        float rstd = rsqrtf(fmaf(square, per, eps)), mean = along * rstd * per;   // mean(g xh)
        const bool wide = isinf(square), far = !(fabsf(along) <= FLT_MAX);
        if (wide || far) {
            const float2 s = sums_again(h + row * ldh, dy + row * ldy, weight, walk.t, walk.threads, d);
            float near_square = s.x, near_along = s.y;
            if (!kWarp) __syncthreads();
            row_add_two<kWarp>(near_square, near_along, again_sums);
            const float root = wide ? rsqrtf(near_square * per) : rstd;   // of 2^-96 h where `wide`
            if (wide) rstd = root * k2m96;
            mean = (far ? near_along : along) * per * root;
            if (far) mean = wide ? mean * 0x1p48f : mean * 0x1p72f * 0x1p72f;
            else mean *= k2m96;
        }
        const f32x2 along_xh = twice(-mean), root = twice(rstd);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.template start<kWay>(i);
            if (kWay == kAhead && c >= d) continue;
            f32x2 a[4], g[4], w[4], v[4];
            values(i, c, a, g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = mul2(a[e], root);   // xh
                dw[i][e] = fma2(g[e], a[e], dw[i][e]);
            }
            if (weight.w) {
                if (kWay == kAhead) ws.get(i, w);
                else weight_pairs<T, kWay>(weight, c, d - c, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = mul2(g[e], w[e]);
            }
            if (dres) {
                if (kWay == kAhead) pairs_of(extra[i], v);
                else read_pairs<kWay>(dres + row * lds + c, d - c, vec, v);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 q = fma2(a[e], along_xh, g[e]);
                v[e] = dres ? fma2(q, root, v[e]) : mul2(q, root);
            }
            if (kWay == kAhead) eight_of<T>(v).store(dx + row * ldx + c);
            else write_pairs<kWay>(dx + row * ldx + c, d - c, vec, v);
        }
    }
    if (!partial) return;
    float* p = partial + (long long)blockIdx.x * d;
    float* own = p;
    if (kWarp) {
        __syncthreads();   // the rows that were on their way have come, or were never asked for
        own = reinterpret_cast<float*>(raw) + (size_t)warp * d;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = walk.template start<kWay>(i);
        write_pairs<kWay>(own + c, d - c, d % 8 == 0, dw[i]);
    }
    if (kWarp) {
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            float t = reinterpret_cast<const float*>(raw)[c];
            for (int w = 1; w < warps; ++w) t += reinterpret_cast<const float*>(raw)[(size_t)w * d + c];
            p[c] = t;
        }
    }
}

// dw[c] = sum of the partials, 32 columns by 32 strided runs of rows per block, the
// runs joined in order.
__global__ void __launch_bounds__(1024)
norm_weight_kernel(const float* __restrict__ partial, int blocks, int d, float* __restrict__ dweight) {
    __shared__ float part[32][33];
    dependent_kernel_start();
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < d) {
#pragma unroll 8
        for (int b = run; b < blocks; b += 32) s += partial[(long long)b * d + c];
    }
    part[run][lane] = s;
    __syncthreads();
    s = norm_warp_add(part[lane][run]);   // of column `run` of the block
    if (lane == 0 && blockIdx.x * 32 + run < d) dweight[blockIdx.x * 32 + run] = s;
}

// dw of no rows
__global__ void norm_zero_kernel(float* __restrict__ dweight, int d) {
    dependent_kernel_start();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < d) dweight[c] = 0.f;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

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
    const Weight wt = {weight, weight && weight_dtype == BITLOGIC_F32, vec_w};
    const RowShape s = row_shape(T, d);
    float* partial = dweight ? static_cast<float*>(workspace) : nullptr;
    int parts = 0;
    const int st = with_row_type(dtype, [&](auto* type) {
        using V = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
        return with_shape(s, [&](auto vecs, auto warp, auto most) {
            constexpr int kVec = decltype(vecs)::value, kThreads = decltype(most)::value;
            constexpr bool kWarp = decltype(warp)::value;
            const int resident = resident_by_registers(s.threads, kVec, kWarp);
            const size_t slots = Slots<V, kVec>::bytes(4, s.threads) + (weight ? WeightSlots<V, kVec>::bytes(s.threads, wt.wide) : 0);
            const bool ahead = vec && d % 8 == 0 && slots <= kMostShared && row_blocks(T, s) > sm_count();
            auto kern = ahead ? norm_backward_kernel<V, kVec, kWarp, kThreads, kAhead>
                        : vec ? norm_backward_kernel<V, kVec, kWarp, kThreads, kDirect>
                              : norm_backward_kernel<V, kVec, kWarp, kThreads, kSpread>;
            const size_t join = kWarp && partial ? (size_t)(s.threads / 32) * d * 4 : 0;   // dw of a block's warps
            const size_t smem = std::max(ahead ? slots : 0, join);
            if (allow_shared(kern, smem, kMostShared) != cudaSuccess) return (int)BITLOGIC_ERR_CUDA;
            const long long blocks = std::min<long long>(kNormPartials, resident_blocks(s, resident, smem, T));
            parts = (int)blocks;
            return done(launch_dependent(kern, (unsigned)blocks, (unsigned)s.threads, smem, stream, static_cast<const V*>(dY),
                                         (long long)ldy, static_cast<const V*>(H), (long long)ldh, wt,
                                         static_cast<const V*>(residual_grad), (long long)ldr, static_cast<V*>(dX), (long long)ldx,
                                         partial, (long long)T, (int)d, eps, vec));
        });
    });
    if (st != BITLOGIC_OK || !dweight) return st;
    return done(launch_dependent(norm_weight_kernel, (unsigned)((d + 31) / 32), 1024, 0, stream, (const float*)partial, parts, (int)d,
                                 dweight));
}
