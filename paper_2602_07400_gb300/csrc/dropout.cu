// Dropout from a counter-based generator, with the addition of a residual:
//
//   out_i = (number_i >= round(p 2^32) ? x_i / (1 - p) : 0) + residual_i
//
// number_i, 32 bits, comes from Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011) under the key `seed`:
// the 8 elements 8 b .. 8 b + 7 share the two counters (b, step, stream) with
// stream = 2 site and 2 site + 1; element 8 b + j takes half-word j of the first
// one's four words as its number's high half and half-word j of the second one's
// as the low half.  Nothing is stored for the gradient, which is the same call on
// the output's gradient.
//
// Bound by reading x (and the residual) and writing out once.  The generator is
// what competes: of 2^28 bf16 values (1.07 GB moved) one Philox call for every 4
// of them took 220 us, one for every 8 took 170, and a plain copy of the same
// bytes 168.  So the high halves decide, and the second counter is only drawn
// where a high half equals the threshold's: one element in 65536.  The round keys
// stay in registers and the comparisons are of whole words (16384 x 8192 bf16 with
// residual, and its gradient: 252 us without either, 212 with: 1.34 GB at 93% of
// the measured HBM rate).
#include <cmath>
#include <type_traits>

#include "rows8.cuh"

namespace bitlogic {
namespace {

constexpr int kDropThreads = 256;
// Outputs past this many bytes are marked as read once: they would only push
// others out of the 126 MB of L2 (16384 x 8192 bf16 with and without a residual:
// 212 us marked, 218 not); what fits is left for its reader.
constexpr long long kKeep = 64LL << 20;

struct DropRule {
    const long long* counter;   // seed, step
    uint32_t threshold;         // round(p 2^32)
    float scale;                // 1 / (1 - p)
    uint32_t stream;            // 2 site
};

// The keys of the ten rounds, kept in registers: they come from memory, so each
// thread would add them up again for every call.
struct RoundKeys {
    uint32_t a[10], b[10];
    __device__ __forceinline__ explicit RoundKeys(unsigned long long seed) {
        a[0] = (uint32_t)seed;
        b[0] = (uint32_t)(seed >> 32);
#pragma unroll
        for (int r = 1; r < 10; ++r) {
            a[r] = a[r - 1] + 0x9E3779B9u;
            b[r] = b[r - 1] + 0xBB67AE85u;
        }
    }
};
__device__ __forceinline__ uint4 philox(uint4 c, const RoundKeys& key) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = (unsigned long long)0xD2511F53u * c.x, b = (unsigned long long)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ key.a[r], (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ key.b[r], (uint32_t)a);
    }
    return c;
}

// The generator of a call: which of a block's 8 elements are kept, a bit each.
struct Keeper {
    RoundKeys key;
    uint32_t step, stream, high, low;

    __device__ __forceinline__ explicit Keeper(const DropRule& r)
        : key((unsigned long long)r.counter[0]), step((uint32_t)r.counter[1]), stream(r.stream), high(r.threshold >> 16),
          low(r.threshold & 0xffffu) {}
    static __device__ __forceinline__ uint32_t half_word(const uint4& w, int j) {
        const uint32_t u = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
        return (j & 1) ? u >> 16 : u & 0xffffu;
    }
    __device__ __forceinline__ uint4 counter(unsigned long long block) const {
        return make_uint4((uint32_t)block, (uint32_t)(block >> 32), step, stream);
    }
    // Whether a half-word of w equals the threshold's high half, and so the low
    // halves decide: a zero half of the difference borrows out of it.
    __device__ __forceinline__ bool level(const uint4& w) const {
        if (low == 0u) return false;   // alike in all threads
        const uint32_t both = high * 0x10001u;
        auto zero_half = [&](uint32_t u) { return ((u ^ both) - 0x10001u) & ~(u ^ both); };
        return (zero_half(w.x) | zero_half(w.y) | zero_half(w.z) | zero_half(w.w)) & 0x80008000u;
    }
    // whether element j is kept where no half is level
    __device__ __forceinline__ bool keeps(const uint4& w, int j) const {
        const uint32_t u = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
        return ((j & 1) ? u : u << 16) >= high << 16;   // the half below cannot decide
    }
    // the same with the low halves looked at, a bit each
    __device__ __forceinline__ uint32_t exact(const uint4& w, unsigned long long block) const {
        uint4 c = counter(block);
        c.w += 1u;
        const uint4 d = philox(c, key);
        uint32_t keep = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t h = half_word(w, j);
            keep |= (h > high || (h == high && half_word(d, j) >= low) ? 1u : 0u) << j;
        }
        return keep;
    }
    __device__ __forceinline__ uint32_t operator()(unsigned long long block) const {
        const uint4 w = philox(counter(block), key);
        if (level(w)) return exact(w, block);
        uint32_t keep = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) keep |= (keeps(w, j) ? 1u : 0u) << j;
        return keep;
    }
};

// Where the 8 elements of a block lie side by side on 16 bytes, in x, residual
// and out.  `width`: blocks of a row; kFlat: the rows follow one another.  Two
// blocks at a time, so that twice the bytes are on their way.
template <typename T, bool kResidual, bool kFlat>
__global__ void __launch_bounds__(kDropThreads)
dropout_vec_kernel(const T* x, long long ldx, const T* residual, long long ldr, T* out, long long ldo, long long blocks,
                   long long width, bool once, DropRule rule) {
    dependent_kernel_start();
    const Keeper keeper(rule);
    auto place = [&](long long b, long long ld) {
        if (kFlat) return b * 8;
        const long long row = b < 0x100000000LL && width < 0x100000000LL ? (long long)((uint32_t)b / (uint32_t)width) : b / width;
        return row * ld + (b - row * width) * 8;
    };
    auto finish = [&](long long b, const Eight<T>& ex, const Eight<T>& er) {
        const uint4 w = philox(keeper.counter((unsigned long long)b), keeper.key);
        float v[8], r[8];
        ex.get(v);
        if (kResidual) er.get(r);
        const bool level = keeper.level(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = v[i] * rule.scale;
            v[i] = keeper.keeps(w, i) ? y : 0.f;
        }
        if (level) {   // one block of eight in 8192
            const uint32_t keep = keeper.exact(w, (unsigned long long)b);
            ex.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (keep >> i & 1u) ? v[i] * rule.scale : 0.f;
        }
        if (kResidual) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += r[i];
        }
        Eight<T> e;
        e.set(v);
        if (once) e.store_once(out + place(b, ldo));
        else e.store(out + place(b, ldo));
    };
    const long long stride = (long long)gridDim.x * kDropThreads;
    for (long long b = (long long)blockIdx.x * kDropThreads + threadIdx.x; b < blocks; b += 2 * stride) {
        Eight<T> x0, x1, r0, r1;
        const bool two = b + stride < blocks;
        x0.load_once(x + place(b, ldx));
        if (two) x1.load_once(x + place(b + stride, ldx));
        if (kResidual) {
            r0.load_once(residual + place(b, ldr));
            if (two) r1.load_once(residual + place(b + stride, ldr));
        }
        finish(b, x0, r0);
        if (two) finish(b + stride, x1, r1);
    }
}

// Any strides and lengths: a warp takes 32 blocks, 256 elements; lane l draws
// block l, and the elements are then visited 32 side by side.
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const T* x, long long ldx, const T* residual, long long ldr, T* out, long long ldo, long long n,
               long long cols, DropRule rule) {
    dependent_kernel_start();
    const Keeper keeper(rule);
    const int lane = threadIdx.x & 31;
    const long long warps = (long long)gridDim.x * (kDropThreads / 32);
    for (long long w = ((long long)blockIdx.x * kDropThreads + threadIdx.x) >> 5; w * 256 < n; w += warps) {
        const uint32_t keep = keeper((unsigned long long)(w * 32 + lane));
        // row and column of the lane's first element; its others are 32 columns on
        const long long e0 = w * 256 + lane;
        long long row = e0 < 0x100000000LL && cols < 0x100000000LL ? (long long)((uint32_t)e0 / (uint32_t)cols) : e0 / cols;
        long long col = e0 - row * cols;
        T v[8], r[8];
        long long at[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            at[i] = row * ldo + col;
            if (e0 + 32 * i < n) {
                v[i] = x[row * ldx + col];
                if (kResidual) r[i] = residual[row * ldr + col];
            }
            col += 32;
            if (col >= cols) {
                const long long over = cols >= 32 ? 1 : col / cols;
                row += over;
                col -= over * cols;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t mine = __shfl_sync(0xffffffffu, keep, 4 * i + (lane >> 3));
            if (e0 + 32 * i < n) {
                float y = (mine >> (lane & 7) & 1u) ? to_f32(v[i]) * rule.scale : 0.f;
                if (kResidual) y += to_f32(r[i]);
                out[at[i]] = from_f32<T>(y);
            }
        }
    }
}

template <typename T>
int launch_dropout(const T* x, int64_t ldx, const T* residual, int64_t ldr, T* out, int64_t ldo, int64_t R, int64_t C,
                   const DropRule& rule, cudaStream_t stream) {
    const bool side_by_side = R == 1 || (ldx == C && ldo == C && (!residual || ldr == C));
    const bool vec = rows_aligned16(x, side_by_side ? 0 : ldx, R, sizeof(T)) && rows_aligned16(out, side_by_side ? 0 : ldo, R, sizeof(T)) &&
                     (!residual || rows_aligned16(residual, side_by_side ? 0 : ldr, R, sizeof(T))) &&
                     (side_by_side ? R * C % 8 == 0 : C % 8 == 0);
    const long long n = R * C, cap = 16LL * sm_count();
    cudaError_t e;
    if (vec) {
        const long long blocks = n / 8, width = side_by_side ? 0 : C / 8;
        const long long grid = (blocks + kDropThreads - 1) / kDropThreads;
        auto kern = side_by_side ? (residual ? dropout_vec_kernel<T, true, true> : dropout_vec_kernel<T, false, true>)
                                 : (residual ? dropout_vec_kernel<T, true, false> : dropout_vec_kernel<T, false, false>);
        e = launch_dependent(kern, (unsigned)(grid < cap ? grid : cap), kDropThreads, 0, stream, x, (long long)ldx, residual,
                             (long long)ldr, out, (long long)ldo, blocks, width, n * (long long)sizeof(T) > kKeep, rule);
    } else {
        const long long grid = (n + 8 * kDropThreads - 1) / (8 * kDropThreads);
        auto kern = residual ? dropout_kernel<T, true> : dropout_kernel<T, false>;
        e = launch_dependent(kern, (unsigned)(grid < cap ? grid : cap), kDropThreads, 0, stream, x, (long long)ldx, residual,
                             (long long)ldr, out, (long long)ldo, n, side_by_side ? n : (long long)C, rule);
    }
    return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

extern "C" int bitlogic_dropout(const void* X, int32_t dtype, int64_t R, int64_t C, int64_t ldx, const void* residual,
                                int64_t ldr, void* out, int64_t ldo, const int64_t* counter, double p, int32_t site,
                                cudaStream_t stream) {
    if (dtype != BITLOGIC_F32 && dtype != BITLOGIC_BF16 && dtype != BITLOGIC_F16) return BITLOGIC_ERR_DTYPE;
    constexpr int64_t kMost = 1LL << 40;
    if (R < 0 || C < 0 || R > kMost || C > kMost || (C > 0 && R > kMost / C)) return BITLOGIC_ERR_SHAPE;
    if (R == 0 || C == 0) return BITLOGIC_OK;
    if (R > 1 && (ldx < C || ldo < C || (residual && ldr < C) || ldx > kMost || ldo > kMost || (residual && ldr > kMost)))
        return BITLOGIC_ERR_SHAPE;
    if (R > 1 && ((ldx > kMost / R) || (ldo > kMost / R) || (residual && ldr > kMost / R))) return BITLOGIC_ERR_SHAPE;
    // not NaN, and a threshold below 2^32
    if (!(p >= 0.0) || !(p * 4294967296.0 < 4294967295.5) || site < 0) return BITLOGIC_ERR_HYPER;
    if (!X || !out || !counter) return BITLOGIC_ERR_NULL;
    const uintptr_t size = (uintptr_t)row_type_bytes(dtype);
    if (reinterpret_cast<uintptr_t>(X) % size || reinterpret_cast<uintptr_t>(out) % size ||
        reinterpret_cast<uintptr_t>(residual) % size || reinterpret_cast<uintptr_t>(counter) % 8)
        return BITLOGIC_ERR_ALIGN;
    DropRule rule;
    rule.counter = reinterpret_cast<const long long*>(counter);
    rule.threshold = (uint32_t)llrint(p * 4294967296.0);
    rule.scale = (float)(1.0 / (1.0 - p));
    rule.stream = 2u * (uint32_t)site;
    return with_row_type(dtype, [&](auto* type) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
        return launch_dropout(static_cast<const T*>(X), ldx, static_cast<const T*>(residual), ldr, static_cast<T*>(out), ldo,
                              R, C, rule, stream);
    });
}
