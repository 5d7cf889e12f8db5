// What the norm of rows and its gradient share (norm.cu, norm_back.cu): how blocks
// walk over rows, how rows come ahead of their turn, sums over a row.
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rows8.cuh"

namespace bitlogic {
namespace {

constexpr int kMaxCols = 32768;   // 1024 threads of four vectors of eight
constexpr size_t kMostShared = 220 * 1024;

__device__ __forceinline__ float norm_warp_add(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The sum over a row's threads, a warp's or the block's; every thread gets it.
// `buf`: 32 floats, free again after the next barrier of the block.
template <bool kWarp>
__device__ __forceinline__ float row_add(float v, float* buf) {
    v = norm_warp_add(v);
    if (kWarp) return v;
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    return norm_warp_add(lane < warps ? buf[lane] : 0.f);
}
// Two sums at once: the halves of a warp take one each after the first step.
// `buf`: 64 floats.
template <bool kWarp>
__device__ __forceinline__ void row_add_two(float& a, float& b, float* buf) {
    const int lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    float v = (half ? b : a) + __shfl_xor_sync(0xffffffffu, half ? a : b, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (!kWarp) {
        const int warps = blockDim.x >> 5;
        if (l == 0) buf[32 * half + (threadIdx.x >> 5)] = v;
        __syncthreads();
        v = l < warps ? buf[32 * half + l] : 0.f;
        if (l + 16 < warps) v += buf[32 * half + l + 16];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    a = __shfl_sync(0xffffffffu, v, 0);
    b = __shfl_sync(0xffffffffu, v, 16);
}
// The largest of |v| by its bits, which NaN and infinity lead.
template <bool kWarp>
__device__ __forceinline__ uint32_t row_largest(uint32_t v, uint32_t* buf) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (kWarp) return v;
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, lane < warps ? buf[lane] : 0u);
}

// How a thread comes to a row's values.
enum Way {
    kDirect,   // as they are wanted, by vectors of 16 bytes where these lie so
    kAhead,    // through shared memory, a row ahead, by vectors that lie in the row in full
    kSpread,   // by element, a warp's lanes side by side
};

// How a block walks over rows: one at a time by all its threads, or one by each
// warp (kWarp).  A thread of a row holds the vectors of eight columns t,
// t + threads, ... of it; with kSpread the same 256 columns of a warp go by lanes.
template <bool kWarp>
struct Walk {
    int t, threads;
    long long first, step;
    __device__ __forceinline__ Walk() {
        const int warps = blockDim.x >> 5;
        t = kWarp ? threadIdx.x & 31 : threadIdx.x;
        threads = kWarp ? 32 : blockDim.x;
        first = kWarp ? (long long)blockIdx.x * warps + (threadIdx.x >> 5) : blockIdx.x;
        step = kWarp ? (long long)gridDim.x * warps : gridDim.x;
    }
    __device__ __forceinline__ int column(int i) const { return 8 * (i * threads + t); }
    // the first of the eight, and how far apart they are
    template <Way kWay>
    __device__ __forceinline__ int start(int i) const {
        return kWay == kSpread ? 8 * (i * threads + (t & ~31)) + (t & 31) : column(i);
    }
};

// A thread's own places in shared memory for a row on its way: the row after next
// is asked for while this one is worked on, without a register.  Nobody else reads
// them, so no barrier guards them.
template <typename T, int kVec>
struct Slots {
    static constexpr int kBytes = 8 * (int)sizeof(T);
    unsigned char* base;
    __device__ __forceinline__ Slots(unsigned char* raw, int row) : base(raw + place(row)) {}
    static size_t bytes(int rows, int threads) { return (size_t)rows * kVec * threads * kBytes; }
    static __device__ __forceinline__ size_t place(int row) { return (size_t)row * kVec * blockDim.x * kBytes; }
    // place `part` of vector i, 16 bytes, lanes side by side
    __device__ __forceinline__ uint4* at(int i, int part) const {
        return reinterpret_cast<uint4*>(base) + ((size_t)i * (kBytes / 16) + part) * blockDim.x + threadIdx.x;
    }
    template <bool kWarp>
    __device__ __forceinline__ void ask(const T* row, const Walk<kWarp>& walk, int d) const {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.column(i);
            if (c < d) {
#pragma unroll
                for (int q = 0; q < kBytes / 16; ++q) cp_async16(at(i, q), reinterpret_cast<const uint4*>(row + c) + q);
            }
        }
    }
    // vector i of a row that has come
    __device__ __forceinline__ void get(int i, f32x2 (&z)[4]) const {
        Eight<T> e;
        e.a = *at(i, 0);
        if constexpr (kBytes == 32) e.b = *at(i, 1);
        pairs_of(e, z);
    }
};

// 1 / sqrt(mean h^2 + eps) from the sum of squares; where that passed fp32, from
// the squares of 2^-96 h, which `again` sums.  per = 1 / d.
template <typename Again>
__device__ __forceinline__ float row_rstd(float sum, float per, float eps, Again again) {
    if (!isinf(sum)) return rsqrtf(fmaf(sum, per, eps));
    constexpr float kBy = 1.262177448e-29f;   // 2^-96
    return rsqrtf(again(kBy) * per) * kBy;
}

// A thread's eight values of a row, the first at p and n columns from the row's
// end: 0 past that.
template <Way kWay = kDirect, typename T>
__device__ __forceinline__ void read_pairs(const T* p, int n, bool vec, f32x2 (&z)[4]) {
    if constexpr (kWay == kSpread) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 32 * i < n ? to_f32(p[32 * i]) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = pack2(v[2 * i], v[2 * i + 1]);
    } else if (vec && n >= 8) {
        Eight<T> e;
        e.load(p);
        pairs_of(e, z);
    } else {
        float v[8];
        load_eight(p, n, false, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = pack2(v[2 * i], v[2 * i + 1]);
    }
}
template <Way kWay = kDirect, typename T>
__device__ __forceinline__ void write_pairs(T* p, int n, bool vec, const f32x2 (&z)[4]) {
    if constexpr (kWay == kSpread) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b;
            unpack2(z[i], a, b);
            if (64 * i < n) p[64 * i] = from_f32<T>(a);
            if (64 * i + 32 < n) p[64 * i + 32] = from_f32<T>(b);
        }
    } else if (vec && n >= 8) {
        eight_of<T>(z).store(p);
    } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(z[i], v[2 * i], v[2 * i + 1]);
        store_eight(p, n, false, v);
    }
}

// The weight of a norm: fp32 or the rows' type, or none.
struct Weight {
    const void* w;
    bool wide, vec;   // fp32; on 16 bytes
};
template <typename T, Way kWay>
__device__ __forceinline__ void weight_pairs(const Weight& weight, int c, int n, f32x2 (&w)[4]) {
    if (weight.wide) read_pairs<kWay>(static_cast<const float*>(weight.w) + c, n, weight.vec, w);
    else read_pairs<kWay>(static_cast<const T*>(weight.w) + c, n, weight.vec, w);
}
// A thread's own columns of the weight in shared memory for all of its rows, for the
// gradient, which reads them twice a row: beside rows on their way L1 has no room
// for them (16384 x 8192 bf16: 195 us with the weight read from L1 and L2, 158 from
// here; the norm itself, which reads them once, 296 and 304).
template <typename T, int kVec>
struct WeightSlots {
    unsigned char* base;
    bool wide;
    static size_t bytes(int threads, bool wide) { return (size_t)kVec * threads * 8 * (wide ? 4 : sizeof(T)); }
    __device__ __forceinline__ uint4* at(int i, int part) const {
        return reinterpret_cast<uint4*>(base) + ((size_t)i * (wide || sizeof(T) == 4 ? 2 : 1) + part) * blockDim.x + threadIdx.x;
    }
    template <bool kWarp>
    __device__ __forceinline__ void fill(const Weight& weight, const Walk<kWarp>& walk, int d) const {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = walk.column(i);
            if (c >= d) continue;
            if (wide) {
                f32x2 w[4];
                read_pairs(static_cast<const float*>(weight.w) + c, 8, weight.vec, w);
                const Eight<float> e = eight_of<float>(w);
                *at(i, 0) = e.a;
                *at(i, 1) = e.b;
            } else {
                f32x2 w[4];
                read_pairs(static_cast<const T*>(weight.w) + c, 8, weight.vec, w);
                const Eight<T> e = eight_of<T>(w);
                *at(i, 0) = e.a;
                if constexpr (sizeof(T) == 4) *at(i, 1) = e.b;
            }
        }
    }
    __device__ __forceinline__ void get(int i, f32x2 (&w)[4]) const {
        if (wide) {
            Eight<float> e;
            e.a = *at(i, 0);
            e.b = *at(i, 1);
            pairs_of(e, w);
        } else {
            Eight<T> e;
            e.a = *at(i, 0);
            if constexpr (sizeof(T) == 4) e.b = *at(i, 1);
            pairs_of(e, w);
        }
    }
};
__device__ __forceinline__ float sum_of(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

// How rows of d columns are taken.  Few rows: a vector per thread, so that a row
// is over soon.  Many: two, so that a block's barriers cost less (32768 rows of
// 8192 bf16 columns to e4m3: one vector 422 us, two 346, four 362).  Up to 1024
// columns a warp has a row to itself where rows are many.
struct RowShape {
    bool warp;
    int threads, vec;   // of a block
};
inline RowShape row_shape(int64_t rows, int d) {
    const int vectors = (d + 7) / 8;
    if (vectors <= 128 && (rows > 16 * sm_count() || vectors <= 32)) {
        return {true, rows > 16 * sm_count() ? 256 : 32, vectors <= 32 ? 1 : vectors <= 64 ? 2 : 4};
    }
    int vec = rows > sm_count() && vectors > 256 ? 2 : 1;
    while ((vectors + vec - 1) / vec > 1024) vec *= 2;
    const int threads = (vectors + vec - 1) / vec;
    return {false, (threads + 31) / 32 * 32, vec};
}
inline long long row_blocks(int64_t rows, const RowShape& s) { return s.warp ? (rows + s.threads / 32 - 1) / (s.threads / 32) : rows; }

// Blocks of a kernel that an SM holds by its registers: 64 a thread, or 128 where
// warps hold four vectors.
constexpr int resident_by_registers(int threads, int vec, bool warp) { return 65536 / (threads * (warp && vec == 4 ? 128 : 64)); }

// Persistent blocks: those that run at once, at most one per row.
inline long long resident_blocks(const RowShape& s, int by_registers, size_t smem, int64_t rows) {
    const long long by_shared = (long long)(227 * 1024 / (smem + 2048)), per = std::min<long long>(by_registers, by_shared);
    return std::min<long long>(row_blocks(rows, s), sm_count() * std::max<long long>(1, std::min<long long>(per, 2048 / s.threads)));
}
// The limit on a kernel's shared memory, set to the most that it is launched with.
template <typename K>
inline cudaError_t allow_shared(K kern, size_t smem, size_t most) {
    return smem > 32 * 1024 ? cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) : cudaSuccess;
}
// f(vectors of a thread, whether a warp has a row, the most threads of a block)
template <typename F>
inline int with_shape(const RowShape& s, F f) {
    using std::integral_constant;
    using k256 = integral_constant<int, 256>;
    using k512 = integral_constant<int, 512>;
    using k1024 = integral_constant<int, 1024>;
    if (s.warp) {
        if (s.vec == 1) return f(integral_constant<int, 1>(), std::true_type(), k256());
        if (s.vec == 2) return f(integral_constant<int, 2>(), std::true_type(), k256());
        return f(integral_constant<int, 4>(), std::true_type(), k256());
    }
    if (s.vec == 1) return f(integral_constant<int, 1>(), std::false_type(), k1024());
    if (s.vec == 2 && s.threads <= 512) return f(integral_constant<int, 2>(), std::false_type(), k512());
    if (s.vec == 2) return f(integral_constant<int, 2>(), std::false_type(), k1024());
    return f(integral_constant<int, 4>(), std::false_type(), k1024());
}

inline int done(cudaError_t e) { return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA; }

inline bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes != 0; }

// Row strides of the [T][d] matrices of a call.
inline bool stride_ok(const void* p, int64_t ld, int64_t T, int d) {
    return !p || T <= 1 || (ld >= d && ld <= (1LL << 40) / T);
}

}  // namespace
}  // namespace bitlogic
