// A row of logits held in the shared memory of one block, or of the blocks of
// one cluster, each a contiguous slice.
//
// Slices are cut at 16-byte boundaries of memory, not of the row, so rows of
// any alignment are copied with 16-byte cp.async; the pieces that reach over
// the row's ends are filled by element, with -inf in the places that are not
// the row's.  Every pass then works on whole pieces.
#pragma once

#include "logits.cuh"
#include "packed.cuh"

namespace bitlogic {

constexpr int kMaxCluster = 8;

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned cluster_size() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// The cluster's barrier; writes to another block's shared memory before the
// arrival are visible after the wait.  Every thread of every block takes part.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Another block's shared memory may be touched only once that block runs: each
// block of a cluster reports at its kernel's start, behind which it asks for its
// slice, and waits for the others just before its first store to one of them.
// The report orders no memory, so it does not wait for loads on their way.
__device__ __forceinline__ void report_running(unsigned blocks) {
    if (blocks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void wait_all_running(unsigned blocks) {
    if (blocks > 1) cluster_wait();
}

// The address of `p` (this block's shared memory) in block `rank`, and a
// store of 4 bytes there.
__device__ __forceinline__ void store_in_block(const void* p, unsigned rank, uint32_t v) {
    const unsigned s = (unsigned)__cvta_generic_to_shared(p);
    asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %0, %1;\nst.shared::cluster.u32 [a], %2;\n}\n"
                 ::"r"(s), "r"(rank), "r"(v) : "memory");
}
// A struct of 4-byte words to the same place in block `rank`.
template <typename S>
__device__ __forceinline__ void put_in_block(S* p, unsigned rank, const S& v) {
    static_assert(sizeof(S) % 4 == 0, "whole words");
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(S) / 4); ++i) store_in_block(reinterpret_cast<uint32_t*>(p) + i, rank, w[i]);
}

// Adds v to a counter in block `rank` and returns what it held.
__device__ __forceinline__ unsigned add_in_block(unsigned* p, unsigned rank, unsigned v) {
    const unsigned s = (unsigned)__cvta_generic_to_shared(p);
    unsigned r;
    asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %1, %2;\natom.shared::cluster.add.u32 %0, [a], %3;\n}\n"
                 : "=r"(r) : "r"(s), "r"(rank), "r"(v) : "memory");
    return r;
}

// Sorts a[0, size) in falling order, size a power of two (bitonic exchanges);
// called by the whole block.  Exchanges over 32 places or fewer stay within the
// 64 places that a warp's 32 pairs cover, so they need no barrier of the block.
__device__ __forceinline__ void block_sort_falling(unsigned long long* a, int size) {
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int i = threadIdx.x; i < size / 2; i += blockDim.x) {
                const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
                const unsigned long long x = a[lo], y = a[hi];
                if ((x < y) == ((lo & k) == 0)) {
                    a[lo] = y;
                    a[hi] = x;
                }
            }
            if (j > 32 || (j == 1 && k >= 64)) __syncthreads();   // the next exchange may span warps
            else __syncwarp();
        }
    __syncthreads();
}

// The logit of a key.
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k); }

// A bound of the largest values that a block's threads hold G of each: the
// largest key of 16 leading bits that at least `need` of them reach (0 when
// fewer rank), by 8 bits at a time.  Called by the whole block.
struct BoundScratch {
    unsigned bins[2][256];
    unsigned digit[2], above;
};
template <int G>
__device__ __forceinline__ uint32_t block_bound(const float (&v)[G], unsigned need, BoundScratch* s) {
    uint32_t key[G];
#pragma unroll
    for (int i = 0; i < G; ++i) key[i] = logit_key(v[i]) >> 16;
    const int tid = threadIdx.x, lane = tid & 31;
    for (int i = tid; i < 256; i += blockDim.x) s->bins[0][i] = s->bins[1][i] = 0u;
    if (tid == 0) s->digit[0] = s->digit[1] = s->above = 0u;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        unsigned* bins = s->bins[pass];
        const uint32_t top = s->digit[0];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            if (pass == 0) atomicAdd(&bins[key[i] >> 8], 1u);
            else if ((key[i] >> 8) == top) atomicAdd(&bins[key[i] & 255u], 1u);
        }
        __syncthreads();
        if (tid < 32) {   // lane l: bins 255 - 8 l down to 248 - 8 l
            const unsigned start = pass == 0 ? 0u : s->above;
            unsigned own = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) own += bins[255 - 8 * lane - i];
            unsigned upto = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned t = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += t;
            }
            const unsigned m = __ballot_sync(0xffffffffu, start + upto >= need);
            if (m && lane == __ffs(m) - 1) {
                unsigned n = start + upto - own;
                int d = 255 - 8 * lane;
                while (n + bins[d] < need) n += bins[d--];
                s->digit[pass] = (unsigned)d;
                s->above = n;
            }
        }
        __syncthreads();
    }
    return (s->digit[0] << 24) | (s->digit[1] << 16);
}
// The smallest logit that such a bound lets through.
__device__ __forceinline__ float bound_logit(uint32_t key) { return key <= kKeyNegInf ? BITLOGIC_NEG_INF : key_logit(key); }

// 16 bytes of logits: their number, their values, their maximum (in two parts,
// each of half the piece's logits), and the rounding of values back into a
// piece.
template <typename T> struct Piece;

template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void load(const uint4& u, float (&z)[4]) {
        z[0] = __uint_as_float(u.x);
        z[1] = __uint_as_float(u.y);
        z[2] = __uint_as_float(u.z);
        z[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&g)[4]) {
        return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
    }
    struct Max {
        float a, b;
    };
    static __device__ __forceinline__ Max lowest() { return {BITLOGIC_NEG_INF, BITLOGIC_NEG_INF}; }
    static __device__ __forceinline__ Max largest(Max m, const uint4& u) {
        return {fmaxf(m.a, fmaxf(__uint_as_float(u.x), __uint_as_float(u.y))),
                fmaxf(m.b, fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)))};
    }
    static __device__ __forceinline__ Max either(Max m, Max n) { return {fmaxf(m.a, n.a), fmaxf(m.b, n.b)}; }
    static __device__ __forceinline__ void parts(Max m, float& a, float& b) { a = m.a, b = m.b; }
    static __device__ __forceinline__ float value(Max m) { return fmaxf(m.a, m.b); }
    static __device__ __forceinline__ float largest_of(const uint4& u) {
        return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
    }
};
template <> struct Piece<int> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void load(const uint4& u, float (&z)[4]) {
        z[0] = logit_value((int)u.x);
        z[1] = logit_value((int)u.y);
        z[2] = logit_value((int)u.z);
        z[3] = logit_value((int)u.w);
    }
    struct Max {
        int a, b;
    };
    static __device__ __forceinline__ Max lowest() { return {INT_MIN, INT_MIN}; }
    static __device__ __forceinline__ Max largest(Max m, const uint4& u) {
        return {max(m.a, max((int)u.x, (int)u.y)), max(m.b, max((int)u.z, (int)u.w))};
    }
    static __device__ __forceinline__ Max either(Max m, Max n) { return {max(m.a, n.a), max(m.b, n.b)}; }
    static __device__ __forceinline__ void parts(Max m, float& a, float& b) { a = logit_value(m.a), b = logit_value(m.b); }
    static __device__ __forceinline__ float value(Max m) { return logit_value(max(m.a, m.b)); }
    static __device__ __forceinline__ float largest_of(const uint4& u) { return value(largest({(int)u.x, (int)u.z}, u)); }
};
template <> struct Piece<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void two(uint32_t u, float& a, float& b) {
        a = __uint_as_float(u << 16);
        b = __uint_as_float(u & 0xffff0000u);
    }
    static __device__ __forceinline__ void load(const uint4& u, float (&z)[8]) {
        two(u.x, z[0], z[1]);
        two(u.y, z[2], z[3]);
        two(u.z, z[4], z[5]);
        two(u.w, z[6], z[7]);
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
    static __device__ __forceinline__ uint4 pack(const float (&g)[8]) {
        return make_uint4(pair(g[0], g[1]), pair(g[2], g[3]), pair(g[4], g[5]), pair(g[6], g[7]));
    }
    using Max = __nv_bfloat162;
    static __device__ __forceinline__ Max as(uint32_t u) { return *reinterpret_cast<const Max*>(&u); }
    static __device__ __forceinline__ Max lowest() { return as(0xff80ff80u); }
    static __device__ __forceinline__ Max largest(Max m, const uint4& u) {   // of two numbers: NaN is passed over
        return __hmax2(__hmax2(m, __hmax2(as(u.x), as(u.y))), __hmax2(as(u.z), as(u.w)));
    }
    static __device__ __forceinline__ Max either(Max m, Max n) { return __hmax2(m, n); }
    static __device__ __forceinline__ void parts(Max m, float& a, float& b) { a = __low2float(m), b = __high2float(m); }
    static __device__ __forceinline__ float value(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
    static __device__ __forceinline__ float largest_of(const uint4& u) { return value(largest(as(u.x), u)); }
};
template <> struct Piece<__half> {
    static constexpr int N = 8;
    static __device__ __forceinline__ __half2 as(uint32_t u) { return *reinterpret_cast<const __half2*>(&u); }
    static __device__ __forceinline__ void load(const uint4& u, float (&z)[8]) {
        const float2 a = __half22float2(as(u.x)), b = __half22float2(as(u.y)), c = __half22float2(as(u.z)),
                     d = __half22float2(as(u.w));
        z[0] = a.x; z[1] = a.y; z[2] = b.x; z[3] = b.y;
        z[4] = c.x; z[5] = c.y; z[6] = d.x; z[7] = d.y;
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b) {
        const __half2 p = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
    static __device__ __forceinline__ uint4 pack(const float (&g)[8]) {
        return make_uint4(pair(g[0], g[1]), pair(g[2], g[3]), pair(g[4], g[5]), pair(g[6], g[7]));
    }
    using Max = __half2;
    static __device__ __forceinline__ Max lowest() { return as(0xfc00fc00u); }
    static __device__ __forceinline__ Max largest(Max m, const uint4& u) {
        return __hmax2(__hmax2(m, __hmax2(as(u.x), as(u.y))), __hmax2(as(u.z), as(u.w)));
    }
    static __device__ __forceinline__ Max either(Max m, Max n) { return __hmax2(m, n); }
    static __device__ __forceinline__ void parts(Max m, float& a, float& b) { a = __low2float(m), b = __high2float(m); }
    static __device__ __forceinline__ float value(Max m) { return fmaxf(__low2float(m), __high2float(m)); }
    static __device__ __forceinline__ float largest_of(const uint4& u) { return value(largest(as(u.x), u)); }
};

template <typename T> __device__ __forceinline__ T masked_logit();
template <> __device__ __forceinline__ float masked_logit<float>() { return BITLOGIC_NEG_INF; }
template <> __device__ __forceinline__ int masked_logit<int>() { return INT_MIN; }
template <> __device__ __forceinline__ __nv_bfloat16 masked_logit<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }
template <> __device__ __forceinline__ __half masked_logit<__half>() { return __ushort_as_half(0xfc00); }

// The values of a piece as pairs, and pairs rounded back into a piece.
template <typename T>
__device__ __forceinline__ void load_pairs(const uint4& u, f32x2 (&z)[Piece<T>::N / 2]) {
    float x[Piece<T>::N];
    Piece<T>::load(u, x);
#pragma unroll
    for (int i = 0; i < Piece<T>::N / 2; ++i) z[i] = pack2(x[2 * i], x[2 * i + 1]);
}

// 2^v of both elements
__device__ __forceinline__ f32x2 exp2_pair(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return pack2(exp2_unit(a), exp2_unit(b));
}

// The exponents c z - base of a slice's powers, the base near c m for the
// slice's largest logit m: one multiply-add each where c m is below 2^28 (the
// base is then rint(c m), so that bases of slices differ by whole numbers), the
// difference z - m first where it is not, which keeps the digits that equal or
// nearby logits of that size differ in.
struct PowerBase {
    float c, m, b;
    bool far, none;   // none: no logit in the sum
    __device__ __forceinline__ PowerBase(float largest, float c_)
        : c(c_), m(largest == BITLOGIC_NEG_INF ? 0.f : largest), none(largest == BITLOGIC_NEG_INF) {
        const float mc = m * c;
        far = !(fabsf(mc) < 268435456.0f);
        b = far ? 0.f : rintf(mc);
    }
    __device__ __forceinline__ float exponent(float z) const { return far ? (z - m) * c : fmaf(z, c, -b); }
    __device__ __forceinline__ float power(float z) const { return exp2_unit(exponent(z)); }
    // whether powers of logits up to `z` about this base stay well inside fp32
    __device__ __forceinline__ bool holds(float z) const { return !none && (far ? z <= m : fmaf(z, c, -b) <= 64.f); }
    // ln of a sum of powers about this base, taken to logits (c = log2(e) / tau)
    __device__ __forceinline__ float log_of(float sum, float inv_tau) const {
        return far ? m * inv_tau + logf(sum) : kLn2 * (b + log2f(sum));
    }
    // the factor that takes a sum about this base to one about `row`
    __device__ __forceinline__ float to(const PowerBase& row) const {
        if (none) return 1.f;   // of a sum of 0, or of NaN
        if (!row.far) return exp2_unit(far ? fmaf(m, c, -row.b) : b - row.b);
        return exp2_unit((m - row.m) * c - (far ? 0.f : fmaf(m, c, -b)));
    }
};
// `p`, far where either of two bases about one logit is.
__device__ __forceinline__ PowerBase far_alike(PowerBase p, const PowerBase& other) {
    p.far = p.far || other.far;
    if (p.far) p.b = 0.f;
    return p;
}
struct NearPairs {
    f32x2 c, nb;
    __device__ __forceinline__ explicit NearPairs(const PowerBase& p) : c(pack2(p.c, p.c)), nb(pack2(-p.b, -p.b)) {}
    __device__ __forceinline__ f32x2 operator()(f32x2 z) const { return exp2_pair(fma2(z, c, nb)); }
};
struct FarPairs {
    f32x2 c, m;
    __device__ __forceinline__ explicit FarPairs(const PowerBase& p) : c(pack2(p.c, p.c)), m(pack2(p.m, p.m)) {}
    __device__ __forceinline__ f32x2 operator()(f32x2 z) const { return exp2_pair(mul2(sub2(z, m), c)); }
};

// A block's slice: pieces [0, n), piece j holding classes first + N j + i.
template <typename T>
struct RowSlice {
    static constexpr int N = Piece<T>::N;
    int first;   // class of the first place (below 0 where the row starts inside the piece)
    int n;

    __device__ __forceinline__ RowSlice(const T* x, int V, unsigned rank, unsigned blocks) {
        const int shift = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
        const int all = (shift + V + N - 1) / N, per = (all + (int)blocks - 1) / (int)blocks;
        const int p0 = min(all, (int)rank * per);
        n = min(all, p0 + per) - p0;
        first = p0 * N - shift;
    }
    // Pieces [whole0, whole1) lie in the row in full; at most one before and
    // one after do not.
    __device__ __forceinline__ int whole0() const { return first < 0 && n > 0 ? 1 : 0; }
    __device__ __forceinline__ int whole1(int V) const { return n > 0 && first + n * N > V ? max(whole0(), n - 1) : n; }
    // Copies on their way; finish with cp_async_wait<0>() and a barrier.
    __device__ __forceinline__ void copy(const T* x, int V, T* tile, int tid, int threads) const {
        const int w0 = whole0(), w1 = whole1(V);
        const T* from = x + first;   // read at whole pieces only
#pragma unroll 4
        for (int j = w0 + tid; j < w1; j += threads) cp_async16(tile + j * N, from + j * N);
        cp_async_commit();
        // the places of the pieces at the row's ends, by element
        if (tid < 2 * N) {
            const int j = tid < N ? 0 : n - 1, p = j * N + tid % N, v = first + p;
            if (n > 0 && (j < w0 || j >= w1)) tile[p] = v >= 0 && v < V ? x[v] : masked_logit<T>();
        }
    }
    // Place of class v in the slice, or -1.
    __device__ __forceinline__ int place(int v) const {
        const int p = v - first;
        return v >= 0 && p >= 0 && p < n * N ? p : -1;
    }
};

// A piece of masked logits.
template <typename T>
__device__ __forceinline__ uint4 masked_piece() {
    constexpr uint32_t w = std::is_same_v<T, float> ? 0xff800000u : std::is_same_v<T, int> ? 0x80000000u
                         : std::is_same_v<T, __nv_bfloat16> ? 0xff80ff80u : 0xfc00fc00u;
    return make_uint4(w, w, w, w);
}

// The whole pieces of a row streamed through registers by a block of kThreads:
// batches of four pieces of every thread, a warp's 128 pieces of a batch side by
// side, a batch loaded while the one before it is used.
template <typename T, int kThreads>
struct PieceStream {
    static constexpr int N = Piece<T>::N;
    const uint4* from;   // piece 0, read at whole pieces
    int j0, j1;          // this thread's first piece, and the end of the whole ones
    int batches;         // that cover all threads' pieces

    static __device__ __forceinline__ int first_of(int tid) { return (tid >> 5) * 128 + (tid & 31); }

    __device__ __forceinline__ PieceStream(const T* x, const RowSlice<T>& slice, int V, int tid)
        : from(reinterpret_cast<const uint4*>(x + slice.first)), j0(slice.whole0() + first_of(tid)), j1(slice.whole1(V)),
          batches((max(0, slice.whole1(V) - slice.whole0()) + 4 * kThreads - 1) / (4 * kThreads)) {}
    __device__ __forceinline__ int piece(int q, int i) const { return j0 + 4 * kThreads * q + 32 * i; }
    __device__ __forceinline__ void load(int q, uint4 (&u)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = piece(q, i);
            u[i] = j < j1 ? __ldcg(from + j) : masked_piece<T>();
        }
    }
};

// A piece at the row's ends, by element; places outside the row are masked.
template <typename T>
__device__ __forceinline__ uint4 end_piece(const T* x, int V, int first_class) {
    T e[Piece<T>::N];
#pragma unroll
    for (int i = 0; i < Piece<T>::N; ++i) {
        const int v = first_class + i;
        e[i] = v >= 0 && v < V ? x[v] : masked_logit<T>();
    }
    uint4 u;
    memcpy(&u, e, 16);
    return u;
}

// Pairs hi + lo of fp32 numbers (lo below half an ulp of hi), by the error-free
// sum and product of Knuth and Dekker: 48 bits of mantissa on the fp32 pipe, for
// the few numbers of a row that need more than fp32.
struct Pair {
    float hi, lo;
};
__device__ __forceinline__ Pair exact_sum(float a, float b) {
    const float s = a + b, t = s - a;
    return {s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Pair exact_product(float a, float b) {
    const float p = a * b;
    return {p, fmaf(a, b, -p)};
}
__device__ __forceinline__ Pair pair_add(Pair x, Pair y) {
    const Pair s = exact_sum(x.hi, y.hi);
    const float lo = s.lo + (x.lo + y.lo), hi = s.hi + lo;
    return {hi, lo - (hi - s.hi)};
}
__device__ __forceinline__ Pair pair_multiply(Pair x, Pair y) {
    const Pair p = exact_product(x.hi, y.hi);
    const float lo = p.lo + (x.hi * y.lo + x.lo * y.hi), hi = p.hi + lo;
    return {hi, lo - (hi - p.hi)};
}
__device__ __forceinline__ Pair warp_add(Pair v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = pair_add(v, Pair{shuffle_xor(v.hi, o), shuffle_xor(v.lo, o)});
    return v;
}


// e^x to about 2^-44 of itself; 0 below -80 and +inf above 88 (2^n is built from
// n's bits).  x = n ln 2 + r with ln 2 in parts whose first n times is exact (Cody
// and Waite's reduction), and the exponential series of r (|r| <= 0.35), whose
// terms from r^7 / 7! on (below 2e-7) are summed in fp32.
__device__ __forceinline__ Pair exp_pair(Pair x) {
    if (!(x.hi > -80.f)) return {x.hi != x.hi ? x.hi : 0.f, 0.f};
    if (x.hi > 88.f) return {HUGE_VALF, 0.f};
    const float n = rintf(x.hi * kLog2E);
    // ln 2 in parts of 11, 24 and 24 bits: n times the first is exact
    constexpr double kLn2Exact = 0.693147180559945309417;
    constexpr float l1 = 0.693359375f, l2 = (float)(kLn2Exact - 0.693359375),
                    l3 = (float)(kLn2Exact - 0.693359375 - (double)l2);
    Pair r = exact_sum(fmaf(-n, l1, x.hi), x.lo);
    const Pair p = exact_product(-n, l2);
    r = pair_add(r, Pair{p.hi, fmaf(-n, l3, p.lo)});
    const float t = r.hi;
    float s = 1.f / 6227020800.f;                      // 1/13!
    s = fmaf(s, t, 1.f / 479001600.f);
    s = fmaf(s, t, 1.f / 39916800.f);
    s = fmaf(s, t, 1.f / 3628800.f);
    s = fmaf(s, t, 1.f / 362880.f);
    s = fmaf(s, t, 1.f / 40320.f);
    s = fmaf(s, t, 1.f / 5040.f);                      // the series from r^7 on, over r^7
    Pair e = {s, 0.f};
    constexpr double k[7] = {1.0, 1.0, 0.5, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720};
#pragma unroll
    for (int i = 6; i >= 0; --i) e = pair_add(pair_multiply(e, r), Pair{(float)k[i], (float)(k[i] - (double)(float)k[i])});
    const float scale = __int_as_float(((int)n + 127) << 23);
    return {e.hi * scale, e.lo * scale};
}

// Bytes of the longest slice of a row of V classes over `blocks` blocks, for
// any alignment of the row.
inline long long slice_bytes(long long V, int element, int blocks) {
    const long long N = 16 / element, all = (N - 1 + V + N - 1) / N;
    return (all + blocks - 1) / blocks * 16;
}

// Blocks per row: as many as the row needs for slices of `fit` bytes (so that
// several blocks share an SM and one loads while another computes), and with
// few rows as many as keep every SM busy on slices of at least `least` bytes.
// 0: the row does not fit slices of `most` bytes.
inline int blocks_per_row(long long T, long long V, int element, long long fit, long long most, long long least) {
    int c = 1;
    while (c < kMaxCluster && slice_bytes(V, element, c) > fit) c *= 2;
    if (slice_bytes(V, element, c) > most) return 0;
    while (c < kMaxCluster && T * c * 2 <= sm_count() && slice_bytes(V, element, 2 * c) >= least) c *= 2;
    return c;
}

// Launch of a kernel over T rows with `blocks` blocks (one cluster) per row,
// as a programmatic dependent launch (see launch_dependent).  The limit on a
// kernel's shared memory belongs to the kernel, not to the call, and calls come
// from any thread: it is set to `most`, the largest `smem` that the kernel is ever
// launched with, and so never below what a launch of another thread needs.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_rows(void (*kernel)(KArgs...), long long T, int blocks, int threads, size_t smem, size_t most,
                               cudaStream_t stream, Args... args) {
    if (smem > 4 * 1024) {   // with the kernels' own arrays perhaps past the 48 KB that need no leave
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(T * blocks));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)blocks;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = blocks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

}  // namespace bitlogic
