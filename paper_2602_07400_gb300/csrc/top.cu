// The record of a row's largest logits: values, classes and log-sum-exp, as a
// teacher hands them to bitlogic_distill_loss.
//
//   order  value descending, class ascending; NaN and -inf do not rank
//   lse    = m / tau + ln sum_v 2^((z_v - m) log2(e) / tau),  m = max z
//
// Bound by reading the logits once: T V bytes_of(type) against 8 T K written.
#include "row_tile.cuh"

namespace bitlogic {
namespace {

constexpr int kTopThreads = 256, kTopWarps = kTopThreads / 32;

struct TopOut {
    int K;
    float inv_tau;
    float* val;
    int* idx;
    float* lse;
};

struct TopScratch {
    SelectScratch select;
    float fbuf[kTopWarps];
    unsigned ubuf[kTopWarps];
    unsigned long long entry[kMaxTop];
    unsigned n_above;
};

// The selection of a row read from memory in every pass, for any row: the
// exact key of the last rank by radix selection, then the classes above it and
// the first ones at it.  Called by the whole block.
template <typename T>
__device__ void top_of_stream(const T* __restrict__ x, int V, const TopOut& o, long long row, TopScratch* s) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = o.K;
    unsigned n = 0;
    for (int v = tid; v < V; v += kTopThreads) n += ranks(logit_key(logit_value(x[v])));
    n = block_add(n, s->ubuf, kTopWarps);
    const unsigned want = min((unsigned)K, n);
    for (int r = tid; r < K; r += kTopThreads)
        if (r >= (int)want) {
            o.val[row * K + r] = BITLOGIC_NEG_INF;
            o.idx[row * K + r] = -1;
        }
    if (want == 0) return;
    unsigned long long above;
    const uint32_t t = select_key([&](int v) { return logit_key(logit_value(x[v])); },
                                  [](int, uint32_t) { return 1ull; }, V, want, &s->select, &above);
    // the classes above t in any order, then the first of those at t by class:
    // every warp takes a contiguous part of the row
    if (tid == 0) s->n_above = 0;
    const int part = (V + kTopWarps - 1) / kTopWarps, v0 = min(V, warp * part), v1 = min(V, v0 + part);
    unsigned eq = 0;
    for (int v = v0 + lane; v < v1; v += 32) eq += logit_key(logit_value(x[v])) == t;
    eq = warp_add(eq);
    __syncthreads();
    if (lane == 0) s->ubuf[warp] = eq;
    __syncthreads();
    unsigned at = (unsigned)above;
    for (int w = 0; w < warp; ++w) at += s->ubuf[w];
    for (int b = v0; b < v1; b += 32) {
        const int v = b + lane;
        const uint32_t k = v < v1 ? logit_key(logit_value(x[v])) : 0u;
        if (v < v1 && k > t) s->entry[atomicAdd(&s->n_above, 1u)] = ((unsigned long long)k << 32) | (uint32_t)~v;
        const bool same = v < v1 && k == t;
        const unsigned mask = __ballot_sync(0xffffffffu, same);
        const unsigned slot = at + __popc(mask & ((1u << lane) - 1u));
        if (same && slot < want) s->entry[slot] = ((unsigned long long)k << 32) | (uint32_t)~v;
        at += __popc(mask);
    }
    __syncthreads();
    if (tid < (int)want) {   // every entry to the place of its rank
        const unsigned long long e = s->entry[tid];
        int r = 0;
        for (unsigned j = 0; j < want; ++j) r += s->entry[j] > e;
        o.val[row * K + r] = key_logit((uint32_t)(e >> 32));
        o.idx[row * K + r] = (int)~(uint32_t)e;
    }
}

// Rows too long for the shared memory of a cluster.
template <typename T>
__global__ void __launch_bounds__(kTopThreads)
top_stream_kernel(const T* __restrict__ X, long long ld, int V, TopOut o) {
    __shared__ TopScratch s;
    grid_dependency_wait();
    const long long row = blockIdx.x;
    const T* x = X + row * ld;
    if (o.lse) {
        float m = BITLOGIC_NEG_INF;
        for (int v = threadIdx.x; v < V; v += kTopThreads) m = fmaxf(m, logit_value(x[v]));
        m = block_largest(m, s.fbuf, kTopWarps);
        const float ms = isinf(m) ? 0.f : m, c = kLog2E * o.inv_tau;
        float sum = 0.f;
        for (int v = threadIdx.x; v < V; v += kTopThreads) sum += exp2_unit((logit_value(x[v]) - ms) * c);
        sum = block_add(sum, s.fbuf, kTopWarps);
        if (threadIdx.x == 0) o.lse[row] = ms * o.inv_tau + logf(sum);
    }
    top_of_stream(x, V, o, row, &s);
}

// Entries (key << 32 | ~class) that a row's selection looks at in the end.
constexpr int kTopList = 1024;

struct TopShared {
    union {
        unsigned long long list[kTopList];   // of the row, in the cluster's first block
        TopScratch scratch;
    };
    union {
        unsigned long long local[kTopList];  // of the slice
        BoundScratch bound;
    };
    struct Stats {
        float m;
        uint32_t bound;
    } stats[kMaxCluster];
    float sums[kMaxCluster];
    float fbuf[kTopWarps];
    unsigned n_list, n_local, base;
};

// A row in the shared memory of one block or one cluster.  Each thread's two
// running maxima give a bound that at least K logits of the row reach: the
// largest key that K / blocks of a block's 512 maxima reach, and the smallest
// of those over the row's blocks.  For logits in no
// particular order little more than K pass it, so the selection sorts a few
// hundred entries; rows on which more than 1024 pass (long runs of equal
// logits, rows sorted by value) are selected from memory.
template <typename T>
__global__ void __launch_bounds__(kTopThreads, 3)
top_tile_kernel(const T* __restrict__ X, long long ld, int V, TopOut o) {
    using P = Piece<T>;
    extern __shared__ __align__(16) unsigned char raw[];
    T* tile = reinterpret_cast<T*>(raw);
    const uint4* tile16 = reinterpret_cast<const uint4*>(raw);
    __shared__ TopShared s;
    grid_dependency_wait();
    allow_dependent_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = o.K;
    const unsigned rank = cluster_rank(), blocks = cluster_size();
    const long long row = blockIdx.x / blocks;
    const T* x = X + row * ld;
    const RowSlice<T> slice(x, V, rank, blocks);
    slice.copy(x, V, tile, tid, kTopThreads);
    if (tid == 0) s.n_list = s.n_local = 0;
    cp_async_wait<0>();
    __syncthreads();

    typename P::Max ma = P::lowest(), mb = P::lowest();
#pragma unroll 4
    for (int j = tid; j < slice.n; j += 2 * kTopThreads) {
        ma = P::largest(ma, tile16[j]);
        if (j + kTopThreads < slice.n) mb = P::largest(mb, tile16[j + kTopThreads]);
    }
    const float za = P::value(ma), zb = P::value(mb);
    const uint32_t bound_here = block_bound(za, zb, (K + blocks - 1) / blocks, &s.bound);
    const float wm = warp_largest(fmaxf(za, zb));
    if (lane == 0) s.fbuf[warp] = wm;
    __syncthreads();
    if (tid < (int)blocks) {
        TopShared::Stats st = {s.fbuf[0], bound_here};
        for (int w = 1; w < kTopWarps; ++w) st.m = fmaxf(st.m, s.fbuf[w]);
        put_in_block(&s.stats[rank], tid, st);
    }
    if (blocks > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    float m = s.stats[0].m;
    uint32_t bound = s.stats[0].bound;
    for (unsigned b = 1; b < blocks; ++b) {
        m = fmaxf(m, s.stats[b].m);
        bound = min(bound, s.stats[b].bound);
    }
    const float ms = isinf(m) ? 0.f : m, c = kLog2E * o.inv_tau, zb_min = bound_logit(bound);

    float s0 = 0.f, s1 = 0.f;
#pragma unroll 2
    for (int j = tid; j < slice.n; j += kTopThreads) {
        const uint4 u = tile16[j];
        float z[P::N];
        P::load(u, z);
        if (o.lse) {
#pragma unroll
            for (int i = 0; i < P::N; i += 2) {
                s0 += exp2_unit((z[i] - ms) * c);
                s1 += exp2_unit((z[i + 1] - ms) * c);
            }
        }
        if (P::largest_of(u) >= zb_min) {
#pragma unroll
            for (int i = 0; i < P::N; ++i)
                if (z[i] >= zb_min && z[i] > BITLOGIC_NEG_INF) {
                    const unsigned at = atomicAdd(&s.n_local, 1u);
                    const int v = slice.first + j * P::N + i;
                    if (at < kTopList) s.local[at] = ((unsigned long long)logit_key(z[i]) << 32) | (uint32_t)~v;
                }
        }
    }
    const float sum = block_add(s0 + s1, s.fbuf, kTopWarps);
    // the slice's entries to the first block
    const unsigned n = min(s.n_local, (unsigned)kTopList);
    if (tid == 0) {
        s.base = add_in_block(&s.n_list, 0, s.n_local);
        store_in_block(&s.sums[rank], 0, __float_as_uint(sum));
    }
    __syncthreads();
    for (unsigned i = tid; i < n; i += kTopThreads)
        if (s.base + i < kTopList) put_in_block(&s.list[s.base + i], 0, s.local[i]);
    if (blocks > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    if (rank != 0) return;

    if (o.lse && tid == 0) {
        float t = 0.f;
        for (unsigned b = 0; b < blocks; ++b) t += s.sums[b];
        o.lse[row] = ms * o.inv_tau + logf(t);
    }
    const unsigned total = s.n_list;
    __syncthreads();
    if (total > kTopList) {
        top_of_stream(x, V, o, row, &s.scratch);
        return;
    }
    if (total <= 256) {
        // every entry to the place of its rank
        const unsigned long long e = tid < (int)total ? s.list[tid] : 0ull;
        unsigned r = 0;
        for (unsigned j = 0; j < total; ++j) r += s.list[j] > e;
        if (tid < (int)total && r < (unsigned)K) {
            o.val[row * K + r] = key_logit((uint32_t)(e >> 32));
            o.idx[row * K + r] = (int)~(uint32_t)e;
        }
    } else {
        const int size = total <= 512 ? 512 : 1024;
        for (int i = total + tid; i < size; i += kTopThreads) s.list[i] = 0ull;
        block_sort_falling(s.list, size);
        if (tid < K) {
            o.val[row * K + tid] = key_logit((uint32_t)(s.list[tid] >> 32));
            o.idx[row * K + tid] = (int)~(uint32_t)s.list[tid];
        }
    }
    if (tid < K && tid >= (int)total) {
        o.val[row * K + tid] = BITLOGIC_NEG_INF;
        o.idx[row * K + tid] = -1;
    }
}

// Rows of few classes: a warp per row, PER keys in the registers of a lane.
constexpr int kNarrow = 1024, kNarrowWarps = 8;

template <typename T, int PER>
__global__ void __launch_bounds__(kNarrowWarps * 32)
top_narrow_kernel(const T* __restrict__ X, long long ld, int V, long long rows, TopOut o) {
    extern __shared__ __align__(16) unsigned char raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, K = o.K;
    unsigned long long* list = reinterpret_cast<unsigned long long*>(raw) + warp * K;
    grid_dependency_wait();
    allow_dependent_launch();
    const long long row = (long long)blockIdx.x * kNarrowWarps + warp;
    if (row >= rows) return;
    const T* x = X + row * ld;
    float z[PER];
    uint32_t key[PER];
    float m = BITLOGIC_NEG_INF;
    unsigned n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int v = i * 32 + lane;
        z[i] = v < V ? logit_value(x[v]) : BITLOGIC_NEG_INF;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        key[i] = logit_key(z[i]);
        m = fmaxf(m, z[i]);
        n += ranks(key[i]);
    }
    if (o.lse) {
        m = warp_largest(m);
        const float ms = isinf(m) ? 0.f : m, c = kLog2E * o.inv_tau;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) s += exp2_unit((z[i] - ms) * c);
        s = warp_add(s);
        if (lane == 0) o.lse[row] = ms * o.inv_tau + logf(s);
    }
    n = __reduce_add_sync(0xffffffffu, n);
    const unsigned want = min((unsigned)K, n);
    for (int r = want + lane; r < K; r += 32) {
        o.val[row * K + r] = BITLOGIC_NEG_INF;
        o.idx[row * K + r] = -1;
    }
    if (want == 0) return;
    // the largest key that `want` reach, a bit at a time; done early where
    // exactly `want` reach it (all that rank: those above -inf)
    uint32_t t = n == want ? kKeyNegInf : 0u;
    unsigned reach = n == want ? want : 0u;
    for (uint32_t bit = 0x80000000u; bit > 0 && reach != want; bit >>= 1) {
        const uint32_t c = t | bit;
        unsigned h = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) h += key[i] >= c;
        h = __reduce_add_sync(0xffffffffu, h);
        if (h >= want) {
            t = c;
            reach = h;
        }
    }
    // those above it, and the first of those at it, by class
    unsigned above = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) above += key[i] > t;
    unsigned ties = want - __reduce_add_sync(0xffffffffu, above), at = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned same = __ballot_sync(0xffffffffu, key[i] == t), below = (1u << lane) - 1u;
        const bool in = key[i] > t || (key[i] == t && __popc(same & below) < ties);
        const unsigned taken = __ballot_sync(0xffffffffu, in);
        if (in && at + __popc(taken & below) < want) list[at + __popc(taken & below)] = ((unsigned long long)key[i] << 32) | (uint32_t)~(i * 32 + lane);
        at += __popc(taken);
        ties -= min(ties, (unsigned)__popc(same));
    }
    __syncwarp();
    for (unsigned a = lane; a < want; a += 32) {   // every entry to the place of its rank
        const unsigned long long e = list[a];
        int r = 0;
        for (unsigned j = 0; j < want; ++j) r += list[j] > e;
        o.val[row * K + r] = key_logit((uint32_t)(e >> 32));
        o.idx[row * K + r] = (int)~(uint32_t)e;
    }
}

// Slices of at most kTileFit bytes leave room for three blocks on an SM.
constexpr int kTileFit = 56 * 1024, kTileMost = 200 * 1024, kTileLeast = 8 * 1024;

template <typename T>
int launch_top(const T* x, long long T_, int V, long long ld, const TopOut& o, cudaStream_t stream) {
    cudaError_t e;
    if (V <= kNarrow) {
        const long long grid = (T_ + kNarrowWarps - 1) / kNarrowWarps;
        const size_t smem = (size_t)kNarrowWarps * o.K * 8;
        auto kern = V <= 32 ? top_narrow_kernel<T, 1> : V <= 128 ? top_narrow_kernel<T, 4>
                  : V <= 256 ? top_narrow_kernel<T, 8> : top_narrow_kernel<T, 32>;
        e = launch_rows(kern, grid, 1, kNarrowWarps * 32, smem, stream, x, ld, V, T_, o);
    } else if (const int blocks = blocks_per_row(T_, V, sizeof(T), kTileFit, kTileMost, kTileLeast)) {
        e = launch_rows(top_tile_kernel<T>, T_, blocks, kTopThreads, (size_t)slice_bytes(V, sizeof(T), blocks), stream,
                        x, ld, V, o);
    } else {
        e = launch_rows(top_stream_kernel<T>, T_, 1, kTopThreads, 0, stream, x, ld, V, o);
    }
    return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

extern "C" int bitlogic_top_logits(const void* X, int32_t dtype, int64_t T, int32_t V, int64_t ld, int32_t K,
                                   float temperature, float* val, int32_t* idx, float* lse, cudaStream_t stream) {
    if (int st = check_logits(X, dtype, true, T, V, ld)) return st;
    if (K < 1 || K > kMaxTop || K > V) return BITLOGIC_ERR_SHAPE;
    if (!(temperature > 0.f) || isinf(temperature)) return BITLOGIC_ERR_HYPER;
    if (T == 0) return BITLOGIC_OK;
    if (!val || !idx) return BITLOGIC_ERR_NULL;
    const TopOut o = {K, 1.0f / temperature, val, idx, lse};
    return with_logit_type(dtype, true, [&](auto* type) {
        return launch_top(static_cast<decltype(type)>(X), T, V, ld, o, stream);
    });
}
