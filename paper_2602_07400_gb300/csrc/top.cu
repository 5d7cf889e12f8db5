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

constexpr int kTopThreads = 256, kTopWarps = kTopThreads / 32;   // at most

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

// ln sum exp of a row that holds +inf: +inf, or NaN with a NaN.
template <typename T>
__device__ float lse_of_inf(const T* x, int V) {
    float s = 0.f;
    for (int v = 0; v < V; ++v) {
        const float z = logit_value(x[v]);
        if (z != z) s = z;
    }
    return s != s ? s : -BITLOGIC_NEG_INF;
}

// The selection of a row read from memory in every pass, for any row: the
// exact key of the last rank by radix selection, then the classes above it and
// the first ones at it.  Called by the whole block.
template <int kThreads, typename T>
__device__ void top_of_stream(const T* __restrict__ x, int V, const TopOut& o, long long row, TopScratch* s) {
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = o.K;
    unsigned n = 0;
    for (int v = tid; v < V; v += kThreads) n += ranks(logit_key(logit_value(x[v])));
    n = block_add(n, s->ubuf, kWarps);
    const unsigned want = min((unsigned)K, n);
    for (int r = tid; r < K; r += kThreads)
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
    const int part = (V + kWarps - 1) / kWarps, v0 = min(V, warp * part), v1 = min(V, v0 + part);
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
    for (unsigned i = tid; i < want; i += kThreads) {   // every entry to the place of its rank
        const unsigned long long e = s->entry[i];
        int r = 0;
        for (unsigned j = 0; j < want; ++j) r += s->entry[j] > e;
        o.val[row * K + r] = key_logit((uint32_t)(e >> 32));
        o.idx[row * K + r] = (int)~(uint32_t)e;
    }
}

// The largest of a sorted or short list to their ranks; the places that no
// class takes are filled.  Called by the whole block; the list has room for
// the next power of two.
template <int kThreads>
__device__ __forceinline__ void write_top(unsigned long long* list, unsigned total, const TopOut& o, long long row) {
    const int tid = threadIdx.x, K = o.K;
    if (total <= 256) {   // every entry to the place of its rank
        for (unsigned i = tid; i < total; i += kThreads) {
            const unsigned long long e = list[i];
            unsigned r = 0;
            for (unsigned j = 0; j < total; ++j) r += list[j] > e;
            if (r < (unsigned)K) {
                o.val[row * K + r] = key_logit((uint32_t)(e >> 32));
                o.idx[row * K + r] = (int)~(uint32_t)e;
            }
        }
    } else {
        const int size = 1 << (32 - __clz(total - 1));
        for (int i = total + tid; i < size; i += kThreads) list[i] = 0ull;
        block_sort_falling(list, size);
        for (int r = tid; r < K; r += kThreads) {
            o.val[row * K + r] = key_logit((uint32_t)(list[r] >> 32));
            o.idx[row * K + r] = (int)~(uint32_t)list[r];
        }
    }
    for (int r = total + tid; r < K; r += kThreads) {
        o.val[row * K + r] = BITLOGIC_NEG_INF;
        o.idx[row * K + r] = -1;
    }
}

constexpr int kRowList = 2048;   // entries of a row

struct TopRowShared {
    union {
        unsigned long long list[kRowList];
        TopScratch scratch;
    };
    BoundScratch bound;
    unsigned short groups[8 * kTopThreads];
    float m[kTopWarps], s[kTopWarps];
    unsigned n, n_groups, inf;
};

// Many rows, of any length: a block per row, which streams it once, keeping
// eight running maxima per thread.  Joined by twos, and in two parts each, the
// 2048 maxima of the row's groups of pieces give a bound that K logits reach, and
// the groups whose maximum reaches it are read again (a sixteenth of a row of 2^17
// bf16 at K = 128; in part from L2: DRAM reads are 1.16 of the logits) for the
// entries: little more than K for logits in no particular order.  A row on which
// more than 2048 pass is selected from memory.  Taking entries
// while streaming, under a bound from the row's beginning that is raised as it
// goes, met four times as many and took 554 us where this takes 221 us
// (4096 x 131072 bf16).
template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
top_row_kernel(const T* __restrict__ X, long long ld, int V, TopOut o) {
    using P = Piece<T>;
    constexpr int N = P::N, H = N / 2, kWarps = kThreads / 32;
    __shared__ TopRowShared s;
    grid_dependency_wait();
    allow_dependent_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = o.K;
    const long long row = blockIdx.x;
    const T* x = X + row * ld;
    const RowSlice<T> slice(x, V, 0, 1);
    const PieceStream<T, kThreads> stream(x, slice, V, tid);
    uint4 ua[4], ub[4];
    stream.load(0, ua);
    stream.load(1, ub);
    if (tid == 0) s.n = s.n_groups = s.inf = 0u;
    __syncthreads();

    // powers about a base of the warp's, which seldom moves
    const float c = kLog2E * o.inv_tau;
    PowerBase base(BITLOGIC_NEG_INF, c);
    f32x2 y0 = 0, y1 = 0;
    typename P::Max mx[8];   // of even and of odd batches
#pragma unroll
    for (int i = 0; i < 8; ++i) mx[i] = P::lowest();
    auto sums = [&](const uint4& u, const auto& power) {
        f32x2 z[H];
        load_pairs<T>(u, z);
#pragma unroll
        for (int i = 0; i < H; i += 2) {
            y0 = add2(y0, power(z[i]));
            y1 = add2(y1, power(z[i + 1]));
        }
    };
    auto add = [&](const uint4 (&u)[4], float top) {   // `top`: of these or more
        if (!base.holds(top)) {
            if (isinf(top) && top > 0.f) {   // the sum is +inf, or NaN
                s.inf = 1u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float z[N];
                    P::load(u[i], z);
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (z[e] != z[e]) y0 = pack2(z[e], z[e]);
                }
                return;
            }
            const PowerBase up(top, c);
            const float f = base.to(up);
            y0 = mul2(y0, pack2(f, f));
            y1 = mul2(y1, pack2(f, f));
            base = up;
        }
        if (base.far) {
            const FarPairs power(base);
#pragma unroll
            for (int i = 0; i < 4; ++i) sums(u[i], power);
        } else {
            const NearPairs power(base);
#pragma unroll
            for (int i = 0; i < 4; ++i) sums(u[i], power);
        }
    };
    auto use = [&](const uint4 (&u)[4], int odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[4 * odd + i] = P::largest(mx[4 * odd + i], u[i]);
        if (o.lse)
            add(u, fmaxf(fmaxf(P::value(mx[4 * odd]), P::value(mx[4 * odd + 1])),
                         fmaxf(P::value(mx[4 * odd + 2]), P::value(mx[4 * odd + 3]))));
    };
    for (int q = 0; q < stream.batches; q += 2) {
        use(ua, 0);
        if (q + 2 < stream.batches) stream.load(q + 2, ua);
        if (q + 1 < stream.batches) use(ub, 1);
        if (q + 3 < stream.batches) stream.load(q + 3, ub);
    }
    // the pieces at the row's ends, of threads 0 and 32
    const int j_end = tid == 0 && slice.whole0() > 0 ? 0 : tid == 32 && slice.whole1(V) < slice.n ? slice.whole1(V) : -1;
    uint4 u_end = masked_piece<T>();
    if (j_end >= 0) {
        u_end = end_piece(x, V, slice.first + j_end * N);
        const uint4 e[4] = {u_end, masked_piece<T>(), masked_piece<T>(), masked_piece<T>()};
        if (o.lse) add(e, fmaxf(base.none ? BITLOGIC_NEG_INF : base.m, P::largest_of(u_end)));
    }

    float part[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) P::parts(P::either(mx[i], mx[4 + i]), part[2 * i], part[2 * i + 1]);
    const float z_min = bound_logit(block_bound(part, K, &s.bound));
    auto take = [&](const uint4& u, int j) {
        if (P::largest_of(u) >= z_min) {
            float z[N];
            P::load(u, z);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (z[i] >= z_min && z[i] > BITLOGIC_NEG_INF) {
                    const unsigned at = atomicAdd(&s.n, 1u);
                    if (at < kRowList) s.list[at] = ((unsigned long long)logit_key(z[i]) << 32) | (uint32_t)~(slice.first + j * N + i);
                }
        }
    };
    if (j_end >= 0) take(u_end, j_end);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float group = P::value(mx[i]);
        if (group >= z_min && group > BITLOGIC_NEG_INF) s.groups[atomicAdd(&s.n_groups, 1u)] = (unsigned short)(8 * tid + i);
    }
    __syncthreads();
    const unsigned half = ((unsigned)stream.batches + 1) / 2, pieces = s.n_groups * half;
    for (unsigned p = tid; p < pieces; p += kThreads) {
        const unsigned which = p / half, g = s.groups[which], q = 2 * (p - which * half) + (g >> 2 & 1u);
        const int j = slice.whole0() + stream.first_of((int)(g >> 3)) + 4 * kThreads * (int)q + 32 * (int)(g & 3u);
        if (j < stream.j1) take(__ldcg(stream.from + j), j);
    }
    if (o.lse) {
        float m = warp_largest(base.none ? BITLOGIC_NEG_INF : base.m), a, b;
        if (lane == 0) s.m[warp] = m;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s.m[w]);
        const PowerBase all(m, c);
        unpack2(add2(y0, y1), a, b);
        const float sum = warp_add((a + b) * base.to(all));
        if (lane == 0) s.s[warp] = sum;
        __syncthreads();
        if (tid == 0) {
            float t = 0.f;
            for (int w = 0; w < kWarps; ++w) t += s.s[w];
            o.lse[row] = t != t ? t : s.inf ? -BITLOGIC_NEG_INF : all.log_of(t, o.inv_tau);
        }
    } else {
        __syncthreads();
    }
    const unsigned total = s.n;
    __syncthreads();
    if (total > kRowList) top_of_stream<kThreads>(x, V, o, row, &s.scratch);
    else write_top<kThreads>(s.list, total, o, row);
}

// Entries (key << 32 | ~class) that a row's selection looks at in the end.
constexpr int kTopList = 1024;

constexpr int kPieces = 1024;    // pieces of a slice that hold an entry

struct TopShared {
    union {
        unsigned long long list[kTopList];   // of the row, in the cluster's first block
        TopScratch scratch;
    };
    union {
        unsigned long long local[kTopList];  // of the slice
        BoundScratch bound;
    };
    unsigned short pieces[kPieces];
    struct Stats {
        float m;
        uint32_t bound;
    } stats[kMaxCluster];
    float sums[kMaxCluster];
    float fbuf[kTopWarps];
    unsigned n_list, n_local, n_pieces, base;
};

// A row in the shared memory of one block or one cluster.  Each thread's two
// running maxima of two parts give a bound that at least K logits of the row
// reach: the largest key that K / blocks of a block's 1024 maxima reach, and the smallest
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
    report_running(blocks);
    slice.copy(x, V, tile, tid, kTopThreads);
    if (tid == 0) s.n_list = s.n_local = s.n_pieces = 0;
    cp_async_wait<0>();
    __syncthreads();

    typename P::Max ma = P::lowest(), mb = P::lowest();
#pragma unroll 4
    for (int j = tid; j < slice.n; j += 2 * kTopThreads) {
        ma = P::largest(ma, tile16[j]);
        if (j + kTopThreads < slice.n) mb = P::largest(mb, tile16[j + kTopThreads]);
    }
    float part[4];
    P::parts(ma, part[0], part[1]);
    P::parts(mb, part[2], part[3]);
    const uint32_t bound_here = block_bound(part, (K + blocks - 1) / blocks, &s.bound);
    const float wm = warp_largest(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    if (lane == 0) s.fbuf[warp] = wm;
    __syncthreads();
    wait_all_running(blocks);
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
    const float c = kLog2E * o.inv_tau, z_min = bound_logit(bound);

    // the powers, and the pieces that hold an entry; their entries after the
    // pass, by threads side by side (a thread that met one in the pass would
    // hold up its warp)
    const PowerBase base(m, c);
    f32x2 y0 = 0, y1 = 0;
    auto pass = [&](const auto& power) {
#pragma unroll 2
        for (int j = tid; j < slice.n; j += kTopThreads) {
            const uint4 u = tile16[j];
            if (o.lse) {
                f32x2 z[P::N / 2];
                load_pairs<T>(u, z);
#pragma unroll
                for (int i = 0; i < P::N / 2; i += 2) {
                    y0 = add2(y0, power(z[i]));
                    y1 = add2(y1, power(z[i + 1]));
                }
            }
            if (P::largest_of(u) >= z_min) {
                const unsigned at = atomicAdd(&s.n_pieces, 1u);
                if (at < kPieces) s.pieces[at] = (unsigned short)j;
            }
        }
    };
    if (base.far) pass(FarPairs(base));
    else pass(NearPairs(base));
    float sum_a, sum_b;
    unpack2(add2(y0, y1), sum_a, sum_b);
    const float sum = block_add(sum_a + sum_b, s.fbuf, kTopWarps);
    const unsigned n_pieces = s.n_pieces;
    if (n_pieces <= kPieces) {
        for (unsigned i = tid; i < n_pieces * P::N; i += kTopThreads) {
            const int p = s.pieces[i / P::N] * P::N + i % P::N;
            const float v = logit_value(tile[p]);
            if (v >= z_min && v > BITLOGIC_NEG_INF) {
                const unsigned at = atomicAdd(&s.n_local, 1u);
                if (at < kTopList) s.local[at] = ((unsigned long long)logit_key(v) << 32) | (uint32_t)~(slice.first + p);
            }
        }
    } else if (tid == 0) {
        s.n_local = kTopList + 1;   // more than the list holds
    }
    __syncthreads();
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
        o.lse[row] = isinf(m) && m > 0.f ? lse_of_inf(x, V) : base.log_of(t, o.inv_tau);
    }
    const unsigned total = s.n_list;
    __syncthreads();
    if (total > kTopList) {
        top_of_stream<kTopThreads>(x, V, o, row, &s.scratch);
        return;
    }
    write_top<kTopThreads>(s.list, total, o, row);
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

// Few rows go by clusters, so that several SMs share one (16 rows of 2^17 bf16
// 10.1 against 16.2 us in a block each, 64 rows 13.5 against 16.5); from half a
// row per SM on a block per row is faster (100 rows 16.6 against 20.6 us, 4096
// rows 220 against 510).  Slices of at most kTileFit bytes leave room for three
// blocks on an SM.
constexpr int kTileFit = 56 * 1024, kTileMost = 200 * 1024, kTileLeast = 8 * 1024;

template <typename T>
int launch_top(const T* x, long long T_, int V, long long ld, const TopOut& o, cudaStream_t stream) {
    cudaError_t e;
    if (V <= kNarrow) {
        const long long grid = (T_ + kNarrowWarps - 1) / kNarrowWarps;
        const size_t smem = (size_t)kNarrowWarps * o.K * 8, most = (size_t)kNarrowWarps * kMaxTop * 8;
        auto kern = V <= 32 ? top_narrow_kernel<T, 1> : V <= 128 ? top_narrow_kernel<T, 4>
                  : V <= 256 ? top_narrow_kernel<T, 8> : V <= 512 ? top_narrow_kernel<T, 16> : top_narrow_kernel<T, 32>;
        e = launch_rows(kern, grid, 1, kNarrowWarps * 32, smem, most, stream, x, ld, V, T_, o);
    } else {
        const int blocks = 2 * T_ <= sm_count() ? blocks_per_row(T_, V, sizeof(T), kTileFit, kTileMost, kTileLeast) : 0;
        if (blocks > 1) {
            e = launch_rows(top_tile_kernel<T>, T_, blocks, kTopThreads, (size_t)slice_bytes(V, sizeof(T), blocks),
                            kTileMost, stream, x, ld, V, o);
        } else {
            // short rows in 128 threads, of which an SM holds more blocks (bf16,
            // 2000 rows: 4096 classes 20.8 against 30.0 us in 256, 16384 classes
            // 35.1 against 36.5, 32768 classes 51.4 against 49.4)
            const bool is_short = V * (long long)sizeof(T) <= 32 * 1024;
            e = launch_rows(is_short ? top_row_kernel<T, 128> : top_row_kernel<T, 256>, T_, 1, is_short ? 128 : 256, 0, 0, stream,
                            x, ld, V, o);
        }
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
    if (!temperature_ok(temperature)) return BITLOGIC_ERR_HYPER;
    if (T == 0) return BITLOGIC_OK;
    if (!val || !idx) return BITLOGIC_ERR_NULL;
    const TopOut o = {K, 1.0f / temperature, val, idx, lse};
    return with_logit_type(dtype, true, [&](auto* type) {
        return launch_top(static_cast<decltype(type)>(X), T, V, ld, o, stream);
    });
}
