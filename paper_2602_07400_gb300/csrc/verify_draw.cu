// The draw behind the accepted drafts: a sequence per block or cluster (verify.cu
// has the mathematics).
//
// Once the refused draft is known, the target's row and the draft's come into the
// shared memory of the sequence's blocks, a slice each, where they are gone over
// three times: the target's weights and the draft's largest logit, the draft's
// weights, and what max(0, p - q) leaves, by chunks of 256 classes; the chunk that
// holds the draw is then looked at class by class.  Bound by instructions and the
// latency between the cluster's barriers: of the 162 us of 256 x 7 drafts over 131072
// bf16 classes 82 are the rows' sums, 14 the slices' copies and 66 the passes, whose
// instructions alone would issue in half of that.  Slices that stay in
// L2 in place of shared memory took 217 us, slices of 32768 classes (a block on an
// SM) 247.
#include "verify.cuh"

namespace bitlogic {
namespace {

// A chunk's logits are held eight to a lane.  Where both rows start on 16 bytes a
// lane's classes are side by side (`along`) and come by vectors; else they lie 32
// apart, so that the lanes of a load are side by side.
__device__ __forceinline__ int place(int q, int lane, int i, bool along) { return q * kChunk + (along ? 8 * lane + i : 32 * i + lane); }

extern __shared__ __align__(16) unsigned char draw_shared[];

// A block's part of a row, classes c0 to c1, in shared memory (kTiled) or where it is.
template <typename T, bool kTiled>
struct Slice {
    static constexpr int N = Piece<T>::N;
    const T* x;      // the row
    int tile;        // of class 0 in the shared memory: its place in values
    int V;
    bool aligned, cut;
    RowRule rule;

    __device__ __forceinline__ Slice(const Rows& rows, long long row, int V_)
        : x(static_cast<const T*>(rows.x) + row * rows.ld), tile(0), V(V_), aligned((reinterpret_cast<uintptr_t>(x) & 15u) == 0),
          rule(rows, row) {
        cut = !(rule.floor == BITLOGIC_NEG_INF);
    }
    __device__ __forceinline__ T* shared() const { return reinterpret_cast<T*>(draw_shared); }
    __device__ __forceinline__ T at(int v) const { return kTiled ? shared()[tile + v] : x[v]; }
    // Copies to `place` bytes into the shared memory; finish with cp_async_wait<0>()
    // and a barrier.
    __device__ __forceinline__ void copy(size_t place, int c0, int c1, int tid) {
        const int shift = (int)((reinterpret_cast<uintptr_t>(x + c0) & 15u) / sizeof(T)), first = c0 - shift;   // class of the first place
        const int n = c1 > c0 ? (shift + c1 - c0 + N - 1) / N : 0;
        const T* from = x + first;   // read at whole pieces only
        tile = (int)(place / sizeof(T)) - first;
        T* to = shared() + place / sizeof(T);
        // pieces [w0, w1) lie in the row in full, at most one before and one after do not
        const int w0 = n > 0 && first < 0 ? 1 : 0, w1 = n > 0 && first + n * N > V ? max(w0, n - 1) : n;
#pragma unroll 4
        for (int j = w0 + tid; j < w1; j += kVerifyThreads) cp_async16(to + j * N, from + j * N);
        if (tid < 2 * N) {
            const int j = tid < N ? 0 : n - 1, v = first + j * N + tid % N;
            if (n > 0 && (j < w0 || j >= w1) && v >= 0 && v < V) to[j * N + tid % N] = x[v];
        }
    }
    // Masks what is not kept of classes c0 to c1 in the tile; copied and with a
    // barrier before and behind.
    __device__ __forceinline__ void mask(int c0, int c1, int tid) const {
        for (int v = c0 + tid; v < c1; v += kVerifyThreads)
            if (!rule.keeps(logit_value(at(v)), v)) shared()[tile + v] = masked_logit<T>();
    }
    // the kept logits of chunk q (what is not kept is masked in a tile already); -inf
    // past the row's end
    __device__ __forceinline__ void load(int q, int lane, bool along, float (&z)[8]) const {
        const bool full = (q + 1) * kChunk <= V;
        if (along && full) {
            const int v0 = q * kChunk + 8 * lane;
            float part[N];
#pragma unroll
            for (int h = 0; h < 8 / N; ++h) {
                if (kTiled) Piece<T>::load(*reinterpret_cast<const uint4*>(shared() + tile + v0 + h * N), part);
                else Piece<T>::load(*reinterpret_cast<const uint4*>(x + v0 + h * N), part);
#pragma unroll
                for (int i = 0; i < N; ++i) z[h * N + i] = part[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int v = place(q, lane, i, along);
                z[i] = v < V ? logit_value(at(v)) : BITLOGIC_NEG_INF;
            }
        }
        if (!kTiled) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = rule.kept(z[i], place(q, lane, i, along));
        }
    }
};

// WeightSum (weights.cuh) of eight weights a lane, the offsets of the floats' bits
// taken off a warp's sum at once.
struct EightSum {
    uint32_t high = 0, low = 0;
    __device__ __forceinline__ void add(f32x2 e) {
        const f32x2 c16 = pack2(16.0f, 16.0f), scale = pack2(kWhole, kWhole), whole = pack2(12582912.0f, 12582912.0f);
        const f32x2 t = add2(e, c16), u = fma2(sub2(e, sub2(t, c16)), scale, whole);
        float a, b;
        unpack2(t, a, b);
        high += __float_as_uint(a) + __float_as_uint(b);
        unpack2(u, a, b);
        low += __float_as_uint(a) + __float_as_uint(b);
    }
    // of the `n` weights of a lane (512 at most)
    __device__ __forceinline__ unsigned long long lane_total(unsigned n) const {
        WeightSum s;
        s.high = high - n * 0x41800000u;
        s.low = low - n * 0x4b400000u;
        return s.total();
    }
    // of the eight of every lane
    __device__ __forceinline__ unsigned long long warp_total() const {
        WeightSum s;
        s.high = __reduce_add_sync(0xffffffffu, high) - 256u * 0x41800000u;
        s.low = __reduce_add_sync(0xffffffffu, low) - 256u * 0x4b400000u;
        return s.total();
    }
};

// The largest of three, NaN where one is.
__device__ __forceinline__ float largest_or_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float warp_largest_or_nan(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = largest_or_nan(v, shuffle_xor(v, o), v);
    return v;
}

// Two powers about m, rounded as RowRule::power rounds one, of logits among which
// there is no NaN.
__device__ __forceinline__ f32x2 two_powers(const RowRule& rule, float a, float b, float m) {
    unpack2(mul2(sub2(pack2(a, b), pack2(m, m)), pack2(rule.slope, rule.slope)), a, b);
    return pack2(exp2_unit(a), exp2_unit(b));
}

struct DrawShared {
    struct Stats {
        unsigned long long mass;
        float m;
        unsigned pad;
    } target[kMaxCluster], nan[kMaxCluster], draft[kMaxCluster], rest[kMaxCluster];
    unsigned long long warp_mass[kVerifyWarps];
    float fbuf[kVerifyWarps];
    int stop, near;                        // of a round, the first draft refused and the first near its bar
    float bar;
    int token;                             // of the draft near its bar
    struct {
        float m;
        int cls, flags;
    } row[kVerifyThreads];                 // of a round's rows
    int chunk;
    unsigned long long before;
};

// The parts of a row joined by as many neighbouring lanes (a power of two of them);
// each gets the result.
__device__ __forceinline__ Part join_parts(const Part& own, int parts, const RowRule& rule) {
    float m = own.m;
    for (int o = parts >> 1; o > 0; o >>= 1) m = fmaxf(m, shuffle_xor(m, o));
    float sum = own.m > BITLOGIC_NEG_INF && !rule.greedy && m <= FLT_MAX ? own.sum * exp2_unit((own.m - m) * rule.slope) : 0.f;
    int cls = own.m == m ? own.cls : INT_MAX, flags = own.flags;
    for (int o = parts >> 1; o > 0; o >>= 1) {
        sum += shuffle_xor(sum, o);
        cls = min(cls, shuffle_xor(cls, o));
        flags |= shuffle_xor(flags, o);
    }
    return {m, sum, cls, flags};
}

// Shared memory behind the chunks' weights: the slices of both rows, of any
// alignment.
__host__ __device__ __forceinline__ size_t tile_offset(int chunks) { return ((size_t)chunks * 8 + 15) / 16 * 16; }
__host__ __device__ __forceinline__ size_t tile_bytes(int chunks, int element) { return (size_t)chunks * kChunk * element + 32; }

template <typename T, typename Q, bool kTiled>
__global__ void __launch_bounds__(kVerifyThreads, 3)
verify_draw_kernel(Rows target, Rows draft, int V, Drafts d, int parts, float error, const Part* __restrict__ sums, Verdict out) {
    unsigned long long* chunks = reinterpret_cast<unsigned long long*>(draw_shared);
    __shared__ DrawShared s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned rank = cluster_rank(), blocks = cluster_size();
    const long long seq = blockIdx.x / blocks;
    // What the call's caller wrote may be read before the wait: the kernel before
    // this one let it start only once its own wait was over.
    const bool writes = rank == 0 && tid == 0;
    Places where;
    if (!where.read(d, seq)) {   // alike in all blocks
        grid_dependency_wait();
        allow_dependent_launch();
        if (writes) {
            flag_index_error();
            out.accepted[seq] = 0;
            out.next_token[seq] = -1;
            if (out.logprob) out.logprob[seq] = BITLOGIC_NEG_INF;
        }
        return;
    }
    report_running(blocks);
    // the drafts before the first that is refused: a row by `parts` lanes, as many as
    // the block has at a time
    const long long first = where.first, k = where.count;
    const int round = kVerifyThreads / parts;
    long long a = k, base = 0;
    bool waited = false;   // for the rows' sums
    for (;; base += round) {
        const long long i = base + tid / parts;   // the row behind the last draft is among them
        float bar = 0.f;
        int v = -1;
        bool near = false;
        if (tid == 0) s.stop = s.near = kVerifyThreads;
        __syncthreads();
        if (base + (tid & ~31) / parts <= k) {    // alike in a warp
            const bool real = i <= k, test = i < k;
            const long long j = first + i, row = first + seq + (real ? i : 0);
            const bool leads = (tid & (parts - 1)) == 0;
            if (parts == 1) {   // decided where the row was read
                if (!waited) grid_dependency_wait();
                const Part p = sums[row];
                if (real) s.row[tid] = {p.m, p.cls, p.flags};
                if (test && (p.flags & kRefused)) atomicMin(&s.stop, tid);
            } else {
                const RowRule rule(target, row);
                v = test ? d.token[j] : -1;
                const bool known = v >= 0 && v < V;
                const float z = known ? kept_logit(target, rule, row, v) : BITLOGIC_NEG_INF, u = test ? d.u[j] : 0.f,
                            q = test && d.logprob ? expf(d.logprob[j]) : 1.f;
                if (!waited) grid_dependency_wait();
                const Part p = join_parts(sums[row * parts + (tid & (parts - 1))], parts, rule);
                if (leads && real) s.row[tid / parts] = {p.m, p.cls, p.flags};
                const float share = share_in(p, rule, z, v);
                bar = bar_of(u, q);
                near = leads && test && known && by_sum(p, rule) && near_bar(bar, share, error);
                if (near) atomicMin(&s.near, tid / parts);
                else if (leads && test && !(known && bar < share)) atomicMin(&s.stop, tid / parts);
            }
            waited = true;
        }
        __syncthreads();
        while (__builtin_expect(s.near < s.stop, 0)) {   // in their order; alike in all blocks
            const int n = s.near;
            if (near && n == tid / parts) {
                s.bar = bar;
                s.token = v;
            }
            __syncthreads();
            const long long border = first + seq + base + n;
            const float share = whole_share(static_cast<const T*>(target.x) + border * target.ld, V, RowRule(target, border), s.row[n].m,
                                            s.token, s.warp_mass);
            if (tid == 0) {
                if (!(s.bar < share)) s.stop = n;
                s.near = kVerifyThreads;
            }
            __syncthreads();
            if (near && tid / parts > n) atomicMin(&s.near, tid / parts);
            __syncthreads();
        }
        if (s.stop < kVerifyThreads) a = base + s.stop;
        if (a < base + round) break;   // refused here, or the last row is here
        __syncthreads();
    }
    if (!waited) grid_dependency_wait();
    allow_dependent_launch();
    const long long row = first + seq + a, j = first + a;
    Slice<T, kTiled> mine_t(target, row, V);
    const Part p = {s.row[a - base].m, 0.f, s.row[a - base].cls, s.row[a - base].flags};
    if (p.flags & kHasNan) mine_t.cut = true;   // a NaN is not kept
    if (writes) {
        out.accepted[seq] = (int)a;
        if (a < k && (d.token[j] < 0 || d.token[j] >= V)) flag_index_error();
    }
    const bool sure = mine_t.rule.greedy || !(p.m > BITLOGIC_NEG_INF) || p.m > FLT_MAX;
    if (sure) {   // one class, or none; alike in all blocks
        if (writes) {
            const bool none = !(p.m > BITLOGIC_NEG_INF);
            out.next_token[seq] = none ? -1 : p.cls;
            if (out.logprob) out.logprob[seq] = none ? BITLOGIC_NEG_INF : 0.f;
        }
        wait_all_running(blocks);
        return;
    }
    const bool refused = a < k;
    Slice<Q, kTiled> mine_q(draft.x && refused ? draft : target, draft.x && refused ? j : row, V);   // not read unless it is the draft's
    Weigher weigh = {mine_t.rule, mine_q.rule, p.m, 0.f, 0.f, 0.f, -1, false};
    if (refused && (!draft.x || mine_q.rule.greedy)) weigh.one = d.token[j];
    bool spread = refused && draft.x && !mine_q.rule.greedy;   // q is over the draft's row

    // the block's chunks of the row, a warp each in turn
    const int all = (V + kChunk - 1) / kChunk, per = (all + (int)blocks - 1) / (int)blocks;
    const int q0 = min(all, (int)rank * per), q1 = min(all, q0 + per);
    const unsigned visits = q0 + warp < q1 ? (unsigned)(q1 - q0 - warp + kVerifyWarps - 1) / kVerifyWarps : 0u;   // of this warp
    auto barrier = [&]() {
        if (blocks > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
    };
    const bool along = mine_t.aligned && (!spread || mine_q.aligned);
    if (kTiled) {
        const int c0 = q0 * kChunk, c1 = min(V, q1 * kChunk);
        mine_t.copy(tile_offset(per), c0, c1, tid);
        if (spread) mine_q.copy(tile_offset(per) + tile_bytes(per, sizeof(T)), c0, c1, tid);
        cp_async_commit();
        cp_async_wait<0>();
        __syncthreads();
        if (mine_t.cut || (spread && mine_q.cut)) {   // alike in all blocks
            if (mine_t.cut) mine_t.mask(c0, c1, tid);
            if (spread && mine_q.cut) mine_q.mask(c0, c1, tid);
            __syncthreads();
        }
    }
    // the sum and the largest over the block's warps to all blocks, and theirs here
    bool met = false;
    auto tell = [&](unsigned long long mass, float top, DrawShared::Stats* to) {
        if (lane == 0) {
            s.warp_mass[warp] = mass;
            s.fbuf[warp] = top;
        }
        __syncthreads();
        if (!met) wait_all_running(blocks);
        met = true;
        if (tid < (int)blocks) {
            DrawShared::Stats own = {0ull, s.fbuf[0], 0u};
            for (int w = 0; w < kVerifyWarps; ++w) {
                own.mass += s.warp_mass[w];
                own.m = largest_or_nan(own.m, s.fbuf[w], s.fbuf[w]);
            }
            put_in_block(to + rank, tid, own);
        }
        barrier();
    };
    // the mass of the blocks before this one, and of all
    auto add_up = [&](const DrawShared::Stats* of, unsigned long long* before) {
        unsigned long long all = 0;
        for (unsigned b = 0; b < blocks; ++b) {
            if (b == rank) *before = all;
            all += of[b].mass;
        }
        return all;
    };
    // the weights of p, or of what is left of it (`rest`), and what they come to told;
    // by chunk where a draw may follow (`by_chunk`)
    using Yes = std::true_type;
    using No = std::false_type;
    auto sum_chunks = [&](auto rest, auto with_draft, auto by_chunk, DrawShared::Stats* to) {
        constexpr bool kRest = decltype(rest)::value, kDraft = decltype(with_draft)::value, kByChunk = decltype(by_chunk)::value;
        unsigned long long mass = 0;
        float top = BITLOGIC_NEG_INF;
        EightSum ws;
        for (int q = q0 + warp; q < q1; q += kVerifyWarps) {
            float z[8], zd[8];
            mine_t.load(q, lane, along, z);
            if (kDraft) mine_q.load(q, lane, along, zd);
            if (kByChunk) ws = EightSum();
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                f32x2 e = two_powers(mine_t.rule, z[i], z[i + 1], weigh.m);
                if (kRest) {
                    float a, b;
                    unpack2(e, a, b);
                    a = __fmul_rn(a, weigh.inv);
                    b = __fmul_rn(b, weigh.inv);
                    if (kDraft) {   // the shares rounded before their difference, as Weigher does
                        float qa, qb;
                        unpack2(two_powers(mine_q.rule, zd[i], zd[i + 1], weigh.dm), qa, qb);
                        e = pack2(fmaxf(__fsub_rn(a, __fmul_rn(qa, weigh.dinv)), 0.f), fmaxf(__fsub_rn(b, __fmul_rn(qb, weigh.dinv)), 0.f));
                    } else {   // q(one) = 1 leaves nothing
                        e = pack2(place(q, lane, i, along) == weigh.one ? 0.f : a, place(q, lane, i + 1, along) == weigh.one ? 0.f : b);
                    }
                }
                ws.add(e);
            }
            if (!kRest && kDraft) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) top = largest_or_nan(top, zd[i], zd[i + 1]);
            }
            if (kByChunk) {
                const unsigned long long w = ws.warp_total();
                if (lane == 0) chunks[q - q0] = w;
                mass += w;
            }
        }
        if (!kByChunk) mass = warp_add(ws.lane_total(8u * visits));
        tell(mass, !kRest && kDraft ? warp_largest_or_nan(top) : top, to);
    };

    // p's own weights, and the draft's largest logit
    if (spread) sum_chunks(No(), Yes(), No(), s.target);
    else if (refused) sum_chunks(No(), No(), No(), s.target);
    else sum_chunks(No(), No(), Yes(), s.target);
    unsigned long long before = 0, mass = add_up(s.target, &before), mine = s.target[rank].mass;
    const unsigned long long whole = mass;
    if (refused) {
        weigh.inv = kWhole / (float)whole;
        auto draft_top = [&](const DrawShared::Stats* of) {
            float t = of[0].m;
            for (unsigned b = 1; b < blocks; ++b) t = largest_or_nan(t, of[b].m, of[b].m);
            return t;
        };
        weigh.dm = draft_top(s.target);
        if (weigh.dm != weigh.dm) {   // a NaN among the draft's logits (only in tiles), which counts nothing
            mine_q.mask(q0 * kChunk, min(V, q1 * kChunk), tid);
            __syncthreads();
            sum_chunks(No(), Yes(), No(), s.nan);
            weigh.dm = draft_top(s.nan);
        }
        if (spread && weigh.dm > FLT_MAX) {   // a draft of +inf: all of q is on the class drawn
            weigh.one = d.token[j];
            spread = false;
        }
        if (spread && weigh.dm > BITLOGIC_NEG_INF) {
            EightSum ws;
            for (int q = q0 + warp; q < q1; q += kVerifyWarps) {
                float zd[8];
                mine_q.load(q, lane, along, zd);
#pragma unroll
                for (int i = 0; i < 8; i += 2) ws.add(two_powers(mine_q.rule, zd[i], zd[i + 1], weigh.dm));
            }
            const unsigned long long sum = warp_add(ws.lane_total(8u * visits));
            tell(sum, 0.f, s.draft);
            unsigned long long unused;
            weigh.dinv = kWhole / (float)add_up(s.draft, &unused);
        }   // a draft without classes: q is 0
        if (spread && !(weigh.dm > BITLOGIC_NEG_INF)) weigh.dm = 0.f;
        weigh.rest = true;
        if (spread) sum_chunks(Yes(), Yes(), Yes(), s.rest);
        else sum_chunks(Yes(), No(), Yes(), s.rest);
        mass = add_up(s.rest, &before);
        mine = s.rest[rank].mass;
        if (mass == 0) {   // p and q differ by less than their roundings
            weigh.rest = false;
            sum_chunks(No(), No(), Yes(), s.draft);   // which every block has read
            mass = add_up(s.draft, &before);
            mine = s.draft[rank].mass;
        }
    }
    const unsigned long long goal = share_of(mass, unit_of(d.draw_u[seq]));
    if (goal < before || goal >= before + mine) return;   // another block's

    // the chunk that holds the draw: a run of chunks per thread
    const int n = q1 - q0, run = (n + kVerifyThreads - 1) / kVerifyThreads;
    const int i0 = min(n, tid * run), i1 = min(n, i0 + run);
    unsigned long long own = 0;
    for (int i = i0; i < i1; ++i) own += chunks[i];
    const unsigned long long upto = lanes_upto(own, lane);
    __syncthreads();
    if (lane == 31) s.warp_mass[warp] = upto;
    __syncthreads();
    unsigned long long at = before + upto - own;
    for (int w = 0; w < warp; ++w) at += s.warp_mass[w];
    if (goal >= at && goal < at + own) {
        int i = i0;
        while (goal >= at + chunks[i]) at += chunks[i++];
        s.chunk = q0 + i;
        s.before = at;
    }
    __syncthreads();
    if (warp != 0) return;
    // side by side, so that lanes follow the order of classes
    const int q = s.chunk, v0 = q * kChunk + 8 * lane;
    float z[8], zd[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        z[i] = v0 + i < V ? mine_t.rule.kept(logit_value(mine_t.at(v0 + i)), v0 + i) : BITLOGIC_NEG_INF;
        zd[i] = weigh.rest && spread && v0 + i < V ? mine_q.rule.kept(logit_value(mine_q.at(v0 + i)), v0 + i) : BITLOGIC_NEG_INF;
    }
    unsigned long long w[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = draw_weight(weigh(z[i], zd[i], v0 + i));
        sum += w[i];
    }
    unsigned long long at_lane = s.before + lanes_upto(sum, lane) - sum;
    if (goal < at_lane || goal >= at_lane + sum) return;
    bool found = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        at_lane += w[i];
        if (!found && at_lane > goal) {
            found = true;
            out.next_token[seq] = v0 + i;
            if (out.logprob) out.logprob[seq] = logf((float)draw_weight(mine_t.rule.power(z[i], p.m)) / (float)whole);
        }
    }
}

constexpr size_t kDrawShared = 200 * 1024;

// Blocks of a sequence's draw: slices of 16384 classes at most (64 KB of two bf16
// rows, three blocks on an SM), and with few sequences as many as run at once, of at
// least 2048.
struct DrawShape {
    int blocks, chunks;   // of a sequence, of a block
    size_t bytes;         // of both slices in shared memory, with the chunks' weights
};
inline DrawShape draw_shape(int64_t S, int V, int element, int draft_element) {
    auto with = [&](int blocks) {
        const int all = (V + kChunk - 1) / kChunk, per = (all + blocks - 1) / blocks;
        return DrawShape{blocks, per, tile_offset(per) + tile_bytes(per, element) + (draft_element ? tile_bytes(per, draft_element) : 0)};
    };
    auto at_once = [](const DrawShape& s) {
        const long long per = 227 * 1024 / (long long)(s.bytes + 6 * 1024);
        return (per < 1 ? 1 : per > 3 ? 3 : per) * sm_count();
    };
    DrawShape s = with(1);
    while (s.blocks < kMaxCluster) {
        const DrawShape more = with(2 * s.blocks);
        if (V / s.blocks <= 16384 && (S * more.blocks > at_once(more) || V / more.blocks < 2048)) break;
        s = more;
    }
    return s;
}

template <typename T, typename Q>
cudaError_t launch_draw(const Rows& target, const Rows& draft, int V, const Drafts& d, int parts, float error, const Part* sums,
                        const Verdict& out, cudaStream_t stream) {
    const DrawShape s = draw_shape(d.S, V, sizeof(T), draft.x ? sizeof(Q) : 0);
    const bool tiled = s.bytes <= kDrawShared;
    return launch_rows(tiled ? verify_draw_kernel<T, Q, true> : verify_draw_kernel<T, Q, false>, d.S, s.blocks, kVerifyThreads,
                       tiled ? s.bytes : (size_t)s.chunks * 8, kDrawShared, stream, target, draft, V, d, parts, error, sums, out);
}

template <typename T>
cudaError_t launch_draw_of(const Rows& target, const Rows& draft, int V, const Drafts& d, int parts, float error, const Part* sums,
                           const Verdict& out, cudaStream_t stream) {
    if (!draft.x) return launch_draw<T, T>(target, draft, V, d, parts, error, sums, out, stream);
    switch (draft.dtype) {
        case BITLOGIC_F32: return launch_draw<T, float>(target, draft, V, d, parts, error, sums, out, stream);
        case BITLOGIC_BF16: return launch_draw<T, __nv_bfloat16>(target, draft, V, d, parts, error, sums, out, stream);
        case BITLOGIC_F16: return launch_draw<T, __half>(target, draft, V, d, parts, error, sums, out, stream);
        default: return launch_draw<T, int>(target, draft, V, d, parts, error, sums, out, stream);
    }
}

}  // namespace

cudaError_t launch_verify_draw(const Rows& target, const Rows& draft, int V, const Drafts& d, int parts, float error, const Part* sums,
                               const Verdict& out, cudaStream_t stream) {
    switch (target.dtype) {
        case BITLOGIC_F32: return launch_draw_of<float>(target, draft, V, d, parts, error, sums, out, stream);
        case BITLOGIC_BF16: return launch_draw_of<__nv_bfloat16>(target, draft, V, d, parts, error, sums, out, stream);
        case BITLOGIC_F16: return launch_draw_of<__half>(target, draft, V, d, parts, error, sums, out, stream);
        default: return launch_draw_of<int>(target, draft, V, d, parts, error, sums, out, stream);
    }
}

}  // namespace bitlogic

using namespace bitlogic;

BITLOGIC_ERROR_READER(verify_draw)
