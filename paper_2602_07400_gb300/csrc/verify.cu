// Drafted classes accepted or rejected by a target's logits and given random
// numbers, and the class that follows the accepted ones (include/bitlogic.h).
//
//   p = softmax of the target's kept logits / temperature, q of the draft's
//   draft i is accepted iff u_i q(d_i) < p(d_i), up to the first that is not;
//   the next class: from max(0, p - q) of the row that refused, by class, or
//   from p of the last row when none did
//
// so that every class that goes out is distributed as p.  q(d_i) comes from the
// draft's draw, so of the draft's logits only the refused row is read; the
// target's rows are read once.  Bound by that reading.
//
//   verify_sums_kernel    a row (or, where rows are few, a part of one) per
//                         block: its largest logit and the sum of its powers
//                         about it, in one pass: every thread keeps a running
//                         maximum and rescales its sum when that rises
//   verify_draw_kernel    a sequence per block or cluster: the accepted drafts
//                         from the rows' sums, then the draw in whole-number
//                         weights, whose sums are exact in any order
//   verify_narrow_kernel  both for few classes: a sequence per warp, a row in
//                         its registers, from the first draft to the refused one
#include <cfloat>

#include "row_tile.cuh"
#include "weights.cuh"

namespace bitlogic {
namespace {

constexpr int kVerifyThreads = 256, kVerifyWarps = kVerifyThreads / 32;
constexpr int kMaxParts = 32;
constexpr int kVerifyNarrow = 1024;   // classes of a row in a warp's registers
constexpr int kChunk = 256;           // classes whose weights are summed together
constexpr float kWhole = 1099511627776.0f;   // 2^40

// A matrix of logits with the settings of its rows.
struct Rows {
    const void* x;
    int dtype;
    long long ld;
    const float* temperature;
    const float* floor;   // kept: z > floor, or z == floor up to class `last`
    const int* last;
};
struct Drafts {
    const int* first;        // [S + 1]
    const int* token;        // [D]
    const float* logprob;    // [D] or NULL: 0
    const float* u;          // [D]
    const float* draw_u;     // [S]
    long long S, D;
};
struct Verdict {
    int* accepted;
    int* next_token;
    float* logprob;
};

// The largest kept logit of a part of a row, the sum of the powers about it, and
// the first class of that logit (in greedy rows and where it is +inf).
struct Part {
    float m, sum;
    int cls, pad;
};

struct RowRule {
    float slope, floor;
    int last;
    bool greedy;
    __device__ __forceinline__ RowRule(const Rows& r, long long row) {
        const float temp = r.temperature ? r.temperature[row] : 1.0f;
        greedy = !(temp > 0.f);
        slope = greedy ? 0.f : fminf((1.0f / temp) * kLog2E, FLT_MAX);
        floor = r.floor ? r.floor[row] : BITLOGIC_NEG_INF;
        last = r.last ? r.last[row] : -1;
    }
    __device__ __forceinline__ bool keeps(float z, int v) const { return z > floor || (z == floor && v <= last); }
    __device__ __forceinline__ float kept(float z, int v) const { return keeps(z, v) ? z : BITLOGIC_NEG_INF; }
    // e of a kept logit about m; 0 for -inf and NaN
    __device__ __forceinline__ float power(float z, float m) const { return fmaxf(exp2_unit((z - m) * slope), 0.f); }
};

// u as the tests use it: 24 bits in [0, 1), NaN reads 0.
__device__ __forceinline__ float unit_of(float u) { return u > 0.f ? floorf(fminf(u, 0.99999994f) * 16777216.0f) * 5.9604645e-08f : 0.f; }

__device__ __forceinline__ bool passes(float u, float q, float p) { return unit_of(u) * q < p; }

// The sum of v over the lanes below this one and itself.
__device__ __forceinline__ unsigned long long lanes_upto(unsigned long long v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// ------------------------------------------------------------ rows' sums --

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, 4)
verify_sums_kernel(Rows rows, int V, Drafts d, int parts, Part* __restrict__ out) {
    using P = Piece<T>;
    constexpr int N = P::N, H = N / 2;
    __shared__ Part s[kVerifyWarps];
    grid_dependency_wait();
    allow_dependent_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = blockIdx.x / (unsigned)parts;
    if (row >= (long long)d.first[d.S] + d.S) return;   // behind the last sequence
    const T* x = static_cast<const T*>(rows.x) + row * rows.ld;
    const RowSlice<T> slice(x, V, blockIdx.x % (unsigned)parts, (unsigned)parts);
    const PieceStream<T, kVerifyThreads> stream(x, slice, V, tid);
    uint4 ua[4], ub[4];
    stream.load(0, ua);
    stream.load(1, ub);
    const RowRule rule(rows, row);
    // every batch of the slice to `use`, of which the first two are loaded
    auto stream_row = [&](auto&& use) {
        for (int q = 0; q < stream.batches; q += 2) {
            use(ua, q);
            if (q + 2 < stream.batches) stream.load(q + 2, ua);
            if (q + 1 < stream.batches) use(ub, q + 1);
            if (q + 3 < stream.batches) stream.load(q + 3, ub);
        }
    };
    // the pieces at the slice's ends that reach over the row's, of threads 0 and 32
    const int j_end = tid == 0 && slice.whole0() > 0 ? 0 : tid == 32 && slice.whole1(V) < slice.n ? slice.whole1(V) : -1;
    const uint4 u_end = j_end >= 0 ? end_piece(x, V, slice.first + j_end * N) : masked_piece<T>();

    float m = BITLOGIC_NEG_INF, sum = 0.f;
    int cls = INT_MAX;
    // the first class of the largest kept logit
    auto first_largest = [&](const uint4& u, int j) {
        if (!(P::largest_of(u) >= fmaxf(m, rule.floor))) return;
        float z[N];
        P::load(u, z);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int v = slice.first + j * N + i;
            if ((z[i] > m || (z[i] == m && v < cls)) && z[i] > BITLOGIC_NEG_INF && rule.keeps(z[i], v)) {
                m = z[i];
                cls = v;
            }
        }
    };
    auto largest_class = [&]() {
        stream_row([&](const uint4 (&u)[4], int q) {
#pragma unroll
            for (int i = 0; i < 4; ++i) first_largest(u[i], stream.piece(q, i));
        });
        if (j_end >= 0) first_largest(u_end, j_end);
    };
    auto rise = [&](float to) {
        if (to > m) {
            sum = m > BITLOGIC_NEG_INF ? sum * exp2_unit((m - to) * rule.slope) : 0.f;
            m = to;
        }
    };
    auto add = [&](const f32x2 (&z)[H], f32x2 acc) {
        const f32x2 mm = pack2(m, m), cc = pack2(rule.slope, rule.slope);
#pragma unroll
        for (int i = 0; i < H; ++i) {
            float a, b;
            unpack2(mul2(sub2(z[i], mm), cc), a, b);
            acc = add2(acc, pack2(exp2_unit(a), exp2_unit(b)));
        }
        return acc;
    };
    auto add_kept = [&](const uint4& u, int j) {
        if (P::largest_of(u) < rule.floor) return;
        float z[N], top = BITLOGIC_NEG_INF;
        P::load(u, z);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            z[i] = rule.kept(z[i], slice.first + j * N + i);
            top = fmaxf(top, z[i]);
        }
        if (top == BITLOGIC_NEG_INF) return;
        rise(top);
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) part += rule.power(z[i], m);
        sum += part;
    };

    auto sum_kept = [&]() {
        stream_row([&](const uint4 (&u)[4], int q) {
#pragma unroll
            for (int i = 0; i < 4; ++i) add_kept(u[i], stream.piece(q, i));
        });
        if (j_end >= 0) add_kept(u_end, j_end);
    };
    if (rule.greedy) {
        largest_class();
    } else if (rule.floor > BITLOGIC_NEG_INF || rule.floor != rule.floor) {
        sum_kept();
    } else {
        stream_row([&](const uint4 (&u)[4], int) {
            typename P::Max top = P::lowest();
#pragma unroll
            for (int i = 0; i < 4; ++i) top = P::largest(top, u[i]);
            const float t = P::value(top);
            if (!(t > BITLOGIC_NEG_INF)) return;
            rise(t);
            f32x2 acc = pack2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 z[H];
                load_pairs<T>(u[i], z);
                acc = add(z, acc);
            }
            float a, b;
            unpack2(acc, a, b);
            sum += a + b;
        });
        if (j_end >= 0) add_kept(u_end, j_end);
    }
    // over the block
    auto join = [&](float m2, float s2, int c2) {
        const float to = fmaxf(m, m2);
        cls = m2 > m ? c2 : m2 == m ? min(cls, c2) : cls;
        const float mine = m == to ? sum : sum * exp2_unit((m - to) * rule.slope);   // not of two infinities
        const float other = m2 == to ? s2 : s2 * exp2_unit((m2 - to) * rule.slope);
        sum = mine + other;
        m = to;
    };
    auto join_block = [&]() {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float m2 = shuffle_xor(m, o), s2 = shuffle_xor(sum, o);
            const int c2 = shuffle_xor(cls, o);
            join(m2, s2, c2);
        }
        __syncthreads();
        if (lane == 0) s[warp] = {m, sum, cls, 0};
        __syncthreads();
        m = s[0].m;
        sum = s[0].sum;
        cls = s[0].cls;
#pragma unroll
        for (int w = 1; w < kVerifyWarps; ++w) join(s[w].m, s[w].sum, s[w].cls);
    };
    join_block();
    if (sum != sum && !(m > FLT_MAX)) {   // a NaN among the logits, which counts nothing
        m = BITLOGIC_NEG_INF;
        sum = 0.f;
        stream.load(0, ua);
        stream.load(1, ub);
        sum_kept();
        join_block();
    }
    if (!rule.greedy && m > FLT_MAX) {   // the first of +inf takes it all
        m = BITLOGIC_NEG_INF;
        cls = INT_MAX;
        stream.load(0, ua);
        stream.load(1, ub);
        largest_class();
        join_block();
    }
    if (tid == 0) out[blockIdx.x] = {m, sum, cls, 0};
}

// ------------------------------------------------------------------- draw --

// A row of any type, its kept logits eight at a time: 32 lanes' eights make a
// chunk.  Where the row starts on 16 bytes a lane's eight classes are side by
// side (`along`), two loads at most; else they lie 32 apart, so that the lanes of
// a load are side by side.  Loads come before conversions, so that a warp has
// many on their way.
struct Raw {
    uint32_t w[8];
};

struct RowReader {
    const unsigned char* x;
    int dtype, V;
    bool wide, aligned, cut;
    RowRule rule;
    __device__ __forceinline__ RowReader(const Rows& rows, long long row, int V_)
        : dtype(rows.dtype), V(V_), wide(rows.dtype == BITLOGIC_F32 || rows.dtype == BITLOGIC_I32), rule(rows, row) {
        x = static_cast<const unsigned char*>(rows.x) + row * rows.ld * (wide ? 4 : 2);
        aligned = (reinterpret_cast<uintptr_t>(x) & 15u) == 0;
        cut = !(rule.floor == BITLOGIC_NEG_INF);
    }
    __device__ __forceinline__ float at(int v) const {
        float z;
        switch (dtype) {
            case BITLOGIC_F32: z = reinterpret_cast<const float*>(x)[v]; break;
            case BITLOGIC_BF16: z = logit_value(reinterpret_cast<const __nv_bfloat16*>(x)[v]); break;
            case BITLOGIC_F16: z = logit_value(reinterpret_cast<const __half*>(x)[v]); break;
            default: z = logit_value(reinterpret_cast<const int*>(x)[v]); break;
        }
        return rule.kept(z, v);
    }
    static __device__ __forceinline__ int place(int q, int lane, int i, bool along) { return q * kChunk + (along ? 8 * lane + i : 32 * i + lane); }
    __device__ __forceinline__ bool full(int q) const { return (q + 1) * kChunk <= V; }
    __device__ __forceinline__ Raw load(int q, int lane, bool along) const {
        Raw r;
        if (along && aligned && full(q)) {
            const uint4* p = reinterpret_cast<const uint4*>(x + (size_t)(q * kChunk + 8 * lane) * (wide ? 4 : 2));
            const uint4 a = p[0];
            if (wide) {
                const uint4 b = p[1];
                r = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
            } else {
                r = {{a.x, a.y, a.z, a.w, 0u, 0u, 0u, 0u}};
            }
        } else if (wide) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int v = place(q, lane, i, along);
                r.w[i] = v < V ? reinterpret_cast<const uint32_t*>(x)[v] : 0u;
            }
        } else {
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int v = place(q, lane, i, along);
                h[i] = v < V ? reinterpret_cast<const unsigned short*>(x)[v] : 0u;
            }
            r = {{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16, 0u, 0u, 0u, 0u}};
        }
        return r;
    }
    // their values; -inf for what is not kept
    __device__ __forceinline__ void kept(const Raw& r, int q, int lane, bool along, float (&z)[8]) const {
        const uint4 a = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]), b = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
        float h[4];
        if (dtype == BITLOGIC_BF16) {
            Piece<__nv_bfloat16>::load(a, z);
        } else if (dtype == BITLOGIC_F16) {
            Piece<__half>::load(a, z);
        } else if (dtype == BITLOGIC_F32) {
            Piece<float>::load(a, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = h[i];
            Piece<float>::load(b, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 + i] = h[i];
        } else {
            Piece<int>::load(a, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = h[i];
            Piece<int>::load(b, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 + i] = h[i];
        }
        if (cut || !full(q)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int v = place(q, lane, i, along);
                z[i] = v < V ? rule.kept(z[i], v) : BITLOGIC_NEG_INF;
            }
        }
    }
};

// What a row of the target and the draft refused there leave for the draw.
struct Weigher {
    RowRule target, draft;
    float m, inv, dm, dinv;   // largest logits, and 2^40 / the sum of the weights
    int one;                  // the class that q has all of, or -1
    bool rest;                // max(0, p - q), or p's own weights

    __device__ __forceinline__ float operator()(float z, float zd, int v) const {
        const float e = target.power(z, m);
        if (!rest) return e;
        // no multiply-add: the differences are those of the rounded shares
        const float p = __fmul_rn(e, inv), q = one >= 0 ? (v == one ? 1.f : 0.f) : __fmul_rn(draft.power(zd, dm), dinv);
        return fmaxf(__fsub_rn(p, q), 0.f);
    }
    // two powers about m, rounded as power() rounds one
    static __device__ __forceinline__ f32x2 powers(const RowRule& rule, float a, float b, float m) {
        unpack2(mul2(sub2(pack2(a, b), pack2(m, m)), pack2(rule.slope, rule.slope)), a, b);
        return pack2(fmaxf(exp2_unit(a), 0.f), fmaxf(exp2_unit(b), 0.f));
    }
    // The weights of a lane's eight logits of chunk q; q(one) = 1 leaves nothing.
    __device__ __forceinline__ WeightSum eight(const float (&z)[8], const float (&zd)[8], bool spread, int q, int lane,
                                               bool along) const {
        WeightSum ws;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            f32x2 e = powers(target, z[i], z[i + 1], m);
            if (rest) {
                e = mul2(e, pack2(inv, inv));
                if (spread) {
                    e = sub2(e, mul2(powers(draft, zd[i], zd[i + 1], dm), pack2(dinv, dinv)));
                    float a, b;
                    unpack2(e, a, b);
                    e = pack2(fmaxf(a, 0.f), fmaxf(b, 0.f));
                } else if (one >= 0 && q == one / kChunk) {
                    float a, b;
                    unpack2(e, a, b);
                    const int v0 = RowReader::place(q, lane, i, along), v1 = RowReader::place(q, lane, i + 1, along);
                    e = pack2(v0 == one ? 0.f : a, v1 == one ? 0.f : b);
                }
            }
            ws.add(e);
        }
        return ws;
    }
};

struct DrawShared {
    struct Stats {
        unsigned long long mass;
        float m;
        unsigned pad;
    } target[kMaxCluster], draft[kMaxCluster];
    struct Mass {
        unsigned long long mass;
    } rest[kMaxCluster];
    unsigned long long warp_mass[kVerifyWarps];
    float fbuf[kVerifyWarps];
    int refused[kVerifyWarps];
    int chunk;
    unsigned long long before;
};

// The parts of a row joined, in order, by a warp; every lane gets the result.
__device__ __forceinline__ Part join_parts(const Part* parts, int n, const RowRule& rule, int lane) {
    Part p = {BITLOGIC_NEG_INF, 0.f, INT_MAX, 0};
    if (lane < n) p = parts[lane];
    const float m = warp_largest(p.m);
    float sum = p.m > BITLOGIC_NEG_INF && !rule.greedy && m <= FLT_MAX ? p.sum * exp2_unit((p.m - m) * rule.slope) : 0.f;
    sum = warp_add(sum);
    const int cls = (int)__reduce_min_sync(0xffffffffu, p.m == m ? (unsigned)p.cls : (unsigned)INT_MAX);
    return {m, sum, cls, 0};
}

// The target's probability of class v.
__device__ __forceinline__ float share_in(const Part& p, const RowRule& rule, float z, int v) {
    if (!(p.m > BITLOGIC_NEG_INF)) return 0.f;
    if (rule.greedy || p.m > FLT_MAX) return v == p.cls ? 1.f : 0.f;
    return rule.power(z, p.m) / p.sum;
}

__global__ void __launch_bounds__(kVerifyThreads, 3)
verify_draw_kernel(Rows target, Rows draft, int V, Drafts d, int parts, const Part* __restrict__ sums, Verdict out) {
    extern __shared__ __align__(16) unsigned char raw[];
    unsigned long long* chunks = reinterpret_cast<unsigned long long*>(raw);
    __shared__ DrawShared s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned rank = cluster_rank(), blocks = cluster_size();
    const long long seq = blockIdx.x / blocks;
    // What the call's caller wrote may be read before the wait: the kernel before
    // this one let it start only once its own wait was over.
    const long long first = d.first[seq], end = d.first[seq + 1];
    const bool writes = rank == 0 && tid == 0;
    if (first < 0 || end < first || end > d.D || end > d.first[d.S]) {   // alike in all blocks
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
    // the drafts before the first that is refused, a warp each
    const long long k = end - first;
    long long a = 0;
    bool waited = false;   // for the rows' sums
    for (; a < k; a += kVerifyWarps) {
        const long long i = a + warp;
        bool refuse = false;
        if (i < k) {
            const long long j = first + i, row = j + seq;
            const RowReader reader(target, row, V);
            const int v = d.token[j];
            const bool known = v >= 0 && v < V;
            if (!known && rank == 0 && lane == 0) flag_index_error();
            const float z = known ? reader.at(v) : BITLOGIC_NEG_INF, u = d.u[j], q = d.logprob ? expf(d.logprob[j]) : 1.f;
            if (!waited) grid_dependency_wait();
            waited = true;
            const Part p = join_parts(sums + row * parts, parts, reader.rule, lane);
            refuse = !(known && passes(u, q, share_in(p, reader.rule, z, v)));
        }
        if (lane == 0) s.refused[warp] = refuse;
        __syncthreads();
        int w = 0;
        while (w < kVerifyWarps && !s.refused[w]) ++w;
        __syncthreads();
        if (w < kVerifyWarps) {
            a += w;
            break;
        }
    }
    if (!waited) grid_dependency_wait();
    allow_dependent_launch();
    a = a < k ? a : k;
    const long long row = first + seq + a, j = first + a;
    const RowReader reader(target, row, V);
    const Part p = join_parts(sums + row * parts, parts, reader.rule, lane);
    if (writes) out.accepted[seq] = (int)a;
    const bool sure = reader.rule.greedy || !(p.m > BITLOGIC_NEG_INF) || p.m > FLT_MAX;
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
    const RowReader other(draft.x && refused ? draft : target, draft.x && refused ? j : row, V);
    Weigher weigh = {reader.rule, other.rule, p.m, 0.f, 0.f, 0.f, -1, false};
    if (refused && (!draft.x || other.rule.greedy)) weigh.one = d.token[j];
    bool spread = refused && draft.x && !other.rule.greedy;   // q is over the draft's row

    // the block's chunks of the row, a warp each in turn
    const int all = (V + kChunk - 1) / kChunk, per = (all + (int)blocks - 1) / (int)blocks;
    const int q0 = min(all, (int)rank * per), q1 = min(all, q0 + per);
    auto barrier = [&]() {
        if (blocks > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
    };
    // two chunks of a warp at a time to `use`, of the target where `with_target` and
    // of the draft where `with_draft`; what is not read is masked
    const bool along = reader.aligned && (!spread || other.aligned);
    auto each_chunk = [&](bool with_target, bool with_draft, auto&& use) {
        for (int q = q0 + warp; q < q1; q += 2 * kVerifyWarps) {
            const int q2 = q + kVerifyWarps;
            const bool two = q2 < q1;
            Raw a0, a1, b0, b1;
            if (with_target) a0 = reader.load(q, lane, along);
            if (with_draft) b0 = other.load(q, lane, along);
            if (with_target && two) a1 = reader.load(q2, lane, along);
            if (with_draft && two) b1 = other.load(q2, lane, along);
            float z[8], zd[8];
            if (with_target) reader.kept(a0, q, lane, along, z);
            if (with_draft) other.kept(b0, q, lane, along, zd);
            use(q, z, zd);
            if (two) {
                if (with_target) reader.kept(a1, q2, lane, along, z);
                if (with_draft) other.kept(b1, q2, lane, along, zd);
                use(q2, z, zd);
            }
        }
    };
    // the chunks' weights into `chunks`; every thread gets the block's sum
    auto sum_chunks = [&](bool with_draft, float* draft_top) {
        unsigned long long mass = 0;
        float top = BITLOGIC_NEG_INF;
        each_chunk(true, with_draft, [&](int q, const float (&z)[8], const float (&zd)[8]) {
            const WeightSum ws = weigh.eight(z, zd, with_draft, q, lane, along);
            if (draft_top && with_draft) {
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, zd[i]);
            }
            const unsigned long long w = ws.warp_total();
            if (lane == 0) chunks[q - q0] = w;
            mass += w;
        });
        if (draft_top) *draft_top = block_largest(top, s.fbuf, kVerifyWarps);
        __syncthreads();
        if (lane == 0) s.warp_mass[warp] = mass;
        __syncthreads();
        unsigned long long t = 0;
        for (int w = 0; w < kVerifyWarps; ++w) t += s.warp_mass[w];
        return t;
    };

    // p's own weights, and the draft's largest logit
    float top = BITLOGIC_NEG_INF;
    unsigned long long mine = sum_chunks(spread, &top);
    wait_all_running(blocks);
    if (tid < (int)blocks) put_in_block(&s.target[rank], tid, DrawShared::Stats{mine, top, 0u});
    barrier();
    unsigned long long mass = 0, before = 0;
    for (unsigned b = 0; b < blocks; ++b) {
        if (b == rank) before = mass;
        mass += s.target[b].mass;
        weigh.dm = b == 0 ? s.target[b].m : fmaxf(weigh.dm, s.target[b].m);
    }
    const unsigned long long whole = mass;
    if (refused) {
        weigh.inv = kWhole / (float)whole;
        if (spread && weigh.dm > FLT_MAX) {   // a draft of +inf: all of q is on the class drawn
            weigh.one = d.token[j];
            spread = false;
        }
        if (spread && weigh.dm > BITLOGIC_NEG_INF) {
            unsigned long long sum = 0;
            each_chunk(false, true, [&](int, const float (&)[8], const float (&zd)[8]) {
                WeightSum ws;
#pragma unroll
                for (int i = 0; i < 8; i += 2)
                    ws.add(Weigher::powers(weigh.draft, zd[i], zd[i + 1], weigh.dm));
                sum += ws.total();
            });
            sum = block_add(sum, s.warp_mass, kVerifyWarps);
            if (tid < (int)blocks) put_in_block(&s.draft[rank], tid, DrawShared::Stats{sum, 0.f, 0u});
            barrier();
            unsigned long long t = 0;
            for (unsigned b = 0; b < blocks; ++b) t += s.draft[b].mass;
            weigh.dinv = kWhole / (float)t;
        }   // a draft without classes: q is 0
        if (spread && !(weigh.dm > BITLOGIC_NEG_INF)) weigh.dm = 0.f;
        weigh.rest = true;
        mine = sum_chunks(spread, nullptr);
        if (tid < (int)blocks) put_in_block(&s.rest[rank], tid, DrawShared::Mass{mine});
        barrier();
        mass = before = 0;
        for (unsigned b = 0; b < blocks; ++b) {
            if (b == rank) before = mass;
            mass += s.rest[b].mass;
        }
        if (mass == 0) {   // p and q differ by less than their roundings
            weigh.rest = false;
            mine = sum_chunks(false, nullptr);
            for (unsigned b = 0; b < blocks; ++b) {
                if (b == rank) before = mass;
                mass += s.target[b].mass;
            }
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
    reader.kept(reader.load(q, lane, true), q, lane, true, z);
    if (weigh.rest && spread) other.kept(other.load(q, lane, true), q, lane, true, zd);
    unsigned long long w[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = draw_weight(weigh(z[i], weigh.rest && spread ? zd[i] : 0.f, v0 + i));
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
            if (out.logprob) out.logprob[seq] = logf((float)draw_weight(reader.rule.power(z[i], p.m)) / (float)whole);
        }
    }
}

// ------------------------------------------------------------ few classes --

// A sequence per warp; class 32 i + lane of a row in a lane's register i.
template <typename T, int PER>
__global__ void __launch_bounds__(kVerifyThreads)
verify_narrow_kernel(Rows target, Rows draft, int V, Drafts d, Verdict out) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    allow_dependent_launch();
    const long long seq = (long long)blockIdx.x * kVerifyWarps + warp;
    if (seq >= d.S) return;
    const long long first = d.first[seq], end = d.first[seq + 1];
    if (first < 0 || end < first || end > d.D || end > d.first[d.S]) {
        if (lane == 0) {
            flag_index_error();
            out.accepted[seq] = 0;
            out.next_token[seq] = -1;
            if (out.logprob) out.logprob[seq] = BITLOGIC_NEG_INF;
        }
        return;
    }
    float z[PER], m = BITLOGIC_NEG_INF;
    unsigned long long whole = 0;
    int sure = -1;   // the class that p has all of
    bool refused = false;
    long long j = first;
    for (;; ++j) {
        const RowRule rule(target, j + seq);
        const T* x = static_cast<const T*>(target.x) + (j + seq) * target.ld;
        const int v = j < end ? d.token[j] : 0;
        const bool known = v >= 0 && v < V;
        m = BITLOGIC_NEG_INF;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 32 * i + lane;
            z[i] = c < V ? rule.kept(logit_value(x[c]), c) : BITLOGIC_NEG_INF;
            m = fmaxf(m, z[i]);
        }
        const float zv = known ? rule.kept(logit_value(x[v]), v) : BITLOGIC_NEG_INF;
        m = warp_largest(m);
        sure = -1;
        whole = 0;
        if (rule.greedy || m > FLT_MAX) {
            unsigned c = 0x7fffffffu;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i)
                if (z[i] == m && m > BITLOGIC_NEG_INF) c = 32 * i + lane;
            sure = (int)__reduce_min_sync(0xffffffffu, c);
        } else if (m > BITLOGIC_NEG_INF) {
            WeightSum ws;
#pragma unroll
            for (int i = 0; i < PER; i += 2)
                ws.add(pack2(rule.power(z[i], m), i + 1 < PER ? rule.power(z[i + 1 < PER ? i + 1 : i], m) : 0.f));
            whole = ws.warp_total();
        }
        if (j >= end) break;
        if (!known && lane == 0) flag_index_error();
        float p = 0.f;
        if (known && m > BITLOGIC_NEG_INF) p = sure >= 0 ? (v == sure ? 1.f : 0.f) : rule.power(zv, m) / ((float)whole * (1.0f / kWhole));
        if (!(known && passes(d.u[j], d.logprob ? expf(d.logprob[j]) : 1.f, p))) {
            refused = true;
            break;
        }
    }
    if (lane == 0) out.accepted[seq] = (int)(j - first);
    if (!(m > BITLOGIC_NEG_INF) || sure >= 0) {
        if (lane == 0) {
            const bool none = !(m > BITLOGIC_NEG_INF);
            out.next_token[seq] = none ? -1 : sure;
            if (out.logprob) out.logprob[seq] = none ? BITLOGIC_NEG_INF : 0.f;
        }
        return;
    }
    const RowReader other(draft.x && refused ? draft : target, draft.x && refused ? j : j + seq, V);
    Weigher weigh = {RowRule(target, j + seq), other.rule, m, kWhole / (float)whole, 0.f, 0.f, -1, refused};
    if (refused && (!draft.x || other.rule.greedy)) weigh.one = d.token[j];
    const bool spread = refused && draft.x && !other.rule.greedy;
    float zd[PER];
    if (spread) {
        float dm = BITLOGIC_NEG_INF;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 32 * i + lane;
            zd[i] = c < V ? other.at(c) : BITLOGIC_NEG_INF;
            dm = fmaxf(dm, zd[i]);
        }
        dm = warp_largest(dm);
        if (dm > FLT_MAX) {
            weigh.one = d.token[j];
        } else if (dm > BITLOGIC_NEG_INF) {
            WeightSum ws;
#pragma unroll
            for (int i = 0; i < PER; i += 2)
                ws.add(pack2(other.rule.power(zd[i], dm), i + 1 < PER ? other.rule.power(zd[i + 1 < PER ? i + 1 : i], dm) : 0.f));
            weigh.dinv = kWhole / (float)ws.warp_total();
            weigh.dm = dm;
        }
    }
    // the weights of the draw; 32 classes at a time, in order
    unsigned long long total = 0;
    for (int attempt = 0; attempt < 2; ++attempt) {
        WeightSum ws;
#pragma unroll
        for (int i = 0; i < PER; i += 2)
            ws.add(pack2(weigh(z[i], spread ? zd[i] : 0.f, 32 * i + lane),
                         i + 1 < PER ? weigh(z[i + 1 < PER ? i + 1 : i], spread ? zd[i + 1 < PER ? i + 1 : i] : 0.f, 32 * (i + 1) + lane) : 0.f));
        total = ws.warp_total();
        if (total) break;
        weigh.rest = false;   // p and q differ by less than their roundings
    }
    const unsigned long long goal = share_of(total, unit_of(d.draw_u[seq]));
    unsigned long long before = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned long long w = draw_weight(weigh(z[i], spread ? zd[i] : 0.f, 32 * i + lane));
        const unsigned long long upto = before + lanes_upto(w, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, upto > goal);
        if (hit) {
            if (lane == __ffs(hit) - 1) {
                out.next_token[seq] = 32 * i + lane;
                if (out.logprob) out.logprob[seq] = logf((float)draw_weight(weigh.target.power(z[i], m)) / (float)whole);
            }
            return;
        }
        before = __shfl_sync(0xffffffffu, upto, 31);
    }
}

// Parts of a row: as many as keep two to four blocks on every SM, of at least 4 KB.
inline int row_parts(long long rows, int V, int element) {
    int parts = 1;
    while (parts < kMaxParts && rows * parts <= 2 * sm_count() && (long long)V * element / (2 * parts) >= 4096) parts *= 2;
    return parts;
}

// Blocks of a sequence's draw: as many as keep up to eight on every SM, of at
// least 2048 classes.
inline int draw_blocks(long long S, int V) {
    int c = 1;
    while (c < kMaxCluster && S * c * 2 <= 8 * sm_count() && V / (2 * c) >= 2048) c *= 2;
    return c;
}

template <typename T>
int launch_verify(const Rows& target, const Rows& draft, int V, const Drafts& d, const Verdict& out, Part* ws, cudaStream_t stream) {
    cudaError_t e;
    if (V <= kVerifyNarrow) {
        auto kern = V <= 32 ? verify_narrow_kernel<T, 1> : V <= 128 ? verify_narrow_kernel<T, 4>
                  : V <= 256 ? verify_narrow_kernel<T, 8> : V <= 512 ? verify_narrow_kernel<T, 16> : verify_narrow_kernel<T, 32>;
        e = launch_rows(kern, (d.S + kVerifyWarps - 1) / kVerifyWarps, 1, kVerifyThreads, 0, 0, stream, target, draft, V, d, out);
    } else {
        const long long rows = d.S + d.D;
        const int parts = row_parts(rows, V, sizeof(T)), blocks = draw_blocks(d.S, V);
        e = launch_rows(verify_sums_kernel<T>, rows * parts, 1, kVerifyThreads, 0, 0, stream, target, V, d, parts, ws);
        if (e == cudaSuccess) {
            const int all = (V + kChunk - 1) / kChunk, per = (all + blocks - 1) / blocks;
            e = launch_rows(verify_draw_kernel, d.S, blocks, kVerifyThreads, (size_t)per * 8, (kMaxClasses / kChunk) * 8, stream,
                            target, draft, V, d, parts, (const Part*)ws, out);
        }
    }
    return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

BITLOGIC_ERROR_READER(verify)

extern "C" size_t bitlogic_verify_drafts_workspace(int64_t S, int64_t D, int32_t V) {
    if (S < 1 || D < 0 || V <= kVerifyNarrow || S > (1LL << 30) || D > (1LL << 30)) return 0;
    return (size_t)(S + D) * kMaxParts * sizeof(Part);
}

extern "C" int bitlogic_verify_drafts(const void* target, int32_t dtype, int64_t S, int64_t D, int32_t V, int64_t ld,
                                      const float* temperature, const float* floor, const int32_t* last, const int32_t* first,
                                      const int32_t* token, const float* u, const float* draw_u, const void* draft,
                                      int32_t draft_dtype, int64_t draft_ld, const float* draft_logprob,
                                      const float* draft_temperature, const float* draft_floor, const int32_t* draft_last,
                                      int32_t* accepted, int32_t* next_token, float* logprob, void* workspace,
                                      size_t workspace_bytes, cudaStream_t stream) {
    if (S < 0 || D < 0 || S > (1LL << 24) || D > (1LL << 24)) return BITLOGIC_ERR_SHAPE;
    if (S == 0) return D == 0 ? BITLOGIC_OK : BITLOGIC_ERR_SHAPE;
    if (int st = check_logits(target, dtype, true, S + D, V, ld)) return st;
    if (draft)
        if (int st = check_logits(draft, draft_dtype, true, D, V, draft_ld)) return st;
    if (!first || !draw_u || !accepted || !next_token || (D > 0 && (!token || !u))) return BITLOGIC_ERR_NULL;
    if ((floor == nullptr) != (last == nullptr) || (draft_floor == nullptr) != (draft_last == nullptr)) return BITLOGIC_ERR_NULL;
    if (D > 0 && (draft == nullptr) != (draft_logprob == nullptr)) return BITLOGIC_ERR_NULL;
    if (!draft && (draft_temperature || draft_floor)) return D > 0 ? BITLOGIC_ERR_NULL : BITLOGIC_OK;
    const size_t need = bitlogic_verify_drafts_workspace(S, D, V);
    if (need) {
        if (!workspace) return BITLOGIC_ERR_NULL;
        if (!aligned16(workspace)) return BITLOGIC_ERR_ALIGN;
        if (workspace_bytes < need) return BITLOGIC_ERR_WORKSPACE;
    }
    const Rows t = {target, dtype, ld, temperature, floor, last};
    const Rows q = {D > 0 ? draft : nullptr, draft_dtype, draft_ld, draft_temperature, draft_floor, draft_last};
    const Drafts d = {first, token, draft_logprob, u, draw_u, S, D};
    const Verdict out = {accepted, next_token, logprob};
    return with_logit_type(dtype, true, [&](auto* type) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
        return launch_verify<T>(t, q, V, d, out, static_cast<Part*>(workspace), stream);
    });
}
