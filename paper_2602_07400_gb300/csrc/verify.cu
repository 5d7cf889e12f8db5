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
// target's rows are read once, and again where u q is so near p that the fp32 sum
// does not decide (near_bar).  Bound by that reading.
//
//   verify_rows_kernel    a row (verify_parts_kernel, where rows are few: a part of
//                         one) per block: its largest logit and the sum of its
//                         powers about it, in one pass: every thread keeps a
//                         running maximum and rescales its sum when that rises
//   verify_draw_kernel    (verify_draw.cu) a sequence per block or cluster: the
//                         accepted drafts from the rows' sums, then the draw in
//                         whole-number weights, whose sums are exact in any order
//   verify_narrow_kernel  both for few classes: a sequence per warp, a row in
//                         its registers, from the first draft to the refused one
#include "verify.cuh"

namespace bitlogic {
namespace {

// ------------------------------------------------------------ rows' sums --

// Part `which` of `parts` of a row, by the whole block; every thread gets it.
template <typename T>
__device__ __forceinline__ Part sum_part(const Rows& rows, long long row, int V, unsigned which, unsigned parts, Part* s) {
    using P = Piece<T>;
    constexpr int N = P::N, H = N / 2;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const T* x = static_cast<const T*>(rows.x) + row * rows.ld;
    const RowSlice<T> slice(x, V, which, parts);
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
        if (to > m) {   // about -inf the sum is 0, or the NaN of a masked batch, which stays
            sum *= exp2_unit((m - to) * rule.slope);
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

    // a NaN into the sum, which then is formed again without them
    auto show_nan = [&](const uint4& u) {
        float z[N];
        P::load(u, z);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (z[i] != z[i]) sum = z[i];
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
            if (!(t > BITLOGIC_NEG_INF)) {   // masked, or NaN, which the maximum passes over
#pragma unroll
                for (int i = 0; i < 4; ++i) show_nan(u[i]);
                return;
            }
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
        if (j_end >= 0) {
            add_kept(u_end, j_end);
            show_nan(u_end);
        }
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
    int flags = 0;
    if (sum != sum && !(m > FLT_MAX)) {   // a NaN among the logits, which counts nothing
        flags = kHasNan;
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
    return {m, sum, cls, flags};
}

// Rows in parts, where they are few; what the parts say of a draft is put together
// by the draw.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, 4)
verify_parts_kernel(Rows rows, int V, Drafts d, int parts, Part* __restrict__ out) {
    __shared__ Part s[kVerifyWarps];
    grid_dependency_wait();
    allow_dependent_launch();
    const long long row = blockIdx.x / (unsigned)parts;
    if (row >= (long long)d.first[d.S] + d.S) return;   // behind the last sequence
    const Part p = sum_part<T>(rows, row, V, blockIdx.x % (unsigned)parts, (unsigned)parts, s);
    if (threadIdx.x == 0) out[blockIdx.x] = p;
}

// Whole rows: block b takes row b / S of sequence b % S, and every `turns`-th one
// behind it.  The row's draft is decided here (kRefused), and where rows come
// in several waves `stop` takes each sequence's first refused draft known so far:
// the rows behind it say nothing about the outcome and are not read.  Whether a
// block sees a refusal in time changes its work, never a result (256 x 7 drafts of
// 131072 bf16 classes: 189 us with all rows read, 169 without those).
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, 4)
verify_rows_kernel(Rows rows, int V, Drafts d, int turns, float error, int* stop, Part* __restrict__ out) {
    __shared__ Part s[kVerifyWarps];
    grid_dependency_wait();
    allow_dependent_launch();
    const long long seq = blockIdx.x % (unsigned)d.S;
    Places at;
    if (!at.read(d, seq)) return;
    for (long long i = blockIdx.x / (unsigned)d.S; i <= at.count; i += turns) {
        __syncthreads();   // the buffers of the row before are free
        if (stop) {
            __shared__ int seen;
            if (threadIdx.x == 0) seen = *(volatile int*)(stop + seq);
            __syncthreads();
            if (seen < i) return;
        }
        const long long row = at.first + seq + i, j = at.first + i;
        Part p = sum_part<T>(rows, row, V, 0u, 1u, s);
        if (i < at.count) {
            __shared__ unsigned long long buf[kVerifyWarps];
            __shared__ int border;   // the drafted class, where its share is near the bar
            const RowRule rule(rows, row);
            float bar = 0.f;
            bool refused = false;
            if (threadIdx.x == 0) {
                const int v = d.token[j];
                const bool known = v >= 0 && v < V;
                const float z = known ? kept_logit(rows, rule, row, v) : BITLOGIC_NEG_INF, q = d.logprob ? expf(d.logprob[j]) : 1.f,
                            share = share_in(p, rule, z, v);
                bar = bar_of(d.u[j], q);
                refused = !(known && bar < share);
                border = known && by_sum(p, rule) && near_bar(bar, share, error) ? v : -1;
            }
            __syncthreads();
            if (border >= 0) {
                const float share = whole_share(static_cast<const T*>(rows.x) + row * rows.ld, V, rule, p.m, border, buf);
                refused = !(bar < share);
            }
            if (threadIdx.x == 0 && refused) {
                p.flags |= kRefused;
                if (stop) atomicMin(stop + seq, (int)i);
            }
        }
        if (threadIdx.x == 0) out[row] = p;
    }
}

__global__ void verify_start_kernel(int* stop, long long S) {
    dependent_kernel_start();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < S) stop[i] = INT_MAX;
}

// ------------------------------------------------------------ few classes --

// A sequence per warp; class 32 i + lane of a row in a lane's register i.  Latency
// of a row after another, so a row's loads go out before the first is used, and
// registers are bounded for several blocks on an SM (2048 sequences of 7 drafts over
// 1024 fp32 classes: 50 us, 125 registers; 258 without either, 213 registers).
template <typename T, int PER>
__global__ void __launch_bounds__(kVerifyThreads, PER > 16 ? 2 : PER > 4 ? 3 : 4)
verify_narrow_kernel(Rows target, Rows draft, int V, Drafts d, Verdict out) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    allow_dependent_launch();
    const long long seq = (long long)blockIdx.x * kVerifyWarps + warp;
    if (seq >= d.S) return;
    Places at;
    if (!at.read(d, seq)) {
        if (lane == 0) {
            flag_index_error();
            out.accepted[seq] = 0;
            out.next_token[seq] = -1;
            if (out.logprob) out.logprob[seq] = BITLOGIC_NEG_INF;
        }
        return;
    }
    const long long first = at.first, end = at.first + at.count;
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
        T raw[PER];   // all loads before the first use
#pragma unroll
        for (int i = 0; i < PER; ++i) raw[i] = 32 * i + lane < V ? x[32 * i + lane] : T(0);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 32 * i + lane;
            z[i] = c < V ? rule.kept(logit_value(raw[i]), c) : BITLOGIC_NEG_INF;
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
        if (!(known && bar_of(d.u[j], d.logprob ? expf(d.logprob[j]) : 1.f) < p)) {
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
    const RowRule other(draft.x && refused ? draft : target, draft.x && refused ? j : j + seq);
    Weigher weigh = {RowRule(target, j + seq), other, m, kWhole / (float)whole, 0.f, 0.f, -1, refused};
    if (refused && (!draft.x || other.greedy)) weigh.one = d.token[j];
    const bool spread = refused && draft.x && !other.greedy;
    float zd[PER];
    if (spread) {
        float dm = BITLOGIC_NEG_INF;
        const bool wide = draft.dtype == BITLOGIC_F32 || draft.dtype == BITLOGIC_I32;
        uint32_t bits[PER];
        if (wide) {
            const uint32_t* x = static_cast<const uint32_t*>(draft.x) + j * draft.ld;
#pragma unroll
            for (int i = 0; i < PER; ++i) bits[i] = 32 * i + lane < V ? x[32 * i + lane] : 0u;
        } else {
            const unsigned short* x = static_cast<const unsigned short*>(draft.x) + j * draft.ld;
#pragma unroll
            for (int i = 0; i < PER; ++i) bits[i] = 32 * i + lane < V ? x[32 * i + lane] : 0u;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            zd[i] = draft.dtype == BITLOGIC_BF16  ? __uint_as_float(bits[i] << 16)
                    : draft.dtype == BITLOGIC_F16 ? __half2float(__ushort_as_half((unsigned short)bits[i]))
                    : draft.dtype == BITLOGIC_F32 ? __uint_as_float(bits[i])
                                                  : logit_value((int)bits[i]);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = 32 * i + lane;
            zd[i] = c < V ? other.kept(zd[i], c) : BITLOGIC_NEG_INF;
            dm = fmaxf(dm, zd[i]);
        }
        dm = warp_largest(dm);
        if (dm > FLT_MAX) {
            weigh.one = d.token[j];
        } else if (dm > BITLOGIC_NEG_INF) {
            WeightSum ws;
#pragma unroll
            for (int i = 0; i < PER; i += 2)
                ws.add(pack2(other.power(zd[i], dm), i + 1 < PER ? other.power(zd[i + 1 < PER ? i + 1 : i], dm) : 0.f));
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

template <typename T>
int launch_verify(const Rows& target, const Rows& draft, int V, const Drafts& d, const Verdict& out, Part* ws, cudaStream_t stream) {
    cudaError_t e;
    if (V <= kVerifyNarrow) {
        auto kern = V <= 32 ? verify_narrow_kernel<T, 1> : V <= 128 ? verify_narrow_kernel<T, 4>
                  : V <= 256 ? verify_narrow_kernel<T, 8> : V <= 512 ? verify_narrow_kernel<T, 16> : verify_narrow_kernel<T, 32>;
        e = launch_rows(kern, (d.S + kVerifyWarps - 1) / kVerifyWarps, 1, kVerifyThreads, 0, 0, stream, target, draft, V, d, out);
    } else {
        const long long rows = d.S + d.D;
        const int parts = row_parts(rows, V, sizeof(T));
        const float error = sum_error(V, sizeof(T), parts);
        if (parts > 1) {
            e = launch_rows(verify_parts_kernel<T>, rows * parts, 1, kVerifyThreads, 0, 0, stream, target, V, d, parts, ws);
        } else {
            const long long turns = (rows + d.S - 1) / d.S, blocks = turns * d.S;
            int* stop = blocks > 2 * 4 * sm_count() ? reinterpret_cast<int*>(ws + rows * kMaxParts) : nullptr;
            e = stop ? launch_dependent(verify_start_kernel, (unsigned)((d.S + 255) / 256), 256, 0, stream, stop, d.S) : cudaSuccess;
            if (e == cudaSuccess)
                e = launch_rows(verify_rows_kernel<T>, blocks, 1, kVerifyThreads, 0, 0, stream, target, V, d, (int)turns, error, stop, ws);
        }
        if (e == cudaSuccess) e = launch_verify_draw(target, draft, V, d, parts, error, ws, out, stream);
    }
    return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

BITLOGIC_ERROR_READER(verify)

extern "C" size_t bitlogic_verify_drafts_workspace(int64_t S, int64_t D, int32_t V) {
    if (S < 1 || D < 0 || V <= kVerifyNarrow || S > (1LL << 30) || D > (1LL << 30)) return 0;
    return (size_t)(S + D) * kMaxParts * sizeof(Part) + ((size_t)S * 4 + 15) / 16 * 16;
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
    if (D > 0 && !draft && (draft_temperature || draft_floor)) return BITLOGIC_ERR_NULL;
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
