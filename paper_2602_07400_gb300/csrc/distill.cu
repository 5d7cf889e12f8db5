// Distillation from a teacher's record (its K largest logits of a row with
// their classes), joined with the cross-entropy against a label, and the
// gradient of both at the student's logits.
//
// Row with logits z, temperature tau, y = z / tau, p = softmax(y); the record
// lists classes v_k with teacher logits a_k = val_k / tau:
//   without teacher_lse  q_k = exp(a_k) / sum_k exp(a_k), q_r = 0
//   with teacher_lse     q_k = exp(a_k - teacher_lse), q_r = max(0, 1 - sum_k q_k):
//                        the classes off the record are one class of the
//                        teacher's remaining probability
//   KL  = sum_k q_k (ln q_k - ln p_{v_k}) + q_r (ln q_r - ln r),
//         r = sum of p over the classes off the record
//   row = kd tau^2 KL + ce (ln sum_v exp(z_v) - z_label)
//   dKL/dy_v = (sum_k q_k + q_r) p_v - q_v          on the record
//            = (sum_k q_k + q_r) p_v - q_r p_v / r  off it
// r is summed over the classes off the record, not formed as 1 - sum_k p_k,
// which would leave no digits of a small remainder; for the same reason q_r is
// formed from pairs of fp32 numbers.  The sum runs about the largest logit off the
// record: about the row's, it underflows where all of them lie 87 tau below, and
// q_r / r overflows before.  With S that sum and F = 2^(base off the record - base
// of the row), r = S F / s and p_v = power F / s, power about the base off the
// record, so the gradient there is power ((sum_k q_k + q_r) F / s - q_r / S).
// Logarithms of probabilities are taken as (z - m) / tau less that of the sum about
// the row's largest m, since c z overflows before they do; ln r likewise, from the
// largest off the record, where fp32 does not hold r.
// Where every class off the record is masked, q_r = 0.
//
// Bound by reading the logits and writing the gradient once.
#include "row_tile.cuh"

namespace bitlogic {
namespace {

struct Distill {
    long long T;
    int V, K;
    long long ld;
    const float* val;
    const int* idx;
    const float* teacher_lse;
    const int* labels;
    const float* weight;
    Pair inv_tau2;           // 1 / tau
    float inv_tau, kd, ce;   // kd = kd_weight tau^2
    float* row_loss;
    long long ldg, incg;
    float grad_scale;
};

// ln q and q of an entry of logit `val` under the teacher's log-sum-exp.
__device__ __forceinline__ Pair teacher_log(float val, const Distill& a, float lse) {
    const Pair p = exact_product(val, a.inv_tau2.hi);
    return pair_add(Pair{p.hi, fmaf(val, a.inv_tau2.lo, p.lo)}, Pair{-lse, 0.f});
}
// An entry's logit over tau less the largest one's: the difference first, which
// keeps the digits that entries of large logits differ in.
__device__ __forceinline__ float below_largest(float val, float largest, const Distill& a) {
    return (val - (isinf(largest) ? 0.f : largest)) * a.inv_tau;
}
// max(0, 1 - Q)
__device__ __forceinline__ float left_of(Pair Q) { return fmaxf(pair_add(Pair{1.f, 0.f}, Pair{-Q.hi, -Q.lo}).hi, 0.f); }

// ln of a sum of powers about a base, less the base's own logit over tau.
__device__ __forceinline__ float log_about(const PowerBase& p, float sum) { return kLn2 * (log2f(sum) - p.exponent(p.m)); }

// ln r of the classes off the record, r = S F / s: the quotient's own logarithm,
// which keeps the digits of an r near 1, as long as fp32 holds the quotient; else
// from the logits (`below`: the largest off the record less the row's, over tau).
__device__ __forceinline__ float log_remainder(float r, float below, float log_rest, float log_s) {
    return r > 1e-30f ? logf(r) : below + log_rest - log_s;
}

// The bases about a logit at tau (y) and at 1 (z): for two softmaxes far alike, as
// one pass takes the powers of both; else the same, since labels come with tau = 1.
template <bool TWO>
struct Bases {
    PowerBase y, z;
    __device__ __forceinline__ Bases(float largest, float cy) : y(largest, cy), z(largest, TWO ? kLog2E : cy) {
        if (TWO) {
            const PowerBase at_tau = y;
            y = far_alike(y, z);
            z = far_alike(z, at_tau);
        }
    }
};

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;

// Rows too long for the shared memory of a cluster: a block per row, which
// streams it once for the statistics and a second time for the gradient, from
// memory again where the rows in flight exceed L2 (8192 x 131072 bf16, which go
// by the tile kernel: 915 us here, 868 there).
// The classes on the record are marked in a bit map by place, and the pieces that
// hold any in a mask per thread; the marked ones are taken out of their sums.
template <typename T, bool TWO>
__global__ void __launch_bounds__(kRowThreads, 3)
distill_row_kernel(const T* Z, T* dZ, Distill a) {
    using P = Piece<T>;
    constexpr int N = P::N, H = N / 2;
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ float tbuf[kRowWarps], nbuf[kRowWarps], qbuf[kRowWarps], mbuf[kRowWarps], obuf[kRowWarps], kbuf[kRowWarps];
    __shared__ float rest_buf[kRowWarps], member_buf[kRowWarps], sz_buf[kRowWarps];
    __shared__ Pair dbuf[kRowWarps];
    __shared__ int classes[kMaxTop];
    __shared__ float probs[kMaxTop];
    __shared__ int any_s, label_on_s, repeated_s;
    grid_dependency_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = blockIdx.x;
    const int V = a.V, K = a.K;
    const T* z = Z + row * a.ld;
    T* g = dZ ? dZ + row * a.ldg : nullptr;
    const RowSlice<T> slice(z, V, 0, 1);
    const int w0 = slice.whole0(), w1 = slice.whole1(V);
    const bool wide = a.incg == 1 && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;
    const PieceStream<T, kRowThreads> stream(z, slice, V, tid);
    const int words = (stream.batches + 7) / 8;   // of a thread's mask
    uint32_t* masks = reinterpret_cast<uint32_t*>(raw);              // [words][kRowThreads]
    uint32_t* marks = masks + words * kRowThreads;                   // a bit per place
    const uint8_t* marks8 = reinterpret_cast<const uint8_t*>(marks);
    const float wt = a.weight ? a.weight[row] : 1.0f / (float)a.T;
    int ev = tid < K ? a.idx[row * K + tid] : -1;
    const float tval = tid < K ? a.val[row * K + tid] : 0.f;
    const int label = a.labels && a.ce != 0.f ? a.labels[row] : -1;
    // the pieces at the row's ends, of threads 0 and 32
    const int j_end = tid == 0 && w0 > 0 ? 0 : tid == 32 && w1 < slice.n ? w1 : -1;

    auto store = [&](int j, const float (&y)[N]) {
        if (wide && j >= w0 && j < w1) {
            __stcs(reinterpret_cast<uint4*>(g + slice.first) + j, P::pack(y));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int v = slice.first + j * N + i;
                if (v >= 0 && v < V) g[(long long)v * a.incg] = logit_of<T>(y[i]);
            }
        }
    };
    auto zero_row = [&]() {
        const float y[N] = {};
        for (int j = tid; g && j < slice.n; j += kRowThreads) store(j, y);
        if (tid == 0) a.row_loss[row] = 0.f;
    };
    if (wt == 0.f) {   // a row left out: whatever its logits hold
        zero_row();
        return;
    }
    uint4 ua[4], ub[4];
    stream.load(0, ua);
    stream.load(1, ub);

    // the record: thread k holds entry k
    for (int i = tid; i < words * kRowThreads + (slice.n * N + 31) / 32; i += kRowThreads) masks[i] = 0u;
    if (tid == 0) any_s = label_on_s = repeated_s = 0;
    if (ev >= V) {
        flag_index_error();
        ev = -1;
    }
    if (ev < 0) ev = -1;
    const float t = ev >= 0 ? tval * a.inv_tau : BITLOGIC_NEG_INF;
    const float zk = ev >= 0 ? logit_value(z[ev]) : 0.f;
    const bool label_ok = label >= 0 && label < V;
    if (label >= V && tid == 0) flag_index_error();
    const float z_label = label_ok ? logit_value(z[label]) : 0.f;
    __syncthreads();
    if (ev >= 0) {
        any_s = 1;
        if (ev == label) label_on_s = 1;
        const int p = ev - slice.first, j = p / N - w0;   // piece j: lane j % 32 of warp j / 128 % 8, its (j / 32 % 4)th of batch j / 1024
        if ((atomicOr(&marks[p >> 5], 1u << (p & 31)) >> (p & 31)) & 1u) repeated_s = 1;
        if (j >= 0 && j < w1 - w0) {
            const int in = j % (4 * kRowThreads), nth = 4 * (j / (4 * kRowThreads)) + in % 128 / 32;
            atomicOr(&masks[(nth >> 5) * kRowThreads + in / 128 * 32 + in % 32], 1u << (nth & 31));
        }
    }
    // the teacher's probabilities
    float q = 0.f, logq = 0.f, Q = 0.f, q_left = 0.f;
    if (a.teacher_lse) {
        Pair q2 = {0.f, 0.f};
        if (t != BITLOGIC_NEG_INF) {
            const Pair d = teacher_log(tval, a, a.teacher_lse[row]);
            logq = d.hi;
            q2 = exp_pair(d);
            q = q2.hi;
        }
        q2 = warp_add(q2);
        if (lane == 0) dbuf[warp] = q2;
        __syncthreads();
    } else {   // softmax over the record
        const float own = ev >= 0 ? tval : BITLOGIC_NEG_INF, wm = warp_largest(own);
        if (lane == 0) tbuf[warp] = wm;
        __syncthreads();
        float tm = tbuf[0];
        for (int w = 1; w < kRowWarps; ++w) tm = fmaxf(tm, tbuf[w]);
        const float d = below_largest(own, tm, a), ws = warp_add(exp2_unit(d * kLog2E));
        if (lane == 0) nbuf[warp] = ws;
        __syncthreads();
        float sum = 0.f;
        for (int w = 0; w < kRowWarps; ++w) sum += nbuf[w];
        logq = d - logf(sum);
        q = own == BITLOGIC_NEG_INF ? 0.f : exp2_unit(logq * kLog2E);
        const float wq = warp_add(q);
        if (lane == 0) qbuf[warp] = wq;
    }

    // statistics, about a base of each thread's own that seldom moves
    const float cy = kLog2E * a.inv_tau;
    float seen = BITLOGIC_NEG_INF;   // the logit of the base, and the largest
    typename P::Max mx = P::lowest();
    PowerBase by(seen, cy), bz(seen, kLog2E);
    f32x2 y0 = 0, y1 = 0, s0 = 0, s1 = 0;
    auto sums = [&](const uint4& u, const auto& py, const auto& pz) {
        f32x2 x[H];
        load_pairs<T>(u, x);
#pragma unroll
        for (int i = 0; i < H; i += 2) {
            y0 = add2(y0, py(x[i]));
            y1 = add2(y1, py(x[i + 1]));
            if (TWO) {
                s0 = add2(s0, pz(x[i]));
                s1 = add2(s1, pz(x[i + 1]));
            }
        }
    };
    auto add = [&](const uint4 (&u)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = P::largest(mx, u[i]);
        const float top = P::value(mx);
        if (!by.holds(top) || !bz.holds(top)) {
            const PowerBase ny(top, cy), nz(top, kLog2E), uy = far_alike(ny, nz), uz = far_alike(nz, ny);
            const float f = by.to(uy);
            y0 = mul2(y0, pack2(f, f));
            y1 = mul2(y1, pack2(f, f));
            if (TWO) {
                const float h = bz.to(uz);
                s0 = mul2(s0, pack2(h, h));
                s1 = mul2(s1, pack2(h, h));
            }
            by = uy;
            bz = uz;
        }
        if (by.far) {
            const FarPairs py(by), pz(bz);
#pragma unroll
            for (int i = 0; i < 4; ++i) sums(u[i], py, pz);
        } else {
            const NearPairs py(by), pz(bz);
#pragma unroll
            for (int i = 0; i < 4; ++i) sums(u[i], py, pz);
        }
    };
    auto without_marked = [&](uint4& u, int j) {
        const unsigned on = ((unsigned)marks8[j * N / 8] >> (j * N % 8)) & ((1u << N) - 1u);
        T x[N];
        memcpy(x, &u, 16);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((on >> i) & 1u) x[i] = masked_logit<T>();
        memcpy(&u, x, 16);
    };
    auto use = [&](uint4 (&u)[4], int q_, uint32_t mask) {
        const unsigned marked = (mask >> (4 * (q_ & 7))) & 15u;
        if (marked) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((marked >> i) & 1u) without_marked(u[i], stream.piece(q_, i));
        }
        add(u);
    };
    for (int b = 0; b < stream.batches; b += 2) {
        const uint32_t mask = masks[(b >> 3) * kRowThreads + tid];
        use(ua, b, mask);
        if (b + 2 < stream.batches) stream.load(b + 2, ua);
        if (b + 1 < stream.batches) use(ub, b + 1, mask);
        if (b + 3 < stream.batches) stream.load(b + 3, ub);
    }
    if (j_end >= 0) {
        uint4 e[4] = {end_piece(z, V, slice.first + j_end * N), masked_piece<T>(), masked_piece<T>(), masked_piece<T>()};
        without_marked(e[0], j_end);
        add(e);
    }
    if (g) {   // the second time, while the statistics come together
        stream.load(0, ua);
        stream.load(1, ub);
    }

    bool first = ev >= 0;
    float q_class = q;   // of all places of the class
    if (repeated_s) {
        if (tid < K) {
            classes[tid] = ev;
            probs[tid] = q;
        }
        __syncthreads();
        if (ev >= 0) {
            q_class = 0.f;
            for (int j = 0; j < K; ++j)
                if (classes[j] == ev) {
                    if (j < tid) first = false;
                    q_class += probs[j];
                }
        }
    }
    // the bases of the row and of its classes off the record, and the sums
    float m_off = warp_largest(P::value(mx)), m = warp_largest(ev >= 0 ? zk : BITLOGIC_NEG_INF);
    if (lane == 0) {
        obuf[warp] = m_off;
        mbuf[warp] = m;
    }
    __syncthreads();
    for (int w = 0; w < kRowWarps; ++w) {
        m_off = fmaxf(m_off, obuf[w]);
        m = fmaxf(m, mbuf[w]);
    }
    m = fmaxf(m, m_off);
    const Bases<TWO> off_bases(m_off, cy);
    const PowerBase ry(m, cy), rz(m, TWO ? kLog2E : cy), &oy = off_bases.y, &oz = off_bases.z;
    {
        float ra, rb, sa, sb;
        unpack2(add2(y0, y1), ra, rb);
        unpack2(add2(s0, s1), sa, sb);
        const float rest = warp_add((ra + rb) * by.to(oy));
        const float member = warp_add(first ? ry.power(zk) : 0.f);
        const float sz = TWO ? warp_add((sa + sb) * bz.to(rz) + (first ? rz.power(zk) : 0.f)) : 0.f;
        if (lane == 0) {
            rest_buf[warp] = rest;
            member_buf[warp] = member;
            sz_buf[warp] = sz;
        }
    }
    __syncthreads();
    float rest = 0.f, s = 0.f, sz = 0.f;
    Pair q_sum = {0.f, 0.f};
    for (int w = 0; w < kRowWarps; ++w) {
        rest += rest_buf[w];
        s += member_buf[w];
        sz += sz_buf[w];
        if (a.teacher_lse) q_sum = pair_add(q_sum, dbuf[w]);
        else Q += qbuf[w];
    }
    const float to_row = oy.to(ry);
    s += rest * to_row;
    if (!TWO) sz = s;   // tau = 1 where a label is
    if (a.teacher_lse) {
        Q = q_sum.hi;
        q_left = left_of(q_sum);
    }
    const bool any = any_s != 0, label_on = label_on_s != 0;
    allow_dependent_launch();
    if (s == 0.f) {   // every class masked: no distribution, no loss
        zero_row();
        return;
    }
    const float qr = a.teacher_lse && any && !oy.none ? q_left : 0.f, log_s = log_about(ry, s);
    const float kl_part = warp_add(q > 0.f ? q * (logq - ((zk - m) * a.inv_tau - log_s)) : 0.f);
    if (lane == 0) kbuf[warp] = kl_part;
    const float ay = wt * a.grad_scale * a.kd * a.inv_tau, az = label_ok ? wt * a.grad_scale * a.ce : 0.f;
    const float p_off = oy.none ? 0.f : to_row;   // the factor F, 0 where no class is off the record
    const float on = ay * (Q + qr) / s, off = ay * ((Q + qr) * p_off / s - (qr > 0.f ? qr / rest : 0.f));
    const float iz = label_ok ? az / sz : 0.f, iz_off = iz * (!TWO ? p_off : oz.none ? 0.f : oz.to(rz)), fy = TWO ? off : off + iz_off;
    if (g) {
        auto gradient = [&](const auto& py, const auto& pz) {
            const f32x2 fy2 = pack2(fy, fy), fz2 = pack2(iz_off, iz_off);
            auto one = [&](const uint4& u, int j) {
                f32x2 x[H];
                load_pairs<T>(u, x);
                float y[N];
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    f32x2 v = mul2(py(x[i]), fy2);
                    if (TWO) v = fma2(pz(x[i]), fz2, v);
                    unpack2(v, y[2 * i], y[2 * i + 1]);
                }
                store(j, y);
            };
            auto all = [&](const uint4 (&u)[4], int b) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (stream.piece(b, i) < stream.j1) one(u[i], stream.piece(b, i));
            };
            for (int b = 0; b < stream.batches; b += 2) {
                all(ua, b);
                if (b + 2 < stream.batches) stream.load(b + 2, ua);
                if (b + 1 < stream.batches) all(ub, b + 1);
                if (b + 3 < stream.batches) stream.load(b + 3, ub);
            }
            if (j_end >= 0) one(end_piece(z, V, slice.first + j_end * N), j_end);
        };
        if (oy.far) gradient(FarPairs(oy), FarPairs(oz));
        else gradient(NearPairs(oy), NearPairs(oz));
    }
    __syncthreads();
    if (g) {
        // the record's classes (whose powers about the base off the record may
        // have overflowed) and the label, over what the pass wrote there
        if (first) {
            float x = ry.power(zk) * on - ay * q_class;
            if (label_ok) x += rz.power(zk) * iz - (ev == label ? az : 0.f);
            g[(long long)ev * a.incg] = logit_of<T>(x);
        }
        if (tid == 0 && label_ok && !label_on)
            g[(long long)label * a.incg] = logit_of<T>(oy.power(z_label) * off + oz.power(z_label) * iz_off - az);
    }
    if (tid == 0) {
        float kl = 0.f;
        for (int w = 0; w < kRowWarps; ++w) kl += kbuf[w];
        if (qr > 0.f) kl += qr * (logf(qr) - log_remainder(rest * to_row / s, (m_off - m) * a.inv_tau, log_about(oy, rest), log_s));
        float loss = a.kd != 0.f ? a.kd * kl : 0.f;   // a loss of +inf without weight is none
        if (label_ok) loss += a.ce * (log_about(rz, sz) - (z_label - m));
        a.row_loss[row] = s != s ? s : Q != Q ? Q : loss;
    }
}

// What the blocks of a row tell each other.
struct DistillStats {
    Pair q;                 // sum of q of the entries in the slice (with teacher_lse)
    float m, m_off;         // largest logit, and the largest off the record
    float rest;             // powers at tau off the record, about m_off
    float member, sz;       // powers at tau on it, and at 1 of all, about m
    float z_label;
    int has_label;
};

// A row in the shared memory of one block or one cluster: the logits are read
// once, and the gradient is written from the same copy.  The record's logits
// are taken out of the slice first (they become -inf), so the passes over the
// slice see the classes off the record only, and the record's own terms and
// gradients are formed by the thread that holds the entry.
// TWO: labels at a temperature other than 1, which need a second softmax.
// kTileThreads: 256, or 128 or 64 for shorter rows, so that as many threads as an
// SM holds work on rows that are too short to keep 256 in step; at least K.
template <typename T, bool TWO, int kTileThreads>
__global__ void __launch_bounds__(kTileThreads, kTileThreads == 64 ? (TWO ? 14 : 16) : kTileThreads == 128 ? (TWO ? 8 : 10) : (TWO ? 4 : 5))
distill_tile_kernel(const T* Z, T* dZ, Distill a) {
    using P = Piece<T>;
    constexpr int H = P::N / 2, kTileWarps = kTileThreads / 32, kClassTable = 2 * kTileThreads;   // open-addressed, of at most K classes
    extern __shared__ __align__(16) unsigned char raw[];
    T* tile = reinterpret_cast<T*>(raw);
    uint4* tile16 = reinterpret_cast<uint4*>(raw);
    __shared__ DistillStats stats[kMaxCluster];
    __shared__ float kl_part[kMaxCluster * kTileWarps];
    __shared__ float mbuf[kTileWarps], obuf[kTileWarps], tbuf[kTileWarps], nbuf[kTileWarps], qbuf[kTileWarps];
    __shared__ float rest_buf[kTileWarps], member_buf[kTileWarps], sz_buf[kTileWarps];
    __shared__ Pair dbuf[kTileWarps];
    __shared__ int table[kClassTable];
    __shared__ int classes[kTileThreads];
    __shared__ float probs[kTileThreads];
    __shared__ int any_s, label_on_s, repeated_s;
    grid_dependency_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned rank = cluster_rank(), blocks = cluster_size();
    const long long row = blockIdx.x / blocks;
    const int V = a.V, K = a.K;
    const T* z = Z + row * a.ld;
    T* g = dZ ? dZ + row * a.ldg : nullptr;
    const RowSlice<T> slice(z, V, rank, blocks);
    const int w0 = slice.whole0(), w1 = slice.whole1(V);
    const bool wide = a.incg == 1 && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;
    const float wt = a.weight ? a.weight[row] : 1.0f / (float)a.T;
    int ev = tid < K ? a.idx[row * K + tid] : -1;
    const float tval = tid < K ? a.val[row * K + tid] : 0.f;
    const int label = a.labels && a.ce != 0.f ? a.labels[row] : -1;

    // the gradient zero, for rows that do not count
    auto zero_row = [&]() {
        if (g) {
            if (wide) {
                for (int j = w0 + tid; j < w1; j += kTileThreads)
                    *reinterpret_cast<uint4*>(g + slice.first + j * P::N) = make_uint4(0, 0, 0, 0);
                if (tid < 2 * P::N) {
                    const int j = tid < P::N ? 0 : slice.n - 1, v = slice.first + j * P::N + tid % P::N;
                    if (slice.n > 0 && (j < w0 || j >= w1) && v >= 0 && v < V) g[v] = logit_of<T>(0.f);
                }
            } else {
                for (int p = tid; p < slice.n * P::N; p += kTileThreads) {
                    const int v = slice.first + p;
                    if (v >= 0 && v < V) g[(long long)v * a.incg] = logit_of<T>(0.f);
                }
            }
        }
        if (rank == 0 && tid == 0) a.row_loss[row] = 0.f;
    };
    if (wt == 0.f) {   // the same for every block of the row
        zero_row();
        return;
    }
    report_running(blocks);
    slice.copy(z, V, tile, tid, kTileThreads);

    // the record: thread k holds entry k; it is this block's when its class
    // lies in the slice
    for (int i = tid; i < kClassTable; i += kTileThreads) table[i] = -1;
    if (tid == 0) any_s = label_on_s = repeated_s = 0;
    if (ev >= V) {
        if (rank == 0) flag_index_error();
        ev = -1;
    }
    if (ev < 0) ev = -1;
    const float t = ev >= 0 ? tval * a.inv_tau : BITLOGIC_NEG_INF;
    const int place = slice.place(ev);
    const bool label_ok = label >= 0 && label < V;
    if (label >= V && rank == 0 && tid == 0) flag_index_error();
    const int label_place = label_ok ? slice.place(label) : -1;
    float q = 0.f, logq = 0.f, Q = 0.f;
    Pair q2 = {0.f, 0.f};
    if (a.teacher_lse) {
        if (place >= 0 && t != BITLOGIC_NEG_INF) {
            const Pair d = teacher_log(tval, a, a.teacher_lse[row]);
            logq = d.hi;
            q2 = exp_pair(d);
            q = q2.hi;
        }
        __syncthreads();
    } else {   // softmax over the record
        const float own = ev >= 0 ? tval : BITLOGIC_NEG_INF, wm = warp_largest(own);
        if (lane == 0) tbuf[warp] = wm;
        __syncthreads();
        float tm = tbuf[0];
        for (int w = 1; w < kTileWarps; ++w) tm = fmaxf(tm, tbuf[w]);
        const float d = below_largest(own, tm, a), ws = warp_add(exp2_unit(d * kLog2E));
        if (lane == 0) nbuf[warp] = ws;
        __syncthreads();
        float sum = 0.f;
        for (int w = 0; w < kTileWarps; ++w) sum += nbuf[w];
        logq = d - logf(sum);
        q = own == BITLOGIC_NEG_INF ? 0.f : exp2_unit(logq * kLog2E);
        const float wq = warp_add(q);
        if (lane == 0) qbuf[warp] = wq;
    }
    // entries of one class: the second finds the first in the table
    if (ev >= 0) any_s = 1;
    if (label_ok && ev == label) label_on_s = 1;
    if (place >= 0) {
        unsigned h = (((unsigned)ev * 2654435761u) >> 16) % kClassTable;
        for (int i = 0; i < kClassTable; ++i, h = (h + 1) % kClassTable) {
            const int was = atomicCAS(&table[h], -1, ev);
            if (was == ev) repeated_s = 1;
            if (was == -1 || was == ev) break;
        }
    }

    cp_async_wait<0>();
    __syncthreads();
    // the record's logits out of the slice
    const float zk = place >= 0 ? logit_value(tile[place]) : BITLOGIC_NEG_INF;
    const float z_label = label_place >= 0 ? logit_value(tile[label_place]) : 0.f;
    if (repeated_s || label_on_s) __syncthreads();   // a place that several threads read
    if (place >= 0) tile[place] = masked_logit<T>();
    const bool any = any_s != 0, label_on = label_on_s != 0;
    if (!a.teacher_lse)
        for (int w = 0; w < kTileWarps; ++w) Q += qbuf[w];
    bool first = place >= 0;
    float q_class = q;   // of all places of the class
    if (repeated_s) {
        if (tid < K) {
            classes[tid] = ev;
            probs[tid] = q;
        }
        __syncthreads();
        if (place >= 0) {
            q_class = 0.f;
            for (int j = 0; j < K; ++j)
                if (classes[j] == ev) {
                    if (j < tid) first = false;
                    q_class += probs[j];
                }
        }
    }
    __syncthreads();
    // the largest of what is left, and of the slice
    typename P::Max mx = P::lowest();
#pragma unroll 4
    for (int j = tid; j < slice.n; j += kTileThreads) mx = P::largest(mx, tile16[j]);
    float m_off = warp_largest(P::value(mx)), m = warp_largest(zk);
    if (lane == 0) {
        obuf[warp] = m_off;
        mbuf[warp] = m;
    }
    __syncthreads();
    for (int w = 0; w < kTileWarps; ++w) {
        m_off = fmaxf(m_off, obuf[w]);
        m = fmaxf(m, mbuf[w]);
    }
    m = fmaxf(m, m_off);

    // powers of the slice
    const float cy = kLog2E * a.inv_tau;
    {
        const Bases<TWO> e(m_off, cy);
        const PowerBase &ey = e.y, &ez = e.z, my(m, cy), mz(m, kLog2E);
        f32x2 r0 = 0, r1 = 0, s0 = 0, s1 = 0;   // two zeros each
        auto sums = [&](const auto& py, const auto& pz) {
#pragma unroll 2
            for (int j = tid; j < slice.n; j += kTileThreads) {
                f32x2 x[H];
                load_pairs<T>(tile16[j], x);
#pragma unroll
                for (int i = 0; i < H; i += 2) {
                    r0 = add2(r0, py(x[i]));
                    r1 = add2(r1, py(x[i + 1]));
                    if (TWO) {
                        s0 = add2(s0, pz(x[i]));
                        s1 = add2(s1, pz(x[i + 1]));
                    }
                }
            }
        };
        if (ey.far) sums(FarPairs(ey), FarPairs(ez));
        else sums(NearPairs(ey), NearPairs(ez));
        float ra, rb, sa, sb;
        unpack2(add2(r0, r1), ra, rb);
        unpack2(add2(s0, s1), sa, sb);
        const float rest = warp_add(ra + rb), member = warp_add(first ? my.power(zk) : 0.f);
        const float sz = TWO ? warp_add((sa + sb) * ez.to(mz) + (first ? mz.power(zk) : 0.f)) : 0.f;
        if (a.teacher_lse) q2 = warp_add(q2);
        if (lane == 0) {
            rest_buf[warp] = rest;
            member_buf[warp] = member;
            sz_buf[warp] = sz;
            dbuf[warp] = q2;
        }
    }
    __syncthreads();
    wait_all_running(blocks);
    if (tid < (int)blocks) {
        DistillStats s = {{0.f, 0.f}, m, m_off, 0.f, 0.f, 0.f, z_label, label_place >= 0};
        for (int w = 0; w < kTileWarps; ++w) {
            s.rest += rest_buf[w];
            s.member += member_buf[w];
            s.sz += sz_buf[w];
            if (a.teacher_lse) s.q = pair_add(s.q, dbuf[w]);
        }
        put_in_block(&stats[rank], tid, s);
    }
    if (blocks > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }

    // statistics of the row
    m = stats[0].m;
    m_off = stats[0].m_off;
    for (unsigned b = 1; b < blocks; ++b) {
        m = fmaxf(m, stats[b].m);
        m_off = fmaxf(m_off, stats[b].m_off);
    }
    const Bases<TWO> off_bases(m_off, cy);
    const PowerBase by(m, cy), bz(m, TWO ? kLog2E : cy), &oy = off_bases.y, &oz = off_bases.z;
    float rest = stats[0].rest, s = stats[0].member, sz = stats[0].sz, zl = stats[0].z_label;
    Pair q_sum = stats[0].q;
    if (blocks > 1) {   // from the blocks' bases
        rest = s = sz = 0.f;
        q_sum = {0.f, 0.f};
        for (unsigned b = 0; b < blocks; ++b) {
            const DistillStats& o = stats[b];
            rest += o.rest * Bases<TWO>(o.m_off, cy).y.to(oy);
            s += o.member * PowerBase(o.m, cy).to(by);
            if (TWO) sz += o.sz * PowerBase(o.m, kLog2E).to(bz);
            if (a.teacher_lse) q_sum = pair_add(q_sum, o.q);
            if (o.has_label) zl = o.z_label;
        }
    }
    const float to_row = oy.to(by);
    s += rest * to_row;
    if (!TWO) sz = s;   // tau = 1 where a label is
    const bool empty = s == 0.f;   // every class masked
    float qr = 0.f;
    if (a.teacher_lse) {
        Q = q_sum.hi;
        if (any && !oy.none) qr = left_of(q_sum);
    }
    const float log_s = log_about(by, s);
    {
        const float term = place >= 0 && q > 0.f ? q * (logq - ((zk - m) * a.inv_tau - log_s)) : 0.f;
        const float part = warp_add(term);
        if (lane == 0) store_in_block(&kl_part[rank * kTileWarps + warp], 0, __float_as_uint(part));
    }
    if (blocks > 1) cluster_arrive();
    else __syncthreads();
    allow_dependent_launch();

    if (empty) {
        zero_row();
    } else if (g) {
        const float ay = wt * a.grad_scale * a.kd * a.inv_tau, az = label_ok ? wt * a.grad_scale * a.ce : 0.f;
        const float p_off = oy.none ? 0.f : to_row;   // the factor F, 0 where no class is off the record
        const float on = ay * (Q + qr) / s, off = ay * ((Q + qr) * p_off / s - (qr > 0.f ? qr / rest : 0.f));
        const float iz = label_ok ? az / sz : 0.f, iz_off = iz * (!TWO ? p_off : oz.none ? 0.f : oz.to(bz)), fy = TWO ? off : off + iz_off;
        auto gradient = [&](const auto& py, const auto& pz) {
            const f32x2 fy2 = pack2(fy, fy), fz2 = pack2(iz_off, iz_off);
            uint4* to16 = wide ? reinterpret_cast<uint4*>(g + slice.first) : tile16;   // written at whole pieces
#pragma unroll 2
            for (int j = tid; j < slice.n; j += kTileThreads) {
                f32x2 x[H];
                load_pairs<T>(tile16[j], x);
                float y[P::N];
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    f32x2 v = mul2(py(x[i]), fy2);
                    if (TWO) v = fma2(pz(x[i]), fz2, v);
                    unpack2(v, y[2 * i], y[2 * i + 1]);
                }
                const uint4 u = P::pack(y);
                if (!wide || (j >= w0 && j < w1)) to16[j] = u;
                else tile16[j] = u;
            }
        };
        if (oy.far) gradient(FarPairs(oy), FarPairs(oz));
        else gradient(NearPairs(oy), NearPairs(oz));
        __syncthreads();
        // the record's classes and the label, over what the pass wrote there
        auto put = [&](int p, float x) {
            const int j = p / P::N;
            if (wide && j >= w0 && j < w1) g[slice.first + p] = logit_of<T>(x);
            else tile[p] = logit_of<T>(x);
        };
        if (first) {
            float x = by.power(zk) * on - ay * q_class;
            if (label_ok) x += bz.power(zk) * iz - (ev == label ? az : 0.f);
            put(place, x);
        }
        if (tid == 0 && label_place >= 0 && !label_on) put(label_place, oy.power(z_label) * off + oz.power(z_label) * iz_off - az);
        __syncthreads();
        if (!wide) {   // gradient places apart from the logits' or at another alignment
            for (int p = tid; p < slice.n * P::N; p += kTileThreads) {
                const int v = slice.first + p;
                if (v >= 0 && v < V) g[(long long)v * a.incg] = tile[p];
            }
        } else if (tid < 2 * P::N) {   // the pieces at the row's ends
            const int j = tid < P::N ? 0 : slice.n - 1, p = j * P::N + tid % P::N, v = slice.first + p;
            if (slice.n > 0 && (j < w0 || j >= w1) && v >= 0 && v < V) g[v] = tile[p];
        }
    }
    if (blocks > 1) cluster_wait();
    if (rank == 0 && tid == 0 && !empty) {
        float kl = 0.f;
        for (unsigned b = 0; b < blocks * kTileWarps; ++b) kl += kl_part[b];
        if (qr > 0.f) kl += qr * (logf(qr) - log_remainder(rest * to_row / s, (m_off - m) * a.inv_tau, log_about(oy, rest), log_s));
        float loss = a.kd != 0.f ? a.kd * kl : 0.f;
        if (label_ok) loss += a.ce * (log_about(bz, sz) - (zl - m));
        a.row_loss[row] = s != s ? s : Q != Q ? Q : loss;
    }
}

// Rows of few classes: a warp per row, the row as fp32 in shared memory.
constexpr int kNarrow = 1024, kNarrowWarps = 8;

struct NarrowEntry {
    int v;
    float q, logq, z;
};

inline int narrow_row_floats(int V) { return V | 1; }   // odd: the rows of a block lie in different banks

template <typename T, bool TWO>
__global__ void __launch_bounds__(kNarrowWarps * 32)
distill_narrow_kernel(const T* Z, T* dZ, Distill a) {
    extern __shared__ __align__(16) unsigned char raw[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int V = a.V, K = a.K, stride = V | 1;
    NarrowEntry* entries = reinterpret_cast<NarrowEntry*>(raw) + warp * K;
    float* rows = reinterpret_cast<float*>(reinterpret_cast<NarrowEntry*>(raw) + kNarrowWarps * K);
    float* x = rows + warp * stride;
    grid_dependency_wait();
    const long long row0 = (long long)blockIdx.x * kNarrowWarps, row = row0 + warp;
    // all that the row needs of memory is asked for at once
    const bool in = row < a.T;
    const float wt = !in ? 0.f : a.weight ? a.weight[row] : 1.0f / (float)a.T;
    const int label = in && a.labels && a.ce != 0.f ? a.labels[row] : -1;
    const float norm = in && a.teacher_lse ? a.teacher_lse[row] : 0.f;
    if (in) {
        const T* z = Z + row * a.ld;
#pragma unroll 4
        for (int v = lane; v < V; v += 32) x[v] = logit_value(z[v]);
        for (int k = lane; k < K; k += 32) {
            NarrowEntry e = {a.idx[row * K + k], 0.f, a.val[row * K + k], 0.f};
            if (e.v < 0) e.v = -1, e.logq = BITLOGIC_NEG_INF;
            entries[k] = e;
        }
    }
    __syncwarp();
    float loss = 0.f;
    bool counts = wt != 0.f;
    if (counts) {
        const bool label_ok = label >= 0 && label < V;
        float tm = BITLOGIC_NEG_INF;
        bool bad = label >= V;
        unsigned any = 0, label_on = 0;
        for (int b = 0; b < K; b += 32) {
            const int k = b + lane;
            int v = -1;
            if (k < K) {
                v = entries[k].v;
                if (v >= V) {
                    bad = true;
                    entries[k].v = v = -1;
                    entries[k].logq = BITLOGIC_NEG_INF;
                }
                tm = fmaxf(tm, entries[k].logq);
            }
            any |= __ballot_sync(0xffffffffu, v >= 0);
            label_on |= __ballot_sync(0xffffffffu, label_ok && v == label);
        }
        if (bad) flag_index_error();
        // the teacher's probabilities
        float Q = 0.f, q_left = 0.f;
        if (a.teacher_lse) {
            Pair sum = {0.f, 0.f};
            for (int k = lane; k < K; k += 32) {
                const float t = entries[k].logq;
                if (t != BITLOGIC_NEG_INF) {
                    const Pair d = teacher_log(t, a, norm), q = exp_pair(d);
                    entries[k].logq = d.hi;
                    entries[k].q = q.hi;
                    sum = pair_add(sum, q);
                }
            }
            sum = warp_add(sum);
            Q = sum.hi;
            q_left = left_of(sum);
        } else {
            tm = warp_largest(tm);
            float sum = 0.f;
            for (int k = lane; k < K; k += 32) sum += exp2_unit(below_largest(entries[k].logq, tm, a) * kLog2E);
            const float log_sum = logf(warp_add(sum));
            for (int k = lane; k < K; k += 32) {
                const float t = entries[k].logq;
                if (t != BITLOGIC_NEG_INF) {
                    const float logq = below_largest(t, tm, a) - log_sum;
                    entries[k].logq = logq;
                    entries[k].q = exp2_unit(logq * kLog2E);
                    Q += entries[k].q;
                }
            }
            Q = warp_add(Q);
        }
        __syncwarp();
        // the record's logits out of the row, as in the tile kernel
        const float z_label = label_ok ? x[label] : 0.f;
        for (int k = lane; k < K; k += 32)
            if (entries[k].v >= 0) entries[k].z = x[entries[k].v];
        __syncwarp();
        for (int k = lane; k < K; k += 32)
            if (entries[k].v >= 0) x[entries[k].v] = __int_as_float(k);
        __syncwarp();
        bool again = false;
        for (int k = lane; k < K; k += 32)
            if (entries[k].v >= 0 && __float_as_int(x[entries[k].v]) != k) again = true;
        const bool repeated = __any_sync(0xffffffffu, again);
        for (int k = lane; k < K; k += 32)
            if (entries[k].v >= 0) x[entries[k].v] = BITLOGIC_NEG_INF;
        __syncwarp();
        auto first_of = [&](int k, float& q_class) {   // whether place k is its class's first, and the class's q
            const int v = entries[k].v;
            q_class = entries[k].q;
            if (v < 0) return false;
            if (!repeated) return true;
            q_class = 0.f;
            bool first = true;
            for (int j = 0; j < K; ++j)
                if (entries[j].v == v) {
                    if (j < k) first = false;
                    q_class += entries[j].q;
                }
            return first;
        };
        float mo = BITLOGIC_NEG_INF;   // largest off the record
        for (int v = lane; v < V; v += 32) mo = fmaxf(mo, x[v]);
        mo = warp_largest(mo);
        float m = mo;
        for (int k = lane; k < K; k += 32)
            if (entries[k].v >= 0) m = fmaxf(m, entries[k].z);
        m = warp_largest(m);
        if (m == BITLOGIC_NEG_INF) m = 0.f;
        const float cy = kLog2E * a.inv_tau;
        const bool off_record = mo > BITLOGIC_NEG_INF;
        if (!off_record) mo = m;   // of a sum of 0, or of NaN
        const float to_row = exp2_unit((mo - m) * cy), to_row_z = exp2_unit((mo - m) * kLog2E);
        float rest = 0.f, member = 0.f, sz = 0.f;
#pragma unroll 4
        for (int v = lane; v < V; v += 32) {
            const float d = x[v] - mo;
            rest += exp2_unit(d * cy);
            if (TWO) sz += exp2_unit(d * kLog2E);
        }
        if (TWO) sz *= to_row_z;
        for (int k = lane; k < K; k += 32) {
            float q_class;
            if (first_of(k, q_class)) {
                const float d = entries[k].z - m;
                member += exp2_unit(d * cy);
                if (TWO) sz += exp2_unit(d * kLog2E);
            }
        }
        rest = warp_add(rest);
        const float s = rest * to_row + warp_add(member);
        sz = TWO ? warp_add(sz) : s;
        if (s == 0.f) {
            counts = false;   // every class masked
        } else {
            const float qr = a.teacher_lse && any && off_record ? q_left : 0.f;
            const float log_s = logf(s);
            float kl = 0.f;
            for (int k = lane; k < K; k += 32)
                if (entries[k].q > 0.f) kl += entries[k].q * (entries[k].logq - ((entries[k].z - m) * a.inv_tau - log_s));
            kl = warp_add(kl);
            if (qr > 0.f) kl += qr * (logf(qr) - log_remainder(rest * to_row / s, (mo - m) * a.inv_tau, logf(rest), log_s));
            loss = a.kd != 0.f ? a.kd * kl : 0.f;
            if (label_ok) loss += a.ce * (logf(sz) - (z_label - m));
            if (s != s) loss = s;
            else if (Q != Q) loss = Q;
            if (dZ) {
                const float ay = wt * a.grad_scale * a.kd * a.inv_tau, az = label_ok ? wt * a.grad_scale * a.ce : 0.f;
                const float on = ay * (Q + qr) / s, off = ay * ((Q + qr) * to_row / s - (qr > 0.f ? qr / rest : 0.f));
                const float iz = label_ok ? az / sz : 0.f, iz_off = iz * to_row_z;
#pragma unroll 4
                for (int v = lane; v < V; v += 32) {
                    const float d = x[v] - mo;
                    x[v] = TWO ? exp2_unit(d * cy) * off + exp2_unit(d * kLog2E) * iz_off : exp2_unit(d * cy) * (off + iz_off);
                }
                __syncwarp();
                for (int k = lane; k < K; k += 32) {
                    float q_class;
                    if (first_of(k, q_class)) {
                        const float d = entries[k].z - m;
                        float y = exp2_unit(d * cy) * on - ay * q_class;
                        if (label_ok) y += exp2_unit(d * kLog2E) * iz - (entries[k].v == label ? az : 0.f);
                        x[entries[k].v] = y;
                    }
                }
                if (lane == 0 && label_ok && !label_on)
                    x[label] = exp2_unit((z_label - mo) * cy) * off + exp2_unit((z_label - mo) * kLog2E) * iz_off - az;
            }
        }
    }
    if (lane == 0 && row < a.T) a.row_loss[row] = loss;
    allow_dependent_launch();
    if (!dZ) return;
    if (!counts)
        for (int v = lane; v < V; v += 32) x[v] = 0.f;
    if (a.incg == 1) {
        __syncwarp();
        if (row < a.T) {
            T* g = dZ + row * a.ldg;
#pragma unroll 4
            for (int v = lane; v < V; v += 32) g[v] = logit_of<T>(x[v]);
        }
    } else {   // a row per class: neighbouring threads store neighbouring rows
        __syncthreads();
        for (int i = tid; i < V * kNarrowWarps; i += kNarrowWarps * 32) {
            const int r = i % kNarrowWarps, v = i / kNarrowWarps;
            if (row0 + r < a.T) dZ[(row0 + r) * a.ldg + (long long)v * a.incg] = logit_of<T>(rows[r * stride + v]);
        }
    }
}

// Blocks per row.  Slices up to 100 KB (two blocks on an SM) beat more and
// shorter ones: what a block does besides its bytes takes 5 us or more, and the
// more so the more blocks exchange statistics (bf16, 2^30 logits in all: rows of
// 64 KB in one block 740 us, of 128 KB in two 813, of 256 KB in four 868; the
// 256 KB rows in eight slices of 32 KB 927 us; 509 fp32 rows of 200 KB are too
// few waves for it to matter: in two 53.6 us, in four 52.4 us).
constexpr int kTileFit = 100 * 1024, kTileMost = 208 * 1024, kTileLeast = 8 * 1024;

// Shared memory of the kernels for rows of few classes and for rows streamed twice.
inline size_t narrow_bytes(int V, int K) { return kNarrowWarps * (K * sizeof(NarrowEntry) + narrow_row_floats(V) * sizeof(float)); }
inline size_t row_bytes(int V, int element) {
    // a thread's mask bits, by 32 of its pieces, and a bit per place of the row
    const long long pieces = slice_bytes(V, element, 1) / 16, words = (pieces + 32 * kRowThreads - 1) / (32 * kRowThreads);
    return (size_t)(words * kRowThreads + (pieces * (16 / element) + 31) / 32) * 4;
}

template <typename T, bool TWO>
int launch_distill(const T* z, T* dz, const Distill& a, cudaStream_t stream) {
    cudaError_t e;
    const int blocks = blocks_per_row(a.T, a.V, sizeof(T), kTileFit, kTileMost, kTileLeast);
    if (a.V <= kNarrow) {
        e = launch_rows(distill_narrow_kernel<T, TWO>, (a.T + kNarrowWarps - 1) / kNarrowWarps, 1, kNarrowWarps * 32,
                        narrow_bytes(a.V, a.K), narrow_bytes(kNarrow, kMaxTop), stream, z, dz, a);
    } else if (blocks > 0) {
        // (bf16: 9024 rows of 6644 classes 55.6 us in 64 threads, 66.5 in 128,
        // 100 in 256; 8192 rows of 16384 classes 103, 102 and 111 us)
        const long long bytes = slice_bytes(a.V, sizeof(T), blocks);
        auto kern = a.K <= 64 && bytes <= 16 * 1024    ? distill_tile_kernel<T, TWO, 64>
                    : a.K <= 128 && bytes <= 40 * 1024 ? distill_tile_kernel<T, TWO, 128>
                                                       : distill_tile_kernel<T, TWO, 256>;
        const int threads = a.K <= 64 && bytes <= 16 * 1024 ? 64 : a.K <= 128 && bytes <= 40 * 1024 ? 128 : 256;
        e = launch_rows(kern, a.T, blocks, threads, (size_t)bytes, kTileMost, stream, z, dz, a);
    } else {
        e = launch_rows(distill_row_kernel<T, TWO>, a.T, 1, kRowThreads, row_bytes(a.V, sizeof(T)),
                        row_bytes(kMaxClasses, sizeof(T)), stream, z, dz, a);
    }
    return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA;
}

// loss = sum_t weight_t row_t, in a fixed order.
constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads)
distill_loss_kernel(const float* __restrict__ row_loss, const float* __restrict__ weight, long long T,
                    float* __restrict__ loss) {
    __shared__ float buf[kLossThreads / 32];
    dependent_kernel_start();
    float s = 0.f;
    for (long long t = threadIdx.x; t < T; t += kLossThreads) s += __ldcg(row_loss + t) * (weight ? __ldg(weight + t) : 1.0f / (float)T);
    s = block_add(s, buf, kLossThreads / 32);
    if (threadIdx.x == 0) loss[0] = s;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

BITLOGIC_ERROR_READER(distill)

extern "C" int bitlogic_distill_loss(const void* Z, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                     const float* teacher_val, const int32_t* teacher_idx, int32_t K,
                                     const float* teacher_lse, const int32_t* labels, const float* row_weight,
                                     float temperature, float kd_weight, float ce_weight, float* row_loss,
                                     float* loss, void* dZ, int64_t ldg, int64_t incg, float grad_scale,
                                     cudaStream_t stream) {
    if (int st = check_logits(Z, dtype, false, T, V, ld)) return st;
    if (K < 1 || K > kMaxTop) return BITLOGIC_ERR_SHAPE;
    if (!temperature_ok(temperature) || !isfinite(kd_weight) || !isfinite(ce_weight) || !isfinite(grad_scale))
        return BITLOGIC_ERR_HYPER;
    const float kd = kd_weight * temperature * temperature;   // of the divergence
    if (!isfinite(kd) || (kd == 0.f) != (kd_weight == 0.f)) return BITLOGIC_ERR_HYPER;
    if (!loss || (T > 0 && (!teacher_val || !teacher_idx || !row_loss))) return BITLOGIC_ERR_NULL;
    if (dZ) {
        // rows and classes of the gradient apart from each other
        if (ldg < 1 || incg < 1 || ldg > (1LL << 40) || incg > (1LL << 40)) return BITLOGIC_ERR_SHAPE;
        // (the rows' extent by division: the product of T and ldg may pass 64 bits)
        if (T > 1 && V > 1 && ldg < (V - 1) * incg + 1 && (incg - 1) / ldg < T - 1) return BITLOGIC_ERR_SHAPE;
        if (reinterpret_cast<uintptr_t>(dZ) % logit_bytes(dtype)) return BITLOGIC_ERR_ALIGN;
    }
    const double inv_tau = 1.0 / (double)temperature;
    Distill a = {T, V, K, ld, teacher_val, teacher_idx, teacher_lse, labels, row_weight,
                 {(float)inv_tau, (float)(inv_tau - (double)(float)inv_tau)},
                 1.0f / temperature,
                 kd, ce_weight, row_loss, ldg, incg, grad_scale};
    if (T > 0) {
        const int st = with_logit_type(dtype, false, [&](auto* type) {
            using E = std::remove_const_t<std::remove_pointer_t<decltype(type)>>;
            if constexpr (std::is_same_v<E, int>) {
                return (int)BITLOGIC_ERR_DTYPE;
            } else {
                const E* z = static_cast<const E*>(Z);
                E* dz = static_cast<E*>(dZ);
                return labels && ce_weight != 0.f && temperature != 1.f ? launch_distill<E, true>(z, dz, a, stream)
                                                                        : launch_distill<E, false>(z, dz, a, stream);
            }
        });
        if (st) return st;
    }
    if (launch_dependent(distill_loss_kernel, 1, kLossThreads, 0, stream, row_loss, row_weight, (long long)T, loss) !=
        cudaSuccess)
        return BITLOGIC_ERR_CUDA;
    return launch_status();
}
