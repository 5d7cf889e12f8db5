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
// formed in double precision.
//
// Bound by reading the logits and writing the gradient once.
#include "row_tile.cuh"

namespace bitlogic {
namespace {

constexpr int kDistillThreads = 512, kDistillWarps = kDistillThreads / 32;

struct Distill {
    long long T;
    int V, K;
    long long ld;
    const float* val;
    const int* idx;
    const float* teacher_lse;
    const int* labels;
    const float* weight;
    double inv_tau64;
    float inv_tau, kd, ce;   // kd = kd_weight tau^2
    float* row_loss;
    long long ldg, incg;
    float grad_scale;
};

// An entry of the record: a repeated class is one entry with the sum of its
// probabilities, kept by its first place.
struct Entry {
    int v;        // class, -1: none
    float q;      // teacher's probability
    float logq;   // its logarithm
};

// Rows too long for the shared memory of a cluster: one block per row, which
// reads it from memory in every pass; the classes on the record are marked in
// a bit map.
template <typename T>
__global__ void __launch_bounds__(kDistillThreads)
distill_stream_kernel(const T* Z, T* dZ, Distill a) {
    extern __shared__ unsigned on_record[];
    __shared__ float fbuf[kDistillWarps];
    __shared__ double dbuf[kDistillWarps];
    __shared__ int classes[kMaxTop];
    __shared__ int repeated;
    grid_dependency_wait();
    const long long row = blockIdx.x;
    const T* z = Z + row * a.ld;
    T* g = dZ ? dZ + row * a.ldg : nullptr;
    const int tid = threadIdx.x, V = a.V, K = a.K;
    const float wt = a.weight ? a.weight[row] : 1.0f / (float)a.T;
    if (wt == 0.f) {   // a row left out: whatever its logits hold
        for (int v = tid; g && v < V; v += kDistillThreads) g[(long long)v * a.incg] = logit_of<T>(0.f);
        if (tid == 0) a.row_loss[row] = 0.f;
        return;
    }
    for (int i = tid; i < (V + 31) / 32; i += kDistillThreads) on_record[i] = 0u;
    if (tid == 0) repeated = 0;
    Entry e = {-1, 0.f, 0.f};
    float t = BITLOGIC_NEG_INF;
    if (tid < K) {
        e.v = a.idx[row * K + tid];
        if (e.v >= V) {
            flag_index_error();
            e.v = -1;
        }
        if (e.v < 0) e.v = -1;
        else t = a.val[row * K + tid] * a.inv_tau;
        classes[tid] = e.v;
    }
    __syncthreads();
    if (e.v >= 0 && (atomicOr(&on_record[e.v >> 5], 1u << (e.v & 31)) >> (e.v & 31)) & 1u) repeated = 1;
    // the teacher's probabilities
    float norm, Q = 0.f, q_left = 0.f;
    if (a.teacher_lse) {
        norm = a.teacher_lse[row];
        double q = 0.0;
        if (t != BITLOGIC_NEG_INF) {
            const double d = (double)a.val[row * K + tid] * a.inv_tau64 - (double)norm;
            e.logq = (float)d;
            q = exp(d);
        }
        e.q = (float)q;
        const double sum = block_add(q, dbuf, kDistillWarps);
        Q = (float)sum;
        q_left = (float)fmax(1.0 - sum, 0.0);
    } else {
        const float tm = block_largest(t, fbuf, kDistillWarps), ts = isinf(tm) ? 0.f : tm;
        norm = ts + logf(block_add(exp2_unit((t - ts) * kLog2E), fbuf, kDistillWarps));
        e.logq = t - norm;
        e.q = t == BITLOGIC_NEG_INF ? 0.f : exp2_unit(e.logq * kLog2E);
        Q = block_add(e.q, fbuf, kDistillWarps);
    }
    const bool any = block_add(e.v >= 0 ? 1.f : 0.f, fbuf, kDistillWarps) > 0.f;
    bool first = e.v >= 0;
    float q_class = e.q;   // of all places of the class
    __syncthreads();
    if (repeated && e.v >= 0) {
        q_class = 0.f;
        for (int j = 0; j < K; ++j)
            if (classes[j] == e.v) {
                if (j < tid) first = false;
                q_class += a.val[row * K + j] == BITLOGIC_NEG_INF ? 0.f : exp2_unit((a.val[row * K + j] * a.inv_tau - norm) * kLog2E);
            }
    }
    // softmax statistics
    float m = BITLOGIC_NEG_INF;
    for (int v = tid; v < V; v += kDistillThreads) m = fmaxf(m, logit_value(z[v]));
    m = block_largest(m, fbuf, kDistillWarps);
    if (isinf(m) && m < 0.f) m = 0.f;
    const float cy = kLog2E * a.inv_tau;
    const int label = a.labels && a.ce != 0.f ? a.labels[row] : -1;
    float rest = 0.f, member = 0.f, sz = 0.f;
    for (int v = tid; v < V; v += kDistillThreads) {
        const float d = logit_value(z[v]) - m, ey = exp2_unit(d * cy);
        if ((on_record[v >> 5] >> (v & 31)) & 1u) member += ey;
        else rest += ey;
        if (label >= 0) sz += exp2_unit(d * kLog2E);
    }
    rest = block_add(rest, fbuf, kDistillWarps);
    const float s = rest + block_add(member, fbuf, kDistillWarps);
    if (label >= 0) sz = block_add(sz, fbuf, kDistillWarps);
    if (s == 0.f) {   // every class masked: no distribution, no loss
        for (int v = tid; g && v < V; v += kDistillThreads) g[(long long)v * a.incg] = logit_of<T>(0.f);
        if (tid == 0) a.row_loss[row] = 0.f;
        return;
    }
    const bool label_ok = label >= 0 && label < V;
    if (label >= V && tid == 0) flag_index_error();
    const float qr = a.teacher_lse && any && rest > 0.f ? q_left : 0.f;
    const float log_s = logf(s);
    // the loss
    float kl = 0.f;
    if (e.q > 0.f) kl = e.q * (e.logq - ((logit_value(z[e.v]) - m) * a.inv_tau - log_s));
    kl = block_add(kl, fbuf, kDistillWarps);
    if (qr > 0.f) kl += qr * (logf(qr) - logf(rest / s));
    if (tid == 0) {
        float loss = a.kd != 0.f ? a.kd * kl : 0.f;   // a loss of +inf without weight is none
        if (label_ok) loss += a.ce * (logf(sz) - (logit_value(z[label]) - m));
        a.row_loss[row] = (s != s) ? s : loss;
    }
    if (!g) return;
    // the gradient
    const float ay = wt * a.grad_scale * a.kd * a.inv_tau, az = label_ok ? wt * a.grad_scale * a.ce : 0.f;
    const float on = ay * (Q + qr) / s, off = ay * ((Q + qr) / s - (qr > 0.f ? qr / rest : 0.f));
    const float iz = label_ok ? az / sz : 0.f;
    const float z_first = first ? logit_value(z[e.v]) : 0.f, z_label = label_ok ? logit_value(z[label]) : 0.f;
    __syncthreads();   // the gradient may take the logits' place
    for (int v = tid; v < V; v += kDistillThreads) {
        const float d = logit_value(z[v]) - m;
        float x = exp2_unit(d * cy) * off;
        if (label_ok) x += exp2_unit(d * kLog2E) * iz;
        g[(long long)v * a.incg] = logit_of<T>(x);
    }
    __syncthreads();
    if (first) {
        const float d = z_first - m;
        float x = exp2_unit(d * cy) * on - ay * q_class;
        if (label_ok) x += exp2_unit(d * kLog2E) * iz - (e.v == label ? az : 0.f);
        g[(long long)e.v * a.incg] = logit_of<T>(x);
    }
    if (tid == 0 && label_ok && !((on_record[label >> 5] >> (label & 31)) & 1u)) {
        const float d = z_label - m;
        g[(long long)label * a.incg] = logit_of<T>(exp2_unit(d * cy) * off + exp2_unit(d * kLog2E) * iz - az);
    }
}

// Powers 2^(c (z - m)) of a slice about its largest.
struct PowerBase {
    float c, m;
    __device__ __forceinline__ PowerBase(float m_, float c_) : c(c_), m(m_) {}
    __device__ __forceinline__ float operator()(float z) const { return exp2_unit((z - m) * c); }
};

// What the blocks of a row tell each other.
struct __align__(8) DistillStats {
    double q;               // sum of q of the entries in the slice (with teacher_lse)
    float m;                // largest logit
    float rest, member, sz; // powers at tau off and on the record, powers at 1
    float z_label;
    int has_label;
};

constexpr int kTileThreads = 256, kTileWarps = kTileThreads / 32;

// A row in the shared memory of one block or one cluster: the logits are read
// once, and the gradient is written from the same copy.  The record's logits
// are taken out of the slice first (they become -inf), so the passes over the
// slice see the classes off the record only, and the record's own terms and
// gradients are formed by the thread that holds the entry.
// TWO: labels at a temperature other than 1, which need a second softmax.
template <typename T, bool TWO>
__global__ void __launch_bounds__(kTileThreads, 3)
distill_tile_kernel(const T* Z, T* dZ, Distill a) {
    using P = Piece<T>;
    extern __shared__ __align__(16) unsigned char raw[];
    T* tile = reinterpret_cast<T*>(raw);
    uint4* tile16 = reinterpret_cast<uint4*>(raw);
    __shared__ DistillStats stats[kMaxCluster];
    __shared__ float kl_part[kMaxCluster];
    __shared__ float fbuf[3][kTileWarps];
    __shared__ double dbuf[kTileWarps];
    __shared__ int classes[kMaxTop];
    __shared__ float probs[kMaxTop];
    grid_dependency_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned rank = cluster_rank(), blocks = cluster_size();
    const long long row = blockIdx.x / blocks;
    const int V = a.V, K = a.K;
    const T* z = Z + row * a.ld;
    T* g = dZ ? dZ + row * a.ldg : nullptr;
    const RowSlice<T> slice(z, V, rank, blocks);
    const bool wide = a.incg == 1 && ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;
    const float wt = a.weight ? a.weight[row] : 1.0f / (float)a.T;

    // the gradient zero, for rows that do not count
    auto zero_row = [&]() {
        if (g)
            for (int j = tid; j < slice.n; j += kTileThreads) {
                const int v = slice.first + j * P::N;
                if (wide && v >= 0 && v + P::N <= V) {
                    *reinterpret_cast<uint4*>(g + v) = make_uint4(0, 0, 0, 0);
                } else {
                    for (int i = 0; i < P::N; ++i)
                        if (v + i >= 0 && v + i < V) g[(long long)(v + i) * a.incg] = logit_of<T>(0.f);
                }
            }
        if (rank == 0 && tid == 0) a.row_loss[row] = 0.f;
    };
    if (wt == 0.f) {   // the same for every block of the row
        zero_row();
        return;
    }
    slice.copy(z, V, tile, tid, kTileThreads);

    // the record: thread k holds entry k; it is this block's when its class
    // lies in the slice
    int ev = -1, place = -1;
    float t = BITLOGIC_NEG_INF, q = 0.f, logq = 0.f;
    double q64 = 0.0;
    if (tid < K) {
        ev = a.idx[row * K + tid];
        if (ev >= V) {
            if (rank == 0) flag_index_error();
            ev = -1;
        }
        if (ev < 0) {
            ev = -1;
        } else {
            t = a.val[row * K + tid] * a.inv_tau;
            place = slice.place(ev);
        }
    }
    const int label = a.labels && a.ce != 0.f ? a.labels[row] : -1;
    const bool label_ok = label >= 0 && label < V;
    if (label >= V && rank == 0 && tid == 0) flag_index_error();
    const bool any = __syncthreads_or(ev >= 0) != 0;
    const bool label_on = label_ok && __syncthreads_or(ev == label) != 0;
    float Q = 0.f;
    if (a.teacher_lse) {
        if (place >= 0 && t != BITLOGIC_NEG_INF) {
            const double d = (double)a.val[row * K + tid] * a.inv_tau64 - (double)a.teacher_lse[row];
            logq = (float)d;
            q64 = exp(d);
            q = (float)q64;
        }
    } else {
        const float tm = block_largest(t, fbuf[0], kTileWarps), ts = isinf(tm) ? 0.f : tm;
        const float norm = ts + logf(block_add(exp2_unit((t - ts) * kLog2E), fbuf[1], kTileWarps));
        logq = t - norm;
        q = t == BITLOGIC_NEG_INF ? 0.f : exp2_unit(logq * kLog2E);
        Q = block_add(q, fbuf[2], kTileWarps);
    }

    cp_async_wait<0>();
    __syncthreads();
    const float zk = place >= 0 ? logit_value(tile[place]) : 0.f;
    const int label_place = label_ok ? slice.place(label) : -1;
    const float z_label = label_place >= 0 ? logit_value(tile[label_place]) : 0.f;
    __syncthreads();
    // entries of one class write their number to the same place: the ones that
    // do not find it there again are repeated
    auto mark = [&](int n) {
        if constexpr (sizeof(T) == 4) reinterpret_cast<int*>(tile)[place] = n;
        else reinterpret_cast<short*>(tile)[place] = (short)n;
    };
    auto marked = [&]() -> int {
        if constexpr (sizeof(T) == 4) return reinterpret_cast<int*>(tile)[place];
        else return reinterpret_cast<short*>(tile)[place];
    };
    if (place >= 0) mark(tid);
    __syncthreads();
    const bool repeated = __syncthreads_or(place >= 0 && marked() != tid) != 0;
    if (place >= 0) tile[place] = masked_logit<T>();
    bool first = place >= 0;
    float q_class = q;   // of all places of the class
    if (repeated) {
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

    // statistics of the slice about its own largest
    typename P::Max mx = P::lowest();
#pragma unroll 4
    for (int j = tid; j < slice.n; j += kTileThreads) mx = P::largest(mx, tile16[j]);
    float m = P::value(mx);
    if (first) m = fmaxf(m, zk);
    m = block_largest(m, fbuf[0], kTileWarps);
    const float cy = kLog2E * a.inv_tau;
    {
        const float ms = m == BITLOGIC_NEG_INF ? 0.f : m;
        const PowerBase py(ms, cy), pz(ms, kLog2E);
        float r0 = 0.f, r1 = 0.f, s0 = 0.f, s1 = 0.f;
#pragma unroll 2
        for (int j = tid; j < slice.n; j += kTileThreads) {
            float x[P::N];
            P::load(tile16[j], x);
#pragma unroll
            for (int i = 0; i < P::N; i += 2) {
                r0 += py(x[i]);
                r1 += py(x[i + 1]);
                if (TWO) {
                    s0 += pz(x[i]);
                    s1 += pz(x[i + 1]);
                }
            }
        }
        const float member = warp_add(first ? py(zk) : 0.f);
        const float rest = warp_add(r0 + r1), sz = TWO ? warp_add(s0 + s1 + (first ? pz(zk) : 0.f)) : 0.f;
        q64 = a.teacher_lse ? warp_add(q64) : 0.0;
        __syncthreads();
        if (lane == 0) {
            fbuf[0][warp] = rest;
            fbuf[1][warp] = member;
            fbuf[2][warp] = sz;
            dbuf[warp] = q64;
        }
        __syncthreads();
        if (tid < (int)blocks) {
            DistillStats s = {0.0, m, 0.f, 0.f, 0.f, z_label, label_place >= 0};
            for (int w = 0; w < kTileWarps; ++w) {
                s.rest += fbuf[0][w];
                s.member += fbuf[1][w];
                s.sz += fbuf[2][w];
                s.q += dbuf[w];
            }
            put_in_block(&stats[rank], tid, s);
        }
    }
    if (blocks > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }

    // statistics of the row
    m = stats[0].m;
    for (unsigned b = 1; b < blocks; ++b) m = fmaxf(m, stats[b].m);
    if (m == BITLOGIC_NEG_INF) m = 0.f;
    float rest = 0.f, s = 0.f, sz = 0.f, zl = 0.f;
    double q_sum = 0.0;
    for (unsigned b = 0; b < blocks; ++b) {
        const DistillStats& o = stats[b];
        const float d = o.m == BITLOGIC_NEG_INF ? 0.f : o.m - m, f = exp2_unit(d * cy);
        rest += o.rest * f;
        s += o.member * f;
        if (TWO) sz += o.sz * exp2_unit(d * kLog2E);
        q_sum += o.q;
        if (o.has_label) zl = o.z_label;
    }
    s += rest;
    if (!TWO) sz = s;   // tau = 1 where a label is
    const bool empty = s == 0.f;   // every class masked
    float qr = 0.f;
    if (a.teacher_lse) {
        Q = (float)q_sum;
        if (any && rest > 0.f) qr = (float)fmax(1.0 - q_sum, 0.0);
    }
    const float log_s = logf(s);
    {
        const float term = place >= 0 && q > 0.f ? q * (logq - ((zk - m) * a.inv_tau - log_s)) : 0.f;
        const float part = block_add(term, fbuf[0], kTileWarps);
        if (tid == 0) put_in_block(&kl_part[rank], 0, part);
    }
    if (blocks > 1) cluster_arrive();
    else __syncthreads();
    allow_dependent_launch();

    if (empty) {
        zero_row();
    } else if (g) {
        const float ay = wt * a.grad_scale * a.kd * a.inv_tau, az = label_ok ? wt * a.grad_scale * a.ce : 0.f;
        const float on = ay * (Q + qr) / s, off = ay * ((Q + qr) / s - (qr > 0.f ? qr / rest : 0.f));
        const float iz = label_ok ? az / sz : 0.f;
        const PowerBase py(m, cy), pz(m, kLog2E);
        const float fy = TWO ? off : off + iz;
#pragma unroll 2
        for (int j = tid; j < slice.n; j += kTileThreads) {
            float x[P::N];
            P::load(tile16[j], x);
#pragma unroll
            for (int i = 0; i < P::N; ++i) x[i] = TWO ? fmaf(py(x[i]), fy, pz(x[i]) * iz) : py(x[i]) * fy;
            const uint4 u = P::pack(x);
            const int v = slice.first + j * P::N;
            if (!wide) {
                tile16[j] = u;
            } else if (v >= 0 && v + P::N <= V) {
                *reinterpret_cast<uint4*>(g + v) = u;
            } else {
#pragma unroll
                for (int i = 0; i < P::N; ++i)
                    if (v + i >= 0 && v + i < V) g[v + i] = logit_of<T>(x[i]);
            }
        }
        __syncthreads();
        // the record's classes and the label, over what the pass wrote there
        T* to = wide ? g + slice.first : tile;
        if (first) {
            float x = exp2_unit((zk - m) * cy) * on - ay * q_class;
            if (label_ok) x += exp2_unit((zk - m) * kLog2E) * iz - (ev == label ? az : 0.f);
            to[place] = logit_of<T>(x);
        }
        if (tid == 0 && label_place >= 0 && !label_on)
            to[label_place] = logit_of<T>(exp2_unit((z_label - m) * cy) * off + exp2_unit((z_label - m) * kLog2E) * iz - az);
        if (!wide) {   // gradient places apart from the logits' or at another alignment
            __syncthreads();
            for (int p = tid; p < slice.n * P::N; p += kTileThreads) {
                const int v = slice.first + p;
                if (v >= 0 && v < V) g[(long long)v * a.incg] = tile[p];
            }
        }
    }
    if (blocks > 1) cluster_wait();
    if (rank == 0 && tid == 0 && !empty) {
        float kl = 0.f;
        for (unsigned b = 0; b < blocks; ++b) kl += kl_part[b];
        if (qr > 0.f) kl += qr * (logf(qr) - logf(rest / s));
        float loss = a.kd != 0.f ? a.kd * kl : 0.f;
        if (label_ok) loss += a.ce * (logf(sz) - (zl - m));
        a.row_loss[row] = s != s ? s : loss;
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
    const float wt = row >= a.T ? 0.f : a.weight ? a.weight[row] : 1.0f / (float)a.T;
    float loss = 0.f;
    bool counts = wt != 0.f;
    if (counts) {
        const T* z = Z + row * a.ld;
#pragma unroll 4
        for (int v = lane; v < V; v += 32) x[v] = logit_value(z[v]);
        const int label = a.labels && a.ce != 0.f ? a.labels[row] : -1;
        const bool label_ok = label >= 0 && label < V;
        float tm = BITLOGIC_NEG_INF;
        bool bad = label >= V;
        unsigned any = 0, label_on = 0;
        for (int b = 0; b < K; b += 32) {
            const int k = b + lane;
            NarrowEntry e = {-1, 0.f, BITLOGIC_NEG_INF, 0.f};
            if (k < K) {
                e.v = a.idx[row * K + k];
                if (e.v >= V) bad = true;
                if (e.v < 0 || e.v >= V) e.v = -1;
                else e.logq = a.val[row * K + k];
                entries[k] = e;
                tm = fmaxf(tm, e.logq * a.inv_tau);
            }
            any |= __ballot_sync(0xffffffffu, e.v >= 0);
            label_on |= __ballot_sync(0xffffffffu, label_ok && e.v == label);
        }
        if (bad) flag_index_error();
        // the teacher's probabilities
        float Q = 0.f, q_left = 0.f;
        if (a.teacher_lse) {
            const double norm = (double)a.teacher_lse[row];
            double sum = 0.0;
            for (int k = lane; k < K; k += 32) {
                const float t = entries[k].logq;
                if (t != BITLOGIC_NEG_INF) {
                    const double d = (double)t * a.inv_tau64 - norm, q = exp(d);
                    entries[k].logq = (float)d;
                    entries[k].q = (float)q;
                    sum += q;
                }
            }
            sum = warp_add(sum);
            Q = (float)sum;
            q_left = (float)fmax(1.0 - sum, 0.0);
        } else {
            tm = warp_largest(tm);
            const float ts = isinf(tm) ? 0.f : tm;
            float sum = 0.f;
            for (int k = lane; k < K; k += 32) sum += exp2_unit((entries[k].logq * a.inv_tau - ts) * kLog2E);
            const float norm = ts + logf(warp_add(sum));
            for (int k = lane; k < K; k += 32) {
                const float t = entries[k].logq * a.inv_tau;
                if (t != BITLOGIC_NEG_INF) {
                    entries[k].logq = t - norm;
                    entries[k].q = exp2_unit((t - norm) * kLog2E);
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
        float m = BITLOGIC_NEG_INF;
        for (int v = lane; v < V; v += 32) m = fmaxf(m, x[v]);
        for (int k = lane; k < K; k += 32)
            if (entries[k].v >= 0) m = fmaxf(m, entries[k].z);
        m = warp_largest(m);
        if (m == BITLOGIC_NEG_INF) m = 0.f;
        const float cy = kLog2E * a.inv_tau;
        float rest = 0.f, member = 0.f, sz = 0.f;
#pragma unroll 4
        for (int v = lane; v < V; v += 32) {
            const float d = x[v] - m;
            rest += exp2_unit(d * cy);
            if (TWO) sz += exp2_unit(d * kLog2E);
        }
        for (int k = lane; k < K; k += 32) {
            float q_class;
            if (first_of(k, q_class)) {
                const float d = entries[k].z - m;
                member += exp2_unit(d * cy);
                if (TWO) sz += exp2_unit(d * kLog2E);
            }
        }
        rest = warp_add(rest);
        const float s = rest + warp_add(member);
        sz = TWO ? warp_add(sz) : s;
        if (s == 0.f) {
            counts = false;   // every class masked
        } else {
            const float qr = a.teacher_lse && any && rest > 0.f ? q_left : 0.f;
            const float log_s = logf(s);
            float kl = 0.f;
            for (int k = lane; k < K; k += 32)
                if (entries[k].q > 0.f) kl += entries[k].q * (entries[k].logq - ((entries[k].z - m) * a.inv_tau - log_s));
            kl = warp_add(kl);
            if (qr > 0.f) kl += qr * (logf(qr) - logf(rest / s));
            loss = a.kd != 0.f ? a.kd * kl : 0.f;
            if (label_ok) loss += a.ce * (logf(sz) - (z_label - m));
            if (s != s) loss = s;
            if (dZ) {
                const float ay = wt * a.grad_scale * a.kd * a.inv_tau, az = label_ok ? wt * a.grad_scale * a.ce : 0.f;
                const float on = ay * (Q + qr) / s, off = ay * ((Q + qr) / s - (qr > 0.f ? qr / rest : 0.f));
                const float iz = label_ok ? az / sz : 0.f;
#pragma unroll 4
                for (int v = lane; v < V; v += 32) {
                    const float d = x[v] - m;
                    x[v] = TWO ? exp2_unit(d * cy) * off + exp2_unit(d * kLog2E) * iz : exp2_unit(d * cy) * (off + iz);
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
                    x[label] = exp2_unit((z_label - m) * cy) * off + exp2_unit((z_label - m) * kLog2E) * iz - az;
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

// Slices of at most this many bytes leave room for three blocks on an SM: one
// loads while another computes or writes.
constexpr int kTileFit = 70 * 1024, kTileMost = 208 * 1024, kTileLeast = 8 * 1024;

template <typename T, bool TWO>
int launch_distill(const T* z, T* dz, const Distill& a, cudaStream_t stream) {
    cudaError_t e;
    const int blocks = a.V <= kNarrow ? 1 : blocks_per_row(a.T, a.V, sizeof(T), kTileFit, kTileMost, kTileLeast);
    if (a.V <= kNarrow) {
        const size_t smem = kNarrowWarps * (a.K * sizeof(NarrowEntry) + narrow_row_floats(a.V) * sizeof(float));
        e = launch_rows(distill_narrow_kernel<T, TWO>, (a.T + kNarrowWarps - 1) / kNarrowWarps, 1, kNarrowWarps * 32, smem,
                        stream, z, dz, a);
    } else if (blocks > 0) {
        const size_t smem = (size_t)slice_bytes(a.V, sizeof(T), blocks);
        e = launch_rows(distill_tile_kernel<T, TWO>, a.T, blocks, kTileThreads, smem, stream, z, dz, a);
    } else {
        const size_t smem = (size_t)(a.V + 31) / 32 * 4;
        e = launch_rows(distill_stream_kernel<T>, a.T, 1, kDistillThreads, smem, stream, z, dz, a);
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
    if (!(temperature > 0.f) || isinf(temperature) || !isfinite(kd_weight) || !isfinite(ce_weight) ||
        !isfinite(grad_scale))
        return BITLOGIC_ERR_HYPER;
    if (!loss || (T > 0 && (!teacher_val || !teacher_idx || !row_loss))) return BITLOGIC_ERR_NULL;
    if (dZ) {
        // rows and classes of the gradient apart from each other
        if (ldg < 1 || incg < 1 || ldg > (1LL << 40) || incg > (1LL << 40)) return BITLOGIC_ERR_SHAPE;
        if (T > 1 && V > 1 && ldg < (V - 1) * incg + 1 && incg < (T - 1) * ldg + 1) return BITLOGIC_ERR_SHAPE;
        if (reinterpret_cast<uintptr_t>(dZ) % logit_bytes(dtype)) return BITLOGIC_ERR_ALIGN;
    }
    Distill a = {T, V, K, ld, teacher_val, teacher_idx, teacher_lse, labels, row_weight, 1.0 / (double)temperature, 1.0f / temperature,
                 kd_weight * temperature * temperature, ce_weight, row_loss, ldg, incg, grad_scale};
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
