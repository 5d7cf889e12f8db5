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
#include "logits.cuh"

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

// One block per row, any V: the row is read from memory in every pass, the
// classes on the record are marked in a bit map.
template <typename T>
__global__ void __launch_bounds__(kDistillThreads)
distill_stream_kernel(const T* Z, T* dZ, Distill a) {
    extern __shared__ unsigned on_record[];
    __shared__ float fbuf[kDistillWarps];
    __shared__ double dbuf[kDistillWarps];
    __shared__ int classes[kMaxTop];
    __shared__ int repeated;
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
                const int smem = (V + 31) / 32 * 4;
                if (smem > 40 * 1024 && cudaFuncSetAttribute(distill_stream_kernel<E>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                             smem) != cudaSuccess)
                    return (int)BITLOGIC_ERR_CUDA;
                distill_stream_kernel<E><<<(unsigned)T, kDistillThreads, smem, stream>>>(
                    static_cast<const E*>(Z), static_cast<E*>(dZ), a);
                return launch_status();
            }
        });
        if (st) return st;
    }
    if (launch_dependent(distill_loss_kernel, 1, kLossThreads, 0, stream, row_loss, row_weight, (long long)T, loss) !=
        cudaSuccess)
        return BITLOGIC_ERR_CUDA;
    return launch_status();
}
