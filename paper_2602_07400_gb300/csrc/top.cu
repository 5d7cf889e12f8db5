// The record of a row's largest logits: values, classes and log-sum-exp, as a
// teacher hands them to bitlogic_distill_loss.
//
//   order  value descending, class ascending; NaN and -inf do not rank
//   lse    = m / tau + ln sum_v 2^((z_v - m) log2(e) / tau),  m = max z
//
// Bound by reading the logits once: T V bytes_of(type) against 8 T K written.
#include "logits.cuh"

namespace bitlogic {
namespace {

constexpr int kTopThreads = 512, kTopWarps = kTopThreads / 32;

// One block per row, any V: the row is read from memory in every pass.
template <typename T>
__global__ void __launch_bounds__(kTopThreads)
top_stream_kernel(const T* __restrict__ X, long long ld, int V, int K, float inv_tau, float* __restrict__ val,
                  int* __restrict__ idx, float* __restrict__ lse) {
    __shared__ SelectScratch sc;
    __shared__ float fbuf[kTopWarps];
    __shared__ unsigned ubuf[kTopWarps];
    __shared__ unsigned long long entry[kMaxTop];
    __shared__ unsigned n_above;
    const long long row = blockIdx.x;
    const T* x = X + row * ld;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    float m = BITLOGIC_NEG_INF;
    unsigned n = 0;
    for (int v = tid; v < V; v += kTopThreads) {
        const float z = logit_value(x[v]);
        m = fmaxf(m, z);
        n += ranks(logit_key(z));
    }
    m = block_largest(m, fbuf, kTopWarps);
    n = block_add(n, ubuf, kTopWarps);
    if (lse) {
        const float ms = isinf(m) ? 0.f : m, c = kLog2E * inv_tau;
        float s = 0.f;
        for (int v = tid; v < V; v += kTopThreads) s += exp2_unit((logit_value(x[v]) - ms) * c);
        s = block_add(s, fbuf, kTopWarps);
        if (tid == 0) lse[row] = ms * inv_tau + logf(s);
    }
    const unsigned want = min((unsigned)K, n);
    for (int r = tid; r < K; r += kTopThreads)
        if (r >= (int)want) {
            val[row * K + r] = BITLOGIC_NEG_INF;
            idx[row * K + r] = -1;
        }
    if (want == 0) return;
    unsigned long long above;
    const uint32_t t = select_key([&](int v) { return logit_key(logit_value(x[v])); },
                                  [](int, uint32_t) { return 1ull; }, V, want, &sc, &above);
    // the classes above t in any order, then the first of those at t by class:
    // every warp takes a contiguous part of the row
    if (tid == 0) n_above = 0;
    const int part = (V + kTopWarps - 1) / kTopWarps, v0 = warp * part, v1 = min(V, v0 + part);
    unsigned eq = 0;
    for (int v = v0 + lane; v < v1; v += 32) eq += logit_key(logit_value(x[v])) == t;
    eq = warp_add(eq);
    __syncthreads();
    if (lane == 0) ubuf[warp] = eq;
    __syncthreads();
    unsigned at = (unsigned)above;
    for (int w = 0; w < warp; ++w) at += ubuf[w];
    for (int b = v0; b < v1; b += 32) {
        const int v = b + lane;
        const uint32_t k = v < v1 ? logit_key(logit_value(x[v])) : 0u;
        if (v < v1 && k > t) entry[atomicAdd(&n_above, 1u)] = ((unsigned long long)k << 32) | (uint32_t)~v;
        const bool same = v < v1 && k == t;
        const unsigned mask = __ballot_sync(0xffffffffu, same);
        const unsigned slot = at + __popc(mask & ((1u << lane) - 1u));
        if (same && slot < want) entry[slot] = ((unsigned long long)k << 32) | (uint32_t)~v;
        at += __popc(mask);
    }
    __syncthreads();
    if (tid < (int)want) {   // every entry to the place of its rank
        const unsigned long long e = entry[tid];
        int r = 0;
        for (unsigned j = 0; j < want; ++j) r += entry[j] > e;
        const int v = (int)~(uint32_t)e;
        val[row * K + r] = logit_value(x[v]);
        idx[row * K + r] = v;
    }
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
    return with_logit_type(dtype, true, [&](auto* type) {
        const auto* x = static_cast<decltype(type)>(X);
        top_stream_kernel<<<(unsigned)T, kTopThreads, 0, stream>>>(x, ld, V, K, 1.0f / temperature, val, idx, lse);
        return launch_status();
    });
}
