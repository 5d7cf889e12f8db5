// A class drawn per row under temperature, top-k, top-p and min-p, from one
// given random number per row.
//
//   m = max z,  e_v = 2^((z_v - m) log2(e) / temperature),  w_v = rint(2^40 e_v)
//   kept: the first top_k classes by (value descending, class ascending); of
//   these the shortest run from the front with at least floor(top_p * their
//   mass); of these e_v >= min_p
//   draw: the first class v, by class, whose kept weights up to and including
//   v exceed floor(u * total)
//
// The weights are whole numbers, so every sum is exact: the draw depends on
// the row and its settings alone, not on the batch, the split of a row over
// threads or the order of additions.  Bound by reading the logits once.
#include <cfloat>

#include "logits.cuh"

namespace bitlogic {
namespace {

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr uint32_t kNoCut = 0u;   // every key of a class with a weight lies above

struct Settings {
    const float* u;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
};

// One block per row, any V: the row is read from memory in every pass.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads)
sample_stream_kernel(const T* __restrict__ X, long long ld, int V, Settings set, int* __restrict__ token,
                     float* __restrict__ logprob) {
    __shared__ SelectScratch sc;
    __shared__ float fbuf[kSampleWarps];
    __shared__ unsigned long long mbuf[kSampleWarps], tbuf[kSampleWarps];
    const long long row = blockIdx.x;
    const T* x = X + row * ld;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    float temp = set.temperature ? set.temperature[row] : 1.0f;
    int k = set.top_k ? set.top_k[row] : 0;
    const float p = set.top_p ? set.top_p[row] : 1.0f;
    float floor_e = set.min_p ? set.min_p[row] : 0.0f, u = set.u[row];
    floor_e = floor_e > 0.f ? fminf(floor_e, 1.0f) : 0.f;
    u = u > 0.f ? fminf(u, 0.99999994f) : 0.f;
    float m = BITLOGIC_NEG_INF;
    for (int v = tid; v < V; v += kSampleThreads) m = fmaxf(m, logit_value(x[v]));
    m = block_largest(m, fbuf, kSampleWarps);
    if (m == BITLOGIC_NEG_INF) {   // nothing to draw from
        if (tid == 0) {
            token[row] = -1;
            if (logprob) logprob[row] = BITLOGIC_NEG_INF;
        }
        return;
    }
    float slope = 0.f;
    if (temp > 0.f && !isinf(m)) slope = fminf((1.0f / temp) * kLog2E, FLT_MAX);
    else k = 1;   // the first of the largest
    const float ms = isinf(m) ? 0.f : m;
    auto key_at = [&](int v) { return logit_key(logit_value(x[v])); };
    auto share = [&](int v) {   // e_v; 0 for what does not rank
        const float z = logit_value(x[v]);
        return z > BITLOGIC_NEG_INF ? exp2_unit((isinf(z) ? 0.f : z - ms) * slope) : 0.f;
    };
    Cut cut = {kNoCut, 0};
    unsigned long long above;
    if (k > 0 && k < V) {
        unsigned long long n = 0;
        for (int v = tid; v < V; v += kSampleThreads) n += ranks(key_at(v));
        n = block_add(n, mbuf, kSampleWarps);
        if ((unsigned long long)k < n) {
            cut.key = select_key(key_at, [](int, uint32_t kk) { return ranks(kk) ? 1ull : 0ull; }, V, k, &sc, &above);
            cut.ties = k - above;
        }
    }
    if (p < 1.0f) {
        const uint32_t kt = cut.key;
        unsigned long long mass = 0, we = 0;   // above the cut; the weight of a class at it
        for (int v = tid; v < V; v += kSampleThreads) {
            const uint32_t kk = key_at(v);
            if (kk > kt) mass += draw_weight(share(v));
            else if (kk == kt && cut.ties) we = draw_weight(share(v));
        }
        mass = block_add(mass, mbuf, kSampleWarps);
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long t = shuffle_xor(we, o);
            we = t > we ? t : we;
        }
        __syncthreads();
        if (lane == 0) tbuf[warp] = we;
        __syncthreads();
        for (int w = 0; w < kSampleWarps; ++w) we = tbuf[w] > we ? tbuf[w] : we;
        unsigned long long want = share_of(mass + cut.ties * we, fmaxf(p, 0.f));
        if (want < 1) want = 1;
        if (want > mass) {   // reached among the ties of the top-k cut
            const unsigned long long need = we ? (want - mass + we - 1) / we : cut.ties;
            if (need < cut.ties) cut.ties = need;
        } else {
            const uint32_t t = select_key(key_at, [&](int v, uint32_t kk) { return kk > kt ? draw_weight(share(v)) : 0ull; },
                                          V, want, &sc, &above);
            unsigned long long wt = 0;
            for (int v = tid; v < V; v += kSampleThreads)
                if (key_at(v) == t) wt = draw_weight(share(v));
            for (int o = 16; o > 0; o >>= 1) {
                const unsigned long long q = shuffle_xor(wt, o);
                wt = q > wt ? q : wt;
            }
            __syncthreads();
            if (lane == 0) tbuf[warp] = wt;
            __syncthreads();
            for (int w = 0; w < kSampleWarps; ++w) wt = tbuf[w] > wt ? tbuf[w] : wt;
            cut.key = t;
            cut.ties = wt ? (want - above + wt - 1) / wt : 1;
        }
    }
    // every warp a contiguous part of the row: its weight above the cut, and its ties
    const int part = (V + kSampleWarps - 1) / kSampleWarps, v0 = warp * part, v1 = min(V, v0 + part);
    unsigned long long mass = 0, eq = 0;
    for (int v = v0 + lane; v < v1; v += 32) {
        const uint32_t kk = key_at(v);
        if (kk > cut.key) {
            const float e = share(v);
            if (e >= floor_e) mass += draw_weight(e);
        } else if (kk == cut.key && cut.ties) {
            ++eq;
        }
    }
    mass = warp_add(mass);
    eq = warp_add(eq);
    __syncthreads();
    if (lane == 0) {
        mbuf[warp] = mass;
        tbuf[warp] = eq;
    }
    __syncthreads();
    // weight of a tie: the same for all of them
    unsigned long long wt = 0;
    if (cut.ties) {
        uint32_t kb = cut.key;
        kb = (kb & 0x80000000u) ? (kb ^ 0x80000000u) : ~kb;
        const float z = __uint_as_float(kb);
        const float e = exp2_unit((isinf(z) ? 0.f : z - ms) * slope);
        wt = e >= floor_e ? draw_weight(e) : 0ull;
    }
    unsigned long long total = 0, before = 0, left = cut.ties, my_left = 0;
    for (int w = 0; w < kSampleWarps; ++w) {
        if (w == warp) {
            before = total;
            my_left = left;
        }
        const unsigned long long q = tbuf[w] < left ? tbuf[w] : left;
        total += mbuf[w] + q * wt;
        left -= q;
    }
    const unsigned long long target = share_of(total, u);
    const unsigned long long mine = mass + (eq < my_left ? eq : my_left) * wt;
    if (target < before || target >= before + mine) return;
    // the warp that holds the class: 32 classes at a time, in order
    unsigned long long run = before;
    for (int b = v0; b < v1; b += 32) {
        const int v = b + lane;
        const uint32_t kk = v < v1 ? key_at(v) : 0u;
        const bool same = v < v1 && kk == cut.key && cut.ties;
        const unsigned mask = __ballot_sync(0xffffffffu, same);
        unsigned long long w = 0;
        if (v < v1 && kk > cut.key) {
            const float e = share(v);
            if (e >= floor_e) w = draw_weight(e);
        } else if (same && __popc(mask & ((1u << lane) - 1u)) < my_left) {
            w = wt;
        }
        unsigned long long upto = w;
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long t = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += t;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, run + upto > target);
        if (hit) {
            if (lane == __ffs(hit) - 1) {
                token[row] = v;
                if (logprob) logprob[row] = logf((float)w / (float)total);
            }
            return;
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
        const unsigned used = __popc(mask);
        my_left = my_left > used ? my_left - used : 0;
    }
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

extern "C" int bitlogic_sample_logits(const void* X, int32_t dtype, int64_t T, int32_t V, int64_t ld, const float* u,
                                      const float* temperature, const int32_t* top_k, const float* top_p,
                                      const float* min_p, int32_t* token, float* logprob, cudaStream_t stream) {
    if (int st = check_logits(X, dtype, true, T, V, ld)) return st;
    if (T == 0) return BITLOGIC_OK;
    if (!u || !token) return BITLOGIC_ERR_NULL;
    const Settings set = {u, temperature, top_k, top_p, min_p};
    return with_logit_type(dtype, true, [&](auto* type) {
        const auto* x = static_cast<decltype(type)>(X);
        sample_stream_kernel<<<(unsigned)T, kSampleThreads, 0, stream>>>(x, ld, V, set, token, logprob);
        return launch_status();
    });
}
