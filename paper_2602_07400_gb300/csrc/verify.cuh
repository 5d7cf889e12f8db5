// What the kernels of the draft check share (verify.cu, verify_draw.cu).
#pragma once

#include <cfloat>

#include "row_tile.cuh"
#include "weights.cuh"

namespace bitlogic {

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
// A sequence's places; read() is false where they break the rules.
struct Places {
    long long first, count;
    __device__ __forceinline__ bool read(const Drafts& d, long long seq) {
        const long long end = d.first[seq + 1];
        first = d.first[seq];
        count = end - first;
        return first >= 0 && count >= 0 && end <= d.D && end <= d.first[d.S];
    }
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
    int cls;
    int flags;   // kRefused (whole rows: the draft of the row), kHasNan
};

constexpr int kRefused = 1, kHasNan = 2;

struct RowRule {
    float slope, floor;
    int last;
    bool greedy;
    __device__ __forceinline__ RowRule(const Rows& r, long long row) {
        const float temp = r.temperature ? r.temperature[row] : 1.0f;
        greedy = !(temp > 0.f);
        // not 0, so that -inf has no power at any temperature
        slope = greedy ? 0.f : fmaxf(fminf((1.0f / temp) * kLog2E, FLT_MAX), FLT_MIN);
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

// What a draft's test compares p with: u q.
__device__ __forceinline__ float bar_of(float u, float q) { return unit_of(u) * q; }

// The sum of v over the lanes below this one and itself.
__device__ __forceinline__ unsigned long long lanes_upto(unsigned long long v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// The target's probability of class v.
__device__ __forceinline__ float share_in(const Part& p, const RowRule& rule, float z, int v) {
    if (!(p.m > BITLOGIC_NEG_INF)) return 0.f;
    if (rule.greedy || p.m > FLT_MAX) return v == p.cls ? 1.f : 0.f;
    return rule.power(z, p.m) / p.sum;
}

// How far the fp32 sum of a row's parts is off, relatively: in units of 2^-24 less
// than 24 a batch (a rise of the maximum and an addition a piece at most, 6 each, four
// pieces) and 190 (the joins 120, the exponents 44, the powers and the whole weights'
// roundings 26); taken are 32 and 512, 2^-14 for 131072 bf16 classes.
inline float sum_error(int V, int element, int parts) {
    const int batches = ((V / (16 / element) + 2) / parts + 1) / (4 * kVerifyThreads) + 1;
    return (float)(4 * batches + 64) / (float)(1 << 21);
}
// A share of which that may turn the verdict is found again from the sum in whole
// numbers, which is the same in any order; so a verdict goes by its row alone.
__device__ __forceinline__ bool near_bar(float bar, float p, float error) { return p > 0.f && fabsf(bar - p) <= p * error; }
// Whether a row's shares come from a sum.
__device__ __forceinline__ bool by_sum(const Part& p, const RowRule& rule) { return !rule.greedy && p.m <= FLT_MAX; }

// The share of class v of a row by its sum in whole numbers about the largest logit m.
// Called by the whole block; `buf`: a value per warp.  Rare, and out of the callers'
// registers.
template <typename T>
__device__ __noinline__ float whole_share(const T* x, int V, RowRule rule, float m, int v, unsigned long long* buf) {
    unsigned long long sum = 0;
#pragma unroll 4
    for (int c = threadIdx.x; c < V; c += kVerifyThreads) sum += draw_weight(rule.power(rule.kept(logit_value(x[c]), c), m));
    sum = block_add(sum, buf, kVerifyWarps);
    return rule.power(rule.kept(logit_value(x[v]), v), m) / ((float)sum * (1.0f / kWhole));
}

// The kept logit of class v of a row of any type.
__device__ __forceinline__ float kept_logit(const Rows& rows, const RowRule& rule, long long row, int v) {
    const long long at = row * rows.ld + v;
    float z;
    switch (rows.dtype) {
        case BITLOGIC_F32: z = static_cast<const float*>(rows.x)[at]; break;
        case BITLOGIC_BF16: z = logit_value(static_cast<const __nv_bfloat16*>(rows.x)[at]); break;
        case BITLOGIC_F16: z = logit_value(static_cast<const __half*>(rows.x)[at]); break;
        default: z = logit_value(static_cast<const int*>(rows.x)[at]); break;
    }
    return rule.kept(z, v);
}

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
};

// The draw behind the accepted drafts of every sequence (verify_draw.cu).
cudaError_t launch_verify_draw(const Rows& target, const Rows& draft, int V, const Drafts& d, int parts, float error,
                               const Part* sums, const Verdict& out, cudaStream_t stream);

}  // namespace bitlogic
