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
//
// The same kernels give a row's support, the last class kept in the order (value
// descending, class ascending) (kSupport): they stop where the cut is known.
// support.cu compiles this file for that entry point, so that the two compile at
// once.
#include <cfloat>

#include "row_tile.cuh"
#include "weights.cuh"

#pragma nv_diag_suppress 128   // loops behind a support's return are not reached

namespace bitlogic {
namespace {

constexpr int kSampleThreads = 256, kSampleWarps = kSampleThreads / 32;
constexpr uint32_t kNoCut = 0u;   // every key of a class with a weight lies above

struct Settings {
    const float* u;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
};
struct Draw {
    int* token;
    float* logprob;
    float* floor;   // of a support: the logit of the last class kept
    int* last;      // and the class
};

template <bool kSupport>
__device__ __forceinline__ void put_nothing(const Draw& out, long long row) {
    if constexpr (kSupport) {
        out.floor[row] = BITLOGIC_NEG_INF;
        out.last[row] = -1;
    } else {
        out.token[row] = -1;
        if (out.logprob) out.logprob[row] = BITLOGIC_NEG_INF;
    }
}
__device__ __forceinline__ void put_support(const Draw& out, long long row, float floor, int last) {
    out.floor[row] = floor;
    out.last[row] = last;
}

// A row's settings as the draw uses them.
struct RowSettings {
    float u, temp, p, floor_e;
    int k;

    __device__ __forceinline__ RowSettings(const Settings& s, long long row, int V) {
        temp = s.temperature ? s.temperature[row] : 1.0f;
        k = s.top_k ? s.top_k[row] : 0;
        if (k <= 0 || k > V) k = V;
        p = s.top_p ? s.top_p[row] : 1.0f;
        p = p < 1.0f ? fmaxf(p, 0.f) : 1.0f;
        floor_e = s.min_p ? s.min_p[row] : 0.0f;
        floor_e = floor_e > 0.f ? fminf(floor_e, 1.0f) : 0.f;
        u = s.u ? s.u[row] : 0.f;
        u = u > 0.f ? fminf(u, 0.99999994f) : 0.f;
    }
};

// e_v about the row's largest logit.  A temperature that is not positive, or a
// largest logit of +inf, leaves the first of the largest: k = 1.
struct Power {
    float m, slope;
    __device__ __forceinline__ Power(float largest, RowSettings& set) {
        slope = 0.f;
        if (set.temp > 0.f && !isinf(largest)) slope = fminf((1.0f / set.temp) * kLog2E, FLT_MAX);
        else set.k = 1;
        m = isinf(largest) ? 0.f : largest;
    }
    // for a logit that ranks
    __device__ __forceinline__ float operator()(float z) const { return exp2_unit((isinf(z) ? 0.f : z - m) * slope); }
    // for any but +inf: 0 for -inf and NaN (0 slope included)
    __device__ __forceinline__ float of(float z) const {
        return z > BITLOGIC_NEG_INF ? exp2_unit((z - m) * slope) : 0.f;
    }
};

// e of two logits, rounded as Power does one; 0 for -inf and NaN.
struct PowerPairs {
    f32x2 m, slope;
    __device__ __forceinline__ explicit PowerPairs(const Power& p) : m(pack2(p.m, p.m)), slope(pack2(p.slope, p.slope)) {}
    __device__ __forceinline__ f32x2 operator()(f32x2 z) const {
        float a, b;
        unpack2(mul2(sub2(z, m), slope), a, b);
        return pack2(fmaxf(exp2_unit(a), 0.f), fmaxf(exp2_unit(b), 0.f));
    }
    __device__ __forceinline__ f32x2 at_least(f32x2 z, float floor_e) const {
        float a, b;
        unpack2((*this)(z), a, b);
        return pack2(a >= floor_e ? a : 0.f, b >= floor_e ? b : 0.f);
    }
};

struct StreamScratch {
    SelectScratch select;
    float fbuf[kSampleWarps];
    unsigned long long mass[kSampleWarps], ties[kSampleWarps];
};

__device__ __forceinline__ unsigned long long block_max(unsigned long long v, unsigned long long* buf) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long t = shuffle_xor(v, o);
        v = t > v ? t : v;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    for (int w = 0; w < kSampleWarps; ++w) v = buf[w] > v ? buf[w] : v;
    return v;
}

// The inclusive sums of v over the lanes of a warp.
__device__ __forceinline__ unsigned long long warp_upto(unsigned long long v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// A logit below which no power exceeds e (some of those above it may not).
__device__ __forceinline__ float logit_below(float e, const Power& p) {
    return p.slope > 0.f ? p.m - fabsf(p.m) * 1e-6f - (0.02f - 1.000001f * log2f(e)) / p.slope : BITLOGIC_NEG_INF;
}

// The last class kept of a row read from memory: at a cut whose power min_p lets
// through the last of its ties, else the last of the classes above the cut with
// e >= min_p.  Called by the whole block.
template <typename T>
__device__ void last_kept(const T* __restrict__ x, int V, const Cut& cut, const RowSettings& set, const Power& power,
                          long long row, const Draw& out, StreamScratch* sc) {
    using P = Piece<T>;
    constexpr int N = P::N;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const RowSlice<T> slice(x, V, 0, 1);
    const uint4* from = reinterpret_cast<const uint4*>(x + slice.first);
    auto piece = [&](int j) {
        return j >= slice.whole0() && j < slice.whole1(V) ? __ldcg(from + j) : end_piece(x, V, slice.first + j * N);
    };
    const float z_cut = cut.key == kNoCut ? BITLOGIC_NEG_INF : key_logit(cut.key);
    if (cut.ties && power(z_cut) >= set.floor_e) {
        // every warp a contiguous part of the row: its ties
        const int part = (slice.n + kSampleWarps - 1) / kSampleWarps, j0 = min(slice.n, warp * part), j1 = min(slice.n, j0 + part);
        auto ties_of = [&](int j, float (&z)[N]) {
            unsigned same = 0;
            if (j < j1) {
                P::load(piece(j), z);
#pragma unroll
                for (int i = 0; i < N; ++i) same += z[i] == z_cut;
            }
            return same;
        };
        float z[N];
        unsigned eq = 0;
        for (int j = j0 + lane; j < j1; j += 32) eq += ties_of(j, z);
        eq = __reduce_add_sync(0xffffffffu, eq);
        __syncthreads();
        if (lane == 0) sc->ties[warp] = eq;
        __syncthreads();
        unsigned long long left = cut.ties;
        for (int w = 0; w < warp; ++w) left -= sc->ties[w] < left ? sc->ties[w] : left;
        if (left == 0 || left > eq) return;
        for (int b = j0; b < j1; b += 32) {   // the warp that holds it: a piece per lane, in order
            const unsigned same = ties_of(b + lane, z);
            const unsigned upto = (unsigned)warp_upto(same, lane);
            if (upto >= left && upto - same < left) {
                unsigned n = (unsigned)left - (upto - same);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (z[i] == z_cut && --n == 0) put_support(out, row, z_cut + 0.0f, slice.first + (b + lane) * N + i);
            }
            const unsigned all = __shfl_sync(0xffffffffu, upto, 31);
            if (all >= left) return;
            left -= all;
        }
        return;
    }
    const float z_min = set.floor_e > 0.f ? logit_below(set.floor_e, power) : BITLOGIC_NEG_INF;
    unsigned long long best = 0;   // ~key << 32 | class, of the least key
    for (int j0 = tid; j0 < slice.n; j0 += 4 * kSampleThreads) {   // four loads on their way
        uint4 u[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) u[r] = j0 + r * kSampleThreads < slice.n ? piece(j0 + r * kSampleThreads) : masked_piece<T>();
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (P::largest_of(u[r]) >= z_min) {
                float z[N];
                P::load(u[r], z);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (z[i] > z_cut && power(z[i]) >= set.floor_e) {
                        const unsigned long long c = ((unsigned long long)~logit_key(z[i]) << 32) |
                                                     (uint32_t)(slice.first + (j0 + r * kSampleThreads) * N + i);
                        best = c > best ? c : best;
                    }
            }
    }
    best = block_max(best, sc->mass);
    if (tid == 0) put_support(out, row, key_logit(~(uint32_t)(best >> 32)), (int)(uint32_t)best);
}

// The draw of a row read from memory in every pass, for any row and settings.
// Called by the whole block.
template <typename T, bool kSupport>
__device__ void sample_of_stream(const T* __restrict__ x, int V, RowSettings set, long long row, const Draw& out,
                                 StreamScratch* sc) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    float m = BITLOGIC_NEG_INF;
    for (int v = tid; v < V; v += kSampleThreads) m = fmaxf(m, logit_value(x[v]));
    m = block_largest(m, sc->fbuf, kSampleWarps);
    if (m == BITLOGIC_NEG_INF) {   // nothing to draw from
        if (tid == 0) put_nothing<kSupport>(out, row);
        return;
    }
    const Power power(m, set);
    auto key_at = [&](int v) { return logit_key(logit_value(x[v])); };
    auto share = [&](int v) {   // e_v; 0 for what does not rank
        const float z = logit_value(x[v]);
        return z > BITLOGIC_NEG_INF ? power(z) : 0.f;
    };
    Cut cut = {kNoCut, 0};
    unsigned long long above;
    if (set.k < V) {
        unsigned long long n = 0;
        for (int v = tid; v < V; v += kSampleThreads) n += ranks(key_at(v));
        n = block_add(n, sc->mass, kSampleWarps);
        if ((unsigned long long)set.k < n) {
            cut.key = select_key(key_at, [](int, uint32_t kk) { return ranks(kk) ? 1ull : 0ull; }, V, set.k, &sc->select, &above);
            cut.ties = set.k - above;
        }
    }
    if (set.p < 1.0f) {
        const uint32_t kt = cut.key;
        unsigned long long mass = 0;   // above the cut
        for (int v = tid; v < V; v += kSampleThreads)
            if (key_at(v) > kt) mass += draw_weight(share(v));
        mass = block_add(mass, sc->mass, kSampleWarps);
        const unsigned long long we = cut.ties ? draw_weight(power(key_logit(kt))) : 0ull;
        unsigned long long want = share_of(mass + cut.ties * we, set.p);
        if (want < 1) want = 1;
        if (want > mass) {   // reached among the ties of the top-k cut
            const unsigned long long need = we ? (want - mass + we - 1) / we : cut.ties;
            if (need < cut.ties) cut.ties = need;
        } else {
            cut.key = select_key(key_at, [&](int v, uint32_t kk) { return kk > kt ? draw_weight(share(v)) : 0ull; }, V, want,
                                 &sc->select, &above);
            const unsigned long long wt = draw_weight(power(key_logit(cut.key)));
            cut.ties = wt ? (want - above + wt - 1) / wt : 1;
        }
    }
    if constexpr (kSupport) {
        last_kept(x, V, cut, set, power, row, out, sc);
        return;
    }
    // every warp a contiguous part of the row: its weight above the cut, and its ties
    const int part = (V + kSampleWarps - 1) / kSampleWarps, v0 = min(V, warp * part), v1 = min(V, v0 + part);
    unsigned long long mass = 0, eq = 0;
    for (int v = v0 + lane; v < v1; v += 32) {
        const uint32_t kk = key_at(v);
        if (kk > cut.key) {
            const float e = share(v);
            if (e >= set.floor_e) mass += draw_weight(e);
        } else if (kk == cut.key && cut.ties) {
            ++eq;
        }
    }
    mass = warp_add(mass);
    eq = warp_add(eq);
    __syncthreads();
    if (lane == 0) {
        sc->mass[warp] = mass;
        sc->ties[warp] = eq;
    }
    __syncthreads();
    // weight of a tie: the same for all of them
    unsigned long long wt = 0;
    if (cut.ties) {
        const float e = power(key_logit(cut.key));
        wt = e >= set.floor_e ? draw_weight(e) : 0ull;
    }
    unsigned long long total = 0, before = 0, left = cut.ties, my_left = 0;
    for (int w = 0; w < kSampleWarps; ++w) {
        if (w == warp) {
            before = total;
            my_left = left;
        }
        const unsigned long long q = sc->ties[w] < left ? sc->ties[w] : left;
        total += sc->mass[w] + q * wt;
        left -= q;
    }
    const unsigned long long target = share_of(total, set.u);
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
            if (e >= set.floor_e) w = draw_weight(e);
        } else if (same && __popc(mask & ((1u << lane) - 1u)) < my_left) {
            w = wt;
        }
        const unsigned long long upto = warp_upto(w, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, run + upto > target);
        if (hit) {
            if (lane == __ffs(hit) - 1) {
                out.token[row] = v;
                if (out.logprob) out.logprob[row] = logf((float)w / (float)total);
            }
            return;
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
        const unsigned used = __popc(mask);
        my_left = my_left > used ? my_left - used : 0;
    }
}

// ------------------------------------------------------------ rows on chip --

constexpr int kList = 2048;       // entries that a cut or a draw looks at in the end
constexpr int kListTop = 1024;    // largest top_k that goes by the list
constexpr int kBinsPerOctave = 64, kBins = 42 * kBinsPerOctave;   // weights of powers below 2^-41 are 0

struct SampleShared {
    union {
        unsigned long long list[kList];   // key << 32 | ~class, of the row, in the first block
        StreamScratch stream;
    };
    union {
        unsigned long long local[kList];  // of the slice
        BoundScratch bound;
        unsigned bins[kBins];             // mass of the slice by the power's exponent
        struct {
            unsigned long long sums[kSampleWarps];
        } scan;
    };
    struct Stats {
        float m;
        uint32_t bound;
    } stats[kMaxCluster];
    struct Sums {
        unsigned long long mass;
        unsigned ties, pad;
    } sums[kMaxCluster];
    unsigned long long warp_mass[kSampleWarps];
    unsigned warp_ties[kSampleWarps];
    float fbuf[kSampleWarps];
    int kept[kSampleWarps];
    struct Found {
        uint32_t key;
        unsigned ties, slow;
        int last;   // class
    } found;
    int bin, last_bin;
    unsigned n_list, n_local, base;
};

// Bins of the powers e, falling: by the exponent and the 6 leading bits of the
// mantissa, so that the powers above bin b are those with e > bin_above(b); bin
// 64 is the first below 1.  A power counts its mantissa's 15 leading bits, so
// that a bin of 2^17 of them sums in 32 bits and is right to 2^-15 of itself.
__device__ __forceinline__ int bin_of(float e) { return (int)((0x3fffffffu - __float_as_uint(e)) >> 17); }   // 2^-41 <= e <= 1
__device__ __forceinline__ unsigned bin_units(float e) { return (((__float_as_uint(e) & 0x7fffffu) | 0x800000u) + 256u) >> 9; }
__device__ __forceinline__ float bin_mass(unsigned units, int b) {
    return (float)units * __uint_as_float((unsigned)(127 - 14 - b / kBinsPerOctave) << 23);
}
__device__ __forceinline__ float bin_above(int b) { return __uint_as_float(0x3fffffffu - ((unsigned)b << 17)); }

// The bins among which a mass is reached from the largest power down, into *bin: the
// first and, 12 bits up, the last (the last bin of all where there is none).  Every
// power counts to 2^-15 of itself (half a unit of 2^14 or more), and so do the bins'
// sums; fp32 sums and goal and the weights' own roundings add less than 2^-18: the
// bins are those that the mass may be reached in if they are off by both.  No more,
// as a bin of many equal powers beside the cut overflows the list.  (One bin more on
// either side than the one found left out the cut of one row in some thousands, where
// bins weigh less than that; a block took 1.5 ms to draw such a row from memory.)
// Called by the whole block.
__device__ __forceinline__ void find_bin(const unsigned* bins, float goal, int* bin, int* last, float* fbuf) {
    constexpr int kPer = (kBins + kSampleThreads - 1) / kSampleThreads;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr float kOff = 0x1p-15f + 0x1p-18f;
    const float least = goal * (1.0f - kOff), most = goal * (1.0f + kOff);
    float sum = 0.f;
    for (int q = 0; q < kPer; ++q) {
        const int b = tid * kPer + q;
        if (b < kBins) sum += bin_mass(bins[b], b);
    }
    float upto = sum;
    for (int o = 1; o < 32; o <<= 1) {
        const float t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
    }
    if (lane == 31) fbuf[warp] = upto;
    if (tid == 0) *bin = *last = kBins - 1;
    __syncthreads();
    float before = upto - sum;
    for (int w = 0; w < warp; ++w) before += fbuf[w];
    if (before * 0.9999f < most && before + sum >= least * 0.9999f)
        for (int q = 0; q < kPer; ++q) {
            const int b = tid * kPer + q;
            if (b < kBins) {
                before += bin_mass(bins[b], b);
                if (before >= least) atomicMin(bin, b);
                if (before >= most) atomicMin(last, b);
            }
        }
    __syncthreads();
    if (tid == 0) *bin |= *last << 12;
    __syncthreads();
}
__device__ __forceinline__ int first_bin(int found) { return found & 4095; }
__device__ __forceinline__ int end_bin(int found) { return min(kBins, (found >> 12) + 1); }

// The sum of v over the block's threads before this one, and over all of them.
__device__ __forceinline__ unsigned long long block_before(unsigned long long v, unsigned long long* buf,
                                                           unsigned long long* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned long long upto = warp_upto(v, lane);
    __syncthreads();
    if (lane == 31) buf[warp] = upto;
    __syncthreads();
    unsigned long long before = 0, t = 0;
    for (int w = 0; w < kSampleWarps; ++w) {
        if (w == warp) before = t;
        t += buf[w];
    }
    *all = t;
    return before + upto - v;
}

__device__ __forceinline__ int power_of_two(unsigned n) { return n <= 32 ? 32 : 1 << (32 - __clz(n - 1)); }

// The last class kept by mass: the exact mass before the list is `first`, the
// list is sorted here, and `kept(entry, e, w)` is called for every class kept
// on it.  found->slow stays set where the mass is not reached on it.  Called by
// the whole block.
template <typename Found, typename Kept>
__device__ __forceinline__ void find_cut(unsigned long long* list, unsigned listed, unsigned long long first,
                                         unsigned long long want, const Power& power, unsigned long long* sums,
                                         Found* found, Kept&& kept) {
    const int tid = threadIdx.x, size = power_of_two(listed), per = ((int)listed + kSampleThreads - 1) / kSampleThreads;
    for (int i = listed + tid; i < size; i += kSampleThreads) list[i] = 0ull;
    block_sort_falling_256(list, size);
    const int i0 = tid * per, i1 = min((int)listed, i0 + per);
    unsigned long long own = 0, all;
    for (int i = i0; i < i1; ++i) own += draw_weight(power.of(key_logit((uint32_t)(list[i] >> 32))));
    unsigned long long run = first + block_before(own, sums, &all);
    for (int i = i0; i < i1 && run < want; ++i) {
        const uint32_t key = (uint32_t)(list[i] >> 32);
        const float e = power.of(key_logit(key));
        const unsigned long long w = draw_weight(e);
        kept(list[i], e, w);
        if (run + w >= want) {   // the last one
            unsigned ties = 1;   // with those of its key before it
            for (int r = i - 1; r >= 0 && (uint32_t)(list[r] >> 32) == key; --r) ++ties;
            found->key = key;
            found->ties = ties;
            found->slow = 0u;
            found->last = (int)~(uint32_t)list[i];
        }
        run += w;
    }
    __syncthreads();
}

// The first block's work where the row's first k classes are all on its list:
// the cut by rank and mass on the sorted list, then the draw among the kept
// sorted by class.
template <bool kSupport, typename S>
__device__ void sample_of_list(S* s, unsigned n, const RowSettings& set, const Power& power, long long row,
                               const Draw& out) {
    constexpr int kPer = kListTop / kSampleThreads;
    const int tid = threadIdx.x;
    const int size = power_of_two(n);
    for (int i = n + tid; i < size; i += kSampleThreads) s->list[i] = 0ull;
    block_sort_falling_256(s->list, size);
    const int k = min((int)n, set.k);   // at most kListTop
    unsigned long long w[kPer], sum = 0, all;
    float e[kPer];
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
        const int i = tid * kPer + q;
        e[q] = i < k ? power(key_logit((uint32_t)(s->list[i] >> 32))) : 0.f;
        w[q] = i < k ? draw_weight(e[q]) : 0ull;
        sum += w[q];
    }
    unsigned long long before = block_before(sum, s->scan.sums, &all);
    unsigned long long want = set.p < 1.0f ? share_of(all, set.p) : all;
    if (want < 1) want = 1;
    int kept = 0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
        const int i = tid * kPer + q;
        if (i < k && (set.p >= 1.0f || before < want) && (!kSupport || e[q] >= set.floor_e)) kept = i + 1;
        before += w[q];
    }
    // the kept are a run from the front: its length
    for (int o = 16; o > 0; o >>= 1) kept = max(kept, __shfl_xor_sync(0xffffffffu, kept, o));
    __syncthreads();
    if ((tid & 31) == 0) s->kept[tid >> 5] = kept;
    __syncthreads();
    for (int v = 0; v < kSampleWarps; ++v) kept = max(kept, s->kept[v]);
    if constexpr (kSupport) {
        if (tid == 0) put_support(out, row, key_logit((uint32_t)(s->list[kept - 1] >> 32)), (int)~(uint32_t)s->list[kept - 1]);
        return;
    }
    // by class: ~class << 32 | key falls as the class rises
    const int size2 = power_of_two(kept);
    for (int i = tid; i < size2; i += kSampleThreads) {
        const unsigned long long x = s->list[i];
        s->list[i] = i < kept ? (x << 32) | (x >> 32) : 0ull;
    }
    block_sort_falling_256(s->list, size2);
    sum = 0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
        const int i = tid * kPer + q;
        w[q] = 0ull;
        if (i < kept) {
            const float p = power(key_logit((uint32_t)s->list[i]));
            if (p >= set.floor_e) w[q] = draw_weight(p);
        }
        sum += w[q];
    }
    before = block_before(sum, s->scan.sums, &all);
    const unsigned long long target = share_of(all, set.u);
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
        if (target >= before && target < before + w[q]) {
            out.token[row] = (int)~(uint32_t)(s->list[tid * kPer + q] >> 32);
            if (out.logprob) out.logprob[row] = logf((float)w[q] / (float)all);
        }
        before += w[q];
    }
}

// A row in the shared memory of one block or one cluster.  What it does past
// the row's largest logit goes by the row's settings, alike in all its blocks:
//   top_k up to 1024 (and greedy rows): the classes that pass a bound which at
//     least k reach go to the first block, which cuts and draws among them;
//   top_p alone: the weights by bins of 1/64 octave show where the mass is
//     reached; the bins that it may be reached in go to the first block, which finds the
//     cut to the class with exact sums; then every block sums its kept weights
//     in the order of classes and the one that holds the draw finds it;
//   neither: the last step alone.
// A larger top_k, and a list that overflows (long runs of equal logits), are
// drawn from memory by the first block.
template <typename T, bool kSupport>
__global__ void __launch_bounds__(kSampleThreads)
sample_tile_kernel(const T* __restrict__ X, long long ld, int V, Settings settings, Draw out) {
    using P = Piece<T>;
    extern __shared__ __align__(16) unsigned char raw[];
    T* tile = reinterpret_cast<T*>(raw);
    const uint4* tile16 = reinterpret_cast<const uint4*>(raw);
    __shared__ SampleShared s;
    grid_dependency_wait();
    allow_dependent_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned rank = cluster_rank(), blocks = cluster_size();
    const long long row = blockIdx.x / blocks;
    const T* x = X + row * ld;
    const RowSlice<T> slice(x, V, rank, blocks);
    report_running(blocks);
    slice.copy(x, V, tile, tid, kSampleThreads);
    RowSettings set(settings, row, V);
    auto row_barrier = [&]() {
        if (blocks > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
    };
    if (tid == 0) s.n_list = s.n_local = 0;
    cp_async_wait<0>();
    __syncthreads();

    // the largest, and a bound that the first k reach
    const int k_asked = set.temp > 0.f ? set.k : 1;
    typename P::Max ma = P::lowest(), mb = P::lowest();
#pragma unroll 4
    for (int j = tid; j < slice.n; j += 2 * kSampleThreads) {
        ma = P::largest(ma, tile16[j]);
        if (j + kSampleThreads < slice.n) mb = P::largest(mb, tile16[j + kSampleThreads]);
    }
    float part[4];
    P::parts(ma, part[0], part[1]);
    P::parts(mb, part[2], part[3]);
    const uint32_t bound_here = k_asked < V ? block_bound(part, (k_asked + blocks - 1) / blocks, &s.bound) : 0u;
    const float wm = warp_largest(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    if (lane == 0) s.fbuf[warp] = wm;
    __syncthreads();
    wait_all_running(blocks);
    if (tid < (int)blocks) {
        SampleShared::Stats st = {s.fbuf[0], bound_here};
        for (int w = 1; w < kSampleWarps; ++w) st.m = fmaxf(st.m, s.fbuf[w]);
        put_in_block(&s.stats[rank], tid, st);
    }
    row_barrier();
    float m = s.stats[0].m;
    uint32_t bound = s.stats[0].bound;
    for (unsigned b = 1; b < blocks; ++b) {
        m = fmaxf(m, s.stats[b].m);
        bound = min(bound, s.stats[b].bound);
    }
    if (m == BITLOGIC_NEG_INF) {   // nothing to draw from
        if (rank == 0 && tid == 0) put_nothing<kSupport>(out, row);
        return;
    }
    const Power power(m, set);
    const PowerPairs pairs(power);
    if (set.k == 1 && k_asked != 1) bound = 0xff800000u;   // a largest of +inf: nothing below it is needed

    // entries of the slice with zmin <= z <= zmax to the first block's list
    auto list_slice = [&](float zmin, float zmax) {
        for (int j = tid; j < slice.n; j += kSampleThreads) {
            const uint4 u = tile16[j];
            if (P::largest_of(u) >= zmin) {
                float z[P::N];
                P::load(u, z);
#pragma unroll
                for (int i = 0; i < P::N; ++i)
                    if (z[i] >= zmin && z[i] <= zmax && z[i] > BITLOGIC_NEG_INF) {
                        const unsigned at = atomicAdd(&s.n_local, 1u);
                        const int v = slice.first + j * P::N + i;
                        if (at < kList) s.local[at] = ((unsigned long long)logit_key(z[i]) << 32) | (uint32_t)~v;
                    }
            }
        }
        __syncthreads();
        const unsigned n = min(s.n_local, (unsigned)kList);
        if (tid == 0) s.base = add_in_block(&s.n_list, 0, s.n_local);
        __syncthreads();
        for (unsigned i = tid; i < n; i += kSampleThreads)
            if (s.base + i < kList) put_in_block(&s.list[s.base + i], 0, s.local[i]);
    };

    if (set.k < V) {
        const bool listed = set.k <= kListTop;
        if (listed) {
            list_slice(bound_logit(bound), __int_as_float(0x7f800000));
            row_barrier();
        }
        if (rank != 0) return;
        const unsigned n = s.n_list;
        __syncthreads();
        if (listed && n <= kList) sample_of_list<kSupport>(&s, n, set, power, row, out);
        else sample_of_stream<T, kSupport>(x, V, set, row, out, &s.stream);
        return;
    }

    if constexpr (kSupport) {
        if (set.p >= 1.0f) {   // min_p alone, or nothing
            if (rank != 0) return;
            if (set.floor_e > 0.f) last_kept(x, V, Cut{kNoCut, 0}, set, power, row, out, &s.stream);
            else if (tid == 0) put_nothing<true>(out, row);
            return;
        }
    }
    // every warp a contiguous part of the slice, so that sums follow the order
    // of classes
    const int run_of = (slice.n + kSampleWarps - 1) / kSampleWarps, j0 = min(slice.n, warp * run_of),
              j1 = min(slice.n, j0 + run_of);
    Cut cut = {kNoCut, 0};
    float z_cut = BITLOGIC_NEG_INF;   // kept: above it, and the first ties at it
    if (set.p < 1.0f) {
        // the mass of the row
        unsigned long long mass = 0;
        for (int j = j0 + lane; j < j1;) {
            WeightSum ws;
#pragma unroll 4
            for (int r = 0; r < 64 && j < j1; ++r, j += 32) {
                f32x2 z[P::N / 2];
                load_pairs<T>(tile16[j], z);
#pragma unroll
                for (int i = 0; i < P::N / 2; ++i) ws.add(pairs(z[i]));
            }
            mass += ws.total();
        }
        mass = block_add(mass, s.warp_mass, kSampleWarps);
        unsigned* row_bins = reinterpret_cast<unsigned*>(s.list);
        for (int b = tid; b < kBins; b += kSampleThreads) s.bins[b] = row_bins[b] = 0u;
        if (tid < (int)blocks) put_in_block(&s.sums[rank], tid, SampleShared::Sums{mass, 0u, 0u});
        row_barrier();
        unsigned long long total = 0;
        for (unsigned b = 0; b < blocks; ++b) total += s.sums[b].mass;
        unsigned long long want = share_of(total, set.p);
        if (want < 1) want = 1;
        // classes with less than a V-th of what top_p leaves off come after it
        const float left_off = fmaxf((float)(total - want) * (1.0f / 1099511627776.0f) / (float)V, 4.5474735e-13f);   // 2^-41 at least
        const float z_min = logit_below(left_off, power);
        for (int j = tid; j < slice.n; j += kSampleThreads) {
            const uint4 u = tile16[j];
            if (P::largest_of(u) >= z_min) {
                f32x2 z[P::N / 2];
                load_pairs<T>(u, z);
#pragma unroll
                for (int i = 0; i < P::N / 2; ++i) {
                    float a, b;
                    unpack2(pairs(z[i]), a, b);
                    if (a >= left_off) atomicAdd(&s.bins[bin_of(a)], bin_units(a));
                    if (b >= left_off) atomicAdd(&s.bins[bin_of(b)], bin_units(b));
                }
            }
        }
        __syncthreads();
        // the bins of all blocks added up where the first one keeps its list (a
        // sum past 32 bits, of more than 2^17 equal logits, picks a wrong bin,
        // which the exact sums below show)
        for (int b = tid; b < kBins; b += kSampleThreads)
            if (s.bins[b]) add_in_block(row_bins + b, 0, s.bins[b]);
        row_barrier();
        if (rank == 0) {
            find_bin(row_bins, (float)want * (1.0f / 1099511627776.0f), &s.bin, &s.last_bin, s.fbuf);
            const int b = s.bin;
            if (tid < (int)blocks) store_in_block(&s.bin, tid, (uint32_t)b);
            if (tid == 0) s.n_list = 0;
        }
        if (tid == 0) s.n_local = 0;
        row_barrier();
        // the exact mass above the bins found, and their entries
        const float e_above = bin_above(first_bin(s.bin)), e_list = bin_above(end_bin(s.bin)), z_list = logit_below(e_list, power);
        WeightSum ws;
        for (int j = tid; j < slice.n; j += kSampleThreads) {
            const uint4 u = tile16[j];
            if (P::largest_of(u) >= z_list) {
                f32x2 z[P::N / 2];
                load_pairs<T>(u, z);
                bool any = false;
#pragma unroll
                for (int i = 0; i < P::N / 2; ++i) {
                    float a, b;
                    unpack2(pairs(z[i]), a, b);
                    ws.add(pack2(a > e_above ? a : 0.f, b > e_above ? b : 0.f));
                    any |= (a > e_list && a <= e_above) || (b > e_list && b <= e_above);
                }
                if (any) {
                    float x_[P::N];
                    P::load(u, x_);
#pragma unroll
                    for (int i = 0; i < P::N; ++i) {
                        const float e = power.of(x_[i]);
                        if (e > e_list && e <= e_above) {
                            const unsigned at = atomicAdd(&s.n_local, 1u);
                            const int v = slice.first + j * P::N + i;
                            if (at < kList) s.local[at] = ((unsigned long long)logit_key(x_[i]) << 32) | (uint32_t)~v;
                        }
                    }
                }
            }
        }
        mass = block_add(ws.total(), s.warp_mass, kSampleWarps);
        const unsigned n = min(s.n_local, (unsigned)kList);
        if (tid == 0) {
            s.base = add_in_block(&s.n_list, 0, s.n_local);
            put_in_block(&s.sums[rank], 0, SampleShared::Sums{mass, 0u, 0u});
        }
        __syncthreads();
        for (unsigned i = tid; i < n; i += kSampleThreads)
            if (s.base + i < kList) put_in_block(&s.list[s.base + i], 0, s.local[i]);
        row_barrier();
        if (rank == 0) {
            unsigned long long first = 0;
            for (unsigned b = 0; b < blocks; ++b) first += s.sums[b].mass;
            const unsigned listed = s.n_list;
            if (tid == 0) s.found = {0u, 0u, 1u, -1};   // not found: from memory
            __syncthreads();
            if (listed <= kList && listed > 0 && first < want)
                find_cut(s.list, listed, first, want, power, s.scan.sums, &s.found, [](unsigned long long, float, unsigned long long) {});
            const SampleShared::Found f = s.found;
            if (tid < (int)blocks && tid > 0) put_in_block(&s.found, tid, f);
        }
        row_barrier();
        if (s.found.slow) {
            if (rank == 0) sample_of_stream<T, kSupport>(x, V, set, row, out, &s.stream);
            return;
        }
        cut = {s.found.key, s.found.ties};
        z_cut = key_logit(cut.key);
        if constexpr (kSupport) {
            if (rank != 0) return;
            const int last = s.found.last;
            __syncthreads();
            if (power.of(z_cut) < set.floor_e) last_kept(x, V, cut, set, power, row, out, &s.stream);
            else if (tid == 0) put_support(out, row, z_cut, last);
            return;
        }
    }

    // kept weights and ties, by warp and by block
    unsigned long long mass = 0;
    unsigned eq = 0;
    if (set.p >= 1.0f) {
        for (int j = j0 + lane; j < j1;) {
            WeightSum ws;
#pragma unroll 4
            for (int r = 0; r < 64 && j < j1; ++r, j += 32) {
                f32x2 z[P::N / 2];
                load_pairs<T>(tile16[j], z);
#pragma unroll
                for (int i = 0; i < P::N / 2; ++i) ws.add(pairs.at_least(z[i], set.floor_e));
            }
            mass += ws.total();
        }
    } else {
        WeightSum ws;
        for (int j = j0 + lane; j < j1; j += 32) {
            const uint4 u = tile16[j];
            if (P::largest_of(u) >= z_cut) {
                f32x2 z[P::N / 2];
                load_pairs<T>(u, z);
#pragma unroll
                for (int i = 0; i < P::N / 2; ++i) {
                    float a, b, za_, zb_;
                    unpack2(pairs.at_least(z[i], set.floor_e), a, b);
                    unpack2(z[i], za_, zb_);
                    ws.add(pack2(za_ > z_cut ? a : 0.f, zb_ > z_cut ? b : 0.f));
                    eq += (za_ == z_cut) + (zb_ == z_cut);
                }
            }
        }
        mass = ws.total();
    }
    mass = warp_add(mass);
    eq = __reduce_add_sync(0xffffffffu, eq);
    __syncthreads();
    if (lane == 0) {
        s.warp_mass[warp] = mass;
        s.warp_ties[warp] = eq;
    }
    __syncthreads();
    if (tid < (int)blocks) {
        SampleShared::Sums mine = {0ull, 0u, 0u};
        for (int w = 0; w < kSampleWarps; ++w) {
            mine.mass += s.warp_mass[w];
            mine.ties += s.warp_ties[w];
        }
        put_in_block(&s.sums[rank], tid, mine);
    }
    row_barrier();
    unsigned long long wt = 0;
    if (cut.ties) {
        const float e = power.of(z_cut);
        wt = e >= set.floor_e ? draw_weight(e) : 0ull;
    }
    unsigned long long total = 0, before = 0, left = cut.ties, my_left = 0;
    for (unsigned b = 0; b < blocks; ++b) {
        if (b == rank) {
            unsigned long long l = left;
            before = total;
            for (int w = 0; w < warp; ++w) {
                const unsigned long long q = s.warp_ties[w] < l ? s.warp_ties[w] : l;
                before += s.warp_mass[w] + q * wt;
                l -= q;
            }
            my_left = l;
        }
        const unsigned long long q = s.sums[b].ties < left ? s.sums[b].ties : left;
        total += s.sums[b].mass + q * wt;
        left -= q;
    }
    const unsigned long long target = share_of(total, set.u);
    const unsigned long long mine = mass + (eq < my_left ? eq : my_left) * wt;
    if (target < before || target >= before + mine) return;
    // the warp that holds the class: a piece per lane, in order
    unsigned long long run = before;
    for (int b = j0; b < j1; b += 32) {
        const int j = b + lane;
        float z[P::N];
        P::load(j < j1 ? tile16[j] : make_uint4(0, 0, 0, 0), z);
        unsigned long long w[P::N], sum = 0;
        unsigned same = 0;
#pragma unroll
        for (int i = 0; i < P::N; ++i) same += j < j1 && cut.ties && z[i] == z_cut;
        unsigned ties_before = same;
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned t = __shfl_up_sync(0xffffffffu, ties_before, o);
            if (lane >= o) ties_before += t;
        }
        const unsigned ties_all = __shfl_sync(0xffffffffu, ties_before, 31);
        ties_before -= same;
#pragma unroll
        for (int i = 0; i < P::N; ++i) {
            w[i] = 0ull;
            if (j < j1) {
                if (z[i] > z_cut) {
                    const float e = power.of(z[i]);
                    if (e >= set.floor_e) w[i] = draw_weight(e);
                } else if (cut.ties && z[i] == z_cut) {
                    if (ties_before < my_left) w[i] = wt;
                    ++ties_before;
                }
            }
            sum += w[i];
        }
        const unsigned long long upto = warp_upto(sum, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, run + upto > target);
        if (hit) {
            if (lane == __ffs(hit) - 1) {
                unsigned long long r = run + upto - sum;
                bool done = false;
#pragma unroll
                for (int i = 0; i < P::N; ++i) {
                    r += w[i];
                    if (!done && r > target) {
                        done = true;
                        out.token[row] = slice.first + j * P::N + i;
                        if (out.logprob) out.logprob[row] = logf((float)w[i] / (float)total);
                    }
                }
            }
            return;
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
        my_left = my_left > ties_all ? my_left - ties_all : 0;
    }
}

// ------------------------------------------------------ rows by one block --

constexpr int kRowList = 4096;   // entries that a cut or a draw looks at in the end

struct SampleRowShared {
    union {
        unsigned long long list[kRowList];   // key << 32 | ~class
        StreamScratch stream;
    };
    union {
        BoundScratch bound;
        unsigned short groups[8 * kSampleThreads];
        unsigned bins[kBins];   // mass by the power's exponent
        struct {
            unsigned long long sums[kSampleWarps];
        } scan;
    };
    float fbuf[kSampleWarps];
    unsigned long long mass[kSampleWarps];
    int kept[kSampleWarps];
    unsigned n, n_groups, ties;
    int bin, last_bin;
    struct {
        uint32_t key;
        unsigned ties, slow;
        int last;   // class
    } found;
};

// The classes in order of their pieces: chunk 0 is the piece at the row's front
// that is not whole, chunk 1 + 8 q + w the 128 pieces of warp w's batch q, and
// the last chunk the piece at the end.
//
// Many rows, of any length: a block per row.  It streams the row once from
// memory for the largest and for the maxima of 2048 groups; what else a row
// needs streams it again, in part from L2 (four rows of 256 KB on every SM exceed
// it: 1024 x 131072 bf16 under mixed settings read 405 MB of DRAM for 268 MB):
//   top_k up to 1024 (and greedy rows): the groups that reach the bound are
//     read again, and their entries cut and drawn among as a list;
//   top_p alone: the mass of the row; then its bins of 1/64 octave down to
//     where top_p can end; then the exact mass above the bin in which it does,
//     by chunk, and that bin's entries as a list, in which the cut is found;
//   neither: the weights by chunk.
// The chunk that holds the draw is read once more by a warp.
template <typename T, bool kSupport>
__global__ void __launch_bounds__(kSampleThreads, 4)
sample_row_kernel(const T* __restrict__ X, long long ld, int V, Settings settings, Draw out) {
    using P = Piece<T>;
    constexpr int N = P::N, H = N / 2;
    extern __shared__ __align__(16) unsigned char raw[];
    unsigned long long* chunks = reinterpret_cast<unsigned long long*>(raw);   // kept weight by chunk
    __shared__ SampleRowShared s;
    grid_dependency_wait();
    allow_dependent_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = blockIdx.x;
    const T* x = X + row * ld;
    const RowSlice<T> slice(x, V, 0, 1);
    const PieceStream<T, kSampleThreads> stream(x, slice, V, tid);
    uint4 ua[4], ub[4];
    stream.load(0, ua);
    stream.load(1, ub);
    RowSettings set(settings, row, V);
    if (tid == 0) s.n = s.n_groups = s.ties = 0u;
    // every batch of the row to `use`, of which the first two are loaded
    auto stream_row = [&](auto&& use) {
        for (int q = 0; q < stream.batches; q += 2) {
            use(ua, q);
            if (q + 2 < stream.batches) stream.load(q + 2, ua);
            if (q + 1 < stream.batches) use(ub, q + 1);
            if (q + 3 < stream.batches) stream.load(q + 3, ub);
        }
    };
    // the pieces at the row's ends, of threads 0 and 32
    const int j_end = tid == 0 && slice.whole0() > 0 ? 0 : tid == 32 && slice.whole1(V) < slice.n ? slice.whole1(V) : -1;
    const uint4 u_end = j_end >= 0 ? end_piece(x, V, slice.first + j_end * N) : masked_piece<T>();
    const int last_chunk = 1 + kSampleWarps * stream.batches, end_chunk = tid == 0 ? 0 : last_chunk;

    typename P::Max mx[8];   // of even and of odd batches
#pragma unroll
    for (int i = 0; i < 8; ++i) mx[i] = P::lowest();
    stream_row([&](const uint4 (&u)[4], int q) {
        if (q & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mx[4 + i] = P::largest(mx[4 + i], u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) mx[i] = P::largest(mx[i], u[i]);
        }
    });
    float m = P::largest_of(u_end);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, P::value(mx[i]));
    m = block_largest(m, s.fbuf, kSampleWarps);
    if (m == BITLOGIC_NEG_INF) {   // nothing to draw from
        if (tid == 0) put_nothing<kSupport>(out, row);
        return;
    }
    const Power power(m, set);
    const PowerPairs pairs(power);

    auto list_entry = [&](float z, int v) {
        const unsigned at = atomicAdd(&s.n, 1u);
        if (at < kRowList) s.list[at] = ((unsigned long long)logit_key(z) << 32) | (uint32_t)~v;
    };
    if (set.k < V) {
        if (set.k > kListTop) {
            sample_of_stream<T, kSupport>(x, V, set, row, out, &s.stream);
            return;
        }
        float part[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) P::parts(P::either(mx[i], mx[4 + i]), part[2 * i], part[2 * i + 1]);
        const float z_min = set.k == 1 ? m : bound_logit(block_bound(part, set.k, &s.bound));
        __syncthreads();
        auto take = [&](const uint4& u, int j) {
            if (P::largest_of(u) >= z_min) {
                float z[N];
                P::load(u, z);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (z[i] >= z_min && z[i] > BITLOGIC_NEG_INF) list_entry(z[i], slice.first + j * N + i);
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
        for (unsigned p = tid; p < pieces; p += kSampleThreads) {
            const unsigned which = p / half, g = s.groups[which], q = 2 * (p - which * half) + (g >> 2 & 1u);
            const int j = slice.whole0() + stream.first_of((int)(g >> 3)) + 4 * kSampleThreads * (int)q + 32 * (int)(g & 3u);
            if (j < stream.j1) take(__ldcg(stream.from + j), j);
        }
        __syncthreads();
        const unsigned n = s.n;
        __syncthreads();
        if (n <= kRowList) sample_of_list<kSupport>(&s, n, set, power, row, out);
        else sample_of_stream<T, kSupport>(x, V, set, row, out, &s.stream);
        return;
    }

    Cut cut = {kNoCut, 0};
    float z_cut = BITLOGIC_NEG_INF;   // kept: above it, and the first ties at it
    if constexpr (kSupport) {
        if (set.p >= 1.0f) {   // min_p alone, or nothing
            if (set.floor_e > 0.f) last_kept(x, V, cut, set, power, row, out, &s.stream);
            else if (tid == 0) put_nothing<true>(out, row);
            return;
        }
    }
    stream.load(0, ua);
    stream.load(1, ub);
    if (set.p < 1.0f) {
        // the mass of the row
        for (int b = tid; b < kBins; b += kSampleThreads) s.bins[b] = 0u;
        unsigned long long mass = 0;
        stream_row([&](const uint4 (&u)[4], int) {
            WeightSum ws;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 z[H];
                load_pairs<T>(u[i], z);
#pragma unroll
                for (int e = 0; e < H; ++e) ws.add(pairs(z[e]));
            }
            mass += ws.total();
        });
        stream.load(0, ua);
        stream.load(1, ub);
        {
            WeightSum ws;
            f32x2 z[H];
            load_pairs<T>(u_end, z);
#pragma unroll
            for (int e = 0; e < H; ++e) ws.add(pairs(z[e]));
            mass += ws.total();
        }
        const unsigned long long total = block_add(mass, s.mass, kSampleWarps);
        unsigned long long want = share_of(total, set.p);
        if (want < 1) want = 1;
        // classes with less than a V-th of what top_p leaves off come after it
        const float left_off = fmaxf((float)(total - want) * (1.0f / 1099511627776.0f) / (float)V, 4.5474735e-13f);   // 2^-41 at least
        const float z_min = logit_below(left_off, power);
        auto count = [&](const uint4& u) {
            if (P::largest_of(u) >= z_min) {
                f32x2 z[H];
                load_pairs<T>(u, z);
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    float a, b;
                    unpack2(pairs(z[i]), a, b);
                    if (a >= left_off) atomicAdd(&s.bins[bin_of(a)], bin_units(a));
                    if (b >= left_off) atomicAdd(&s.bins[bin_of(b)], bin_units(b));
                }
            }
        };
        stream_row([&](const uint4 (&u)[4], int) {
#pragma unroll
            for (int i = 0; i < 4; ++i) count(u[i]);
        });
        stream.load(0, ua);
        stream.load(1, ub);
        count(u_end);
        __syncthreads();
        find_bin(s.bins, (float)want * (1.0f / 1099511627776.0f), &s.bin, &s.last_bin, s.fbuf);
        // the exact mass above the bins found, and its kept part by
        // chunk; the pieces that hold entries of those bins wait until the pass
        // is over (where the bins were)
        const float e_above = bin_above(first_bin(s.bin)), e_list = bin_above(end_bin(s.bin)), z_list = logit_below(e_list, power);
        __syncthreads();
        mass = 0;
        auto above = [&](const uint4& u, int j, WeightSum& kept, WeightSum& cut_off) {
            if (P::largest_of(u) < z_list) return;
            f32x2 z[H];
            load_pairs<T>(u, z);
            float rest = 0.f;   // the largest that is not above
#pragma unroll
            for (int i = 0; i < H; ++i) {
                float a, b;
                unpack2(pairs(z[i]), a, b);
                const float ra = a > e_above ? 0.f : a, rb = b > e_above ? 0.f : b;
                rest = fmaxf(rest, fmaxf(ra, rb));
                a -= ra;
                b -= rb;
                if (set.floor_e > 0.f) {   // counts for the cut, but is not kept
                    cut_off.add(pack2(a < set.floor_e ? a : 0.f, b < set.floor_e ? b : 0.f));
                    a = a < set.floor_e ? 0.f : a;
                    b = b < set.floor_e ? 0.f : b;
                }
                kept.add(pack2(a, b));
            }
            if (rest > e_list) {
                const unsigned at = atomicAdd(&s.n_groups, 1u);
                if (at < kBins) s.bins[at] = (unsigned)j;
            }
        };
        stream_row([&](const uint4 (&u)[4], int q) {
            WeightSum kept, cut_off;
#pragma unroll
            for (int i = 0; i < 4; ++i) above(u[i], stream.piece(q, i), kept, cut_off);
            mass += cut_off.total();
            const unsigned long long w = kept.warp_total();
            if (lane == 0) {
                chunks[1 + kSampleWarps * q + warp] = w;
                mass += w;
            }
        });
        if (tid == 0) chunks[0] = chunks[last_chunk] = 0ull;
        __syncthreads();
        if (j_end >= 0) {
            WeightSum kept, cut_off;
            above(u_end, j_end, kept, cut_off);
            chunks[end_chunk] = kept.total();
            mass += kept.total() + cut_off.total();
        }
        const unsigned long long first = block_add(mass, s.mass, kSampleWarps);
        const unsigned waiting = s.n_groups;
        for (unsigned i = tid; i < min(waiting, (unsigned)kBins) * N; i += kSampleThreads) {
            const int v = slice.first + (int)s.bins[i / N] * N + (int)(i % N);
            if (v >= 0 && v < V) {
                const float z = logit_value(x[v]), e = power.of(z);
                if (e > e_list && e <= e_above) list_entry(z, v);
            }
        }
        if (tid == 0) s.found = {0u, 0u, 1u, -1};   // not found: from memory
        __syncthreads();
        const unsigned listed = s.n;
        __syncthreads();
        if (waiting <= kBins && listed <= kRowList && listed > 0 && first < want)
            find_cut(s.list, listed, first, want, power, s.scan.sums, &s.found, [&](unsigned long long entry, float e, unsigned long long w) {
                if (e >= set.floor_e && w) {   // its weight to its chunk
                    const int j = ((int)~(uint32_t)entry - slice.first) / N - slice.whole0();
                    atomicAdd(&chunks[j < 0 ? 0 : j >= slice.whole1(V) - slice.whole0() ? last_chunk : 1 + j / 128], w);
                }
            });
        if (s.found.slow) {
            sample_of_stream<T, kSupport>(x, V, set, row, out, &s.stream);
            return;
        }
        cut = {s.found.key, s.found.ties};
        z_cut = key_logit(cut.key);
        if constexpr (kSupport) {
            if (power.of(z_cut) < set.floor_e) last_kept(x, V, cut, set, power, row, out, &s.stream);
            else if (tid == 0) put_support(out, row, z_cut, s.found.last);
            return;
        }
    } else {
        stream_row([&](const uint4 (&u)[4], int q) {
            WeightSum ws;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 z[H];
                load_pairs<T>(u[i], z);
#pragma unroll
                for (int e = 0; e < H; ++e) ws.add(pairs.at_least(z[e], set.floor_e));
            }
            const unsigned long long w = ws.warp_total();
            if (lane == 0) chunks[1 + kSampleWarps * q + warp] = w;
        });
        if (tid == 0) chunks[0] = chunks[last_chunk] = 0ull;
        __syncthreads();
        if (j_end >= 0) {
            WeightSum ws;
            f32x2 z[H];
            load_pairs<T>(u_end, z);
#pragma unroll
            for (int e = 0; e < H; ++e) ws.add(pairs.at_least(z[e], set.floor_e));
            chunks[end_chunk] = ws.total();
        }
        __syncthreads();
    }

    // the chunk that holds the draw, and what lies before it
    const int per = (last_chunk + kSampleThreads) / kSampleThreads;
    unsigned long long own = 0, total;
    for (int i = tid * per; i < min(last_chunk + 1, (tid + 1) * per); ++i) own += chunks[i];
    unsigned long long before = block_before(own, s.mass, &total);
    const unsigned long long target = share_of(total, set.u);
    if (tid == 0) s.kept[1] = -1;
    __syncthreads();
    if (target >= before && target < before + own) {
        int i = tid * per;
        while (target >= before + chunks[i]) before += chunks[i++];
        s.kept[0] = i;
        s.kept[1] = 0;
        s.mass[0] = before;
    }
    __syncthreads();
    if (warp != 0 || s.kept[1] < 0) return;
    // read by one warp, a piece per lane, in order
    const int chunk = s.kept[0], w0 = slice.whole0();
    const int c0 = chunk == 0 ? 0 : chunk == last_chunk ? slice.whole1(V) : w0 + (chunk - 1) * 128;
    const int c1 = chunk == 0 ? w0 : chunk == last_chunk ? slice.n : min(slice.whole1(V), c0 + 128);
    unsigned long long run = s.mass[0];
    unsigned my_left = 0;
    unsigned long long wt = 0;
    if (cut.ties) {
        const float e = power.of(z_cut);
        wt = e >= set.floor_e ? draw_weight(e) : 0ull;
        // ties before the chunk: all of them are on the list
        const int v_first = slice.first + c0 * N;
        unsigned ties = 0;
        for (unsigned i = lane; i < s.n; i += 32)
            ties += (uint32_t)(s.list[i] >> 32) == cut.key && (int)~(uint32_t)s.list[i] < v_first;
        ties = __reduce_add_sync(0xffffffffu, ties);
        my_left = (unsigned)cut.ties > ties ? (unsigned)cut.ties - ties : 0u;
    }
    for (int b = c0; b < c1; b += 32) {
        const int j = b + lane;
        float z[N];
        P::load(j >= c1 ? masked_piece<T>() : j >= w0 && j < slice.whole1(V) ? __ldcg(stream.from + j) : end_piece(x, V, slice.first + j * N), z);
        unsigned long long w[N], sum = 0;
        unsigned same = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) same += cut.ties && z[i] == z_cut;
        unsigned ties_before = same;
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned t = __shfl_up_sync(0xffffffffu, ties_before, o);
            if (lane >= o) ties_before += t;
        }
        const unsigned ties_all = __shfl_sync(0xffffffffu, ties_before, 31);
        ties_before -= same;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = 0ull;
            if (z[i] > z_cut) {
                const float e = power.of(z[i]);
                if (e >= set.floor_e) w[i] = draw_weight(e);
            } else if (cut.ties && z[i] == z_cut) {
                if (ties_before < my_left) w[i] = wt;
                ++ties_before;
            }
            sum += w[i];
        }
        const unsigned long long upto = warp_upto(sum, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, run + upto > target);
        if (hit) {
            if (lane == __ffs(hit) - 1) {
                unsigned long long r = run + upto - sum;
                bool done = false;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    r += w[i];
                    if (!done && r > target) {
                        done = true;
                        out.token[row] = slice.first + j * N + i;
                        if (out.logprob) out.logprob[row] = logf((float)w[i] / (float)total);
                    }
                }
            }
            return;
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
        my_left = my_left > ties_all ? my_left - ties_all : 0;
    }
}

// Rows of few classes: a warp per row, PER keys and weights in the registers of
// a lane (class 32 i + lane).  A weight is held as w = 2^21 high + low (see
// WeightSum), so that a warp's sums are two 32-bit reductions.
constexpr int kNarrow = 1024, kNarrowWarps = 8;

template <typename T, int PER, bool kSupport>
__global__ void __launch_bounds__(kNarrowWarps * 32)
sample_narrow_kernel(const T* __restrict__ X, long long ld, int V, long long rows, Settings settings, Draw out) {
    constexpr int kKeyBits = sizeof(T) == 2 ? 19 : 32;   // leading bits of a key that differ (fp16 fills 19)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    allow_dependent_launch();
    const long long row = (long long)blockIdx.x * kNarrowWarps + warp;
    if (row >= rows) return;
    const T* x = X + row * ld;
    RowSettings set(settings, row, V);
    float z[PER], m = BITLOGIC_NEG_INF;
#pragma unroll
    for (int i = 0; i < PER; ++i) z[i] = 32 * i + lane < V ? logit_value(x[32 * i + lane]) : BITLOGIC_NEG_INF;
#pragma unroll
    for (int i = 0; i < PER; ++i) m = fmaxf(m, z[i]);
    m = warp_largest(m);
    if (m == BITLOGIC_NEG_INF) {   // nothing to draw from
        if (lane == 0) put_nothing<kSupport>(out, row);
        return;
    }
    const Power power(m, set);
    uint32_t key[PER], high[PER];
    int low[PER];
    unsigned ranked = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        key[i] = logit_key(z[i]);
        ranked += ranks(key[i]);
        const float e = ranks(key[i]) ? power(z[i]) : 0.f, t = e + 16.0f;
        high[i] = __float_as_uint(t) - 0x41800000u;
        low[i] = (int)(__float_as_uint(fmaf(e - (t - 16.0f), 1099511627776.0f, 12582912.0f)) - 0x4b400000u);
        if (!ranks(key[i])) key[i] = 0u;
    }
    // the weight of the keys that `in` takes, over the warp
    auto weigh = [&](auto&& in) {
        unsigned h = 0;
        int l = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (in(key[i])) {
                h += high[i];
                l += low[i];
            }
        h = __reduce_add_sync(0xffffffffu, h);
        l = (int)__reduce_add_sync(0xffffffffu, (unsigned)l);
        return ((unsigned long long)h << 21) + (unsigned long long)(long long)l;
    };
    Cut cut = {kNoCut, 0};
    unsigned long long wt = 0;   // of a class at the cut
    auto weight_at = [&](uint32_t k) { return draw_weight(power(key_logit(k))); };
    if (set.k < V && (unsigned)set.k < __reduce_add_sync(0xffffffffu, ranked)) {
        uint32_t t = 0;
        unsigned reach = 0;
#pragma unroll 1
        for (uint32_t bit = 0x80000000u; bit > 0 && reach != (unsigned)set.k; bit >>= 1) {
            unsigned h = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) h += key[i] >= (t | bit);
            h = __reduce_add_sync(0xffffffffu, h);
            if (h >= (unsigned)set.k) {
                t |= bit;
                reach = h;
            }
        }
        unsigned above = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) above += key[i] > t;
        above = __reduce_add_sync(0xffffffffu, above);
        cut.key = t;
        cut.ties = set.k - above;
        if (cut.ties) wt = weight_at(cut.key);
    }
    if (set.p < 1.0f) {
        const uint32_t kt = cut.key;
        const unsigned long long mass = weigh([&](uint32_t k) { return k > kt; });
        unsigned long long want = share_of(mass + cut.ties * wt, set.p);
        if (want < 1) want = 1;
        if (want > mass) {   // reached among the ties of the top-k cut
            const unsigned long long need = wt ? (want - mass + wt - 1) / wt : cut.ties;
            if (need < cut.ties) cut.ties = need;
        } else {
            // the largest key that the mass is reached at, a bit at a time (the
            // bits of a key that the type does not fill follow the sign), until
            // one key is left in [t, t + bit)
            uint32_t t = 0;
#pragma unroll 1
            for (uint32_t bit = 0x80000000u; bit >= 1u << (32 - kKeyBits); bit >>= 1) {
                const uint32_t c = t | bit;
                if (weigh([&](uint32_t k) { return k >= c && k > kt; }) >= want) t = c;
                if (bit == 1u) break;
                if (bit & 0x00888800u) {   // a look at what is left, now and then
                    uint32_t lo = 0xffffffffu, hi = 0u;
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        const bool left = key[i] >= t && key[i] > kt && key[i] - t < bit;
                        lo = left ? min(lo, key[i]) : lo;
                        hi = left ? max(hi, key[i]) : hi;
                    }
                    if (__reduce_min_sync(0xffffffffu, lo) == __reduce_max_sync(0xffffffffu, hi)) break;
                }
            }
            uint32_t lowest = 0xffffffffu;
#pragma unroll
            for (int i = 0; i < PER; ++i) lowest = key[i] >= t && key[i] > kt ? min(lowest, key[i]) : lowest;
            t = __reduce_min_sync(0xffffffffu, lowest);
            const unsigned long long above = weigh([&](uint32_t k) { return k > t; });
            wt = weight_at(t);
            cut.key = t;
            cut.ties = wt ? (want - above + wt - 1) / wt : 1;
        }
    }
    unsigned left = (unsigned)cut.ties;
    const float floor_e = set.floor_e;
    if constexpr (kSupport) {
        if (set.k >= V && set.p >= 1.0f && floor_e == 0.f) {
            if (lane == 0) put_nothing<true>(out, row);
            return;
        }
        // the least key kept, and the last of its classes
        uint32_t least = 0xffffffffu;
        unsigned last = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const bool same = cut.ties && key[i] == cut.key;
            const unsigned mask = __ballot_sync(0xffffffffu, same);
            const bool kept = ranks(key[i]) && (key[i] > cut.key || (same && __popc(mask & ((1u << lane) - 1u)) < left)) &&
                              (floor_e == 0.f || power(key_logit(key[i])) >= floor_e);
            left -= min(left, (unsigned)__popc(mask));
            if (kept && key[i] <= least) {
                least = key[i];
                last = 32 * i + lane;
            }
        }
        const uint32_t all = __reduce_min_sync(0xffffffffu, least);
        last = __reduce_max_sync(0xffffffffu, least == all ? last : 0u);
        if (lane == 0) put_support(out, row, key_logit(all), (int)last);
        return;
    }
    // kept weights, then the draw: the 32 classes it falls in, and the class
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool same = cut.ties && key[i] == cut.key;
        const unsigned mask = __ballot_sync(0xffffffffu, same);
        const bool kept = (key[i] > cut.key || (same && __popc(mask & ((1u << lane) - 1u)) < left)) &&
                          (floor_e == 0.f || power(key_logit(key[i])) >= floor_e);
        left -= min(left, (unsigned)__popc(mask));
        if (!kept || !ranks(key[i])) high[i] = 0u, low[i] = 0;
    }
    const unsigned long long total = weigh([](uint32_t) { return true; }), target = share_of(total, set.u);
    unsigned long long before = 0, w = 0;
    int at = -1;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (at < 0) {
            const unsigned h = __reduce_add_sync(0xffffffffu, high[i]);
            const int l = (int)__reduce_add_sync(0xffffffffu, (unsigned)low[i]);
            const unsigned long long sum = ((unsigned long long)h << 21) + (unsigned long long)(long long)l;
            if (before + sum > target) {
                at = i;
                w = ((unsigned long long)high[i] << 21) + (unsigned long long)(long long)low[i];
            } else {
                before += sum;
            }
        }
    const unsigned long long upto = warp_upto(w, lane);
    const unsigned hit = __ballot_sync(0xffffffffu, before + upto > target);
    if (hit && lane == __ffs(hit) - 1) {
        out.token[row] = 32 * at + lane;
        if (out.logprob) out.logprob[row] = logf((float)w / (float)total);
    }
}

// Slices of at most kTileFit bytes leave room for three blocks on an SM beside
// their lists.
constexpr int kTileFit = 40 * 1024, kTileMost = 184 * 1024, kTileLeast = 8 * 1024;

// Shared memory of the chunks' weights of a row.
inline size_t chunk_bytes(int V, int element) {
    const long long pieces = slice_bytes(V, element, 1) / 16, batches = (pieces + 4 * kSampleThreads - 1) / (4 * kSampleThreads);
    return (size_t)(2 + kSampleWarps * batches) * 8;
}

template <typename T, bool kSupport>
int launch_sample(const T* x, long long T_, int V, long long ld, const Settings& set, const Draw& out,
                  cudaStream_t stream) {
    cudaError_t e;
    if (V <= kNarrow) {
        auto kern = V <= 32 ? sample_narrow_kernel<T, 1, kSupport> : V <= 128 ? sample_narrow_kernel<T, 4, kSupport>
                  : V <= 256 ? sample_narrow_kernel<T, 8, kSupport> : V <= 512 ? sample_narrow_kernel<T, 16, kSupport> : sample_narrow_kernel<T, 32, kSupport>;
        e = launch_rows(kern, (T_ + kNarrowWarps - 1) / kNarrowWarps, 1, kNarrowWarps * 32, 0, 0, stream, x, ld, V, T_, set, out);
    } else {
        // where a cluster per row is faster (50001 fp32 and 131072 bf16 classes:
        // top_k at 60 rows 21.4 and 21.6 against 17.1 and 18.7 us in a block each,
        // top_p at 100 rows 50.4 and 89 against 58 and 112 us, at 250 rows 111
        // and 180 against 68 and 131)
        const long long few = set.top_p ? sm_count() : sm_count() / 4;
        const int blocks = T_ <= few ? blocks_per_row(T_, V, sizeof(T), kTileFit, kTileMost, kTileLeast) : 0;
        if (blocks > 1) {
            e = launch_rows(sample_tile_kernel<T, kSupport>, T_, blocks, kSampleThreads, (size_t)slice_bytes(V, sizeof(T), blocks),
                            kTileMost, stream, x, ld, V, set, out);
        } else {
            e = launch_rows(sample_row_kernel<T, kSupport>, T_, 1, kSampleThreads, chunk_bytes(V, sizeof(T)),
                            chunk_bytes(kMaxClasses, sizeof(T)), stream, x, ld, V, set, out);
        }
    }
    return e == cudaSuccess ? launch_status() : (int)BITLOGIC_ERR_CUDA;
}

}  // namespace
}  // namespace bitlogic

using namespace bitlogic;

#ifndef BITLOGIC_SUPPORT_UNIT
extern "C" int bitlogic_sample_logits(const void* X, int32_t dtype, int64_t T, int32_t V, int64_t ld, const float* u,
                                      const float* temperature, const int32_t* top_k, const float* top_p,
                                      const float* min_p, int32_t* token, float* logprob, cudaStream_t stream) {
    if (int st = check_logits(X, dtype, true, T, V, ld)) return st;
    if (T == 0) return BITLOGIC_OK;
    if (!u || !token) return BITLOGIC_ERR_NULL;
    const Settings set = {u, temperature, top_k, top_p, min_p};
    const Draw out = {token, logprob, nullptr, nullptr};
    return with_logit_type(dtype, true, [&](auto* type) {
        return launch_sample<std::remove_const_t<std::remove_pointer_t<decltype(type)>>, false>(
            static_cast<decltype(type)>(X), T, V, ld, set, out, stream);
    });
}
#else
extern "C" int bitlogic_support_logits(const void* X, int32_t dtype, int64_t T, int32_t V, int64_t ld,
                                       const float* temperature, const int32_t* top_k, const float* top_p,
                                       const float* min_p, float* floor, int32_t* last, cudaStream_t stream) {
    if (int st = check_logits(X, dtype, true, T, V, ld)) return st;
    if (T == 0) return BITLOGIC_OK;
    if (!floor || !last) return BITLOGIC_ERR_NULL;
    const Settings set = {nullptr, temperature, top_k, top_p, min_p};
    const Draw out = {nullptr, nullptr, floor, last};
    return with_logit_type(dtype, true, [&](auto* type) {
        return launch_sample<std::remove_const_t<std::remove_pointer_t<decltype(type)>>, true>(
            static_cast<decltype(type)>(X), T, V, ld, set, out, stream);
    });
}
#endif
