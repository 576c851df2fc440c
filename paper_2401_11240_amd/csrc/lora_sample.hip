// gfx950 kernels of the next token of every row (include/lora_sample.h).
//
// A logit's order is that of a 32-bit key.  The way to the token:
//
//   1. the largest key of the row (weights are relative to it);
//   2. a histogram over bins of 1/16 in (l_max - l) / T: logits, and weights where they are needed, per bin.  From
//      its running sums come a first bin `lo` and a last bin `hi`: logits of bins below lo are kept by all
//      filters, those above hi by none (what lies past 32 weighs nothing);
//   3. the logits of bins lo .. hi in a list, in the order of their indices, and where lo is not 0 the
//      weights below it, summed by segments of the row;
//   4. in the list, which one workgroup holds, both thresholds exactly: the top_k-th largest logit and
//      the last one of the top_p start, found digit by digit of the key from sums per digit, from the largest down;
//      what equal logits share of a threshold goes to the lowest indices.  Then the segment, and
//      in it the logit, where the running sum passes the target.
//
// A list holds kList logits.  Rows that need a longer one (a top_k of thousands, thousands of equal logits at a
// threshold) are done by one workgroup from memory, digit by digit over the whole row (slow_row).
//
// Sums are whole numbers, so neither the order of atomic additions nor the division of a row over workgroups changes
// a bit.
#include <cmath>

#include <algorithm>

#include "lora_device.h"
#include "lora_mx_internal.h"
#include "lora_sample.h"

namespace lora {
namespace {

constexpr int kSampleThreads = 1024, kWaves = kSampleThreads / 64;
constexpr int kDigits = 2048;
constexpr int kBins = 512, kBinsPerNat = 16;   // the last bin: 31.9 and more, whose weights are zero
constexpr int kList = 4096;                // logits of a list
constexpr int kMaxSlices = 16;
constexpr int kMaxVocab = 1 << 19;
constexpr int kWeightBits = 43;            // sums of 2^19 weights stay below 2^62 (and exact)
constexpr double kOne = 8796093022208.0;   // 2^43
constexpr uint32_t kKeyNone = 0x007fffffu; // the key of -infinity

struct SampleArgs {
    const void* logits;
    int64_t ld;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* tokens;
    float* probs;
    unsigned char* ws;
    int64_t ws_row;                        // bytes of a row's workspace
    int n_vocab, slices;
};

template <int DT>
__device__ __forceinline__ float logit(const void* row, int i) {
    if (DT == LORA_F32) return ((const float*)row)[i];
    if (DT == LORA_F16) return FmtF16::to_f32(((const uint16_t*)row)[i]);
    return FmtBF16::to_f32(((const uint16_t*)row)[i]);
}

// Larger logits have larger keys, -0 and 0 the same; NaN is as -infinity.
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(l + 0.f);
    const uint32_t k = b ^ ((int)b < 0 ? 0xffffffffu : 0x80000000u);
    return l != l ? kKeyNone : k;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

// The weight 2^43 exp((l - max) / T), rounded: exp(d / T) = 2^(k / 64) e^r, k = round(64 d / (T ln 2)),
// |r| <= ln 2 / 128, 2^(k / 64) from a table of its 64 fractions and e^r by its series up to r^5 (the
// next term is below 4e-17).  Adding 2^52 leaves the rounded whole number in the low bits.
__device__ __forceinline__ uint64_t weight(uint32_t key, uint32_t top, double lmax, double rate, const double* frac) {
    if (key == top) return 1ull << kWeightBits;
    const double d = ((double)logit_of(key) - lmax) * rate;
    if (!(d > -64.0 * (kWeightBits + 2))) return 0;
    const double k = __builtin_rint(d);
    const double r = (d - k) * 0x1.62e42fefa39efp-7;          // ln 2 / 64
    double p = 1.0 / 120;
    p = fma(p, r, 1.0 / 24);
    p = fma(p, r, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const int ki = (int)k;
    const double v = ldexp(frac[ki & 63] * p, (ki >> 6) + kWeightBits);
    return (uint64_t)__double_as_longlong(v + 0x1p52) - 0x4330000000000000ull;
}

__device__ __forceinline__ uint64_t shfl_up64(uint64_t v, int d) { return __shfl_up((unsigned long long)v, d, 64); }
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int d) { return __shfl_xor((unsigned long long)v, d, 64); }

// What the filters leave open (step 2).
struct Cut {
    uint64_t all;                          // sum of all weights (0 where it is not needed)
    uint64_t below;                        // of bins below lo
    int mode, lo, hi, n;                   // kListed ..; the list's bins and logits
    int k_cuts;                            // whether top_k leaves out a logit that weighs anything
};
enum { kListed, kSlow };

struct Shared {
    unsigned long long hist[kDigits];      // per digit
    unsigned long long mass[kBins];
    uint32_t count[kBins], before[kBins];  // before: of the slices in front
    uint64_t list[kList];                  // key << 32 | index
    uint64_t segs[kMaxSlices * kWaves];
    double frac[64];
    uint64_t part[kWaves], parts[kWaves], ties[kWaves];
    uint64_t above;
    uint32_t digit;
    Cut cut;
};

// Sum over the workgroup, in every thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared& sh) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += shfl_xor64(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) v += sh.part[i];
    return v;
}

// The lowest digit that holds something and whose larger digits hold less than `limit`
// together with `above`; sh.digit, and sh.above what all larger ones hold.  Whole workgroup.
__device__ __forceinline__ void find_digit(uint64_t above, double limit, Shared& sh) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    // thread t: digits kDigits - 1 - 2 t and the one below, falling
    const int d0 = kDigits - 1 - 2 * t;
    const uint64_t a = sh.hist[d0], b = sh.hist[d0 - 1];
    uint64_t s = a + b;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = shfl_up64(s, d);
        if (l >= d) s += o;
    }
    if (l == 63) sh.parts[w] = s;
    if (t == 0) sh.digit = kDigits;
    __syncthreads();
    uint64_t before = above + s - a - b;
    for (int i = 0; i < w; ++i) before += sh.parts[i];
    uint32_t mine = kDigits;
    if (a && (double)before < limit) mine = d0;
    if (b && (double)(before + a) < limit) mine = d0 - 1;
    if (mine < kDigits) atomicMin(&sh.digit, mine);
    __syncthreads();
    if (sh.digit == mine && mine < kDigits) sh.above = mine == (uint32_t)d0 ? before : before + a;
    __syncthreads();
}

// A row's settings.
struct Row {
    const void* z;
    float T, p, m, lmax_f, bin_rate;
    double lmax, rate, least, u;           // least: the weight that min_p asks for
    int row, V, k;
    uint32_t top;
    int top_at;
    bool has_k, has_p, done;               // done: nothing to draw (nothing left, or the largest logit alone)

    __device__ __forceinline__ Row(const SampleArgs& a, int r, int dt) : row(r), V(a.n_vocab) {
        z = (const unsigned char*)a.logits + r * a.ld * (dt == LORA_F32 ? 4 : 2);
        T = a.temperature ? a.temperature[r] : 1.f;
        p = a.top_p ? a.top_p[r] : 1.f;
        m = a.min_p ? a.min_p[r] : 0.f;
        k = a.top_k ? a.top_k[r] : 0;
        const float uf = a.u[r];
        u = uf >= 1.f ? 1.0 : uf > 0.f ? (double)uf : 0.0;
        has_k = k > 0 && k < V;
        has_p = p < 1.f;
        least = m > 0.f ? (double)(m < 1.f ? m : 1.f) * kOne : 0;
    }
    // best: the largest key and, complemented, the lowest of its indices
    __device__ __forceinline__ void set_top(uint64_t best) {
        top = (uint32_t)(best >> 32);
        top_at = (int)(0xffffffffu - (uint32_t)best);
        done = top <= kKeyNone || !(T > 0.f);
        lmax_f = logit_of(top);
        lmax = lmax_f;
        rate = 64 * 1.4426950408889634 / (double)T;
        bin_rate = (float)kBinsPerNat / T;
    }
    __device__ __forceinline__ uint64_t weight_of(uint32_t key, const double* frac) const { return weight(key, top, lmax, rate, frac); }
    __device__ __forceinline__ uint64_t kept(uint64_t w) const { return (double)w >= least ? w : 0; }
    // (each step is monotone in the key; a difference that is not a number, of infinities, is the last bin)
    __device__ __forceinline__ int bin_of(uint32_t key) const {
        const float f = (lmax_f - logit_of(key)) * bin_rate;
        return key == top ? 0 : f < (float)(kBins - 1) ? (int)f : kBins - 1;
    }
    __device__ __forceinline__ void finish(const SampleArgs& a) const {
        a.tokens[row] = top <= kKeyNone ? -1 : top_at;
        if (a.probs) a.probs[row] = top <= kKeyNone ? 0.f : 1.f;
    }
    __device__ __forceinline__ void choose(const SampleArgs& a, int i, uint64_t w, uint64_t total) const {
        a.tokens[row] = i;
        if (a.probs) a.probs[row] = (float)((double)w / (double)total);
    }
    __device__ __forceinline__ uint64_t target(uint64_t total) const {
        const uint64_t t = (uint64_t)floor(u * (double)total);
        return t < total - 1 ? t : total - 1;
    }
};

// Thresholds of `n` logits, key(i) of the i-th: the whole workgroup calls it.  BY_WEIGHT: the sums are of
// weights, otherwise of ones, each with `above` in front of them; the lowest key whose larger ones sum to less than
// `limit`, and what they sum to.  With weights, keys below floor_key do not count and those of floor_key weigh
// floor_sum together.
template <bool BY_WEIGHT, class Key>
__device__ __forceinline__ uint32_t threshold(const Row& R, Shared& sh, int n, const Key& key_at, double limit, uint32_t floor_key,
                                              uint64_t floor_sum, uint64_t& above) {
    uint32_t prefix = 0;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
        __syncthreads();
        for (int i = threadIdx.x; i < kDigits; i += kSampleThreads) sh.hist[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kSampleThreads) {
            const uint32_t key = key_at(i);
            if (key <= kKeyNone || (level > 0 && (key >> (shift + bits)) != prefix)) continue;
            uint64_t v = 1;
            if (BY_WEIGHT) v = key > floor_key ? R.weight_of(key, sh.frac) : 0;
            if (v) atomicAdd(&sh.hist[(key >> shift) & ((1u << bits) - 1)], (unsigned long long)v);
        }
        if (BY_WEIGHT && threadIdx.x == 0 && floor_sum && (level == 0 || (floor_key >> (shift + bits)) == prefix))
            atomicAdd(&sh.hist[(floor_key >> shift) & ((1u << bits) - 1)], (unsigned long long)floor_sum);
        __syncthreads();
        find_digit(above, limit, sh);
        if (sh.digit >= kDigits) return kKeyNone;      // (nothing that weighs)
        prefix = prefix << bits | sh.digit;
        above = sh.above;
    }
    return prefix;
}

// Both thresholds over `n` logits that hold everything the filters leave open: kept are keys above
// tkey, and of those equal the first `share`.  all, below: of Cut, with `outside` logits' weights in
// them that are not among the n (0 and 0 if the n are the whole row).
template <class Key>
__device__ __forceinline__ void thresholds(const Row& R, Shared& sh, int n, const Key& key_at, bool has_k, uint64_t all, uint64_t below,
                                           uint32_t& tkey, uint32_t& share) {
    tkey = kKeyNone;
    share = 0;
    if (has_k) {
        uint64_t above = 0;
        tkey = threshold<false>(R, sh, n, key_at, (double)R.k, 0, 0, above);
        share = (uint32_t)(R.k - above);   // (at least 1; more than there are if few logits are left)
    }
    if (!R.has_p) return;
    if (!(R.p > 0.f)) {
        tkey = R.top;
        share = 1;
        return;
    }
    uint64_t floor_sum = 0;
    if (has_k || !all) {                   // the sum over K
        uint64_t sum = 0, ties = 0;
        for (int i = threadIdx.x; i < n; i += kSampleThreads) {
            const uint32_t key = key_at(i);
            if (key <= kKeyNone) continue;
            if (key > tkey) sum += R.weight_of(key, sh.frac);
            else if (key == tkey) ++ties;
        }
        sum = block_sum(sum, sh);
        ties = block_sum(ties, sh);
        if (tkey > kKeyNone) floor_sum = min((uint64_t)share, ties) * R.weight_of(tkey, sh.frac);
        all = sum + floor_sum;
    }
    const double limit = (double)R.p * (double)all;
    uint64_t above = below;
    const uint32_t key = threshold<true>(R, sh, n, key_at, limit, tkey, floor_sum, above);
    if (key <= kKeyNone) return;
    const uint64_t each = R.weight_of(key, sh.frac);
    // the first `few` of the equal ones begin below the limit
    uint32_t few = 1, most = key == tkey ? share : (uint32_t)R.V;
    while (few < most) {
        const uint32_t mid = few + (most - few + 1) / 2;
        if ((double)(above + (mid - 1) * each) < limit) few = mid;
        else most = mid - 1;
    }
    tkey = key;
    share = few;
}

// The row from memory by one workgroup, however it is.
template <int DT>
__device__ __noinline__ void slow_row(const SampleArgs& a, const Row& R, Shared& sh) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6, V = R.V;
    auto key_at = [&](int i) { return key_of(logit<DT>(R.z, i)); };
    uint32_t tkey, share;
    thresholds(R, sh, V, key_at, R.has_k, 0, 0, tkey, share);
    const uint64_t tie_weight = tkey > kKeyNone ? R.kept(R.weight_of(tkey, sh.frac)) : 0;
    // weights and ties of each wave's part of the row, in the order of the indices
    const int per = ((V + kWaves - 1) / kWaves + 63) & ~63;
    const int i0 = min(w * per, V), i1 = min(i0 + per, V);
    uint64_t sum = 0, ties = 0;
    for (int i = i0 + l; i < i1; i += 64) {
        const uint32_t key = key_at(i);
        if (key <= kKeyNone) continue;
        if (key > tkey) sum += R.kept(R.weight_of(key, sh.frac));
        else if (key == tkey) ++ties;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        sum += shfl_xor64(sum, d);
        ties += shfl_xor64(ties, d);
    }
    __syncthreads();
    if (l == 0) {
        sh.parts[w] = sum;
        sh.ties[w] = ties;
    }
    __syncthreads();
    uint64_t total = 0, at = 0, ties_before = 0, seen = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i == w) {
            at = total;
            ties_before = seen;
        }
        const uint64_t left = share > seen ? share - seen : 0;
        total += sh.parts[i] + min(left, sh.ties[i]) * tie_weight;
        seen += sh.ties[i];
    }
    const uint64_t target = R.target(total);
    // the wave in whose part the target lies comes to it
    for (int i = i0; i < i1; i += 64) {
        const uint32_t key = i + l < i1 ? key_at(i + l) : 0;
        const bool tie = key == tkey && key > kKeyNone;
        const uint64_t ballot = __ballot(tie);
        const uint64_t rank = ties_before + __popcll(ballot & ((1ull << l) - 1));
        uint64_t v = key > kKeyNone && key > tkey ? R.kept(R.weight_of(key, sh.frac)) : tie && rank < share ? tie_weight : 0;
        const uint64_t own = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t o = shfl_up64(v, d);
            if (l >= d) v += o;
        }
        if (own && at + v > target && at + v - own <= target) R.choose(a, i + l, own, total);
        at += __shfl((unsigned long long)v, 63, 64);
        ties_before += __popcll(ballot);
        if (at > target) break;
    }
}

// A slice of a row in registers: wave w holds 64 EPT consecutive logits, lane l every 64th of them.
template <int DT, int EPT>
struct Slice {
    uint32_t key[EPT];                     // 0 past the row
    int i0;                                // this lane's first
    __device__ __forceinline__ Slice(const Row& R, int slice) {
        i0 = (slice * kWaves + (threadIdx.x >> 6)) * 64 * EPT + (threadIdx.x & 63);
        float v[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) v[e] = i0 + 64 * e < R.V ? logit<DT>(R.z, i0 + 64 * e) : 0.f;
#pragma unroll
        for (int e = 0; e < EPT; ++e) key[e] = i0 + 64 * e < R.V ? key_of(v[e]) : 0u;
    }
    // Largest key and, complemented, the lowest of its indices: in every thread of the workgroup.
    __device__ __forceinline__ uint64_t best(Shared& sh) const {
        uint32_t k = 0;
        int at = i0;
#pragma unroll
        for (int e = 0; e < EPT; ++e)
            if (key[e] > k) {
                k = key[e];
                at = i0 + 64 * e;
            }
        uint64_t b = (uint64_t)k << 32 | (0xffffffffu - (uint32_t)at);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) b = max(b, shfl_xor64(b, d));
        if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = b;
        __syncthreads();
        for (int i = 0; i < kWaves; ++i) b = max(b, sh.part[i]);
        return b;
    }
};

// Whether the histogram has to hold weights: not where the list will be the top_k's.
__device__ __forceinline__ bool needs_mass(const Row& R) { return !(R.has_k && R.k <= kList); }

template <class S, int EPT>
__device__ __forceinline__ void fill_bins(const Row& R, Shared& sh, const S& s) {
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) {
        sh.count[i] = 0;
        sh.mass[i] = 0;
    }
    __syncthreads();
    const bool mass = needs_mass(R);
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        const uint32_t key = s.key[e];
        const int b = R.bin_of(key);
        if (key > kKeyNone && b < kBins - 1) {
            atomicAdd(&sh.count[b], 1u);
            if (mass) atomicAdd(&sh.mass[b], (unsigned long long)R.weight_of(key, sh.frac));
        }
    }
    __syncthreads();
}

// Step 2's decision from the row's histogram in sh.count and sh.mass; into sh.cut.
__device__ __forceinline__ void decide(const Row& R, Shared& sh) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    // running sums up to and with bin t
    uint64_t c = t < kBins ? sh.count[t] : 0, m = t < kBins ? sh.mass[t] : 0;
    const uint64_t own_m = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t oc = shfl_up64(c, d), om = shfl_up64(m, d);
        if (l >= d) {
            c += oc;
            m += om;
        }
    }
    if (l == 63) {
        sh.parts[w] = m;
        sh.ties[w] = c;
    }
    __syncthreads();
    uint64_t all = 0;
    for (int i = 0; i < kBins / 64; ++i) {
        if (i < w) {
            m += sh.parts[i];
            c += sh.ties[i];
        }
        all += sh.parts[i];
    }
    // the bin of the top_k-th logit, and the weights up to it, which K's are not above
    if (t == 0) {
        sh.digit = kBins - 1;
        sh.above = all;
    }
    __syncthreads();
    const uint64_t before = c - (t < kBins ? sh.count[t] : 0);
    if (R.has_k && t < kBins - 1 && before < (uint64_t)R.k && c >= (uint64_t)R.k) {
        sh.digit = t;
        sh.above = m;
    }
    __syncthreads();
    const int kb = sh.digit;
    const double limit = (double)R.p * (double)sh.above;
    __syncthreads();
    // the last bin that begins below top_p's limit (or, with K's sum smaller, later than that)
    if (t == 0) sh.digit = R.has_p && !(R.p > 0.f) ? 0 : kBins - 2;
    __syncthreads();
    const bool by_p = R.has_p && R.p > 0.f && needs_mass(R);
    if (by_p && t < kBins - 1 && own_m && (double)(m - own_m) < limit && (double)m >= limit) sh.digit = t;
    __syncthreads();
    const int pb = sh.digit;
    __syncthreads();
    // bins in which min_p may cut, with a bin to spare on either side for the roundings
    int m0 = kBins - 1, m1 = kBins - 2;
    if (R.least > 0) {
        const float f = (float)kBinsPerNat * -logf((float)(R.least / kOne));
        // (weights of a few units are rounded by up to ln 2)
        const int spare = R.least < 256 ? 12 : 1;
        if (f < (float)(kBins - 2)) {
            m0 = max((int)f - spare, 0);
            m1 = (int)f + spare;
        }
    }
    const bool k_cuts = R.has_k && kb < kBins - 1;
    // (top_p needs the sum over K: all of it is in the list, if the bins do not have the row's)
    const bool whole_k = R.has_p && R.p > 0.f && (k_cuts || !needs_mass(R));
    const int hi = whole_k ? min(kb, kBins - 2) : min(min(kb, pb), min(m1, kBins - 2));
    if (t == hi) {                         // all of it fits the list, or else ...
        sh.digit = c <= (uint64_t)kList;
        sh.cut.n = (int)min(c, (uint64_t)1 << 30);
    }
    __syncthreads();
    int lo = 0;
    if (!sh.digit) lo = !R.has_p && R.least <= 0 ? kBins - 1 : min(pb < kBins - 2 || by_p ? pb : kBins - 1, m0);
    if (t == 0) {
        sh.cut.lo = lo;
        sh.cut.hi = hi;
        sh.cut.all = needs_mass(R) && !k_cuts ? all : 0;
        sh.cut.below = 0;
        sh.cut.mode = kListed;
        sh.cut.k_cuts = k_cuts;
        if (!sh.digit && (lo == 0 || k_cuts || !needs_mass(R))) sh.cut.mode = kSlow;
        if (lo > hi) sh.cut.n = 0;
    }
    __syncthreads();
    if (lo > 0) {                          // ... its last bins, with what is kept below them
        if (t == lo - 1) {
            sh.cut.below = m;
            sh.above = c;
        }
        __syncthreads();
        if (t == hi && lo <= hi) {
            const uint64_t n = c - sh.above;
            sh.cut.n = (int)min(n, (uint64_t)1 << 30);
            if (n > (uint64_t)kList) sh.cut.mode = kSlow;
        }
    }
    __syncthreads();
}

// Step 3 for a slice: its logits of the cut's bins into `list`, from entry `first` on in the order of their indices,
// and, where lo is not 0, each wave's sum of weights below it into segs.
template <class S, int EPT>
__device__ __forceinline__ void collect(const Row& R, Shared& sh, const S& s, int first, uint64_t* list, uint64_t* segs) {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int lo = sh.cut.lo, hi = sh.cut.hi;
    int mine = 0;
    uint64_t sum = 0;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        const uint32_t key = s.key[e];
        const int b = key > kKeyNone ? R.bin_of(key) : kBins;
        mine += __popcll(__ballot(b >= lo && b <= hi));
        if (lo > 0 && b < lo && b <= hi) sum += R.weight_of(key, sh.frac);
    }
    if (lo > 0) {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) sum += shfl_xor64(sum, d);
        if (l == 0) segs[w] = sum;
    }
    __syncthreads();
    if (l == 0) sh.ties[w] = mine;
    __syncthreads();
    for (int i = 0; i < w; ++i) first += (int)sh.ties[i];
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        const uint32_t key = s.key[e];
        const int b = key > kKeyNone ? R.bin_of(key) : kBins;
        const bool in = b >= lo && b <= hi;
        const uint64_t ballot = __ballot(in);
        const int at = first + __popcll(ballot & ((1ull << l) - 1));
        if (in && at < kList) list[at] = (uint64_t)key << 32 | (uint32_t)(s.i0 + 64 * e);
        first += __popcll(ballot);
    }
    __syncthreads();
}

// Step 4, from the list and the segments' sums in sh.  EPT: the slices' (a segment is a wave's share of a slice).
template <int DT, int EPT>
__device__ __forceinline__ void pick(const SampleArgs& a, const Row& R, Shared& sh) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    constexpr int kSeg = 64 * EPT, kEach = kList / kSampleThreads;
    const Cut cut = sh.cut;
    const int n = cut.n;
    auto key_at = [&](int i) { return (uint32_t)(sh.list[i] >> 32); };
    uint32_t tkey = kKeyNone, share = 0;
    if (n > 0) thresholds(R, sh, n, key_at, cut.k_cuts, cut.all, cut.below, tkey, share);
    const uint64_t tie_weight = tkey > kKeyNone ? R.kept(R.weight_of(tkey, sh.frac)) : 0;
    // thread t: entries kEach t ..; ranks of equal ones, then kept weights, then their running sums
    uint64_t v[kEach], ties = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = kEach * t + j;
        const uint32_t key = i < n ? key_at(i) : 0;
        v[j] = key > tkey && key > kKeyNone ? R.kept(R.weight_of(key, sh.frac)) : 0;
        ties += key == tkey && key > kKeyNone;
    }
    auto scan = [&](uint64_t x) {          // exclusive, over the workgroup; sh.above: the sum
        uint64_t s = x;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t o = shfl_up64(s, d);
            if (l >= d) s += o;
        }
        __syncthreads();
        if (l == 63) sh.parts[w] = s;
        __syncthreads();
        uint64_t before = 0, all = 0;
        for (int i = 0; i < kWaves; ++i) {
            if (i < w) before += sh.parts[i];
            all += sh.parts[i];
        }
        if (t == 0) sh.above = all;
        return before + s - x;
    };
    uint64_t rank = scan(ties);
    uint64_t mine = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = kEach * t + j;
        const uint32_t key = i < n ? key_at(i) : 0;
        if (key == tkey && key > kKeyNone) {
            if (rank < share) v[j] = tie_weight;
            ++rank;
        }
        mine += v[j];
    }
    if (cut.lo == 0) {
        const uint64_t at = scan(mine);
        __syncthreads();
        const uint64_t total = sh.above, target = R.target(total);
        uint64_t run = at;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (v[j] && run <= target && target < run + v[j]) R.choose(a, (int)(uint32_t)sh.list[kEach * t + j], v[j], total);
            run += v[j];
        }
        return;
    }
    // the list's kept weights into their segments; the first of equal ones that is not kept, in tie_end
    const int n_segs = a.slices * kWaves;
    if (t == 0) sh.digit = 0x7fffffff;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = kEach * t + j;
        if (v[j]) atomicAdd((unsigned long long*)&sh.segs[(uint32_t)sh.list[i] / kSeg], (unsigned long long)v[j]);
        else if (i < n && key_at(i) == tkey) atomicMin(&sh.digit, (uint32_t)sh.list[i]);
    }
    __syncthreads();
    const uint32_t tie_end = sh.digit;
    const uint64_t s = t < n_segs ? sh.segs[t] : 0;
    const uint64_t at = scan(s);
    __syncthreads();
    const uint64_t total = sh.above, target = R.target(total);
    if (s && at <= target && target < at + s) {
        sh.digit = t;
        sh.part[0] = at;
    }
    __syncthreads();
    // the segment again
    const int seg = sh.digit;
    const uint64_t begin = sh.part[0];
    constexpr int kOf = EPT >= 16 ? EPT / 16 : 1;      // consecutive logits of a thread
    uint64_t x[kOf], sum = 0;
#pragma unroll
    for (int j = 0; j < kOf; ++j) {
        const int o = t * kOf + j, i = seg * kSeg + o;
        const uint32_t key = o < kSeg && i < R.V ? key_of(logit<DT>(R.z, i)) : 0;
        const int b = key > kKeyNone ? R.bin_of(key) : kBins;
        x[j] = 0;
        if (b <= cut.hi && key >= tkey && (key != tkey || (uint32_t)i < tie_end)) x[j] = R.weight_of(key, sh.frac);
        if (b >= cut.lo) x[j] = R.kept(x[j]);
        sum += x[j];
    }
    uint64_t run = begin + scan(sum);
#pragma unroll
    for (int j = 0; j < kOf; ++j) {
        if (x[j] && run <= target && target < run + x[j]) R.choose(a, seg * kSeg + t * kOf + j, x[j], total);
        run += x[j];
    }
}

__device__ __forceinline__ void fill_fractions(Shared& sh) {
    if (threadIdx.x < 64) sh.frac[threadIdx.x] = exp2(threadIdx.x / 64.0);
}

// Rows that one workgroup holds.
template <int DT, int EPT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_row_kernel(SampleArgs a) {
    __shared__ Shared sh;
    Row R(a, blockIdx.x, DT);
    using S = Slice<DT, EPT>;
    S s(R, 0);
    fill_fractions(sh);
    R.set_top(s.best(sh));
    if (R.done) {
        if (threadIdx.x == 0) R.finish(a);
        return;
    }
    __syncthreads();
    fill_bins<S, EPT>(R, sh, s);
    decide(R, sh);
    if (sh.cut.mode == kSlow) {
        slow_row<DT>(a, R, sh);
        return;
    }
    collect<S, EPT>(R, sh, s, 0, sh.list, sh.segs);
    pick<DT, EPT>(a, R, sh);
}

// Rows of several slices, a launch for each of the four steps.  A row's workspace: every slice's best, counts and
// weights per bin, segment sums; the list; the cut.
struct RowSpace {
    uint64_t *best, *mass, *segs, *list;
    uint32_t* count;
    Cut* cut;
    __host__ __device__ RowSpace(unsigned char* p, int slices) {
        cut = (Cut*)p;
        best = (uint64_t*)(p + 64);
        mass = best + kMaxSlices;
        segs = mass + (int64_t)slices * kBins;
        list = segs + (int64_t)slices * kWaves;
        count = (uint32_t*)(list + kList);
    }
    static int64_t bytes(int slices) { return 64 + 8ll * (kMaxSlices + slices * (kBins + kWaves) + kList) + 4ll * slices * kBins; }
};

__device__ __forceinline__ uint64_t row_best(const RowSpace& ws, int slices) {
    uint64_t b = 0;
    for (int i = 0; i < slices; ++i) b = max(b, ws.best[i]);
    return b;
}

template <int DT, int EPT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_best_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const Row R(a, blockIdx.y, DT);
    const Slice<DT, EPT> s(R, blockIdx.x);
    const uint64_t b = s.best(sh);
    if (threadIdx.x == 0) RowSpace(a.ws + blockIdx.y * a.ws_row, a.slices).best[blockIdx.x] = b;
}

template <int DT, int EPT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_bins_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const RowSpace ws(a.ws + blockIdx.y * a.ws_row, a.slices);
    Row R(a, blockIdx.y, DT);
    using S = Slice<DT, EPT>;
    const S s(R, blockIdx.x);
    fill_fractions(sh);
    R.set_top(row_best(ws, a.slices));
    if (R.done) return;
    __syncthreads();
    fill_bins<S, EPT>(R, sh, s);
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) {
        ws.count[blockIdx.x * kBins + i] = sh.count[i];
        ws.mass[blockIdx.x * kBins + i] = sh.mass[i];
    }
}

template <int DT, int EPT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_list_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const RowSpace ws(a.ws + blockIdx.y * a.ws_row, a.slices);
    Row R(a, blockIdx.y, DT);
    using S = Slice<DT, EPT>;
    const S s(R, blockIdx.x);
    fill_fractions(sh);
    R.set_top(row_best(ws, a.slices));
    if (R.done) return;
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) {
        uint32_t c = 0, before = 0;
        uint64_t m = 0;
        for (int j = 0; j < a.slices; ++j) {
            if (j == (int)blockIdx.x) before = c;
            c += ws.count[j * kBins + i];
            m += ws.mass[j * kBins + i];
        }
        sh.count[i] = c;
        sh.before[i] = before;
        sh.mass[i] = m;
    }
    __syncthreads();
    decide(R, sh);
    if (blockIdx.x == 0 && threadIdx.x == 0) *ws.cut = sh.cut;
    if (sh.cut.mode == kSlow) return;
    const int t = threadIdx.x;
    const int first = (int)block_sum(t < kBins && t >= sh.cut.lo && t <= sh.cut.hi ? sh.before[t] : 0, sh);
    collect<S, EPT>(R, sh, s, first, ws.list, ws.segs + blockIdx.x * kWaves);
}

template <int DT, int EPT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_pick_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const RowSpace ws(a.ws + blockIdx.x * a.ws_row, a.slices);
    Row R(a, blockIdx.x, DT);
    fill_fractions(sh);
    R.set_top(row_best(ws, a.slices));
    if (R.done) {
        if (threadIdx.x == 0) R.finish(a);
        return;
    }
    if (threadIdx.x == 0) sh.cut = *ws.cut;
    __syncthreads();
    if (sh.cut.mode == kSlow) {
        slow_row<DT>(a, R, sh);
        return;
    }
    for (int i = threadIdx.x; i < sh.cut.n; i += kSampleThreads) sh.list[i] = ws.list[i];
    if (sh.cut.lo > 0)
        for (int i = threadIdx.x; i < a.slices * kWaves; i += kSampleThreads) sh.segs[i] = ws.segs[i];
    __syncthreads();
    pick<DT, EPT>(a, R, sh);
}

// Slices of a row: kSampleThreads * ept logits each.
struct SamplePlan {
    int ept, slices;
};

SamplePlan plan_sample(int n_rows, int n_vocab) {
    SamplePlan p{};
    for (p.ept = 8; p.ept < 32; p.ept *= 2) {
        const int64_t per = (int64_t)kSampleThreads * p.ept;
        p.slices = (int)((n_vocab + per - 1) / per);
        if (p.slices <= kMaxSlices && (int64_t)n_rows * p.slices <= 512) break;
    }
    p.slices = (int)((n_vocab + (int64_t)kSampleThreads * p.ept - 1) / ((int64_t)kSampleThreads * p.ept));
#ifdef MX_PROBE
    if (const char* e = getenv("SA_EPT")) { p.ept = atoi(e); p.slices = (int)((n_vocab + (int64_t)kSampleThreads * p.ept - 1) / ((int64_t)kSampleThreads * p.ept)); }
#endif
    return p;
}

template <int DT, int EPT>
void launch_sample(const SampleArgs& a, int n_rows, hipStream_t st) {
    const dim3 block(kSampleThreads);
    if (a.slices == 1) {
        hipLaunchKernelGGL((lora_sample_row_kernel<DT, EPT>), dim3(n_rows), block, 0, st, a);
        return;
    }
    const dim3 grid(a.slices, n_rows);
    hipLaunchKernelGGL((lora_sample_best_kernel<DT, EPT>), grid, block, 0, st, a);
    hipLaunchKernelGGL((lora_sample_bins_kernel<DT, EPT>), grid, block, 0, st, a);
    hipLaunchKernelGGL((lora_sample_list_kernel<DT, EPT>), grid, block, 0, st, a);
    hipLaunchKernelGGL((lora_sample_pick_kernel<DT, EPT>), dim3(n_rows), block, 0, st, a);
}

template <int DT>
void launch_sample(const SampleArgs& a, int ept, int n_rows, hipStream_t st) {
    if (ept == 8) launch_sample<DT, 8>(a, n_rows, st);
    else if (ept == 16) launch_sample<DT, 16>(a, n_rows, st);
    else launch_sample<DT, 32>(a, n_rows, st);
}

}  // namespace
}  // namespace lora

using namespace lora;

extern "C" {

int lora_sample_workspace_bytes(int32_t n_rows, int32_t n_vocab, int32_t dtype, size_t* bytes) {
    if (n_rows < 0) return set_error(LORA_E_ARG, "negative n_rows");
    if (n_vocab < 1 || n_vocab > kMaxVocab) return set_error(LORA_E_SHAPE, "n_vocab must be in [1, 2^19]");
    if (dtype != LORA_F16 && dtype != LORA_BF16 && dtype != LORA_F32)
        return set_error(LORA_E_ARG, "dtype must be LORA_F16, LORA_BF16 or LORA_F32");
    if (!bytes) return set_error(LORA_E_ARG, "bytes is NULL");
    const SamplePlan p = plan_sample(n_rows, n_vocab);
    *bytes = p.slices > 1 ? std::max<size_t>(16, (size_t)n_rows * RowSpace::bytes(p.slices)) : 16;
    return LORA_OK;
}

int lora_sample(const void* logits, int64_t ld, int32_t dtype, int32_t n_rows, int32_t n_vocab,
                const lora_sample_t* params, const float* u, int32_t* tokens, float* probs, void* ws, size_t ws_bytes,
                void* stream) {
    size_t need = 0;
    if (int rc = lora_sample_workspace_bytes(n_rows, n_vocab, dtype, &need)) return rc;
    if (ld < n_vocab || ld > (1ll << 40)) return set_error(LORA_E_SHAPE, "ld must be n_vocab to 2^40");
    if (n_rows > 0 && (!logits || !u || !tokens)) return set_error(LORA_E_ARG, "logits, u or tokens is NULL");
    const int64_t e = dtype == LORA_F32 ? 4 : 2;
    if ((uintptr_t)logits % (uintptr_t)e) return set_error(LORA_E_ALIGN, "logits not aligned to their elements");
    const lora_sample_t none = {nullptr, nullptr, nullptr, nullptr};
    if (!params) params = &none;
    const void* words[7] = {params->temperature, params->top_k, params->top_p, params->min_p, u, tokens, probs};
    for (const void* p : words)
        if ((uintptr_t)p & 3u) return set_error(LORA_E_ALIGN, "parameters, u, tokens and probs must be 4-byte aligned");
    if (!ws || ws_bytes < need) return set_error(LORA_E_WORKSPACE, "workspace smaller than lora_sample_workspace_bytes");
    if (!is_aligned16(ws)) return set_error(LORA_E_ALIGN, "ws not 16-byte aligned");
    Span in[6] = {Span(logits, n_rows, ld * e, n_vocab * e)};
    for (int i = 0; i < 5; ++i) in[1 + i] = Span(words[i], 1, 0, 4ll * n_rows);
    const Span out[3] = {Span(tokens, 1, 0, 4ll * n_rows), Span(probs, 1, 0, 4ll * n_rows), Span(ws, 1, 0, (int64_t)need)};
    for (int i = 0; i < 3; ++i) {
        for (const Span& s : in)
            if (out[i].meets(s)) return set_error(LORA_E_OVERLAP, "an output or ws overlaps an input");
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return set_error(LORA_E_OVERLAP, "tokens, probs and ws overlap");
    }
    if (n_rows == 0) return LORA_OK;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_sample: no device for the stream");
    SampleArgs a;
    a.logits = logits;
    a.ld = ld;
    a.temperature = params->temperature;
    a.top_p = params->top_p;
    a.min_p = params->min_p;
    a.u = u;
    a.top_k = params->top_k;
    a.tokens = tokens;
    a.probs = probs;
    a.n_vocab = n_vocab;
    a.ws = (unsigned char*)ws;
    const SamplePlan p = plan_sample(n_rows, n_vocab);
    a.slices = p.slices;
    a.ws_row = RowSpace::bytes(p.slices);
    if (dtype == LORA_F16) launch_sample<LORA_F16>(a, p.ept, n_rows, st);
    else if (dtype == LORA_BF16) launch_sample<LORA_BF16>(a, p.ept, n_rows, st);
    else launch_sample<LORA_F32>(a, p.ept, n_rows, st);
    return check_launch("lora_sample");
}

}  // extern "C"
