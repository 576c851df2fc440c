// gfx950 kernels of the next token of every row (include/lora_sample.h).
//
// The way to the token:
//
//   1. the largest logit of the row (weights are relative to it);
//   2. a histogram over bins of 1/32 in (l_max - l) / T: logits and weights per bin.  From its running sums come a
//      first bin `lo` and a last bin `hi`: logits of bins below lo are kept by all filters, those above hi by none
//      (what lies past 32 weighs nothing).  Where top_k is small, every thread's largest logit is enough: at
//      least top_k logits are as large as the top_k-th of those, and not many more;
//   3. the logits of bins lo .. hi in a list, in the order of their indices, and where lo is not 0 the
//      weights below it, summed by segments of the row;
//   4. one workgroup finds the last logit of the list that is kept (by comparing all with all where they are few, else with a
//      finer histogram, whose one bin at the border is compared, or is sorted with the list where it is large); then, in the
//      order of the indices again, the segment and in it the logit where the running sum passes the target.
//
// Where there are rows enough a workgroup takes a row all the way, otherwise a row is divided into slices, a workgroup
// each, with a launch for each step.  A list holds kList logits, a sixteenth for each wave of a workgroup; where a wave has more
// (the likely logits are neighbours) the waves collect again, in any order, and the token's segment is read once more.  Rows that
// need a longer list (a top_k of thousands,
// thousands of equal logits at a threshold) are done by one workgroup, thresholds digit by digit of an ordered key (slow_row).
//
// Sums are whole numbers, so neither the order of atomic additions nor the division of a row over workgroups changes
// a bit.
//
// What bounds it: a few rows, the four launches (3 to 9 us each in a trace; one row of 32000: 22 us, most of it the way of the first loads, of
// code that every workgroup runs through once, and of barriers of sixteen waves); many rows with top_p and no small top_k (64 rows of
// 128000 in bfloat16: 49 us), that a compute unit has one workgroup: its 1024 threads take 72 to 98 registers each in the launches
// that weigh 16-bit logits, of 64 that two workgroups would leave them, so nothing runs beside what it waits for (first loads, atomic
// additions, barriers).  The weights by themselves, about 20 binary64 instructions of 4 cycles, are 4 us of the 32000 logits of a
// workgroup, twice that where the list does not hold all that is kept or where nothing but min_p filters; and in a batch of
// all kinds the workgroups of the rows with a small top_k have none of that work.  Many rows with a small top_k: the reading of the logits
// (256 x 50257 in float32: 21 us, 51 MB, of which 8 are that reading, 3 the second, of the threads that have a listed logit, and 8 the
// way from there to the token, through some twenty barriers of sixteen waves).
#include <cmath>

#include <algorithm>

#include "lora_device.h"
#include "lora_mx_internal.h"
#include "lora_sample.h"

namespace lora {
namespace {

constexpr int kSampleThreads = 1024, kWaves = kSampleThreads / 64;
constexpr int kDigits = 2048;
constexpr int kBins = 1024, kBinsPerNat = 32;  // the last bin: 31.9 and more, whose weights are zero
constexpr int kList = 4096;                // logits of a list
constexpr int kWaveList = kList / kWaves;  // of one wave's part of it
constexpr int kFits = kList * 3 / 4;       // up to which the waves' parts are expected to hold them
constexpr int kRanked = 256;               // up to which a list is ranked by comparing all with all
constexpr int kSmallK = 512;               // top_k up to which threads' largest logits bound it
constexpr int kMaxSlices = 16;
constexpr int kMaxVocab = 1 << 19;
constexpr int kLaunchRows = 1 << 20;       // of one launch: its threads stay below 2^32
constexpr float kLeastT = 0x1p-100f, kMostT = 0x1p100f;   // within which bins and logits' differences stay in range
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
    int seg;                               // logits of a wave's segment
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

// Larger for larger logits, of equal ones for the lowest index.
__device__ __forceinline__ uint64_t ranked(float l, int i) { return (uint64_t)key_of(l) << 32 | (0xffffffffu - (uint32_t)i); }
__device__ __forceinline__ int index_of(uint64_t r) { return (int)(0xffffffffu - (uint32_t)r); }

// The weight 2^43 exp((l - max) / T), rounded: exp(d / T) = 2^(k / 64) 2^(x / 64) with k + x = 64 d / (T ln 2), k whole and
// |x| at most 1/2.  2^(43 + k / 64) comes from a table of its 64 fractions, 2^(x / 64) from its series in x up to x^5 (the
// next term is below 4e-17).  Adding 1.5 2^52 leaves the whole number k in the low bits, adding 2^52 the rounded weight.
// (Without branches, so that several run side by side: their number of instructions is what the histogram costs.)
__device__ __forceinline__ uint64_t weight(float l, double lmax, double rate, const double* frac) {
    constexpr double c = 0x1.62e42fefa39efp-7;                // ln 2 / 64
    double d = ((double)l - lmax) * rate;
    d = __builtin_fmin(__builtin_fmax(d, -64.0 * (kWeightBits + 2)), 0.0);   // (rounds to nothing; infinities)
    const double kd = d + 0x1.8p52, x = d - (kd - 0x1.8p52);
    const int k = (int)(uint32_t)__double_as_longlong(kd);
    double p = c * c * c * c * c / 120;
    p = fma(p, x, c * c * c * c / 24);
    p = fma(p, x, c * c * c / 6);
    p = fma(p, x, c * c / 2);
    p = fma(p, x, c);
    p = fma(p, x, 1.0);
    return (uint64_t)__double_as_longlong(fma(ldexp(frac[k & 63], k >> 6), p, 0x1p52)) - 0x4330000000000000ull;
}

// The value of the lane that the DPP control names, in the rows of ROWS; 0 elsewhere and where there is none.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t moved(uint64_t v) {
    return (uint64_t)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v);
}
// Sums over the four lanes of a quad, in all four.
template <class T>
__device__ __forceinline__ T quad_sum(T v) {
    v += moved<0xB1>(v);                   // lanes 1 0 3 2
    return v + moved<0x4E>(v);             // lanes 2 3 0 1
}
// f over the lanes up to and with each of a wave's 64, all of them active (0 must change nothing): over 1, 2, 4 and 8 lanes
// of a row of 16, then the rows' ends into the rows behind them.
template <class T, class F>
__device__ __forceinline__ T wave_scan(T v, const F& f) {
    v = f(v, moved<0x111>(v));             // 1 lane down
    v = f(v, moved<0x112>(v));
    v = f(v, moved<0x114>(v));
    v = f(v, moved<0x118>(v));
    v = f(v, moved<0x142, 0xa>(v));        // a row's last lane to rows 1 and 3
    return f(v, moved<0x143, 0xc>(v));     // lane 31 to rows 2 and 3
}
template <class T>
__device__ __forceinline__ T wave_sums(T v) {
    return wave_scan(v, [](T a, T b) { return a + b; });
}
// A lane's value, in every lane; l is the same in all.
__device__ __forceinline__ uint32_t at_lane(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ uint64_t at_lane(uint64_t v, int l) { return (uint64_t)at_lane((uint32_t)(v >> 32), l) << 32 | at_lane((uint32_t)v, l); }
template <class T>
__device__ __forceinline__ T wave_sum(T v) { return at_lane(wave_sums(v), 63); }
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    return at_lane(wave_scan(v, [](uint64_t a, uint64_t b) { return max(a, b); }), 63);
}

// Of the sums of a workgroup's waves, one behind the other in LDS: what lies in front of this wave's, and their whole.  (By
// lanes: sixteen conditional additions are four times the code, and a workgroup that runs through code once waits for it.)
template <class T>
__device__ __forceinline__ T in_front(const T* sums, T& all) {
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T own = sums[l & (kWaves - 1)];
    T v = own + moved<0x111>(own);         // (a row of 16 lanes holds all)
    v += moved<0x112>(v);
    v += moved<0x114>(v);
    v += moved<0x118>(v);
    all = at_lane(v, kWaves - 1);
    return at_lane(T(v - own), w);
}
static_assert(kWaves == 16, "a lane of a row for each wave");

// What the filters leave open (step 2).
struct Cut {                               // (read as whole words)
    uint64_t all;                          // sum of all weights (0 where it is not needed)
    uint64_t below;                        // of bins below lo
    int lo, hi;                            // the list's bins
    int k_cuts;                            // whether top_k may leave out a logit that weighs anything
    int slow;
};

struct Shared {
    unsigned long long hist[kDigits];      // per digit
    unsigned long long mass[kBins];
    uint32_t count[kBins];
    uint64_t list[kList];                  // ranked() of logits
    uint64_t weights[kRanked];
    uint64_t segs[kMaxSlices * kWaves];
    uint32_t seg_n[kMaxSlices * kWaves];
    double frac[64];                       // 2^(43 + i / 64)
    uint64_t part[kWaves], parts[kWaves], ties[kWaves];
    uint32_t counts[kWaves];
    uint64_t above;
    int found[2];
    uint32_t digit;
    Cut cut;
};

// Sum over the workgroup, in every thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared& sh) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    in_front(sh.part, v);
    return v;
}

// The lowest digit that holds something and whose larger digits hold less than `limit`
// together with `above`; sh.digit, and sh.above what all larger ones hold.  Whole workgroup.
__device__ __forceinline__ void find_digit(uint64_t above, double limit, Shared& sh) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    // thread t: digits kDigits - 1 - 2 t and the one below, falling
    const int d0 = kDigits - 1 - 2 * t;
    const uint64_t a = sh.hist[d0], b = sh.hist[d0 - 1];
    const uint64_t s = wave_sums(a + b);
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
    float T, p, m, lmax_f, bin_top, bin_rate;
    double lmax, rate, u;
    uint64_t least;                        // the weight that min_p asks for
    int row, V, k, top_at;
    bool has_k, has_p, done;               // done: nothing to draw (nothing left, or the largest logit alone)

    __device__ __forceinline__ Row(const SampleArgs& a, int r, int dt) : row(r), V(a.n_vocab) {
        z = (const unsigned char*)a.logits + r * a.ld * (dt == LORA_F32 ? 4 : 2);
        // (without branches: the loads are on their way together; for an array that is not there u is read)
        const float uf = a.u[r];
        const float t = *((a.temperature ? a.temperature : a.u) + r), q = *((a.top_p ? a.top_p : a.u) + r),
                    n = *((a.min_p ? a.min_p : a.u) + r);
        const int i = *((a.top_k ? a.top_k : (const int32_t*)a.u) + r);
        T = !a.temperature ? 1.f : t > kMostT ? kMostT : t;
        p = a.top_p ? q : 1.f;
        m = a.min_p ? n : 0.f;
        k = a.top_k ? i : 0;
        u = uf >= 1.f ? 1.0 : uf > 0.f ? (double)uf : 0.0;
        has_k = k > 0 && k < V;
        has_p = p < 1.f;
        least = m > 0.f ? (uint64_t)ceil((double)(m < 1.f ? m : 1.f) * kOne) : 0;
    }
    __device__ __forceinline__ void set_top(uint64_t best) {
        lmax_f = logit_of((uint32_t)(best >> 32));
        top_at = index_of(best);
        done = (uint32_t)(best >> 32) <= kKeyNone || !(T >= kLeastT);
        lmax = lmax_f < INFINITY ? (double)lmax_f : 0x1p130;   // (infinity weighs 2^43, what is finite nothing)
        rate = 64 * 1.4426950408889634 / (double)T;
        bin_rate = (float)kBinsPerNat / T;
        bin_top = fminf(lmax_f, 3.402823466e38f);
    }
    // top_k is small: the histogram is of threads' largest logits, and K's weights are summed in the list
    __device__ __forceinline__ bool small_k() const { return has_k && k <= kSmallK; }
    __device__ __forceinline__ uint64_t weight_of(float l, const double* frac) const { return weight(l, lmax, rate, frac); }
    __device__ __forceinline__ uint64_t kept(uint64_t w) const { return w >= least ? w : 0; }
    // (each step is monotone; what is -infinity or weighs nothing is in the last bin)
    __device__ __forceinline__ int bin_of(float l) const {
        return (int)__builtin_amdgcn_fmed3f((bin_top - l) * bin_rate, 0.f, (float)(kBins - 1));
    }
    __device__ __forceinline__ void finish(const SampleArgs& a) const {
        const bool none = !(lmax_f > -INFINITY);
        a.tokens[row] = none ? -1 : top_at;
        if (a.probs) a.probs[row] = none ? 0.f : 1.f;
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

// f(logits, index of the first) for the logits of segment `seg`, by one wave, whose lanes hold kVec consecutive ones each,
// lane by lane and step by step in the order of the indices.  NaN is as -infinity, and so is what lies past the
// segment, and all that lanes have whose `want` is false.  (16 bytes a lane and load, at whatever alignment the row has; U
// loads on their way together.  A segment is a multiple of 256 logits and a step of a 16-bit row 512: where the multiple is odd the
// last half step is read logit by logit, and so is all of segments of 256, which rows of up to 4096 logits have, and
// few rows of up to 65536.)
template <int DT>
struct Vec {
    static constexpr int kVec = DT == LORA_F32 ? 4 : 8;
    u32x4 w;
    __device__ __forceinline__ void load(const Row& R, int i, bool want) {
        constexpr uint32_t kNone = DT == LORA_F32 ? 0xff800000u : DT == LORA_F16 ? 0xfc00fc00u : 0xff80ff80u;
        w = u32x4{kNone, kNone, kNone, kNone};
        if (want) __builtin_memcpy(&w, (const unsigned char*)R.z + (int64_t)i * (DT == LORA_F32 ? 4 : 2), 16);
    }
    __device__ __forceinline__ float get(int e) const {
        const uint32_t x = DT == LORA_F32 ? w[e & 3] : w[(e >> 1) & 3] >> (16 * (e & 1)) & 0xffffu;
        const float l = DT == LORA_F32 ? __uint_as_float(x) : DT == LORA_F16 ? FmtF16::to_f32(x) : FmtBF16::to_f32(x);
        return l == l ? l : -INFINITY;
    }
};
template <int DT, int U = 2, class F>
__device__ __forceinline__ void for_segment(const SampleArgs& a, const Row& R, int seg, const F& f, bool want = true) {
    constexpr int kVec = Vec<DT>::kVec, kStep = 64 * kVec;
    const int l = threadIdx.x & 63, end = min(R.V, (seg + 1) * a.seg);
    int c = seg * a.seg;
    float v[kVec];
    for (; c + U * kStep <= end; c += U * kStep) {
        Vec<DT> x[U];
#pragma unroll
        for (int q = 0; q < U; ++q) x[q].load(R, c + kStep * q + kVec * l, want);
#pragma unroll
        for (int q = 0; q < U; ++q) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] = x[q].get(e);
            f(v, c + kStep * q + kVec * l);
        }
    }
    for (; c < end; c += kStep) {
        if (c + kStep <= end) {
            Vec<DT> x;
            x.load(R, c + kVec * l, want);
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] = x.get(e);
            f(v, c + kVec * l);
            continue;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const int i = c + kVec * l + e;
            v[e] = want && i < end ? logit<DT>(R.z, i) : -INFINITY;
            v[e] = v[e] == v[e] ? v[e] : -INFINITY;
        }
        f(v, c + kVec * l);
    }
}

// f(logit) for wave w's sixteenth of the row, which lies behind those of the waves before it.
template <int DT, class F>
__device__ __forceinline__ void for_part(const SampleArgs& a, const Row& R, const F& f) {
    constexpr int kVec = Vec<DT>::kVec;
    const int w = threadIdx.x >> 6;
    for (int seg = w * a.slices; seg < (w + 1) * a.slices; ++seg)
        for_segment<DT>(a, R, seg, [&](const float (&v)[kVec], int) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) f(v[e]);
        });
}

// Running sum in front of x over the workgroup's threads; `all` gets the whole.
__device__ __forceinline__ uint64_t scan(Shared& sh, uint64_t x, uint64_t& all) {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint64_t s = wave_sums(x);
    __syncthreads();
    if (l == 63) sh.parts[w] = s;
    __syncthreads();
    return in_front(sh.parts, all) + s - x;
}

// A threshold over the row in memory, by the whole workgroup: the lowest key whose larger ones sum to less than `limit`,
// and in `above` what they sum to.  BY_WEIGHT: of weights, otherwise of ones.  With weights, keys below floor_key do not
// count and those of floor_key weigh floor_sum together.
template <int DT, bool BY_WEIGHT>
__device__ __forceinline__ uint32_t threshold(const SampleArgs& a, const Row& R, Shared& sh, double limit, uint32_t floor_key, uint64_t floor_sum,
                                              uint64_t& above) {
    uint32_t prefix = 0;
    above = 0;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
        __syncthreads();
        for (int i = threadIdx.x; i < kDigits; i += kSampleThreads) sh.hist[i] = 0;
        __syncthreads();
        for_part<DT>(a, R, [&](float l) __attribute__((always_inline)) {
            const uint32_t key = key_of(l);
            if (key <= kKeyNone || (level > 0 && (key >> (shift + bits)) != prefix)) return;
            uint64_t v = 1;
            if (BY_WEIGHT) v = key > floor_key ? R.weight_of(l, sh.frac) : 0;
            if (v) atomicAdd(&sh.hist[(key >> shift) & ((1u << bits) - 1)], (unsigned long long)v);
        });
        if (BY_WEIGHT && threadIdx.x == 0 && floor_sum && (level == 0 || (floor_key >> (shift + bits)) == prefix))
            atomicAdd(&sh.hist[(floor_key >> shift) & ((1u << bits) - 1)], (unsigned long long)floor_sum);
        __syncthreads();
        find_digit(above, limit, sh);
        prefix = prefix << bits | sh.digit;
        above = sh.above;
    }
    return prefix;
}

// The row from memory by one workgroup, however it is.
template <int DT>
__device__ __forceinline__ void slow_row(const SampleArgs& a, const Row& R, Shared& sh) {
    const int t = threadIdx.x, w = t >> 6, V = R.V;
    auto weight_at = [&](uint32_t key) { return R.weight_of(logit_of(key), sh.frac); };
    // kept are keys above tkey, and of those equal the first `share`
    uint32_t tkey = kKeyNone, share = 0;
    if (R.has_k) {
        uint64_t above;
        tkey = threshold<DT, false>(a, R, sh, (double)R.k, 0, 0, above);
        share = (uint32_t)(R.k - above);   // (at least 1; more than there are if few logits are left)
    }
    if (R.has_p && !(R.p > 0.f)) {
        tkey = key_of(R.lmax_f);
        share = 1;
    } else if (R.has_p) {
        uint64_t sum = 0, ties = 0;        // over K
        for_part<DT>(a, R, [&](float l) __attribute__((always_inline)) {
            const uint32_t key = key_of(l);
            if (key > kKeyNone && key > tkey) sum += weight_at(key);
            ties += key > kKeyNone && key == tkey;
        });
        sum = block_sum(sum, sh);
        ties = block_sum(ties, sh);
        const uint64_t floor_sum = tkey > kKeyNone ? min((uint64_t)share, ties) * weight_at(tkey) : 0;
        const double limit = (double)R.p * (double)(sum + floor_sum);
        uint64_t above;
        const uint32_t key = threshold<DT, true>(a, R, sh, limit, tkey, floor_sum, above);
        const uint64_t each = weight_at(key);
        // the first `few` of the equal ones begin below the limit
        uint32_t few = 1, most = key == tkey ? share : (uint32_t)V;
        while (few < most) {
            const uint32_t mid = few + (most - few + 1) / 2;
            if ((double)(above + (mid - 1) * each) < limit) few = mid;
            else most = mid - 1;
        }
        tkey = key;
        share = few;
    }
    const uint64_t tie_weight = tkey > kKeyNone ? R.kept(weight_at(tkey)) : 0;
    // weights and ties of each wave's part of the row
    uint64_t sum = 0, ties = 0;
    for_part<DT>(a, R, [&](float l) __attribute__((always_inline)) {
        const uint32_t key = key_of(l);
        if (key > kKeyNone && key > tkey) sum += R.kept(weight_at(key));
        ties += key > kKeyNone && key == tkey;
    });
    sum = wave_sum(sum);
    ties = wave_sum(ties);
    __syncthreads();
    if ((t & 63) == 0) {
        sh.part[w] = sum;
        sh.ties[w] = ties;
    }
    __syncthreads();
    auto part_of = [&](int i, uint64_t seen) { return sh.part[i] + min(share > seen ? share - seen : 0, sh.ties[i]) * tie_weight; };
    uint64_t total = 0, seen = 0;
    for (int i = 0; i < kWaves; ++i) {
        total += part_of(i, seen);
        seen += sh.ties[i];
    }
    const uint64_t target = R.target(total);
    // the part in which the target lies, and in it the logit, by all
    uint64_t at = 0;
    int p = 0;
    seen = 0;
    for (; p < kWaves - 1 && target >= at + part_of(p, seen); ++p) {
        at += part_of(p, seen);
        seen += sh.ties[p];
    }
    const int first = p * a.slices * a.seg, end = min(V, first + a.slices * a.seg);
    for (int i = first; i < end && at <= target; i += kSampleThreads) {
        const uint32_t key = i + t < end ? key_of(logit<DT>(R.z, i + t)) : 0;
        const bool tie = key == tkey && key > kKeyNone;
        uint64_t here, all;
        const uint64_t rank = seen + scan(sh, tie ? 1 : 0, here);
        const uint64_t own = key > kKeyNone && key > tkey ? R.kept(weight_at(key)) : tie && rank < share ? tie_weight : 0;
        const uint64_t before = at + scan(sh, own, all);
        if (own && before <= target && target < before + own) R.choose(a, i + t, own, total);
        at += all;
        seen += here;
    }
}

// ranked() of a slice's largest logit, in every thread of the workgroup; `most`: this thread's largest.
template <int DT>
__device__ __forceinline__ uint64_t best_of(const SampleArgs& a, const Row& R, Shared& sh, int slice, float& most) {
    float top = -INFINITY;
    int at = 0;
    constexpr int kVec = Vec<DT>::kVec;
    for_segment<DT>(a, R, slice * kWaves + (threadIdx.x >> 6), [&](const float (&v)[kVec], int i) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            at = v[e] > top ? i + e : at;
            top = fmaxf(top, v[e]);
        }
    });
    most = top;
    uint64_t b = wave_max(ranked(top, at));
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = b;
    __syncthreads();
    return wave_max(sh.part[threadIdx.x & (kWaves - 1)]);
}

__device__ __forceinline__ void clear_bins(Shared& sh) {
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) {
        sh.count[i] = 0;
        sh.mass[i] = 0;
    }
    __syncthreads();
}

// A slice's histogram into sh.count and sh.mass, or that of the threads' largest.
template <int DT>
__device__ __forceinline__ void fill_bins(const SampleArgs& a, const Row& R, Shared& sh, int slice, float most) {
    clear_bins(sh);
    if (R.small_k()) {
        const int b = R.bin_of(most);
        if (b < kBins - 1) atomicAdd(&sh.count[b], 1u);
    } else {
        constexpr int kVec = Vec<DT>::kVec;
        for_segment<DT>(a, R, slice * kWaves + (threadIdx.x >> 6), [&](const float (&v)[kVec], int) __attribute__((always_inline)) {
            uint64_t w[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) w[e] = R.weight_of(v[e], sh.frac);
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const int b = R.bin_of(v[e]);
                if (b < kBins - 1) {
                    atomicAdd(&sh.count[b], 1u);
                    atomicAdd(&sh.mass[b], (unsigned long long)w[e]);
                }
            }
        });
    }
    __syncthreads();
}

// The histogram in sh.count and sh.mass into its running sums, a bin a thread: up to and with the thread's bin, and
// in front of it.  Whole workgroup.
struct BinSums {
    uint32_t c, c0;
    uint64_t m, m0;
    __device__ __forceinline__ BinSums(Shared& sh) {
        const int t = threadIdx.x, w = t >> 6;
        c0 = sh.count[t];
        m0 = sh.mass[t];
        c = wave_sums(c0);
        m = wave_sums(m0);
        if ((t & 63) == 63) {
            sh.counts[w] = c;
            sh.parts[w] = m;
        }
        if (t < 2) sh.found[t] = kBins - 1;
        __syncthreads();
        uint32_t n;
        uint64_t all;
        c += in_front(sh.counts, n);
        m += in_front(sh.parts, all);
        sh.count[t] = c;
        sh.mass[t] = m;
        c0 = c - c0;
        m0 = m - m0;
        __syncthreads();
    }
    // the first bin at which `ok` of the running sums holds (it holds from there on, and not of 0 and 0), or the last
    // bin; `i` is 0 or 1, once each
    template <class Ok>
    __device__ __forceinline__ int first(Shared& sh, int i, const Ok& ok) const {
        if (ok(c, m) && !ok(c0, m0)) sh.found[i] = threadIdx.x;
        __syncthreads();
        return sh.found[i];
    }
};
static_assert(kBins == kSampleThreads, "a bin a thread");
template <class T>
__device__ __forceinline__ T up_to(const T* sums, int b) { return b < 0 ? 0 : sums[b]; }

// Step 2's decision from the row's histogram in sh.count and sh.mass, into sh.cut.
__device__ __forceinline__ void decide(const Row& R, Shared& sh) {
    const BinSums S(sh);
    const uint64_t all = sh.mass[kBins - 1];
    // the bin of the top_k-th logit, and the weights up to it, which K's are not above
    const bool small = R.small_k();
    const int kb = R.has_k ? S.first(sh, 0, [&](uint32_t c, uint64_t) { return c >= (uint32_t)R.k; }) : kBins - 1;
    const bool k_cuts = R.has_k && (small || kb < kBins - 1);
    // the last bin that begins below top_p's limit (or, with K's sum smaller, later than that)
    int pb = kBins - 2;
    const bool by_p = R.has_p && R.p > 0.f && !small;
    if (R.has_p && !(R.p > 0.f)) pb = 0;
    if (by_p) {
        const double limit = (double)R.p * (double)sh.mass[kb];
        pb = min(pb, S.first(sh, 1, [&](uint32_t, uint64_t m) { return (double)m >= limit; }));
    }
    // the last bin with a logit that min_p keeps, with some to spare for the roundings (weights of a few units
    // are rounded by up to ln 2)
    int m1 = kBins - 2;
    if (R.least > 0) {
        const float f = (float)kBinsPerNat * -logf((float)((double)R.least / kOne));
        const int spare = R.least < 256 ? kBinsPerNat * 3 / 4 : 2;
        if (f < (float)(kBins - 2)) m1 = min((int)f + spare, kBins - 2);
    }
    // (top_p needs the sum over K: all of it is in the list, if the bins do not have the row's)
    const bool whole_k = R.has_p && R.p > 0.f && k_cuts;
    const int hi = whole_k ? min(kb, kBins - 2) : min(min(min(kb, pb), m1), kBins - 2);
    int lo = 0, slow = 0;
    const uint32_t upto = sh.count[hi];
    if (!small && upto > (uint32_t)kFits) {            // more than a list: top_p's last bin, if it is among them
        lo = R.has_p && pb <= hi ? pb : hi + 1;
        slow = lo == 0 || k_cuts || (lo <= hi && upto - up_to(sh.count, lo - 1) > (uint32_t)kFits);
    }
    if (threadIdx.x == 0) {
        sh.cut.all = k_cuts ? 0 : all;
        sh.cut.below = up_to(sh.mass, lo - 1);
        sh.cut.lo = lo;
        sh.cut.hi = hi;
        sh.cut.k_cuts = k_cuts;
        sh.cut.slow = slow;
    }
    __syncthreads();
}

// Step 3 for segment `seg`, by one wave: its logits of the cut's bins into `list` of kWaveList, in the order of their
// indices, and, where lo is not 0, the sum of weights below it into `sum`.  Their number, which may be more than the room.
// `most`: the thread's largest of the segment, where top_k is small; a thread without a listed one reads nothing.
// ANY: into a list of kList that all waves share, in any order, sh.digit (0 before) counting.
template <int DT, bool ANY>
__device__ __forceinline__ uint32_t collect(const SampleArgs& a, const Row& R, Shared& sh, int seg, float most, uint64_t* list, uint64_t& sum) {
    const int lo = sh.cut.lo, hi = sh.cut.hi;
    constexpr int kVec = Vec<DT>::kVec;
    uint32_t n = 0;
    // a lane's logits of one step that are in, bit by bit; lanes in order
    auto add = [&](uint32_t in, const float (&v)[kVec], int i) __attribute__((always_inline)) {
        if (!__any(in)) return;
        const uint32_t own = __popc(in), sums = wave_sums(own);
        if (ANY) n = (uint32_t)__builtin_amdgcn_readlane((int)((threadIdx.x & 63) == 63 ? atomicAdd(&sh.digit, sums) : 0u), 63);
        uint32_t at = n + sums - own;
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (in >> e & 1) {
                if (at < (uint32_t)(ANY ? kList : kWaveList)) list[at] = ranked(v[e], i + e);
                ++at;
            }
        n += at_lane(sums, 63);
    };
    sum = 0;
    if (lo == 0) {
        for_segment<DT, 4>(a, R, seg, [&](const float (&v)[kVec], int i) __attribute__((always_inline)) {
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) in |= (uint32_t)(R.bin_of(v[e]) <= hi) << e;
            add(in, v, i);
        }, !R.small_k() || R.bin_of(most) <= hi);
    } else {
        for_segment<DT>(a, R, seg, [&](const float (&v)[kVec], int i) __attribute__((always_inline)) {
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const int b = R.bin_of(v[e]);
                in |= (uint32_t)(b >= lo && b <= hi) << e;
                if (b < lo) sum += R.kept(R.weight_of(v[e], sh.frac));
            }
            add(in, v, i);
        });
        sum = wave_sum(sum);
    }
    return n;
}

// How many of list[0 .. n) are larger than `mine`, and their weights' sum, by the quad that holds `mine` (0 for none).
__device__ __forceinline__ void rank_among(const uint64_t* list, const uint64_t* weights, int n, uint64_t mine, int& rank,
                                           uint64_t& before) {
    uint32_t r = 0;
    before = 0;
    if (mine) {
#pragma unroll 4
        for (int i = threadIdx.x & 3; i < n; i += 4) {
            const bool larger = list[i] > mine;
            const uint64_t w = weights[i];
            r += larger;
            before += larger ? w : 0;
        }
    }
    rank = (int)quad_sum(r);
    before = quad_sum(before);
}

// What top_k and top_p keep of a list (n logits, 4 entries a thread in `mine`): ranked() of the last.  A finer histogram
// of the list's bins leads to the one bin in which each of the two ends, whose few logits are compared with one another.
// False if they are not few.
__device__ __forceinline__ bool select(const Row& R, Shared& sh, const Cut& cut, const uint64_t (&mine)[kList / kSampleThreads], int n,
                                       uint64_t& last) {
    constexpr int kEach = kList / kSampleThreads;
    const int t = threadIdx.x;
    const float scale = (float)kBins / (float)(cut.hi + 1 - cut.lo);
    int fine[kEach];
    clear_bins(sh);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const float l = logit_of((uint32_t)(mine[j] >> 32));
        const float f = __builtin_amdgcn_fmed3f((R.bin_top - l) * R.bin_rate, 0.f, (float)(kBins - 1));
        fine[j] = mine[j] ? (int)__builtin_amdgcn_fmed3f((f - (float)cut.lo) * scale, 0.f, (float)(kBins - 1)) : kBins;
        if (fine[j] < kBins) {
            atomicAdd(&sh.count[fine[j]], 1u);
            if (R.has_p) atomicAdd(&sh.mass[fine[j]], (unsigned long long)R.weight_of(l, sh.frac));
        }
    }
    __syncthreads();
    // a bin's logits, one a quad (and in its first lane), with their rank in it and the weights in front of them in it;
    // false if too many
    uint64_t own = 0, weight = 0, before = 0;
    int rank = 0;
    const BinSums S(sh);                   // (and the running sums in sh)
    auto compare = [&](int bin) __attribute__((always_inline)) {
        const int m = (int)(sh.count[bin] - up_to(sh.count, bin - 1));
        if (m > kRanked) return false;
        if (t == 0) sh.digit = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (fine[j] == bin) sh.hist[atomicAdd(&sh.digit, 1u)] = mine[j];
        __syncthreads();
        own = t >> 2 < m ? sh.hist[t >> 2] : 0;
        weight = own ? R.weight_of(logit_of((uint32_t)(own >> 32)), sh.frac) : 0;
        if (own) sh.weights[t >> 2] = weight;
        __syncthreads();
        rank_among((const uint64_t*)sh.hist, sh.weights, m, own, rank, before);
        if (t & 3) own = 0;
        return true;
    };
    last = 0;
    uint64_t sum = cut.all;
    if (cut.k_cuts) {
        sum = sh.mass[kBins - 1];
        if (n > R.k) {
            const int b = S.first(sh, 0, [&](uint32_t c, uint64_t) { return c >= (uint32_t)R.k; });
            const int c0 = (int)up_to(sh.count, b - 1);
            const uint64_t m0 = up_to((const uint64_t*)sh.mass, b - 1);
            if (!compare(b)) return false;
            if (own && c0 + rank == R.k - 1) {
                sh.part[4] = own;
                sh.part[5] = m0 + before + weight;
            }
            __syncthreads();
            last = sh.part[4];
            sum = sh.part[5];
        }
    }
    if (R.has_p) {
        const double limit = (double)R.p * (double)sum;
        const int b = S.first(sh, 1, [&](uint32_t c, uint64_t m) { return R.p > 0.f ? (double)(cut.below + m) >= limit : c > 0; });
        const uint64_t m0 = cut.below + up_to((const uint64_t*)sh.mass, b - 1);
        if (!compare(b)) return false;
        // the last of the bin that begins below the limit (none: what lies in front of the bin is all)
        const bool in = own && ((double)(m0 + before) < limit || (!(R.p > 0.f) && rank == 0));
        if (t == 0) sh.digit = 0, sh.part[2] = 0;
        __syncthreads();
        if (in) atomicMax(&sh.digit, (uint32_t)rank + 1);
        __syncthreads();
        if (in && (uint32_t)rank + 1 == sh.digit) sh.part[2] = own;
        __syncthreads();
        // (the weights of all bins may stay below the limit: then nothing is cut here)
        if (sh.digit > 0) last = max(last, sh.part[2]);
        __syncthreads();
    }
    return true;
}

// sh.list[0 .. n) falling, by compare and exchange in the order of a bitonic sort; from n on zeros.  Exchanges over
// less than 128 stay inside a wave's 128 entries, whose reads and writes are in order.
__device__ __forceinline__ void sort_list(Shared& sh, int n) {
    int size = 256;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kSampleThreads) sh.list[i] = 0;
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            if (j >= 128 || k == 2) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (int t = threadIdx.x; t < size / 2; t += kSampleThreads) {
                const int i = 2 * t - (t & (j - 1)), o = i + j;
                const uint64_t x = sh.list[i], y = sh.list[o];
                if ((x < y) == ((i & k) == 0)) {
                    sh.list[i] = y;
                    sh.list[o] = x;
                }
            }
            if (j == 128) __syncthreads();
        }
    __syncthreads();
}

// Step 4, from the list (n logits, `ordered` by their indices or not) and the segments' sums in sh.
template <int DT>
__device__ __forceinline__ void pick(const SampleArgs& a, const Row& R, Shared& sh, int n, bool ordered) {
    const int t = threadIdx.x;
    constexpr int kEach = kList / kSampleThreads;
    const Cut cut = sh.cut;
    const bool direct = cut.lo == 0 && ordered;    // the token is found in the list itself
    auto weight_at = [&](uint64_t r) __attribute__((always_inline)) { return R.weight_of(logit_of((uint32_t)(r >> 32)), sh.frac); };
    const bool cuts = n > 0 && (cut.k_cuts || R.has_p);
    const int most = cut.k_cuts ? min(R.k, n) : n;
    uint64_t all, last = 0;                // last: the last that top_k and top_p keep
    if (n <= kRanked) {
        // one entry a quad: its rank and the weights in front of it, from a comparison with every other, which the four
        // lanes share; from then on it is the first lane's
        const uint64_t mine = t >> 2 < n ? sh.list[t >> 2] : 0;
        uint64_t w = mine ? weight_at(mine) : 0;
        if (cuts) {
            if (mine) sh.weights[t >> 2] = w;
            __syncthreads();
            uint64_t before;
            int rank;
            rank_among(sh.list, sh.weights, n, mine, rank, before);
            bool in = mine && (t & 3) == 0 && rank < most;
            if (R.has_p) {
                all = cut.all;
                if (cut.k_cuts) scan(sh, in ? w : 0, all);
                in &= rank == 0 || (double)(cut.below + before) < (double)R.p * (double)all;
            }
            if (!in) w = 0;
            if (!direct) {                 // (the segment's search asks for the last)
                if (t == 0) sh.digit = 0;
                __syncthreads();
                if (in) atomicMax(&sh.digit, (uint32_t)rank);
                __syncthreads();
                if (in && (uint32_t)rank == sh.digit) sh.part[1] = mine;
                __syncthreads();
                last = sh.part[1];
            }
        }
        w = (t & 3) == 0 ? R.kept(w) : 0;
        if (direct) {
            const uint64_t run = scan(sh, w, all), target = R.target(all);
            if (w && run <= target && target < run + w) R.choose(a, index_of(mine), w, all);
            return;
        }
        if (w) atomicAdd((unsigned long long*)&sh.segs[index_of(mine) / a.seg], (unsigned long long)w);
    } else {
        // thread t: entries kEach t ..
        uint64_t mine[kEach], v[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) mine[j] = kEach * t + j < n ? sh.list[kEach * t + j] : 0;
        if (cuts && !select(R, sh, cut, mine, n, last)) {
            __syncthreads();
            sort_list(sh, n);
            int kept = most;
            if (R.has_p) {
                uint64_t sum = 0;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    v[j] = kEach * t + j < kept ? weight_at(sh.list[kEach * t + j]) : 0;
                    sum += v[j];
                }
                uint64_t before = cut.below + scan(sh, sum, all);
                const double limit = (double)R.p * (double)(cut.k_cuts ? all : cut.all);
                int end = 1;               // (running sums: the kept ones are the first)
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    if (kEach * t + j < kept && (double)before < limit) end = kEach * t + j + 1;
                    before += v[j];
                }
                if (t == 0) sh.digit = 1;
                __syncthreads();
                if (end > 1) atomicMax(&sh.digit, (uint32_t)end);
                __syncthreads();
                kept = (int)sh.digit;
            }
            last = sh.list[kept - 1];
        }
        uint64_t sum = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            v[j] = mine[j] && mine[j] >= last ? R.kept(weight_at(mine[j])) : 0;
            sum += v[j];
        }
        if (direct) {
            uint64_t run = scan(sh, sum, all);
            const uint64_t target = R.target(all);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (v[j] && run <= target && target < run + v[j]) R.choose(a, index_of(mine[j]), v[j], all);
                run += v[j];
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (v[j]) atomicAdd((unsigned long long*)&sh.segs[index_of(mine[j]) / a.seg], (unsigned long long)v[j]);
    }
    // the segment in which the target lies, and the segment again
    __syncthreads();
    const uint64_t s = t < a.slices * kWaves ? sh.segs[t] : 0;
    const uint64_t at = scan(sh, s, all);
    const uint64_t total = all, target = R.target(total);
    if (s && at <= target && target < at + s) {
        sh.digit = t;
        sh.part[0] = at;
    }
    __syncthreads();
    const int first = (int)sh.digit * a.seg, end = min(R.V, first + a.seg);
    uint64_t run = sh.part[0];
    for (int i = first + t; i - t < end && run <= target; i += kSampleThreads) {
        float l = i < end ? logit<DT>(R.z, i) : -INFINITY;
        l = l == l ? l : -INFINITY;
        const int b = R.bin_of(l);
        uint64_t x = 0;
        if (b < cut.lo || (b <= cut.hi && ranked(l, i) >= last)) x = R.kept(R.weight_of(l, sh.frac));
        const uint64_t mine = run + scan(sh, x, all);
        if (x && mine <= target && target < mine + x) R.choose(a, i, x, total);
        run += all;
    }
}

// The waves' lists, from[kWaveList g ..] for wave g, one behind the other in sh.list (which `from` may be itself, of one
// slice); numbers in sh.seg_n[0 .. segs).  kFull if all do not fit; kCrowded if one is longer than a wave's part: of one
// slice it is not whole then and nothing is moved, of several the list is whole, but in any order.
enum Gathered { kOrdered, kCrowded, kFull };
__device__ __forceinline__ Gathered gather(Shared& sh, const uint64_t* from, int segs, int& n) {
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    const uint64_t mine = t < segs ? sh.seg_n[t] : 0;
    uint64_t all;                          // (in the upper half how many are longer)
    const uint64_t first = scan(sh, mine > (uint64_t)kWaveList ? mine + (1ull << 32) : mine, all) & 0xffffffffu;
    n = (int)(uint32_t)all;
    const Gathered how = (uint32_t)all > (uint32_t)kList ? kFull : all >> 32 ? kCrowded : kOrdered;
    if (how == kFull || (how == kCrowded && segs == kWaves)) return how;
    if (t < segs) sh.segs[t] = first;      // (for a moment)
    __syncthreads();
    if (segs == kWaves) {
        constexpr int kPer = kWaveList / 64;
        uint64_t r[kPer];
        const int of = (int)sh.seg_n[w], to = (int)sh.segs[w];
#pragma unroll
        for (int q = 0; q < kPer; ++q) r[q] = l + 64 * q < of ? from[w * kWaveList + l + 64 * q] : 0;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kPer; ++q)
            if (l + 64 * q < of) sh.list[to + l + 64 * q] = r[q];
    } else {
        // the first 64 of eight of the wave's parts at once, more where there are
        constexpr int kPer = 8;
        for (int j0 = 0; j0 * kWaves < segs; j0 += kPer) {
            uint64_t r[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int g = w + kWaves * (j0 + j);
                r[j] = g < segs && l < (int)sh.seg_n[g] ? from[(int64_t)g * kWaveList + l] : 0;
            }
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int g = w + kWaves * (j0 + j);
                if (g >= segs) break;
                const int of = (int)sh.seg_n[g], to = (int)sh.segs[g];
                if (l < of) sh.list[to + l] = r[j];
#pragma unroll 4
                for (int i = l + 64; i < of; i += 64) sh.list[to + i] = from[(int64_t)g * kWaveList + i];
            }
        }
    }
    __syncthreads();
    return how;
}

// 2^(43 + i / 64), by the series of e^x: past x^20 nothing is left of it.
struct Fractions {
    double f[64];
    constexpr Fractions() : f() {
        for (int i = 0; i < 64; ++i) {
            const long double x = 0.693147180559945309417232121458176568L * i / 64;
            long double p = 1;
            for (int n = 24; n > 0; --n) p = 1 + p * x / n;
            f[i] = (double)p * kOne;
        }
    }
};
__constant__ const Fractions kFractions;
// (loaded early, needed late)
__device__ __forceinline__ double fraction() { return kFractions.f[threadIdx.x & 63]; }
__device__ __forceinline__ void put_fraction(Shared& sh, double f) {
    if (threadIdx.x < 64) sh.frac[threadIdx.x] = f;
}

// A row's workspace: the cut; every slice's best; of every wave the number of listed logits, its sum and its list; of
// every slice counts and weights per bin, or its threads' largest logits.
struct RowSpace {
    Cut* cut;
    uint64_t *best, *mass, *segs, *list;
    uint32_t *count, *n;
    float* most;
    static constexpr int64_t kHead = 64 + 8 * kMaxSlices;
    static constexpr int64_t kSlice = kWaves * (8 + 4 + 8 * kWaveList) + 12 * kBins + 4 * kSampleThreads;
    __device__ RowSpace(unsigned char* p, int slices) {
        cut = (Cut*)p;
        best = (uint64_t*)(p + 64);
        mass = best + kMaxSlices;
        segs = mass + (int64_t)slices * kBins;
        list = segs + (int64_t)slices * kWaves;
        n = (uint32_t*)(list + (int64_t)slices * kWaves * kWaveList);
        count = n + (int64_t)slices * kWaves;
        most = (float*)(count + (int64_t)slices * kBins);
    }
    static int64_t bytes(int slices) { return kHead + slices * kSlice; }
};
static_assert(4 * kRanked == kSampleThreads, "a quad for each of a ranked list");
static_assert((sizeof(Cut) & (sizeof(Cut) - 1)) == 0 && sizeof(Cut) <= 64 && RowSpace::kHead % 16 == 0 && RowSpace::kSlice % 16 == 0, "rows' workspaces");

template <int DT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_row_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, w = t >> 6;
    Row R(a, blockIdx.x, DT);
    const double f = fraction();
    float most;
    R.set_top(best_of<DT>(a, R, sh, 0, most));
    if (R.done) {
        if (t == 0) R.finish(a);
        return;
    }
    put_fraction(sh, f);
    fill_bins<DT>(a, R, sh, 0, most);
    decide(R, sh);
    int n = 0;
    Gathered how = sh.cut.slow ? kFull : kOrdered;
    if (how != kFull) {
        uint64_t sum;
        const uint32_t of = collect<DT, false>(a, R, sh, w, most, sh.list + w * kWaveList, sum);
        if ((t & 63) == 0) sh.seg_n[w] = of;
        __syncthreads();
        how = gather(sh, sh.list, kWaves, n);
        __syncthreads();
        if ((t & 63) == 0) sh.segs[w] = sum;
        if (t == 0) sh.digit = 0;
        __syncthreads();
        if (how == kCrowded) {
            collect<DT, true>(a, R, sh, w, most, sh.list, sum);
            __syncthreads();
        }
    }
    if (how == kFull) {
        slow_row<DT>(a, R, sh);
        return;
    }
    pick<DT>(a, R, sh, n, how == kOrdered);
}

// The row's best of its slices', which lanes hold.
__device__ __forceinline__ uint64_t largest(uint64_t b, int slices) {
    return wave_max((threadIdx.x & (kMaxSlices - 1)) < (unsigned)slices ? b : 0);
}

template <int DT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_best_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const RowSpace ws(a.ws + blockIdx.y * a.ws_row, a.slices);
    const Row R(a, blockIdx.y, DT);
    float most;
    const uint64_t b = best_of<DT>(a, R, sh, blockIdx.x, most);
    if (threadIdx.x == 0) ws.best[blockIdx.x] = b;
    if (R.small_k()) ws.most[blockIdx.x * kSampleThreads + threadIdx.x] = most;
}

template <int DT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_bins_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const RowSpace ws(a.ws + blockIdx.y * a.ws_row, a.slices);
    const uint64_t bests = ws.best[threadIdx.x & (kMaxSlices - 1)];
    Row R(a, blockIdx.y, DT);
    if (R.small_k()) return;
    put_fraction(sh, fraction());
    R.set_top(largest(bests, a.slices));
    if (R.done) return;
    fill_bins<DT>(a, R, sh, blockIdx.x, 0.f);
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) {
        ws.count[blockIdx.x * kBins + i] = sh.count[i];
        ws.mass[blockIdx.x * kBins + i] = sh.mass[i];
    }
}

template <int DT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_list_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, seg = blockIdx.x * kWaves + (t >> 6);
    const RowSpace ws(a.ws + blockIdx.y * a.ws_row, a.slices);
    const uint64_t bests = ws.best[t & (kMaxSlices - 1)];
    Row R(a, blockIdx.y, DT);
    const double f = fraction();
    // (of four slices at once, those past the last read as the last again and not counted)
    float own = 0.f;
    if (R.small_k()) {
        own = ws.most[blockIdx.x * kSampleThreads + t];
        float most[kMaxSlices] = {};
#pragma unroll
        for (int j = 0; j < kMaxSlices; ++j)
            if ((j & ~3) < a.slices) most[j] = ws.most[min(j, a.slices - 1) * kSampleThreads + t];
        R.set_top(largest(bests, a.slices));
        if (R.done) return;
        clear_bins(sh);
#pragma unroll
        for (int j = 0; j < kMaxSlices; ++j) {
            const int b = R.bin_of(most[j]);
            if (j < a.slices && b < kBins - 1) atomicAdd(&sh.count[b], 1u);
        }
    } else {
        uint32_t c[kMaxSlices];
        uint64_t m[kMaxSlices];
#pragma unroll
        for (int j = 0; j < kMaxSlices; ++j) {
            c[j] = 0, m[j] = 0;
            if ((j & ~3) < a.slices) {
                c[j] = ws.count[min(j, a.slices - 1) * kBins + t];
                m[j] = ws.mass[min(j, a.slices - 1) * kBins + t];
            }
        }
        R.set_top(largest(bests, a.slices));
        if (R.done) return;
#pragma unroll
        for (int j = 1; j < kMaxSlices; ++j) {
            c[0] += j < a.slices ? c[j] : 0;
            m[0] += j < a.slices ? m[j] : 0;
        }
        sh.count[t] = c[0];
        sh.mass[t] = m[0];
    }
    put_fraction(sh, f);
    __syncthreads();
    decide(R, sh);
    if (blockIdx.x == 0 && t == 0) *ws.cut = sh.cut;
    if (sh.cut.slow) return;
    uint64_t sum;
    uint32_t n = collect<DT, false>(a, R, sh, seg, own, ws.list + (int64_t)seg * kWaveList, sum);
    if (t == 0) sh.digit = 0;
    if (__syncthreads_or(n > (uint32_t)kWaveList)) {   // the slice's waves share their parts, and the first has all
        collect<DT, true>(a, R, sh, seg, own, ws.list + (int64_t)blockIdx.x * kList, sum);
        __syncthreads();
        n = t < 64 ? sh.digit : 0;
    }
    if ((t & 63) == 0) {
        ws.n[seg] = n;
        ws.segs[seg] = sum;
    }
}

template <int DT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_pick_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, segs = a.slices * kWaves;
    const RowSpace ws(a.ws + blockIdx.x * a.ws_row, a.slices);
    // (all that is read from the workspace, at once)
    constexpr int kCutWords = sizeof(Cut) / 8;
    const uint64_t cut = ((const uint64_t*)ws.cut)[t & (kCutWords - 1)];
    const uint32_t listed = ws.n[min(t, segs - 1)];
    const uint64_t sum = ws.segs[min(t, segs - 1)];
    const uint64_t bests = ws.best[t & (kMaxSlices - 1)];
    Row R(a, blockIdx.x, DT);
    put_fraction(sh, fraction());
    if (t < kCutWords) ((uint64_t*)&sh.cut)[t] = cut;
    if (t < segs) sh.seg_n[t] = listed;
    const uint64_t best = largest(bests, a.slices);
    R.set_top(best);
    if (R.done) {
        if (t == 0) R.finish(a);
        return;
    }
    __syncthreads();
    int n = 0;
    Gathered how = sh.cut.slow ? kFull : kOrdered;
    if (how != kFull) {
        how = gather(sh, ws.list, segs, n);
        __syncthreads();
        if (t < segs) sh.segs[t] = sum;
        __syncthreads();
    }
    if (how == kFull) {
        slow_row<DT>(a, R, sh);
        return;
    }
    pick<DT>(a, R, sh, n, how == kOrdered);
}

struct SamplePlan {
    int slices, seg;
};

// One launch and a workgroup a row from 129 rows on, or where a row is short; slices of 4096 logits at least, as many as
// give every compute unit a workgroup, otherwise.  What a row costs depends on its parameters, which are on the device: with a
// small top_k one workgroup is faster further up than with top_p alone.  Measured (us), one launch against 2, 4 and 8 slices:
// 256 rows of 50257 with top_k 50 21 against 33, 39, 49, with top_p alone 57 against 68, 80, 92; of 128000 in bfloat16, one launch
// against 2, 3 and 4 slices, all kinds, top_p 0.95 and top_k 50: 86 rows 100 against 70, 64, 56, 103 against 73, 82, 80 and 27 against 27, 37, 33;
// 129 rows 103 against 74, 75, 70, 107 against 106, 109, 96 and 28 against 40, 39, 42; 200 rows 104 against 87, 106, 91, 107 against 123,
// 146, 127 and 29 against 42, 54, 53; 300 rows 140 against 125, 131, 120, 200 against 181, 197, 176 and 53 against 62, 73, 70; 128 rows of 50257 18 against
// 23, 26 and 55 against 50, 52, of 32000 14 against 21, 23 and 36 against 35, 42; 60 rows of 24000 12 against 19, 19 and 29
// against 35, 29, of 50257 17 against 21, 20 and 54 against 49, 36; 64 rows of 128000, all kinds, 103 against 70, 49, 50; 16 rows
// of 32000 without filters 28 against 26, 22, 22; one row of 20000 with top_p 22 against 25, 23, 22, of 32000 28 against 27, 23, 22.
SamplePlan plan_sample(int n_rows, int n_vocab) {
    const bool one = n_vocab <= 24576 || (n_rows > 64 && n_vocab <= 49152);
    int64_t slices = one ? 1 : std::min<int64_t>({kMaxSlices, (n_vocab + 4095) / 4096, 256 / std::max(1, n_rows)});
    slices = std::max<int64_t>(1, slices);
    SamplePlan p;
    p.seg = (int)((n_vocab + slices * kWaves * 256 - 1) / (slices * kWaves * 256)) * 256;
    p.slices = (n_vocab + p.seg * kWaves - 1) / (p.seg * kWaves);
    return p;
}

template <int DT>
void launch_sample(const SampleArgs& a, int n_rows, hipStream_t st) {
    const dim3 block(kSampleThreads);
    if (a.slices == 1) {
        hipLaunchKernelGGL(lora_sample_row_kernel<DT>, dim3(n_rows), block, 0, st, a);
        return;
    }
    const dim3 grid(a.slices, n_rows);
    hipLaunchKernelGGL(lora_sample_best_kernel<DT>, grid, block, 0, st, a);
    hipLaunchKernelGGL(lora_sample_bins_kernel<DT>, grid, block, 0, st, a);
    hipLaunchKernelGGL(lora_sample_list_kernel<DT>, grid, block, 0, st, a);
    hipLaunchKernelGGL(lora_sample_pick_kernel<DT>, dim3(n_rows), block, 0, st, a);
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
    a.ld = ld;
    a.n_vocab = n_vocab;
    a.ws = (unsigned char*)ws;
    const SamplePlan p = plan_sample(n_rows, n_vocab);
    a.slices = p.slices;
    a.seg = p.seg;
    a.ws_row = RowSpace::bytes(p.slices);
    for (int r = 0, n; r < n_rows; r += n) {
        n = std::min(n_rows - r, kLaunchRows);
        a.logits = (const unsigned char*)logits + r * ld * e;
        a.temperature = params->temperature ? params->temperature + r : nullptr;
        a.top_k = params->top_k ? params->top_k + r : nullptr;
        a.top_p = params->top_p ? params->top_p + r : nullptr;
        a.min_p = params->min_p ? params->min_p + r : nullptr;
        a.u = u + r;
        a.tokens = tokens + r;
        a.probs = probs ? probs + r : nullptr;
        if (dtype == LORA_F16) launch_sample<LORA_F16>(a, n, st);
        else if (dtype == LORA_BF16) launch_sample<LORA_BF16>(a, n, st);
        else launch_sample<LORA_F32>(a, n, st);
        if (int rc = check_launch("lora_sample")) return rc;
    }
    return LORA_OK;
}

}  // extern "C"
