// gfx950 kernel of the next token of every row (include/lora_sample.h).
//
// One workgroup per row.  A logit's order is that of a 32-bit key; both thresholds, the
// top_k-th largest logit and the last one of the top_p start, are found digit by digit of the
// key from sums per digit (of ones or of weights), from the largest down.  What equal logits
// share of a threshold goes to the lowest indices.  Sums are whole numbers, so that neither the
// order of the atomic additions nor the division of the row changes a bit.
#include <cmath>

#include <algorithm>

#include "lora_device.h"
#include "lora_mx_internal.h"
#include "lora_sample.h"

namespace lora {
namespace {

constexpr int kSampleThreads = 1024, kWaves = kSampleThreads / 64;
constexpr int kDigits = 2048;
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
    int n_vocab;
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

struct Shared {
    unsigned long long hist[kDigits];
    double frac[64];
    uint64_t part[kWaves], parts[kWaves], ties[kWaves];
    uint64_t above;
    uint32_t digit;
    uint64_t best;
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

template <int DT>
__global__ void __launch_bounds__(kSampleThreads) lora_sample_kernel(SampleArgs a) {
    __shared__ Shared sh;
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    const int row = blockIdx.x, V = a.n_vocab;
    const void* z = (const unsigned char*)a.logits + row * a.ld * (DT == LORA_F32 ? 4 : 2);
    const float T = a.temperature ? a.temperature[row] : 1.f;
    const float p = a.top_p ? a.top_p[row] : 1.f, m = a.min_p ? a.min_p[row] : 0.f;
    const int k = a.top_k ? a.top_k[row] : 0;

    if (t < 64) sh.frac[t] = exp2(t / 64.0);
    // the largest key, and of its indices the lowest
    uint64_t best = 0;
    for (int i = t; i < V; i += kSampleThreads) {
        const uint64_t c = (uint64_t)key_of(logit<DT>(z, i)) << 32 | (0xffffffffu - (uint32_t)i);
        best = best > c ? best : c;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const uint64_t o = shfl_xor64(best, d);
        best = best > o ? best : o;
    }
    if (l == 0) sh.part[w] = best;
    __syncthreads();
    for (int i = 0; i < kWaves; ++i) best = best > sh.part[i] ? best : sh.part[i];
    const uint32_t top = (uint32_t)(best >> 32);
    if (top <= kKeyNone || !(T > 0.f)) {
        if (t == 0) {
            a.tokens[row] = top <= kKeyNone ? -1 : (int)(0xffffffffu - (uint32_t)best);
            if (a.probs) a.probs[row] = top <= kKeyNone ? 0.f : 1.f;
        }
        return;
    }
    const double lmax = logit_of(top), rate = 64 * 1.4426950408889634 / (double)T;
    auto wt = [&](uint32_t key) { return weight(key, top, lmax, rate, sh.frac); };

    // Threshold of `of` (1: counts, 2: weights) up to `limit`: a key, and what is above it.
    // With weights, keys below floor_key do not count and those of floor_key weigh floor_sum together.
    auto threshold = [&](int of, double limit, uint32_t floor_key, uint64_t floor_sum, uint64_t& above) {
        uint32_t prefix = 0;
        above = 0;
        for (int level = 0; level < 3; ++level) {
            const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
            __syncthreads();
            for (int i = t; i < kDigits; i += kSampleThreads) sh.hist[i] = 0;
            __syncthreads();
            for (int i = t; i < V; i += kSampleThreads) {
                const uint32_t key = key_of(logit<DT>(z, i));
                if (key <= kKeyNone || (level > 0 && (key >> (shift + bits)) != prefix)) continue;
                uint64_t v = 1;
                if (of == 2) v = key > floor_key ? wt(key) : 0;
                if (v) atomicAdd(&sh.hist[(key >> shift) & ((1u << bits) - 1)], (unsigned long long)v);
            }
            if (of == 2 && t == 0 && floor_sum && (level == 0 || (floor_key >> (shift + bits)) == prefix))
                atomicAdd(&sh.hist[(floor_key >> shift) & ((1u << bits) - 1)], (unsigned long long)floor_sum);
            __syncthreads();
            find_digit(above, limit, sh);
            prefix = prefix << bits | sh.digit;
            above = sh.above;
        }
        return prefix;
    };

    // kept so far: keys above tkey, and of those equal the first `share`
    uint32_t tkey = kKeyNone;
    uint32_t share = 0;
    if (k > 0 && k < V) {
        uint64_t above;
        tkey = threshold(1, (double)k, 0, 0, above);
        share = (uint32_t)(k - above);     // (at least 1; more than there are if few logits are left)
    }
    if (p < 1.f) {
        if (!(p > 0.f)) {
            tkey = top;
            share = 1;
        } else {
            uint64_t sum = 0, ties = 0;
            for (int i = t; i < V; i += kSampleThreads) {
                const uint32_t key = key_of(logit<DT>(z, i));
                if (key <= kKeyNone) continue;
                if (key > tkey) sum += wt(key);
                else if (key == tkey) ++ties;
            }
            sum = block_sum(sum, sh);
            ties = block_sum(ties, sh);
            const uint64_t floor_sum = tkey > kKeyNone ? min((uint64_t)share, ties) * wt(tkey) : 0;
            const double limit = (double)p * (double)(sum + floor_sum);
            uint64_t above;
            const uint32_t key = threshold(2, limit, tkey, floor_sum, above);
            const uint64_t each = wt(key);
            // the first `lo` of the equal ones begin below the limit
            uint32_t lo = 1, hi = key == tkey ? share : (uint32_t)V;
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo + 1) / 2;
                if ((double)(above + (mid - 1) * each) < limit) lo = mid;
                else hi = mid - 1;
            }
            tkey = key;
            share = lo;
        }
    }
    const double least = m > 0.f ? (double)(m < 1.f ? m : 1.f) * kOne : 0;
    auto kept = [&](uint64_t v) { return (double)v >= least ? v : 0; };
    const uint64_t tie_weight = tkey > kKeyNone ? kept(wt(tkey)) : 0;

    // weights and ties of each wave's part of the row, in the order of the indices
    const int per = ((V + kWaves - 1) / kWaves + 63) & ~63;
    const int i0 = min(w * per, V), i1 = min(i0 + per, V);
    uint64_t sum = 0, ties = 0;
    for (int i = i0 + l; i < i1; i += 64) {
        const uint32_t key = key_of(logit<DT>(z, i));
        if (key <= kKeyNone) continue;
        if (key > tkey) sum += kept(wt(key));
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
    uint64_t total = 0, mine = 0, ties_before = 0, seen = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i == w) {
            mine = total;
            ties_before = seen;
        }
        const uint64_t left = share > seen ? share - seen : 0;
        total += sh.parts[i] + min(left, sh.ties[i]) * tie_weight;
        seen += sh.ties[i];
    }
    const float uf = a.u[row];
    const double u = uf >= 1.f ? 1.0 : uf > 0.f ? (double)uf : 0.0;
    uint64_t target = (uint64_t)floor(u * (double)total);
    target = min(target, total - 1);
    // the wave in whose part the target lies goes through it
    uint64_t at = mine;
    for (int i = i0; i < i1; i += 64) {
        const uint32_t key = i + l < i1 ? key_of(logit<DT>(z, i + l)) : 0;
        const bool tie = key == tkey && key > kKeyNone;
        const uint64_t ballot = __ballot(tie);
        const uint64_t rank = ties_before + __popcll(ballot & ((1ull << l) - 1));
        uint64_t v = key > kKeyNone && key > tkey ? kept(wt(key)) : tie && rank < share ? tie_weight : 0;
        const uint64_t own = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t o = shfl_up64(v, d);
            if (l >= d) v += o;
        }
        if (own && at + v > target && at + v - own <= target) {
            a.tokens[row] = i + l;
            if (a.probs) a.probs[row] = (float)((double)own / (double)total);
        }
        at += __shfl((unsigned long long)v, 63, 64);
        ties_before += __popcll(ballot);
        if (at > target) break;
    }
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
    *bytes = 16;
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
    if (dtype == LORA_F16) hipLaunchKernelGGL(lora_sample_kernel<LORA_F16>, dim3(n_rows), dim3(kSampleThreads), 0, st, a);
    else if (dtype == LORA_BF16) hipLaunchKernelGGL(lora_sample_kernel<LORA_BF16>, dim3(n_rows), dim3(kSampleThreads), 0, st, a);
    else hipLaunchKernelGGL(lora_sample_kernel<LORA_F32>, dim3(n_rows), dim3(kSampleThreads), 0, st, a);
    return check_launch("lora_sample");
}

}  // extern "C"
