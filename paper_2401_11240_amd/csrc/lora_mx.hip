// gfx950 kernels of rows in blocks (include/lora_mx.h): the norm between two layers, and
// values into blocks and back.  The product is in lora_mx_gemm.hip.
//
// All three read and write every element once: large calls are bound by HBM, a few rows by
// the launch and its chain of dependent loads.  A thread works on chunks of 8 consecutive
// elements (16 bytes of 16-bit values), so a block of 32 is the four lanes of a quad, and its
// largest magnitude two DPP steps.
#include <cmath>

#include <algorithm>
#include <type_traits>

#include "lora_device.h"
#include "lora_mx_internal.h"

namespace lora {

int check_mx(const char* name, const lora_mx_t* q) {
    const std::string n(name);
    if (!q) return set_error(LORA_E_ARG, n + " is NULL");
    if (q->format != LORA_E4M3 && q->format != LORA_E2M1)
        return set_error(LORA_E_ARG, n + ": format must be LORA_E4M3 or LORA_E2M1");
    if (q->n_rows < 0) return set_error(LORA_E_ARG, n + ": negative n_rows");
    if (q->h < 8 || q->h % 8) return set_error(LORA_E_SHAPE, n + ": h must be a positive multiple of 8");
    if (q->ld_codes % 16 || q->ld_codes < mx_row_bytes(q->h, q->format) || q->ld_codes > (1ll << 40))
        return set_error(LORA_E_SHAPE, n + ": ld_codes must be a multiple of 16 and hold a row's blocks");
    if (q->ld_scales % 4 || q->ld_scales < mx_blocks(q->h) || q->ld_scales > (1ll << 40))
        return set_error(LORA_E_SHAPE, n + ": ld_scales must be a multiple of 4 and hold a row's scales");
    if (q->n_rows > 0 && (!q->codes || !q->scales)) return set_error(LORA_E_ARG, n + ": codes or scales is NULL");
    if (!is_aligned16(q->codes)) return set_error(LORA_E_ALIGN, n + ": codes not 16-byte aligned");
    if ((uintptr_t)q->scales & 3u) return set_error(LORA_E_ALIGN, n + ": scales not 4-byte aligned");
    return LORA_OK;
}

namespace {

constexpr int kNormMax = 65536;            // elements of a row: 1024 threads of 8 chunks
constexpr int kNormRows = 1 << 20;         // of one launch: its threads stay below 2^32

// 32-bit rows in memory, beside FmtF16 and FmtBF16.
struct FmtF32 {};
template <class Fmt>
struct Chunk {                             // 8 consecutive elements
    static constexpr int kBytes = 16;
    u32x4 w;
    __device__ __forceinline__ void load(const unsigned char* p) { w = *(const u32x4*)p; }
    __device__ __forceinline__ void load_far(const unsigned char* p) { w = __builtin_nontemporal_load((const u32x4*)p); }
    __device__ __forceinline__ void clear() { w = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = Fmt::to_f32(lo16(w[i]));
            v[2 * i + 1] = Fmt::to_f32(hi16(w[i]));
        }
    }
    static __device__ __forceinline__ void put(unsigned char* p, const float (&v)[8]) {
        *(u32x4*)p = u32x4{Fmt::pack2(v[0], v[1]), Fmt::pack2(v[2], v[3]), Fmt::pack2(v[4], v[5]), Fmt::pack2(v[6], v[7])};
    }
    // past the caches: 16 bytes a lane of consecutive lanes are whole lines
    static __device__ __forceinline__ void put_far(unsigned char* p, const float (&v)[8]) {
        __builtin_nontemporal_store(u32x4{Fmt::pack2(v[0], v[1]), Fmt::pack2(v[2], v[3]), Fmt::pack2(v[4], v[5]), Fmt::pack2(v[6], v[7])}, (u32x4*)p);
    }
};
template <>
struct Chunk<FmtF32> {
    static constexpr int kBytes = 32;
    u32x4 w[2];
    __device__ __forceinline__ void load(const unsigned char* p) {
        w[0] = ((const u32x4*)p)[0];
        w[1] = ((const u32x4*)p)[1];
    }
    __device__ __forceinline__ void load_far(const unsigned char* p) {
        w[0] = __builtin_nontemporal_load((const u32x4*)p);
        w[1] = __builtin_nontemporal_load((const u32x4*)p + 1);
    }
    __device__ __forceinline__ void clear() { w[0] = w[1] = u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i >> 2][i & 3]);
    }
    static __device__ __forceinline__ void put(unsigned char* p, const float (&v)[8]) {
        ((f32x4*)p)[0] = f32x4{v[0], v[1], v[2], v[3]};
        ((f32x4*)p)[1] = f32x4{v[4], v[5], v[6], v[7]};
    }
    // (halves of lines, which the L2 has to put together: past it 8192 x 8192 into 8 bits and back took 146 us, through it 142)
    static __device__ __forceinline__ void put_far(unsigned char* p, const float (&v)[8]) { put(p, v); }
};

// The larger of the quad's values, in all four lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true)); // lanes 2 3 0 1
}

// One chunk of a block into its codes (8 bytes of E4M3, 4 of E2M1), the four lanes of a quad
// together; every lane returns the block's scale byte.  Magnitudes compare as integers, NaN above
// infinity above the rest; the factor 2^(127 - scale) is a float for every scale below 255, and
// the product with it exact but for results below 2^-126, which round to the code 0 either way.
__device__ __forceinline__ uint32_t encode(const float (&v)[8], int format, u32x2& codes) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = quad_max(m);
    codes = u32x2{0, 0};
    if (m >= 0x7f800000u) return 255;
    const int top = (int)(m >> 23), emax = format == LORA_E4M3 ? 8 : 2;
    const int scale = top > emax ? top - emax : 0;
    const float f = __uint_as_float((uint32_t)(254 - scale) << 23);
    float s[8];
    if (format == LORA_E4M3) {
        // (conversions past 448 give NaN)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = __builtin_amdgcn_fmed3f(v[i] * f, -448.f, 448.f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * i], s[4 * i + 1], 0, false);
            codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[4 * i + 2], s[4 * i + 3], w, true);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = v[i] * f;
        uint32_t w = 0;                    // (conversions past 6 give 6)
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[0], s[1], 1.f, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[2], s[3], 1.f, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[4], s[5], 1.f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, s[6], s[7], 1.f, 3);
        codes[0] = w;
    }
    return (uint32_t)scale;
}

// Chunk c of a row's codes and, by the quad's first lane, the block's scale.
__device__ __forceinline__ void put_codes(unsigned char* codes, unsigned char* scales, int c, int format, const u32x2& w,
                                          uint32_t scale) {
    if (format == LORA_E4M3) *(u32x2*)(codes + 8 * (int64_t)c) = w;
    else *(uint32_t*)(codes + 4 * (int64_t)c) = w[0];
    if ((c & 3) == 0) scales[c >> 2] = (unsigned char)scale;
}

// ---------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------

struct NormArgs {
    const unsigned char *x, *residual, *weight;
    unsigned char *total, *y, *codes, *scales;
    int64_t ldx, ldr, ldt, ldy;            // bytes
    int64_t ld_codes, ld_scales;
    int n_rows, chunks, format;            // chunks of a row
    float eps;
    double inv_h;
};

// The float32 y with a rest of the exact value beyond it, moved by its last bit towards the rest.
__device__ __forceinline__ float towards(float y, float rest) {
    const uint32_t b = __float_as_uint(y);
    constexpr int kFinite = 0x198;         // normal and subnormal, of either sign: not zero, infinity or NaN
    return __builtin_amdgcn_classf(rest, kFinite) ? __uint_as_float(b + ((int)(b ^ __float_as_uint(rest)) >> 31 | 1)) : y;
}

// A row by TPR threads (a wave, or a workgroup of 256 or 1024), CH chunks each, which stay in
// registers between the sum of squares and the outputs: x and the residual are read once.  HBM bounds many rows (8437 x
// 5120 with all outputs 70-71 us, 5.5 TB/s), the launch and the chain of load, sum and barrier a few (one row of 4096: 3.3 us).
// Rows of 16 bits are written past the caches (256 x 8192 6.6 -> 5.6 us, 1024 x 8192 18.4 -> 14.2, 8437 x 5120 73.5 -> 71.3); the
// products that read them next take the same time either way.  Rows of more than 32768 elements, eight chunks a thread, are held to 128
// registers by their 1024 threads and spill 88 (binary16) and 72 bytes (bfloat16) a lane: 256 x 65536 36 and 32 us, 4.2 and 4.8 TB/s.
// Every output of a row is written after all of its inputs are read where that is asked
// for: y depends on the whole row, and total[i] only on x[i] and residual[i].
template <class Fmt, int CH, int TPR>
__global__ void __launch_bounds__(TPR < kThreads ? kThreads : TPR) lora_norm_kernel(NormArgs a) {
    constexpr int kRows = TPR < kThreads ? kThreads / TPR : 1;     // of a workgroup
    const int t = threadIdx.x % TPR;
    const int row = blockIdx.x * kRows + threadIdx.x / TPR;
    if (row >= a.n_rows) return;           // (a whole wave: without a barrier below)
    const unsigned char* x = a.x + row * a.ldx;
    constexpr uint32_t kOnes = std::is_same<Fmt, FmtF16>::value ? 0x3c003c00u : 0x3f803f80u;
    Chunk<Fmt> in[CH], res[CH], g[CH];       // (zeros and ones for a residual and a weight that are not there)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TPR + t;
        in[i].clear();
        res[i].clear();
        g[i].w = u32x4{kOnes, kOnes, kOnes, kOnes};
        if (c < a.chunks) {
            in[i].load(x + 16 * c);
            if (a.residual) res[i].load(a.residual + row * a.ldr + 16 * c);
            if (a.weight) g[i].load(a.weight + 16 * c);
        }
    }
    float s[CH][8];
    double sum = 0.;                       // (the squares of a chunk in float32, chunks in binary64)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        float r[8];
        in[i].get(s[i]);
        res[i].get(r);
        float q = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[i][e] += r[e];
            q = fmaf(s[i][e], s[i][e], q);
        }
        sum += q;
        if (a.total && i * TPR + t < a.chunks) Chunk<Fmt>::put_far(a.total + row * a.ldt + 16 * (i * TPR + t), s[i]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if constexpr (TPR > 64) {
        __shared__ double part[TPR / 64];
        if ((t & 63) == 0) part[t >> 6] = sum;
        __syncthreads();
        sum = 0.;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) sum += part[i];
    }
    // 1 / sqrt in binary64 (an estimate and one Newton step), as a float32 and what it leaves: with them the product
    // s rstd w below is off by little more than its rounding to float32.  That one matters to the outputs' only where it
    // ends half way between two of their values: there the rest decides.  (Without that about one of 2 million 8-bit
    // codes comes out next to the right one; with the rest carried through every product 8437 x 5120 takes 82.7 us, so
    // 73.7.)
    const double ms = sum * a.inv_h + (double)a.eps;
    double r64 = __builtin_amdgcn_rsq(ms);
    r64 = ms < INFINITY ? r64 * (1.5 - 0.5 * ms * r64 * r64) : r64;    // (0 for infinity, NaN for NaN)
    const float rstd = (float)r64, rest = (float)(r64 - (double)rstd);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TPR + t;
        constexpr uint32_t kHalfWay = std::is_same<Fmt, FmtF16>::value ? 0xfff : 0x7fff;
        float w[8], v[8];
        g[i].get(w);
        uint32_t half_way = ~0u;           // 0 if one of the chunk may lie half way between two values of an output
        auto product = [&](int e, float& lo_by) __attribute__((always_inline)) {
            const float hi = s[i][e] * rstd, lo = fmaf(s[i][e], rest, fmaf(s[i][e], rstd, -hi));
            lo_by = lo * w[e];
            return hi;
        };
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float lo_by;
            const float hi = product(e, lo_by);
            v[e] = fmaf(hi, w[e], lo_by);
            half_way = min(half_way, __float_as_uint(v[e]) & kHalfWay);
        }
        if (__builtin_expect(__any(half_way == 0 && c < a.chunks), 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float lo_by;
                const float hi = product(e, lo_by);
                if ((__float_as_uint(v[e]) & kHalfWay) == 0) v[e] = towards(v[e], fmaf(hi, w[e], -v[e]) + lo_by);
            }
        }
        if (a.y && c < a.chunks) Chunk<Fmt>::put_far(a.y + row * a.ldy + 16 * c, v);
        if (a.codes && i * TPR < a.chunks) {
            if (c >= a.chunks) {           // (rows of zeros may not be: 0 times infinity)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
            }
            u32x2 codes;
            const uint32_t scale = encode(v, a.format, codes);
            if (c < ((a.chunks + 3) & ~3))
                put_codes(a.codes + row * a.ld_codes, a.scales + row * a.ld_scales, c, a.format, codes, scale);
        }
    }
}

template <class Fmt, int CH, int TPR>
void launch_norm_form(const NormArgs& a, hipStream_t st) {
    constexpr int kRows = TPR < kThreads ? kThreads / TPR : 1;
    hipLaunchKernelGGL((lora_norm_kernel<Fmt, CH, TPR>), dim3((a.n_rows + kRows - 1) / kRows), dim3(TPR * kRows), 0, st, a);
}
// MOST: the most chunks a thread that TPR threads are given
template <class Fmt, int TPR, int MOST>
void launch_norm_tpr(const NormArgs& a, hipStream_t st) {
    const int ch = (a.chunks + TPR - 1) / TPR;
    if (ch <= 1) launch_norm_form<Fmt, 1, TPR>(a, st);
    else if (ch <= 2) launch_norm_form<Fmt, 2, TPR>(a, st);
    else if (ch <= 4) launch_norm_form<Fmt, std::min(MOST, 4), TPR>(a, st);
    else launch_norm_form<Fmt, MOST, TPR>(a, st);
}

template <class Fmt>
void launch_norm(const NormArgs& a, hipStream_t st) {
    // many short rows: a wave each, without barriers; long ones, and rather long ones that are few: as many threads as there are
    // chunks, for the sake of the loads on their way (us with 256 against 1024 threads, h 8192: 64 rows 5.9 against 4.4, 256 rows
    // 7.2 against 5.8, 2048 rows 31.6 against 30.3; h 4096: one row 3.7 against 3.3, 256 rows 4.5 against 4.1, 512 rows 5.9 against
    // 6.2; 8437 x 5120 70.0 against 72.2; a wave against 256 threads: 4000 x 1024 8.1 against 9.8, 1024 x 2048 7.2 against 5.7)
    const int tpr = a.n_rows >= 1024 && a.chunks <= 128 ? 64 : a.chunks > 768 || (a.chunks >= 512 && a.n_rows <= 256) ? 1024 : 256;
    if (tpr == 64) launch_norm_tpr<Fmt, 64, 2>(a, st);
    else if (tpr == 256) launch_norm_tpr<Fmt, 256, 4>(a, st);
    else launch_norm_tpr<Fmt, 1024, kNormMax / 8 / 1024>(a, st);
}

// ---------------------------------------------------------------------------
// values into blocks and back
// ---------------------------------------------------------------------------

struct BlocksArgs {
    unsigned char *values, *codes, *scales;
    int64_t ld, ld_codes, ld_scales;       // bytes
    uint32_t total;                        // chunks of the launch, whole blocks
    uint32_t per_row;                      // chunks of a row's blocks
    uint32_t chunks;                       // chunks of a row
    int format;
};

// A chunk a thread, blocks in the order of memory, rows written past the caches: a 28672 x 8192 weight into 4 bits and back takes
// 189 us, 5.7 TB/s (254 through the caches; a large copy runs at 4.9 TB/s); 203 rows of 4096 into 8 bits and back 4.4, two launches.
// FAR: values are read past the caches.
template <class Fmt, bool FAR>
__global__ void __launch_bounds__(kThreads) lora_mx_quantize_kernel(BlocksArgs a) {
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.total) return;              // (whole quads: total is a multiple of 4)
    const uint32_t row = i / a.per_row, c = i - row * a.per_row;
    Chunk<Fmt> in;
    in.clear();
    const unsigned char* from = a.values + row * a.ld + (uint32_t)Chunk<Fmt>::kBytes * (uint64_t)c;
    if (c < a.chunks) {
        if (FAR) in.load_far(from);
        else in.load(from);
    }
    float v[8];
    in.get(v);
    u32x2 w;
    const uint32_t scale = encode(v, a.format, w);
    put_codes(a.codes + row * a.ld_codes, a.scales + row * a.ld_scales, (int)c, a.format, w, scale);
}

template <class Fmt>
__global__ void __launch_bounds__(kThreads) lora_mx_dequantize_kernel(BlocksArgs a) {
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.total) return;
    const uint32_t row = i / a.chunks, c = i - row * a.chunks;
    const unsigned char* codes = a.codes + row * a.ld_codes;
    const uint32_t s = a.scales[row * a.ld_scales + (c >> 2)];
    const float f = s == 255 ? __uint_as_float(0x7fc00000u) : s ? __uint_as_float(s << 23) : __uint_as_float(0x00400000u);
    float v[8];
    if (a.format == LORA_E4M3) {
        const u32x2 w = *(const u32x2*)(codes + 8 * (uint64_t)c);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
            v[4 * j] = lo[0];
            v[4 * j + 1] = lo[1];
            v[4 * j + 2] = hi[0];
            v[4 * j + 3] = hi[1];
        }
    } else {
        const uint32_t w = *(const uint32_t*)(codes + 4 * (uint64_t)c);
        const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1),
                   p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
        v[0] = p0[0], v[1] = p0[1], v[2] = p1[0], v[3] = p1[1], v[4] = p2[0], v[5] = p2[1], v[6] = p3[0], v[7] = p3[1];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= f;
    Chunk<Fmt>::put_far(a.values + row * a.ld + (uint32_t)Chunk<Fmt>::kBytes * (uint64_t)c, v);
}

int element_bytes(int32_t dtype) { return dtype == LORA_F32 ? 4 : 2; }

// A matrix [n_rows, ld] of h elements a row.
int check_values(const char* name, const void* p, const char* ld_name, int64_t ld, int64_t h, int32_t n_rows) {
    if (ld > (1ll << 40)) return set_error(LORA_E_SHAPE, std::string(ld_name) + " exceeds 2^40");
    return check_kv_rows(name, p, ld_name, ld, h, n_rows);
}

constexpr uint32_t kLaunchChunks = 1u << 30;   // of one launch, at most (or one row)
constexpr int64_t kFar = 256 << 20;            // bytes of the memory-side cache

template <bool BACK>
int enqueue_blocks(const char* name, const lora_mx_t* q, const void* values, int64_t ld, int32_t dtype, void* stream) {
    if (q->n_rows == 0) return LORA_OK;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return set_error(LORA_E_HIP, std::string(name) + ": no device for the stream");
    BlocksArgs a;
    a.ld = ld * element_bytes(dtype);
    a.ld_codes = q->ld_codes;
    a.ld_scales = q->ld_scales;
    a.chunks = (uint32_t)q->h / 8;
    a.per_row = 4 * (uint32_t)mx_blocks(q->h);
    a.format = q->format;
    // (more than the memory-side cache holds, of which nothing is there and nothing would stay: 28672 x 8192 in bfloat16 into 4
    // bits and back 189 us against 221 through the caches; 13824 x 5120 72.0 against 70.7, 203 x 4096 4.7 against 4.5)
    const bool far = (int64_t)q->n_rows * q->h * element_bytes(dtype) > kFar;
    const uint32_t row = BACK ? a.chunks : a.per_row;
    const int32_t step = (int32_t)std::max(1u, kLaunchChunks / row);
    for (int64_t r = 0; r < q->n_rows; r += step) {
        const int64_t n = std::min<int64_t>(step, q->n_rows - r);
        a.values = (unsigned char*)const_cast<void*>(values) + r * a.ld;
        a.codes = (unsigned char*)q->codes + r * a.ld_codes;
        a.scales = (unsigned char*)q->scales + r * a.ld_scales;
        a.total = (uint32_t)n * row;
        const dim3 grid((a.total + kThreads - 1) / kThreads);
        if constexpr (BACK) {
            if (dtype == LORA_F16) hipLaunchKernelGGL(lora_mx_dequantize_kernel<FmtF16>, grid, dim3(kThreads), 0, st, a);
            else if (dtype == LORA_BF16) hipLaunchKernelGGL(lora_mx_dequantize_kernel<FmtBF16>, grid, dim3(kThreads), 0, st, a);
            else hipLaunchKernelGGL(lora_mx_dequantize_kernel<FmtF32>, grid, dim3(kThreads), 0, st, a);
        } else {
            auto kernel = dtype == LORA_F16    ? far ? lora_mx_quantize_kernel<FmtF16, true> : lora_mx_quantize_kernel<FmtF16, false>
                          : dtype == LORA_BF16 ? far ? lora_mx_quantize_kernel<FmtBF16, true> : lora_mx_quantize_kernel<FmtBF16, false>
                          : far ? lora_mx_quantize_kernel<FmtF32, true> : lora_mx_quantize_kernel<FmtF32, false>;
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, a);
        }
        if (int rc = check_launch(name)) return rc;
    }
    return LORA_OK;
}

int check_blocks(const lora_mx_t* q, const char* name, const void* p, const char* ld_name, int64_t ld, int32_t dtype) {
    if (int rc = check_mx("q", q)) return rc;
    if (dtype != LORA_F16 && dtype != LORA_BF16 && dtype != LORA_F32)
        return set_error(LORA_E_ARG, "dtype must be LORA_F16, LORA_BF16 or LORA_F32");
    if (int rc = check_values(name, p, ld_name, ld, q->h, q->n_rows)) return rc;
    const int64_t e = element_bytes(dtype);
    const Span v(p, q->n_rows, ld * e, q->h * e), c = codes_span(q), s = scales_span(q);
    if (v.meets(c) || v.meets(s) || c.meets(s)) return set_error(LORA_E_OVERLAP, std::string(name) + ", codes and scales overlap");
    return LORA_OK;
}

}  // namespace
}  // namespace lora

using namespace lora;

extern "C" {

int lora_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, float eps,
              int32_t n_rows, int32_t h, int32_t dtype, void* total, int64_t ldt, void* y, int64_t ldy,
              const lora_mx_t* q, void* stream) {
    if (dtype != LORA_F16 && dtype != LORA_BF16) return set_error(LORA_E_ARG, "dtype must be LORA_F16 or LORA_BF16");
    if (n_rows < 0) return set_error(LORA_E_ARG, "negative n_rows");
    if (h < 8 || h % 8 || h > kNormMax) return set_error(LORA_E_SHAPE, "h must be a multiple of 8 in [8, 65536]");
    if (!(eps > 0.f) || !std::isfinite(eps)) return set_error(LORA_E_ARG, "eps must be positive and finite");
    if (!y && !q) return set_error(LORA_E_ARG, "y and q are NULL");
    if (int rc = check_values("x", x, "ldx", ldx, h, n_rows)) return rc;
    if (residual)
        if (int rc = check_values("residual", residual, "ldr", ldr, h, n_rows)) return rc;
    if (total)
        if (int rc = check_values("total", total, "ldt", ldt, h, n_rows)) return rc;
    if (y)
        if (int rc = check_values("y", y, "ldy", ldy, h, n_rows)) return rc;
    if (!is_aligned16(weight)) return set_error(LORA_E_ALIGN, "weight not 16-byte aligned");
    if (q) {
        if (int rc = check_mx("q", q)) return rc;
        if (q->h != h || q->n_rows != n_rows) return set_error(LORA_E_SHAPE, "q has other rows or another h");
    }
    struct Part {
        const char* name;
        const void* p;
        int64_t ld;
        Span s;
    };
    const Part in[3] = {{"x", x, ldx, Span(x, n_rows, 2 * ldx, 2 * h)},
                        {"residual", residual, ldr, Span(residual, n_rows, 2 * ldr, 2 * h)},
                        {"weight", weight, 0, Span(weight, 1, 0, 2 * h)}};
    const Part out[4] = {{"total", total, ldt, Span(total, n_rows, 2 * ldt, 2 * h)},
                         {"y", y, ldy, Span(y, n_rows, 2 * ldy, 2 * h)},
                         {"codes", q ? q->codes : nullptr, 0, q ? codes_span(q) : Span(nullptr, 0, 0, 0)},
                         {"scales", q ? q->scales : nullptr, 0, q ? scales_span(q) : Span(nullptr, 0, 0, 0)}};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 3; ++j) {
            const bool same = i < 2 && j < 2 && out[i].p == in[j].p && out[i].ld == in[j].ld;
            if (out[i].s.meets(in[j].s) && !same)
                return set_error(LORA_E_OVERLAP, std::string(out[i].name) + " and " + in[j].name + " overlap");
        }
        for (int j = 0; j < i; ++j)
            if (out[i].s.meets(out[j].s))
                return set_error(LORA_E_OVERLAP, std::string(out[i].name) + " and " + out[j].name + " overlap");
    }
    if (n_rows == 0) return LORA_OK;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_norm: no device for the stream");
    NormArgs a;
    a.x = (const unsigned char*)x;
    a.residual = (const unsigned char*)residual;
    a.weight = (const unsigned char*)weight;
    a.total = (unsigned char*)total;
    a.y = (unsigned char*)y;
    a.codes = q ? (unsigned char*)q->codes : nullptr;
    a.scales = q ? (unsigned char*)q->scales : nullptr;
    a.ldx = 2 * ldx;
    a.ldr = 2 * ldr;
    a.ldt = 2 * ldt;
    a.ldy = 2 * ldy;
    a.ld_codes = q ? q->ld_codes : 0;
    a.ld_scales = q ? q->ld_scales : 0;
    a.chunks = h / 8;
    a.format = q ? q->format : 0;
    a.eps = eps;
    a.inv_h = 1.0 / h;
    for (int left = n_rows; left > 0; left -= kNormRows) {
        a.n_rows = std::min(left, kNormRows);
        if (dtype == LORA_F16) launch_norm<FmtF16>(a, st);
        else launch_norm<FmtBF16>(a, st);
        if (int rc = check_launch("lora_norm")) return rc;
        a.x += kNormRows * a.ldx;
        if (a.residual) a.residual += kNormRows * a.ldr;
        if (a.total) a.total += kNormRows * a.ldt;
        if (a.y) a.y += kNormRows * a.ldy;
        if (a.codes) {
            a.codes += kNormRows * a.ld_codes;
            a.scales += kNormRows * a.ld_scales;
        }
    }
    return LORA_OK;
}

int lora_mx_quantize(const void* x, int64_t ldx, int32_t dtype, const lora_mx_t* q, void* stream) {
    if (int rc = check_blocks(q, "x", x, "ldx", ldx, dtype)) return rc;
    return enqueue_blocks<false>("lora_mx_quantize", q, x, ldx, dtype, stream);
}

int lora_mx_dequantize(const lora_mx_t* q, void* y, int64_t ldy, int32_t dtype, void* stream) {
    if (int rc = check_blocks(q, "y", y, "ldy", ldy, dtype)) return rc;
    return enqueue_blocks<true>("lora_mx_dequantize", q, y, ldy, dtype, stream);
}

}  // extern "C"
