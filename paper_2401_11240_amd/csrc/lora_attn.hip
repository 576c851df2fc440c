// gfx950 kernels of attention over the paged key-value cache (include/lora_kv.h).
//
// Decode: one new token per sequence. Per visible token and key-value head 4 head_dim
// bytes are read and 4 group head_dim operations done on them (group: the q heads
// that share the head), far below what the chip computes per byte read: the launch is
// bound by HBM, so what counts is that every compute unit reads all the time and that
// nothing is read twice.
//
//   Work: the visible tokens of every (sequence, key-value head) are cut into tiles
//   of kTile tokens; all tiles of the launch lie in one line, and workgroup w takes
//   tiles [w R, (w + 1) R), R from the lengths as they are on the device. So the load
//   is even whatever the lengths, one long sequence fills the chip, and a recorded
//   launch serves every later token.
//
//   Tile: four waves of 32 tokens. S^T = K Q^T on v_mfma_f32_16x16x32 with the tokens
//   as rows, so that a lane's four results are four tokens of one head; in the
//   product O^T = V^T P^T the 32 tokens may stand in any order, and the one taken is
//   that of the lanes that hold their weights: P goes from one product into the other
//   without leaving its lane. V^T comes from 8 tokens x head_dim / 16 elements per
//   lane, transposed in registers (one v_perm per word). No LDS in the loop, each
//   byte of K and V is loaded once, 16 bytes per lane. The group's heads are the 16
//   columns; most of the arithmetic is on empty columns when few heads share keys,
//   and free beside the reads.
//
//   Join: a head's partial results (float32 sums with their maximum) of the four
//   waves meet in LDS, those of several workgroups in device memory: the last one to
//   arrive, counted by an atomic, adds them up, in an order that does not depend on
//   which one that is. (16 at a time: a sequence of 100000 tokens, 16/1 heads, in
//   25 us, where one workgroup that joined all of them took 83.)
//
//   Measured: 128 sequences of 64 to 1024 tokens, 40/40 heads, 911 MB read in 185 us
//   (4.9 TB/s; a large copy reads and writes 4.8 TB/s); 256 sequences of 64 to 8192
//   tokens, 64/8 heads, 2.1 GB in 389 us (5.4 TB/s). Bound by HBM there, the matrix
//   cores busy for 4% of the time; by the length of the chain page, key, score, sum,
//   join where there is little to read (one sequence of 300 tokens 8.7 us).
//
// Prompt: rows of segments, each row and q head a column of the products. Per
// key-value head, tile of columns and token 4 head_dim operations per column: with
// hundreds of columns per token read this is matrix work, bound by the MFMA rate and
// by the vector instructions that make weights of the scores, which share a SIMD's
// issue slots. With m the running maximum of a column:
//
//   s_j = scale log2(e) q . K[j],  w_j = 2^(s_j - m),  O = sum w_j V[j],  S = sum w_j
//
// and when a maximum rises by more than kSlack powers of two, O and S are multiplied
// by 2^(old - new). Smaller rises leave m as it is, so that the product is needed in few
// steps. Weights are then up to 2^kSlack, and the heaviest, 1 with the exact maximum, is
// rounded like the others. What rounding weights costs, as relative error against 64 bits (the
// output's own rounding alone, with weights in float32: 0.0016-0.0017 in bf16, 0.00020 in f16): with the
// exact maximum, in the decode kernel, 0.0019 and 0.00022; here 0.0020 (prompts of 256 to 1024 rows) to 0.0023
// (16384 tokens) and 0.00023 to 0.00026.
//
//   Tile: 128 columns, 32 per wave; steps of 64 tokens. S^T = K Q^T and O^T = V^T P^T
//   on v_mfma_f32_32x32x16: a lane has one column's scores, so maximum and sum need
//   one exchange between two lanes, and the weights of a lane are the operand of the
//   second product as they are. Q stays in registers.
//
//   K and V go through LDS, two buffers each, by buffer-to-LDS loads that the four
//   waves share: 16-byte chunks in slots permuted by their token, so that neither the
//   reads of K nor the transposing reads of V meet in a bank (1% of the cycles). One
//   barrier per step. A step's loads are issued one at a time between the products of
//   its scores, its weights made between its products with V; every LDS read is two
//   to four products ahead of its use.
//
//   Order: a launch's tiles are taken from the end, where a row sees the most; the
//   heads of a tile are next to each other, so that an XCD keeps to its heads (block
//   i runs on XCD i % 8). Few tiles: the tokens are divided over up to 16 workgroups
//   (parts), and few columns go to lora_attn_prompt_few_kernel.
//
//   A hidden token's value may be anything. Its weight is zero, which keeps it out
//   unless it is an infinity or a NaN. So a tile whose output is not finite is
//   computed again by run_careful(), and so is one whose scores reach 2^21 powers of two.
//
//   Measured: 2048 rows behind 14336 tokens, 64/8 heads of width 128, bf16: 0.94-1.0
//   ms, 1.03-1.09 PFLOP/s (library products reach 1.3 at their best), matrix cores
//   busy for 55% of the cycles; four prompts of 2500 to 6000 rows under a window of
//   1024, 24/8 heads of width 64, f16: 130 us, 0.6 PFLOP/s (twice the weights per
//   product: vector instructions are issued in 72% of the cycles); sixteen prompts of
//   256 to 1024 rows, 32/32 heads: 85 us, 3 TB/s (tiles of six steps on average,
//   whose start and end count). Widths between 64, 128 and 256 do the work of the next of them: the first case takes
//   620 us at 64, 853-888 at 72 to 96, 944 at 128, 1639-1722 at 136 to 192, 1828 at 256.
#include <algorithm>
#include <cmath>
#include <new>

#include "lora_device.h"
#include "lora_kv_internal.h"

using namespace lora;

namespace {
// Workgroups of the decode kernel per compute unit: registers for a tile's K and V
// in flight beside the output.  (Two of width 256 spill: 64 sequences of 64 to 8192
// tokens, 32/8 heads, 199 against 190 us.)
constexpr int decode_per_cu(int dp) { return dp == 256 ? 1 : dp == 128 ? 3 : 4; }
}

struct lora_attn_s {
    int device = 0;
    int n_cu = 0;
    uint32_t* counters = nullptr;          // a cache line each: partial results that have arrived; 0 between launches
    float* slots = nullptr;                // two partial results per workgroup
};

namespace {

struct AttnArgs {
    const uint16_t *k, *v;                 // the layer's
    const uint16_t* q;
    uint16_t* out;
    const int32_t *tables, *lens, *seg_offset;
    int64_t page_stride, head_stride, row_stride, ldq, ldo;
    int32_t n_rows, n_seqs, ld_table, max_len, n_pages, page_shift;
    int32_t group, head_dim;
    int32_t window, n_sinks;
    float scale;
};

constexpr int kTile = 128;                 // tokens per tile: 32 per wave
constexpr int kWaveTokens = 32;
constexpr int kHeads = 16;                 // q heads per group tile (columns of the MFMA)
constexpr float kLog2e = 1.44269504088896340736f;

// Weights are taken 2^kLift above their maximum's 1, in binary16, and the factor cancels in the division by their
// sum: what is rounded to zero begins 2^-32 below the largest instead of 2^-25 (131072 tokens just below
// 2^-25, behind a first token that holds the maximum, were 0.4% of a sum and came out as none).
// With kSlack more the largest is 2^15.
template <class Fmt>
constexpr float kLift = Fmt::kNarrowRange ? 7.f : 0.f;

constexpr int kCounters = 3;               // per workgroup: see arrive()

// The join gives a tile's q heads 16 threads each, of 256; what they leave goes to parts.
__host__ __device__ constexpr int head_slots(int heads) { return heads > 8 ? 16 : heads > 4 ? 8 : heads > 2 ? 4 : heads; }
// Parts that one workgroup joins: four for each group of threads at once, or 16.
__host__ __device__ constexpr int join_width(int heads) { return heads > 2 ? 16 : 64 / head_slots(heads); }

// One partial result in device memory: kHeads rows of the unnormalised output, then the
// maxima and the sums.
constexpr int slot_floats(int dp) { return kHeads * dp + 2 * kHeads; }

// The visible tokens of a decode row: [0, sinks) and [first, len), in tiles
// [0, sink_tiles) and [win_tile, ..).  At least one tile, so that a row that
// sees nothing is written as well.
struct Span {
    int len, first, sinks, sink_tiles, win_tile, n;
};
__device__ __forceinline__ Span decode_span(const AttnArgs& a, int len) {
    Span p;
    p.len = len;
    p.first = a.window ? max(0, p.len - a.window) : 0;
    p.sinks = min(a.n_sinks, p.first);
    p.sink_tiles = (p.sinks + kTile - 1) / kTile;
    p.win_tile = max(p.first / kTile, p.sink_tiles);
    p.n = max(1, p.sink_tiles + (p.len + kTile - 1) / kTile - p.win_tile);
    return p;
}
__device__ __forceinline__ int tile_token(const Span& p, int i) {
    return (i < p.sink_tiles ? i : p.win_tile + i - p.sink_tiles) * kTile;
}

struct DecodeArgs {
    AttnArgs a;
    uint32_t* counters;
    float* slots;
    int32_t heads_per_seq;                 // kv heads times group tiles
    int32_t group_tiles;
};

// The largest of v over the four lanes l % 16 + 16 i, in each of them.
__device__ __forceinline__ float max_over_quarters(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_over_quarters(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

template <class Fmt, int DP>
struct DecodeWave {
    static constexpr int NS = DP / 32;     // MFMA steps of a score
    static constexpr int NV = DP / 16;     // elements of V per lane and token
    static constexpr int VW = NV / 2;      // the same in words
    const AttnArgs& a;
    const int l, w;
    u32x4 q[NS];
    u32x4 kf[2][NS];
    uint32_t vf[8][VW];
    f32x4 o[NV];
    float m, sum;
    uint32_t koff[NS], voff[(NV + 7) / 8];
    uint32_t page_bytes, row_bytes;
    int pages;                             // lane i: page of subtile i of the next 32 tiles
    int pages_at;                          // the first of those tiles
    bool has_page[2];                      // of the tile in kf, for its two subtiles
    __device__ __forceinline__ DecodeWave(const AttnArgs& args)
        : a(args), l(threadIdx.x & 63), w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) {
        row_bytes = (uint32_t)a.row_stride * 2u;
        page_bytes = ((1u << a.page_shift) - 1) * row_bytes + (uint32_t)a.head_dim * 2u;
#pragma unroll
        for (int i = 0; i < NS; ++i) koff[i] = 32 * i + 8 * (l >> 4) < a.head_dim ? 64u * i + 16u * (l >> 4) : (uint32_t)kOut;
#pragma unroll
        for (int i = 0; i < (NV + 7) / 8; ++i)
            voff[i] = (l & 15) * NV + 8 * i < a.head_dim ? (l & 15) * NV * 2u + 16u * i : (uint32_t)kOut;
    }

    // Pages of the subtiles of tiles [i, i + 32): lane 2 t + u that of tile i + t's tokens 32 w + 16 u on, -1 where none is seen.
    __device__ __forceinline__ void load_pages(const Span& p, int s, int i, int end) {
        const int t = i + (l >> 1);
        const int token = tile_token(p, t) + kWaveTokens * w + 16 * (l & 1);
        const bool seen = t < end && token < p.len && (token < p.sinks || token + 15 >= p.first);
        int page = -1;
        if (seen) page = a.tables[(int64_t)s * a.ld_table + (token >> a.page_shift)];
        pages = (uint32_t)page < (uint32_t)a.n_pages ? page : -1;
        pages_at = i;
    }
    __device__ __forceinline__ rsrc_t page_rsrc(const uint16_t* base, int page, int kh) const {
        const int64_t at = max(page, 0) * a.page_stride + kh * a.head_stride;
        return make_rsrc(base + at, page < 0 ? 0u : page_bytes);
    }
    __device__ __forceinline__ void load_k(const Span& p, int kh, int i) {
        const int base = tile_token(p, i) + kWaveTokens * w;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * (i - pages_at) + u);
            has_page[u] = page >= 0;
            const rsrc_t r = page_rsrc(a.k, page, kh);
            const uint32_t row = (uint32_t)(((base + 16 * u) & ((1 << a.page_shift) - 1)) + (l & 15)) * row_bytes;
#pragma unroll
            for (int x = 0; x < NS; ++x) kf[u][x] = bload16(r, (int)(row + koff[x]));
        }
    }
    // Which tokens of a tile this lane sees: x stands for token x + 4 (l / 16) of the wave's 32.
    struct Seen {
        int sinks, first, end;
        __device__ __forceinline__ Seen(const Span& p, int base, int l)
            : sinks(p.sinks - base - 4 * (l >> 4)), first(p.first - base - 4 * (l >> 4)), end(p.len - base - 4 * (l >> 4)) {}
        __device__ __forceinline__ bool operator()(int x) const { return (x < sinks) | ((x >= first) & (x < end)); }
    };
    __device__ __forceinline__ void load_v(const Span& p, int kh, int i) {
        const int base = tile_token(p, i) + kWaveTokens * w;
        const Seen seen(p, base, l);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * (i - pages_at) + u);
            const rsrc_t r = page_rsrc(a.v, page, kh);
            // (an empty buffer with no scalar offset, so that every offset is out of its range)
            const int step = page < 0 ? 0 : (int)row_bytes;
            const uint32_t row = (uint32_t)(((base + 16 * u) & ((1 << a.page_shift) - 1)) + 4 * (l >> 4)) * row_bytes;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // values of tokens that are not seen are not read: their weight is
                // zero, but zero times an infinity or a NaN is not
                const uint32_t at = seen(16 * u + j) ? row : (uint32_t)kOut;
                const int so = j * step;
                if constexpr (NV == 4) {
                    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)(at + voff[0]), so, 0));
                    vf[4 * u + j][0] = x[0];
                    vf[4 * u + j][1] = x[1];
                } else {
#pragma unroll
                    for (int x = 0; x < NV / 8; ++x) {
                        const u32x4 y = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(at + voff[x]), so, 0));
#pragma unroll
                        for (int z = 0; z < 4; ++z) vf[4 * u + j][4 * x + z] = y[z];
                    }
                }
            }
        }
    }
    // Scores of the tile from kf, weights, and the statistics; returns the weights as the B operand of the product with V.
    __device__ __forceinline__ u32x4 weights(const Span& p, int i) {
        const int base = tile_token(p, i) + kWaveTokens * w;
        f32x4 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < NS; ++x) c = Fmt::mma32(kf[u][x], q[x], c);
            sc[u] = c;
        }
        const float c = a.scale * kLog2e;
        const Seen seen(p, base, l);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[u][j] = (seen(16 * u + j) & has_page[u]) ? sc[u][j] * c : -INFINITY;
        float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                          fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        top = max_over_quarters(top);
        const float mn = fmaxf(m, top);
        const float most = mn == -INFINITY ? 0.f : mn, ref = most - kLift<Fmt>;
        const float f = __builtin_amdgcn_exp2f(m - most);
        m = mn;
        u32x4 pw;
        float add = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t x = Fmt::pack2(__builtin_amdgcn_exp2f(sc[u][2 * h] - ref),
                                              __builtin_amdgcn_exp2f(sc[u][2 * h + 1] - ref));
                pw[2 * u + h] = x;
                add += Fmt::to_f32(lo16(x)) + Fmt::to_f32(hi16(x));
            }
        sum = sum * f + add;
#pragma unroll
        for (int t = 0; t < NV; ++t) o[t] *= f;
        return pw;
    }
    __device__ __forceinline__ void add_v(const u32x4& pw) {
#pragma unroll
        for (int t = 0; t < NV; ++t) {
            u32x4 x;
#pragma unroll
            for (int z = 0; z < 4; ++z)
                x[z] = (t & 1) ? pack_hi(vf[2 * z][t >> 1], vf[2 * z + 1][t >> 1])
                               : pack_lo(vf[2 * z][t >> 1], vf[2 * z + 1][t >> 1]);
            o[t] = Fmt::mma32(x, pw, o[t]);
        }
    }
    // Tiles [i0, i1) of sequence s, key-value head kh, group tile g.
    __device__ __forceinline__ void run(const Span& p, int s, int kh, int g, int i0, int i1) {
        const int head = g * kHeads + (l & 15);
        const uint16_t* qr = a.q + s * a.ldq + (int64_t)(kh * a.group) * a.head_dim;
        const rsrc_t r = make_rsrc(qr, (uint32_t)a.group * a.head_dim * 2u);
        load_pages(p, s, i0, i1);
        load_k(p, kh, i0);
        load_v(p, kh, i0);
#pragma unroll
        for (int x = 0; x < NS; ++x)
            q[x] = bload16(r, head < a.group ? (int)((uint32_t)head * a.head_dim * 2u + koff[x]) : kOut);
        m = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int t = 0; t < NV; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int i = i0; i < i1; ++i) {
            const u32x4 pw = weights(p, i);
            // kf and vf are refilled as soon as they have been used, and not before: a
            // second set of registers costs more waves than it brings (128 sequences
            // x 40 heads 249 against 185 us).  (tile i1 has no pages: its loads
            // return zeros and read nothing)
            if (i + 1 - pages_at == 32) load_pages(p, s, i + 1, i1);
            __builtin_amdgcn_sched_barrier(0);
            load_k(p, kh, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            add_v(pw);
            __builtin_amdgcn_sched_barrier(0);
            load_v(p, kh, i + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        sum = sum_over_quarters(sum);
    }
};

template <class Fmt, int DP>
__global__ void __launch_bounds__(256, decode_per_cu(DP)) lora_attn_decode_kernel(DecodeArgs d) {
    constexpr int NV = DP / 16;
    constexpr int LD = DP + 4;
    __shared__ float lo[4][kHeads][LD];
    __shared__ float lm[4][kHeads], ls[4][kHeads];
    __shared__ int last[2];
    const AttnArgs& a = d.a;
    const int t = threadIdx.x, l = t & 63, w = t >> 6;
    // the line of all tiles; each wave finds its own way: lane l has sequences per l on
    const int per = (a.n_seqs + 63) / 64;
    int s = l * per, len = 0, mine = 0;
    if (s < a.n_seqs) {
        len = kv_len(a.lens, s, a.max_len);
        mine = decode_span(a, len).n;
    }
    int longest = mine;
    for (int x = s + 1; x < min(s + per, a.n_seqs); ++x) {
        const int n = decode_span(a, kv_len(a.lens, x, a.max_len)).n;
        mine += n;
        longest = max(longest, n);
    }
    int seq_before = mine;                 // tiles of the sequences before
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int o = __shfl_up(seq_before, i, 64);
        if (l >= i) seq_before += o;
        longest = max(longest, __shfl_xor(longest, i, 64));
    }
    longest = __builtin_amdgcn_readfirstlane(longest);
    const int64_t total = (int64_t)__builtin_amdgcn_readlane(seq_before, 63) * d.heads_per_seq;
    // Tiles per workgroup: an even share, but up to 4 where that keeps a head's parts to
    // what one workgroup joins (8 x 33 tiles of 2 heads: 18.3 us with 3 tiles each, 22.2
    // with one).
    const int64_t R = max((total + gridDim.x - 1) / gridDim.x,
                          (int64_t)min(4, (longest + join_width(a.group) - 1) / join_width(a.group)));
    const int64_t start = blockIdx.x * R;
    if (start >= total) return;
    const int at = (int)(start / d.heads_per_seq);
    seq_before -= mine;
    const int lane = __builtin_ctzll(__ballot(at >= seq_before && at < seq_before + mine));
    seq_before = __builtin_amdgcn_readlane(seq_before, lane);
    s = __builtin_amdgcn_readlane(s, lane);
    Span p = decode_span(a, __builtin_amdgcn_readlane(len, lane));
    while (at >= seq_before + p.n) {       // one of the lane's others
        seq_before += p.n;
        p = decode_span(a, __builtin_amdgcn_readfirstlane(kv_len(a.lens, ++s, a.max_len)));
    }
    int hs, i0;
    {
        const int64_t in = start - (int64_t)seq_before * d.heads_per_seq;
        hs = (int)(in / p.n);
        i0 = (int)(in - (int64_t)hs * p.n);
    }
    int64_t left = min(R, total - start);
    DecodeWave<Fmt, DP> wave(a);
    while (true) {
        const int take = (int)min(left, (int64_t)(p.n - i0));
        const int kh = hs / d.group_tiles, g = hs - kh * d.group_tiles;
        wave.run(p, s, kh, g, i0, i0 + take);
        // the waves' results meet in LDS
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < NV; x += 4)
                *(f32x4*)&lo[w][l & 15][(4 * (l >> 4) + i) * NV + x] =
                    f32x4{wave.o[x][i], wave.o[x + 1][i], wave.o[x + 2][i], wave.o[x + 3][i]};
        if (l < 16) {
            lm[w][l] = wave.m;
            ls[w][l] = wave.sum;
        }
        __syncthreads();
        // thread t: elements NV (t % 16) .. of head t / 16
        const int h = t >> 4, e0 = (t & 15) * NV;
        const int head = g * kHeads + h;
        float M = fmaxf(fmaxf(lm[0][h], lm[1][h]), fmaxf(lm[2][h], lm[3][h]));
        float S = 0.f;
        f32x4 acc[NV / 4];
#pragma unroll
        for (int x = 0; x < NV / 4; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
        {
            const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = __builtin_amdgcn_exp2f(lm[i][h] - ref);
                S += ls[i][h] * f;
#pragma unroll
                for (int x = 0; x < NV / 4; ++x) acc[x] += *(const f32x4*)&lo[i][h][e0 + 4 * x] * f;
            }
        }
        bool store = true;
        if (take != p.n) {
            // a part of the head's tokens: to device memory, and on only with all parts there.
            // Many parts are joined 16 or more at a time first, by as many workgroups: a single
            // one took a microsecond for every few of them.
            const int64_t first = (int64_t)seq_before * d.heads_per_seq + (int64_t)hs * p.n;
            const int w0 = (int)(first / R), w1 = (int)((first + p.n - 1) / R);   // the head's workgroups
            constexpr int SF = slot_floats(DP);
            const rsrc_t all = make_rsrc(d.slots, gridDim.x * 2u * SF * 4u);
            // this thread's place in the partial result of workgroup w: its first part if w is w0, its last
            auto place = [&](int x, int hh) { return ((2 * x + (x == w0)) * SF + hh * DP + e0) * 4; };
            auto place_ms = [&](int x, int hh) { return ((2 * x + (x == w0)) * SF + kHeads * DP + 2 * hh) * 4; };
            auto put = [&](int x) {
                if (head < a.group) {
#pragma unroll
                    for (int y = 0; y < NV / 4; ++y) bstore16<kCoherent>(as_u4(acc[y]), all, place(x, h) + 16 * y);
                    if ((t & 15) == 0)
                        bstore8<kCoherent>(u32x2{__float_as_uint(M), __float_as_uint(S)}, all, place_ms(x, h));
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
                __builtin_amdgcn_s_waitcnt(0);           // every thread's stores have reached the device
                __syncthreads();
            };
            // Is this the last of n workgroups to come here?
            auto arrive = [&](int kind, int x, int n) {
                if (t == 0) {
                    uint32_t* c = d.counters + (kind * (int)gridDim.x + x) * kSyncStride;
                    const bool r = __hip_atomic_fetch_add(c, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(n - 1);
                    if (r) __hip_atomic_store(c, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    last[kind >> 1] = r;
                }
                __syncthreads();
                return last[kind >> 1] != 0;
            };
            // The partial results of workgroups x0, x0 + step, .. up to x1 into M, S and acc
            // of the threads that hold them.  Threads of heads that the tile does not have take
            // parts as well: group k of the ng takes parts k, k + ng, .., four at a
            // time in flight, and the groups' sums meet in LDS.
            const int gp = head_slots(min(kHeads, a.group - g * kHeads));
            const int ng = kHeads / gp, k = h / gp, hk = h - k * gp;
            auto join = [&](int x0, int x1, int step) {
                M = -INFINITY;
                S = 0.f;
#pragma unroll
                for (int x = 0; x < NV / 4; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
                auto add = [&](float m1, float s1, const f32x4 (&y)[NV / 4]) {
                    const float mn = fmaxf(M, m1), ref = mn == -INFINITY ? 0.f : mn;
                    const float f0 = __builtin_amdgcn_exp2f(M - ref), f1 = __builtin_amdgcn_exp2f(m1 - ref);
                    M = mn;
                    S = S * f0 + s1 * f1;
#pragma unroll
                    for (int x = 0; x < NV / 4; ++x) acc[x] = acc[x] * f0 + y[x] * f1;
                };
                for (int v = x0 + k * step; v <= x1; v += 4 * ng * step) {
                    u32x2 ms[4];
                    f32x4 y[4][NV / 4];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int u = v + b * ng * step;
                        ms[b] = bload8<kCoherent>(all, u <= x1 ? place_ms(u, hk) : kOut);
#pragma unroll
                        for (int x = 0; x < NV / 4; ++x)
                            y[b][x] = as_f4(bload16<kCoherent>(all, u <= x1 ? place(u, hk) + 16 * x : kOut));
                    }
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        add(v + b * ng * step <= x1 ? __uint_as_float(ms[b][0]) : -INFINITY, __uint_as_float(ms[b][1]), y[b]);
                }
                if (ng > 1) {
#pragma unroll
                    for (int x = 0; x < NV / 4; ++x) *(f32x4*)&lo[0][h][e0 + 4 * x] = acc[x];
                    if ((t & 15) == 0) {
                        lm[0][h] = M;
                        ls[0][h] = S;
                    }
                    __syncthreads();
                    const int used = min(ng, (x1 - x0) / step + 1);
                    for (int o = 1; o < used && k == 0; ++o) {
                        f32x4 y[NV / 4];
#pragma unroll
                        for (int x = 0; x < NV / 4; ++x) y[x] = *(const f32x4*)&lo[0][o * gp + hk][e0 + 4 * x];
                        add(lm[0][o * gp + hk], ls[0][o * gp + hk], y);
                    }
                }
            };
            const int kJoin = join_width(a.group - g * kHeads);
            const int n = w1 - w0 + 1;
            const int x0 = w0 + ((int)blockIdx.x - w0) / kJoin * kJoin, x1 = min(x0 + kJoin - 1, w1);
            put(blockIdx.x);
            store = arrive(x0 != w0, x0, x1 - x0 + 1);
            if (store) {
                join(x0, x1, 1);
                if (n > kJoin) {
                    put(x0);                             // (a barrier: what join() left in LDS has been read)
                    store = arrive(2, w0, (n + kJoin - 1) / kJoin);
                    if (store) join(w0, w1, kJoin);
                }
            }
        }
        if (store && head < a.group) {
            const float f = S != 0.f ? 1.f / S : 0.f;
            uint16_t* dst = a.out + s * a.ldo + (int64_t)(kh * a.group + head) * a.head_dim + e0;
#pragma unroll
            for (int x = 0; x < NV / 4; x += NV == 4 ? 1 : 2) {
                if (e0 + 4 * x >= a.head_dim) continue;
                const f32x4 y = acc[x] * f;
                if constexpr (NV == 4) {
                    *(u32x2*)dst = u32x2{Fmt::pack2(y[0], y[1]), Fmt::pack2(y[2], y[3])};
                } else {
                    const f32x4 z = acc[x + 1] * f;
                    *(u32x4*)(dst + 4 * x) = u32x4{Fmt::pack2(y[0], y[1]), Fmt::pack2(y[2], y[3]),
                                                   Fmt::pack2(z[0], z[1]), Fmt::pack2(z[2], z[3])};
                }
            }
        }
        left -= take;
        if (left == 0) return;
        // the next head, or the next sequence's first
        i0 = 0;
        if (++hs == d.heads_per_seq) {
            seq_before += p.n;
            hs = 0;
            p = decode_span(a, __builtin_amdgcn_readfirstlane(kv_len(a.lens, ++s, a.max_len)));
        }
        __syncthreads();                   // lo, lm, ls have been read
    }
}

template <int DP>
void launch_decode(const DecodeArgs& d, int dtype, int blocks, hipStream_t st) {
    if (dtype == LORA_F16)
        hipLaunchKernelGGL((lora_attn_decode_kernel<FmtF16, DP>), dim3(blocks), dim3(256), 0, st, d);
    else
        hipLaunchKernelGGL((lora_attn_decode_kernel<FmtBF16, DP>), dim3(blocks), dim3(256), 0, st, d);
}

__global__ void __launch_bounds__(256) lora_attn_clear_kernel(uint32_t* p, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0u;
}

// ---------------------------------------------------------------------------
// prompt
// ---------------------------------------------------------------------------

typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kCols = 128;                 // columns (row, head) of a workgroup: 32 per wave
constexpr int kKeys = 64;                  // tokens per step
constexpr float kSlack = 8.f;              // how far (in powers of two) a maximum may rise before the sums are rescaled
// A score of this many powers of two and more: s c - m in one rounding is then off from s c rounded, which
// m is, by half an ulp of m, an eighth of a power of two here, and from 2^31 on by more than weights hold.
constexpr float kWild = 0x1p21f;

struct PromptArgs {
    AttnArgs a;
    uint32_t* counters;
    float* slots;
    int32_t kv_heads;
    int32_t parts;                         // workgroups that share a tile's tokens
};

// Workgroups per compute unit: what the registers allow.
constexpr int prompt_per_cu(int dp) { return dp == 256 ? 1 : dp == 128 ? 2 : 3; }
// Floats of a partial result: the outputs, then maximum and sum of every column.
constexpr int part_floats(int dp) { return kCols * dp + 2 * kCols; }

template <class Fmt>
__device__ __forceinline__ f32x16 mma32x32(const u32x4& a, const u32x4& b, f32x16 c);
template <>
__device__ __forceinline__ f32x16 mma32x32<FmtF16>(const u32x4& a, const u32x4& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16 mma32x32<FmtBF16>(const u32x4& a, const u32x4& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// s + the two 16-bit values of x.
template <class Fmt>
__device__ __forceinline__ float add_pair(uint32_t x, float s);
template <>
__device__ __forceinline__ float add_pair<FmtF16>(uint32_t x, float s) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2v, x), __builtin_bit_cast(f16x2v, 0x3c003c00u), s, false);
}
template <>
__device__ __forceinline__ float add_pair<FmtBF16>(uint32_t x, float s) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v, x), __builtin_bit_cast(bf16x2v, 0x3f803f80u), s, false);
}

// 16 bytes per lane from buffer r at byte offset off + so (zeros when out of
// range) into LDS at lds + 16 * lane; lds, so and r are the same in every lane.
// Inline assembly without an output: for the builtin the compiler waits for
// every such load in flight before each LDS read.  A wait and a barrier order the
// reads after it.  The wait states are those of a scalar register that a vector
// instruction wrote (v_readfirstlane, or v_readlane where the compiler had put it
// aside); they cover the write of m0.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is reserved: nothing to preserve, the clobber is what is said
__device__ __forceinline__ void lds_load16(const u32x4& r, uint32_t lds, uint32_t off, uint32_t so) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(lds), "v"(off), "s"(r), "s"(so) : "memory", "m0");
}
#pragma clang diagnostic pop
// The resource of make_rsrc() as four scalar words.
__device__ __forceinline__ u32x4 uniform_rsrc(const void* base, uint32_t bytes) {
    const uint64_t b = (uint64_t)base;
    return {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b),
            (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) & 0xffffu,
            (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), (uint32_t)kRsrcWord3};
}

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
// Transposing read: lane j of each 16 lanes gets element j % 4 of the 8-byte
// values that lanes j / 4, 4 + j / 4, 8 + j / 4 and 12 + j / 4 address.
__device__ __forceinline__ u32x2 lds_read_tr16(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at));
}

// s_waitcnt lgkmcnt(0), vmcnt and expcnt left free.
__device__ __forceinline__ void wait_lgkm0() { __builtin_amdgcn_s_waitcnt(0xC07F); }
// s_waitcnt vmcnt(N), the other counters left free.
template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// The larger of v in lane l and lane l ^ 32, in both; their sum.
__device__ __forceinline__ float max_over_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_over_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A workgroup's tile: 128 columns of one segment and key-value head, and the
// tokens that some row of it sees, [0, sinks) and [first, last], in steps of 64.
struct PromptTile {
    int seq, row0, n;                      // segment, its first row, its rows
    int col0;                              // the tile's first column: row col0 / group, head col0 % group
    int pos0;                              // position of the segment's first row
    int lowest, last;                      // positions of the tile's first and last row
    int first, sinks, sink_steps, win_step, steps;
};

// KS 1: the four waves have 32 columns each and share the tokens of a step.
// KS 4 (launches of few columns): all have the same 32 columns, and each its own 64
// tokens of a step of 256, which no other wave touches.
template <class Fmt, int DP, int KS>
struct PromptBlock {
    static constexpr int CH = DP / 8;      // 16-byte chunks of a token
    static constexpr int NS = DP / 16;     // MFMA steps of a score
    static constexpr int ND = DP / 32;     // 32-row blocks of the output
    static constexpr int KD = 2;           // MFMA steps of a score read ahead from LDS
    static constexpr int VD = 4;           // products with V read ahead from LDS
    static constexpr int NL = CH / 4;      // loads of K (and of V) per wave and step
    static constexpr int NVO = CH == 32 ? 2 : 1;     // see vo
    static constexpr int kStage = kKeys * CH * 16;   // bytes of K (or V) of 64 tokens
    static constexpr int kV = KS == 1 ? 2 * kStage : kStage;       // V in LDS: behind two buffers of K, or one
    static constexpr int kLds = 4 * kStage * (KS == 1 ? 1 : 2);
    static constexpr bool kAcc = DP == 256 || KS == 4;   // o in accumulation registers
    static constexpr int kGroups = 4 * KS;           // 16-token groups of a step
    const AttnArgs& a;
    const PromptTile& p;
    unsigned char* lds;
    const int kh, l, w;
    const int pos;                         // of this lane's column, -1 for none
    u32x4 q[NS];
    f32x16 o[ND];
    float m, sum;
    // byte offsets of this lane's chunks in its 16 tokens, kOut past the head; of V only
    // those that differ by more than whole tokens
    uint32_t ko[NL], vo[NVO];
    uint32_t row_bytes, lbase;
    uint32_t ka, va[ND];                   // see set_reads()
    int pages, next_pages;                 // lane kGroups t + g: page of tokens 16 g on of step t, -1 for none seen
    uint64_t has_pages;                    // which of pages there are
    int pages_at, pages_end;               // the first step of pages; the end of this run's
    int k_page;                            // this wave's page of the step whose K was loaded last
    uint32_t has_load;                     // which pages there are of the four of the step whose K came last
    float c, top;                          // scale in powers of two; the step's largest score

    __device__ __forceinline__ PromptBlock(const AttnArgs& args, const PromptTile& tile, unsigned char* smem, int kv_head,
                                           int position)
        : a(args), p(tile), lds(smem), kh(kv_head), l(threadIdx.x & 63),
          w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), pos(position) {
        if (KS > 1) lds += w * 2 * kStage;
        lbase = (uint32_t)(uintptr_t)(lds_u8*)lds;
        row_bytes = (uint32_t)a.row_stride * 2u;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int at = i * 64 + l, r = at / CH;
            const int kc = (at % CH) ^ k_key(r), vc = (at % CH) ^ v_key(r);
            ko[i] = 8 * kc < a.head_dim ? r * row_bytes + 16u * kc : (uint32_t)kOut;
            if (i < NVO) vo[i] = 8 * vc < a.head_dim ? r * row_bytes + 16u * vc : (uint32_t)kOut;
        }
    }
    // Chunk c of token r stands in slot c ^ key(r) of its row.  K: the 16 rows
    // that a quarter wave reads one chunk of lie in 16 bank groups.  V: the four
    // rows that a transposing read takes 64 bytes of lie in four.
    static __device__ __forceinline__ int k_key(int r) { return CH >= 16 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int v_key(int r) { return CH >= 16 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }

    // The first token of step i; of this wave's 64 of it.
    __device__ __forceinline__ int first_token(int i) const {
        return (i < p.sink_steps ? i : p.win_step + i - p.sink_steps) * (kKeys * KS);
    }
    __device__ __forceinline__ int step_token(int i) const { return first_token(i) + (KS == 1 ? 0 : kKeys * w); }
    __device__ __forceinline__ void fetch_pages(int i) {
        const int t = i + l / kGroups, token = first_token(t) + 16 * (l % kGroups);
        const bool seen = t < pages_end && token <= p.last && (token < p.sinks || token + 15 >= p.first);
        next_pages = -1;
        if (seen) next_pages = a.tables[(int64_t)p.seq * a.ld_table + (token >> a.page_shift)];
    }
    __device__ __forceinline__ void turn_pages(int i) {
        pages = (uint32_t)next_pages < (uint32_t)a.n_pages ? next_pages : -1;
        has_pages = __ballot(pages >= 0);
        pages_at = i;
        fetch_pages(i + 64 / kGroups);
    }
    // 16 tokens of K or V, `token` on, on their way from their page to `to` in LDS.
    // Tokens past the last one that the tile sees are past the end of the resource:
    // zeros.  (Those it does not see before a window are read, and kept out as hidden
    // values.)
    struct Source {
        u32x4 r;
        uint32_t so, step, most, to;
    };
    __device__ __forceinline__ Source source(const uint16_t* base, int token, int page, uint32_t to) const {
        const int row = token & ((1 << a.page_shift) - 1);
        const int rows = min((1 << a.page_shift) - 1, p.last - token + row);      // the last row of the page to read
        Source s;
        s.r = uniform_rsrc(base + max(page, 0) * a.page_stride + kh * a.head_stride,
                           page < 0 ? 0u : (uint32_t)rows * row_bytes + (uint32_t)a.head_dim * 2u);
        // (an empty buffer with no scalar offset, so that every offset is out of its range)
        s.step = page < 0 ? 0u : row_bytes;
        s.so = (uint32_t)row * s.step;
        s.most = (uint32_t)rows * s.step;
        s.to = lbase + to;
        return s;
    }
    // Load j of NL of a source.  (The range of a buffer is counted from its scalar offset on,
    // which therefore stays below its end: where all tokens of a load of V are past the
    // last one, the last stands in for the first of them, with weight zero as well.)
    template <bool kOfV>
    __device__ __forceinline__ void issue(const Source& s, int j) const {
        lds_load16(s.r, s.to + j * 1024u, kOfV ? vo[j % NVO] : ko[j],
                   kOfV ? min(s.so + (j - j % NVO) * (64 / CH) * s.step, s.most) : s.so);
    }
    template <bool kOfV>
    __device__ __forceinline__ void issue_all(const Source& s) const {
#pragma unroll
        for (int j = 0; j < NL; ++j) issue<kOfV>(s, j);
    }
    // KS 1.  K of step i into buffer b (steps in order), wave w its tokens 16 w .. + 15;
    // V of the step whose K came last.
    __device__ __forceinline__ Source next_k(int i, int b) {
        if (i - pages_at == 16) turn_pages(i);
        k_page = __builtin_amdgcn_readlane(pages, 4 * (i - pages_at) + w);
        has_load = (uint32_t)(has_pages >> (4 * (i - pages_at))) & 15u;
        return source(a.k, step_token(i) + 16 * w, k_page, (uint32_t)(b * kStage + w * 16 * CH * 16));
    }
    __device__ __forceinline__ Source next_v(int i, int b) const {
        return source(a.v, step_token(i) + 16 * w, k_page, (uint32_t)(kV + b * kStage + w * 16 * CH * 16));
    }
    // KS 4.  This wave's 64 tokens of step i (steps in order, K before V).
    template <bool kOfV>
    __device__ __forceinline__ void issue_own(int i) {
        if (!kOfV && i - pages_at == 64 / kGroups) turn_pages(i);
        const int lane = kGroups * (i - pages_at) + 4 * w;
        if (!kOfV) has_load = (uint32_t)(has_pages >> lane) & 15u;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            issue_all<kOfV>(source(kOfV ? a.v : a.k, step_token(i) + 16 * g, __builtin_amdgcn_readlane(pages, lane + g),
                                   (uint32_t)((kOfV ? kV : 0) + g * 16 * CH * 16)));
    }

    // LDS addresses of this lane's reads in the first buffers: K chunk l / 32 of token
    // l % 32 (chunk 2 x + l / 32 is 2 x in the chunk's bits away); 4 elements of V's block d of token 4 (l / 32) + (l % 16) / 4, which
    // the 16 lanes exchange.  Other tokens of the step are constants away.
    __device__ __forceinline__ void set_reads() {
        const int h = l >> 5, row = l & 31;
        ka = lbase + (row * CH + (h ^ k_key(row))) * 16;
        const int r = 4 * h + ((l & 15) >> 2), e = (l & 16) + 4 * (l & 3);
#pragma unroll
        for (int d = 0; d < ND; ++d) va[d] = lbase + kV + (r * CH + ((4 * d + (e >> 3)) ^ v_key(r))) * 16 + 2 * (e & 7);
    }
    __device__ __forceinline__ void read_k(u32x4 (&f)[2], int x, int b) const {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) f[kt] = *(const lds_u32x4*)(uintptr_t)((ka ^ (32u * x)) + b * kStage + kt * 32 * CH * 16);
    }
    // V of product f: 16 tokens f / ND, output block f % ND.
    __device__ __forceinline__ u32x4 read_v(int f, int b) const {
        const uint32_t at = va[f % ND] + b * kStage + 16 * (f / ND) * CH * 16;
        const u32x2 x = lds_read_tr16(at), y = lds_read_tr16(at + 8 * CH * 16);
        return u32x4{x[0], x[1], y[0], y[1]};
    }
    __device__ __forceinline__ bool visible(int token) const {
        return (token <= pos) & ((a.window == 0) | (token > pos - a.window) | (token < a.n_sinks));
    }

    // The two 16-bit values of x, infinities and NaN replaced by zero.
    static constexpr uint32_t kExponent = Fmt::kNarrowRange ? 0x7c00u : 0x7f80u;
    static __device__ __forceinline__ uint32_t finite_pair(uint32_t x) {
        const uint32_t lo = (x & kExponent) == kExponent ? 0u : lo16(x);
        return (x >> 16 & kExponent) == kExponent ? lo : lo | (x & 0xffff0000u);
    }

    // Do all columns see all tokens of step i?
    __device__ __forceinline__ bool all_see(int i, uint32_t has) const {
        const int base = step_token(i);
        return (base + kKeys - 1 <= p.lowest) & (has == 15u) &
               ((a.window == 0) | (base > p.last - a.window) | (base + kKeys <= a.n_sinks));
    }
    __device__ __forceinline__ void hide(f32x16 (&s)[2], int i, uint32_t has) const {
        const int base = step_token(i) + 4 * (l >> 5);
        const int first = a.window ? pos - a.window + 1 : 0;              // seen: first .. pos, and the sinks
        const uint32_t span = (uint32_t)(pos - max(first, 0)), from = (uint32_t)(base - max(first, 0));
        const bool simple = (has == 15u) & (step_token(i) >= a.n_sinks) & (pos >= 0);
        if (__all(simple)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[kt][r] = from + (uint32_t)(32 * kt + 8 * (r >> 2) + (r & 3)) <= span ? s[kt][r] : -INFINITY;
        } else {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int x = 32 * kt + 8 * (r >> 2) + (r & 3);
                    s[kt][r] = (visible(base + x) & ((has >> (x >> 4)) & 1u)) ? s[kt][r] : -INFINITY;
                }
        }
    }
    // Scores of the step whose K is in buffer b; filler(x) after the products of dimensions 16 x on.
    template <class F>
    __device__ __forceinline__ void score(f32x16 (&s)[2], int b, F filler) {
        u32x4 kf[KD][2];
#pragma unroll
        for (int x = 0; x < KD; ++x) read_k(kf[x], x, b);
        __builtin_amdgcn_sched_barrier(0);
        filler(-1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < NS; ++x) {
            const f32x16 zero = {};
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) s[kt] = mma32x32<Fmt>(kf[x % KD][kt], q[x], x ? s[kt] : zero);
            if (x + KD < NS) read_k(kf[x % KD], x + KD, b);
            filler(x);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __device__ __forceinline__ void rescale() {
        // (a column's maximum does not depend on the others': no value that it does not see reaches it)
        const bool rise = top > m + kSlack;
        if (__any(rise)) {
            const float f = rise ? __builtin_amdgcn_exp2f(m - top) : 1.f;
            m = rise ? top : m;
            sum *= f;
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                // (where o is in accumulation registers: without this the compiler moves all of it out
                // of them in every step, for a product that few steps need)
                if (kAcc) asm volatile("" : "+a"(o[d]));
                o[d] *= f;
                if (kAcc) asm volatile("" : "+a"(o[d]));
            }
        }
    }
    // A score relative to ref, in powers of two.  kAnySize: also where they are very large (kWild); the product is
    // then rounded as that of the maximum was.
    template <bool kAnySize>
    __device__ __forceinline__ float relative(float s, float ref) const {
        const float x = __builtin_fmaf(s, c, -ref);
        if (!kAnySize) return x;
        float y = s * c;
        asm volatile("" : "+v"(y));                      // not one rounding after all
        return fabsf(ref) >= kWild ? y - m + kLift<Fmt> : x;     // (ref itself would be rounded)
    }
    // Weights of pair z of this lane's 32 tokens: pw[t] is the B operand of tokens 16 t on.
    template <bool kAnySize = false>
    __device__ __forceinline__ void weigh_pair(const f32x16 (&s)[2], u32x4 (&pw)[4], int z, float ref) {
        const int kt = z >> 3, r = 2 * (z & 7);
        uint32_t x = Fmt::pack2(__builtin_amdgcn_exp2f(relative<kAnySize>(s[kt][r], ref)),
                                __builtin_amdgcn_exp2f(relative<kAnySize>(s[kt][r + 1], ref)));
        asm volatile("" : "+v"(x));                      // here, and not where the compiler would rather have it
        pw[z >> 2][z & 3] = x;
        sum = add_pair<Fmt>(x, sum);
    }

    // Step i, its K and V in buffers B; the next step's go into the other ones.
    template <int B>
    __device__ __forceinline__ void step(int i) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070);              // this wave's loads have landed, its reads are done;
        __builtin_amdgcn_s_barrier();                    // every wave's
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t has = has_load;
        const Source sk = next_k(i + 1, B ^ 1), sv = next_v(i + 1, B ^ 1);   // (past the end: zeros)
        f32x16 s[2];
        // the next step's loads behind the products, one at a time: each takes 16 cycles
        // of the path into LDS, and all at once they held every wave up for 800 of
        // a step's 3600 cycles
        score(s, B, [&](int x) {
#pragma unroll
            for (int j = 2 * NL * x / NS; x >= 0 && j < 2 * NL * (x + 1) / NS; ++j) {
                if (j < NL) issue<false>(sk, j);
                else issue<true>(sv, j - NL);
            }
        });
        u32x4 vf[VD];
        first_v(vf, B);
        __builtin_amdgcn_sched_barrier(0);
        u32x4 pw[4];
        const float ref = settle(s, i, has, pw);
        products(s, pw, vf, ref, B);
    }
    __device__ __forceinline__ void first_v(u32x4 (&vf)[VD], int b) const {
#pragma unroll
        for (int f = 0; f < VD; ++f) vf[f] = read_v(f, b);
    }
    // Step i's scores, those not seen hidden, against the maximum so far; the first
    // weights.  Returns what the scores are taken relative to.
    __device__ __forceinline__ float settle(f32x16 (&s)[2], int i, uint32_t has, u32x4 (&pw)[4]) {
        if (!all_see(i, has)) hide(s, i, has);
        top = highest(s);
        rescale();
        const float ref = m == -INFINITY ? 0.f : m - kLift<Fmt>;
#pragma unroll
        for (int z = 0; z < 4; ++z) weigh_pair(s, pw, z, ref);
        __builtin_amdgcn_sched_barrier(0);
        return ref;
    }
    // The products with V, the weights of 16 tokens behind the products of the 16 before.
    __device__ __forceinline__ void products(const f32x16 (&s)[2], u32x4 (&pw)[4], u32x4 (&vf)[VD], float ref, int b) {
#pragma unroll
        for (int f = 0; f < 4 * ND; ++f) {
            o[f % ND] = mma32x32<Fmt>(vf[f % VD], pw[f / ND], o[f % ND]);
            if (f + VD < 4 * ND) vf[f % VD] = read_v(f + VD, b);
            if (f < 3 * ND) {
#pragma unroll
                for (int z = 4 + 4 * f / ND; z < 4 + 4 * (f + 1) / ND; ++z) weigh_pair(s, pw, z, ref);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    __device__ __forceinline__ void start(int i0, int i1) {
        c = a.scale * kLog2e;
        m = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
        set_reads();
        pages_end = i1;
        fetch_pages(i0);
        turn_pages(i0);
    }
    __device__ __forceinline__ float highest(const f32x16 (&s)[2]) const {
        float high = s[0][0];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) high = fmaxf(high, s[kt][r]);
        return max_over_halves(high) * c;
    }
    __device__ __forceinline__ void finish() {
        sum = sum_over_halves(sum);
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_s_barrier();                    // the buffers have been read
    }

    // Steps [i0, i1) into o, m and sum.
    __device__ __forceinline__ void run(int i0, int i1) {
        start(i0, i1);
        if (i0 < i1) {
            issue_all<false>(next_k(i0, 0));
            issue_all<true>(next_v(i0, 0));
            for (int i = i0;;) {
                step<0>(i);
                if (++i == i1) break;
                step<1>(i);
                if (++i == i1) break;
            }
        }
        finish();
    }

    // Steps [i0, i1) of a block of few columns: this wave's tokens of them, by itself.
    __device__ __forceinline__ void run_own(int i0, int i1) {
        start(i0, i1);
        if (i0 < i1) {
            issue_own<false>(i0);
            issue_own<true>(i0);
        }
        for (int i = i0; i < i1; ++i) {
            const uint32_t has = has_load;
            __builtin_amdgcn_sched_barrier(0);
            wait_vm<4 * NL>();                           // K has landed, V may be on its way
            __builtin_amdgcn_sched_barrier(0);
            f32x16 s[2];
            score(s, 0, [](int) {});
            wait_lgkm0();
            if (i + 1 < i1) issue_own<false>(i + 1);     // (K has been read)
            __builtin_amdgcn_sched_barrier(0);
            u32x4 pw[4];
            const float ref = settle(s, i, has, pw);
            if (i + 1 < i1) wait_vm<4 * NL>();           // V has landed
            else wait_vm<0>();
            __builtin_amdgcn_sched_barrier(0);
            u32x4 vf[VD];
            first_v(vf, 0);
            products(s, pw, vf, ref, 0);
            wait_lgkm0();
            if (i + 1 < i1) issue_own<true>(i + 1);
        }
        sum = sum_over_halves(sum);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0);
    }

    // The same as run() and run_own() with infinities and NaN among the values, or with scores of any
    // size (kWild).  A token that a column
    // does not see has weight zero, which is as good as leaving it out unless its
    // value is one of those.  Here such values, in steps that only some columns see,
    // are kept out of the product and added to the columns that see them; the
    // other columns' sums are made in the same order, to the same bits.  One step at a time.
    __device__ __forceinline__ void run_careful(int i0, int i1) {
        start(i0, i1);
        const int h = l >> 5;
        for (int i = i0; i < i1; ++i) {
            if constexpr (KS == 1) {
                issue_all<false>(next_k(i, 0));
                issue_all<true>(next_v(i, 0));
            } else {
                issue_own<false>(i);
                issue_own<true>(i);
            }
            wait_vm<0>();
            if (KS == 1) __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            f32x16 s[2];
            score(s, 0, [](int) {});
            const bool edge = !all_see(i, has_load);
            if (edge) hide(s, i, has_load);
            top = highest(s);
            rescale();
            const float ref = m == -INFINITY ? 0.f : m - kLift<Fmt>;
            u32x4 pw[4];
#pragma unroll
            for (int z = 0; z < 16; ++z) weigh_pair<true>(s, pw, z, ref);
#pragma unroll
            for (int f = 0; f < 4 * ND; ++f) {
                u32x4 x = read_v(f, 0);
                if (edge) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) x[z] = finite_pair(x[z]);
                }
                o[f % ND] = mma32x32<Fmt>(x, pw[f / ND], o[f % ND]);
            }
            if (edge) {
                const int base = step_token(i);
                const unsigned char* vb = lds + kV;
                for (int j = 0; j < kKeys; ++j) {
                    // token j's weight: word 2 (j / 8) + (j % 4) / 2 of the lanes of half (j / 4) % 2
                    const int word = 2 * (j >> 3) + ((j & 3) >> 1);
                    uint32_t x = pw[0][0];
#pragma unroll
                    for (int e = 1; e < 16; ++e) x = word == e ? pw[e >> 2][e & 3] : x;
                    x = (uint32_t)__shfl((int)x, (l & 31) + 8 * (j & 4), 64);
                    const float pj = Fmt::to_f32(j & 1 ? hi16(x) : lo16(x));
                    const bool in = visible(base + j) & ((has_load >> (j >> 4)) & 1u);
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const u32x2 y = *(const u32x2*)(vb + (j * CH + ((4 * d + e) ^ v_key(j))) * 16 + 8 * h);
#pragma unroll
                            for (int z = 0; z < 4; ++z) {
                                const uint32_t v = z & 1 ? hi16(y[z >> 1]) : lo16(y[z >> 1]);
                                const bool add = in & ((v & kExponent) == kExponent);
                                o[d][4 * e + z] = add ? __builtin_fmaf(pj, Fmt::to_f32(v), o[d][4 * e + z]) : o[d][4 * e + z];
                            }
                        }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0070);          // the buffer has been read
            if (KS == 1) __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
        sum = sum_over_halves(sum);
        __builtin_amdgcn_s_waitcnt(0);
        if (KS == 1) __builtin_amdgcn_s_barrier();
    }
    // Is an output not finite?  It may come from a token that the column does not see.  Or was the column's
    // largest score too large for the fast weights?  (One that was on the way to a maximum nearer to zero
    // has left nothing, or infinities.)
    __device__ __forceinline__ bool doubtful() const {
        float x = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) x += o[d][r] * 0.f;
        return !(x == 0.f) || (fabsf(m) >= kWild && m != -INFINITY);
    }
    // The queries of this lane's column at q, if there is one.
    __device__ __forceinline__ void load_q(const uint16_t* at, bool real) {
#pragma unroll
        for (int x = 0; x < NS; ++x) {
            const int d = 16 * x + 8 * (l >> 5);
            q[x] = u32x4{0u, 0u, 0u, 0u};
            if (real && d < a.head_dim) q[x] = *(const u32x4*)(at + d);
        }
    }
};

// Row tile `index` of the launch, of `cols` columns and with steps of `keys` tokens:
// the tiles of all segments lie in one line, the last, which see the most, first.
// Each wave finds its own way: lane l has segments per l on.  False past the last tile.
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int cols, int keys, int index, PromptTile& p) {
    const int l = threadIdx.x & 63;
    const int per = (a.n_seqs + 63) / 64;
    auto rows_of = [&](int s, int& row0) {
        const int lo = a.seg_offset[s], hi = a.seg_offset[s + 1];
        row0 = min(max(lo, 0), a.n_rows);
        return max(min(max(hi, 0), a.n_rows) - row0, 0);       // (both in [0, n_rows]: no difference wraps)
    };
    auto tiles_of = [&](int n) { return (int)(((int64_t)n * a.group + cols - 1) / cols); };
    int seq = l * per, row0 = 0, n = 0, len = 0, mine = 0;     // the lane's first segment
    if (seq < a.n_seqs) {
        n = rows_of(seq, row0);
        len = kv_len(a.lens, seq, a.max_len);
        mine = tiles_of(n);
    }
    for (int s = seq + 1; s < min(seq + per, a.n_seqs); ++s) {
        int r;
        mine += tiles_of(rows_of(s, r));
    }
    int before = mine;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int o = __shfl_up(before, i, 64);
        if (l >= i) before += o;
    }
    const int tile = __builtin_amdgcn_readlane(before, 63) - 1 - index;
    if (tile < 0) return false;
    before -= mine;
    const int lane = __builtin_ctzll(__ballot(tile >= before && tile < before + mine));
    before = __builtin_amdgcn_readlane(before, lane);
    p.seq = __builtin_amdgcn_readlane(seq, lane);
    p.row0 = __builtin_amdgcn_readlane(row0, lane);
    p.n = __builtin_amdgcn_readlane(n, lane);
    len = __builtin_amdgcn_readlane(len, lane);
    if (per > 1 && tile >= before + tiles_of(p.n)) {           // one of the lane's others
        do {
            before += tiles_of(p.n);
            p.n = rows_of(++p.seq, p.row0);
        } while (tile >= before + tiles_of(p.n));
        len = kv_len(a.lens, p.seq, a.max_len);
        p.n = __builtin_amdgcn_readfirstlane(p.n);
        p.row0 = __builtin_amdgcn_readfirstlane(p.row0);
        len = __builtin_amdgcn_readfirstlane(len);
    }
    p.col0 = (tile - before) * cols;
    p.pos0 = len - p.n;
    p.lowest = p.pos0 + p.col0 / a.group;
    p.last = p.pos0 + min((p.col0 + cols - 1) / a.group, p.n - 1);
    p.first = a.window && p.lowest > 0 ? max(0, p.lowest - a.window + 1) : 0;
    p.sinks = min(a.n_sinks, p.first);
    p.sink_steps = (p.sinks + keys - 1) / keys;
    p.win_step = max(p.first / keys, p.sink_steps);
    p.steps = p.last < 0 ? 0 : max(0, p.sink_steps + p.last / keys + 1 - p.win_step);
    return true;
}

template <class Fmt, int DP>
__global__ void __launch_bounds__(256, prompt_per_cu(DP)) lora_attn_prompt_kernel(PromptArgs pa) {
    using Block = PromptBlock<Fmt, DP, 1>;
    constexpr int ND = DP / 32;
    __shared__ __align__(1024) unsigned char smem[Block::kLds];   // (rows of 512 bytes whose chunks are told apart by XOR)
    __shared__ int last_part, bad;
    const AttnArgs& a = pa.a;
    const int t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int kh = blockIdx.x % pa.kv_heads;
    const int rest = blockIdx.x / pa.kv_heads;
    const int part = rest % pa.parts;
    if (t == 0) bad = 0;                   // (run() has barriers)
    PromptTile p;
    if (!find_tile(a, kCols, kKeys, rest / pa.parts, p)) return;
    const int col = p.col0 + 32 * w + (l & 31);
    const int row = col / a.group, head = kh * a.group + col - row * a.group;
    const bool real = row < p.n;
    Block blk(a, p, smem, kh, real ? p.pos0 + row : -1);
    blk.load_q(a.q + (p.row0 + (real ? row : 0)) * a.ldq + (int64_t)head * a.head_dim, real);
    const int i0 = (int)((int64_t)p.steps * part / pa.parts), i1 = (int)((int64_t)p.steps * (part + 1) / pa.parts);
    blk.run(i0, i1);
    if (blk.doubtful()) bad = 1;
    __syncthreads();
    if (bad) blk.run_careful(i0, i1);
    if (pa.parts > 1) {
        constexpr int PF = part_floats(DP);
        const int64_t slot = (int64_t)(kh + pa.kv_heads * (rest / pa.parts)) * pa.parts;
        const rsrc_t r = make_rsrc(pa.slots + (slot + part) * PF, PF * 4u);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                bstore16<kCoherent>(u32x4{__float_as_uint(blk.o[d][4 * e]), __float_as_uint(blk.o[d][4 * e + 1]),
                                          __float_as_uint(blk.o[d][4 * e + 2]), __float_as_uint(blk.o[d][4 * e + 3])},
                                    r, ((4 * d + e) * 256 + t) * 16);
        if (l < 32) bstore8<kCoherent>(u32x2{__float_as_uint(blk.m), __float_as_uint(blk.sum)}, r,
                                       (kCols * DP + 2 * (32 * w + l)) * 4);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        uint32_t* counter = pa.counters + (kh + pa.kv_heads * (rest / pa.parts)) * kSyncStride;
        if (t == 0)
            last_part = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                        (uint32_t)(pa.parts - 1);
        __syncthreads();
        if (!last_part) return;
        if (t == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const rsrc_t all = make_rsrc(pa.slots + slot * PF, (uint32_t)pa.parts * PF * 4u);
        const int at_ms = (kCols * DP + 2 * (32 * w + (l & 31))) * 4;
        blk.m = -INFINITY;
        for (int z = 0; z < pa.parts; ++z) blk.m = fmaxf(blk.m, __uint_as_float(bload8<kCoherent>(all, z * PF * 4 + at_ms)[0]));
        const float ref = blk.m == -INFINITY ? 0.f : blk.m;
        blk.sum = 0.f;
        // block by block of the output, four parts in flight
#pragma unroll
        for (int d = 0; d < ND; ++d) {
#pragma unroll
            for (int x = 0; x < 16; ++x) blk.o[d][x] = 0.f;
            for (int z = 0; z < pa.parts; z += 4) {
                u32x2 ms[4];
                f32x4 y[4][4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const uint32_t at = z + b < pa.parts ? (uint32_t)(z + b) * PF * 4 : (uint32_t)kOut;
                    ms[b] = bload8<kCoherent>(all, (int)(at + at_ms));
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[b][e] = as_f4(bload16<kCoherent>(all, (int)(at + ((4 * d + e) * 256 + t) * 16)));
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float f = z + b < pa.parts ? __builtin_amdgcn_exp2f(__uint_as_float(ms[b][0]) - ref) : 0.f;
                    if (d == 0) blk.sum += __uint_as_float(ms[b][1]) * f;
#pragma unroll
                    for (int x = 0; x < 16; ++x) blk.o[d][x] += y[b][x >> 2][x & 3] * f;
                }
            }
        }
    }
    // Out through LDS, whole rows of a head at a time: a lane holds 8 bytes here and
    // there of its column, and storing those took 2 us of a workgroup's time.  Each
    // wave has its own part; chunk c of column j is in slot c ^ j % 16 (or % 8).
    constexpr int CH = Block::CH;
    const float f = blk.sum != 0.f ? 1.f / blk.sum : 0.f;
    unsigned char* part_lds = smem + w * 32 * CH * 16;
    constexpr int kMask = CH < 16 ? 7 : 15;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *(u32x2*)(part_lds + ((l & 31) * CH + ((4 * d + e) ^ (l & kMask))) * 16 + 8 * (l >> 5)) =
                u32x2{Fmt::pack2(blk.o[d][4 * e] * f, blk.o[d][4 * e + 1] * f),
                      Fmt::pack2(blk.o[d][4 * e + 2] * f, blk.o[d][4 * e + 3] * f)};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    const int64_t to = real ? (p.row0 + row) * a.ldo + (int64_t)head * a.head_dim : -1;
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
        const int j = i * (64 / CH) + l / CH, ch = l % CH;     // column, chunk
        const int64_t at = (int64_t)(uint32_t)__shfl((int)(uint32_t)to, j, 64) | (int64_t)__shfl((int)(to >> 32), j, 64) << 32;
        const u32x4 y = *(const u32x4*)(part_lds + (j * CH + (ch ^ (j & kMask))) * 16);
        if (at >= 0 && 8 * ch < a.head_dim) *(u32x4*)(a.out + at + 8 * ch) = y;
    }
}

// Launches whose tiles of 128 columns would leave most of the chip idle (one short
// prompt, a few rows behind a long cache): tiles of 32 columns, whose tokens the four
// waves divide and whose results meet in LDS.  One workgroup per compute unit, its
// tokens 64 per wave in one buffer: bound by the latency of the loads, so what counts
// is how few of them follow one another.  (203 rows of 32 heads: 9.1 us; in tiles of 128 columns 11.9 us.)
constexpr int kFewCols = 32;
constexpr int few_floats(int dp) { return kFewCols * dp + 2 * kFewCols; }

template <class Fmt, int DP>
__global__ void __launch_bounds__(256, 1) lora_attn_prompt_few_kernel(PromptArgs pa) {
    using Block = PromptBlock<Fmt, DP, 4>;
    constexpr int ND = DP / 32, CH = DP / 8, kMask = CH < 16 ? 7 : 15;
    __shared__ __align__(1024) unsigned char smem[Block::kLds];
    __shared__ float lm[4][kFewCols], ls[4][kFewCols];
    __shared__ int last_part;
    const AttnArgs& a = pa.a;
    const int t = threadIdx.x, l = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), c = l & 31;
    const int kh = blockIdx.x % pa.kv_heads;
    const int rest = blockIdx.x / pa.kv_heads;
    const int part = rest % pa.parts;
    PromptTile p;
    if (!find_tile(a, kFewCols, 4 * kKeys, rest / pa.parts, p)) return;
    float M, S;
    f32x4 y[4];                            // block w of the output of column c
    {
        const int col = p.col0 + c, row = col / a.group, head = kh * a.group + col - row * a.group;
        const bool real = row < p.n;
        Block blk(a, p, smem, kh, real ? p.pos0 + row : -1);
        blk.load_q(a.q + (p.row0 + (real ? row : 0)) * a.ldq + (int64_t)head * a.head_dim, real);
        const int i0 = (int)((int64_t)p.steps * part / pa.parts), i1 = (int)((int64_t)p.steps * (part + 1) / pa.parts);
        blk.run_own(i0, i1);
        if (__any(blk.doubtful())) blk.run_careful(i0, i1);
        // the waves' results meet: each has its own part of LDS, read by itself so far
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(f32x4*)(blk.lds + ((4 * d + e) * 64 + l) * 16) =
                    f32x4{blk.o[d][4 * e], blk.o[d][4 * e + 1], blk.o[d][4 * e + 2], blk.o[d][4 * e + 3]};
        if (l < 32) {
            lm[w][l] = blk.m;
            ls[w][l] = blk.sum;
        }
    }
    __syncthreads();
    {
        M = fmaxf(fmaxf(lm[0][c], lm[1][c]), fmaxf(lm[2][c], lm[3][c]));
        const float ref = M == -INFINITY ? 0.f : M;
        S = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = __builtin_amdgcn_exp2f(lm[i][c] - ref);
            S += ls[i][c] * f;
            if (w < ND)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[e] += *(const f32x4*)(smem + i * 2 * Block::kStage + ((4 * w + e) * 64 + l) * 16) * f;
        }
    }
    if (pa.parts > 1) {
        constexpr int PF = few_floats(DP);
        const int slot = (kh + pa.kv_heads * (rest / pa.parts)) * pa.parts;
        const rsrc_t all = make_rsrc(pa.slots + (int64_t)slot * PF, (uint32_t)pa.parts * PF * 4u);
        if (w < ND)
#pragma unroll
            for (int e = 0; e < 4; ++e) bstore16<kCoherent>(as_u4(y[e]), all, (part * PF + ((4 * w + e) * 64 + l) * 4) * 4);
        if (t < 32)
            bstore8<kCoherent>(u32x2{__float_as_uint(M), __float_as_uint(S)}, all, (part * PF + kFewCols * DP + 2 * t) * 4);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);                   // every thread's stores have reached the device
        __syncthreads();
        uint32_t* counter = pa.counters + (kh + pa.kv_heads * (rest / pa.parts)) * kSyncStride;
        if (t == 0) {
            last_part = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                        (uint32_t)(pa.parts - 1);
            if (last_part) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last_part) return;
        M = -INFINITY;
        S = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int block = min(w, ND - 1);
        for (int z = 0; z < pa.parts; z += 4) {          // four in flight
            u32x2 ms[4];
            f32x4 x[4][4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const uint32_t at = z + b < pa.parts ? (uint32_t)(z + b) * PF * 4 : (uint32_t)kOut;
                ms[b] = bload8<kCoherent>(all, (int)(at + (kFewCols * DP + 2 * c) * 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) x[b][e] = as_f4(bload16<kCoherent>(all, (int)(at + ((4 * block + e) * 64 + l) * 16)));
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float m1 = z + b < pa.parts ? __uint_as_float(ms[b][0]) : -INFINITY;
                const float mn = fmaxf(M, m1), ref = mn == -INFINITY ? 0.f : mn;
                const float f0 = __builtin_amdgcn_exp2f(M - ref), f1 = __builtin_amdgcn_exp2f(m1 - ref);
                M = mn;
                S = S * f0 + __uint_as_float(ms[b][1]) * f1;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = y[e] * f0 + x[b][e] * f1;
            }
        }
    }
    // out through LDS, past the sums: chunk i of column j in slot i ^ j % 16 (or % 8)
    const float f = S != 0.f ? 1.f / S : 0.f;
    unsigned char* rows = smem + Block::kStage;
    static_assert(kFewCols * DP * 4 <= Block::kStage, "the sums end before the second half of a wave's part");
    if (w < ND)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *(u32x2*)(rows + (c * CH + ((4 * w + e) ^ (c & kMask))) * 16 + 8 * (l >> 5)) =
                u32x2{Fmt::pack2(y[e][0] * f, y[e][1] * f), Fmt::pack2(y[e][2] * f, y[e][3] * f)};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewCols * CH / 256; ++i) {
        const int at = i * 256 + t, j = at / CH, ch = at % CH;
        const int col = p.col0 + j, row = col / a.group, head = kh * a.group + col - row * a.group;
        if (row < p.n && 8 * ch < a.head_dim)
            *(u32x4*)(a.out + (p.row0 + row) * a.ldo + (int64_t)head * a.head_dim + 8 * ch) =
                *(const u32x4*)(rows + (j * CH + (ch ^ (j & kMask))) * 16);
    }
}

template <int DP>
void launch_prompt_few(const PromptArgs& p, int dtype, unsigned blocks, hipStream_t st) {
    if (dtype == LORA_F16)
        hipLaunchKernelGGL((lora_attn_prompt_few_kernel<FmtF16, DP>), dim3(blocks), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((lora_attn_prompt_few_kernel<FmtBF16, DP>), dim3(blocks), dim3(256), 0, st, p);
}

template <int DP>
void launch_prompt(const PromptArgs& p, int dtype, unsigned blocks, hipStream_t st) {
    if (dtype == LORA_F16)
        hipLaunchKernelGGL((lora_attn_prompt_kernel<FmtF16, DP>), dim3(blocks), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((lora_attn_prompt_kernel<FmtBF16, DP>), dim3(blocks), dim3(256), 0, st, p);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

int check_attn(const lora_attn_s* h, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, int32_t n_rows,
               int32_t n_heads, const void* q, int64_t ldq, const void* out, int64_t ldo, float scale, int32_t window,
               int32_t n_sinks) {
    if (!h) return set_error(LORA_E_ARG, "attention handle is NULL");
    if (int rc = check_kv_cache(c)) return rc;
    if (int rc = check_kv_layer(c, layer)) return rc;
    if (int rc = check_kv_seqs(c, s)) return rc;
    if (n_rows < 0) return set_error(LORA_E_ARG, "negative n_rows");
    if (n_heads < 1 || n_heads % c->n_kv_heads)
        return set_error(LORA_E_SHAPE, "n_heads must be a positive multiple of n_kv_heads");
    const int64_t width = (int64_t)n_heads * c->head_dim;
    if (width > (1 << 24)) return set_error(LORA_E_SHAPE, "n_heads * head_dim exceeds 2^24");
    if (int rc = check_kv_rows("q", q, "ldq", ldq, width, n_rows)) return rc;
    if (int rc = check_kv_rows("out", out, "ldo", ldo, width, n_rows)) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale)) return set_error(LORA_E_ARG, "scale must be positive and finite");
    if (window < 0 || n_sinks < 0) return set_error(LORA_E_ARG, "negative window or n_sinks");
    if (n_rows > 0) {
        const uintptr_t qs = (uintptr_t)q, os = (uintptr_t)out;
        const uintptr_t qe = qs + ((uintptr_t)(n_rows - 1) * ldq + width) * 2;
        const uintptr_t oe = os + ((uintptr_t)(n_rows - 1) * ldo + width) * 2;
        if (qs < oe && os < qe) return set_error(LORA_E_OVERLAP, "q and out overlap");
    }
    return LORA_OK;
}

AttnArgs attn_args(const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, const int32_t* seg_offset,
                   int32_t n_rows, int32_t n_heads, const void* q, int64_t ldq, void* out, int64_t ldo, float scale,
                   int32_t window, int32_t n_sinks) {
    AttnArgs a;
    a.k = (const uint16_t*)c->k + layer * c->layer_stride;
    a.v = (const uint16_t*)c->v + layer * c->layer_stride;
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.tables = s->tables;
    a.lens = s->lens;
    a.seg_offset = seg_offset;
    a.page_stride = c->page_stride;
    a.head_stride = c->head_stride;
    a.row_stride = c->row_stride;
    a.ldq = ldq;
    a.ldo = ldo;
    a.n_rows = n_rows;
    a.n_seqs = s->n_seqs;
    a.ld_table = s->ld_table;
    a.max_len = s->max_len;
    a.n_pages = c->n_pages;
    a.page_shift = 0;
    while ((1 << a.page_shift) < c->page_rows) ++a.page_shift;
    a.group = n_heads / c->n_kv_heads;
    a.head_dim = c->head_dim;
    a.window = window < s->max_len ? window : 0;    // (one that long hides nothing)
    a.n_sinks = std::min(n_sinks, s->max_len);
    a.scale = scale;
    return a;
}

// Parts that a row tile's tokens are cut into, so that `tiles` of them come near
// `fill` workgroups: at least `least` tokens each, and 16 at most, which the last
// workgroup to end joins.
int prompt_parts(int64_t fill, int64_t tiles, int32_t tokens, int32_t least) {
    const int64_t n = std::min<int64_t>({fill / std::max<int64_t>(1, tiles), tokens / least, 16});
    return (int)std::max<int64_t>(1, n);
}

struct HandleDevice {
    int prev = -1;
    bool ok = false, moved = false;
    explicit HandleDevice(int device) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        moved = prev != device;
        ok = !moved || hipSetDevice(device) == hipSuccess;
    }
    ~HandleDevice() {
        if (moved) (void)hipSetDevice(prev);
    }
};

}  // namespace

extern "C" {

int lora_attn_create(lora_attn_t* out, int device, void* stream) {
    if (!out) return set_error(LORA_E_ARG, "out is NULL");
    *out = nullptr;
    if (device < 0) return set_error(LORA_E_ARG, "negative device");
    HandleDevice g(device);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_attn_create: cannot select the device");
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing((hipStream_t)stream, &cs) != hipSuccess)
        return set_error(LORA_E_HIP, "lora_attn_create: the stream's capture status");
    if (cs != hipStreamCaptureStatusNone) return set_error(LORA_E_CAPTURE, "lora_attn_create cannot be recorded in a graph");
    auto* h = new (std::nothrow) lora_attn_s();
    if (!h) return set_error(LORA_E_NOMEM, "handle allocation failed");
    h->device = device;
    int n_cu = 0;
    if (hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n_cu < 1) n_cu = 256;
    h->n_cu = n_cu;
    const size_t n_counters = (size_t)n_cu * decode_per_cu(64) * kCounters * kSyncStride;
    size_t n_floats = 0;
    for (int dp = 64; dp <= 256; dp *= 2)
        n_floats = std::max({n_floats, (size_t)n_cu * decode_per_cu(dp) * 2 * slot_floats(dp),
                             (size_t)n_cu * 2 * part_floats(dp)});
    hipError_t e = hipMalloc((void**)&h->counters, n_counters * 4);
    if (e == hipSuccess) e = hipMalloc((void**)&h->slots, n_floats * 4);
    if (e != hipSuccess) {
        lora_attn_destroy(h);
        return set_error(LORA_E_NOMEM, std::string("hipMalloc of the attention handle: ") + hipGetErrorString(e));
    }
    hipLaunchKernelGGL(lora_attn_clear_kernel, dim3((unsigned)((n_counters + 255) / 256)), dim3(256), 0,
                       (hipStream_t)stream, h->counters, (int)n_counters);
    e = hipGetLastError();
    if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
    if (e != hipSuccess) {
        lora_attn_destroy(h);
        return set_error(LORA_E_HIP, std::string("lora_attn_create: ") + hipGetErrorString(e));
    }
    *out = h;
    return LORA_OK;
}

int lora_attn_destroy(lora_attn_t a) {
    if (!a) return set_error(LORA_E_ARG, "attention handle is NULL");
    {
        HandleDevice g(a->device);
        (void)hipFree(a->counters);
        (void)hipFree(a->slots);
    }
    delete a;
    return LORA_OK;
}

int lora_attn_decode(lora_attn_t h, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, int32_t n_heads,
                     const void* q, int64_t ldq, void* out, int64_t ldo, float scale, int32_t window, int32_t n_sinks,
                     void* stream) {
    if (int rc = check_attn(h, c, layer, s, s ? s->n_seqs : 0, n_heads, q, ldq, out, ldo, scale, window, n_sinks)) return rc;
    if (s->n_seqs == 0) return LORA_OK;
    HandleDevice g(h->device);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_attn_decode: cannot select the device");
    const AttnArgs a = attn_args(c, layer, s, nullptr, s->n_seqs, n_heads, q, ldq, out, ldo, scale, window, n_sinks);
    DecodeArgs d;
    d.a = a;
    d.counters = h->counters;
    d.slots = h->slots;
    d.group_tiles = (a.group + kHeads - 1) / kHeads;
    d.heads_per_seq = c->n_kv_heads * d.group_tiles;
    const int64_t tiles = std::max(1, (s->max_len + kTile - 1) / kTile + 1);   // of a sequence, at most
    if (tiles * s->n_seqs > 0x7fffffff || tiles * d.heads_per_seq > 0x7fffffff)
        return set_error(LORA_E_SHAPE, "lora_attn_decode: more than 2^31 tiles of 128 tokens");
    const int dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
    const int blocks = (int)std::min<int64_t>((int64_t)h->n_cu * decode_per_cu(dp), tiles * s->n_seqs * d.heads_per_seq);
    if (dp == 64) launch_decode<64>(d, c->dtype, blocks, (hipStream_t)stream);
    else if (dp == 128) launch_decode<128>(d, c->dtype, blocks, (hipStream_t)stream);
    else launch_decode<256>(d, c->dtype, blocks, (hipStream_t)stream);
    return check_launch("lora_attn_decode");
}

int lora_attn_prompt(lora_attn_t h, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s,
                     const int32_t* seg_offset, int32_t n_rows, int32_t n_heads, const void* q, int64_t ldq, void* out,
                     int64_t ldo, float scale, int32_t window, int32_t n_sinks, void* stream) {
    if (int rc = check_attn(h, c, layer, s, n_rows, n_heads, q, ldq, out, ldo, scale, window, n_sinks)) return rc;
    if (!seg_offset) return set_error(LORA_E_ARG, "seg_offset is NULL");
    if ((uintptr_t)seg_offset & 3) return set_error(LORA_E_ALIGN, "seg_offset not 4-byte aligned");
    if (n_rows == 0 || s->n_seqs == 0) return LORA_OK;
    HandleDevice g(h->device);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_attn_prompt: cannot select the device");
    const AttnArgs a = attn_args(c, layer, s, seg_offset, n_rows, n_heads, q, ldq, out, ldo, scale, window, n_sinks);
    PromptArgs pa;
    pa.a = a;
    pa.counters = h->counters;
    pa.slots = h->slots;
    pa.kv_heads = c->n_kv_heads;
    // row tiles: every segment's last may be partly filled
    const int64_t cols = (int64_t)n_rows * a.group;
    auto tiles_of = [&](int n) { return std::min((cols + (int64_t)s->n_seqs * (n - 1)) / n, cols) * pa.kv_heads; };
    // (columns and tiles are counted in 32 bits, also where device offsets are not what they should be)
    if (cols > 0x7fffff00 || (cols / kFewCols + 1) * s->n_seqs > 0x7fffffff)
        return set_error(LORA_E_SHAPE, "lora_attn_prompt: too many rows and sequences");
    const int dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
    const int32_t tokens = window > 0 ? (int32_t)std::min<int64_t>(s->max_len, (int64_t)window + n_sinks + n_rows) : s->max_len;
    hipStream_t st = (hipStream_t)stream;
    // Tiles of 32 columns (head_dim to 128, where the tokens of four waves fit the LDS) where they run in one round: one
    // workgroup per compute unit, two of width 64; past 1024 tokens, which tiles of 128 columns share out as well, in
    // half a round. Both sides, us, tiles of 128 / of 32, 32/32 heads, f16:
    //   width 128, tokens:    the rows'   512        1024       2048       4096       16384
    //     128 tiles, 128 rows  8.5/9.1    15.9/11.5  21.3/14.1  22.3/18.1  30.4/28.8  73.8/86.9
    //     256 tiles, 256 rows  11.1/9.3   15.9/12.0  21.6/16.2  23.9/24.0  46.6/44.5  103/148
    //     320 tiles, 300 rows  12.2/16.8  16.9/21.2  22.5/29.0  30.5/45.0  46.3/78.5  131/282
    //   width 64, 512 tiles, 512 rows     12.6/10.0  17.1/14.0  23.0/22.4  33.5/38.2  106/145
    // and 7.2/8.9 for 64 rows of 64 tokens. What counts is max_len, as the lengths are on the device: with 4096 and more
    // there, 203 rows of 203 tokens take tiles of 128, most of whose parts are empty (25.6 us, 9.3 in tiles of 32).
    const int64_t few = tiles_of(kFewCols);
    if (dp <= 128 && tokens > kKeys && few <= (dp == 64 ? 2 : 1) * h->n_cu && (tokens <= 1024 || few <= h->n_cu / 2)) {
        pa.parts = prompt_parts(h->n_cu, few, tokens, 2 * 4 * kKeys);
        if (dp == 64) launch_prompt_few<64>(pa, c->dtype, (unsigned)(few * pa.parts), st);
        else launch_prompt_few<128>(pa, c->dtype, (unsigned)(few * pa.parts), st);
        return check_launch("lora_attn_prompt");
    }
    const int64_t tiles = tiles_of(kCols);
    pa.parts = prompt_parts(2 * (int64_t)h->n_cu, tiles, tokens, 8 * kKeys);
    const int64_t blocks = tiles * pa.parts;
    if (blocks > 0x7fffff) return set_error(LORA_E_SHAPE, "lora_attn_prompt: too many rows");
    if (dp == 64) launch_prompt<64>(pa, c->dtype, (unsigned)blocks, st);
    else if (dp == 128) launch_prompt<128>(pa, c->dtype, (unsigned)blocks, st);
    else launch_prompt<256>(pa, c->dtype, (unsigned)blocks, st);
    return check_launch("lora_attn_prompt");
}

}  // extern "C"
