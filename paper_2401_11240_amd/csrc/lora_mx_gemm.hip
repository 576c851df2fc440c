// gfx950 kernels of the product of rows in blocks (include/lora_mx.h): y = x W^T with
// x in E4M3 or E2M1 and W in E2M1 blocks, on v_mfma_scale_f32_*_f8f6f4, which takes codes and
// scale bytes as they are stored.
//
// The instruction, as measured (A here the weight, B the rows x; M = 16 with K 128 or M = 32
// with K 64): lane l holds row l % M of its operand; of 4-bit codes K 32 g .. + 31 (g = l / M:
// one block, 16 bytes), of 8-bit codes K 16 g .. + 15 and the same of the upper half of K; its scale
// byte (one of four of a word, chosen by the instruction) is that of block g of row l % M.  Accumulators:
// D[4 g + i][l % 16], or D[8 (i / 4) + 4 g + i % 4][l % 32].  The weight as A puts four consecutive
// columns of y into a lane.
//
// Two forms: lora_mx_stream_kernel for few rows, which reads the weight once from memory straight into
// registers, and lora_mx_tile_kernel for many, tiles through LDS.  Either may split K over workgroups, whose
// float32 sums lora_mx_join_kernel adds in order.
#include <stddef.h>

#include <algorithm>

#include "lora_device.h"
#include "lora_mx_internal.h"

namespace lora {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) unsigned char lds_u8;

constexpr int kUnits = 256, kXcds = 8;     // compute units and XCDs of the card
constexpr int64_t kJoinMost = 1 << 30;     // elements of y that may be joined from split K
constexpr int64_t kMostTiles = 1 << 22;    // of a launch; a product of more goes to several
constexpr int64_t kMostY = 1ll << 42;      // elements of y
constexpr int kTileSpan = 256;             // rows that one buffer resource covers, at most

struct GemmArgs {
    const unsigned char *x, *xs, *w, *ws;
    void* y;
    float* part;                           // [splits][n_rows][h_out] where splits > 1
    int64_t ldx, ldxs, ldw, ldws, ldy;     // bytes; ldy elements
    int n_rows, h_out, blocks;
    int dtype;
    int splits, split_blocks;              // K in ranges of split_blocks blocks, a multiple of 16
    int n_nt, n_tt, per_xcd;               // tiles
};

// s_waitcnt lgkmcnt(0), vmcnt and expcnt left free (gfx9 encoding).
__device__ __forceinline__ void wait_lgkm0() { __builtin_amdgcn_s_waitcnt(0xC07F); }
// s_waitcnt with lgkmcnt(0) and vmcnt(0).
__device__ __forceinline__ void wait_vm0_lgkm0() { __builtin_amdgcn_s_waitcnt(0x0070); }
// s_waitcnt vmcnt(N), the other counters left free.
template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// 16 bytes per lane from buffer r at byte offset off (zeros when out of range, word by word)
// into LDS at lds + 16 * lane; lds is the same in every lane.  In assembly, with no output: for the
// builtin the compiler waits for every such load in flight before each LDS read.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is reserved: nothing to preserve, the clobber is what is said
__device__ __forceinline__ void lds_load16(const u32x4& r, uint32_t lds, int off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(off), "s"(r) : "memory", "m0");
}
#pragma clang diagnostic pop
// The resource of make_rsrc() as four scalar words, five wait states (gfx9) after the
// vector instructions that write them.
__device__ __forceinline__ u32x4 rsrc_words(const void* base, uint32_t bytes) {
    const uint64_t b = (uint64_t)base;
    u32x4 r = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) & 0xffffu,
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), (uint32_t)kRsrcWord3};
    asm volatile("s_nop 4" : "+s"(r));
    return r;
}

// Four consecutive columns of a row of y, rounded.
__device__ __forceinline__ void store4(const GemmArgs& a, int row, int n, const f32x4& v) {
    const int64_t at = row * a.ldy + n;
    if (a.dtype == LORA_F32) *(f32x4*)((float*)a.y + at) = v;
    else if (a.dtype == LORA_F16) *(u32x2*)((uint16_t*)a.y + at) = u32x2{FmtF16::pack2(v[0], v[1]), FmtF16::pack2(v[2], v[3])};
    else *(u32x2*)((uint16_t*)a.y + at) = u32x2{FmtBF16::pack2(v[0], v[1]), FmtBF16::pack2(v[2], v[3])};
}
__device__ __forceinline__ f32x4* part4(const GemmArgs& a, int split, int row, int n) {
    return (f32x4*)(a.part + ((int64_t)split * a.n_rows + row) * a.h_out + n);
}

// y from the sums of the K ranges, added in their order.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) lora_mx_join_kernel(GemmArgs a) {
    const int per_row = a.h_out / 4;
    const int64_t i = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    const int row = (int)(i / per_row), n = 4 * (int)(i - (int64_t)row * per_row);
    if (row >= a.n_rows) return;
    f32x4 v = *part4(a, 0, row, n);
    for (int s = 1; s < a.splits; ++s) v += *part4(a, s, row, n);
    store4(a, row, n, v);
}

// ---------------------------------------------------------------------------
// tiles: many rows
// ---------------------------------------------------------------------------

// TN columns of y (rows of W) by TT rows of y, by WN x WT waves; XF is the format of x.  K in steps of kStep blocks
// of 32, two slices of K 64.  Loads go from memory to LDS without registers, RING - 1 steps ahead; a slice's
// fragments are read while the slice before is multiplied; one barrier a step.
//
// 8437 rows, 5120 -> 13824, 8-bit x: 482-490 us, 2.4 PFLOP/s (550 on another card); 2048 rows, 8192 -> 8192, 4-bit x: 75-81 us,
// 3.5 PFLOP/s; 64 rows, 8192 -> 28672: 36-38 us, 3.4 TB/s of W, bound by loads.  Of the first the matrix instructions alone
// take 300 us (they are 4 PFLOP/s with 8-bit x, 6 with 4-bit x), the loads alone 347, and the whole with codes of zero 400 where
// random ones take 550: the clock, which the power limit sets by what the data make the units switch, is a good part of
// what is left.  Tried without gain: four waves of 128 x 128 (no registers for a second wave on a SIMD), steps of K 256
// (spills: 143 us for the second), a ring of four, two workgroups of 256 x 128 on a unit, K begun at another place on every
// XCD, sixteen waves for a band of one row tile.
constexpr int kStep = 4;                   // blocks of a step

template <int XF, int TN, int TT, int WN, int WT, int RING>
struct TileCfg {
    static constexpr int kWaves = WN * WT, kThreads = 64 * kWaves;
    static constexpr int NB = TN / WN / 32, TB = TT / WT / 32;     // 32 x 32 blocks of a wave
    static constexpr int kXRow = XF == LORA_E4M3 ? 2 * kStep : kStep, kWRow = kStep;   // 16-byte chunks of a row and step
    static constexpr int kXChunks = TT * kXRow, kWChunks = TN * kWRow, kStage = kXChunks + kWChunks;
    static constexpr int XL = kXChunks / 64 / kWaves, WL = kWChunks / 64 / kWaves, NL = XL + WL;   // loads of a wave and step
    static constexpr int RB = RING;
    static constexpr int kTurn = 16 / kStep;                          // steps of 16 blocks, whose scales are a 16-byte word
    static constexpr int kScales = TN + TT;                        // such words: W's rows, then x's
    static constexpr int SL = (kScales / 64 + kWaves - 1) / kWaves;
    static constexpr int kLds = RB * kStage + 2 * kScales;         // 16-byte chunks
    static_assert(kXChunks % (64 * kWaves) == 0 && kWChunks % (64 * kWaves) == 0 && kScales % 64 == 0, "whole loads");
    static_assert(kLds * 16 <= 160 * 1024 && RB * NL + SL < 64, "ring");
    // (scales, asked for kTurn - 1 steps before they are read, have come when at most RB - 2 steps' loads are out)
    static_assert(RB >= 2 && RB - 2 < kTurn, "ring");
};

// Slot of chunk c of row r among the row's: rows that are read together (16 or 32 lanes) fall in all of
// the 16 bank groups.
template <int ROW>
__device__ __forceinline__ int slot_of(int r, int c) {
    static_assert(ROW == 4 || ROW == 8, "chunks of a row");
    return c ^ (ROW == 4 ? (r >> 2) & 3 : (r >> 1) & 7);
}

template <class C, int XF, int TN, int TT, int WN, int WT>
struct Tile {
    static constexpr int NB = C::NB, TB = C::TB, NW = C::kWaves, RB = C::RB, NL = C::NL;
    const GemmArgs& a;
    const int w, l, wn, wt, n0, t0;
    u32x4* lds;
    uint32_t lbase;
    u32x4 xr, wr, sxr, swr;
    uint32_t xo[C::XL], wo[C::WL], so[C::SL];
    int xblk[C::XL], wblk[C::WL];          // block of a step that this lane's chunk belongs to
    f32x16 acc[NB][TB];

    __device__ __forceinline__ Tile(const GemmArgs& args, u32x4* smem, int nt, int tt)
        : a(args), w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), l(threadIdx.x & 63), wn(w / WT), wt(w % WT),
          n0(nt * TN), t0(tt * TT), lds(smem) {
        lbase = (uint32_t)(uintptr_t)(lds_u8*)(unsigned char*)smem;
        const int nr = min_i(TN, a.h_out - n0), tr = min_i(TT, a.n_rows - t0);
        const int words = 4 * ((a.blocks + 3) >> 2);
        xr = rsrc_words(a.x + t0 * a.ldx, (uint32_t)((tr - 1) * a.ldx) + (uint32_t)a.blocks * (XF == LORA_E4M3 ? 32u : 16u));
        wr = rsrc_words(a.w + n0 * a.ldw, (uint32_t)((nr - 1) * a.ldw) + (uint32_t)a.blocks * 16u);
        sxr = rsrc_words(a.xs + t0 * a.ldxs, (uint32_t)((tr - 1) * a.ldxs) + (uint32_t)words);
        swr = rsrc_words(a.ws + n0 * a.ldws, (uint32_t)((nr - 1) * a.ldws) + (uint32_t)words);
#pragma unroll
        for (int i = 0; i < C::XL; ++i) {
            const int at = 64 * (NW * i + w) + l, r = at / C::kXRow, c = slot_of<C::kXRow>(r, at % C::kXRow);
            xblk[i] = XF == LORA_E4M3 ? c >> 1 : c;
            xo[i] = r < tr ? (uint32_t)(r * a.ldx) + 16u * c : (uint32_t)kOut;
        }
#pragma unroll
        for (int i = 0; i < C::WL; ++i) {
            const int at = 64 * (NW * i + w) + l, r = at / C::kWRow, c = slot_of<C::kWRow>(r, at % C::kWRow);
            wblk[i] = c;
            wo[i] = r < nr ? (uint32_t)(r * a.ldw) + 16u * c : (uint32_t)kOut;
        }
#pragma unroll
        for (int i = 0; i < C::SL; ++i) {
            const int r = 64 * (NW * i + w) + l;                   // W's rows, then x's
            so[i] = r < TN ? (r < nr ? (uint32_t)(r * a.ldws) : (uint32_t)kOut)
                           : (r - TN < tr ? (uint32_t)((r - TN) * a.ldxs) : (uint32_t)kOut);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }

    // Load i of step k into ring buffer b; blocks from `end` on are zeros.
    __device__ __forceinline__ void load(int k, int end, int b, int i) {
        const uint32_t at = lbase + (uint32_t)(b * C::kStage) * 16u;
        if (i < C::XL) {
            const uint32_t kb = kStep * k + xblk[i] < end ? (uint32_t)k * (16u * C::kXRow) : (uint32_t)kOut;
            lds_load16(xr, at + (uint32_t)(NW * i + w) * 1024u, (int)(xo[i] + kb));
        } else {
            const int j = i - C::XL;
            const uint32_t kb = kStep * k + wblk[j] < end ? (uint32_t)k * (16u * C::kWRow) : (uint32_t)kOut;
            lds_load16(wr, at + C::kXChunks * 16u + (uint32_t)(NW * j + w) * 1024u, (int)(wo[j] + kb));
        }
    }
    // The scales of blocks 16 s .. 16 s + 15 into half `half`.
    __device__ __forceinline__ void load_scales(int s, int half) {
        const uint32_t at = lbase + (uint32_t)(RB * C::kStage + half * C::kScales) * 16u;
#pragma unroll
        for (int i = 0; i < C::SL; ++i)
            if (NW * i + w < C::kScales / 64)
                lds_load16(NW * i + w < TN / 64 ? swr : sxr, at + (uint32_t)(NW * i + w) * 1024u, (int)(so[i] + 16u * (uint32_t)s));
    }

    // Fragments of slice j: e < NB of W, then x's two parts of each block (one of 4-bit x).
    static constexpr int kXParts = XF == LORA_E4M3 ? 2 : 1, NF = NB + TB * kXParts;
    __device__ __forceinline__ u32x4 frag(const u32x4* buf, int j, int e) const {
        const int r = l & 31, h = l >> 5;
        if (e < NB) return buf[C::kXChunks + ((wn * NB + e) * 32 + r) * C::kWRow + slot_of<C::kWRow>(r, 2 * j + h)];
        const int x = e - NB, row = (wt * TB + x / kXParts) * 32 + r;
        return buf[row * C::kXRow + slot_of<C::kXRow>(r, XF == LORA_E4M3 ? 4 * j + h + 2 * (x % 2) : 2 * j + h)];
    }
    // Scale words of the k-th step taken: byte 2 j of the shifted word is that of this lane's block of slice j.
    __device__ __forceinline__ void read_scales(uint32_t (&s)[NB + TB], int k) const {
        const uint32_t* p = (const uint32_t*)(lds + RB * C::kStage + ((k / C::kTurn) & 1) * C::kScales) + k % C::kTurn;
#pragma unroll
        for (int i = 0; i < NB; ++i) s[i] = p[((wn * NB + i) * 32 + (l & 31)) * 4];
#pragma unroll
        for (int i = 0; i < TB; ++i) s[NB + i] = p[(TN + (wt * TB + i) * 32 + (l & 31)) * 4];
    }

    template <int J>
    __device__ __forceinline__ void mma(f32x16& c, const u32x4& fw, const u32x4& x0, const u32x4& x1, uint32_t sw, uint32_t sx) {
        const i32x8 A = {(int)fw[0], (int)fw[1], (int)fw[2], (int)fw[3], 0, 0, 0, 0};
        const i32x8 B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
        c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, XF == LORA_E4M3 ? 0 : 4, 2 * J, (int)sw, 2 * J, (int)sx);
    }

    // Slice J: its MFMAs, between them the fragments of the next slice (in `next`) and loads [l0, l1) of step kl.
    template <int J>
    __device__ __forceinline__ void slice(u32x4 (&f)[2][NF], const uint32_t (&s)[NB + TB], const u32x4* next, int kl, int end,
                                          int b, int l0, int l1) {
        constexpr int NM = NB * TB;
        int re = 0, ld = l0;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            const int i = m / TB, jt = m % TB;
            mma<J>(acc[i][jt], f[J][i], f[J][NB + jt * kXParts], f[J][NB + jt * kXParts + kXParts - 1], s[i], s[NB + jt]);
            const int want = min_i(NF, ((m + 1) * NF * 4 + NM * 3 - 1) / (NM * 3));
            for (; re < want; ++re) f[1 - J][re] = frag(next, 1 - J, re);
            for (; ld < l0 + ((m + 1) * (l1 - l0)) / NM; ++ld) load(kl, end, b, ld);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // The product over steps [k0, k1), k0 a multiple of kTurn, begun at step k0 + turn (a multiple of kTurn; 0 if their
    // number is none).  On return no load is in flight and every wave's LDS reads are done.
    __device__ __forceinline__ void product(int k0, int k1, int turn) {
        constexpr int kFirst = NL / 2;
        const int end = min_i(a.blocks, kStep * k1), n = k1 - k0;
        // the i-th step taken; from n on one whose blocks are all past the end
        auto at = [&](int i) __attribute__((always_inline)) { return i >= n ? k1 : i + turn < n ? k0 + i + turn : k0 + i + turn - n; };
        load_scales(at(0) / C::kTurn, 0);
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < (b < RB - 1 ? NL : kFirst); ++i) load(at(b), end, b, i);
        wait_vm<(RB - 2) * NL + kFirst>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        u32x4 f[2][NF];
        uint32_t s[NB + TB], sn[NB + TB];
#pragma unroll
        for (int e = 0; e < NF; ++e) f[0][e] = frag(lds, 0, e);
        read_scales(sn, 0);
        int b = 0;
        for (int i = 0; i < n; ++i) {
            const int bn = b + 1 == RB ? 0 : b + 1, bp = b == 0 ? RB - 1 : b - 1;
            const u32x4* cur = lds + b * C::kStage;
            const u32x4* nxt = lds + bn * C::kStage;
            // scales of blocks past the end, whatever lies there, are zeros (255 would make NaN of their zeros)
            const int left = a.blocks - kStep * at(i);
            const uint32_t mask = left >= 4 ? 0xffffffffu : left > 0 ? (1u << (8 * left)) - 1 : 0u;
#pragma unroll
            for (int e = 0; e < NB + TB; ++e) s[e] = (sn[e] & mask) >> (8 * (l >> 5));
            if (i % C::kTurn == 0) load_scales(at(i + C::kTurn) / C::kTurn, (i / C::kTurn + 1) & 1);
            slice<0>(f, s, cur, at(i - 1 + RB), end, bp, kFirst, NL);
            // this wave's reads of cur are done and its loads of the next step have landed; past the barrier every
            // wave's are and have
            wait_lgkm0();
            wait_vm<(RB - 2) * NL>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            read_scales(sn, i + 1);
            slice<1>(f, s, nxt, at(i + RB), end, b, 0, kFirst);
            b = bn;
        }
        wait_vm0_lgkm0();
        __builtin_amdgcn_s_barrier();
    }
};

template <int XF, int TN, int TT, int WN, int WT, int RING>
__global__ void __launch_bounds__(64 * WN * WT) lora_mx_tile_kernel(GemmArgs a) {
    using C = TileCfg<XF, TN, TT, WN, WT, RING>;
    __shared__ __attribute__((aligned(1024))) u32x4 smem[C::kLds];
    const int q = blockIdx.x / kXcds, tile = (blockIdx.x % kXcds) * a.per_xcd + q;
    if (tile >= a.n_nt * a.n_tt) return;
    // panels of kPanel row tiles, column by column
    constexpr int kPanel = 8;
    const int panel = tile / (kPanel * a.n_nt), u = tile - panel * kPanel * a.n_nt;
    const int high = min_i(kPanel, a.n_tt - panel * kPanel);
    const int nt = u / high, tt = panel * kPanel + u - nt * high;
    Tile<C, XF, TN, TT, WN, WT> T(a, smem, nt, tt);
    const int steps = (a.blocks + kStep - 1) / kStep, k0 = blockIdx.y * (a.split_blocks / kStep);
    const int k1 = min_i(steps, k0 + a.split_blocks / kStep);
    // workgroups that share no W begin K at different places, so that the rows of a step, whose distance is often a
    // power of two, do not all come from the same few memory channels (64 rows, 8192 -> 28672: 42.0 -> 38.1 us; where
    // workgroups share W it would cost them the L2's copy: 8437 rows, 5120 -> 13824: 485 -> 570 us)
    const int fours = (k1 - k0) / C::kTurn;
    const int turn = a.n_tt == 1 && (k1 - k0) % C::kTurn == 0 ? C::kTurn * (q % fours) : 0;
    T.product(k0, k1, turn);

    const int tb = T.t0 + 32 * C::TB * T.wt, nb = T.n0 + 32 * C::NB * T.wn;
    const int r = T.l & 31, h = T.l >> 5;
    if (a.splits > 1 || a.dtype == LORA_F32) {
#pragma unroll
        for (int i = 0; i < C::NB; ++i)
#pragma unroll
            for (int j = 0; j < C::TB; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16& c = T.acc[i][j];
                    const int row = tb + 32 * j + r, n = nb + 32 * i + 8 * g + 4 * h;
                    const f32x4 v = {c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
                    if (row < a.n_rows && n < a.h_out) {
                        if (a.splits > 1) *part4(a, blockIdx.y, row, n) = v;
                        else *(f32x4*)((float*)a.y + row * a.ldy + n) = v;
                    }
                }
        return;
    }
    // 16-bit y: 32 rows at a time through the wave's own share of LDS (16-byte chunk q of row r at slot
    // q ^ r % 16, its halves swapped for odd r / 16) and out by rows, 16 bytes per lane, past the caches, which keep x and W
    // (8437 rows, 5120 -> 13824: 490 -> 483 us, 2048 rows, 8192 -> 8192 with 4-bit x 86 -> 81)
    constexpr int QC = 4 * C::NB, kMask = QC < 16 ? QC - 1 : 15;
    u32x2* q8 = (u32x2*)(smem + T.w * 32 * QC);
    const u32x4* q16 = (const u32x4*)q8;
#pragma unroll
    for (int j = 0; j < C::TB; ++j) {
#pragma unroll
        for (int i = 0; i < C::NB; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x16& c = T.acc[i][j];
                const int at = (r * QC + ((4 * i + g) ^ (r & kMask))) * 2 + (h ^ ((r >> 4) & 1));
                if (a.dtype == LORA_F16) q8[at] = u32x2{FmtF16::pack2(c[4 * g], c[4 * g + 1]), FmtF16::pack2(c[4 * g + 2], c[4 * g + 3])};
                else q8[at] = u32x2{FmtBF16::pack2(c[4 * g], c[4 * g + 1]), FmtBF16::pack2(c[4 * g + 2], c[4 * g + 3])};
            }
#pragma unroll
        for (int it = 0; it < QC / 2; ++it) {
            const int ro = it * (64 / QC) + T.l / QC, qc = T.l % QC;
            const u32x4 v = q16[ro * QC + (qc ^ (ro & kMask))];
            const int row = tb + 32 * j + ro, n = nb + 8 * qc;
            if (row < a.n_rows && n < a.h_out)
                __builtin_nontemporal_store((ro >> 4) & 1 ? u32x4{v.z, v.w, v.x, v.y} : v, (u32x4*)((uint16_t*)a.y + row * a.ldy + n));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// ---------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------

// Waves of a workgroup: eight (two per SIMD) where two units of loads and the accumulators fit half
// of a SIMD's registers, else four.
template <int XF, int NR, int TG>
struct StreamCfg {
    static constexpr int kXParts = XF == LORA_E4M3 ? 2 : 1;        // 16-byte parts of a lane's K 128 of a row of x
    static constexpr int kUnitRegs = 2 * 4 * (NR + TG * kXParts) + 2 * (NR + TG);
    static constexpr int kWaves = 2 * kUnitRegs + 4 * NR * TG <= 200 ? 8 : 4;
};

constexpr int kStreamTurn = 5;

// 16 NR rows of W by 16 TG rows of x.  Wave w takes the units (of K 256) w, w + kWaves, ...: every
// element of W and x goes from memory to the registers of one lane, the next unit's on the
// way while this one's MFMAs run.  A load instruction covers 64 consecutive bytes of 16 rows.  The waves'
// sums are added through LDS in their order.
template <int XF, int NR, int TG>
struct Stream {
    using C = StreamCfg<XF, NR, TG>;
    static constexpr int kXBlock = XF == LORA_E4M3 ? 32 : 16, kXParts = C::kXParts;
    struct Unit {
        u32x4 w[2][NR], x[2][TG][kXParts];
        u32x2 sw[NR], sx[TG];
    };
    const GemmArgs& a;
    const int l, g;
    rsrc_t rw, rx, rsw, rsx;
    int ow[NR], osw[NR], ox[TG], osx[TG];
    f32x4 acc[NR][TG];

    __device__ __forceinline__ Stream(const GemmArgs& args, int n0, int t0) : a(args), l(threadIdx.x & 63), g((threadIdx.x & 63) >> 4) {
        const int nr = min_i(16 * NR, a.h_out - n0), tr = min_i(16 * TG, a.n_rows - t0), r = l & 15;
        const int words = (a.blocks + 3) >> 2;
        rw = make_rsrc(a.w + n0 * a.ldw, (uint32_t)((nr - 1) * a.ldw) + 16u * a.blocks);
        rx = make_rsrc(a.x + t0 * a.ldx, (uint32_t)((tr - 1) * a.ldx) + (uint32_t)kXBlock * a.blocks);
        rsw = make_rsrc(a.ws + n0 * a.ldws, (uint32_t)((nr - 1) * a.ldws) + 4u * words);
        rsx = make_rsrc(a.xs + t0 * a.ldxs, (uint32_t)((tr - 1) * a.ldxs) + 4u * words);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            ow[i] = 16 * i + r < nr ? (int)((16 * i + r) * a.ldw) + 16 * g : kOut;
            osw[i] = 16 * i + r < nr ? (int)((16 * i + r) * a.ldws) : kOut;
        }
#pragma unroll
        for (int i = 0; i < TG; ++i) {
            ox[i] = 16 * i + r < tr ? (int)((16 * i + r) * a.ldx) + 16 * g : kOut;
            osx[i] = 16 * i + r < tr ? (int)((16 * i + r) * a.ldxs) : kOut;
        }
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int j = 0; j < TG; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    static __device__ __forceinline__ u32x4 load16(rsrc_t r, int off, int soff) {
        return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, soff, 0));
    }
    // WHOLE: all of the unit's blocks are there; otherwise those past the end are zeros.
    template <bool WHOLE>
    __device__ __forceinline__ void load(Unit& q, int u) const {
#pragma unroll
        for (int i = 0; i < NR; ++i) q.sw[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rsw, osw[i], 8 * u, 0));
#pragma unroll
        for (int i = 0; i < TG; ++i) q.sx[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rsx, osx[i], 8 * u, 0));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int left = a.blocks - 8 * u - 4 * j;
#pragma unroll
            for (int i = 0; i < NR; ++i) q.w[j][i] = load16(rw, WHOLE || g < left ? ow[i] + 64 * j : kOut, 128 * u);
            // (a lane's part p of 8-bit x is half of block g / 2 + 2 p)
#pragma unroll
            for (int i = 0; i < TG; ++i)
#pragma unroll
                for (int p = 0; p < kXParts; ++p)
                    q.x[j][i][p] = load16(rx, WHOLE || (kXParts == 2 ? (g >> 1) + 2 * p : g) < left ? ox[i] + 4 * kXBlock * j + 64 * p : kOut,
                                          8 * kXBlock * u);
        }
    }
    __device__ __forceinline__ void load(Unit& q, int u) const {
        if (8 * u + 8 <= a.blocks) load<true>(q, u);
        else load<false>(q, u);
    }

    __device__ __forceinline__ void multiply(const Unit& q, int u) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // scales of blocks past the end, whatever lies there, are zeros (255 would make NaN of their zeros)
            const int left = a.blocks - 8 * u - 4 * j;
            const uint32_t mask = left >= 4 ? 0xffffffffu : left > 0 ? (1u << (8 * left)) - 1 : 0u;
            uint32_t sw[NR], sx[TG];
#pragma unroll
            for (int i = 0; i < NR; ++i) sw[i] = (q.sw[i][j] & mask) >> (8 * g);
#pragma unroll
            for (int i = 0; i < TG; ++i) sx[i] = (q.sx[i][j] & mask) >> (8 * g);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const u32x4& w = q.w[j][i];
                const i32x8 A = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < TG; ++t) {
                    const u32x4 &x0 = q.x[j][t][0], &x1 = q.x[j][t][kXParts - 1];
                    const i32x8 B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
                    acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc[i][t], 4, XF == LORA_E4M3 ? 0 : 4, 0,
                                                                                 (int)sw[i], 0, (int)sx[t]);
                }
            }
        }
    }
};

template <int XF, int NR, int TG>
__global__ void __launch_bounds__((64 * StreamCfg<XF, NR, TG>::kWaves)) lora_mx_stream_kernel(GemmArgs a) {
    constexpr int NW = StreamCfg<XF, NR, TG>::kWaves;
    __shared__ f32x4 red[NW][TG][64];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
    const int n0 = blockIdx.x * 16 * NR, t0 = blockIdx.y * 16 * TG;
    Stream<XF, NR, TG> S(a, n0, t0);
    // the units in a ring, entered at another place by every workgroup
    const int n_units = (a.blocks + 7) / 8;
    const int turn = blockIdx.x * kStreamTurn % n_units;
    auto at = [&](int i) __attribute__((always_inline)) { return i + turn < n_units ? i + turn : i + turn - n_units; };
    int i = w;
    if (i < n_units) {
        typename Stream<XF, NR, TG>::Unit p, q;
        S.load(p, at(i));
        for (;;) {
            if (i + NW >= n_units) {
                S.multiply(p, at(i));
                break;
            }
            S.load(q, at(i + NW));
            S.multiply(p, at(i));
            i += NW;
            if (i + NW >= n_units) {
                S.multiply(q, at(i));
                break;
            }
            S.load(p, at(i + NW));
            S.multiply(q, at(i));
            i += NW;
        }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
#pragma unroll
        for (int t = 0; t < TG; ++t) red[w][t][l] = S.acc[i][t];
        __syncthreads();
        for (int e = threadIdx.x; e < TG * 64; e += 64 * NW) {
            const int t = e >> 6, le = e & 63;
            f32x4 v = red[0][t][le];
#pragma unroll
            for (int k = 1; k < NW; ++k) v += red[k][t][le];
            const int row = t0 + 16 * t + (le & 15), n = n0 + 16 * i + 4 * (le >> 4);
            if (row < a.n_rows && n < a.h_out) store4(a, row, n, v);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// which form, in which tiles
// ---------------------------------------------------------------------------

struct Plan {
    bool tiles;
    int nr, tg;                            // stream: 16-row groups of W and x
    int tn, tt;                            // tiles
    int splits, split_blocks;
};

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Few rows and a weight that is not very large go straight to registers: nothing is shared, so the small
// launches' latency is what counts (16 rows: 4096 -> 4096 6.3 us against 9.5 in tiles, 5120 -> 13824 12.2
// against 15.7, 8192 -> 28672 41.0 against 36.4; 24 rows: 7.8 against 10.0, 14.3 against 16.4, 46 against 36.5).
// Tiles are chosen by what has to be loaded, which bounds them (the latency of what the L2 does not have yet): a
// compute unit gets about 34 GB/s with one workgroup on it and 60 with two or more, all together 11.8 TB/s, W's first
// reading slower; 4 us around a launch, and for split K another launch and the sums' way through memory.  Over 60
// shapes from 24 to 2048 rows and 1 to 8 ranges the choice was within 10% of the fastest in all but a few.
Plan plan_product(int n_rows, int h_out, int blocks, int format) {
    Plan p{};
    const int sixteens = ceil_div(blocks, 16);
    const double weight = 16.0 * blocks * h_out;           // bytes
    if (n_rows <= 32 && weight <= (n_rows <= 4 ? 1.5e8 : n_rows <= 16 ? 6e7 : 3e7)) {
        p.tg = n_rows <= 16 ? 1 : 2;
        const int groups = ceil_div(h_out, 16);
        p.nr = groups <= kUnits ? 1 : groups <= 2 * kUnits || n_rows <= 4 ? 2 : 4;
        p.splits = 1;
        p.split_blocks = 16 * sixteens;
        return p;
    }
    static const int kTiles[4][3] = {{64, 64, 3}, {128, 64, 2}, {128, 128, 2}, {256, 256, 1}};   // edges, workgroups a unit holds
    double best = 0;
    p.tiles = true;
    for (const auto& t : kTiles)
        for (int want = 1; want <= 8; want *= 2) {
            const int range = 16 * ceil_div(sixteens, want), splits = ceil_div(blocks, range);
            const int64_t each_range = (int64_t)ceil_div(h_out, t[0]) * ceil_div(n_rows, t[1]);
            if (want > 1 && (splits <= want / 2 || (int64_t)n_rows * h_out > kJoinMost || each_range > kMostTiles)) break;
            const double bytes = (double)std::min(range, blocks) * (t[0] * 16 + t[1] * (format == LORA_E4M3 ? 32 : 16)) * 1e-3;
            const int64_t groups = each_range * splits;
            const int64_t each = (groups + kUnits - 1) / kUnits, rest = each % t[2];    // of the unit with most
            const double unit = (double)(each - rest) * bytes / (t[2] > 1 ? 60 : 34) + (double)rest * bytes / (rest > 1 ? 60 : 34);
            double us = 4 + std::max(unit, (double)groups * bytes / 11800 + weight / 1e7);
            if (splits > 1) us += 2.5 + 8.0 * splits * n_rows * h_out / 5e6;
            if (best == 0 || us < best) {
                best = us;
                p.tn = t[0];
                p.tt = t[1];
                p.splits = splits;
                p.split_blocks = range;
            }
        }
    return p;
}

int check_product(const lora_mx_t* x, const lora_mx_t* w) {
    if (int rc = check_mx("x", x)) return rc;
    if (int rc = check_mx("w", w)) return rc;
    if (w->format != LORA_E2M1) return set_error(LORA_E_ARG, "w: format must be LORA_E2M1");
    if (x->h != w->h) return set_error(LORA_E_SHAPE, "x and w differ in h");
    if (w->n_rows < 8 || w->n_rows % 8) return set_error(LORA_E_SHAPE, "w: n_rows must be a positive multiple of 8");
    if ((int64_t)x->n_rows * w->n_rows > kMostY) return set_error(LORA_E_SHAPE, "y has more than 2^42 elements");
    for (const lora_mx_t* q : {x, w})
        if (std::max(q->ld_codes, q->ld_scales) * kTileSpan > (int64_t)kMaxSpan)
            return set_error(LORA_E_SHAPE, "256 rows of x or w span more than 0x7fff0000 bytes");
    return LORA_OK;
}

size_t part_bytes(const Plan& p, const lora_mx_t* x, const lora_mx_t* w) {
    return p.splits > 1 ? (size_t)p.splits * x->n_rows * w->n_rows * 4 : 16;
}

template <int XF, int NR>
void launch_stream(const GemmArgs& a, const Plan& p, hipStream_t st) {
    const dim3 grid(ceil_div(a.h_out, 16 * NR), ceil_div(a.n_rows, 16 * p.tg));
    if (p.tg == 1)
        hipLaunchKernelGGL((lora_mx_stream_kernel<XF, NR, 1>), grid, dim3(64 * StreamCfg<XF, NR, 1>::kWaves), 0, st, a);
    else
        hipLaunchKernelGGL((lora_mx_stream_kernel<XF, NR, 2>), grid, dim3(64 * StreamCfg<XF, NR, 2>::kWaves), 0, st, a);
}

template <int XF, int TN, int TT, int WN, int WT, int RING>
void launch_tiles(GemmArgs& a, const Plan& p, hipStream_t st) {
    a.n_nt = ceil_div(a.h_out, TN);
    a.n_tt = ceil_div(a.n_rows, TT);
    a.per_xcd = ceil_div((int64_t)a.n_nt * a.n_tt, kXcds);
    hipLaunchKernelGGL((lora_mx_tile_kernel<XF, TN, TT, WN, WT, RING>), dim3(kXcds * a.per_xcd, p.splits), dim3(64 * WN * WT), 0,
                       st, a);
}

template <int XF>
void launch_product(GemmArgs& a, const Plan& p, hipStream_t st) {
    if (!p.tiles) {
        if (p.nr == 1) launch_stream<XF, 1>(a, p, st);
        else if (p.nr == 2) launch_stream<XF, 2>(a, p, st);
        else launch_stream<XF, 4>(a, p, st);
    } else if (p.tn == 256) {
        launch_tiles<XF, 256, 256, 2, 4, 3>(a, p, st);
    } else if (p.tn == 128 && p.tt == 64) {
        launch_tiles<XF, 128, 64, 4, 1, 4>(a, p, st);
    } else if (p.tn == 64 && p.tt == 64) {
        launch_tiles<XF, 64, 64, 2, 2, 4>(a, p, st);
    } else {
        launch_tiles<XF, 128, 128, 2, 2, 3>(a, p, st);
    }
}

}  // namespace
}  // namespace lora

using namespace lora;

extern "C" {

int lora_mx_workspace_bytes(const lora_mx_t* x, const lora_mx_t* w, size_t* bytes) {
    if (int rc = check_product(x, w)) return rc;
    if (!bytes) return set_error(LORA_E_ARG, "bytes is NULL");
    *bytes = part_bytes(plan_product(x->n_rows, w->n_rows, (int)mx_blocks(x->h), x->format), x, w);
    return LORA_OK;
}

int lora_mx_apply(const lora_mx_t* x, const lora_mx_t* w, void* y, int64_t ldy, int32_t dtype, void* ws,
                  size_t ws_bytes, void* stream) {
    size_t need = 0;
    if (int rc = lora_mx_workspace_bytes(x, w, &need)) return rc;
    if (dtype != LORA_F16 && dtype != LORA_BF16 && dtype != LORA_F32)
        return set_error(LORA_E_ARG, "dtype must be LORA_F16, LORA_BF16 or LORA_F32");
    if (int rc = check_kv_rows("y", y, "ldy", ldy, w->n_rows, x->n_rows)) return rc;
    if (ldy > (1ll << 40)) return set_error(LORA_E_SHAPE, "ldy exceeds 2^40");
    if (!ws || ws_bytes < need) return set_error(LORA_E_WORKSPACE, "workspace smaller than lora_mx_workspace_bytes");
    if (!is_aligned16(ws)) return set_error(LORA_E_ALIGN, "ws not 16-byte aligned");
    const int64_t e = dtype == LORA_F32 ? 4 : 2;
    const Span out[2] = {Span(y, x->n_rows, ldy * e, w->n_rows * e), Span(ws, 1, 0, (int64_t)need)};
    const Span in[4] = {codes_span(x), scales_span(x), codes_span(w), scales_span(w)};
    for (const Span& o : out)
        for (const Span& i : in)
            if (o.meets(i)) return set_error(LORA_E_OVERLAP, "y or ws overlaps x or w");
    if (out[0].meets(out[1])) return set_error(LORA_E_OVERLAP, "y and ws overlap");
    if (x->n_rows == 0) return LORA_OK;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return set_error(LORA_E_HIP, "lora_mx_apply: no device for the stream");
    GemmArgs a{};
    a.x = (const unsigned char*)x->codes;
    a.xs = (const unsigned char*)x->scales;
    a.w = (const unsigned char*)w->codes;
    a.ws = (const unsigned char*)w->scales;
    a.y = y;                               // (of several launches, each has its own)
    a.part = (float*)ws;
    a.ldx = x->ld_codes;
    a.ldxs = x->ld_scales;
    a.ldw = w->ld_codes;
    a.ldws = w->ld_scales;
    a.ldy = ldy;
    a.n_rows = x->n_rows;
    a.h_out = w->n_rows;
    a.blocks = (int)mx_blocks(x->h);
    a.dtype = dtype;
    const Plan p = plan_product(a.n_rows, a.h_out, a.blocks, x->format);
    a.splits = p.splits;
    a.split_blocks = p.split_blocks;
    // rows and columns of a launch: whole tiles, at most kMostTiles
    const int cols = p.tiles ? (int)std::min<int64_t>(a.h_out, kMostTiles * p.tn) : a.h_out;
    const int rows = p.tiles ? (int)std::min<int64_t>(a.n_rows, kMostTiles / ceil_div(cols, p.tn) * p.tt) : a.n_rows;
    for (int64_t n = 0; n < w->n_rows; n += cols)
        for (int64_t t = 0; t < x->n_rows; t += rows) {
            GemmArgs b = a;
            b.x += t * a.ldx;
            b.xs += t * a.ldxs;
            b.w += n * a.ldw;
            b.ws += n * a.ldws;
            b.y = (char*)y + (t * ldy + n) * e;
            b.n_rows = (int)std::min<int64_t>(rows, a.n_rows - t);
            b.h_out = (int)std::min<int64_t>(cols, a.h_out - n);
            if (x->format == LORA_E4M3) launch_product<LORA_E4M3>(b, p, st);
            else launch_product<LORA_E2M1>(b, p, st);
            if (int rc = check_launch("lora_mx_apply")) return rc;
        }
    if (p.splits == 1) return LORA_OK;
    hipLaunchKernelGGL(lora_mx_join_kernel, dim3(ceil_div((int64_t)a.n_rows * (a.h_out / 4), kJoinThreads)), dim3(kJoinThreads), 0,
                       st, a);
    return check_launch("lora_mx_apply");
}

}  // extern "C"
