// gfx950 kernels of the paged key-value cache (include/lora_kv.h): new rows
// into their pages, and the book of who holds which page.
//
// All of it moves bits: a launch is bound by HBM where it moves pages or many
// rows, and by launch and dependent-load latency where it changes a few
// integers.  The book's single-workgroup kernels (grow, the fork's page
// search, the compaction's numbering) read refs once or twice front to back,
// 8 pages per thread and step, with a running count over the workgroup: page
// numbers are handed out in ascending order, so the result does not depend on
// timing.
#include <stddef.h>

#include <algorithm>
#include <new>
#include <vector>

#include "lora_device.h"
#include "lora_kv_internal.h"

namespace lora {

int check_kv_cache(const lora_kv_cache_t* c) {
    if (!c) return set_error(LORA_E_ARG, "cache is NULL");
    if (c->dtype != LORA_F16 && c->dtype != LORA_BF16) return set_error(LORA_E_ARG, "dtype must be LORA_F16 or LORA_BF16");
    if (c->n_layers < 1 || c->n_pages < 0 || c->n_kv_heads < 1)
        return set_error(LORA_E_ARG, "cache needs n_layers >= 1, n_pages >= 0 and n_kv_heads >= 1");
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8)
        return set_error(LORA_E_SHAPE, "head_dim must be a multiple of 8 in [8, 256]");
    if (c->page_rows < 16 || c->page_rows > 65536 || (c->page_rows & (c->page_rows - 1)))
        return set_error(LORA_E_SHAPE, "page_rows must be a power of two in [16, 65536]");
    const int64_t st[4] = {c->layer_stride, c->page_stride, c->head_stride, c->row_stride};
    const int64_t n[4] = {c->n_layers, c->n_pages, c->n_kv_heads, c->page_rows};
    for (int i = 0; i < 4; ++i) {
        if (st[i] % 8 || st[i] < 0) return set_error(LORA_E_SHAPE, "cache strides must be multiples of 8, not negative");
        if (n[i] > 1 && st[i] < c->head_dim) return set_error(LORA_E_SHAPE, "cache strides must be at least head_dim");
    }
    // (an offset in elements stays far below 2^63)
    double span = 0;
    for (int i = 0; i < 4; ++i) span += (double)n[i] * (double)st[i];
    if (span > 1e15) return set_error(LORA_E_SHAPE, "the cache's strides span more than 10^15 elements");
    if ((c->page_rows * c->row_stride + c->head_dim) * 2 > (int64_t)kMaxSpan)
        return set_error(LORA_E_SHAPE, "a page's rows of one head span more than 2 GiB");
    if (c->n_pages > 0 && (!c->k || !c->v)) return set_error(LORA_E_ARG, "k or v is NULL");
    if (!is_aligned16(c->k) || !is_aligned16(c->v)) return set_error(LORA_E_ALIGN, "k or v not 16-byte aligned");
    return LORA_OK;
}

int check_kv_layer(const lora_kv_cache_t* c, int32_t layer) {
    if (layer < 0 || layer >= c->n_layers)
        return set_error(LORA_E_INDEX, "layer " + std::to_string(layer) + " of " + std::to_string(c->n_layers));
    return LORA_OK;
}

int check_kv_seqs(const lora_kv_cache_t* c, const lora_kv_seqs_t* s) {
    if (!s) return set_error(LORA_E_ARG, "sequences are NULL");
    if (s->n_seqs < 0 || s->ld_table < 0 || s->max_len < 0)
        return set_error(LORA_E_ARG, "negative n_seqs, ld_table or max_len");
    if (s->n_seqs > 0 && (!s->lens || (s->ld_table > 0 && !s->tables)))
        return set_error(LORA_E_ARG, "tables or lens is NULL");
    if ((int64_t)s->max_len > (int64_t)s->ld_table * c->page_rows)
        return set_error(LORA_E_SHAPE, "max_len exceeds ld_table * page_rows");
    if (s->max_len > (1 << 30)) return set_error(LORA_E_SHAPE, "max_len exceeds 2^30");
    if (((uintptr_t)s->lens | (uintptr_t)s->tables) & 3) return set_error(LORA_E_ALIGN, "tables or lens not 4-byte aligned");
    return LORA_OK;
}

int check_kv_rows(const char* name, const void* p, const char* ld_name, int64_t ld, int64_t h, int32_t n_rows) {
    if (ld < h || ld % 8)
        return set_error(LORA_E_SHAPE, std::string(ld_name) + " must be a multiple of 8 and >= " + std::to_string(h));
    if (n_rows > 0 && !p) return set_error(LORA_E_ARG, std::string(name) + " is NULL");
    if (!is_aligned16(p)) return set_error(LORA_E_ALIGN, std::string(name) + " not 16-byte aligned");
    return LORA_OK;
}

int check_launch(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(LORA_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
    return LORA_OK;
}

}  // namespace lora

using namespace lora;

namespace {

constexpr int kCopyThreads = 256;
constexpr int kBookThreads = 1024;
constexpr int kBookPages = 8;              // pages per thread and step of a scan of refs
constexpr int kArgIds = 480;               // ids (or 240 pairs) that one launch carries in its arguments

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------

struct AppendArgs {
    uint16_t *k, *v;                       // the layer's
    const uint16_t *k_new, *v_new;
    const int32_t *tables, *lens, *seg_offset;
    int64_t page_stride, head_stride, row_stride, ldk, ldv;
    int32_t n_rows, n_seqs, ld_table, max_len, n_pages;
    int32_t page_shift, row_chunks, dim_chunks;   // 16-byte chunks of a row, of one head's part of it
    int32_t group_rows;                    // rows per workgroup
};

// A workgroup finds where each of its rows goes (one thread per row: a binary
// search of the offsets, the length, the table entry), then all threads move
// the rows' 16-byte chunks.  Bound by HBM for the rows of prompts (7812 rows of
// 32 heads of 128: 256 MB read and written in 52 us, 4.9 TB/s), by the chain offset,
// length, table, row for single tokens (256 rows: 3 us, less than the launch costs
// the host).
constexpr int kAppendRows = 64;

__global__ void __launch_bounds__(kCopyThreads) lora_kv_append_kernel(AppendArgs a) {
    __shared__ int64_t at[kAppendRows];
    const int t = threadIdx.x;
    const int row0 = blockIdx.x * a.group_rows;
    const int rows = min(a.group_rows, a.n_rows - row0);
    if (t < rows) {
        const int row = row0 + t;
        int s = row, n = 1, i = 0;
        if (a.seg_offset) {
            int lo = 0, hi = a.n_seqs;     // the first segment that ends past the row
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (a.seg_offset[mid + 1] > row) hi = mid;
                else lo = mid + 1;
            }
            s = lo;
            if (s < a.n_seqs) {
                const int first = a.seg_offset[s];
                n = min(a.seg_offset[s + 1], a.n_rows) - first;
                i = row - first;
                if (first < 0 || i < 0) s = a.n_seqs;
            }
        }
        int64_t to = -1;
        if (s < a.n_seqs) {
            const int pos = kv_len(a.lens, s, a.max_len) - n + i;   // max_len keeps it inside the table
            if (pos >= 0) {
                const int page = a.tables[(int64_t)s * a.ld_table + (pos >> a.page_shift)];
                if ((uint32_t)page < (uint32_t)a.n_pages)
                    to = page * a.page_stride + (pos & ((1 << a.page_shift) - 1)) * a.row_stride;
            }
        }
        at[t] = to;
    }
    __syncthreads();
    const int n = rows * a.row_chunks;
    for (int i = t; i < n; i += kCopyThreads) {
        const int r = i / a.row_chunks, c = i - r * a.row_chunks;
        const int h = c / a.dim_chunks, e = c - h * a.dim_chunks;
        const int64_t to = at[r];
        if (to < 0) continue;
        const u32x4 kw = *(const u32x4*)(a.k_new + (int64_t)(row0 + r) * a.ldk + 8 * c);
        const u32x4 vw = *(const u32x4*)(a.v_new + (int64_t)(row0 + r) * a.ldv + 8 * c);
        const int64_t o = to + h * a.head_stride + 8 * e;
        *(u32x4*)(a.k + o) = kw;
        *(u32x4*)(a.v + o) = vw;
    }
}

// ---------------------------------------------------------------------------
// page copies
// ---------------------------------------------------------------------------

// Bound by HBM: a compaction that moves 257 MB reads and writes at 4.9 TB/s (105 us), and so does a copy of 240 pages
// (251 MB, 102 us).  A
// workgroup moves 32 KiB at a time, all of it in flight, so a few pages fill the chip.
struct PageDims {
    uint16_t *k, *v;
    int64_t layer_stride, page_stride, head_stride, row_stride;
    int32_t n_layers, n_kv_heads, page_rows, dim_chunks;
    int32_t row_inner;                     // rows of a head lie closer together than heads of a row
    int32_t blocks;                        // parts of kPartChunks chunks of a whole page
};

constexpr int kPartChunks = 2048;          // 32 KiB of k or v: one step of a workgroup, 8 loads in flight per thread

// Part `part` of the first `rows` rows of page src to page dst, in one layer of k or v.
__device__ __forceinline__ void copy_part(const PageDims& d, uint16_t* base, int src, int dst, int rows, int part) {
    const int n = d.n_kv_heads * rows * d.dim_chunks;
    const uint16_t* from = base + src * d.page_stride;
    uint16_t* to = base + dst * d.page_stride;
    u32x4 w[kPartChunks / kCopyThreads];
    int64_t o[kPartChunks / kCopyThreads];
#pragma unroll
    for (int i = 0; i < kPartChunks / kCopyThreads; ++i) {
        const int c = part * kPartChunks + i * kCopyThreads + (int)threadIdx.x;
        o[i] = -1;
        if (c < n) {
            const int x = c / d.dim_chunks, e = c - x * d.dim_chunks;
            const int m = d.row_inner ? rows : d.n_kv_heads;
            const int hi = x / m, lo = x - hi * m;
            const int h = d.row_inner ? hi : lo, r = d.row_inner ? lo : hi;
            o[i] = h * d.head_stride + r * d.row_stride + 8 * e;
            w[i] = *(const u32x4*)(from + o[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kPartChunks / kCopyThreads; ++i)
        if (o[i] >= 0) *(u32x4*)(to + o[i]) = w[i];
}

// Unit u of a page's copy: its part, then k or v, then the layer.
__device__ __forceinline__ void copy_unit(const PageDims& d, int u, int src, int dst, int rows) {
    const int part = u % d.blocks, kv = (u / d.blocks) & 1, layer = u / (2 * d.blocks);
    copy_part(d, (kv ? d.v : d.k) + layer * d.layer_stride, src, dst, rows, part);
}

struct IdArgs {
    int32_t id[kArgIds];
};

// Pairs (src, dst) in the arguments: workgroup (x, y) runs unit x of pair y.
__global__ void __launch_bounds__(kCopyThreads) lora_kv_copy_kernel(PageDims d, IdArgs ids) {
    const int src = ids.id[2 * blockIdx.y], dst = ids.id[2 * blockIdx.y + 1];
    copy_unit(d, blockIdx.x, src, dst, d.page_rows);
}

// ---------------------------------------------------------------------------
// the book
// ---------------------------------------------------------------------------

struct Book {
    int32_t *tables, *lens, *refs;
    int32_t n_seqs, ld_table, n_pages, page_shift;
};

// Table entries that a sequence of len tokens holds.
__device__ __forceinline__ int held(const Book& b, int len) {
    if (len <= 0) return 0;
    const int n = (int)(((int64_t)len + (1 << b.page_shift) - 1) >> b.page_shift);
    return min(n, b.ld_table);
}
__device__ __forceinline__ bool is_page(const Book& b, int p) { return (uint32_t)p < (uint32_t)b.n_pages; }

// Exclusive sum of v over the workgroup's threads in order; total gets the sum.
__device__ __forceinline__ int block_scan(int v, int* wave_sum, int& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int o = __shfl_up(s, i, 64);
        if (lane >= i) s += o;
    }
    __syncthreads();                       // wave_sum of the last call has been read
    if (lane == 63) wave_sum[w] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kBookThreads / 64; ++i) {
        const int x = wave_sum[i];
        before += i < w ? x : 0;
        all += x;
    }
    total = all;
    return before + s - v;
}

// refs of this thread's pages of a step; pages past the last read as in use.
__device__ __forceinline__ int thread_pages(const Book& b, int step, int (&r)[kBookPages]) {
    const int p0 = (step * kBookThreads + (int)threadIdx.x) * kBookPages;
#pragma unroll
    for (int i = 0; i < kBookPages; ++i) r[i] = p0 + i < b.n_pages ? b.refs[p0 + i] : 1;
    return p0;
}

// The first `want` free pages in ascending order into list; returns how many there are of them.
__device__ int find_free(const Book& b, int want, int32_t* list, int* wave_sum) {
    int found = 0;
    for (int step = 0; found < want && (int64_t)step * kBookThreads * kBookPages < b.n_pages; ++step) {
        int r[kBookPages];
        const int p0 = thread_pages(b, step, r);
        int n = 0, total;
#pragma unroll
        for (int i = 0; i < kBookPages; ++i) n += r[i] == 0;
        int at = found + block_scan(n, wave_sum, total);
#pragma unroll
        for (int i = 0; i < kBookPages; ++i)
            if (r[i] == 0) {
                if (at < want) list[at] = p0 + i;
                ++at;
            }
        found += total;
    }
    __syncthreads();                       // the list, written by other threads, can be read
    return min(found, want);
}

// Workspace: int32 words.  [0, n_pages) and [n_pages, 2 n_pages): page lists;
// [2 n_pages, 3 n_pages): the compaction's numbering; then n_seqs running
// sums (a fork's pages by pair: its children are distinct, so at most n_seqs), and two counters.
struct BookWs {
    int32_t *list, *list2, *map, *sums, *count;
};

__host__ __device__ inline BookWs book_ws(void* ws, int n_pages, int n_seqs) {
    int32_t* w = (int32_t*)ws;
    return {w, w + n_pages, w + 2 * (int64_t)n_pages, w + 3 * (int64_t)n_pages, w + 3 * (int64_t)n_pages + n_seqs};
}

// One workgroup: the counts of 1024 sequences at a time in a scan, the free pages in another.  Bound by latency:
// 3.2 us where no sequence needs a page, 6.2 for 24 and 14 for 256 that all need one. The scan of free pages reads
// the counts from the first page on until there are enough, so a cache that is full to the last
// pages costs more: 111 us with 199680 of 200000 in use.
// No length passes room; step_lens may be NULL.
__global__ void __launch_bounds__(kBookThreads) lora_kv_grow_kernel(Book b, const int32_t* add, int64_t room,
                                                                    int32_t* step_lens, int32_t* info, BookWs w) {
    __shared__ int wave_sum[kBookThreads / 64];
    __shared__ int stayed;
    const int t = threadIdx.x;
    if (t == 0) stayed = 0;
    // pages wanted by the sequences up to and including each, those too long for their table left out
    auto wanted = [&](int s, int& len, int& to) {
        len = max(b.lens[s], 0);
        const int64_t sum = (int64_t)len + max(add[s], 0);
        if (sum > room || sum > 0x7fffffff) {
            to = -1;
            return 0;
        }
        to = (int)sum;
        return held(b, to) - held(b, len);
    };
    int total = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += kBookThreads) {
        const int s = s0 + t;
        int len, to, sum;
        const int n = s < b.n_seqs ? wanted(s, len, to) : 0;
        const int before = block_scan(n, wave_sum, sum);
        // (sums saturate: the pages of all tables together may pass 32 bits)
        if (s < b.n_seqs) w.sums[s] = (int)min((int64_t)total + before + n, (int64_t)0x7fffffff);
        total = (int)min((int64_t)total + sum, (int64_t)0x7fffffff);
    }
    const int found = find_free(b, min(total, b.n_pages), w.list, wave_sum);
    // the sequences that fit: sums up to `found`
    __syncthreads();
    int taken = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += kBookThreads) {
        const int s = s0 + t;
        int n = 0, sum;
        if (s < b.n_seqs) {
            int len, to;
            n = wanted(s, len, to);
            const bool stays = to < 0 || (n > 0 && w.sums[s] > found);
            if (stays) {
                n = 0;
                atomicAdd(&stayed, 1);
            }
        }
        block_scan(n, wave_sum, sum);
        taken += sum;
    }
    // page i goes to the sequence whose running sum first passes i
    for (int i = t; i < taken; i += kBookThreads) {
        int lo = 0, hi = b.n_seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (w.sums[mid] > i) hi = mid;
            else lo = mid + 1;
        }
        int len, to;
        const int n = wanted(lo, len, to);
        const int page = w.list[i];
        b.tables[(int64_t)lo * b.ld_table + held(b, len) + i - (w.sums[lo] - n)] = page;
        b.refs[page] = 1;
    }
    __syncthreads();
    for (int s = t; s < b.n_seqs; s += kBookThreads) {
        int len, to;
        const int n = wanted(s, len, to);
        const bool grows = to >= 0 && (n == 0 || w.sums[s] <= found);
        if (grows) b.lens[s] = to;
        // (a sequence that got nothing has no row in the step: stored at its length's end, it
        // would go over the last token, which others may share)
        if (step_lens) step_lens[s] = grows && to > len ? to : 0;
    }
    if (info && t == 0) {
        info[0] = taken;
        info[1] = stayed;
    }
}

// Sequence ids in the arguments give their pages back: one workgroup each, which
// leaves length 0 and entries -1 (48 sequences of 60 to 800 pages: 3.2 to 4.2 us).  (stride 2, first 1: the children of pairs; step_lens may be NULL)
__global__ void __launch_bounds__(kCopyThreads) lora_kv_release_kernel(Book b, IdArgs ids, int stride, int first,
                                                                       int32_t* step_lens) {
    const int s = ids.id[blockIdx.x * stride + first];
    const int n = held(b, b.lens[s]);
    int32_t* table = b.tables + (int64_t)s * b.ld_table;
    for (int e = threadIdx.x; e < b.ld_table; e += kCopyThreads) {
        const int p = table[e];
        if (e < n && is_page(b, p)) atomicSub(b.refs + p, 1);
        table[e] = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        b.lens[s] = 0;
        // (rows that a child had in a step under way would land in pages that it shares from here on)
        if (step_lens) step_lens[s] = 0;
    }
}

// One workgroup per sequence (256 sequences of 60 to 800 pages: 3 to 5 us), in strides where a grid's threads
// would pass 32 bits.
constexpr int kTrimBlocks = 1 << 20;

__global__ void __launch_bounds__(kCopyThreads) lora_kv_trim_kernel(Book b, int32_t window, int32_t n_sinks) {
    for (int64_t s = blockIdx.x; s < b.n_seqs; s += gridDim.x) {
        const int len = b.lens[s];
        const int n = held(b, len);
        int32_t* table = b.tables + s * b.ld_table;
        for (int e = threadIdx.x; e < n; e += kCopyThreads) {
            const int64_t first = (int64_t)e << b.page_shift, last = first + (1 << b.page_shift) - 1;
            // the row at position len sees tokens from len + 1 - window on; later rows later ones
            if (last > (int64_t)len - window || first < n_sinks) continue;
            const int p = table[e];
            if (is_page(b, p)) atomicSub(b.refs + p, 1);
            table[e] = -1;
        }
    }
}

// Does a child of this parent need a page of its own, and which is copied into it?
__device__ __forceinline__ bool fork_tail(const Book& b, int parent, int& len, int& src) {
    len = max(b.lens[parent], 0);
    const int e = len >> b.page_shift;
    src = -1;
    if (!(len & ((1 << b.page_shift) - 1)) || e >= b.ld_table) return false;
    src = b.tables[(int64_t)parent * b.ld_table + e];
    return is_page(b, src);
}

// A fork is three launches: the children's pages come back, the new ones are found, tables
// and rows are copied (48 children: 3.2 + 5.2 + 12.3 us, 62 MB).  With the first two
// in one it took longer (22.8 against 19.6 us): one workgroup then releases what 48 did.
//
// The pages of n children: sums[i] gets pair i's, or -1 where it needs none, or -2 where none is left.
struct ForkArgs {
    Book book;
    BookWs w;
    int32_t* info;
    int32_t n, first;
    IdArgs pairs;
};
__global__ void __launch_bounds__(kBookThreads) lora_kv_fork_pages_kernel(ForkArgs a) {
    __shared__ int wave_sum[kBookThreads / 64];
    // read through the argument segment: a lane-dependent index into the
    // parameter would copy it to private memory
    const int32_t* ids = (const int32_t*)((const unsigned char*)__builtin_amdgcn_kernarg_segment_ptr() +
                                          offsetof(ForkArgs, pairs));
    const Book& b = a.book;
    const BookWs& w = a.w;
    const int t = threadIdx.x, n = a.n, first = a.first;
    int32_t* info = a.info;
    int len, src, want = 0;
    const bool need = t < n && fork_tail(b, ids[2 * t], len, src);
    const int at = block_scan(need ? 1 : 0, wave_sum, want);
    const int found = find_free(b, want, w.list, wave_sum);
    if (t < n) {
        const int page = !need ? -1 : at < found ? w.list[at] : -2;
        w.sums[t] = page;
        if (page >= 0) b.refs[page] = 1;
    }
    if (info && t == 0) {
        info[0] = (first ? 0 : info[0]) + found;
        info[1] = (first ? 0 : info[1]) + want - found;
    }
}

// Workgroups y < n: row y of the children's tables and lengths (x == 0), and unit x of
// the copy of its last page's rows.
__global__ void __launch_bounds__(kCopyThreads) lora_kv_fork_kernel(Book b, PageDims d, IdArgs ids, BookWs w) {
    const int pair = blockIdx.y;
    const int parent = ids.id[2 * pair], child = ids.id[2 * pair + 1];
    const int fresh = w.sums[pair];
    if (fresh == -2) return;               // the child is empty already
    int len, src;
    fork_tail(b, parent, len, src);
    if (blockIdx.x == 0) {
        const int32_t* from = b.tables + (int64_t)parent * b.ld_table;
        int32_t* to = b.tables + (int64_t)child * b.ld_table;
        const int full = min(len >> b.page_shift, b.ld_table);
        for (int e = threadIdx.x; e < b.ld_table; e += kCopyThreads) {
            int p = e < full ? from[e] : -1;
            if (!is_page(b, p)) p = -1;
            if (p >= 0) atomicAdd(b.refs + p, 1);
            if (e == full && fresh >= 0) p = fresh;
            to[e] = p;
        }
        if (threadIdx.x == 0) b.lens[child] = len;
    } else if (fresh >= 0) {
        copy_unit(d, blockIdx.x - 1, src, fresh, len & ((1 << b.page_shift) - 1));
    }
}

// Numbers the pages in use: map[p] is p's new id for p < L (-1 where it is free), L + i for the
// i-th one in use from L on; list[i] and list2[i] are its old and new id.
__global__ void __launch_bounds__(kBookThreads) lora_kv_number_kernel(Book b, int32_t* info, BookWs w) {
    __shared__ int wave_sum[kBookThreads / 64];
    const int per_step = kBookThreads * kBookPages;
    const int steps = (b.n_pages + per_step - 1) / per_step;
    int live = 0;
    for (int step = 0; step < steps; ++step) {
        int r[kBookPages];
        const int p0 = thread_pages(b, step, r);
#pragma unroll
        for (int i = 0; i < kBookPages; ++i) live += p0 + i < b.n_pages && r[i] != 0;
    }
    int L, moved = 0, holes = 0;
    block_scan(live, wave_sum, L);
    for (int step = 0; step < steps; ++step) {
        int r[kBookPages];
        const int p0 = thread_pages(b, step, r);
        int m = 0, h = 0, sum;
#pragma unroll
        for (int i = 0; i < kBookPages; ++i) {
            const int p = p0 + i;
            h += p < L && r[i] == 0;
            m += p >= L && p < b.n_pages && r[i] != 0;
        }
        const int before = block_scan(h | m << 16, wave_sum, sum);   // at most 8192 of either in a step
        int hi = holes + (before & 0xffff), mi = moved + (before >> 16);
#pragma unroll
        for (int i = 0; i < kBookPages; ++i) {
            const int p = p0 + i;
            if (p >= b.n_pages) continue;
            int to = -1;
            if (p < L) {
                if (r[i] == 0) w.list2[hi++] = p;
                else to = p;
            } else if (r[i] != 0) {
                to = L + mi;
                w.list[mi++] = p;
            }
            w.map[p] = to;
        }
        holes += sum & 0xffff;
        moved += sum >> 16;
    }
    if (threadIdx.x == 0) {
        w.count[0] = L;
        w.count[1] = moved;
        if (info) {
            info[0] = L;
            info[1] = moved;
        }
    }
    __syncthreads();
    // the moved pages' counts, before the next launch writes over them: behind the moved pages in list
    // (they are at most half of all)
    for (int i = threadIdx.x; i < moved; i += kBookThreads) w.list[moved + i] = b.refs[w.list[i]];
}

// The first `book_blocks` workgroups write the tables and counts for the new ids, the others move pages.
__global__ void __launch_bounds__(kCopyThreads) lora_kv_move_kernel(Book b, PageDims d, int32_t* tables_out,
                                                                    int32_t* refs_out, BookWs w, int book_blocks) {
    const int L = w.count[0], moved = w.count[1];
    if ((int)blockIdx.x < book_blocks) {
        const int64_t entries = (int64_t)b.n_seqs * b.ld_table;
        const int64_t stride = (int64_t)book_blocks * kCopyThreads;
        for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += stride) {
            const int s = (int)(i / b.ld_table), e = (int)(i - (int64_t)s * b.ld_table);
            const int p = b.tables[i];
            int to = -1;
            if (e < held(b, b.lens[s]) && is_page(b, p)) {
                to = w.map[p];
                if (to >= L) to = w.list2[to - L];
            }
            tables_out[i] = to;
        }
        for (int64_t p = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; p < b.n_pages; p += stride) {
            if (p >= L) refs_out[p] = 0;
            else if (w.map[p] >= 0) refs_out[p] = b.refs[p];
        }
        for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < moved; i += stride)
            refs_out[w.list2[i]] = w.list[moved + i];
        return;
    }
    const int units = 2 * d.n_layers * d.blocks;
    const int64_t n = (int64_t)moved * units;
    for (int64_t u = (int)blockIdx.x - book_blocks; u < n; u += gridDim.x - book_blocks) {
        const int i = (int)(u / units);
        copy_unit(d, (int)(u - (int64_t)i * units), w.list[i], w.list2[i], d.page_rows);
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

int log2_of(int v) {
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}

int check_book(const lora_kv_book_t* b) {
    if (!b) return set_error(LORA_E_ARG, "book is NULL");
    if (b->n_seqs < 0 || b->ld_table < 0 || b->n_pages < 0)
        return set_error(LORA_E_ARG, "negative n_seqs, ld_table or n_pages");
    if ((int64_t)b->n_seqs * b->ld_table > 0x7fffffff)   // (the page counts of a book add up in 32 bits)
        return set_error(LORA_E_SHAPE, "the book's tables have 2^31 entries or more");
    if (b->n_pages > (1 << 30)) return set_error(LORA_E_SHAPE, "n_pages exceeds 2^30");
    if (b->page_rows < 16 || b->page_rows > 65536 || (b->page_rows & (b->page_rows - 1)))
        return set_error(LORA_E_SHAPE, "page_rows must be a power of two in [16, 65536]");
    if ((b->n_seqs > 0 && (!b->lens || (b->ld_table > 0 && !b->tables))) || (b->n_pages > 0 && !b->refs))
        return set_error(LORA_E_ARG, "tables, lens or refs is NULL");
    if (((uintptr_t)b->lens | (uintptr_t)b->tables | (uintptr_t)b->refs) & 3)
        return set_error(LORA_E_ALIGN, "tables, lens or refs not 4-byte aligned");
    return LORA_OK;
}

int check_book_cache(const lora_kv_cache_t* c, const lora_kv_book_t* b) {
    if (c->page_rows != b->page_rows || c->n_pages != b->n_pages)
        return set_error(LORA_E_SHAPE, "cache and book differ in page_rows or n_pages");
    return LORA_OK;
}

size_t ws_bytes_of(const lora_kv_book_t* b) { return 4 * (3 * (size_t)b->n_pages + (size_t)b->n_seqs + 2); }

int check_ws(const lora_kv_book_t* b, const void* ws, size_t bytes) {
    if (!ws) return set_error(LORA_E_ARG, "workspace is NULL");
    if (!is_aligned16(ws)) return set_error(LORA_E_ALIGN, "workspace not 16-byte aligned");
    if (bytes < ws_bytes_of(b))
        return set_error(LORA_E_WORKSPACE, "workspace has " + std::to_string(bytes) + " bytes, needs " +
                                               std::to_string(ws_bytes_of(b)));
    return LORA_OK;
}

// Ids in [0, n_ids), no two alike; mark gets 1 for each.
int check_ids(const char* what, const int32_t* ids, int32_t n, int32_t n_ids, std::vector<uint8_t>& mark) {
    for (int32_t i = 0; i < n; ++i) {
        if (ids[i] < 0 || ids[i] >= n_ids)
            return set_error(LORA_E_INDEX, std::string(what) + " " + std::to_string(ids[i]) + " of " + std::to_string(n_ids));
        if (mark[ids[i]]) return set_error(LORA_E_ARG, std::string(what) + " " + std::to_string(ids[i]) + " is given twice");
        mark[ids[i]] = 1;
    }
    return LORA_OK;
}

// from[] in [0, n_ids) and to[] too, the latter distinct and none of the former.
int check_pairs(const char* from_name, const char* to_name, const int32_t* from, const int32_t* to, int32_t n,
                int32_t n_ids) {
    if (n < 0) return set_error(LORA_E_ARG, "negative count");
    if (n > 0 && (!from || !to)) return set_error(LORA_E_ARG, std::string(from_name) + " or " + to_name + " array is NULL");
    try {
        std::vector<uint8_t> mark((size_t)n_ids, 0);
        if (int rc = check_ids(to_name, to, n, n_ids, mark)) return rc;
        for (int32_t i = 0; i < n; ++i) {
            if (from[i] < 0 || from[i] >= n_ids)
                return set_error(LORA_E_INDEX, std::string(from_name) + " " + std::to_string(from[i]) + " of " +
                                                   std::to_string(n_ids));
            if (mark[from[i]])
                return set_error(LORA_E_ARG, std::string(from_name) + " " + std::to_string(from[i]) + " is also a " + to_name);
        }
    } catch (const std::bad_alloc&) {
        return set_error(LORA_E_NOMEM, "host memory for the argument check");
    }
    return LORA_OK;
}

int check_words(const char* what, const void* p) {
    if ((uintptr_t)p & 3) return set_error(LORA_E_ALIGN, std::string(what) + " not 4-byte aligned");
    return LORA_OK;
}

Book device_book(const lora_kv_book_t* b) {
    return {b->tables, b->lens, b->refs, b->n_seqs, b->ld_table, b->n_pages, log2_of(b->page_rows)};
}

PageDims page_dims(const lora_kv_cache_t* c) {
    PageDims d;
    d.k = (uint16_t*)c->k;
    d.v = (uint16_t*)c->v;
    d.layer_stride = c->layer_stride;
    d.page_stride = c->page_stride;
    d.head_stride = c->head_stride;
    d.row_stride = c->row_stride;
    d.n_layers = c->n_layers;
    d.n_kv_heads = c->n_kv_heads;
    d.page_rows = c->page_rows;
    d.dim_chunks = c->head_dim / 8;
    d.row_inner = c->row_stride <= c->head_stride;
    d.blocks = (int)(((int64_t)c->n_kv_heads * c->page_rows * d.dim_chunks + kPartChunks - 1) / kPartChunks);
    return d;
}

// One page's chunks fit 31 bits, the threads that copy one page 32.
int check_page_size(const lora_kv_cache_t* c) {
    const int64_t chunks = (int64_t)c->n_kv_heads * c->page_rows * (c->head_dim / 8);
    if (chunks > 0x3fffffff || ((chunks + kPartChunks - 1) / kPartChunks) * 2 * c->n_layers > 0x7fffff)
        return set_error(LORA_E_SHAPE, "a page of all layers holds more than 256 GiB");
    return LORA_OK;
}

int no_device(const char* what) { return set_error(LORA_E_HIP, std::string(what) + ": cannot select the stream's device"); }

// step_lens of a step's calls: an array of its own beside the book's lengths.
int check_step_lens(const lora_kv_book_t* b, const int32_t* step_lens) {
    if (b->n_seqs > 0 && !step_lens) return set_error(LORA_E_ARG, "step_lens is NULL");
    if (int rc = check_words("step_lens", step_lens)) return rc;
    const uintptr_t x = (uintptr_t)step_lens, y = (uintptr_t)b->lens, n = 4 * (uintptr_t)b->n_seqs;
    if (x < y + n && y < x + n) return set_error(LORA_E_OVERLAP, "step_lens and lens overlap");
    return LORA_OK;
}

int enqueue_grow(const char* name, const lora_kv_book_t* b, const int32_t* add, int64_t room, int32_t* step_lens,
                 int32_t* info, void* ws, size_t ws_bytes, void* stream) {
    if (b->n_seqs > 0 && !add) return set_error(LORA_E_ARG, "add is NULL");
    if (int rc = check_words("add", add)) return rc;
    if (int rc = check_words("info", info)) return rc;
    if (int rc = check_ws(b, ws, ws_bytes)) return rc;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device(name);
    hipLaunchKernelGGL(lora_kv_grow_kernel, dim3(1), dim3(kBookThreads), 0, st, device_book(b), add, room, step_lens,
                       info, book_ws(ws, b->n_pages, b->n_seqs));
    return check_launch(name);
}

int enqueue_fork(const char* name, const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t n, const int32_t* parents,
                 const int32_t* children, int32_t* step_lens, int32_t* info, void* ws, size_t ws_bytes, void* stream) {
    if (int rc = check_kv_cache(c)) return rc;
    if (int rc = check_page_size(c)) return rc;
    if (int rc = check_book(b)) return rc;
    if (int rc = check_book_cache(c, b)) return rc;
    if (int rc = check_pairs("parent", "child", parents, children, n, b->n_seqs)) return rc;
    if (int rc = check_words("info", info)) return rc;
    if (int rc = check_ws(b, ws, ws_bytes)) return rc;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device(name);
    const Book book = device_book(b);
    const PageDims d = page_dims(c);
    const BookWs w = book_ws(ws, b->n_pages, b->n_seqs);
    constexpr int kPairs = kArgIds / 2;
    static_assert(kPairs <= kBookThreads, "one thread per pair");
    const int units = 2 * d.n_layers * d.blocks;
    IdArgs ids{};
    // every child's pages come back before any is handed out
    for (int pass = 0; pass < 2; ++pass)
        for (int32_t i0 = 0; i0 < n || (pass && n == 0 && i0 == 0); i0 += kPairs) {
            const int m = std::min(kPairs, n - i0);
            for (int i = 0; i < m; ++i) {
                ids.id[2 * i] = parents[i0 + i];
                ids.id[2 * i + 1] = children[i0 + i];
            }
            if (pass == 0) {
                hipLaunchKernelGGL(lora_kv_release_kernel, dim3(m), dim3(kCopyThreads), 0, st, book, ids, 2, 1, step_lens);
            } else {
                hipLaunchKernelGGL(lora_kv_fork_pages_kernel, dim3(1), dim3(kBookThreads), 0, st,
                                   ForkArgs{book, w, info, m, (int)(i0 == 0), ids});
                if (m > 0)
                    hipLaunchKernelGGL(lora_kv_fork_kernel, dim3(1 + units, m), dim3(kCopyThreads), 0, st, book, d, ids, w);
            }
            if (int rc = check_launch(name)) return rc;
        }
    return LORA_OK;
}

}  // namespace

extern "C" {

int lora_kv_append(const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, const int32_t* seg_offset,
                   int32_t n_rows, const void* k_new, int64_t ldk, const void* v_new, int64_t ldv, void* stream) {
    if (int rc = check_kv_cache(c)) return rc;
    if (int rc = check_kv_layer(c, layer)) return rc;
    if (int rc = check_kv_seqs(c, s)) return rc;
    if (n_rows < 0) return set_error(LORA_E_ARG, "negative n_rows");
    if (!seg_offset && n_rows != s->n_seqs)
        return set_error(LORA_E_SHAPE, "without seg_offset, n_rows must be n_seqs");
    if (int rc = check_words("seg_offset", seg_offset)) return rc;
    const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
    if (int rc = check_kv_rows("k_new", k_new, "ldk", ldk, width, n_rows)) return rc;
    if (int rc = check_kv_rows("v_new", v_new, "ldv", ldv, width, n_rows)) return rc;
    if (width > (1 << 24)) return set_error(LORA_E_SHAPE, "n_kv_heads * head_dim exceeds 2^24");
    if (n_rows == 0 || s->n_seqs == 0 || c->n_pages == 0) return LORA_OK;
    // rows of a workgroup: two chunks per thread
    const int group_rows = std::max(1, std::min(kAppendRows, 2 * kCopyThreads / (int)(width / 8)));
    const int64_t blocks = ((int64_t)n_rows + group_rows - 1) / group_rows;
    if (blocks > 0xffffff) return set_error(LORA_E_SHAPE, "lora_kv_append: too many rows");
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device("lora_kv_append");
    AppendArgs a;
    a.k = (uint16_t*)c->k + layer * c->layer_stride;
    a.v = (uint16_t*)c->v + layer * c->layer_stride;
    a.k_new = (const uint16_t*)k_new;
    a.v_new = (const uint16_t*)v_new;
    a.tables = s->tables;
    a.lens = s->lens;
    a.seg_offset = seg_offset;
    a.page_stride = c->page_stride;
    a.head_stride = c->head_stride;
    a.row_stride = c->row_stride;
    a.ldk = ldk;
    a.ldv = ldv;
    a.n_rows = n_rows;
    a.n_seqs = s->n_seqs;
    a.ld_table = s->ld_table;
    a.max_len = s->max_len;
    a.n_pages = c->n_pages;
    a.page_shift = log2_of(c->page_rows);
    a.row_chunks = (int)(width / 8);
    a.dim_chunks = c->head_dim / 8;
    a.group_rows = group_rows;
    hipLaunchKernelGGL(lora_kv_append_kernel, dim3((unsigned)blocks), dim3(kCopyThreads), 0, st, a);
    return check_launch("lora_kv_append");
}

int lora_kv_workspace_bytes(const lora_kv_book_t* b, size_t* bytes) {
    if (int rc = check_book(b)) return rc;
    if (!bytes) return set_error(LORA_E_ARG, "bytes is NULL");
    *bytes = ws_bytes_of(b);
    return LORA_OK;
}

int lora_kv_grow(const lora_kv_book_t* b, const int32_t* add, int32_t* info, void* ws, size_t ws_bytes, void* stream) {
    if (int rc = check_book(b)) return rc;
    return enqueue_grow("lora_kv_grow", b, add, (int64_t)b->ld_table * b->page_rows, nullptr, info, ws, ws_bytes, stream);
}

int lora_kv_grow_step(const lora_kv_book_t* b, const int32_t* add, int32_t max_len, int32_t* step_lens, int32_t* info,
                      void* ws, size_t ws_bytes, void* stream) {
    if (int rc = check_book(b)) return rc;
    if (max_len < 0) return set_error(LORA_E_ARG, "negative max_len");
    if ((int64_t)max_len > (int64_t)b->ld_table * b->page_rows)
        return set_error(LORA_E_SHAPE, "max_len exceeds ld_table * page_rows");
    if (int rc = check_step_lens(b, step_lens)) return rc;
    return enqueue_grow("lora_kv_grow_step", b, add, max_len, step_lens, info, ws, ws_bytes, stream);
}

int lora_kv_fork(const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t n, const int32_t* parents,
                 const int32_t* children, int32_t* info, void* ws, size_t ws_bytes, void* stream) {
    return enqueue_fork("lora_kv_fork", c, b, n, parents, children, nullptr, info, ws, ws_bytes, stream);
}

int lora_kv_fork_step(const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t n, const int32_t* parents,
                      const int32_t* children, int32_t* step_lens, int32_t* info, void* ws, size_t ws_bytes,
                      void* stream) {
    if (int rc = check_book(b)) return rc;
    if (int rc = check_step_lens(b, step_lens)) return rc;
    return enqueue_fork("lora_kv_fork_step", c, b, n, parents, children, step_lens, info, ws, ws_bytes, stream);
}

int lora_kv_free(const lora_kv_book_t* b, int32_t n, const int32_t* seqs, void* stream) {
    if (int rc = check_book(b)) return rc;
    if (n < 0) return set_error(LORA_E_ARG, "negative count");
    if (n > 0 && !seqs) return set_error(LORA_E_ARG, "seqs is NULL");
    try {
        std::vector<uint8_t> mark((size_t)b->n_seqs, 0);
        if (int rc = check_ids("sequence", seqs, n, b->n_seqs, mark)) return rc;
    } catch (const std::bad_alloc&) {
        return set_error(LORA_E_NOMEM, "host memory for the argument check");
    }
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device("lora_kv_free");
    IdArgs ids{};
    for (int32_t i0 = 0; i0 < n; i0 += kArgIds) {
        const int m = std::min(kArgIds, n - i0);
        for (int i = 0; i < m; ++i) ids.id[i] = seqs[i0 + i];
        hipLaunchKernelGGL(lora_kv_release_kernel, dim3(m), dim3(kCopyThreads), 0, st, device_book(b), ids, 1, 0,
                           (int32_t*)nullptr);
        if (int rc = check_launch("lora_kv_free")) return rc;
    }
    return LORA_OK;
}

int lora_kv_trim(const lora_kv_book_t* b, int32_t window, int32_t n_sinks, void* stream) {
    if (int rc = check_book(b)) return rc;
    if (window < 1 || n_sinks < 0) return set_error(LORA_E_ARG, "needs window >= 1 and n_sinks >= 0");
    if (b->n_seqs == 0) return LORA_OK;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device("lora_kv_trim");
    hipLaunchKernelGGL(lora_kv_trim_kernel, dim3(std::min(b->n_seqs, kTrimBlocks)), dim3(kCopyThreads), 0, st,
                       device_book(b), window, n_sinks);
    return check_launch("lora_kv_trim");
}

int lora_kv_copy(const lora_kv_cache_t* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
    if (int rc = check_kv_cache(c)) return rc;
    if (int rc = check_page_size(c)) return rc;
    if (int rc = check_pairs("src", "dst", src, dst, n, c->n_pages)) return rc;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device("lora_kv_copy");
    const PageDims d = page_dims(c);
    IdArgs ids{};
    for (int32_t i0 = 0; i0 < n; i0 += kArgIds / 2) {
        const int m = std::min(kArgIds / 2, n - i0);
        for (int i = 0; i < m; ++i) {
            ids.id[2 * i] = src[i0 + i];
            ids.id[2 * i + 1] = dst[i0 + i];
        }
        hipLaunchKernelGGL(lora_kv_copy_kernel, dim3(2 * d.n_layers * d.blocks, m), dim3(kCopyThreads), 0, st, d, ids);
        if (int rc = check_launch("lora_kv_copy")) return rc;
    }
    return LORA_OK;
}

int lora_kv_compact(const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t* tables_out, int32_t* refs_out,
                    int32_t* info, void* ws, size_t ws_bytes, void* stream) {
    if (int rc = check_kv_cache(c)) return rc;
    if (int rc = check_page_size(c)) return rc;
    if (int rc = check_book(b)) return rc;
    if (int rc = check_book_cache(c, b)) return rc;
    if ((b->n_seqs > 0 && b->ld_table > 0 && !tables_out) || (b->n_pages > 0 && !refs_out))
        return set_error(LORA_E_ARG, "tables_out or refs_out is NULL");
    if (((uintptr_t)tables_out | (uintptr_t)refs_out) & 3)
        return set_error(LORA_E_ALIGN, "tables_out or refs_out not 4-byte aligned");
    if (int rc = check_words("info", info)) return rc;
    if (int rc = check_ws(b, ws, ws_bytes)) return rc;
    hipStream_t st = (hipStream_t)stream;
    StreamDevice g(st);
    if (!g.ok) return no_device("lora_kv_compact");
    const Book book = device_book(b);
    const PageDims d = page_dims(c);
    const BookWs w = book_ws(ws, b->n_pages, b->n_seqs);
    hipLaunchKernelGGL(lora_kv_number_kernel, dim3(1), dim3(kBookThreads), 0, st, book, info, w);
    if (int rc = check_launch("lora_kv_compact")) return rc;
    // workgroups for the book (one word per thread, 256 at most) and for the pages (at most half of all move)
    const int64_t words = std::max((int64_t)b->n_seqs * b->ld_table, (int64_t)b->n_pages);
    const int book_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(256, (words + kCopyThreads - 1) / kCopyThreads));
    const int64_t units = (int64_t)(b->n_pages / 2) * 2 * d.n_layers * d.blocks;
    const int copy_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(4096, units));
    hipLaunchKernelGGL(lora_kv_move_kernel, dim3(book_blocks + copy_blocks), dim3(kCopyThreads), 0, st, book, d,
                       tables_out, refs_out, w, book_blocks);
    return check_launch("lora_kv_compact");
}

}  // extern "C"
