// prompt_kernels.cu — attention of many query rows over the same pages of a
// paged cache, on the 5th-generation tensor cores.
//
// Two calls use it: a prompt's rows over its sequence (Sec. 3.2: new queries
// are computed on top of a restored block), and the rows of a batch over the
// pages of a block that its sequences share.  Query row i attends to the valid
// rows (below their page's fill) in slots [lo_i, hi_i]:
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j
// For a prompt hi_i is the row's own slot and lo_i 0 or the slot of the last
// `window` valid rows up to it; for a shared block hi_i is its last slot.
//
// A work item is a KV head, a tile of query rows (tokens x the group's heads,
// so that a KV head's queries share its keys) and a range of key tiles; a CTA
// takes one, or for head_dim 256 a pair of CTAs (a cluster), each with half of
// the query rows, of the keys' columns and of the values' dimensions: a single
// CTA's shared memory held 2.5 key or value tiles there, which made it wait for
// copies (8,191 rows of the 12B shape: 506 us; 392 us as pairs, all else the same).
// Key tiles are 128 columns, made of units of 128 (pairs: 64): a page's rows,
// or as many whole pages as fit when pages are smaller, each at a multiple of 8
// rows so that its copy starts on a swizzle atom.
//
// Warps: four per stream of 128 query rows form weights (a thread has a row);
// one loads pages, one thread issues products, one zeroes the value rows that
// hold nothing, one works out the next item and fetches its queries (for an fp8
// cache four convert E4M3 codes to fp16, exact, zero those rows and fetch the
// queries).
//
// What bounds it: the tensor cores and, with two streams, the softmax between
// them.  A tile of 256 x 128 is 2,150 cycles of products; it takes 2,400 for
// head_dim 256 (1.68 PFLOP/s over 8,191 rows of the 12B shape, 327 us) and
// 2,650 for 128 (1.53, 8,192 rows of the 31B shape on 16,384 in 1,795 us): each
// stream's scores, weights and products follow one another, and the weights of
// one take longer (1,350 cycles) than the products of the other.  Packed fp8
// prompts of 1 .. 1,501 rows with windows of 1,024 (161 us) spend 6,500 of
// 34,000 cycles an item between items.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "tcgen05.cuh"

namespace kvg {

namespace {

constexpr int kTile = 128;       // query rows of a stream, columns of a key tile
constexpr int kMaskSlots = 16;   // key tiles whose column masks are kept
constexpr int kConvertWarps = 4;
constexpr int kRowWarps = 8;     // 32 rows of an item each, at most
// The running maximum that the weights refer to is moved only when a row's
// maximum passes it by more than this (in powers of two): weights then reach
// at most 2^8, which costs no precision in bf16 or fp16, and the accumulator
// is rarely rescaled.
constexpr float kMaxSlack = 8.f;

// STREAMS tiles of query rows share each key tile: with two, one's products
// run while the other's weights are formed.  With one there are two score
// buffers instead, so that the next tile's scores are formed ahead.
template <int D_, bool FP8_, int STREAMS_>
struct Cfg {
    static constexpr int D = D_, STREAMS = STREAMS_;
    static constexpr bool FP8 = FP8_, PAIR = D == 256;
    static constexpr int CTAS = PAIR ? 2 : 1;
    static constexpr int DV = D / CTAS;              // dimensions of a CTA's values
    static constexpr int UNIT = kTile / CTAS;        // columns of a CTA's keys
    static constexpr int CHUNK = kTile * DV * 2;     // a CTA's keys or values of a tile, 16 bits
    // boxes of 128 bytes x UNIT (keys) or 128 (values) rows
    static constexpr int K_BOX = UNIT * 128, V_BOX = kTile * 128, K_BOXES = D / 64, V_BOXES = DV / 64;
    static constexpr int RAW = FP8 ? CHUNK / 2 : 0;  // the same as fp8, as it is in the cache
    static constexpr int Q_BYTES = STREAMS * kTile * D * 2;
    static constexpr int STAGES = D == 64 ? 8 : FP8 ? (Q_BYTES > 32768 ? 4 : 5) : Q_BYTES > 32768 ? 5 : 6;
    static constexpr int RAW_STAGES = FP8 ? 2 : 0;
    static constexpr int LANDS = FP8 ? RAW_STAGES : STAGES;  // the ring that copies land in
    // Chunks come as K0, then K(j + 1) and V(j) in turn, the last V alone.  Two
    // streams hand over and give back K(j + 1) and V(j) together (an MMA commit
    // holds up the issuing thread): chunk c is of group (c + 1) / 2.
    static constexpr bool GROUPED = STREAMS == 2;
    // (As many barriers as a ring may hold groups: items of one tile have a chunk to
    // each, and two groups that land on one barrier would be one phase ahead.)
    static constexpr int GROUPS = GROUPED ? 8 : STAGES;
    static_assert(GROUPS >= STAGES && GROUPS <= 8, "groups in flight");
    static constexpr int SOFTMAX_WARPS = 4 * STREAMS;
    static constexpr int LOAD_WARP = SOFTMAX_WARPS, MMA_WARP = LOAD_WARP + 1, TIDY_WARP = LOAD_WARP + 2, CONVERT_WARP = LOAD_WARP + 4;
    // (for an fp8 cache the converting warps tidy and fetch queries)
    static constexpr int NEXT_WARP = LOAD_WARP + 3;
    static constexpr int THREADS = 32 * (CONVERT_WARP + (FP8 ? kConvertWarps : 0));
    // Registers of a softmax thread and of the others, moved between the
    // warpgroups where the launch's even share is too few for a row of scores:
    // 3 groups of 168 (200 + 200 + 96 of 504, or 224 + 136 + 136), 4 of 128 (176
    // + 176 + 80 + 80 of 512).  (A call in the kernel would void it.)
    static constexpr int MORE_REGS = THREADS == 512 ? 176 : THREADS == 384 ? (STREAMS == 2 ? 200 : 224) : 0;
    static constexpr int FEWER_REGS = THREADS == 512 ? 80 : STREAMS == 2 ? 96 : 136;
    static constexpr int SMEM = Q_BYTES + STAGES * CHUNK + RAW_STAGES * RAW + 1024;  // + alignment slack
    static_assert(!PAIR || STREAMS == 1, "tensor memory");
    static_assert(SMEM <= 230400 + 1024, "shared memory");
    static __device__ __forceinline__ int group(int chunk) { return GROUPED ? (chunk + 1) / 2 : chunk; }
};
constexpr int kScoreCols = 0, kOutCols = 256;  // tensor memory: scores (and weights), outputs

// ------------------------------------------------------------ a work item --
struct Item {
    int b, split, lr, g;
    int gs;         // log2 of the group
    int row0, rows; // of the sequence's rows (token x head of the group), those of the item
    int k0, k1;     // key tiles
    int last_slot;  // of the sequence's pages that the item reads
    int at;         // of the launch's items
};

// Items that a CTA knows of at once.
constexpr int kItems = 4;
// The next item is asked for kAskTiles key tiles before an item's end (the
// answer, the first pages and the queries take some 8,000 cycles), so that CTAs
// end close together: 20 us apart instead of 35 in packed fp8 prompts of up to 9
// tiles an item (161 us; 167 to 171 asked for at its start).
constexpr int kAskTiles = 5;

struct Bars {
    uint64_t landed[8], freed[2];            // copies: there; (fp8) converted, their place is free
    uint64_t ready[8], empty[8];             // groups of chunks: may be multiplied; have been
    uint64_t scores[2], out[2];              // a score tile is there; its weights' product is added
    uint64_t weights[2][2];                  // the halves of its weights are there
    uint64_t queries, scored;                // an item's queries are there, have been multiplied
    uint64_t taken[2], drained;              // its outputs have been read
    uint64_t next[kItems], known[kItems];    // of item k (k % kItems): the answer is there, what it is
    uint4 answer[kItems];
    Item item[kItems];                       // b < 0: no more
    uint32_t mask[kMaskSlots][4];            // valid columns of key tile j % kMaskSlots
    uint32_t tmem;
    int abort;
    int redo;                                // last entry of p.redo that the CTA made, or -1
};

// Bounded wait that also ends when another warp gave up.
__device__ __forceinline__ bool wait_slow(uint64_t *bar, uint32_t parity, volatile int *abort, DevStatus *status) {
    const uint64_t t0 = global_timer_ns();
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 63) == 0) {
            if (*abort) return false;
            if (global_timer_ns() - t0 > 2000000000ull) {
                *abort = 1;
                record_error(status, KVG_ERR_DEVICE_CHECK, 20);
                return false;
            }
        }
    }
}
__device__ __forceinline__ bool wait_bar(Bars &s, uint64_t *bar, uint32_t parity, DevStatus *status) {
    const bool ok = mbar_try_wait(bar, parity) || wait_slow(bar, parity, &s.abort, status);
    return __all_sync(0xffffffffu, ok);
}

// ------------------------------------------------------------ a work item --

// Key tile and column of a slot.
__device__ __forceinline__ void tile_of(const PromptParams &p, int slot, int &tile, int &col) {
    const int pg = p.by_page.div(slot), r = slot - pg * p.page_size;
    int u;
    if (p.pages_per_unit) {
        u = p.by_pages.div(pg);
        col = (pg - u * p.pages_per_unit) * p.page_rows + r;
    } else {
        u = pg * p.units_per_page + r / p.unit;
        col = r % p.unit;
    }
    const int per = kTile / p.unit;
    tile = u / per;
    col += (u - tile * per) * p.unit;
}
__device__ __forceinline__ int first_slot(const PromptParams &p, int tile) {
    const int u = tile * (kTile / p.unit);
    return p.pages_per_unit ? u * p.pages_per_unit * p.page_size
                            : p.by_pages.div(u) * p.page_size + (u - p.by_pages.div(u) * p.units_per_page) * p.unit;
}

// First slot that the row at `slot` attends to.
__device__ __forceinline__ int window_first(const PromptParams &p, int b, int slot) {
    if (p.window <= 0) return 0;
    const int from = max(0, slot - p.window + 1);
    if (from >= p.solid[b]) return from;
    // pages that are not full lie in between: count valid rows back
    const int32_t *fill = p.page_fill + (int64_t)p.seq[b] * p.max_pages;
    int pg = slot / p.page_size, n = slot % p.page_size + 1, left = p.window;
    while (n < left && pg > 0) {
        left -= n;
        n = fill[--pg];
    }
    return pg * p.page_size + max(0, n - left);
}
__device__ __forceinline__ int row_first(const PromptParams &p, const Item &it, int tok) {
    return p.shared ? p.lo[p.row0[it.b] + tok] : window_first(p, it.b, p.slot0[it.b] + tok);
}
__device__ __forceinline__ int row_last(const PromptParams &p, const Item &it, int tok) {
    return p.slot0[it.b] + (p.shared ? 0 : tok);
}
// Row of q and out.
__device__ __forceinline__ int64_t q_row(const PromptParams &p, const Item &it, int row) {
    const int at = p.row0[it.b] + (row >> it.gs);
    return ((int64_t)p.qlayers[it.lr] * p.q_rows + (p.shared ? p.member[at] : at)) * p.n_q_heads + (it.g << it.gs) +
           (row & ((1 << it.gs) - 1));
}
// Slot of a row's partial result.
__device__ __forceinline__ int64_t part_slot(const PromptParams &p, const Item &it, int split, int row) {
    const int64_t n = (int64_t)(p.first[it.b + 1] - p.first[it.b]) << it.gs;
    const int unit = it.lr * p.n_kv_heads + it.g;
    return p.part0[it.b] + ((int64_t)split * p.n_units + unit) * n + row;
}

__device__ __forceinline__ int search(const int32_t *first, int n, int64_t at) {
    int b = 0;
    for (int hi = n - 1; b < hi;) {  // largest b with first[b] <= at
        const int mid = (b + hi + 1) >> 1;
        if (first[mid] <= at)
            b = mid;
        else
            hi = mid - 1;
    }
    return b;
}

// The longest tiles of a sequence (its last rows) come first.
__device__ __forceinline__ Item item_of(const PromptParams &p, int at, int tile_rows) {
    Item it;
    it.at = at;
    const int b = search(p.item0, p.n_seq, at);
    it.b = b;
    it.gs = p.log2_group;
    const int n = (p.first[b + 1] - p.first[b]) << it.gs, nt = (n + tile_rows - 1) / tile_rows;
    const int splits = p.splits[b], of_unit = at - p.item0[b];
    const int rem = p.by_units.div(of_unit), unit = of_unit - rem * p.n_units;
    const int tile = splits == 1 ? rem : rem / splits, t = nt - 1 - tile;
    it.split = rem - tile * splits;
    it.lr = p.by_kv_heads.div(unit);
    it.g = unit - it.lr * p.n_kv_heads;
    it.row0 = t * tile_rows;
    it.rows = min(tile_rows, n - it.row0);
    it.last_slot = row_last(p, it, (it.row0 + it.rows - 1) >> it.gs);
    int from = p.window <= 0 ? 0 : p.begin[b];
    if (p.window > 0 && !p.shared) {
        const int reach = max(0, p.slot0[b] + (it.row0 >> it.gs) - p.window + 1);
        if (reach >= p.solid[b]) from = reach;
    }
    int ka, kb, col;
    tile_of(p, from, ka, col);
    tile_of(p, it.last_slot, kb, col);
    const int len = max(0, kb + 1 - ka);  // (a shared block may end before the rows' windows)
    const int part = splits == 1 ? len : len / splits, rest = len - part * splits;  // the first `rest` splits have one more
    it.k0 = ka + part * it.split + min(it.split, rest);
    it.k1 = it.k0 + max(1, part + (it.split < rest));  // (one tile past the last: no valid column)
    return it;
}

// ------------------------------------------------------- one row, scalar ----
// D / 32 consecutive elements of a row as floats.
template <int D, bool FP8>
__device__ __forceinline__ void load_row(const uint8_t *row, int lane, float (&x)[D / 32]) {
    constexpr int N = D / 32;
    if constexpr (FP8) {
        const uint16_t *c = reinterpret_cast<const uint16_t *>(row + lane * N);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c[i]));
            asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
                : "=f"(x[2 * i]), "=f"(x[2 * i + 1])
                : "r"(h));
        }
    } else {
        const uint32_t *c = reinterpret_cast<const uint32_t *>(row + lane * N * 2);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            x[2 * i] = __uint_as_float(c[i] << 16);
            x[2 * i + 1] = __uint_as_float(c[i] & 0xffff0000u);
        }
    }
}

// K row (V: + v_off bytes) of a slot, null where it is not valid.
template <int D, bool FP8>
__device__ __forceinline__ const uint8_t *row_at(const PromptParams &p, const Item &it, int slot, int64_t &v_off) {
    constexpr int E = FP8 ? 1 : 2;
    const int pg = slot / p.page_size, r = slot - pg * p.page_size;
    const int64_t at = (int64_t)p.seq[it.b] * p.max_pages + pg;
    const int pid = p.page_table[at];
    v_off = p.pool_pages * p.n_kv_heads * p.page_size * D * E;
    if (r >= p.page_fill[at] || pid < 0 || pid >= p.pool_pages) return nullptr;
    const int64_t page = (int64_t)p.layers[it.lr] * 2 * p.pool_pages + pid;
    return p.pool + (((page * p.n_kv_heads + it.g) * p.page_size) + r) * D * E;
}

// A warp: attention of one query row over slots [first, last], from the last one
// back, some slots' loads in flight together.
template <int D, bool FP8>
__device__ __forceinline__ void attend_row(const PromptParams &p, const Item &it, int row, int first, int last,
                                        float (&o)[D / 32], float &m, float &l) {
    constexpr int N = D / 32, U = 4;
    const int lane = threadIdx.x & 31;
    float q[N];
    load_row<D, false>(reinterpret_cast<const uint8_t *>(p.q + q_row(p, it, row) * D), lane, q);
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
    for (int slot = last; slot >= first; slot -= U) {
        const uint8_t *k[U];
        int64_t v_off;
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = slot - u >= first ? row_at<D, FP8>(p, it, slot - u, v_off) : nullptr;
            s[u] = 0.f;
            if (!k[u]) continue;
            float x[N];
            load_row<D, FP8>(k[u], lane, x);
#pragma unroll
            for (int i = 0; i < N; ++i) s[u] = __fmaf_rn(q[i], x[i], s[u]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] += __shfl_xor_sync(0xffffffffu, s[u], d);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!k[u]) continue;
            s[u] *= p.negate ? -p.qscale : p.qscale;
            const float mn = fmaxf(m, s[u]);
            const float base = mn == -INFINITY ? 0.f : mn;
            const float a = exp2f(m - base), w = exp2f(s[u] - base);
            m = mn;
            l = __fmaf_rn(l, a, w);
            float x[N];
            load_row<D, FP8>(k[u] + v_off, lane, x);
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = __fmaf_rn(o[i], a, w * x[i]);
        }
        bool nan = true;
#pragma unroll
        for (int i = 0; i < N; ++i) nan = nan && o[i] != o[i];
        if (__all_sync(0xffffffffu, nan)) break;  // (stays so)
    }
}

__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// A value row that is not finite reaches, as 0 x inf, the outputs of rows of
// its tile that do not attend to it.  So a softmax warp whose outputs are not
// finite notes its 32 rows, and when the CTA has done all its items (nothing
// waits for those warps then, however long it takes) they compute the ones that
// such a row reached over from the definition, each a row at a time.

// Of some of the CTA's warps, always the same.
__device__ __forceinline__ void sync_warps(int warps) { asm volatile("bar.sync 1, %0;" ::"r"(32 * warps) : "memory"); }

// A warp: of 32 rows from first_row on, those that a value row which is not
// finite reached without being attended to, among the columns that their tiles
// masked.  (Other outputs that are not finite are as they should be.)
template <int D, bool FP8>
__device__ __forceinline__ uint32_t reached(const PromptParams &p, const Item &it, int first_row) {
    constexpr int N = D / 32;
    const int lane = threadIdx.x & 31, row = first_row + lane;
    const bool mine = row < it.row0 + it.rows;
    const int lo = mine ? row_first(p, it, row >> it.gs) : 0, hi = mine ? row_last(p, it, row >> it.gs) : -1;
    int tile_lo, tile_hi = 0x7fffffff, col;
    tile_of(p, lo, tile_lo, col);
    if (mine) tile_of(p, hi, tile_hi, col);
    const int from = __reduce_min_sync(0xffffffffu, tile_hi), to = __reduce_max_sync(0xffffffffu, tile_lo);
    bool redo = false;
    for (int kt = it.k0; kt < it.k1; ++kt) {
        if (kt < from && kt > to) continue;  // no row of the warp masks valid columns of it
        const int end = min(first_slot(p, kt + 1), it.last_slot / p.page_size * p.page_size + p.page_size);
        for (int slot = first_slot(p, kt); slot < end; ++slot) {
            int64_t v_off;
            const uint8_t *k = row_at<D, FP8>(p, it, slot, v_off);
            if (!k) continue;
            float x[N];
            load_row<D, FP8>(k + v_off, lane, x);
            bool fine = true;
#pragma unroll
            for (int i = 0; i < N; ++i) fine = fine && isfinite(x[i]);
            if (__any_sync(0xffffffffu, !fine)) redo = redo || slot < lo || slot > hi;
        }
    }
    return __ballot_sync(0xffffffffu, mine && redo);
}

// The CTA's softmax warps (all of them), of the entries up to `last`: first each
// takes entries and keeps the rows that are to be computed, then rows.  8,192
// rows of the 31B shape on 4,096 whose queries are all NaN take 1.56 ms (finite
// ones 0.69), with all values NaN 2.2.
template <int D, bool FP8>
__device__ __forceinline__ void compute_over(const PromptParams &p, int last, int tile_rows, int warp, int warps) {
    constexpr int N = D / 32;
    const int lane = threadIdx.x & 31;
    int n = 0;  // entries, then rows so far
    for (int id = last; id >= 0; id = p.redo[id].y, ++n) {
        if (n % warps != warp) continue;
        const Item it = item_of(p, id / kRowWarps, tile_rows);
        const uint32_t rows = reached<D, FP8>(p, it, it.row0 + id % kRowWarps * 32);
        if (lane == 0) p.redo[id].x &= (int)rows;
    }
    sync_warps(warps);
    n = 0;
    for (int id = last; id >= 0;) {
        const int2 entry = p.redo[id];
        const Item it = item_of(p, id / kRowWarps, tile_rows);
        const int first_row = it.row0 + id % kRowWarps * 32;
        const bool partial = p.splits[it.b] > 1 || p.shared;
        for (uint32_t left = entry.x; left; left &= left - 1, ++n) {
            if (n % warps != warp) continue;
            const int row = first_row + __ffs(left) - 1, token = row >> it.gs;
            const int from = max(row_first(p, it, token), first_slot(p, it.k0));
            const int to = min(row_last(p, it, token), first_slot(p, it.k1) - 1);
            float o[N], m, l;
            attend_row<D, FP8>(p, it, row, from, to, o, m, l);
            if (partial) {
                const int64_t at = part_slot(p, it, it.split, row);
#pragma unroll
                for (int e = 0; e < N; ++e) p.part_o[at * D + lane * N + e] = o[e];
                if (lane == 0) p.part_ml[at] = make_float2(l == l ? m : 0.f, l);
            } else {
                const float inv = p.vscale / l;
                uint32_t *out = reinterpret_cast<uint32_t *>(p.out + q_row(p, it, row) * D + lane * N);
#pragma unroll
                for (int e = 0; e < N / 2; ++e) out[e] = pack_out(o[2 * e] * inv, o[2 * e + 1] * inv);
            }
        }
        id = entry.y;
    }
}

// Tiles land as K0, then K(j + 1) and V(j) in turn, the last V alone: whether
// the i-th is a value tile, and of which key tile the keys or values are.
__device__ __forceinline__ bool value_tile(int i, int n, int &j) {
    const bool last = i == 2 * n - 1, values = last || (i > 0 && i % 2 == 0);
    j = last ? n - 1 : values ? i / 2 - 1 : (i + 1) / 2;
    return values;
}

// A lane's page of a key tile: lane i has page i % 16 of the tile's unit i / 16.
struct Page {
    int rows;    // valid rows of it in the tile
    int32_t at;  // its first row in the pool, of the layer's keys
};
struct Entry {  // the same as it is in the tables, on its way
    int pid, fill, sub;  // sub: first row in the page
};
template <class C>
struct Pages {
    const int32_t *table, *fill;  // of the item's sequence
    int32_t base;                 // the pool's row where page 0 would start
    int last;                     // the item's last page
    __device__ __forceinline__ void of(const PromptParams &p, const Item &it) {
        const int64_t e = (int64_t)p.seq[it.b] * p.max_pages;
        table = p.page_table + e;
        fill = p.page_fill + e;
        base = (int32_t)(((int64_t)p.layers[it.lr] * 2 * p.pool_pages * p.n_kv_heads + it.g) * p.page_size);
        last = p.by_page.div(it.last_slot);
    }
    // of key tile kt (none from k1 on)
    __device__ __forceinline__ Entry load(const PromptParams &p, int kt, int k1, int lane) const {
        const int unit = lane / 16, place = lane % 16, u = kt * C::CTAS + unit;
        int pg = u * p.pages_per_unit + place;
        bool has = unit < C::CTAS && place < p.pages_per_unit;
        Entry e{0, 0, 0};
        if (!p.pages_per_unit) {
            pg = p.by_pages.div(u);
            e.sub = (u - pg * p.units_per_page) * C::UNIT;
            has = unit < C::CTAS && place == 0;
        }
        if (has && pg <= last && kt < k1) {
            e.pid = table[pg];
            e.fill = fill[pg];
        }
        return e;
    }
    __device__ __forceinline__ Page page(const PromptParams &p, const Entry &e) const {
        Page r;
        r.rows = max(0, min(p.pages_per_unit ? p.page_size : C::UNIT, e.fill - e.sub));
        if (r.rows && (e.pid < 0 || e.pid >= p.pool_pages)) {
            record_error(p.status, KVG_ERR_DEVICE_CHECK, 21);
            r.rows = 0;
        }
        r.at = base + e.pid * (p.n_kv_heads * p.page_size) + e.sub;
        return r;
    }
};

// Query rows of an item on their way to the swizzled rows of their tiles, by
// warps that each have CHUNKS times 32 of a CTA's rows: rows 32 w, w = from,
// from + step, ...  (What runs once per item is kept to short loops here and for
// the outputs: unrolled, it waited for its instructions.)
template <class C, int CHUNKS>
struct Queries {
    static constexpr int D = C::D, LPR = D / 8, RPI = 32 / LPR, N = 32 / RPI;  // lanes of a row, rows of a copy
    const __nv_bfloat16 *src;  // the lane's piece of the item's first row
    int off[CHUNKS];           // the lane's row of each 32, in rows from there; INT_MIN: past the item's end

    __device__ __forceinline__ void find(const PromptParams &p, const Item &it, int first, int from, int step, int lane,
                                         bool prefetch) {
        const int64_t base = q_row(p, it, it.row0);
        src = p.q + base * D + lane % LPR * 8;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int r = first + (from + c * step) * 32 + lane;
            off[c] = r < it.rows ? (int)(q_row(p, it, it.row0 + r) - base) : INT_MIN;  // (a tile's rows: less than 2^31 apart)
            if (prefetch && r < it.rows)
#pragma unroll 1
                for (int x = 0; x < D; x += 64) prefetch_l2(p.q + (base + off[c]) * D + x);
        }
    }
    // the lane's piece of copy i of rows 32 w
    static __device__ __forceinline__ uint8_t *at(uint8_t *q_tiles, int w, int i, int lane) {
        const int u = lane % LPR, h = lane / LPR;
        return q_tiles + w / 4 * (kTile * D * 2) + w % 4 * (32 * 128) + u / 8 * (kTile * 128) + h * 128 + i * RPI * 128 +
               (((u % 8 ^ h) << 4) ^ (i * RPI % 8 << 4));
    }
    __device__ __forceinline__ void copy(int from, int step, int lane, uint8_t *q_tiles) const {
#pragma unroll 1
        for (int c = 0; c < CHUNKS; ++c) {
            int mine = off[0];
#pragma unroll
            for (int x = 1; x < CHUNKS; ++x) mine = c == x ? off[x] : mine;
#pragma unroll 1
            for (int i0 = 0; i0 < N; i0 += 8) {
                int o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = __shfl_sync(0xffffffffu, mine, (i0 + i) * RPI + lane / LPR);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    async_copy16(at(q_tiles, from + c * step, i0 + i, lane), src + (int64_t)(o[i] == INT_MIN ? 0 : o[i]) * D,
                                 o[i] != INT_MIN);
            }
        }
    }
    // After the lane's copies, for an fp8 cache's products: bf16 to fp16, in place.
    static __device__ __forceinline__ void convert(int from, int step, int lane, uint8_t *q_tiles) {
        constexpr int BATCH = 4;
#pragma unroll 1
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll 1
            for (int i0 = 0; i0 < N; i0 += BATCH) {
                uint4 x[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) x[i] = *reinterpret_cast<const uint4 *>(at(q_tiles, from + c * step, i0 + i, lane));
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __half2 h = __floats2half2_rn(__uint_as_float(y[e] << 16), __uint_as_float(y[e] & 0xffff0000u));
                        y[e] = *reinterpret_cast<const uint32_t *>(&h);
                    }
                    *reinterpret_cast<uint4 *>(at(q_tiles, from + c * step, i0 + i, lane)) = make_uint4(y[0], y[1], y[2], y[3]);
                }
            }
    }
};

// Lane q of four has row q of a 4 x 4 block: column q of it, for each.
__device__ __forceinline__ void transpose4(uint32_t (&v)[4], int q) {
#pragma unroll
    for (int d = 1; d <= 2; d *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!(i & d)) {
                const bool odd = q & d;
                const uint32_t x = __shfl_xor_sync(0xffffffffu, odd ? v[i] : v[i | d], d);
                (odd ? v[i] : v[i | d]) = x;
            }
}

// Which group's commit frees each place of the ring: a lane remembers the group
// of the chunk that its place holds.
template <class C>
struct Groups {
    int held = 0, before = 0;  // the lane's place; groups of the items before
    // place st is for the item's i-th chunk: the group of the chunk it held
    __device__ __forceinline__ int take(int st, int lane, int i) {
        const int g = of(st);
        if (lane == st) held = before + C::group(i);
        return g;
    }
    __device__ __forceinline__ int of(int st) const { return __shfl_sync(0xffffffffu, held, st); }
    __device__ __forceinline__ void end(int n) { before += C::group(2 * n - 1) + 1; }
};

// ------------------------------------------------------------------ kernel --
template <class C>
__global__ void __launch_bounds__(C::THREADS, 1)
    prompt_kernel(const __grid_constant__ PromptParams p, const __grid_constant__ CUtensorMap map) {
    constexpr int D = C::D, STREAMS = C::STREAMS, STAGES = C::STAGES, LANDS = C::LANDS, CTAS = C::CTAS;
    constexpr bool FP8 = C::FP8;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ Bars s;
    uint8_t *const smem = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    uint8_t *const ring = smem + C::Q_BYTES;
    uint8_t *const raw = ring + STAGES * C::CHUNK;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;  // uniform in the warp
    const int rank = CTAS == 2 ? (int)cluster_rank() : 0;
    const int first = rank * kTile;  // of an item's rows
    // a warp's arrival for the issuing thread (of a pair's first CTA), one for its lanes together
    auto arrive_issuer = [&](uint64_t *bar, int times = 1) {
        __syncwarp();
        if (lane == 0)
            for (int i = 0; i < times; ++i) {
                if constexpr (CTAS == 2)
                    mbar_arrive_first(bar);
                else
                    mbar_arrive(bar);
            }
    };

    if (warp == C::LOAD_WARP && lane == 0)
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::GROUPS; ++i) {
            mbar_init(&s.ready[i], CTAS * (C::GROUPED ? 2 : 1) * (FP8 ? kConvertWarps : 1));
            mbar_init(&s.empty[i], 1);
        }
        for (int i = 0; i < LANDS; ++i) mbar_init(&s.landed[i], 1);
        for (int i = 0; i < C::RAW_STAGES; ++i) mbar_init(&s.freed[i], kConvertWarps);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.scores[i], 1);
            mbar_init(&s.weights[i][0], CTAS * 4);
            mbar_init(&s.weights[i][1], CTAS * 4);
            mbar_init(&s.out[i], 1);
        }
        mbar_init(&s.queries, CTAS * C::SOFTMAX_WARPS);
        mbar_init(&s.scored, 1);
        mbar_init(&s.taken[0], CTAS * 4);
        mbar_init(&s.taken[1], CTAS * 4);
        for (int i = 0; i < kItems; ++i) {
            mbar_init(&s.next[i], 1);
            mbar_init(&s.known[i], 1);
        }
        mbar_init(&s.drained, 1);
        s.abort = 0;
        s.redo = -1;
        fence_mbar_init();
    }
    if (warp == C::MMA_WARP) tmem_alloc<512, CTAS>(&s.tmem);
    // The first item (from the launch's parameters alone), its first pages and its
    // queries, all beside the set-up.
    Item it;
    Pages<C> pages;
    Entry coming{0, 0, 0}, after{0, 0, 0};
    Queries<C, 1> first_queries;
    if (warp <= C::LOAD_WARP) {
        it = item_of(p, blockIdx.x / CTAS, STREAMS * CTAS * kTile);
        after_previous();
        if (warp < C::LOAD_WARP) {
            first_queries.find(p, it, first, warp, 0, lane, false);
        } else {
            pages.of(p, it);
            coming = pages.load(p, it.k0, it.k1, lane);
            after = pages.load(p, it.k0 + 1, it.k1, lane);
            if (lane == 0) s.item[0] = it;
        }
    }
    tc_before_sync();
    if constexpr (CTAS == 2)
        cluster_sync();
    else
        __syncthreads();
    tc_after_sync();
    const uint32_t tmem = s.tmem;

    // The CTA's items: its own, then those of CTAs that have not started, so that
    // copies run ahead into the next item while an item's outputs are stored.
    // The issuing thread asks for item k + 1 while it is in item k (every warp has
    // left item k - 3, whose places it takes), one warp works out what the answer
    // means for all.  The CTA's item k >= 1, for a warp:
    auto has_item = [&](int k) {
        return wait_bar(s, &s.known[k % kItems], ((k - 1) / kItems) & 1, p.status) && s.item[k % kItems].b >= 0;
    };

    if (warp < C::SOFTMAX_WARPS) {
        if constexpr (C::MORE_REGS > 0) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::MORE_REGS));
        const int stream = warp / 4;
        first_queries.copy(warp, 0, lane, smem);
        async_wait_all();
        if constexpr (FP8) first_queries.convert(warp, 0, lane, smem);
        fence_proxy_async_shared();
        arrive_issuer(&s.queries);
        bool ok = true;
        int tiles = 0;  // of the items before
        for (int k = 0; ok; ++k) {
            const Item &it = s.item[k % kItems];  // (there until item k + 4 is known)
            const int k0 = it.k0, n = it.k1 - k0;
            // ---- weights: a thread has a query row
            const uint32_t lanes = (uint32_t)(warp % 4) << 21;  // tensor memory lanes of the warp
            const int r = first + threadIdx.x;                   // the thread's row of the item
            const bool mine = r < it.rows;
            int tile_lo = 0, col_lo = 0, tile_hi = -1, col_hi = 0;
            if (mine) {
                const int token = (it.row0 + r) >> it.gs;
                tile_of(p, row_first(p, it, token), tile_lo, col_lo);
                tile_of(p, row_last(p, it, token), tile_hi, col_hi);
            }
            const float c = p.qscale;
            float m = -INFINITY;               // what the weights refer to
            float2 sum = make_float2(0.f, 0.f);
            const uint32_t o_at = tmem + lanes + kOutCols + stream * kTile;
            for (int j = 0; j < n; ++j) {
                const int J = tiles + j, buf = STREAMS == 1 ? J & 1 : stream;
                const uint32_t s_at = tmem + lanes + kScoreCols + buf * kTile;
                ok = wait_bar(s, &s.scores[buf], (STREAMS == 1 ? J >> 1 : J) & 1, p.status);
                if (!ok) break;
                tc_after_sync();
                float x[kTile];
#pragma unroll
                for (int i = 0; i < kTile; i += 32) tmem_ld32(s_at + i, reinterpret_cast<uint32_t *>(x) + i);
                // columns [from, to) of the tile are the row's
                const int kt = k0 + j;
                const int from = kt < tile_lo ? kTile : kt == tile_lo ? col_lo : 0;
                const int to = kt > tile_hi ? 0 : kt == tile_hi ? col_hi + 1 : kTile;
                const uint32_t *valid = s.mask[J % kMaskSlots];
                const bool whole = from == 0 && to == kTile && (valid[0] & valid[1] & valid[2] & valid[3]) == ~0u;
                const bool all = __all_sync(0xffffffffu, whole);
                tmem_wait_ld();
                if (!all) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int a = from - 32 * w, e = to - 32 * w;
                        const uint32_t bits = valid[w] & (e >= 32 ? ~0u : e <= 0 ? 0u : (1u << e) - 1) &
                                              (a >= 32 ? 0u : a <= 0 ? ~0u : ~((1u << a) - 1));
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[32 * w + i] = bits >> i & 1 ? x[32 * w + i] : -INFINITY;
                    }
                }
                float t[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = fmaxf(x[e], x[4 + e]);
#pragma unroll
                for (int i = 8; i < kTile; i += 8)  // (three operands to an instruction)
#pragma unroll
                    for (int e = 0; e < 4; ++e) t[e] = fmaxf(fmaxf(t[e], x[i + e]), x[i + 4 + e]);
                const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
                // move the reference?  (-inf: no column so far, nothing to rescale)
                const bool move = top > m && (m == -INFINITY || (top - m) * c > kMaxSlack);
                const bool rescale = move && m != -INFINITY;
                if (__any_sync(0xffffffffu, rescale)) {
                    const float a = rescale ? exp2_approx((m - top) * c) : 1.f;
                    sum.x *= a;
                    sum.y *= a;
                    // (two streams: the scores came after the previous product)
                    if (STREAMS == 1) ok = wait_bar(s, &s.out[0], (J - 1) & 1, p.status);
                    if (!ok) break;
                    tc_after_sync();
#pragma unroll 1
                    for (int i = 0; i < D; i += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_at + i, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
                        tmem_st32(o_at + i, o);
                    }
                }
                if (move) m = top;
                const float base = m == -INFINITY ? 0.f : -m * c;
                const float2 c2 = make_float2(c, c), b2 = make_float2(base, base);
                // weights in the products' 16 bits, a half of the tile at a time so that
                // its product starts while the other half is formed
                uint32_t w[kTile / 2];
                float2 part[4] = {};
                auto weigh = [&](int from_pair, int to_pair) {
#pragma unroll
                    for (int e = from_pair; e < to_pair; ++e) {
                        float2 y = fma2(make_float2(x[2 * e], x[2 * e + 1]), c2, b2);
                        y = make_float2(exp2_approx(y.x), exp2_approx(y.y));
                        if constexpr (FP8) {  // fp16's rounding (2^-12) stays below the output's: summed as they are
                            const __half2 h = __floats2half2_rn(y.x, y.y);
                            w[e] = *reinterpret_cast<const uint32_t *>(&h);
                            part[e % 4] = add2(part[e % 4], y);
                        } else {
                            w[e] = pack_out(y.x, y.y);
                        }
                    }
                };
                weigh(0, 32);
                tmem_st32(s_at, w);
                weigh(32, 48);
                tmem_wait_st();
                tc_before_sync();
                arrive_issuer(&s.weights[buf][0]);
                weigh(48, 64);
                tmem_st32(s_at + 32, w + 32);
                tmem_wait_st();
                tc_before_sync();
                // the wait after the last tile tells its product from the one before
                // only if that one is known to be done
                if (STREAMS == 1 && j > 0 && j == n - 1) ok = wait_bar(s, &s.out[0], (J - 1) & 1, p.status);
                if (!ok) break;
                arrive_issuer(&s.weights[buf][1]);
                // The sum adds the rounded bf16 weights: where one is far above the
                // others, its rounding then divides out.  (Beside the products.)
                if constexpr (!FP8) {
#pragma unroll
                    for (int e = 0; e < kTile / 2; ++e)
                        part[e % 4] = add2(part[e % 4], make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u)));
                }
                sum = add2(sum, add2(add2(part[0], part[1]), add2(part[2], part[3])));
            }
            tiles += n;
            if (!ok) break;
            // ---- output
            const float l = sum.x + sum.y;
            const bool empty = m == -INFINITY && l == 0.f;  // no column of the item's is the row's
            const int row = it.row0 + r;
            const bool partial = p.splits[it.b] > 1 || p.shared;
            const int64_t at = !mine ? 0 : partial ? part_slot(p, it, it.split, row) : q_row(p, it, row);
            const float inv = __fdiv_rn(p.vscale, l);
            const bool put = mine && !(partial && empty);
            ok = wait_bar(s, &s.out[stream], STREAMS == 1 ? (tiles - 1) & 1 : k & 1, p.status);
            if (ok) {
                tc_after_sync();
                // (scores that are all NaN leave m at -inf, which would read as no column)
                if (mine && partial) p.part_ml[at] = make_float2(l == l ? m * c : 0.f, l);
                bool bad = false;
                // 16 of the warp's rows at a time: a lane has two columns of every eight of
                // rows lane / 4 and lane / 4 + 8, so that a store has 32 bytes (partials) or,
                // with blocks of 4 x 4 lanes transposed, 64 bytes (outputs) of 8 rows each
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    int64_t to[2];
                    float f[2], z[2] = {};
                    bool puts[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int from = h * 16 + e * 8 + lane / 4;
                        to[e] = __shfl_sync(0xffffffffu, at, from) * D;
                        f[e] = __shfl_sync(0xffffffffu, inv, from);
                        puts[e] = __shfl_sync(0xffffffffu, put, from);
                    }
                    float o[16], next_o[16];
                    tmem_ld16(o_at + (h << 20), reinterpret_cast<uint32_t *>(next_o));
#pragma unroll 2
                    for (int i = 0; i < D; i += 32) {
                        tmem_wait_ld();
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] = next_o[x];
                        if (i + 32 < D) tmem_ld16(o_at + (h << 20) + i + 32, reinterpret_cast<uint32_t *>(next_o));
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float2 y[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                y[x] = make_float2(o[4 * x + 2 * e], o[4 * x + 2 * e + 1]);
                                z[e] = __fmaf_rn(y[x].x, 0.f, __fmaf_rn(y[x].y, 0.f, z[e]));
                            }
                            if (partial) {
                                float2 *const out = reinterpret_cast<float2 *>(p.part_o + to[e] + i) + lane % 4;
                                if (puts[e])
#pragma unroll
                                    for (int x = 0; x < 4; ++x) out[4 * x] = y[x];
                            } else {
                                uint32_t v[4];
#pragma unroll
                                for (int x = 0; x < 4; ++x) v[x] = pack_out(y[x].x * f[e], y[x].y * f[e]);
                                transpose4(v, lane % 4);
                                if (puts[e])
                                    reinterpret_cast<uint4 *>(p.out + to[e] + i)[lane % 4] = make_uint4(v[0], v[1], v[2], v[3]);
                            }
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t not_finite = __ballot_sync(0xffffffffu, !(z[e] == 0.f));
                        if (lane / 8 == 2 * h + e) bad = not_finite >> lane % 8 * 4 & 15;
                    }
                }
                bad = bad && put;
                // (read: the next item's products may be added there)
                tc_before_sync();
                arrive_issuer(&s.taken[stream]);
                const uint32_t rows = __ballot_sync(0xffffffffu, bad);
                if (rows && lane == 0) {
                    const int id = it.at * kRowWarps + rank * 4 + warp;
                    p.redo[id] = make_int2((int)rows, atomicExch(&s.redo, id));
                }
            }
            if (!has_item(k + 1)) break;
        }
        // Nothing waits for these warps any more.  (Here and not after the last barrier,
        // where all warps would be left with the few registers of the others: packed fp8
        // prompts of 1 .. 1,501 rows 166 us and 170, although nothing is computed over.)
        sync_warps(C::SOFTMAX_WARPS);
        if (s.redo >= 0 && !s.abort) compute_over<D, FP8>(p, s.redo, STREAMS * CTAS * kTile, warp, C::SOFTMAX_WARPS);
    } else {
        if constexpr (C::MORE_REGS > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::FEWER_REGS));
        if (warp == C::LOAD_WARP) {
            // ---- keys and values of tile j: K0, then K(j + 1) and V(j) in turn
            const int64_t plane = p.pool_pages * p.n_kv_heads * p.page_size;  // rows of a layer's keys
            const int unit = lane / 16, row = lane % 16 * p.page_rows;         // of the lane's page
            int chunk = 0, st = 0, round = 0;  // the next chunk, its place, how often that was filled
            Groups<C> groups;
            const int box_bytes = p.box_rows * 128;
            // the lane's rows of a tile without invalid columns (-1: there is none)
            const int whole = p.pages_per_unit && p.pages_per_unit * p.page_size != C::UNIT ? -1
                              : unit >= C::CTAS || lane % 16 >= max(1, p.pages_per_unit)    ? 0
                                                                                            : min(p.page_size, C::UNIT);
            // the i-th copy of the item
            auto copy = [&](const Page &r, bool values, int i) {
                if constexpr (FP8) {
                    if (round && !wait_bar(s, &s.freed[st], (round - 1) & 1, p.status)) return false;
                } else {
                    const int g = groups.take(st, lane, i);
                    if (round && !wait_bar(s, &s.empty[g % C::GROUPS], (g / C::GROUPS) & 1, p.status)) return false;
                }
                // a pair's keys are split by columns, its values by dimensions
                const bool mine = r.rows > 0 && (values || CTAS == 1 || unit == rank);
                const int boxes = (values ? C::V_BOXES : C::K_BOXES) / (FP8 ? 2 : 1);
                const uint32_t pages = __ballot_sync(0xffffffffu, mine);
                if (elect_one()) {
                    if (pages)
                        mbar_arrive_expect_tx(&s.landed[st], __popc(pages) * box_bytes * boxes);
                    else
                        mbar_arrive(&s.landed[st]);
                }
                __syncwarp();
                // (one elected thread issues: a copy that any lane might make took over 100 cycles)
                uint8_t *const to = FP8 ? raw + st * C::RAW : ring + st * C::CHUNK;
                for (uint32_t left = pages; left; left &= left - 1) {
                    const int from = __ffs(left) - 1;
                    const int32_t y = __shfl_sync(0xffffffffu, r.at, from) + (values ? (int32_t)plane : 0);
                    uint8_t *const dst = to + ((values ? from / 16 * C::UNIT : 0) + from % 16 * p.page_rows) * 128;
                    if (elect_one())
#pragma unroll
                        for (int x = 0; x < C::K_BOXES; ++x)
                            if (x < boxes)
                                tma_load_2d(dst + x * (values ? C::V_BOX : C::K_BOX), &map,
                                            (values ? rank * C::DV : 0) + x * (FP8 ? 128 : 64), y, &s.landed[st]);
                }
                ++chunk;
                if (++st == LANDS) st = 0, ++round;
                return true;
            };
            auto note_mask = [&](const Page &r, int j) {
                // (a tile of whole pages without padding rows)
                if (__all_sync(0xffffffffu, r.rows == whole)) {
                    if (lane < 4) s.mask[j % kMaskSlots][lane] = ~0u;
                    __syncwarp();
                    return;
                }
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int a = unit * C::UNIT + row - 32 * w, e = a + r.rows;  // the lane's columns [a, e) of the word
                    uint32_t bits = 0;
                    if (r.rows > 0 && a < 32 && e > 0)
                        bits = (e >= 32 ? ~0u : (1u << e) - 1) & ~(a > 0 ? (1u << a) - 1 : 0u);
                    bits = __reduce_or_sync(0xffffffffu, bits);
                    if (lane == 0) s.mask[j % kMaskSlots][w] = bits;
                }
                __syncwarp();
            };
            bool ok = true;
            Page now{0, 0}, before{0, 0};  // of the last key tile, of the one before; `coming` and `after` are of the next two
            for (int k = 0, tiles = 0; ok; ++k) {
                const int n = it.k1 - it.k0;
                bool more = true;
                for (int i = 0; ok && i < 2 * n; ++i) {
                    int j;
                    const bool values = value_tile(i, n, j);
                    if (!values) {
                        before = now;
                        now = pages.page(p, coming);
                        note_mask(now, tiles + j);
                    }
                    ok = copy(values && j + 1 < n ? before : now, values, i);
                    if (!ok) break;
                    // the pages of another key tile, or of the next item's first two
                    int kt = it.k0 + j + 2, loads = !values;
                    if (i == 2 * n - 1) {
                        more = has_item(k + 1);
                        if (!more) break;
                        it = s.item[(k + 1) % kItems];
                        pages.of(p, it);
                        kt = it.k0;
                        loads = 2;
                    }
                    for (; loads > 0; --loads, ++kt) {
                        coming = after;
                        after = pages.load(p, kt, it.k1, lane);
                    }
                }
                tiles += n;
                groups.end(n);
                if (!more) break;
            }
            // every commit's arrival is awaited before the CTA ends
            if constexpr (!FP8)
                for (int c = max(0, chunk - LANDS); ok && c < chunk; ++c) {
                    const int g = groups.of(c % LANDS);
                    ok = wait_bar(s, &s.empty[g % C::GROUPS], (g / C::GROUPS) & 1, p.status);
                }
            if (!ok)  // gave up: no copy may still be landing when the CTA ends
                for (int c = max(0, chunk - LANDS); c < chunk; ++c)
                    (void)mbar_wait_bounded(&s.landed[c % LANDS], (c / LANDS) & 1);
        } else if (warp == C::MMA_WARP) {
            // ---- products: one thread (of a pair's first CTA) issues
            constexpr uint32_t QK = mma_desc(CTAS * kTile, kTile, FP8, false), PV = mma_desc(CTAS * kTile, D, FP8, true);
            const uint32_t qk = QK | (p.negate ? kMmaNegateA : 0u);
            const uint32_t q_d = smem_desc(smem_addr(smem), 0), k_d = smem_desc(smem_addr(ring), 0);
            const uint32_t v_d = smem_desc(smem_addr(ring), C::V_BOX);
            if (rank == 1) {  // its part in the questions, while the first CTA issues
                for (int k = 1;; ++k) {
                    if (lane == 0) mbar_arrive_expect_tx(&s.next[k % kItems], sizeof(uint4));
                    __syncwarp();
                    if (!wait_bar(s, &s.next[k % kItems], ((k - 1) / kItems) & 1, p.status)) break;
                    if (answered_cta(&s.answer[k % kItems]) < 0) break;
                }
                (void)mbar_wait_bounded(&s.drained, 0);
            }
            if (rank == 0 && elect_one()) {
                auto wait = [&](uint64_t *bar, uint32_t parity) {
                    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, &s.abort, p.status);
                };
                int chunk = 0, group = 0;  // of the next chunk; groups of the items before
                // the group of the item's i-th chunk is there; its place is free
                auto arrived = [&](int i) {
                    const int g = group + C::group(i);
                    return wait(&s.ready[g % C::GROUPS], (g / C::GROUPS) & 1);
                };
                auto release = [&](int i) { mma_commit<CTAS>(&s.empty[(group + C::group(i)) % C::GROUPS]); };
                // S = Q K^T of a stream into score columns `buf`, keys in chunk c
                auto scores = [&](int stream, int buf, int c) {
                    const uint32_t q = q_d + stream * (kTile * D * 2 / 16), k = k_d + c % STAGES * (C::CHUNK / 16);
                    const uint32_t to = tmem + kScoreCols + buf * kTile;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
                        mma_ss<CTAS>(to, q + (i / 4 * (kTile * 128) + i % 4 * 32) / 16, k + (i / 4 * C::K_BOX + i % 4 * 32) / 16,
                                     qk, i > 0);
                    mma_commit<CTAS>(&s.scores[buf]);
                };
                // O += P V of a stream, half of the weights in score columns `buf`, values in chunk c
                auto product = [&](int stream, int buf, int half, int c, bool add) {
                    const uint32_t v = v_d + c % STAGES * (C::CHUNK / 16) + half * (kTile / 2 * 128 / 16);
                    const uint32_t to = tmem + kOutCols + stream * kTile;
                    const uint32_t w = tmem + kScoreCols + buf * kTile + half * (kTile / 4);
                    mma_ts<CTAS>(to, w, v, PV, add || half > 0);
#pragma unroll
                    for (int i = 1; i < kTile / 32; ++i) mma_ts<CTAS>(to, w + i * 8, v + i * (2048 / 16), PV, true);
                };
                auto ask = [&](int k) {
                    mbar_arrive_expect_tx(&s.next[k % kItems], sizeof(uint4));
                    ask_for_cta<CTAS>(&s.answer[k % kItems], &s.next[k % kItems]);
                };
                bool ok = true;
                int n = s.item[0].k1 - s.item[0].k0;
                for (int k = 0, tiles = 0; ok; ++k) {
                    ok = wait(&s.queries, k & 1) && arrived(0);
                    if (!ok) break;
                    tc_after_sync();
                    for (int st = 0; st < STREAMS; ++st) scores(st, STREAMS == 1 ? tiles & 1 : st, chunk);
                    if (n == 1) mma_commit<CTAS>(&s.scored);
                    release(0);
                    ++chunk;
                    int i = 1;  // chunk of the item
                    // (asked between two runs of tiles: within the loop, 8,192 rows of the 31B shape
                    // on 16,384 took 1,645 us for 1,629)
#pragma unroll 1
                    for (int part = 0, j = 0; ok && part < 2; ++part) {
                        const int end = part ? n : max(0, n - kAskTiles);
                        if (part) ask(k + 1);
                        for (; ok && j < end; ++j) {
                            const int J = tiles + j, k_at = chunk;
                            const bool more = j + 1 < n;
                            if (more) {
                                ok = arrived(i);
                                if (!ok) break;
                                if (STREAMS == 1) {  // the next scores, beside this tile's weights
                                    // (their buffer's weights, of tile j - 1, were multiplied before)
                                    scores(0, (J + 1) & 1, k_at);
                                    if (j + 2 == n) mma_commit<CTAS>(&s.scored);
                                    release(i);
                                }
                                ++i, ++chunk;
                            }
                            if (!C::GROUPED || !more) ok = arrived(i);
                            for (int st = 0; ok && st < STREAMS; ++st) {
                                const int buf = STREAMS == 1 ? J & 1 : st;
                                // (the first product of an item takes the place of the outputs before)
                                if (j == 0 && k > 0) ok = wait(&s.taken[st], (k - 1) & 1);
#pragma unroll
                                for (int half = 0; half < 2; ++half) {
                                    ok = ok && wait(&s.weights[buf][half], (STREAMS == 1 ? J >> 1 : J) & 1);
                                    if (!ok) break;
                                    tc_after_sync();
                                    product(st, buf, half, chunk, j > 0);
                                }
                                if (!ok) break;
                                if (STREAMS == 1 || !more) mma_commit<CTAS>(&s.out[st]);
                                if (STREAMS == 2 && more) scores(st, st, k_at);
                            }
                            if (!ok) break;
                            if (STREAMS == 2 && j + 2 == n) mma_commit<CTAS>(&s.scored);
                            release(i);
                            ++i, ++chunk;
                        }
                    }
                    if (!ok) break;
                    tiles += n;
                    group += C::group(2 * n - 1) + 1;
                    ok = wait(&s.known[(k + 1) % kItems], (k / kItems) & 1);
                    if (!ok || s.item[(k + 1) % kItems].b < 0) break;
                    n = s.item[(k + 1) % kItems].k1 - s.item[(k + 1) % kItems].k0;
                }
                // all products have completed before the tensor memory is given back
                mma_commit<CTAS>(&s.drained);
                (void)mbar_wait_bounded(&s.drained, 0);
            }
            __syncwarp();
        } else if (warp == C::NEXT_WARP) {
            // ---- the next item, for all, and its queries as soon as nothing reads this
            // one's: its first products run beside the output
            for (int k = 0;; ++k) {
                const int slot = (k + 1) % kItems;
                if (!wait_bar(s, &s.next[slot], (k / kItems) & 1, p.status)) break;
                const int x = answered_cta(&s.answer[slot]);
                fence_proxy_async_shared();  // read before another answer lands there
                Item after = item_of(p, max(x, 0) / CTAS, STREAMS * CTAS * kTile);
                if (x < 0) after.b = -1;
                if (lane == 0) {
                    s.item[slot] = after;
                    mbar_arrive(&s.known[slot]);
                }
                __syncwarp();
                if constexpr (!FP8) {
                    Queries<C, C::SOFTMAX_WARPS> q;
                    if (x >= 0) q.find(p, after, first, 0, 1, lane, true);
                    if (!wait_bar(s, &s.scored, k & 1, p.status)) break;
                    if (x < 0) break;
                    q.copy(0, 1, lane, smem);
                    async_wait_all();
                    fence_proxy_async_shared();
                    arrive_issuer(&s.queries, C::SOFTMAX_WARPS);
                }
                if (x < 0) break;
            }
        } else if (!FP8 && warp == C::TIDY_WARP) {
            // ---- value rows that are not valid hold anything: zero weights must meet zeros
            bool ok = true;
            for (int k = 0, tiles = 0, chunk = 0, group = 0; ok; ++k) {
                const int n = s.item[k % kItems].k1 - s.item[k % kItems].k0;
                for (int i = 0; ok && i < 2 * n; ++i, ++chunk) {
                    const int st = chunk % STAGES;
                    ok = wait_bar(s, &s.landed[st], (chunk / STAGES) & 1, p.status);
                    if (!ok) break;
                    int j;
                    if (value_tile(i, n, j)) {
                        const uint32_t *m = s.mask[(tiles + j) % kMaskSlots];
                        if ((m[0] & m[1] & m[2] & m[3]) != ~0u) {
                            uint8_t *v = ring + st * C::CHUNK;
                            for (int r = lane / 8; r < kTile; r += 4)
                                if (!(m[r / 32] >> (r % 32) & 1))
#pragma unroll
                                    for (int x = 0; x < C::V_BOXES; ++x)
                                        reinterpret_cast<uint4 *>(v + x * C::V_BOX + r * 128)[lane % 8] = make_uint4(0, 0, 0, 0);
                            fence_proxy_async_shared();
                        }
                    }
                    // (twice for a group of one)
                    arrive_issuer(&s.ready[(group + C::group(i)) % C::GROUPS], C::GROUPED && (i == 0 || i == 2 * n - 1) ? 2 : 1);
                }
                tiles += n;
                group += C::group(2 * n - 1) + 1;
                ok = ok && has_item(k + 1);
            }
        } else if (FP8 && warp >= C::CONVERT_WARP) {
            // ---- E4M3 codes to fp16 (exact), chunk by chunk
            const int t = threadIdx.x - 32 * C::CONVERT_WARP, u = t % 8;
            bool ok = true;
            Groups<C> groups;
            // the queries of the items after the first, as soon as nothing reads the item's
            // before: its first products run beside the output
            const int from = warp - C::CONVERT_WARP;
            int chunk = 0, k = 0;
            for (int tiles = 0, group = 0; ok; ++k) {
                const int n = s.item[k % kItems].k1 - s.item[k % kItems].k0;
                for (int i = 0; ok && i < 2 * n; ++i, ++chunk) {
                    if (i == 0 && k > 0) {
                        Queries<C, C::SOFTMAX_WARPS / kConvertWarps> q;
                        q.find(p, s.item[k % kItems], first, from, kConvertWarps, lane, true);
                        ok = wait_bar(s, &s.scored, (k - 1) & 1, p.status);
                        if (!ok) break;
                        q.copy(from, kConvertWarps, lane, smem);
                        async_wait_all();
                        q.convert(from, kConvertWarps, lane, smem);
                        fence_proxy_async_shared();
                        arrive_issuer(&s.queries, C::SOFTMAX_WARPS / kConvertWarps);
                    }
                    const int rs = chunk % LANDS, st = chunk % STAGES;
                    int j;
                    const bool values = value_tile(i, n, j);
                    j += tiles;
                    ok = wait_bar(s, &s.landed[rs], (chunk / LANDS) & 1, p.status);
                    const int g = groups.take(st, lane, i);
                    if (ok && chunk >= STAGES) ok = wait_bar(s, &s.empty[g % C::GROUPS], (g / C::GROUPS) & 1, p.status);
                    if (!ok) break;
                    const uint8_t *src = raw + rs * C::RAW;
                    uint8_t *dst = ring + st * C::CHUNK;
                    constexpr int N = C::CHUNK / 2 / (128 * 4 * kConvertWarps);  // rows of 128 codes that a thread has
                    uint4 x[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int r = t / 8 + k * 4 * kConvertWarps;
                        x[k] = *reinterpret_cast<const uint4 *>(src + r * 128 + ((u ^ (r & 7)) << 4));
                    }
                    if (values) {  // rows that are not valid hold anything: zero weights must meet zeros
                        const uint32_t *m = s.mask[j % kMaskSlots];
                        if ((m[0] & m[1] & m[2] & m[3]) != ~0u)
#pragma unroll
                            for (int k = 0; k < N; ++k) {
                                const int r = t / 8 + k * 4 * kConvertWarps;
                                if (!(m[r / 32] >> (r % 32) & 1)) x[k] = make_uint4(0, 0, 0, 0);
                            }
                    }
                    const int box = values ? C::V_BOX : C::K_BOX;
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int r = t / 8 + k * 4 * kConvertWarps;
                        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
                        uint32_t y[8];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint16_t lo = (uint16_t)w[e], hi = (uint16_t)(w[e] >> 16);
                            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y[2 * e]) : "h"(lo));
                            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y[2 * e + 1]) : "h"(hi));
                        }
                        // a pair's keys: two boxes of codes, 64 rows each, become four
                        const int half = values ? 0 : r / C::UNIT, rb = values ? r : r % C::UNIT, u2 = u % 4 * 2;
                        uint8_t *to = dst + (half * 2 + u / 4) * box + rb * 128;
                        // (lanes of the second box take the other half first: 8 lanes, 8 bank groups)
                        const uint4 a = make_uint4(y[0], y[1], y[2], y[3]), b = make_uint4(y[4], y[5], y[6], y[7]);
                        const int odd = u / 4;
                        *reinterpret_cast<uint4 *>(to + (((u2 + odd) ^ (r & 7)) << 4)) = odd ? b : a;
                        *reinterpret_cast<uint4 *>(to + (((u2 + 1 - odd) ^ (r & 7)) << 4)) = odd ? a : b;
                    }
                    fence_proxy_async_shared();
                    arrive_issuer(&s.ready[(group + C::group(i)) % C::GROUPS], C::GROUPED && (i == 0 || i == 2 * n - 1) ? 2 : 1);
                    if (lane == 0) mbar_arrive(&s.freed[rs]);
                }
                tiles += n;
                group += C::group(2 * n - 1) + 1;
                groups.end(n);
                if (!ok || !has_item(k + 1)) break;
            }
            // every commit's arrival is awaited before the CTA ends
            if (ok) ok = wait_bar(s, &s.scored, k & 1, p.status);
            for (int c = max(0, chunk - STAGES); ok && c < chunk; ++c) {
                const int g = groups.of(c % STAGES);
                ok = wait_bar(s, &s.empty[g % C::GROUPS], (g / C::GROUPS) & 1, p.status);
            }
        }
    }
    // (a pair: the other CTA's arrivals and products reach into this one's memory)
    tc_before_sync();
    if constexpr (CTAS == 2)
        cluster_sync();
    else
        __syncthreads();
    tc_after_sync();
    if (warp == C::MMA_WARP) tmem_free<512, CTAS>(tmem);
}

// Joins the splits of each row: a warp per row of the sequences that were split.
template <int D>
__global__ void __launch_bounds__(128) prompt_join_kernel(const __grid_constant__ PromptParams p) {
    constexpr int N = D / 32;
    after_previous();
    let_next_start();  // a few microseconds to its end, and room for the next beside it
    const int rows4 = p.by_units.div(blockIdx.x), unit = blockIdx.x - rows4 * p.n_units;
    const int lane = threadIdx.x & 31, gs = p.log2_group;
    const int64_t row_of_all = (int64_t)rows4 * 4 + threadIdx.x / 32;
    if (row_of_all >= (int64_t)p.first[p.n_seq] << gs) return;
    Item it{};
    it.gs = gs;
    it.b = search(p.first, p.n_seq, row_of_all >> gs);
    if (p.splits[it.b] == 1) return;
    const int row = (int)(row_of_all - ((int64_t)p.first[it.b] << gs));
    it.lr = p.by_kv_heads.div(unit);
    it.g = unit - it.lr * p.n_kv_heads;
    float M = -INFINITY, L = 0.f, o[N] = {};
    for (int i = 0; i < p.splits[it.b]; ++i) M = fmaxf(M, p.part_ml[part_slot(p, it, i, row)].x);
    for (int i = 0; i < p.splits[it.b]; ++i) {
        const int64_t slot = part_slot(p, it, i, row);
        const float2 ml = p.part_ml[slot];
        if (ml.y == 0.f) continue;
        const float a = exp2f(ml.x - M);
        L = __fmaf_rn(ml.y, a, L);
        using Vec = std::conditional_t<N == 2, float2, float4>;
        constexpr int W = sizeof(Vec) / 4;
        float x[N];
#pragma unroll
        for (int e = 0; e < N / W; ++e)
            reinterpret_cast<Vec *>(x)[e] = reinterpret_cast<const Vec *>(p.part_o + slot * D + lane * N)[e];
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = __fmaf_rn(x[e], a, o[e]);
    }
    const float inv = __fdiv_rn(p.vscale, L);
    uint32_t *out = reinterpret_cast<uint32_t *>(p.out + q_row(p, it, row) * D + lane * N);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) out[e] = pack_out(o[2 * e] * inv, o[2 * e + 1] * inv);
}

template <class C>
struct PromptLaunch {
    static cudaError_t run(const PromptParams &p, const CUtensorMap &map, cudaStream_t s) {
        static std::atomic<int> ready[kMaxDevices];  // the shared-memory attribute is per device
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
        if (!ready[dev].load()) {
            e = cudaFuncSetAttribute(prompt_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
            if (e != cudaSuccess) return e;
            ready[dev].store(1);
        }
        if (C::CTAS == 1) return launch_after(prompt_kernel<C>, p.item0[p.n_seq], C::THREADS, C::SMEM, s, p, map);
        cudaLaunchAttribute attr[2]{};
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim = {C::CTAS, 1, 1};
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(p.item0[p.n_seq] * C::CTAS);
        cfg.blockDim = dim3(C::THREADS);
        cfg.dynamicSmemBytes = C::SMEM;
        cfg.stream = s;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        e = cudaLaunchKernelEx(&cfg, prompt_kernel<C>, p, map);
        count_launches(1);
        return e != cudaSuccess ? e : cudaGetLastError();
    }
};

}  // namespace

// Two streams of query tiles unless no sequence has rows for the second (single
// calls on an idle GPU): 8,192
// rows of the 31B shape on 16,384 1,617 us (one stream 2,331), packed fp8 prompts
// of 1 .. 1,501 rows 176 (240); 7 x 40 .. 60 rows, a tile or less, on 3,000 ..
// 5,000 77.5 (one stream 67.8).  (head_dim 256 fills the tensor memory with one.)
int prompt_streams(int head_dim, int64_t most_rows) { return head_dim <= 128 && most_rows > kTile ? 2 : 1; }

// Query rows of a work item, and the CTAs that share it.
int prompt_tile_rows(int head_dim, int streams) { return kTile * (head_dim == 256 ? 2 : streams); }
int prompt_ctas(int head_dim) { return head_dim == 256 ? 2 : 1; }
uint64_t prompt_redo_bytes(int64_t items) { return (uint64_t)items * kRowWarps * sizeof(int2); }

// How pages fill the columns of a key tile.
void prompt_tiling(int page_size, int head_dim, PromptParams *p) {
    const int rows = (page_size + 7) / 8 * 8;
    p->unit = kTile / prompt_ctas(head_dim);
    p->page_rows = rows;
    p->pages_per_unit = rows <= p->unit ? p->unit / rows : 0;
    p->units_per_page = (page_size + p->unit - 1) / p->unit;
    p->box_rows = std::min(rows, p->unit);
}

cudaError_t launch_prompt(int head_dim, bool fp8, int streams, const PromptParams &p, const CUtensorMap &map,
                          cudaStream_t s) {
    if (head_dim == 64 && !fp8)
        return streams == 2 ? PromptLaunch<Cfg<64, false, 2>>::run(p, map, s) : PromptLaunch<Cfg<64, false, 1>>::run(p, map, s);
    if (head_dim == 128 && !fp8)
        return streams == 2 ? PromptLaunch<Cfg<128, false, 2>>::run(p, map, s) : PromptLaunch<Cfg<128, false, 1>>::run(p, map, s);
    if (head_dim == 128)
        return streams == 2 ? PromptLaunch<Cfg<128, true, 2>>::run(p, map, s) : PromptLaunch<Cfg<128, true, 1>>::run(p, map, s);
    if (head_dim == 256)
        return fp8 ? PromptLaunch<Cfg<256, true, 1>>::run(p, map, s) : PromptLaunch<Cfg<256, false, 1>>::run(p, map, s);
    return cudaErrorInvalidValue;
}

cudaError_t launch_prompt_join(int head_dim, const PromptParams &p, cudaStream_t s) {
    const int64_t grid = ((((int64_t)p.first[p.n_seq] << p.log2_group) + 3) / 4) * p.n_units;
    switch (head_dim) {
        case 64: return launch_after(prompt_join_kernel<64>, (unsigned)grid, 128, 0, s, p);
        case 128: return launch_after(prompt_join_kernel<128>, (unsigned)grid, 128, 0, s, p);
        case 256: return launch_after(prompt_join_kernel<256>, (unsigned)grid, 128, 0, s, p);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
