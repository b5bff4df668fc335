// weigh_kernels.cu — the weight that each cached row received from a prompt's
// rows, on the 5th-generation tensor cores:
//   weight[j] = sum over layers, query heads and rows i that attend to j of
//               2^(c s_ij - lse_i),   lse_i = log2 sum_j 2^(c s_ij),  c = scale log2(e)
// The prompt kernel leaves each row's lse.  The scores are formed a second time,
// the other way round: keys are the rows of a tile (tensor memory lanes), so that
// a thread has a key and adds up its row of weights in registers; no weight leaves
// the SM.  One row of sums per work item goes to memory, and a last pass adds those
// of all KV heads, layers and query ranges in a fixed order.
//
// A work item is a KV head, two tiles of 128 keys and a range of query tiles (128
// token x head rows).  For head_dim up to 128 one CTA has both key tiles; for 256 a
// pair of CTAs has one each and half of every query tile.  An item's keys are put
// into tensor memory once, query tiles stream through a ring of copies; scores have
// two or three buffers in tensor memory, so that a tile's products run beside the
// exponentials of the one before.
//
// What bounds it: the products, and the hand-overs between warps.  2,047 rows of the
// 12B shape on 6,145: 81 us, of which the products alone are 59; with the CTAs' shares
// less even than now, and their items worked out one by one, 92, of that 77 without sums, 84 without the rows' logarithms
// from shared memory, and 92 with sixteen summing warps or a third score buffer too.
// With both operands in shared memory that memory's 128 bytes a cycle bounded it (a
// pair's products of 128 keys and 128 rows read 8 KB in their 64 cycles).
//
// Few rows on long contexts are bound by what an item costs beside its products: 17
// sequences of 65 to 125 rows on 3,872 to 5,027 of the 31B shape 308 us a call with
// items worked out one by one, 265 so.
//
// CTAs are persistent: item by item, the ring of query tiles running on from one to
// the next, and the next item's keys on their way while one is worked on.
//
// Warps: eight form and sum weights, four put keys into tensor memory (of an fp8
// cache as fp16, exact), one loads, one thread issues products, in a pair one hands
// the query tiles over to the first CTA's issuing thread.
#include <math.h>

#include "prompt.cuh"

namespace kvg {

namespace {

template <int D_, bool FP8_>
struct Weigh {
    static constexpr int D = D_;
    static constexpr bool FP8 = FP8_, PAIR = D == 256;
    static constexpr int CTAS = PAIR ? 2 : 1, STREAMS = PAIR ? 1 : 2;  // key tiles of a CTA
    static constexpr int KEYS = kTile * D * (FP8 ? 1 : 2);             // bytes of a key tile
    static constexpr int Q_ROWS = kTile / CTAS, Q_BYTES = Q_ROWS * D * 2;  // a CTA's part of a query tile
    static constexpr int STAGES = D == 64 ? 6 : 4;
    // tensor memory: score buffers, then the keys' (D / 2 columns a tile), of a pair two
    static constexpr int SCORES = PAIR ? 2 : 3, KEY_SETS = PAIR ? 2 : 1, KEY_COL = SCORES * kTile;
    static_assert(KEY_COL + KEY_SETS * STREAMS * D / 2 <= 512, "tensor memory");
    static constexpr int SUM_WARPS = 8, KEY_WARP = 8, LOAD_WARP = 12, MMA_WARP = 13, RELAY_WARP = 14;
    static constexpr int THREADS = 32 * (PAIR ? 15 : 14);
    static constexpr int LINES = 2 / STREAMS;                          // a key's sums: a pair's CTA has two warps to it
    static constexpr int COLS = kTile / LINES;                         // of a query tile that a summing warp has
    static constexpr int SMEM = STREAMS * KEYS + STAGES * Q_BYTES + 1024;
    static_assert(SMEM <= 210 * 1024, "shared memory beside the barriers, the logarithms and the items");
};

// Of the launch: a KV head of a layer, a pair of key tiles, a range of query tiles.
struct WeighItem {
    int n, q0;               // query tiles [q0, q0 + n)
    int rows;                // query rows of the sequence, token x head
    int tile;                // first key tile
    int seq, slot0, solid, head;  // head: first query head
    int token, key;          // first row of the queries; of the KV head's plane in the pool
    int line, pad;           // floats between the lines of sums
    int64_t lse, sums;       // the sequence's logarithms; the first line of sums, its first key
};
__device__ __forceinline__ WeighItem weigh_item(const WeighParams &w, int at) {
    const PromptParams &p = w.p;
    WeighItem it;
    const int b = search(w.item0, p.n_seq, at), splits = w.splits[b];
    const int units = w.n_lr * p.n_kv_heads, of_seq = at - w.item0[b], of_unit = of_seq / units;
    const int unit = of_seq - of_unit * units, lr = w.lr0 + unit / p.n_kv_heads, g = unit % p.n_kv_heads;
    const int block = of_unit / splits, split = of_unit - block * splits, gs = p.log2_group;
    const int n = p.first[b + 1] - p.first[b], row0 = p.row0[b];
    it.rows = n << gs;
    it.tile = w.tile0[b] + 2 * block;
    it.seq = p.seq[b];
    it.slot0 = p.slot0[b];
    it.solid = p.solid[b];
    it.head = g << gs;
    it.token = p.qlayers[lr] * (int)p.q_rows + row0;
    it.key = (int)(((int64_t)p.layers[lr] * 2 * p.pool_pages * p.n_kv_heads + g) * p.page_size);
    it.line = 2 * w.blocks[b] * kTile;
    it.pad = 0;
    it.lse = ((int64_t)(lr * p.n_kv_heads + g) * p.q_rows + row0) << gs;
    it.sums = w.sum0[b] + ((int64_t)split * units + unit) * w.lines * it.line + 2 * block * kTile;
    // the tokens that may attend to its slots
    const int from = first_slot(p, it.tile), end = first_slot(p, it.tile + 2);
    const int t0 = max(0, from - it.slot0);
    const int64_t reach = p.window > 0 ? (int64_t)end - 1 + p.window - it.slot0 + w.gaps[b] : n;
    const int t1 = (int)min((int64_t)n, max(reach, (int64_t)0));
    const int a = (t0 << gs) / kTile, e = max(a, ((t1 << gs) + kTile - 1) / kTile), len = e - a;
    it.q0 = a + (int)((int64_t)len * split / splits);
    it.n = t0 < t1 ? a + (int)((int64_t)len * (split + 1) / splits) - it.q0 : 0;
    return it;
}

constexpr int kItemsAhead = 96;  // of a CTA, worked out at its start, a thread each
struct WeighBars {
    uint64_t k_landed, k_taken;              // keys: there; their place is free
    uint64_t k_ready[2], k_free[2];          // in tensor memory (of a pair both); multiplied
    uint64_t landed[8], ready[8], empty[8];  // query tiles: there; in both CTAs; multiplied
    uint64_t scores[3], taken[3];            // of a buffer: there; read
    uint64_t drained;
    uint32_t tmem;
    int abort;
    alignas(16) float lse[8][2][kTile];      // of each summing warp: minus lse of its rows of two tiles
    alignas(16) WeighItem items[kItemsAhead];
};

__device__ __forceinline__ bool wait_weigh(WeighBars &s, uint64_t *bar, uint32_t parity, DevStatus *status) {
    const bool ok = mbar_try_wait(bar, parity) || wait_slow(bar, parity, &s.abort, status);
    return __all_sync(0xffffffffu, ok);
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1)
    weigh_kernel(const __grid_constant__ WeighParams w, const __grid_constant__ CUtensorMap k_map,
                 const __grid_constant__ CUtensorMap q_map) {
    constexpr int D = C::D, STREAMS = C::STREAMS, STAGES = C::STAGES, CTAS = C::CTAS;
    constexpr bool FP8 = C::FP8;
    const PromptParams &p = w.p;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ WeighBars s;
    uint8_t *const keys = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    uint8_t *const ring = keys + STREAMS * C::KEYS;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;  // uniform in the warp
    const int rank = CTAS == 2 ? (int)cluster_rank() : 0;
    auto arrive_issuer = [&](uint64_t *bar) {  // a warp, for its lanes together
        __syncwarp();
        if (lane == 0) {
            if constexpr (CTAS == 2)
                mbar_arrive_first(bar);
            else
                mbar_arrive(bar);
        }
    };
    if (threadIdx.x == 0) {
        mbar_init(&s.k_landed, 1);
        mbar_init(&s.k_taken, 4);
        for (int i = 0; i < C::KEY_SETS; ++i) {
            mbar_init(&s.k_ready[i], CTAS * 4);
            mbar_init(&s.k_free[i], 1);
        }
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&s.landed[i], 1);
            mbar_init(&s.ready[i], CTAS);
            mbar_init(&s.empty[i], 1);
        }
        for (int i = 0; i < C::SCORES; ++i) {
            mbar_init(&s.scores[i], 1);
            mbar_init(&s.taken[i], CTAS * C::SUM_WARPS / STREAMS);
        }
        mbar_init(&s.drained, 1);
        s.abort = 0;
        fence_mbar_init();
    }
    // The CTA's items: one of each round of grid / CTAS, every other round backwards (the
    // items of a sequence get shorter).  Working one out takes 3,000 cycles where the
    // launch's parameters are not in the constant cache.
    const int n_at = gridDim.x / CTAS, me = blockIdx.x / CTAS, n_items = w.item0[p.n_seq];
    auto item_of = [&](int round) { return round * n_at + (round & 1 ? n_at - 1 - me : me); };
    if (threadIdx.x < kItemsAhead && item_of(threadIdx.x) < n_items) s.items[threadIdx.x] = weigh_item(w, item_of(threadIdx.x));
    if (warp == C::MMA_WARP) tmem_alloc<512, CTAS>(&s.tmem);
    tc_before_sync();
    if constexpr (CTAS == 2)
        cluster_sync();
    else
        __syncthreads();
    tc_after_sync();
    after_previous();
    const uint32_t tmem = s.tmem;
    const int gs = p.log2_group;
    // tiles: query tiles of the items before; items: how many of those had any.
    auto each_item = [&](auto &&work) {
        int tiles = 0, items = 0;
        for (int round = 0;; ++round) {
            const int at = item_of(round);
            if (at >= n_items) return;
            WeighItem it;
            if (round < kItemsAhead)
                it = s.items[round];
            else
                it = weigh_item(w, at);
            if (!work(it, tiles, items)) return;
            tiles += it.n;
            items += it.n > 0;
        }
    };

    if (warp < C::SUM_WARPS) {
        each_item([&](const WeighItem &it, int tiles, int items) {
            // ---- a thread has a key
            const int stream = STREAMS == 2 ? warp / 4 : 0, half = STREAMS == 2 ? 0 : warp / 4;
            const int shift = STREAMS == 2 ? stream : rank, col = warp % 4 * 32 + lane, n = it.n, rows = it.rows;
            // its slot
            const int u = (it.tile + shift) * (kTile / p.unit) + col / p.unit, c0 = col % p.unit;
            int pg, r0;
            bool valid;
            if (p.pages_per_unit) {
                const int place = c0 / p.page_rows;
                pg = u * p.pages_per_unit + place;
                r0 = c0 - place * p.page_rows;
                valid = place < p.pages_per_unit && r0 < p.page_size;
            } else {
                pg = p.by_pages.div(u);
                r0 = (u - pg * p.units_per_page) * p.unit + c0;
                valid = r0 < p.page_size;
            }
            const int slot0 = it.slot0, slot = pg * p.page_size + r0;
            valid = valid && slot < slot0 + (rows >> gs);
            const int32_t *fill = p.page_fill + (int64_t)it.seq * p.max_pages;
            const int filled = valid ? fill[pg] : 0;
            // the logarithms of the first tiles, beside it
            bool ok = true;
            constexpr int COLS = C::COLS, PER = COLS / 32;  // PER: logarithms that a lane fetches
            const float *lse = p.row_lse + it.lse;
            float *const mine[2] = {s.lse[warp][0], s.lse[warp][1]};
            // of the tile after this one, and of the one after that: their loads take as long as a tile
            float next[PER], after[PER];
            auto fetch = [&](int i, float (&to)[PER]) {
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    const int r = (it.q0 + i) * kTile + half * COLS + k * 32 + lane;
                    to[k] = i < n && r < rows ? lse[r] : INFINITY;  // (2^-inf: no weight)
                }
            };
            fetch(0, next);
            fetch(1, after);
            // the query rows [lo, hi) of the sequence that attend to it
            int lo = 0, hi = rows;
            valid = r0 < filled;
            if (valid) {
                lo = max(0, slot - slot0) << gs;
                if (p.window > 0) {
                    // valid rows from here up to the query rows
                    int64_t between = (int64_t)slot0 - slot;
                    if (slot < it.solid) {
                        between = filled - r0;
                        const int end = slot0 / p.page_size;
                        for (int i = pg + 1; i < end && between < p.window; ++i) between += fill[i];
                        if (end > pg) between += slot0 - end * p.page_size;
                        else between = slot0 - slot;
                    }
                    hi = (int)max((int64_t)0, min((int64_t)(rows >> gs), p.window - between)) << gs;
                }
            }
            auto put = [&](int buf) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < PER; ++i) mine[buf][i * 32 + lane] = -next[i];
                __syncwarp();
            };
            const float c = p.negate ? -p.qscale : p.qscale;
            const float2 c2 = make_float2(c, c);
            const uint32_t at = tmem + ((uint32_t)(warp % 4) << 21) + half * COLS;
            float2 sum[4] = {};
            put(0);
            for (int i = 0; ok && i < n; ++i) {
                const int t = (tiles + i) * STREAMS + stream, buf = t % C::SCORES, lbuf = i & 1, row0 = (it.q0 + i) * kTile + half * COLS;
#pragma unroll
                for (int k = 0; k < PER; ++k) next[k] = after[k];
                fetch(i + 2, after);
                ok = wait_weigh(s, &s.scores[buf], (t / C::SCORES) & 1, p.status);
                if (!ok) break;
                tc_after_sync();
                const bool whole = !valid || (lo <= row0 && hi >= row0 + COLS);
                const bool all = __all_sync(0xffffffffu, whole);
                float x[64];
#pragma unroll
                for (int j = 0; j < COLS; j += 64) {
                    const int left = rows - row0 - j;  // of the sequence's rows
                    if (j > 0 && left <= 0) break;
                    tmem_ld32(at + buf * kTile + j, reinterpret_cast<uint32_t *>(x));
                    tmem_ld32(at + buf * kTile + j + 32, reinterpret_cast<uint32_t *>(x) + 32);
                    tmem_wait_ld();
                    if (j + 64 == COLS || left <= 64) {  // the next scores may be put there
                        tc_before_sync();
                        arrive_issuer(&s.taken[buf]);
                    }
                    auto add = [&](int r, float2 y0, float2 y1) {
                        sum[r / 2 % 4] = add2(sum[r / 2 % 4], make_float2(exp2_approx(y0.x), exp2_approx(y0.y)));
                        sum[r / 2 % 4 + 1] = add2(sum[r / 2 % 4 + 1], make_float2(exp2_approx(y1.x), exp2_approx(y1.y)));
                    };
                    if (all) {
#pragma unroll
                        for (int r = 0; r < 64; r += 4) {
                            const float4 l = *reinterpret_cast<const float4 *>(&mine[lbuf][j + r]);
                            add(r, fma2(make_float2(x[r], x[r + 1]), c2, make_float2(l.x, l.y)),
                                fma2(make_float2(x[r + 2], x[r + 3]), c2, make_float2(l.z, l.w)));
                        }
                    } else {
                        const int a = lo - row0 - j, e = hi - row0 - j;
                        const uint64_t bits = (e >= 64 ? ~0ull : e <= 0 ? 0ull : (1ull << e) - 1) &
                                              (a >= 64 ? 0ull : a <= 0 ? ~0ull : ~((1ull << a) - 1));
#pragma unroll
                        for (int r = 0; r < 64; r += 4) {
                            const float4 l = *reinterpret_cast<const float4 *>(&mine[lbuf][j + r]);
                            float2 y0 = fma2(make_float2(x[r], x[r + 1]), c2, make_float2(l.x, l.y));
                            float2 y1 = fma2(make_float2(x[r + 2], x[r + 3]), c2, make_float2(l.z, l.w));
                            y0.x = bits >> r & 1 ? y0.x : -INFINITY;
                            y0.y = bits >> (r + 1) & 1 ? y0.y : -INFINITY;
                            y1.x = bits >> (r + 2) & 1 ? y1.x : -INFINITY;
                            y1.y = bits >> (r + 3) & 1 ? y1.y : -INFINITY;
                            // (or the compiler makes one form of both, with a selection for every weight)
                            asm volatile("" : "+f"(y0.x), "+f"(y0.y), "+f"(y1.x), "+f"(y1.y));
                            add(r, y0, y1);
                        }
                    }
                }
                put(lbuf ^ 1);
            }
            if (!ok) return false;
            const float2 total = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
            w.sums[it.sums + half * it.line + shift * kTile + col] = valid ? total.x + total.y : 0.f;
            return true;
        });
    } else if (warp < C::KEY_WARP + 4) {
        // ---- keys from shared to tensor memory: a thread has a key of each tile, 64
        // elements (of a bf16 cache 128 swizzled bytes, of an fp8 cache 64) at a time
        const int row = warp % 4 * 32 + lane;
        each_item([&](const WeighItem &it, int tiles, int items) {
            if (it.n == 0) return true;
            const int set = items % C::KEY_SETS;
            if (!wait_weigh(s, &s.k_landed, items & 1, p.status)) return false;
            if (items >= C::KEY_SETS && !wait_weigh(s, &s.k_free[set], (items / C::KEY_SETS - 1) & 1, p.status)) return false;
            tc_after_sync();
#pragma unroll
            for (int st = 0; st < STREAMS; ++st)
#pragma unroll
                for (int x = 0; x < D / 64; ++x) {
                    uint32_t y[32];
                    const uint8_t *from = keys + st * C::KEYS + (FP8 ? x / 2 : x) * (kTile * 128) + row * 128;
#pragma unroll
                    for (int u = 0; u < (FP8 ? 4 : 8); ++u) {
                        const int chunk = FP8 ? x % 2 * 4 + u : u;
                        const uint4 v = *reinterpret_cast<const uint4 *>(from + ((chunk ^ (row & 7)) << 4));
                        const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if constexpr (FP8) {
                                const uint16_t a = (uint16_t)words[e], b = (uint16_t)(words[e] >> 16);
                                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y[8 * u + 2 * e]) : "h"(a));
                                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y[8 * u + 2 * e + 1]) : "h"(b));
                            } else {
                                y[4 * u + e] = words[e];
                            }
                        }
                    }
                    tmem_st32(tmem + ((uint32_t)(warp % 4) << 21) + C::KEY_COL + (set * STREAMS + st) * (D / 2) + x * 32, y);
                }
            tmem_wait_st();
            tc_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.k_taken);
            arrive_issuer(&s.k_ready[set]);
            return true;
        });
    } else if (warp == C::LOAD_WARP) {
        bool ok = true;
        int i = 0, k = 0;  // query tiles and keys that were asked for
        each_item([&](const WeighItem &it, int tiles, int items) {
            // ---- the keys of the CTA's tiles, then its part of each query tile
            const int n = it.n;
            if (n == 0) return true;
            const int64_t entry = (int64_t)it.seq * p.max_pages;
            const int slot_end = it.slot0 + (it.rows >> gs), last = (slot_end - 1) / p.page_size;
            const int per = kTile / p.unit, unit = lane / 16, place = lane % 16;
            constexpr int BOXES = FP8 ? D / 128 : D / 64;
            int32_t y[STREAMS];
            uint32_t has[STREAMS];
            int boxes = 0;
#pragma unroll
            for (int st = 0; st < STREAMS; ++st) {
                const int u = (it.tile + (STREAMS == 2 ? st : rank)) * per + unit;
                int pg = u * p.pages_per_unit + place, sub = 0;
                bool mine = unit < per && place < p.pages_per_unit;
                if (!p.pages_per_unit) {
                    pg = u / p.units_per_page;
                    sub = (u - pg * p.units_per_page) * p.unit;
                    mine = unit < per && place == 0;
                }
                mine = mine && pg <= last;
                int pid = 0;
                if (mine) {
                    pid = p.page_table[entry + pg];
                    mine = p.page_fill[entry + pg] > sub;
                    if (mine && (pid < 0 || pid >= p.pool_pages)) {
                        record_error(p.status, KVG_ERR_DEVICE_CHECK, 31);
                        mine = false;
                    }
                }
                y[st] = it.key + pid * (p.n_kv_heads * p.page_size) + sub;
                has[st] = __ballot_sync(0xffffffffu, mine);
                boxes += __popc(has[st]);
            }
            const int token0 = it.token + ((rank * C::Q_ROWS) >> gs);
            auto load = [&](int t) {
                const int st = i % STAGES;
                if (i >= STAGES) ok = wait_weigh(s, &s.empty[st], (i / STAGES - 1) & 1, p.status);
                if (!ok) return;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&s.landed[st], C::Q_BYTES);
#pragma unroll
                    for (int x = 0; x < D / 64; ++x)
                        tma_load_3d(ring + st * C::Q_BYTES + x * (C::Q_ROWS * 128), &q_map, x * 64, it.head,
                                    token0 + (((it.q0 + t) * kTile) >> gs), &s.landed[st]);
                }
                __syncwarp();
                ++i;
            };
            if (items > 0) ok = wait_weigh(s, &s.k_taken, (items - 1) & 1, p.status);
            if (!ok) return false;
            ++k;
            if (elect_one()) {
                if (boxes)
                    mbar_arrive_expect_tx(&s.k_landed, boxes * p.box_rows * 128 * BOXES);
                else
                    mbar_arrive(&s.k_landed);
            }
            __syncwarp();
#pragma unroll
            for (int st = 0; st < STREAMS; ++st)
                for (uint32_t left = has[st]; left; left &= left - 1) {
                    const int from = __ffs(left) - 1;
                    const int32_t row = __shfl_sync(0xffffffffu, y[st], from);
                    uint8_t *const to = keys + st * C::KEYS + (from / 16 * p.unit + from % 16 * p.page_rows) * 128;
                    if (elect_one())
#pragma unroll
                        for (int x = 0; x < BOXES; ++x)
                            tma_load_2d(to + x * (kTile * 128), &k_map, x * (FP8 ? 128 : 64), row, &s.k_landed);
                }
            for (int t = 0; ok && t < n; ++t) load(t);
            return ok;
        });
        // no copy may still be landing, nor a commit arriving, when the CTA ends
        if (k > 0) (void)mbar_wait_bounded(&s.k_landed, (k - 1) & 1);
        for (int t = max(0, i - STAGES); t < i; ++t) {
            (void)mbar_wait_bounded(&s.landed[t % STAGES], (t / STAGES) & 1);
            if (ok) ok = wait_weigh(s, &s.empty[t % STAGES], (t / STAGES) & 1, p.status);
        }
        for (int t = max(0, k - C::KEY_SETS); ok && t < k; ++t)
            ok = wait_weigh(s, &s.k_free[t % C::KEY_SETS], (t / C::KEY_SETS) & 1, p.status);
        if (rank == 1 && k > 0) (void)mbar_wait_bounded(&s.drained, 0);  // (the first CTA's commits reach this one's barriers)
    } else if (warp == C::MMA_WARP) {
        if (rank == 0 && elect_one()) {
            constexpr uint32_t KQ = mma_desc(CTAS * kTile, kTile, FP8, false);
            const uint32_t q_d = smem_desc(smem_addr(ring), 0);
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                return mbar_try_wait(bar, parity) || wait_slow(bar, parity, &s.abort, p.status);
            };
            constexpr bool DIRECT = CTAS == 1;  // the copies' own barriers
            bool any = false;
            each_item([&](const WeighItem &it, int tiles, int items) {
                const int n = it.n;
                if (n == 0) return true;
                any = true;
                const int set = items % C::KEY_SETS;
                bool ok = wait(&s.k_ready[set], (items / C::KEY_SETS) & 1);
                for (int i = tiles; ok && i < tiles + n; ++i) {
                    const int st = i % STAGES;
                    ok = wait(DIRECT ? &s.landed[st] : &s.ready[st], (i / STAGES) & 1);
                    for (int stream = 0; ok && stream < STREAMS; ++stream) {
                        const int t = i * STREAMS + stream, buf = t % C::SCORES;
                        if (t >= C::SCORES) ok = wait(&s.taken[buf], (t / C::SCORES - 1) & 1);
                        if (!ok) break;
                        tc_after_sync();
                        const uint32_t k = tmem + C::KEY_COL + (set * STREAMS + stream) * (D / 2);
                        const uint32_t q = q_d + st * (C::Q_BYTES / 16), to = tmem + buf * kTile;
#pragma unroll
                        for (int x = 0; x < D / 16; ++x)
                            mma_ts<CTAS>(to, k + x * 8, q + (x / 4 * (C::Q_ROWS * 128) + x % 4 * 32) / 16, KQ, x > 0);
                        mma_commit<CTAS>(&s.scores[buf]);
                    }
                    if (ok) mma_commit<CTAS>(&s.empty[st]);
                }
                if (ok) mma_commit<CTAS>(&s.k_free[set]);
                return ok;
            });
            // all products have completed before the tensor memory is given back
            if (any) {
                mma_commit<CTAS>(&s.drained);
                (void)mbar_wait_bounded(&s.drained, 0);
            }
        }
        __syncwarp();
    } else if (warp == C::RELAY_WARP) {
        // ---- a pair: the query tiles that have landed here, for the first CTA's issuing thread
        each_item([&](const WeighItem &it, int tiles, int items) {
            bool ok = true;
            for (int i = tiles; ok && i < tiles + it.n; ++i) {
                ok = wait_weigh(s, &s.landed[i % STAGES], (i / STAGES) & 1, p.status);
                if (ok) arrive_issuer(&s.ready[i % STAGES]);
            }
            return ok;
        });
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

// A block: kSlots slots of a sequence, kLines threads for each that share the lines
// of sums.
constexpr int kSlots = 64, kLines = 4;
__global__ void __launch_bounds__(kSlots * kLines) weigh_sum_kernel(const __grid_constant__ WeighParams w) {
    const PromptParams &p = w.p;
    __shared__ float part[kLines][kSlots];
    const int b = blockIdx.y, x = threadIdx.x % kSlots, line = threadIdx.x / kSlots;
    const int n = p.slot0[b] + p.first[b + 1] - p.first[b], slot = blockIdx.x * kSlots + x;
    if (blockIdx.x * kSlots >= n) return;
    after_previous();
    float sum = 0.f;
    if (slot < n) {
        const int pg = p.by_page.div(slot);
        int tile, col;
        tile_of(p, slot, tile, col);
        tile -= w.tile0[b];
        if (tile >= 0 && slot - pg * p.page_size < p.page_fill[(int64_t)p.seq[b] * p.max_pages + pg]) {
            const int lines = w.splits[b] * w.n_lr * p.n_kv_heads * w.lines;
            const int64_t step = (int64_t)2 * w.blocks[b] * kTile;
            const float *s = w.sums + w.sum0[b] + (int64_t)tile * kTile + col;
#pragma unroll 8
            for (int i = line; i < lines; i += kLines) sum += s[i * step];
        }
    }
    part[line][x] = sum;
    __syncthreads();
    if (line > 0 || slot >= n) return;
#pragma unroll
    for (int i = 1; i < kLines; ++i) sum += part[i][x];
    float *to = w.weights + (int64_t)p.seq[b] * w.max_slots + slot;
    const float decay = w.met[b] ? 1.f : w.decay;
    *to = decay == 0.f ? sum : __fmaf_rn(decay, *to, sum);
}

// bf16 queries as fp16, as products with an fp8 cache's codes take them; n: a multiple of 8.
__global__ void __launch_bounds__(256) query_halves_kernel(const uint4 *q, int64_t n8, uint4 *out) {
    after_previous();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n8; i += (int64_t)gridDim.x * blockDim.x) {
        const uint4 x = q[i];
        uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __half2 h = __floats2half2_rn(__uint_as_float(y[e] << 16), __uint_as_float(y[e] & 0xffff0000u));
            y[e] = *reinterpret_cast<const uint32_t *>(&h);
        }
        out[i] = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

template <class C>
cudaError_t run_weigh(const WeighParams &w, const CUtensorMap &k_map, const CUtensorMap &q_map, int n_sm, cudaStream_t s) {
    static std::atomic<int> ready[kMaxDevices];  // the shared-memory attribute is per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (!ready[dev].load()) {
        e = cudaFuncSetAttribute(weigh_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev].store(1);
    }
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {C::CTAS, 1, 1};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(std::min(w.item0[w.p.n_seq], n_sm / C::CTAS) * C::CTAS);
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = C::CTAS == 2 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, weigh_kernel<C>, w, k_map, q_map);
    count_launches(1);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_prompt_lse(int head_dim, bool fp8, int streams, const PromptParams &p, const CUtensorMap &map,
                              cudaStream_t s) {
    if (head_dim == 64 && !fp8)
        return streams == 2 ? PromptLaunch<Cfg<64, false, 2, true>>::run(p, map, s)
                            : PromptLaunch<Cfg<64, false, 1, true>>::run(p, map, s);
    if (head_dim == 128 && !fp8)
        return streams == 2 ? PromptLaunch<Cfg<128, false, 2, true>>::run(p, map, s)
                            : PromptLaunch<Cfg<128, false, 1, true>>::run(p, map, s);
    if (head_dim == 128)
        return streams == 2 ? PromptLaunch<Cfg<128, true, 2, true>>::run(p, map, s)
                            : PromptLaunch<Cfg<128, true, 1, true>>::run(p, map, s);
    if (head_dim == 256)
        return fp8 ? PromptLaunch<Cfg<256, true, 1, true>>::run(p, map, s)
                   : PromptLaunch<Cfg<256, false, 1, true>>::run(p, map, s);
    return cudaErrorInvalidValue;
}

int weigh_lines(int head_dim) { return head_dim == 256 ? Weigh<256, false>::LINES : Weigh<128, false>::LINES; }
int weigh_tokens(int head_dim, int group) { return (head_dim == 256 ? kTile / 2 : kTile) / group; }

cudaError_t launch_query_halves(const void *q, int64_t n, void *out, int n_sm, cudaStream_t s) {
    const int64_t grid = std::min<int64_t>((n / 8 + 255) / 256, 8 * (int64_t)n_sm);
    return launch_after(query_halves_kernel, (unsigned)grid, 256, 0, s, static_cast<const uint4 *>(q), n / 8,
                        static_cast<uint4 *>(out));
}

cudaError_t launch_weigh(int head_dim, bool fp8, const WeighParams &w, const CUtensorMap &k_map, const CUtensorMap &q_map,
                         int n_sm, cudaStream_t s) {
    switch (head_dim) {
        case 64: return run_weigh<Weigh<64, false>>(w, k_map, q_map, n_sm, s);
        case 128: return fp8 ? run_weigh<Weigh<128, true>>(w, k_map, q_map, n_sm, s) : run_weigh<Weigh<128, false>>(w, k_map, q_map, n_sm, s);
        case 256: return fp8 ? run_weigh<Weigh<256, true>>(w, k_map, q_map, n_sm, s) : run_weigh<Weigh<256, false>>(w, k_map, q_map, n_sm, s);
    }
    return cudaErrorInvalidValue;
}

cudaError_t launch_weigh_sum(const WeighParams &w, cudaStream_t s) {
    int most = 0;
    for (int b = 0; b < w.p.n_seq; ++b) most = std::max(most, w.p.slot0[b] + w.p.first[b + 1] - w.p.first[b]);
    return launch_after(weigh_sum_kernel, dim3((most + kSlots - 1) / kSlots, w.p.n_seq), kSlots * kLines, 0, s, w);
}

}  // namespace kvg
