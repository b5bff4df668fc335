// evict_kernels.cu — a sequence thinned to a number of its rows: the first few,
// the last ones, and of those in between the ones of most weight (a restored
// context, Sec. 4.4, that has to take less room).
//
// Of n rows with weights w the kept ones are i < first, i >= n - last, and the m
// heaviest others, m = rows - first - last; of equal weights the earlier.  They
// keep their order, so the j-th kept row moves from slot s_j >= j to slot j.
//
// Selection: a cluster of CTAs per sequence, a thread up to four slots at a time.
// The m-th largest weight is found digit by digit (8 bits of a key that orders like
// the weights), each digit a histogram of the rows that agree so far, the CTAs'
// added up through their shared memories; then ballots rank the rows that are kept
// for certain and the ties, and each kept row is noted where it goes: behind the
// certain ones before it and as many of the ties before it as are kept.  The
// sequence's tags, weights and tables move in the same pass, all of the slots at
// hand read before any is written, and nothing is written behind them.  Latency
// bounds it: three sequences of up to 16,384 rows take 15 us (one CTA each, 16 slots
// a thread: 28, four slots at a time: 37), one of 293 rows 9.
//
// Move: a CTA takes one KV head of a layer's keys or values of a sequence, chunk
// by chunk of kept rows in order: a chunk's rows come from behind the chunk before
// it, so a barrier between a chunk's loads and its stores is all that moving rows
// within a sequence's own pages takes.  Rows that go to another sequence's pages
// are divided among several CTAs.  Memory bounds it: each kept row is read and
// written once, with the next chunk's loads in flight while one is stored (403 MB of
// the 12B shape's rows read and written in 119 us, 6.8 TB/s).  In place there are no
// more CTAs than planes and heads, and each one's chunks in turn bound it until those
// fill the SMs: 4,096 of 8,192 rows of the 12B shape take 243 us for 1 or 4 layers and
// 567 for 40 (bytes 10, 40 and 396), to another sequence 32, 65 and 423.
#include <algorithm>

#include "tcgen05.cuh"

namespace kvg {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kItems = 4;        // slots of a thread at once
constexpr int kMaxCluster = 8;
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 4;  // 16-byte pieces of a thread in a chunk

// Orders like the weights (-0 as 0, NaN below everything).
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0;
    const uint32_t b = w == 0.f ? 0u : __float_as_uint(w);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
    __shared__ int hist[2][256];     // of a digit, this CTA's rows
    __shared__ int all_hist[256];    // the cluster's
    __shared__ int found[2];         // digit, rows that have larger ones
    __shared__ int counts[kItems][32];  // rows of a warp: kept for certain, ties << 16
    __shared__ int2 totals[2];       // the CTA's
    const int n_cta = (int)cluster_size(), rank = (int)cluster_rank();
    const EvictSeq q = p.seq[blockIdx.x / n_cta];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, P = p.page_size;
    if (tid < 256) hist[0][tid] = 0;
    let_next_start();  // (all CTAs run by then, and what waits takes no room that they need)
    after_previous();
    const int32_t *table = p.page_table + (int64_t)q.src * p.max_pages, *fill = p.page_fill + (int64_t)q.src * p.max_pages;
    const float *w_src = p.weights + (int64_t)q.src * p.max_slots;
    const int32_t *pos_src = p.positions + (int64_t)q.src * p.max_slots;
    float *w_dst = p.weights + (int64_t)q.dst * p.max_slots;
    int32_t *pos_dst = p.positions + (int64_t)q.dst * p.max_slots;
    int32_t *to = p.to + q.page0;
    if (p.n_pids && rank == 0)  // the sequence's new pages came with the launch
        for (int i = tid; i < q.n_pages; i += kSelectThreads) to[i] = p.pids[q.page0 - p.pid0 + i];

    // The cluster has `span` slots at once, a CTA adjacent ones; a thread's items are
    // the slots first + i * kSelectThreads + tid.
    const int items = min(kItems, (q.n_slots + n_cta * kSelectThreads - 1) / (n_cta * kSelectThreads));
    const int span = max(1, n_cta * items * kSelectThreads);
    float w[kItems];
    int pos[kItems], from[kItems];
    uint32_t valid = 0;
    auto load = [&](int base) {
        valid = 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int s = base + (rank * items + i) * kSelectThreads + tid;
            w[i] = 0.f;
            if (i >= items || s >= q.n_slots) continue;
            const int pg = p.by_page.div(s), r = s - pg * P, pid = table[pg];
            w[i] = w_src[s];
            pos[i] = pos_src[s];
            from[i] = pid * (p.n_kv_heads * P) + r;
            if (!q.gaps || r < fill[pg]) {
                valid |= 1u << i;
                if (pid < 0 || pid >= p.pool_pages) {
                    record_error(p.status, KVG_ERR_DEVICE_CHECK, 30);
                    from[i] = -1;
                }
            }
        }
    };
    auto middle = [&](int base, int i) {  // may be chosen by weight
        const int s = base + (rank * items + i) * kSelectThreads + tid;
        return s >= q.lo && s < q.hi && !q.all;
    };
    load(0);
    const bool at_once = q.n_slots <= span;  // loaded once for all

    // ---- the weight that decides: of the rows in slots [lo, hi) those whose key's
    // digits so far (mask) are above `prefix` are kept, and `ties` of the equal ones
    uint32_t prefix = 0xffffffffu, mask = 0xffffffffu;
    int ties = 0;
    if (q.middle > 0) {
        prefix = mask = 0;
        ties = q.middle;
        __syncthreads();
        for (int shift = 24, buf = 0; shift >= 0; shift -= 8, buf ^= 1) {
            for (int base = 0; base < q.n_slots; base += span) {
                if (!at_once) load(base);
#pragma unroll
                for (int i = 0; i < kItems; ++i) {
                    const uint32_t key = weight_key(w[i]);
                    if ((valid >> i & 1) && middle(base, i) && (key & mask) == prefix)
                        atomicAdd(&hist[buf][key >> shift & 255], 1);
                }
            }
            cluster_sync();
            if (tid < 256) {
                int n = 0;
                for (int c = 0; c < n_cta; ++c) n += load_of_cta(&hist[buf][tid], c);
                all_hist[tid] = n;
                hist[buf ^ 1][tid] = 0;  // (read by all before the barrier)
            }
            __syncthreads();
            if (warp == 0) {  // a lane has eight digits, the last lane the largest
                int n[8], sum = 0;
#pragma unroll
                for (int i = 7; i >= 0; --i) sum += n[i] = all_hist[lane * 8 + i];
                int above = sum;  // of this lane and the ones after it
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int x = __shfl_down_sync(0xffffffffu, above, d);
                    if (lane + d < 32) above += x;
                }
                above -= sum;
                if (above < ties && ties <= above + sum) {
#pragma unroll
                    for (int i = 7; i >= 0; --i) {
                        if (above < ties && ties <= above + n[i]) {
                            found[0] = lane * 8 + i;
                            found[1] = above;
                        }
                        above += n[i];
                    }
                }
            }
            __syncthreads();
            const int digit = found[0];
            ties -= found[1];
            prefix |= (uint32_t)digit << shift;
            mask |= 255u << shift;
            if (all_hist[digit] == ties) break;  // all of them
        }
    }

    // ---- in slot order: what is kept, and where it goes
    int sure0 = 0, tie0 = 0;  // of the slots before: kept for certain, ties
    for (int base = 0, buf = 0; base < q.n_slots; base += span, buf ^= 1) {
        if (!at_once) load(base);
        uint32_t sure[kItems], tie[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const bool mid = middle(base, i), is = valid >> i & 1;
            const uint32_t key = weight_key(w[i]) & mask;
            sure[i] = __ballot_sync(0xffffffffu, is && (!mid || key > prefix));
            tie[i] = __ballot_sync(0xffffffffu, is && mid && key == prefix);
            if (lane == 0) counts[i][warp] = __popc(sure[i]) | __popc(tie[i]) << 16;
        }
        __syncthreads();
        int before[kItems], sum = 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int x = counts[i][lane];
            before[i] = sum + __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
            sum += __reduce_add_sync(0xffffffffu, x);
        }
        if (tid == 0) totals[buf] = make_int2(sum & 0xffff, sum >> 16);
        cluster_sync();  // (and every slot at hand has been read)
        int sure_all = sure0, tie_all = tie0;
        for (int c = 0; c < n_cta; ++c) {
            if (c == rank) sure0 = sure_all, tie0 = tie_all;
            sure_all += load_of_cta(&totals[buf].x, c);
            tie_all += load_of_cta(&totals[buf].y, c);
        }
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const uint32_t below = (1u << lane) - 1;
            const int ties_before = tie0 + (before[i] >> 16) + __popc(tie[i] & below);
            const int j = sure0 + (before[i] & 0xffff) + __popc(sure[i] & below) + min(ties, ties_before);
            const bool keep = (sure[i] >> lane & 1) || ((tie[i] >> lane & 1) && ties_before < ties);
            if (!keep || j >= q.kept) continue;
            p.from[q.list + j] = from[i];
            pos_dst[j] = pos[i];
            w_dst[j] = w[i];
        }
        sure0 = sure_all;
        tie0 = tie_all;
    }
    cluster_sync();  // nothing reads this CTA's memory, the tables, or what is cleared next
    const int at = rank * kSelectThreads + tid, step = n_cta * kSelectThreads;
    for (int s = q.kept + at; s < q.old_slots; s += step) {
        pos_dst[s] = -1;
        w_dst[s] = 0.f;
    }
    int32_t *table_dst = p.page_table + (int64_t)q.dst * p.max_pages, *fill_dst = p.page_fill + (int64_t)q.dst * p.max_pages;
    if (rank == 0)  // (the CTA that wrote the new pages' ids)
        for (int j = tid; j < max(q.n_pages, q.old_pages); j += kSelectThreads) {
            table_dst[j] = j < q.n_pages ? to[j] : -1;
            fill_dst[j] = j < q.n_pages ? min(P, q.kept - j * P) : 0;
        }
}

// SHIFT: log2 of a row's bytes.
template <int SHIFT>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictParams p) {
    constexpr int U = kMoveUnroll, ROWS = kMoveThreads * U * 16 >> SHIFT;  // of a chunk
    const EvictSeq q = p.seq[blockIdx.y];
    const int part = blockIdx.z;
    if (q.in_place && part > 0) return;
    const int parts = q.in_place ? 1 : gridDim.z, n = q.kept - q.start, P = p.page_size;
    // (whole chunks of rows to a part)
    const int chunks = (n + ROWS - 1) / ROWS;
    const int begin = q.start + (int)((int64_t)chunks * part / parts) * ROWS;
    const int end = min(q.kept, q.start + (int)((int64_t)chunks * (part + 1) / parts) * ROWS);
    if (begin >= end) return;
    const int plane = blockIdx.x / p.n_kv_heads, head = blockIdx.x - plane * p.n_kv_heads;
    uint8_t *const rows = p.pool + ((((int64_t)plane * p.pool_pages * p.n_kv_heads + head) * P) << SHIFT);
    after_previous();
    const int32_t *from = p.from + q.list, *to = p.to + q.page0;
    uint4 x[U], y[U];
    int32_t tx[U], ty[U];  // where they go; -1: nowhere
    auto load = [&](int j0, uint4 (&v)[U], int32_t (&t)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (u * kMoveThreads + threadIdx.x) * 16, j = j0 + (at >> SHIFT);
            t[u] = -1;
            if (j < end) {
                const int pg = p.by_page.div(j), f = from[j];
                t[u] = to[pg] * (p.n_kv_heads * P) + j - pg * P;
                if (t[u] == f || f < 0)  // stays
                    t[u] = -1;
                else
                    v[u] = *reinterpret_cast<const uint4 *>(rows + ((int64_t)f << SHIFT) + (at & ((1 << SHIFT) - 1)));
            }
        }
    };
    auto store = [&](const uint4 (&v)[U], const int32_t (&t)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t[u] >= 0)
                *reinterpret_cast<uint4 *>(rows + ((int64_t)t[u] << SHIFT) +
                                           (((u * kMoveThreads + threadIdx.x) * 16) & ((1 << SHIFT) - 1))) = v[u];
    };
    load(begin, x, tx);
    for (int j = begin; j < end; j += 2 * ROWS) {
        load(j + ROWS, y, ty);
        if (q.in_place) __syncthreads();
        store(x, tx);
        load(j + 2 * ROWS, x, tx);
        if (q.in_place) __syncthreads();
        store(y, ty);
    }
}

}  // namespace

cudaError_t launch_evict(const EvictParams &p, int64_t most_slots, int64_t most_rows, int n_sm, cudaStream_t s) {
    // a slot to each thread, up to a cluster's CTAs
    int cluster = 1;
    while (cluster < kMaxCluster && (int64_t)cluster * kSelectThreads < most_slots) cluster *= 2;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(p.n_seq * cluster);
    cfg.blockDim = dim3(kSelectThreads);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, evict_select_kernel, p);
    count_launches(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess || most_rows <= 0) return e;
    // parts of a plane's rows: some four waves of CTAs, a chunk or more to each
    const int64_t units = (int64_t)p.n_planes * p.n_kv_heads * p.n_seq;
    const int64_t chunks = (most_rows * p.row_bytes + kMoveThreads * kMoveUnroll * 16 - 1) / (kMoveThreads * kMoveUnroll * 16);
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({chunks, 32 * (int64_t)n_sm / units, 65535}));
    const dim3 grid((unsigned)(p.n_planes * p.n_kv_heads), p.n_seq, (unsigned)parts);
    switch (p.row_bytes) {
        case 64: return launch_after(evict_move_kernel<6>, grid, kMoveThreads, 0, s, p);
        case 128: return launch_after(evict_move_kernel<7>, grid, kMoveThreads, 0, s, p);
        case 256: return launch_after(evict_move_kernel<8>, grid, kMoveThreads, 0, s, p);
        case 512: return launch_after(evict_move_kernel<9>, grid, kMoveThreads, 0, s, p);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
