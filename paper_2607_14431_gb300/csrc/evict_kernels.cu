// evict_kernels.cu — a sequence thinned to a number of its rows: the first few,
// the last ones, and of those in between the ones of most weight (a restored
// context, Sec. 4.4, that has to take less room).
//
// Of n rows with weights w the kept ones are i < first, i >= n - last, and the m
// heaviest others, m = rows - first - last; of equal weights the earlier.  They
// keep their order, so the j-th kept row moves from slot s_j >= j to slot j.
//
// Selection: a CTA per sequence.  The m-th largest weight is found digit by digit
// (8 bits of a key that orders like the weights), each digit a histogram of the
// rows that agree so far; then one pass in slot order ranks ties and kept rows by
// ballots and writes where each row comes from.  The sequence's tags, weights and
// tables move in the same pass: a chunk of slots is read before it is written,
// and no later chunk is written to.
//
// Move: a CTA takes one KV head of a layer's keys or values of a sequence, chunk
// by chunk of kept rows in order: a chunk's rows come from behind the chunk before
// it, so a barrier between a chunk's loads and its stores is all that moving rows
// within a sequence's own pages takes.  Rows that go to another sequence's pages
// are divided among several CTAs.  Memory bounds it: each kept row is read and
// written once, with the next chunk's loads in flight while one is stored.
#include <algorithm>

#include "common.cuh"

namespace kvg {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 4;  // 16-byte pieces of a thread in a chunk

// Orders like the weights (-0 as 0, NaN below everything).
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0;
    const uint32_t b = w == 0.f ? 0u : __float_as_uint(w);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
    __shared__ int hist[256];
    __shared__ int counts[2][2][32];  // of a chunk: ties, kept rows of each warp
    __shared__ int found[2];          // digit, rows that have larger ones
    const EvictSeq q = p.seq[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, P = p.page_size;
    after_previous();
    const int32_t *table = p.page_table + (int64_t)q.src * p.max_pages, *fill = p.page_fill + (int64_t)q.src * p.max_pages;
    const float *w_src = p.weights + (int64_t)q.src * p.max_slots;
    const int32_t *pos_src = p.positions + (int64_t)q.src * p.max_slots;
    float *w_dst = p.weights + (int64_t)q.dst * p.max_slots;
    int32_t *pos_dst = p.positions + (int64_t)q.dst * p.max_slots;
    int32_t *to = p.to + q.page0;
    if (p.n_pids)  // the sequence's new pages came with the launch
        for (int i = tid; i < q.n_pages; i += kSelectThreads) to[i] = p.pids[q.page0 - p.pid0 + i];
    auto valid = [&](int s) {
        if (!q.gaps) return true;
        const int pg = p.by_page.div(s);
        return s - pg * P < fill[pg];
    };

    // ---- the weight that decides: of the rows in slots [lo, hi) those whose key's
    // digits so far (mask) are above `prefix` are kept, and `ties` of the equal ones
    uint32_t prefix = 0xffffffffu, mask = 0xffffffffu;
    int ties = 0;
    if (q.middle > 0) {
        prefix = mask = 0;
        ties = q.middle;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int s = q.lo + tid; s < q.hi; s += kSelectThreads) {
                const uint32_t key = weight_key(w_src[s]);
                if ((key & mask) == prefix && valid(s)) atomicAdd(&hist[key >> shift & 255], 1);
            }
            __syncthreads();
            if (warp == 0) {  // a lane has eight digits, the last lane the largest
                int n[8], sum = 0;
#pragma unroll
                for (int i = 7; i >= 0; --i) sum += n[i] = hist[lane * 8 + i];
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
            if (hist[digit] == ties) break;  // all of them
            __syncthreads();
        }
    }

    // ---- chunk by chunk: what is kept, and where it goes
    int tie0 = 0, kept0 = 0, buf = 0;  // of the chunks before
    struct Slot {
        float w;
        int pos, from;
        bool valid;
    };
    auto load = [&](int s) {
        Slot x{0.f, 0, 0, false};
        if (s < q.n_slots) {
            const int pg = p.by_page.div(s), r = s - pg * P;
            x.valid = !q.gaps || r < fill[pg];
            x.w = w_src[s];
            x.pos = pos_src[s];
            const int pid = table[pg];
            x.from = pid * (p.n_kv_heads * P) + r;
            if (x.valid && (pid < 0 || pid >= p.pool_pages)) {
                record_error(p.status, KVG_ERR_DEVICE_CHECK, 30);
                x.from = -1;
            }
        }
        return x;
    };
    auto before = [&](const int *n, int &total) {  // of the warps before; all warps'
        int x = n[lane];
        total = __reduce_add_sync(0xffffffffu, x);
        return __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
    };
    Slot next = load(tid);
    for (int base = 0; base < q.n_slots; base += kSelectThreads, buf ^= 1) {
        const Slot x = next;
        next = load(base + kSelectThreads + tid);  // (slots that nothing is moved to before they are read)
        const int s = base + tid;
        const bool mid = s >= q.lo && s < q.hi && !q.all;
        const uint32_t key = weight_key(x.w) & mask;
        const bool tie = x.valid && mid && key == prefix;
        const uint32_t tied = __ballot_sync(0xffffffffu, tie);
        if (lane == 0) counts[buf][0][warp] = __popc(tied);
        __syncthreads();
        int n_tied, n_kept;
        const int rank = tie0 + before(counts[buf][0], n_tied) + __popc(tied & ((1u << lane) - 1));
        const bool keep = x.valid && (!mid || key > prefix || (tie && rank < ties));
        const uint32_t kept = __ballot_sync(0xffffffffu, keep);
        if (lane == 0) counts[buf][1][warp] = __popc(kept);
        __syncthreads();  // (and the chunk has been read)
        const int j = kept0 + before(counts[buf][1], n_kept) + __popc(kept & ((1u << lane) - 1));
        if (keep && j < q.kept) {
            p.from[q.list + j] = x.from;
            pos_dst[j] = x.pos;
            w_dst[j] = x.w;
        }
        tie0 += n_tied;
        kept0 += n_kept;
    }
    __syncthreads();  // the tables have been read
    for (int s = q.kept + tid; s < q.old_slots; s += kSelectThreads) {
        pos_dst[s] = -1;
        w_dst[s] = 0.f;
    }
    int32_t *table_dst = p.page_table + (int64_t)q.dst * p.max_pages, *fill_dst = p.page_fill + (int64_t)q.dst * p.max_pages;
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

cudaError_t launch_evict(const EvictParams &p, int64_t most_rows, bool move, int n_sm, cudaStream_t s) {
    cudaError_t e = launch_after(evict_select_kernel, p.n_seq, kSelectThreads, 0, s, p);
    if (e != cudaSuccess || !move) return e;
    const int shift = p.row_bytes == 64 ? 6 : p.row_bytes == 128 ? 7 : p.row_bytes == 256 ? 8 : 9;
    // parts of a plane's rows: some four waves of CTAs, a chunk or more to each
    const int64_t units = (int64_t)p.n_planes * p.n_kv_heads * p.n_seq;
    const int64_t chunks = (most_rows * p.row_bytes + kMoveThreads * kMoveUnroll * 16 - 1) / (kMoveThreads * kMoveUnroll * 16);
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({chunks, 32 * (int64_t)n_sm / units, 65535}));
    const dim3 grid((unsigned)(p.n_planes * p.n_kv_heads), p.n_seq, (unsigned)parts);
    switch (shift) {
        case 6: return launch_after(evict_move_kernel<6>, grid, kMoveThreads, 0, s, p);
        case 7: return launch_after(evict_move_kernel<7>, grid, kMoveThreads, 0, s, p);
        case 8: return launch_after(evict_move_kernel<8>, grid, kMoveThreads, 0, s, p);
        default: return launch_after(evict_move_kernel<9>, grid, kMoveThreads, 0, s, p);
    }
}

}  // namespace kvg
