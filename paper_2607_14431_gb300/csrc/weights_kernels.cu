// weights_kernels.cu — what weight each cached row received from the query rows
// that attended to it (the measure by which kvg_cache_evict thins a restored
// context, Sec. 4.4):
//   weight[j] = sum over layers, query heads and rows i of 2^(s_ij - m_i) / l_i,
// s_ij the scores scaled by log2(e), m_i a row's maximum, l_i its sum of 2^(s_ij -
// m_i), all in fp32 (the attention's own sums add 16-bit weights).
//
// A decode step's scores are G / D of its keys' and values' bytes (fp8: 2 G / D), to
// be written and read once: the decode kernel stores them on its way.  Behind it one
// launch merges its partial results into outputs (the blocks of the combine) and adds
// up a slot's weights over layers and heads, in a fixed order, so that keys are read
// once and results are bitwise reproducible.  A block of the latter has up to 128 slots
// of a batch row and finds (m, l) of all its heads itself, a few partials each: as a
// launch of its own behind the combine, which had merged them, one token on 2,111 rows
// of the 31B shape took 13.9 us.
#include <algorithm>

#include "decode.cuh"
#include "tcgen05.cuh"

namespace kvg {

namespace {

constexpr int kHeads = 512;  // layers x query heads whose (m, 1 / l) are kept at once

// Slots of a block with that many threads: two to a thread; the threads of one
// slot share its heads.
__host__ __device__ constexpr int block_slots(int threads) { return 2 * (threads < 64 ? threads : 64); }

__device__ __forceinline__ void accumulate(const DecodeParams &p, const AccumulateParams &a, int block, int b) {
    __shared__ float2 ml[kHeads];
    __shared__ UnitPartials units[kHeads];
    __shared__ float part[2][kCombineMaxThreads];
    const int slots = block_slots(blockDim.x), half = slots / 2, lines = blockDim.x / half;
    const int x = threadIdx.x % half, line = threadIdx.x / half, n = a.scores.n[b], slot = block * slots + x;
    if (block * slots >= n) return;
    const int G = p.n_q_heads / p.n_kv_heads, heads = p.n_layers_run * p.n_q_heads;
    after_previous();
    bool valid[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int s = slot + k * half;
        valid[k] = s < n;
        if (valid[k]) {
            const int pg = a.by_page.div(s);
            valid[k] = s - pg * p.page_size < p.page_fill[(int64_t)p.seq[b] * p.max_pages + pg];
        }
    }
    const int from[2] = {a.first[0][b], a.first[1][b]};  // of the layers' groups
    constexpr int U = 8;  // a slot's scores in flight.  (Where their use was behind a branch, the loads were too:
                          // 10,000 cycles for 16 heads.  So what lies outside is read again, and left out.)
    const float *const at[2] = {a.scores.scores + a.scores.at[b] + min(slot, n - 1),
                                a.scores.scores + a.scores.at[b] + min(slot + half, n - 1)};
    float sum[2] = {};
    for (int r0 = 0; r0 < heads; r0 += kHeads) {
        const int end = min(heads - r0, kHeads);
        float ahead[2][U];
        auto fetch = [&](int r) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = (int64_t)(r0 + min(r + u * lines, end - 1)) * n;
                ahead[0][u] = at[0][i];
                ahead[1][u] = at[1][i];
            }
        };
        fetch(line);
        // where a KV head's partials are: a thread each (64-bit divisions); kHeads is a multiple of G
        for (int u = threadIdx.x; u < end / G; u += blockDim.x) {
            const int lr = (r0 / G + u) / p.n_kv_heads;
            units[u] = unit_partials(p, r0 / G + u - lr * p.n_kv_heads, b, lr);
        }
        __syncthreads();
        // (m, 1 / l) of a head: four threads, eight partials of each in flight
        const int lane = threadIdx.x % 4;
        for (int i0 = threadIdx.x / 4; i0 - (int)threadIdx.x / 4 < end; i0 += blockDim.x / 4) {  // (whole warps)
            const int r = min(i0, end - 1);
            const UnitPartials of = units[r / G];
            const int64_t from0 = of.slot * G + r % G;
            float M = -INFINITY, L = 0.f;
            auto join = [&](float m, float l) {
                const float top = fmaxf(M, m), base = top == -INFINITY ? 0.f : top;
                L = __fmaf_rn(L, exp2_approx(M - base), l * exp2_approx(m - base));
                M = top;
            };
            for (int i = lane; i < of.n; i += 32) {
                float2 x[8];
                float l[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int64_t k = from0 + (int64_t)min(i + 4 * u, of.n - 1) * G;
                    x[u] = p.part_ml[k];
                    l[u] = a.scores.part_lx[k];
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const bool in = i + 4 * u < of.n;
                    join(in ? x[u].x : -INFINITY, in ? l[u] : 0.f);
                }
            }
#pragma unroll
            for (int d = 2; d; d >>= 1) {
                const float m = __shfl_xor_sync(0xffffffffu, M, d), l = __shfl_xor_sync(0xffffffffu, L, d);
                join(m, l);
            }
            if (lane == 0 && i0 < end) ml[r] = make_float2(M == -INFINITY ? 0.f : M, __fdiv_rn(1.f, L));
        }
        __syncthreads();
        const int border = p.layer1 * p.n_q_heads - r0;  // heads of the other group from here on
        for (int r = line; r < end; r += U * lines) {
            float x[2][U];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int u = 0; u < U; ++u) x[k][u] = ahead[k][u];
            fetch(r + U * lines);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int head = r + u * lines, first = head < border ? from[0] : from[1];
                const float2 of = ml[min(head, end - 1)];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float w = exp2_approx(x[k][u] - of.x) * of.y;
                    sum[k] += head < end && slot + k * half >= first ? w : 0.f;
                }
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (!valid[k]) sum[k] = 0.f;
    part[0][threadIdx.x] = sum[0];
    part[1][threadIdx.x] = sum[1];
    __syncthreads();
    if (line > 0) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (slot + k * half >= n) return;
        for (int i = 1; i < lines; ++i) sum[k] += part[k][i * half + x];
        float *w = a.weights + (int64_t)p.seq[b] * a.max_slots + slot + k * half;
        *w = a.decay == 0.f ? sum[k] : __fmaf_rn(a.decay, *w, sum[k]);
    }
}

template <int D, int COLS>
__global__ void __launch_bounds__(kCombineMaxThreads)
    combine_weights_kernel(const __grid_constant__ DecodeParams p, const __grid_constant__ AccumulateParams a) {
    constexpr int PARTS = D / COLS;
    const int outputs = p.n_q_heads * PARTS * p.n_layers_run;
    int i = blockIdx.x;
    if (i >= outputs) {
        accumulate(p, a, i - outputs, blockIdx.y);
        return;
    }
    const int lr = i / (p.n_q_heads * PARTS);
    i -= lr * p.n_q_heads * PARTS;
    const int h = i / PARTS, col0 = i % PARTS * COLS, b = blockIdx.y;
    write_output<COLS>(p, merge_partials<D, COLS>(p, h, col0, b, lr), out_head(p, h, b, lr), col0, D);
}

}  // namespace

int decode_scores_max_warps(int head_dim, int group, bool fp8, int page_size, int n_sm) {
    const int tok = decode_tile_tokens(head_dim, fp8, page_size);
#define KVG_CASE(DD, GG, FF, TT)                                        \
    if (head_dim == DD && group == GG && fp8 == FF && tok == TT)        \
        return DecodeLaunch<DD, GG, FF, TT, ScoreParams>::max_blocks_per_sm() * n_sm;
    KVG_DECODE_CASES(KVG_CASE)
#undef KVG_CASE
    return 0;
}

cudaError_t launch_decode_weights(int head_dim, int group, bool fp8, const DecodeParams &p, const AccumulateParams &a,
                                  const CUtensorMap &pool_map, int n_sm, cudaStream_t s) {
    const int tok = decode_tile_tokens(head_dim, fp8, p.page_size);
    cudaError_t e = cudaErrorInvalidValue;
#define KVG_CASE(DD, GG, FF, TT)                                        \
    if (head_dim == DD && group == GG && fp8 == FF && tok == TT)        \
        e = DecodeLaunch<DD, GG, FF, TT, ScoreParams>::run(p, pool_map, a.scores, s);
    KVG_DECODE_CASES(KVG_CASE)
#undef KVG_CASE
    if (e != cudaSuccess) return e;
    // (the combine's blocks are those of launch_combine: outputs are those of the decode alone, bit for bit, where
    // both split the tiles alike, among as many warps and over the same layers and rows; else within the sums' rounding)
    const int cols = (int64_t)p.n_q_heads * p.B * p.n_layers_run <= n_sm ? 64 : head_dim;
    const int n = combine_threads(cols, p), slots = block_slots(n);
    const int64_t outputs = (int64_t)p.n_q_heads * (head_dim / cols) * p.n_layers_run;
    const dim3 grid((unsigned)(outputs + (a.most_slots + slots - 1) / slots), p.B);
    switch (head_dim * 1000 + cols) {
        case 64064: return launch_after(combine_weights_kernel<64, 64>, grid, n, 0, s, p, a);
        case 128064: return launch_after(combine_weights_kernel<128, 64>, grid, n, 0, s, p, a);
        case 128128: return launch_after(combine_weights_kernel<128, 128>, grid, n, 0, s, p, a);
        case 256064: return launch_after(combine_weights_kernel<256, 64>, grid, n, 0, s, p, a);
        case 256256: return launch_after(combine_weights_kernel<256, 256>, grid, n, 0, s, p, a);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
