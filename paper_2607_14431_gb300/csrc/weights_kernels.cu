// weights_kernels.cu — what weight each cached row received from the query rows
// that attended to it (the measure by which kvg_cache_evict thins a restored
// context, Sec. 4.4):
//   weight[j] = sum over layers, query heads and rows i of 2^(s_ij - m_i) / l_i,
// s_ij the scores scaled by log2(e), m_i a row's maximum, l_i its sum of 2^(s_ij -
// m_i), all in fp32 (the attention's own sums add 16-bit weights).
//
// A decode step's scores are 2 G / D of its keys' and values' bytes: the decode
// kernel stores them on its way, the combine leaves (m, 1 / l) of each head, and
// one more pass over the scores adds up a slot's weights, in a fixed order, so
// keys are read once and results are bitwise reproducible.
#include <algorithm>

#include "decode.cuh"

namespace kvg {

namespace {

template <int D, int COLS>
__global__ void __launch_bounds__(kCombineMaxThreads)
    combine_scores_kernel(const DecodeParams p, const __grid_constant__ ScoreParams sp) {
    constexpr int PARTS = D / COLS;
    const int h = blockIdx.x / PARTS, col0 = blockIdx.x % PARTS * COLS, b = blockIdx.y, lr = blockIdx.z;
    const Merged m = merge_partials<D, COLS, true>(p, h, col0, b, lr, sp.part_lx);
    if (threadIdx.x == 0 && col0 == 0) sp.ml[((int64_t)lr * p.B + b) * p.n_q_heads + h] = make_float2(m.M, __fdiv_rn(1.f, m.LX));
    write_output<COLS>(p, m, h, col0, b, lr, D);
}

// A block: kSlots slots of a batch row, kLines threads for each that share its
// layers and heads.
constexpr int kSlots = 64, kLines = 4;
__global__ void __launch_bounds__(kSlots * kLines) accumulate_kernel(const __grid_constant__ AccumulateParams p) {
    __shared__ float part[kLines][kSlots];
    const int b = blockIdx.y, x = threadIdx.x % kSlots, line = threadIdx.x / kSlots, n = p.n[b];
    const int slot = blockIdx.x * kSlots + x;
    if (blockIdx.x * kSlots >= n) return;
    after_previous();
    bool valid = slot < n;
    if (valid) {
        const int pg = p.by_page.div(slot);
        valid = slot - pg * p.page_size < p.page_fill[(int64_t)p.seq[b] * p.max_pages + pg];
    }
    float sum = 0.f;
    auto add = [&](int lr0, int lr1, int first) {
        if (!valid || slot < first) return;
        const int r1 = lr1 * p.n_q_heads;
        const float *s = p.scores + p.at[b] + slot;
#pragma unroll 8
        for (int r = lr0 * p.n_q_heads + line; r < r1; r += kLines) {
            const int lr = r / p.n_q_heads;
            const float2 ml = p.ml[((int64_t)lr * p.B + b) * p.n_q_heads + r - lr * p.n_q_heads];
            sum = __fmaf_rn(exp2f(s[(int64_t)r * n] - ml.x), ml.y, sum);
        }
    };
    add(0, p.layer1, p.first[0][b]);
    add(p.layer1, p.n_layers_run, p.first[1][b]);
    part[line][x] = sum;
    __syncthreads();
    if (line > 0 || slot >= n) return;
#pragma unroll
    for (int i = 1; i < kLines; ++i) sum += part[i][x];
    float *w = p.weights + (int64_t)p.seq[b] * p.max_slots + slot;
    *w = p.decay == 0.f ? sum : __fmaf_rn(p.decay, *w, sum);
}

}  // namespace

int decode_scores_max_warps(int head_dim, int group, bool fp8, int page_size, int n_sm) {
    const int tok = decode_tile_tokens(head_dim, fp8, page_size);
#define KVG_CASE(DD, GG, FF, TT)                                        \
    if (head_dim == DD && group == GG && fp8 == FF && tok == TT)        \
        return DecodeLaunch<DD, GG, FF, TT, true>::max_blocks_per_sm() * n_sm;
    KVG_DECODE_CASES(KVG_CASE)
#undef KVG_CASE
    return 0;
}

cudaError_t launch_decode_scores(int head_dim, int group, bool fp8, const DecodeParams &p, const ScoreParams &sp,
                                 const CUtensorMap &pool_map, int n_sm, cudaStream_t s) {
    const int tok = decode_tile_tokens(head_dim, fp8, p.page_size);
    cudaError_t e = cudaErrorInvalidValue;
#define KVG_CASE(DD, GG, FF, TT)                                        \
    if (head_dim == DD && group == GG && fp8 == FF && tok == TT)        \
        e = DecodeLaunch<DD, GG, FF, TT, true>::run(p, pool_map, sp, s);
    KVG_DECODE_CASES(KVG_CASE)
#undef KVG_CASE
    if (e != cudaSuccess) return e;
    const int cols = (int64_t)p.n_q_heads * p.B * p.n_layers_run <= n_sm ? 64 : head_dim;
    const dim3 grid(p.n_q_heads * (head_dim / cols), p.B, p.n_layers_run);
    const int n = combine_threads(cols, p);
    switch (head_dim * 1000 + cols) {
        case 64064: return launch_after(combine_scores_kernel<64, 64>, grid, n, 0, s, p, sp);
        case 128064: return launch_after(combine_scores_kernel<128, 64>, grid, n, 0, s, p, sp);
        case 128128: return launch_after(combine_scores_kernel<128, 128>, grid, n, 0, s, p, sp);
        case 256064: return launch_after(combine_scores_kernel<256, 64>, grid, n, 0, s, p, sp);
        case 256256: return launch_after(combine_scores_kernel<256, 256>, grid, n, 0, s, p, sp);
    }
    return cudaErrorInvalidValue;
}

cudaError_t launch_accumulate(const AccumulateParams &p, cudaStream_t s) {
    int most = 0;
    for (int b = 0; b < p.B; ++b) most = std::max(most, p.n[b]);
    if (most == 0) return cudaSuccess;
    return launch_after(accumulate_kernel, dim3((most + kSlots - 1) / kSlots, p.B), kSlots * kLines, 0, s, p);
}

}  // namespace kvg
