// prompt_kernels.cu — launches of the prompt kernel, and the join of rows whose
// keys were split.
#include "prompt.cuh"

namespace kvg {

namespace {

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
    if (p.row_lse && lane == 0) {
        float top = -INFINITY, sum = 0.f;
        for (int i = 0; i < p.splits[it.b]; ++i) top = fmaxf(top, p.part_lse[part_slot(p, it, i, row)]);
        for (int i = 0; i < p.splits[it.b]; ++i) sum += exp2f(p.part_lse[part_slot(p, it, i, row)] - top);
        p.row_lse[lse_row(p, it, row)] = top + log2f(sum);
    }
    const float inv = __fdiv_rn(p.vscale, L);
    uint32_t *out = reinterpret_cast<uint32_t *>(p.out + q_row(p, it, row) * D + lane * N);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) out[e] = pack_out(o[2 * e] * inv, o[2 * e + 1] * inv);
}

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
