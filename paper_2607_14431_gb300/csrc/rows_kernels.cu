// rows_kernels.cu — the decode kernel for a few query rows of a sequence at a time
// (cross attention of a decoder's candidates to an encoder's states): the heads of
// its eight-column products are those of as many rows as fit, so that keys and
// values are read once for all of them, at a decode's rate.
#include <algorithm>

#include "decode.cuh"

namespace kvg {

namespace {

template <int D, int COLS>
__global__ void __launch_bounds__(kCombineMaxThreads)
    combine_rows_kernel(const __grid_constant__ DecodeParams p, const __grid_constant__ RowParams rows) {
    constexpr int PARTS = D / COLS;
    const int h = blockIdx.x / PARTS, col0 = blockIdx.x % PARTS * COLS, b = blockIdx.y, lr = blockIdx.z;
    const int g = h / kRowHeads, j = h % kRowHeads, gs = rows.log2_group;
    if (j >= rows.heads[b]) return;
    const int64_t row = p.qlayers[lr] * rows.q_rows + rows.row0[b] + (j >> gs);
    write_output<COLS>(p, merge_partials<D, COLS>(p, h, col0, b, lr),
                       row * rows.n_q_heads + (g << gs) + (j & ((1 << gs) - 1)), col0, D);
}

}  // namespace

#define KVG_ROWS_CASES(X)                                                                                       \
    X(64, false, 64) X(64, false, 16) X(128, false, 64) X(128, false, 16) X(256, false, 16) X(128, true, 32)   \
    X(128, true, 16) X(256, true, 16)

int decode_rows_max_warps(int head_dim, bool fp8, int page_size, int n_sm) {
    const int tok = decode_tile_tokens(head_dim, fp8, page_size);
#define KVG_CASE(DD, FF, TT)                              \
    if (head_dim == DD && fp8 == FF && tok == TT)         \
        return DecodeLaunch<DD, kRowHeads, FF, TT, RowParams>::max_blocks_per_sm() * n_sm;
    KVG_ROWS_CASES(KVG_CASE)
#undef KVG_CASE
    return 0;
}

cudaError_t launch_decode_rows(int head_dim, bool fp8, const DecodeParams &p, const RowParams &rows,
                               const CUtensorMap &pool_map, int n_sm, cudaStream_t s) {
    const int tok = decode_tile_tokens(head_dim, fp8, p.page_size);
    cudaError_t e = cudaErrorInvalidValue;
#define KVG_CASE(DD, FF, TT)                              \
    if (head_dim == DD && fp8 == FF && tok == TT)         \
        e = DecodeLaunch<DD, kRowHeads, FF, TT, RowParams>::run(p, pool_map, rows, s);
    KVG_ROWS_CASES(KVG_CASE)
#undef KVG_CASE
    if (e != cudaSuccess) return e;
    const int cols = (int64_t)p.n_q_heads * p.B * p.n_layers_run <= n_sm ? 64 : head_dim;
    const dim3 grid(p.n_q_heads * (head_dim / cols), p.B, p.n_layers_run);
    const int n = combine_threads(cols, p);
    switch (head_dim * 1000 + cols) {
        case 64064: return launch_after(combine_rows_kernel<64, 64>, grid, n, 0, s, p, rows);
        case 128064: return launch_after(combine_rows_kernel<128, 64>, grid, n, 0, s, p, rows);
        case 128128: return launch_after(combine_rows_kernel<128, 128>, grid, n, 0, s, p, rows);
        case 256064: return launch_after(combine_rows_kernel<256, 64>, grid, n, 0, s, p, rows);
        case 256256: return launch_after(combine_rows_kernel<256, 256>, grid, n, 0, s, p, rows);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
