// attn_kernels.cu — launches of the decode kernel, the merges of its partial
// results, and the tensor maps of a pool.
#include "decode.cuh"

namespace kvg {

namespace {

template <int D, int COLS>
__global__ void __launch_bounds__(kCombineMaxThreads) combine_kernel(const DecodeParams p) {
    constexpr int PARTS = D / COLS;
    const int h = blockIdx.x / PARTS, col0 = blockIdx.x % PARTS * COLS, b = blockIdx.y, lr = blockIdx.z;
    write_output<COLS>(p, merge_partials<D, COLS>(p, h, col0, b, lr), out_head(p, h, b, lr), col0, D);
}

// Merge of a decode whose rows read some of their pages together
// (kvg_decode_attention_shared): the row's partials over the shared pages, then
// its own.  Few of each (an SM has a key range of the shared pages, a short tail
// is a warp or two), so a warp takes a row, a lane D / 32 of its columns, four
// partials in flight: 96 sequences of the 31B shape over 9 ranges 8.3 us, with
// a block per row as above 12.1 us.
constexpr int kCombineRows = 8;  // of a block
template <int D>
__global__ void __launch_bounds__(32 * kCombineRows)
    combine_shared_kernel(const __grid_constant__ DecodeParams p, const __grid_constant__ SharedParts sp) {
    constexpr int N = D / 32, U = 4;
    using Vec = std::conditional_t<N == 2, float2, float4>;
    constexpr int W = sizeof(Vec) / 4;
    const int lane = threadIdx.x & 31, G = p.n_q_heads / p.n_kv_heads;
    const int at = blockIdx.x * kCombineRows + threadIdx.x / 32;
    if (at >= p.n_q_heads * p.B * p.n_layers_run) return;
    const int h = at % p.n_q_heads, b = at / p.n_q_heads % p.B, lr = at / p.n_q_heads / p.B;
    const int g = h / G, hh = h - g * G, grp = lr >= p.layer1;
    // the row's own partials: of the decode's warps wa, wa + 1, ...
    const int32_t *pref = p.rows[grp].pref_tiles;
    const int64_t Tb = pref[b + 1] - pref[b], T = p.group_tiles(grp), WN = p.n_warps[grp];
    const int64_t unit = ((int64_t)lr * p.B + b) * p.n_kv_heads + g;
    int n_own = 0;
    int64_t own = 0;
    if (Tb > 0) {
        const int64_t first = (int64_t)g * Tb +  // of the group's tiles
                              (int64_t)p.n_kv_heads * ((int64_t)(lr - (grp ? p.layer1 : 0)) * pref[p.B] + pref[b]);
        const int64_t wa = warp_of(first, T, WN);
        n_own = (int)(warp_of(first + Tb - 1, T, WN) - wa) + 1;
        own = (unit + wa + (grp ? p.n_warps[0] : 0)) * G + hh;
    }
    const int n_shared = sp.splits[grp][b], n = n_shared + n_own;
    const int64_t part = sp.at[grp][b] + (int64_t)((lr - (grp ? p.layer1 : 0)) * p.n_kv_heads + g) * sp.rows[grp][b] + hh;
    const int64_t part_step = (int64_t)sp.units[grp] * sp.rows[grp][b];
    after_previous();
    let_next_start();  // a few microseconds to its end, and room for the next beside it
    auto ml_at = [&](int i) { return i < n_shared ? sp.part_ml[part + i * part_step] : p.part_ml[own + (int64_t)(i - n_shared) * G]; };
    float M = -INFINITY;
    for (int i = lane; i < n; i += 32) M = fmaxf(M, ml_at(i).x);
#pragma unroll
    for (int x = 16; x; x >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
    float o[N] = {}, L = 0.f;
    for (int i0 = 0; i0 < n; i0 += U) {
        Vec v[U][N / W];
        float2 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u;
            if (i >= n) continue;
            x[u] = ml_at(i);
            const float *src = i < n_shared ? sp.part_o + (part + i * part_step) * D : p.part_o + (own + (int64_t)(i - n_shared) * G) * D;
#pragma unroll
            for (int e = 0; e < N / W; ++e) v[u][e] = reinterpret_cast<const Vec *>(src + lane * N)[e];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u >= n || x[u].y == 0.f) continue;  // (no rows: not even written)
            const float sc = exp2f(x[u].x - M);
            L = __fmaf_rn(x[u].y, sc, L);
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = __fmaf_rn(reinterpret_cast<const float *>(v[u])[e], sc, o[e]);
        }
    }
    uint32_t *out = reinterpret_cast<uint32_t *>(
        p.out + ((int64_t)(p.qlayers[lr] * p.q_row_stride_b + p.b0 + b) * p.n_q_heads + h) * D + lane * N);
#pragma unroll
    for (int e = 0; e < N; e += 2) {  // (a sum that is NaN gives NaN)
        const float y0 = L != 0.f ? __fdiv_rn(o[e], L) * p.vscale : 0.f, y1 = L != 0.f ? __fdiv_rn(o[e + 1], L) * p.vscale : 0.f;
        const __nv_bfloat162 y = __floats2bfloat162_rn(y0, y1);
        out[e / 2] = *reinterpret_cast<const uint32_t *>(&y);
    }
}

// The same merge for a split decode: the unit's partials give (M, L, O) for
// this call's rows, scaled by vscale, and the result is stored as the state
// (o, m, l) of query head h, or merged into the state already there:
// m' = max(m0, M), o' = o0 2^(m0 - m') + O 2^(M - m'), l' likewise (a side
// with l = 0 holds no rows and is left out).
template <int D>
__global__ void __launch_bounds__(kCombineMaxThreads) combine_state_kernel(const DecodeParams p) {
    const int h = blockIdx.x, b = blockIdx.y, lr = blockIdx.z;
    const Merged m = merge_partials<D, D>(p, h, 0, b, lr);
    float L = m.L, M = m.M;
    float O[4] = {__fmul_rn(m.o.x, p.vscale), __fmul_rn(m.o.y, p.vscale), __fmul_rn(m.o.z, p.vscale),
                  __fmul_rn(m.o.w, p.vscale)};
    float *st = p.state + ((int64_t)(p.qlayers[lr] * p.q_row_stride_b + p.b0 + b) * p.n_q_heads + h) * (D + 4);
    const bool mine = threadIdx.x < D / 4;
    if (p.state_merge) {
        const float m0 = st[D], l0 = st[D + 1];
        float4 o0 = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine) o0 = reinterpret_cast<const float4 *>(st)[threadIdx.x];
        __syncthreads();  // every thread has read (m0, l0) before thread 0 rewrites them
        if (l0 > 0.f) {
            const float oo[4] = {o0.x, o0.y, o0.z, o0.w};
            if (L > 0.f) {
                const float mm = fmaxf(m0, M);
                const float a = exp2f(m0 - mm), c = exp2f(M - mm);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e] = __fmaf_rn(oo[e], a, __fmul_rn(O[e], c));
                L = __fmaf_rn(l0, a, __fmul_rn(L, c));
                M = mm;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e] = oo[e];
                L = l0;
                M = m0;
            }
        }
    }
    if (!mine) return;
    if (L == 0.f) {
        O[0] = O[1] = O[2] = O[3] = 0.f;
        M = -INFINITY;
    }
    reinterpret_cast<float4 *>(st)[threadIdx.x] = make_float4(O[0], O[1], O[2], O[3]);
    if (threadIdx.x == 0) reinterpret_cast<float4 *>(st)[D / 4] = make_float4(M, L, 0.f, 0.f);
}

__global__ void state_finish_kernel(const float *state, int64_t n_rows, int D, __nv_bfloat16 *out) {
    after_previous();
    const int64_t n = n_rows * D;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = i / D;
        const int d = (int)(i - r * D);
        const float *st = state + r * (D + 4);
        const float l = st[D + 1];
        out[i] = __float2bfloat16_rn(l > 0.f ? __fdiv_rn(st[d], l) : 0.f);
    }
}

}  // namespace

namespace {
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up once (thread-safe static init).
EncodeTiled tensor_map_encoder() {
    static const EncodeTiled fn = []() -> EncodeTiled {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}
}  // namespace

cudaError_t encode_tensor_map(CUtensorMap *out, int rank, void *base, const cuuint64_t *dims,
                              const cuuint64_t *strides, const cuuint32_t *box) {
    const EncodeTiled encode = tensor_map_encoder();
    if (!encode) return cudaErrorSymbolNotFound;
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, base, dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t make_pool_tensor_map(CUtensorMap *out, void *pool, int head_dim, bool fp8, int box_rows, uint64_t rows) {
    const EncodeTiled encode = tensor_map_encoder();
    if (!encode) return cudaErrorSymbolNotFound;
    if (fp8 && head_dim % 128) {  // no fp8 decode for this head_dim: nothing to map
        memset(out, 0, sizeof *out);
        return cudaSuccess;
    }
    if (box_rows <= 0 || rows == 0 || rows > 0x7fffffffull) return cudaErrorInvalidValue;
    // 128-byte rows per box: 64 bf16 columns, or 128 fp8 columns
    const cuuint64_t dims[2] = {(cuuint64_t)head_dim, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)head_dim * (fp8 ? 1 : 2)};
    const cuuint32_t box[2] = {fp8 ? 128u : 64u, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = encode(out, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, pool,
                              dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t make_query_tensor_map(CUtensorMap *out, const void *q, int head_dim, int n_q_heads, int group, int tokens,
                                  uint64_t rows) {
    const EncodeTiled encode = tensor_map_encoder();
    if (!encode) return cudaErrorSymbolNotFound;
    if (rows == 0 || rows > 0x7fffffffull) return cudaErrorInvalidValue;
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)n_q_heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)n_q_heads * head_dim * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)tokens}, estr[3] = {1, 1, 1};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(q), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

bool decode_supported(int head_dim, int group, bool fp8) {
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return false;
    if (fp8 && head_dim == 64) return false;
    if (group != 1 && group != 2 && group != 4 && group != 8) return false;
    return head_dim * group <= 512;
}

// The usual tile where it reads at most a tenth more rows of a page than
// 16-row tiles do (the two are within 2% of each other on whole tiles, so what
// decides is the rows read in vain), else those.
int decode_tile_tokens(int head_dim, bool fp8, int page_size) {
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
    if (fp8 && head_dim == 64) return 0;
    const int tok = usual_tok(head_dim, fp8);
    const int64_t usual = ((int64_t)page_size + tok - 1) / tok * tok;
    const int64_t small = ((int64_t)page_size + kSmallTok - 1) / kSmallTok * kSmallTok;
    return usual * 10 <= small * 11 ? tok : kSmallTok;
}

int decode_max_warps(int head_dim, int group, bool fp8, int page_size, int n_sm) {
    const int tok = decode_tile_tokens(head_dim, fp8, page_size);
#define KVG_CASE(DD, GG, FF, TT)                                        \
    if (head_dim == DD && group == GG && fp8 == FF && tok == TT)        \
        return DecodeLaunch<DD, GG, FF, TT>::max_blocks_per_sm() * n_sm;
    KVG_DECODE_CASES(KVG_CASE)
#undef KVG_CASE
    return 0;
}

cudaError_t launch_decode(int head_dim, int group, bool fp8, const DecodeParams &p, const CUtensorMap &pool_map,
                          cudaStream_t s) {
    const int tok = decode_tile_tokens(head_dim, fp8, p.page_size);
#define KVG_CASE(DD, GG, FF, TT)                                        \
    if (head_dim == DD && group == GG && fp8 == FF && tok == TT)        \
        return DecodeLaunch<DD, GG, FF, TT>::run(p, pool_map, {}, s);
    KVG_DECODE_CASES(KVG_CASE)
#undef KVG_CASE
    return cudaErrorInvalidValue;
}

// Threads of a combine block over `cols` columns of a head: a group of cols / 4
// lanes per up to four partials of the row with the most of them (the loads
// one thread keeps in flight).
int combine_threads(int cols, const DecodeParams &p) {
    int64_t most = 1;
    for (int g = 0; g < kMaxWindowGroups; ++g) {
        if (p.group_tiles(g) <= 0) continue;
        int64_t tb = 0;
        for (int b = 0; b < p.B; ++b)
            tb = std::max<int64_t>(tb, p.rows[g].pref_tiles[b + 1] - p.rows[g].pref_tiles[b]);
        most = std::max(most, tb * p.n_warps[g] / p.group_tiles(g) + 2);
    }
    const int lanes = cols / 4;
    int threads = std::max(lanes, 32);
    while (threads < kCombineMaxThreads && (int64_t)(threads / lanes) * 4 < most) threads *= 2;
    return threads;
}

cudaError_t launch_combine(int head_dim, const DecodeParams &p, int n_sm, cudaStream_t s) {
    const bool narrow = !p.state && (int64_t)p.n_q_heads * p.B * p.n_layers_run <= n_sm;
    const int cols = narrow ? 64 : head_dim;
    const dim3 grid(p.n_q_heads * (head_dim / cols), p.B, p.n_layers_run);
    const int n = combine_threads(cols, p);
    switch (head_dim) {
        case 64: return launch_after(p.state ? combine_state_kernel<64> : combine_kernel<64, 64>, grid, n, 0, s, p);
        case 128:
            return launch_after(p.state ? combine_state_kernel<128>
                                        : narrow ? combine_kernel<128, 64> : combine_kernel<128, 128>, grid, n, 0, s, p);
        case 256:
            return launch_after(p.state ? combine_state_kernel<256>
                                        : narrow ? combine_kernel<256, 64> : combine_kernel<256, 256>, grid, n, 0, s, p);
    }
    return cudaErrorInvalidValue;
}

cudaError_t launch_combine_shared(int head_dim, const DecodeParams &p, const SharedParts &parts, cudaStream_t s) {
    const int64_t rows = (int64_t)p.n_q_heads * p.B * p.n_layers_run;
    const unsigned grid = (unsigned)((rows + kCombineRows - 1) / kCombineRows);
    switch (head_dim) {
        case 64: return launch_after(combine_shared_kernel<64>, grid, 32 * kCombineRows, 0, s, p, parts);
        case 128: return launch_after(combine_shared_kernel<128>, grid, 32 * kCombineRows, 0, s, p, parts);
        case 256: return launch_after(combine_shared_kernel<256>, grid, 32 * kCombineRows, 0, s, p, parts);
    }
    return cudaErrorInvalidValue;
}

cudaError_t launch_state_finish(const float *state, int64_t n_rows, int head_dim, __nv_bfloat16 *out,
                                cudaStream_t s) {
    const int64_t n = n_rows * head_dim;
    if (n == 0) return cudaSuccess;
    int64_t grid = (n + 255) / 256;
    if (grid > 65535) grid = 65535;
    return launch_after(state_finish_kernel, (int)grid, 256, 0, s, state, n_rows, head_dim, out);
}

}  // namespace kvg
