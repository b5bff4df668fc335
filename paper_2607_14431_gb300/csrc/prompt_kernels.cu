// prompt_kernels.cu — causal attention of packed prompt rows over a paged
// cache (Sec. 3.2: new queries are computed on top of a restored block).
//
// Query row i of a sequence, at slot s_i, attends to its valid rows (below
// their page's fill) in slots [lo_i, s_i]:
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j
// with lo_i = 0, or the slot of the last `window` valid rows up to s_i.
//
// A warp takes a query head's row and walks its slots, a lane D / 32 of the
// dimensions: right for every case, and bound by the reduction per key.
#include "common.cuh"

namespace kvg {

namespace {

constexpr int kRowThreads = 128;

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

// First slot that the row at `slot` attends to.
__device__ __forceinline__ int window_first(const PromptParams &p, int b, int slot) {
    if (p.window <= 0) return 0;
    if (!p.holes[b]) return max(0, slot - p.window + 1);
    // pages that are not full lie in between: count valid rows back
    const int32_t *fill = p.page_fill + (int64_t)p.seq[b] * p.max_pages;
    int pg = slot / p.page_size, n = slot % p.page_size + 1, left = p.window;
    while (n < left && pg > 0) {
        left -= n;
        n = fill[--pg];
    }
    return pg * p.page_size + max(0, n - left);
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kRowThreads) prompt_rows_kernel(const __grid_constant__ PromptParams p) {
    constexpr int N = D / 32;
    after_previous();
    const int lane = threadIdx.x & 31;
    const int64_t n = (int64_t)p.first[p.n_seq] * p.n_q_heads;
    const int64_t at = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 5;
    if (at >= n) return;
    const int row = (int)(at / p.n_q_heads), h = (int)(at - (int64_t)row * p.n_q_heads), lr = blockIdx.y;
    int b = 0;
    for (int hi = p.n_seq - 1; b < hi;) {
        const int mid = (b + hi + 1) >> 1;
        if (p.first[mid] <= row)
            b = mid;
        else
            hi = mid - 1;
    }
    const int t = row - p.first[b], slot = p.slot0[b] + t, P = p.page_size;
    const int g = h / (p.n_q_heads / p.n_kv_heads);
    const int64_t qrow = ((int64_t)p.qlayers[lr] * p.q_rows + p.row0[b] + t) * p.n_q_heads + h;
    float q[N], o[N], m = -INFINITY, l = 0.f;
    load_row<D, false>(reinterpret_cast<const uint8_t *>(p.q + qrow * D), lane, q);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
    const int first = window_first(p, b, slot);
    constexpr int E = FP8 ? 1 : 2;
    for (int pg = first / P; pg <= slot / P; ++pg) {
        const int pid = p.page_table[(int64_t)p.seq[b] * p.max_pages + pg];
        const int fill = p.page_fill[(int64_t)p.seq[b] * p.max_pages + pg];
        if (pid < 0 || pid >= p.pool_pages) {
            record_error(p.status, KVG_ERR_DEVICE_CHECK, 1);
            continue;
        }
        const int64_t page = (int64_t)p.layers[lr] * 2 * p.pool_pages + pid;
        const uint8_t *k = p.pool + ((page * p.n_kv_heads + g) * P) * D * E;
        const uint8_t *v = k + p.pool_pages * p.n_kv_heads * P * D * E;
        const int r1 = min(fill, slot - pg * P + 1);
        for (int r = max(0, first - pg * P); r < r1; ++r) {
            float x[N], s = 0.f;
            load_row<D, FP8>(k + (int64_t)r * D * E, lane, x);
#pragma unroll
            for (int i = 0; i < N; ++i) s = __fmaf_rn(q[i], x[i], s);
#pragma unroll
            for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            s *= p.qscale;
            const float mn = fmaxf(m, s);
            const float base = mn == -INFINITY ? 0.f : mn;
            const float a = exp2f(m - base), w = exp2f(s - base);
            m = mn;
            l = __fmaf_rn(l, a, w);
            load_row<D, FP8>(v + (int64_t)r * D * E, lane, x);
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = __fmaf_rn(o[i], a, w * x[i]);
        }
    }
    const float inv = p.vscale / l;
    uint32_t *out = reinterpret_cast<uint32_t *>(p.out + qrow * D + lane * N);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const __nv_bfloat162 y = __floats2bfloat162_rn(o[2 * i] * inv, o[2 * i + 1] * inv);
        out[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
}

}  // namespace

cudaError_t launch_prompt(int head_dim, bool fp8, const PromptParams &p, cudaStream_t s) {
    const int64_t warps = (int64_t)p.first[p.n_seq] * p.n_q_heads;
    const dim3 grid((unsigned)((warps + kRowThreads / 32 - 1) / (kRowThreads / 32)), p.n_layers_run);
    switch (head_dim) {
        case 64: return launch_after(prompt_rows_kernel<64, false>, grid, kRowThreads, 0, s, p);
        case 128: return launch_after(fp8 ? prompt_rows_kernel<128, true> : prompt_rows_kernel<128, false>, grid, kRowThreads, 0, s, p);
        case 256: return launch_after(fp8 ? prompt_rows_kernel<256, true> : prompt_rows_kernel<256, false>, grid, kRowThreads, 0, s, p);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
