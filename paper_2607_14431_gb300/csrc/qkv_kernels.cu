// qkv_kernels.cu — new tokens' projections become cache rows: norm of each
// query and key head, rotary positions, and the append, in one pass.
//
// Of a head x[0, D) with rotary dimension R:
//   y[d]  = x[d] / sqrt(mean(x^2) + eps) * (w[d] + offset)     (w given)
//   z[a]  = m (y[a] cos(p f_i) - y[b] sin(p f_i))
//   z[b]  = m (y[b] cos(p f_i) + y[a] sin(p f_i))   for the R / 2 pairs (a, b)
//   z[d]  = y[d] for d >= R
// in fp32, rounded once: to bf16 (queries, bf16 caches) or to E4M3 codes.
//
// Every value is read once and written once, so memory bounds it; for a
// decode step's few rows the launch and one dependent load do.  A CTA takes a
// token: the cos and sin of its position are the same for all its heads, so a
// thread makes each pair's once, in shared memory, while the head rows' loads
// are in flight.  A row is D / 8 lanes of 16 bytes each; a lane keeps the same
// columns for all its rows, so its weights, cos and sin stay in registers, and
// the other half of a pair comes from its lane by a shuffle.
//
// The angle: p f_i / (2 pi) turns as a 64-bit fixed-point product that wraps at
// whole turns, so the fraction is good to 2^-33 turns at any position, where
// an fp32 product would be off by 6e-3 radians at position 100,000.
#include "common.cuh"

namespace kvg {

namespace {

constexpr int kQkvThreads = 256;
constexpr int kQkvUnroll = 4;  // rows of a lane in flight

__device__ __forceinline__ void unpack_bf16x8(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack_bf16x8(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&t);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// fp32 times the reciprocal scale (one rounding), to the E4M3 grid (nearest
// even, saturating at +-448), as every append into an fp8 cache.
__device__ __forceinline__ uint2 pack_e4m3x8(const float (&f)[8], float inv_scale) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __fmul_rn(f[2 * i], inv_scale), hi = __fmul_rn(f[2 * i + 1], inv_scale);
        uint16_t c;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
        h[i] = c;
    }
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kQkvThreads) append_qkv_kernel(const __grid_constant__ QkvParams p) {
    constexpr int LPR = D / 8;               // lanes of a row
    constexpr int RPP = kQkvThreads / LPR;   // rows that the CTA's threads hold at once
    __shared__ float2 trig[D / 2];
    const int t = blockIdx.x, lr = blockIdx.y;
    const int lane = threadIdx.x % LPR, grp = threadIdx.x / LPR;
    int b = 0;
    for (int hi = p.n_seg - 1; b < hi;) {  // largest segment that starts at or before t
        const int mid = (b + hi + 1) >> 1;
        if (p.first[mid] <= t)
            b = mid;
        else
            hi = mid - 1;
    }
    const int P = p.page_size;
    const int slot = p.slot0[b] + (t - p.first[b]);
    const int pg = slot / P, row = slot - pg * P;
    const int pid = p.pids[p.pid0[b] + pg - p.slot0[b] / P];
    const int64_t tok = p.tok0 + t;  // of the call's packed tokens
    const int n_rows = p.n_q_heads + 2 * p.n_kv_heads;
    const uint16_t *const q = p.q + lr * p.q_layer + tok * p.q_token + 8 * lane;
    const uint16_t *const k = p.k + lr * p.k_layer + tok * p.k_token + 8 * lane;
    const uint16_t *const v = p.v + lr * p.v_layer + tok * p.v_token + 8 * lane;

    after_previous();
    const int pos = p.pos[tok];
    if (p.write_meta && lr == 0 && threadIdx.x == 0) {
        const int64_t seq = p.seq[b];
        p.positions[seq * p.max_slots + slot] = pos;
        // a page's last row of this launch knows its fill
        if (row == P - 1 || t + 1 == p.first[b + 1]) {
            p.page_table[seq * p.max_pages + pg] = pid;
            p.page_fill[seq * p.max_pages + pg] = row + 1;
        }
    }

    const int R = p.rotary_dim;
    const bool half = p.rotary_half;
    const bool turns = 8 * lane < R;           // the lane's columns are rotated
    const bool upper = half && 16 * lane >= R; // its columns are the second of their pairs
    const int partner = (threadIdx.x & 31) + (!half || !turns ? 0 : upper ? -(R / 16) : R / 16);
    float c[8], s[8];
    uint4 wq = make_uint4(0, 0, 0, 0), wk = wq;
    if (p.q_norm) wq = reinterpret_cast<const uint4 *>(p.q_norm + (int64_t)lr * D)[lane];
    if (p.k_norm) wk = reinterpret_cast<const uint4 *>(p.k_norm + (int64_t)lr * D)[lane];

    for (int base = 0; base < n_rows; base += RPP * kQkvUnroll) {
        uint4 x[kQkvUnroll];
#pragma unroll
        for (int u = 0; u < kQkvUnroll; ++u) {
            const int h = base + u * RPP + grp;
            x[u] = make_uint4(0, 0, 0, 0);
            if (h < n_rows) {
                const int hk = h - p.n_q_heads, hv = hk - p.n_kv_heads;
                x[u] = *reinterpret_cast<const uint4 *>(hk < 0 ? q + h * D : hv < 0 ? k + hk * D : v + hv * D);
            }
        }
        if (base == 0) {
            for (int i = threadIdx.x; i < R / 2; i += kQkvThreads) {
                const uint64_t frac = (uint64_t)(int64_t)pos * p.turn[i];  // of a turn, times 2^64
                float sv, cv;
                sincospif((float)(int32_t)(frac >> 32) * 0x1p-31f, &sv, &cv);
                trig[i] = make_float2(cv * p.attention_factor, sv * p.attention_factor);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                c[j] = 1.f;
                s[j] = 0.f;
                if (turns) {
                    const float2 cs = trig[half ? 8 * lane + j - (upper ? R / 2 : 0) : 4 * lane + j / 2];
                    c[j] = cs.x;
                    s[j] = (half ? upper : j & 1) ? cs.y : -cs.y;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kQkvUnroll; ++u) {
            const int h = base + u * RPP + grp;
            const int hk = h - p.n_q_heads, hv = hk - p.n_kv_heads;
            float f[8], y[8];
            unpack_bf16x8(x[u], f);
            if (p.q_norm || p.k_norm) {
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = __fmaf_rn(f[j], f[j], ss);
#pragma unroll
                for (int o = LPR / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                if (hv < 0 && (hk < 0 ? p.q_norm : p.k_norm)) {
                    const float rms = rsqrtf(ss * (1.f / D) + p.eps);
                    float w[8];
                    unpack_bf16x8(hk < 0 ? wq : wk, w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] *= rms * (w[j] + p.norm_offset);
                }
            }
            if (R) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = half ? __shfl_sync(0xffffffffu, f[j], partner) : f[j ^ 1];
                if (turns && hv < 0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = __fmaf_rn(y[j], s[j], f[j] * c[j]);
                }
            }
            if (h >= n_rows) continue;
            if (hk < 0) {
                uint16_t *const out = p.q_out + ((lr * p.n_tokens + tok) * p.n_q_heads + h) * D;
                reinterpret_cast<uint4 *>(out)[lane] = pack_bf16x8(f);
                continue;
            }
            const int kv = hv >= 0, head = kv ? hv : hk;
            const int64_t page = ((int64_t)(p.layer0 + lr) * 2 + kv) * p.pool_pages + pid;
            const int64_t at = ((page * p.n_kv_heads + head) * P + row) * D;  // element of the pool
            if constexpr (FP8)
                reinterpret_cast<uint2 *>(p.pool + at)[lane] = pack_e4m3x8(f, kv ? p.v_inv_scale : p.k_inv_scale);
            else
                reinterpret_cast<uint4 *>(p.pool + 2 * at)[lane] = kv ? x[u] : pack_bf16x8(f);
        }
    }
    let_next_start();
}

}  // namespace

cudaError_t launch_append_qkv(int head_dim, bool fp8, const QkvParams &p, cudaStream_t s) {
    const dim3 grid(p.first[p.n_seg], p.n_layers_run);
    switch (head_dim) {
        case 64: return launch_after(fp8 ? append_qkv_kernel<64, true> : append_qkv_kernel<64, false>, grid, kQkvThreads, 0, s, p);
        case 128: return launch_after(fp8 ? append_qkv_kernel<128, true> : append_qkv_kernel<128, false>, grid, kQkvThreads, 0, s, p);
        case 256: return launch_after(fp8 ? append_qkv_kernel<256, true> : append_qkv_kernel<256, false>, grid, kQkvThreads, 0, s, p);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
