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
// run of tokens, one after the other, the next one's rows on their way while
// the current one's are worked on; the cos and sin of a token's position, the
// same for all its heads, are made once, in shared memory.  A head is D / 8
// lanes of two 8-byte pieces: of a rotated half-pair head the same 4 columns of
// both halves, so that no pair is split over lanes.  A lane keeps its columns
// for all rows: weights, cos and sin stay in registers.
// One layer of 8,191 rows of the 12B shape (268 MB): 95.6 us with a CTA per
// token and the other half of a pair fetched by shuffles, 56.3 us this way (4.8
// TB/s; the rest of the time is instruction issue: some 60 a piece of a row).
//
// The angle: p f_i / (2 pi) turns as a 64-bit fixed-point product that wraps at
// whole turns.  What it is off by: the fraction in fp32 2^-26 turns, and p f_i /
// (2 pi) times 2^-50 of the host's fp64 f_i, as much at position 2^26; an fp32
// product would be off by 6e-3 radians (10^-3 turns) at position 100,000.
#include <algorithm>

#include "common.cuh"

namespace kvg {

namespace {

constexpr int kQkvThreads = 256;
constexpr int kQkvUnroll = 4;  // rows of a lane in flight
constexpr int kQkvTurns = 8;   // tokens whose angles are made together

// Eight columns of a row as they are handled: pairs (a[i], b[i]).  A lane's two
// pieces hold a and b (half pairs), or pairs side by side.
template <bool HALF>
__device__ __forceinline__ void unpack(const uint2 &x, const uint2 &y, float (&a)[4], float (&b)[4]) {
    const uint32_t w[4] = {x.x, x.y, y.x, y.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
        if constexpr (HALF) {
            (i < 2 ? a : b)[2 * i % 4] = lo;
            (i < 2 ? a : b)[2 * i % 4 + 1] = hi;
        } else {
            a[i] = lo;
            b[i] = hi;
        }
    }
}

// The eight values in the order of their columns.
template <bool HALF>
__device__ __forceinline__ float in_order(const float (&a)[4], const float (&b)[4], int i) {
    return HALF ? (i < 4 ? a[i % 4] : b[i % 4]) : (i % 2 ? b[i / 2] : a[i / 2]);
}

template <bool HALF>
__device__ __forceinline__ void pack_bf16(const float (&a)[4], const float (&b)[4], uint2 &x, uint2 &y) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(in_order<HALF>(a, b, 2 * i), in_order<HALF>(a, b, 2 * i + 1));
        w[i] = *reinterpret_cast<const uint32_t *>(&t);
    }
    x = make_uint2(w[0], w[1]);
    y = make_uint2(w[2], w[3]);
}

// fp32 times the reciprocal scale (one rounding), to the E4M3 grid (nearest
// even, saturating at +-448), as every append into an fp8 cache.
template <bool HALF>
__device__ __forceinline__ void pack_e4m3(const float (&a)[4], const float (&b)[4], float inv_scale, uint32_t &x, uint32_t &y) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __fmul_rn(in_order<HALF>(a, b, 2 * i), inv_scale);
        const float hi = __fmul_rn(in_order<HALF>(a, b, 2 * i + 1), inv_scale);
        uint16_t c;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
        h[i] = c;
    }
    x = h[0] | (h[1] << 16);
    y = h[2] | (h[3] << 16);
}

template <int D, bool FP8, bool HALF>
__global__ void __launch_bounds__(kQkvThreads, 2) append_qkv_kernel(const __grid_constant__ QkvParams p) {
    constexpr int LPR = D / 8;               // lanes of a row
    constexpr int RPP = kQkvThreads / LPR;   // rows that the CTA's threads hold at once
    constexpr int E = FP8 ? 1 : 2;           // bytes of a cached element
    __shared__ float2 trig[kQkvTurns][D / 2];  // of some tokens
    __shared__ int places[2][kQkvTurns];     // positions of them and of the next
    const int lr = blockIdx.y;
    const int lane = threadIdx.x % LPR, grp = threadIdx.x / LPR;
    // the CTA's tokens [t0, end) of the launch
    const int n_tokens = p.first[p.n_seg];
    const int t0 = (int)((int64_t)n_tokens * blockIdx.x / gridDim.x);
    const int end = (int)((int64_t)n_tokens * (blockIdx.x + 1) / gridDim.x);
    int b0 = 0;
    for (int hi = p.n_seg - 1; b0 < hi;) {  // largest segment that starts at or before t0
        const int mid = (b0 + hi + 1) >> 1;
        if (p.first[mid] <= t0)
            b0 = mid;
        else
            hi = mid - 1;
    }
    const int P = p.page_size, R = p.rotary_dim;
    const bool turns = 8 * lane < R;  // the lane's columns are rotated
    // its pieces: columns [c0, c0 + 4) and [c0 + c1, c0 + c1 + 4)
    const int c0 = HALF && turns ? 4 * lane : 8 * lane, c1 = HALF && turns ? R / 2 : 4;
    const int n_q = p.n_q_heads, n_qk = n_q + p.n_kv_heads, n_rows = n_qk + p.n_kv_heads;
    const bool norms = p.q_norm || p.k_norm;
    const float eps = p.eps, k_inv = p.k_inv_scale, v_inv = p.v_inv_scale;
    const int64_t page_elems = (int64_t)p.n_kv_heads * P * D, out_token = (int64_t)n_q * D;

    after_previous();
    float wq[8], wk[8];  // weights and offset, a then b of the lane's pairs
#pragma unroll
    for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 1.f;
    auto weights = [&](const uint16_t *w, float (&to)[8]) {
        w += (int64_t)lr * D + c0;
        float a[4], d[4];
        unpack<HALF>(*reinterpret_cast<const uint2 *>(w), *reinterpret_cast<const uint2 *>(w + c1), a, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            to[i] = a[i] + p.norm_offset;
            to[4 + i] = d[i] + p.norm_offset;
        }
    };
    if (p.q_norm) weights(p.q_norm, wq);
    if (p.k_norm) weights(p.k_norm, wk);
    // Cos and sin of the tokens [t, t + kQkvTurns): all threads for all of them,
    // so that two barriers serve eight tokens and no warp waits for another's
    // few pairs (with a barrier per token half of the stalls were there).
    const int pairs = R / 2;
    auto fetch = [&](int t, int buf) {
        if (threadIdx.x < kQkvTurns && t + (int)threadIdx.x < end) places[buf][threadIdx.x] = p.pos[p.tok0 + t + threadIdx.x];
    };
    auto turn = [&](int t, int buf) {
        __syncthreads();  // the angles before are used, the positions are there
        const int n = min(kQkvTurns, end - t) * pairs;
        for (int i = threadIdx.x; i < n; i += kQkvThreads) {
            const int k = i / pairs, pair = i - k * pairs;
            const uint64_t frac = (uint64_t)(int64_t)places[buf][k] * p.turn[pair];  // of a turn, times 2^64
            float sv, cv;
            sincospif((float)(int32_t)(frac >> 32) * 0x1p-31f, &sv, &cv);
            trig[k][pair] = make_float2(cv * p.attention_factor, sv * p.attention_factor);
        }
        __syncthreads();
    };

    // head rows in batches of RPP * kQkvUnroll; most models have one
    for (int base = 0; base < n_rows; base += RPP * kQkvUnroll) {
        // The lane's rows: where their first token is, how far the next one, and
        // where they go (queries: from token to token; rows: from the page's slot)
        const uint16_t *src[kQkvUnroll];
        int64_t step[kQkvUnroll];
        uint8_t *dst[kQkvUnroll];
        int kind[kQkvUnroll];  // 0 query, 1 key, 2 value, 3 none
#pragma unroll
        for (int u = 0; u < kQkvUnroll; ++u) {
            const int h = base + u * RPP + grp;
            kind[u] = h < n_q ? 0 : h < n_qk ? 1 : h < n_rows ? 2 : 3;
            const int head = h - (kind[u] == 0 ? 0 : kind[u] == 1 ? n_q : n_qk);
            const uint16_t *x = kind[u] == 0 ? p.q + lr * p.q_layer : kind[u] == 1 ? p.k + lr * p.k_layer : p.v + lr * p.v_layer;
            step[u] = kind[u] == 0 ? p.q_token : kind[u] == 1 ? p.k_token : p.v_token;
            src[u] = x + (p.tok0 + t0) * step[u] + (kind[u] == 3 ? 0 : head * D) + c0;
            dst[u] = kind[u] == 0
                         ? reinterpret_cast<uint8_t *>(p.q_out + (lr * p.n_tokens + p.tok0 + t0) * out_token + head * D + c0)
                         : p.pool + ((((int64_t)(p.layer0 + lr) * 2 + (kind[u] == 2)) * p.pool_pages * p.n_kv_heads + head) * P * D + c0) * E;
        }
        auto load = [&](uint2 (&x)[kQkvUnroll][2]) {
#pragma unroll
            for (int u = 0; u < kQkvUnroll; ++u) {
                if (kind[u] < 3) {
                    x[u][0] = *reinterpret_cast<const uint2 *>(src[u]);
                    x[u][1] = *reinterpret_cast<const uint2 *>(src[u] + c1);
                }
                src[u] += step[u];
            }
        };
        // where token t goes: kept from token to token, looked up at a page's or a segment's end
        int b = b0 - 1, seg_end = t0, pg = 0, row = P - 1, buf = 0, k = kQkvTurns;
        int64_t at_slot = 0, at_query = 0;
        uint2 xa[kQkvUnroll][2] = {}, xb[kQkvUnroll][2] = {};
        __syncthreads();  // (a batch before is done with the positions)
        fetch(t0, 0);
        load(xa);
        auto token = [&](int t, const uint2 (&x)[kQkvUnroll][2], uint2 (&ahead)[kQkvUnroll][2]) {
            if (k == kQkvTurns) {
                turn(t, buf);
                fetch(t + kQkvTurns, buf ^= 1);
                k = 0;
            }
            const bool new_segment = t == seg_end, new_page = !new_segment && ++row == P;
            if (new_segment) {
                ++b;
                seg_end = p.first[b + 1];
                const int slot = p.slot0[b] + (t - p.first[b]);
                pg = slot / P;
                row = slot - pg * P;
            } else if (new_page) {
                ++pg;
                row = 0;
            }
            at_slot += D * E;
            if (new_segment || new_page)
                at_slot = (p.pids[p.pid0[b] + pg - p.slot0[b] / P] * page_elems + (int64_t)row * D) * E;
            if (p.write_meta && base == 0 && lr == 0 && threadIdx.x == 0) {
                const int64_t seq = p.seq[b];
                p.positions[seq * p.max_slots + (int64_t)pg * P + row] = places[buf ^ 1][k];
                // a page's last row of this launch knows its fill
                if (row == P - 1 || t + 1 == seg_end) {
                    p.page_table[seq * p.max_pages + pg] = p.pids[p.pid0[b] + pg - p.slot0[b] / P];
                    p.page_fill[seq * p.max_pages + pg] = row + 1;
                }
            }
            float c[4], s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 cs = turns ? trig[k][4 * lane + i] : make_float2(1.f, 0.f);
                c[i] = cs.x;
                s[i] = cs.y;
            }
            ++k;
            if (t + 1 < end) load(ahead);  // the next token's, while this one's are worked on
#pragma unroll
            for (int u = 0; u < kQkvUnroll; ++u) {
                float f[4], g[4];
                unpack<HALF>(x[u][0], x[u][1], f, g);
                if (norms && __any_sync(0xffffffffu, kind[u] < 2)) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) ss = __fmaf_rn(f[i], f[i], __fmaf_rn(g[i], g[i], ss));
#pragma unroll
                    for (int o = LPR / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                    const float rms = rsqrtf(ss * (1.f / D) + eps);
                    auto scale = [&](const float (&w)[8]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f[i] *= rms * w[i];
                            g[i] *= rms * w[4 + i];
                        }
                    };
                    if (kind[u] == 0 && p.q_norm) scale(wq);
                    if (kind[u] == 1 && p.k_norm) scale(wk);
                }
                if (kind[u] == 3) continue;
                if (turns && kind[u] < 2) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = f[i], d = g[i];
                        f[i] = __fmaf_rn(-d, s[i], a * c[i]);
                        g[i] = __fmaf_rn(a, s[i], d * c[i]);
                    }
                }
                uint8_t *const to = dst[u] + (kind[u] ? at_slot : at_query);
                if (!FP8 && kind[u] == 2) {
                    *reinterpret_cast<uint2 *>(to) = x[u][0];
                    *reinterpret_cast<uint2 *>(to + 2 * c1) = x[u][1];
                } else if (FP8 && kind[u]) {
                    uint32_t y0, y1;
                    pack_e4m3<HALF>(f, g, kind[u] == 2 ? v_inv : k_inv, y0, y1);
                    *reinterpret_cast<uint32_t *>(to) = y0;
                    *reinterpret_cast<uint32_t *>(to + c1) = y1;
                } else {
                    uint2 y0, y1;
                    pack_bf16<HALF>(f, g, y0, y1);
                    *reinterpret_cast<uint2 *>(to) = y0;
                    *reinterpret_cast<uint2 *>(to + 2 * c1) = y1;
                }
            }
            at_query += out_token * 2;
        };
        for (int t = t0; t < end; t += 2) {
            token(t, xa, xb);
            if (t + 1 < end) token(t + 1, xb, xa);
        }
    }
}

template <int D, bool FP8>
cudaError_t run_qkv(const QkvParams &p, int n_sm, cudaStream_t s) {
    const dim3 grid(std::min(p.first[p.n_seg], std::max(1, 2 * n_sm / p.n_layers_run)), p.n_layers_run);
    return launch_after(p.rotary_half ? append_qkv_kernel<D, FP8, true> : append_qkv_kernel<D, FP8, false>, grid,
                        kQkvThreads, 0, s, p);
}

}  // namespace

cudaError_t launch_append_qkv(int head_dim, bool fp8, const QkvParams &p, int n_sm, cudaStream_t s) {
    switch (head_dim) {
        case 64: return fp8 ? run_qkv<64, true>(p, n_sm, s) : run_qkv<64, false>(p, n_sm, s);
        case 128: return fp8 ? run_qkv<128, true>(p, n_sm, s) : run_qkv<128, false>(p, n_sm, s);
        case 256: return fp8 ? run_qkv<256, true>(p, n_sm, s) : run_qkv<256, false>(p, n_sm, s);
    }
    return cudaErrorInvalidValue;
}

}  // namespace kvg
