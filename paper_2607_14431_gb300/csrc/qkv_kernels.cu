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
// same for all its heads, are made once, in shared memory.  A head is D / 16
// lanes of two 16-byte pieces: of a rotated half-pair head the same 8 columns of
// both halves, so that no pair is split over lanes, and two columns go through
// each instruction (f32x2).
// One layer of 8,191 rows of the 12B shape (268 MB): 95.6 us with a CTA per
// token and the other half of a pair fetched by shuffles, 56.3 us with a CTA per
// run of tokens and two 8-byte pieces a lane (136 instructions for a warp's 256
// columns), 47.9 us this way (98; 5.6 TB/s), with the same bits.  What is left is
// instruction issue and the latency of a lane's chain (half of the issue slots).
//
// The angle: p f_i / (2 pi) turns as a 64-bit fixed-point product that wraps at
// whole turns.  What it is off by: the fraction in fp32 2^-26 turns, and p f_i /
// (2 pi) times 2^-50 of the host's fp64 f_i, as much at position 2^26; an fp32
// product would be off by 6e-3 radians (10^-3 turns) at position 100,000.
//
// Positions on several axes (images and video: time, height, width): pair i
// turns by the token's position on the pair's axis.  Only the angles differ, and
// they are made once a token, so a row costs what it does with one axis; the
// axis is in the top two bits of the pair's turns, which leaves the loop over
// the pairs without a second table.
#include <algorithm>

#include "common.cuh"
#include "tcgen05.cuh"

namespace kvg {

namespace {

constexpr int kQkvThreads = 256;
constexpr int kQkvUnroll = 2;  // rows of a lane in flight
constexpr int kQkvTurns = 8;   // tokens whose angles are made together

// Sixteen columns of a row as they are handled: pairs (a, b), two to an
// instruction.  A lane's two pieces of eight hold a and b (half pairs), or pairs
// side by side.
struct Columns {
    float2 a[4], b[4];
};
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
template <bool HALF>
__device__ __forceinline__ Columns unpack(const uint4 &x, const uint4 &y) {
    const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    Columns c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (HALF) {
            c.a[i] = make_float2(lo16(w[i]), hi16(w[i]));
            c.b[i] = make_float2(lo16(w[4 + i]), hi16(w[4 + i]));
        } else {
            c.a[i] = make_float2(lo16(w[2 * i]), lo16(w[2 * i + 1]));
            c.b[i] = make_float2(hi16(w[2 * i]), hi16(w[2 * i + 1]));
        }
    }
    return c;
}

// Neighbouring columns 2 i and 2 i + 1 of the lane's.
template <bool HALF>
__device__ __forceinline__ float2 in_order(const Columns &c, int i) {
    if constexpr (HALF)
        return i < 4 ? c.a[i % 4] : c.b[i % 4];
    else
        return i % 2 ? make_float2(c.a[i / 2].y, c.b[i / 2].y) : make_float2(c.a[i / 2].x, c.b[i / 2].x);
}

template <bool HALF>
__device__ __forceinline__ void pack_bf16(const Columns &c, uint4 &x, uint4 &y) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 v = in_order<HALF>(c, i);
        const __nv_bfloat162 t = __floats2bfloat162_rn(v.x, v.y);
        w[i] = *reinterpret_cast<const uint32_t *>(&t);
    }
    x = make_uint4(w[0], w[1], w[2], w[3]);
    y = make_uint4(w[4], w[5], w[6], w[7]);
}

// fp32 times the reciprocal scale (one rounding), to the E4M3 grid (nearest
// even, saturating at +-448), as every append into an fp8 cache.
template <bool HALF>
__device__ __forceinline__ void pack_e4m3(const Columns &c, float inv_scale, uint2 &x, uint2 &y) {
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 v = mul2(in_order<HALF>(c, i), make_float2(inv_scale, inv_scale));
        uint16_t e;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(e) : "f"(v.y), "f"(v.x));
        h[i] = e;
    }
    x = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
    y = make_uint2(h[4] | (h[5] << 16), h[6] | (h[7] << 16));
}

template <int D, bool FP8, bool HALF>
__global__ void __launch_bounds__(kQkvThreads, 2) append_qkv_kernel(const __grid_constant__ QkvParams p) {
    constexpr int LPR = D / 16;              // lanes of a row
    constexpr int RPP = kQkvThreads / LPR;   // rows that the CTA's threads hold at once
    constexpr int E = FP8 ? 1 : 2;           // bytes of a cached element
    // A lane's eight pairs lie in four float4s, LPR apart (no bank conflicts).
    __shared__ float4 trig[kQkvTurns][4][LPR];      // cos and sin of two pairs each, of some tokens
    __shared__ float4 weight[2][4][LPR];            // of queries and keys, offset included: a of two pairs, b of them
    __shared__ int places[2][kMaxAxes][kQkvTurns];  // positions of those tokens and of the next
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
    const bool turns = 16 * lane < R;  // the lane's columns are rotated
    // its pieces: columns [c0, c0 + 8) and [c0 + c1, c0 + c1 + 8)
    const int c0 = HALF && turns ? 8 * lane : 16 * lane, c1 = HALF && turns ? R / 2 : 8;
    const int n_q = p.n_q_heads, n_qk = n_q + p.n_kv_heads, n_rows = n_qk + p.n_kv_heads;
    const bool norms = p.q_norm || p.k_norm;
    const float eps = p.eps, k_inv = p.k_inv_scale, v_inv = p.v_inv_scale;
    const int64_t page_elems = (int64_t)p.n_kv_heads * P * D, out_token = (int64_t)n_q * D;

    after_previous();
    // (the first group of lanes for queries, the second for keys)
    if (grp < 2 && (grp ? p.k_norm : p.q_norm)) {
        const uint16_t *const from = (grp ? p.k_norm : p.q_norm) + (int64_t)lr * D + c0;
        const float2 offset = make_float2(p.norm_offset, p.norm_offset);
        const Columns w = unpack<HALF>(*reinterpret_cast<const uint4 *>(from), *reinterpret_cast<const uint4 *>(from + c1));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = add2(w.a[i], offset), b = add2(w.b[i], offset);
            weight[grp][i][lane] = make_float4(a.x, a.y, b.x, b.y);
        }
    }
    // Cos and sin of the tokens [t, t + kQkvTurns): all threads for all of them,
    // so that two barriers serve eight tokens and no warp waits for another's
    // few pairs (with a barrier per token half of the stalls were there).  A thread
    // makes those of one pair.
    const int pair = threadIdx.x % (D / 2);
    const uint64_t turn_of = pair < R / 2 ? p.turn[pair] : 0;
    auto fetch = [&](int t, int buf) {
        const int axis = threadIdx.x / kQkvTurns, k = threadIdx.x % kQkvTurns;
        if (axis < p.n_axes && t + k < end) places[buf][axis][k] = p.pos[axis * p.n_tokens + p.tok0 + t + k];
    };
    auto turn = [&](int t, int buf) {
        __syncthreads();  // the angles before are used, the positions are there
        const int n = min(kQkvTurns, end - t);
        if (pair < R / 2)
            for (int k = threadIdx.x / (D / 2); k < n; k += kQkvThreads / (D / 2)) {
                // of a turn, times 2^64
                const uint64_t frac = (uint64_t)(int64_t)places[buf][turn_of >> kAxisShift][k] *
                                      (turn_of & (((uint64_t)1 << kAxisShift) - 1));
                float sv, cv;
                sincospif((float)(int32_t)(frac >> 32) * 0x1p-31f, &sv, &cv);
                reinterpret_cast<float2 *>(&trig[k][pair % 8 / 2][pair / 8])[pair % 2] =
                    make_float2(cv * p.attention_factor, sv * p.attention_factor);
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
        auto load = [&](uint4 (&x)[kQkvUnroll][2]) {
#pragma unroll
            for (int u = 0; u < kQkvUnroll; ++u) {
                if (kind[u] < 3) {
                    x[u][0] = *reinterpret_cast<const uint4 *>(src[u]);
                    x[u][1] = *reinterpret_cast<const uint4 *>(src[u] + c1);
                }
                src[u] += step[u];
            }
        };
        // where token t goes: kept from token to token, looked up at a page's or a segment's end
        int b = b0 - 1, seg_end = t0, pg = 0, row = P - 1, buf = 0, k = kQkvTurns;
        int64_t at_slot = 0, at_query = 0;
        uint4 xa[kQkvUnroll][2] = {}, xb[kQkvUnroll][2] = {};
        __syncthreads();  // (a batch before is done with the positions)
        fetch(t0, 0);
        load(xa);
        auto token = [&](int t, const uint4 (&x)[kQkvUnroll][2], uint4 (&ahead)[kQkvUnroll][2]) {
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
                p.positions[seq * p.max_slots + (int64_t)pg * P + row] = places[buf ^ 1][0][k];
                // a page's last row of this launch knows its fill
                if (row == P - 1 || t + 1 == seg_end) {
                    p.page_table[seq * p.max_pages + pg] = p.pids[p.pid0[b] + pg - p.slot0[b] / P];
                    p.page_fill[seq * p.max_pages + pg] = row + 1;
                }
            }
            if (t + 1 < end) load(ahead);  // the next token's, while this one's are worked on
#pragma unroll
            for (int u = 0; u < kQkvUnroll; ++u) {
                Columns y = unpack<HALF>(x[u][0], x[u][1]);
                if (norms && __any_sync(0xffffffffu, kind[u] < 2)) {
                    // the first eight columns' sum and the others', each over the row's lanes
                    float ss[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // (columns that are not rotated: four and four of a piece)
                        const bool side = HALF && !turns;
                        ss[h] = 0.f;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 a = h && side ? y.b[i] : y.a[2 * h + i];
                            const float2 d = side && !h ? y.a[2 + i] : y.b[2 * h + i];
                            ss[h] = __fmaf_rn(a.x, a.x, __fmaf_rn(d.x, d.x, ss[h]));
                            ss[h] = __fmaf_rn(a.y, a.y, __fmaf_rn(d.y, d.y, ss[h]));
                        }
                    }
                    // (the lanes' halves take one sum each from the first step on)
                    const bool second = lane & (LPR / 2);
                    float v = second ? ss[1] : ss[0];
                    v += __shfl_xor_sync(0xffffffffu, second ? ss[0] : ss[1], LPR / 2);
#pragma unroll
                    for (int o = LPR / 4; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                    v += __shfl_xor_sync(0xffffffffu, v, LPR / 2);
                    const float rms = rsqrtf(v * (1.f / D) + eps);
                    if (kind[u] < 2 && (kind[u] ? p.k_norm : p.q_norm)) {
                        const float2 r = make_float2(rms, rms);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 w = weight[kind[u]][i][lane];
                            y.a[i] = mul2(y.a[i], mul2(r, make_float2(w.x, w.y)));
                            y.b[i] = mul2(y.b[i], mul2(r, make_float2(w.z, w.w)));
                        }
                    }
                }
                if (kind[u] == 3) continue;
                if (turns && kind[u] < 2) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 cs = trig[k][i][lane];
                        const float2 a = y.a[i], d = y.b[i], c = make_float2(cs.x, cs.z);
                        y.a[i] = fma2(d, make_float2(-cs.y, -cs.w), mul2(a, c));
                        y.b[i] = fma2(a, make_float2(cs.y, cs.w), mul2(d, c));
                    }
                }
                uint8_t *const to = dst[u] + (kind[u] ? at_slot : at_query);
                if (!FP8 && kind[u] == 2) {
                    *reinterpret_cast<uint4 *>(to) = x[u][0];
                    *reinterpret_cast<uint4 *>(to + 2 * c1) = x[u][1];
                } else if (FP8 && kind[u]) {
                    uint2 y0, y1;
                    pack_e4m3<HALF>(y, kind[u] == 2 ? v_inv : k_inv, y0, y1);
                    *reinterpret_cast<uint2 *>(to) = y0;
                    *reinterpret_cast<uint2 *>(to + c1) = y1;
                } else {
                    uint4 y0, y1;
                    pack_bf16<HALF>(y, y0, y1);
                    *reinterpret_cast<uint4 *>(to) = y0;
                    *reinterpret_cast<uint4 *>(to + 2 * c1) = y1;
                }
            }
            ++k;
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
