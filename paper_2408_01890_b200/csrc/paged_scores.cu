// Scores of a shared layer over a paged 8-bit cache, for the new token: the first of the decode step's two kernels (paged_decode.cu has the other).
//
//   a = W2^T act(W1^T prev + b1) + b2 + q'.K'_j / sqrt(r)     (Eq. 3-4; and the other forms of Integrate)
//
// A CTA takes CH positions of a sequence and all heads, because the aligner mixes them.  Phase 1: the differences of all heads into shared memory, a
// warp per KV head.  K' lies with the 16 positions of a block side by side, so 16 bytes are one rank at 16 positions: on mma m16n8k16 the
// rows of tile mt are positions 2 mt and 2 mt + 1 of the eight blocks, k are the ranks (up to 32, zeros beyond r), the columns the two fp16 terms of q'
// for four query heads.  Phase 2: the FFN, a warp to 16 positions (M), on mma m16n8k16 with every fp32 operand as three bf16 terms (24 bits) against the
// bf16 weights, whose products are exact: rows handed on in fp32 are what fp32 arithmetic gives.  A row that is bf16 is one term.
// With fewer than 128 positions to a CTA (small batches) the hidden units are divided over the warps and their sums added in a fixed order.
// Bytes: r of K' a KV head and position, the row in and out; bound by HBM for large batches, else by the latency of its two phases.
#include <algorithm>

#include "decode_fast.cuh"
#include "paged_decode.cuh"

namespace lisa {
namespace {

__device__ __forceinline__ void put_score(const ScoresParams& p, int b, int h, int pos, float v) {
    p.scores[b * p.s_sb + h * p.s_sh + pos] = v;
    if (p.out_scores) {
        const int64_t to = b * p.sc_sb + h * p.sc_sh + pos;
        if (p.row_bf16) st_row<true>(p.out_scores, to, v);
        else st_row<false>(p.out_scores, to, v);
    }
}

// Any head count, width, Integrate and weight type: a thread per position, fp32 throughout, weights in shared memory.
constexpr int kGeneralThreads = 128;
template <int FMT>
__global__ void __launch_bounds__(kGeneralThreads) paged_scores_general_kernel(const __grid_constant__ ScoresParams p) {
    extern __shared__ __align__(16) float smem[];
    const int b = blockIdx.y, tid = threadIdx.x, pos = blockIdx.x * kGeneralThreads + tid;
    const int Hq = p.Hq, r = p.pool.r, m = p.integrate == LISA_INTEGRATE_PLUS ? 0 : p.m;
    const int h_in = p.integrate == LISA_INTEGRATE_CONCAT ? 2 * Hq : Hq;
    float* w1_s = smem;                     // [h_in][m]
    float* w2_s = w1_s + h_in * m;          // [m][Hq]
    float* b1_s = w2_s + m * Hq;            // [m]
    float* b2_s = b1_s + m;                 // [Hq]
    float* qp_s = b2_s + Hq;                // [Hq][r]
    chain_release();
    if (m) {
        for (int e = tid; e < h_in * m; e += kGeneralThreads) w1_s[e] = ld_elem(p.w1, e, p.w_dtype);
        for (int e = tid; e < m; e += kGeneralThreads) b1_s[e] = ldw(p.b1, e, p.w_dtype);
        if (p.ffn_layers == 2) {
            for (int e = tid; e < m * Hq; e += kGeneralThreads) w2_s[e] = ld_elem(p.w2, e, p.w_dtype);
            for (int e = tid; e < Hq; e += kGeneralThreads) b2_s[e] = ldw(p.b2, e, p.w_dtype);
        }
    }
    chain_wait();
    const int L = length_of(p.seq_lens, b, p.L);
    if (blockIdx.x * kGeneralThreads >= L) return;
    for (int e = tid; e < Hq * r; e += kGeneralThreads) qp_s[e] = ld_elem(p.qp.ptr, b * p.qp.sb + e / r * p.qp.sh + e % r, p.qp.dtype);
    __syncthreads();
    if (pos >= L) return;
    const int id = p.pool.page_of(b, pos, (pos & (kPageBlock - 1)) == 0);
    uint8_t* page = p.pool.page(max(id, 0));
    const float inv_sqrt_r = rsqrtf((float)r);
    float a[kMaxHeads], dl[kMaxHeads], hid[kMaxHidden];
    for (int h = 0; h < Hq; ++h) {
        const int64_t at = b * p.prev_sb + h * p.prev_sh + pos;
        a[h] = p.row_bf16 ? ld_row<true>(p.prev, at) : ld_row<false>(p.prev, at);
        float s = 0.f;
        if (id >= 0) {
            const uint8_t* k = page + p.pool.kp_block(h / p.G, pos) + (pos & (kPageBlock - 1));
            for (int x = 0; x < r; ++x) s = fmaf(qp_s[h * r + x], code_value<FMT>(k[x * kPageBlock], 0), s);
            s *= p.pool.scales(page, h / p.G, pos)[0] * inv_sqrt_r;
        }
        dl[h] = s;
    }
    if (p.integrate == LISA_INTEGRATE_PLUS) {
        for (int h = 0; h < Hq; ++h) a[h] += dl[h];
    } else {
        for (int u = 0; u < m; ++u) {
            float s = b1_s[u];
            for (int x = 0; x < Hq; ++x) s = fmaf(a[x], w1_s[x * m + u], s);
            if (p.integrate == LISA_INTEGRATE_CONCAT)
                for (int x = 0; x < Hq; ++x) s = fmaf(dl[x], w1_s[(Hq + x) * m + u], s);
            hid[u] = s;
        }
        if (p.ffn_layers == 1) {
            for (int h = 0; h < Hq; ++h) a[h] = hid[h];
        } else {
            for (int u = 0; u < m; ++u) hid[u] = act_apply(hid[u], p.act);
            for (int h = 0; h < Hq; ++h) {
                float s = b2_s[h];
                for (int u = 0; u < m; ++u) s = fmaf(hid[u], w2_s[u * Hq + h], s);
                a[h] = s;
            }
        }
        if (p.integrate == LISA_INTEGRATE_ADD)
            for (int h = 0; h < Hq; ++h) a[h] += dl[h];
    }
    if (id < 0) return;
    for (int h = 0; h < Hq; ++h) put_score(p, b, h, pos, a[h]);
}

size_t general_smem(const ScoresParams& p) {
    const int h_in = p.integrate == LISA_INTEGRATE_CONCAT ? 2 * p.Hq : p.Hq, m = p.integrate == LISA_INTEGRATE_PLUS ? 0 : p.m;
    return sizeof(float) * ((size_t)h_in * m + (size_t)m * p.Hq + m + p.Hq + (size_t)p.Hq * p.pool.r);
}

// ---------------------------------------------------------------------------------------------
// 32 or 40 heads, bf16 weights, hidden widths that are multiples of 8 up to 256, adding or concatenating Integrate
// ---------------------------------------------------------------------------------------------
constexpr int kScoresThreads = 256;
constexpr int kScoresWarps = kScoresThreads / 32;

// Shared memory of a CTA (byte offsets): differences [HQ][CH + 4], partial FFN outputs [HS][HQ][CH + 4] (HS > 1), q' [HQ][32] and its scales, weights, biases
struct ScoresLayout {
    int y, qp, q_scale, w1, w2, b1, b2, total;
};
__host__ __device__ inline ScoresLayout scores_layout(int HQ, int CH, bool concat, int m) {
    ScoresLayout l;
    const int HS = 128 / CH, mp = (m + 15) / 16 * 16, kp = concat ? 2 * HQ : (HQ + 15) / 16 * 16;
    int off = HQ * (CH + 4) * 4;
    l.y = off; off += HS > 1 ? HS * HQ * (CH + 4) * 4 : 0;
    l.qp = off; off += HQ * kMaxRank * 4;
    l.q_scale = off; off += HQ * 4;
    l.w1 = off; off += kp * (mp + 8) * 2;
    l.w2 = off; off += mp * (HQ + 8) * 2;
    l.b1 = off; off += mp * 4;
    l.b2 = off; off += HQ * 4;
    l.total = off;
    return l;
}

// Differences of one KV head's up to four query heads h0 .. h0 + nh - 1 at the 16 positions of this lane's block
template <int FMT>
__device__ __forceinline__ void delta_blocks(const PagedView& pool, const uint8_t* page, int pos, int kvh, int h0, int nh, bool on, const float* qp_s,
                                             const float* q_scale, float* s_s, int ld) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, r = pool.r;
    const uint8_t* at = page + pool.kp_block(kvh, pos) + t * kPageBlock;
    uint32_t w[2][4][4];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = ld_stream16_or_zero(at + (16 * s + 4 * i) * kPageBlock, on && 16 * s + 4 * i + t < r);
            w[s][i][0] = v.x; w[s][i][1] = v.y; w[s][i][2] = v.z; w[s][i][3] = v.w;
        }
    const float scale = on ? pool.scales(const_cast<uint8_t*>(page), kvh, pos)[0] : 0.f;
    // column g: head g / 2's leading (even g) or second term; k-step s: ranks 16 s + 4 i + t
    uint32_t bf[2][2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float* q = qp_s + (h0 + (g >> 1)) * kMaxRank + 16 * s + 8 * e + t;
            bf[s][e] = (g >> 1) < nh ? pack16(term_of(q[0], g & 1), term_of(q[4], g & 1)) : 0u;
        }
    float c[8][4];
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) c[mt][0] = c[mt][1] = c[mt][2] = c[mt][3] = 0.f;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t y0 = biased<FMT>(w[s][0][k]), y1 = biased<FMT>(w[s][1][k]), y2 = biased<FMT>(w[s][2][k]), y3 = biased<FMT>(w[s][3][k]);
            const uint32_t lo01 = __byte_perm(y0, y1, 0x5140), hi01 = __byte_perm(y0, y1, 0x7362);
            const uint32_t lo23 = __byte_perm(y2, y3, 0x5140), hi23 = __byte_perm(y2, y3, 0x7362);
            mma_f16(c[2 * k], pair16<FMT>(lo01, false), pair16<FMT>(lo01, true), pair16<FMT>(lo23, false), pair16<FMT>(lo23, true), bf[s][0], bf[s][1]);
            mma_f16(c[2 * k + 1], pair16<FMT>(hi01, false), pair16<FMT>(hi01, true), pair16<FMT>(hi23, false), pair16<FMT>(hi23, true), bf[s][0], bf[s][1]);
        }
    if (t >= nh || !on) return;
    const float f = scale * q_scale[h0 + t];
    float4* dst = reinterpret_cast<float4*>(s_s + (h0 + t) * ld + g * kPageBlock);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        dst[k] = make_float4((c[2 * k][0] + c[2 * k][1]) * f, (c[2 * k][2] + c[2 * k][3]) * f, (c[2 * k + 1][0] + c[2 * k + 1][1]) * f,
                             (c[2 * k + 1][2] + c[2 * k + 1][3]) * f);
}

template <int HQ, int CH, bool CONCAT>
__global__ void __launch_bounds__(kScoresThreads, 2) paged_scores_kernel(const __grid_constant__ ScoresParams p, int dtype) {
    constexpr int HS = 128 / CH, LD = CH + 4, NT2 = HQ / 8, KPH = (HQ + 15) / 16, KS1 = CONCAT ? 2 * HQ / 16 : KPH, W2_LD = HQ + 8;
    extern __shared__ __align__(16) uint8_t smem_b[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int b = blockIdx.y, j0 = blockIdx.x * CH, m = p.m, mp = (m + 15) / 16 * 16, w1_ld = mp + 8;
    const ScoresLayout lay = scores_layout(HQ, CH, CONCAT, m);
    float* s_s = reinterpret_cast<float*>(smem_b);
    float* y_s = reinterpret_cast<float*>(smem_b + lay.y);
    float* qp_s = reinterpret_cast<float*>(smem_b + lay.qp);
    float* q_scale = reinterpret_cast<float*>(smem_b + lay.q_scale);
    __nv_bfloat16* w1_s = reinterpret_cast<__nv_bfloat16*>(smem_b + lay.w1);     // [inputs][mp + 8], zero rows and columns beyond the FFN's sizes
    __nv_bfloat16* w2_s = reinterpret_cast<__nv_bfloat16*>(smem_b + lay.w2);     // [mp][HQ + 8]
    float* b1_s = reinterpret_cast<float*>(smem_b + lay.b1);
    float* b2_s = reinterpret_cast<float*>(smem_b + lay.b2);
    chain_release();
    // the aligner's weights are constants of the model: staged while the kernel before this one may still be running
    const int c8 = mp / 8;
    for (int e = tid; e < KS1 * 16 * c8; e += kScoresThreads) {
        const int k = e / c8, c = (e - k * c8) * 8;
        *reinterpret_cast<uint4*>(w1_s + k * w1_ld + c) = k < (CONCAT ? 2 * HQ : HQ) && c < m
            ? *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.w1) + k * m + c) : make_uint4(0u, 0u, 0u, 0u);
    }
    for (int e = tid; e < mp * NT2; e += kScoresThreads) {
        const int k = e / NT2, c = e % NT2 * 8;
        *reinterpret_cast<uint4*>(w2_s + k * W2_LD + c) = k < m
            ? *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.w2) + k * HQ + c) : make_uint4(0u, 0u, 0u, 0u);
    }
    for (int e = tid; e < mp; e += kScoresThreads) b1_s[e] = e < m ? ldw(p.b1, e, p.w_dtype) : 0.f;
    for (int e = tid; e < HQ; e += kScoresThreads) b2_s[e] = ldw(p.b2, e, p.w_dtype);
    chain_wait();
    const int L = length_of(p.seq_lens, b, p.L);
    if (j0 >= L) return;

    // this lane's block of the chunk
    const int blk_pos = j0 + g * kPageBlock;
    const int id = g < CH / kPageBlock && blk_pos < L ? p.pool.page_of(b, blk_pos, warp == 0 && t == 0) : -1;
    const uint8_t* page = p.pool.page(max(id, 0));
    // the previous scores of the FFN phase: asked for now
    const int strip = warp % (CH / 16), hs = warp / (CH / 16), p0 = strip * 16 + g, p1 = p0 + 8;
    const bool ok0 = j0 + p0 < L, ok1 = j0 + p1 < L;
    float pv[KPH * 4][2];               // slots 2 i, 2 i + 1: heads 8 i + 2t, + 1
    auto load_prev = [&](const auto* row) {
        row += b * p.prev_sb + j0 + 2 * t * p.prev_sh;
#pragma unroll
        for (int i = 0; i < KPH * 2; ++i) {
            const bool in = i < HQ / 8;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const auto* at = row + (8 * i + e) * p.prev_sh;
                pv[2 * i + e][0] = in && ok0 ? (float)at[p0] : 0.f;
                pv[2 * i + e][1] = in && ok1 ? (float)at[p1] : 0.f;
            }
        }
    };
    if (p.row_bf16) load_prev(static_cast<const __nv_bfloat16*>(p.prev));
    else load_prev(static_cast<const float*>(p.prev));

    // q', each head brought to [2^13, 2^14) by a power of two
    for (int h = warp; h < HQ; h += kScoresWarps) {
        const float x = lane < p.pool.r ? ld_elem(p.qp.ptr, b * p.qp.sb + h * p.qp.sh + lane, p.qp.dtype) : 0.f;
        const int ex = exponent(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu)));
        qp_s[h * kMaxRank + lane] = x * pow2(13 - ex);
        if (lane == 0) q_scale[h] = pow2(ex - 13) * rsqrtf((float)p.pool.r);
    }
    if (CH < 128 || j0 + CH > L)        // absent blocks: their differences are zeros
        for (int e = tid; e < HQ * LD; e += kScoresThreads) s_s[e] = 0.f;
    __syncthreads();
    const int passes = (p.G + 3) / 4, nv = p.pool.Hkv * passes;
    for (int v = warp; v < nv; v += kScoresWarps) {
        const int kvh = v / passes, q0 = v % passes * 4, nh = min(4, p.G - q0);
        if (dtype == LISA_S8) delta_blocks<LISA_S8>(p.pool, page, blk_pos, kvh, kvh * p.G + q0, nh, id >= 0, qp_s, q_scale, s_s, LD);
        else delta_blocks<LISA_E4M3>(p.pool, page, blk_pos, kvh, kvh * p.G + q0, nh, id >= 0, qp_s, q_scale, s_s, LD);
    }
    __syncthreads();

    // the FFN: a warp owns 16 positions and every HS-th block of 16 hidden units
    float yacc[NT2][4];
#pragma unroll
    for (int j = 0; j < NT2; ++j) {
        const float x = hs == 0 ? b2_s[j * 8 + 2 * t] : 0.f, y = hs == 0 ? b2_s[j * 8 + 2 * t + 1] : 0.f;
        yacc[j][0] = x; yacc[j][1] = y; yacc[j][2] = x; yacc[j][3] = y;
    }
    uint32_t afr[KS1][3][4];
#pragma unroll
    for (int ks = 0; ks < KS1; ++ks)
#pragma unroll
        for (int q = 0; q < 4; ++q) {   // operand register q: rows g (+ 8), inputs 2t, 2t + 1 (+ 8)
            const int k8 = ks * 16 + (q & 2 ? 8 : 0);
            float x, y;
            if (k8 < KPH * 16 && !(CONCAT && k8 >= HQ)) {
                x = pv[k8 / 4][q & 1]; y = pv[k8 / 4 + 1][q & 1];
            } else {
                const float* d = s_s + (k8 - HQ + 2 * t) * LD + (q & 1 ? p1 : p0);
                x = d[0]; y = d[LD];
            }
            split3(x, y, afr[ks][0][q], afr[ks][1][q], afr[ks][2][q]);
        }
    const bool one_term = p.row_bf16 && !CONCAT;      // (a bf16 row is its own first term)
    const int lk = (lane & 7) + (lane & 8 ? 8 : 0), ln = lane & 16 ? 8 : 0;   // row and column half this lane addresses for ldmatrix
    for (int blk = hs; blk < mp / 16; blk += HS) {
        float hacc[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            hacc[u][0] = hacc[u][2] = b1_s[blk * 16 + u * 8 + 2 * t];
            hacc[u][1] = hacc[u][3] = b1_s[blk * 16 + u * 8 + 2 * t + 1];
        }
#pragma unroll
        for (int ks = 0; ks < KS1; ++ks) {
            uint32_t w[4];
            ldsm_x4_trans(w, w1_s + (ks * 16 + lk) * w1_ld + blk * 16 + ln);
            if (!one_term) {
#pragma unroll
                for (int q = 2; q >= 1; --q) {        // smallest terms first
                    mma_bf16(hacc[0], afr[ks][q], w[0], w[1]);
                    mma_bf16(hacc[1], afr[ks][q], w[2], w[3]);
                }
            }
            mma_bf16(hacc[0], afr[ks][0], w[0], w[1]);
            mma_bf16(hacc[1], afr[ks][0], w[2], w[3]);
        }
        uint32_t hfr[3][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                split3(act_apply(hacc[u][2 * e], p.act), act_apply(hacc[u][2 * e + 1], p.act), hfr[0][2 * u + e], hfr[1][2 * u + e], hfr[2][2 * u + e]);
#pragma unroll
        for (int j = 0; j < NT2; j += 2) {
            uint32_t w[4];
            const __nv_bfloat16* src = w2_s + (blk * 16 + lk) * W2_LD + j * 8;
            if (j + 1 < NT2) ldsm_x4_trans(w, src + ln);
            else ldsm_x2_trans(w, src);
#pragma unroll
            for (int q = 2; q >= 0; --q) {
                mma_bf16(yacc[j], hfr[q], w[0], w[1]);
                if (j + 1 < NT2) mma_bf16(yacc[j + 1], hfr[q], w[2], w[3]);
            }
        }
    }
    // yacc[j]: [0] (p0, head 8 j + 2t), [1] (p0, + 1), [2] (p1, 2t), [3] (p1, + 1)
    if constexpr (HS == 1) {
        // whether a position's page is there is known to the lanes that hold its block: lanes 4 strip .. 4 strip + 3
        const bool there = __shfl_sync(0xffffffffu, id, 4 * strip) >= 0;
        if (!there) return;
#pragma unroll
        for (int j = 0; j < NT2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = j * 8 + 2 * t + (e & 1), pos = e & 2 ? p1 : p0;
                if (e & 2 ? ok1 : ok0) put_score(p, b, h, j0 + pos, yacc[j][e] + (CONCAT ? 0.f : s_s[h * LD + pos]));
            }
    } else {
#pragma unroll
        for (int j = 0; j < NT2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) y_s[(hs * HQ + j * 8 + 2 * t + (e & 1)) * LD + (e & 2 ? p1 : p0)] = yacc[j][e];
        __syncthreads();
        // pages of the chunk's blocks: lane 4 i holds block i's
        const uint32_t there = __ballot_sync(0xffffffffu, id >= 0);
        for (int e = tid; e < HQ * CH; e += kScoresThreads) {
            const int h = e / CH, pos = e % CH;
            if (j0 + pos >= L || !(there >> (pos / kPageBlock * 4) & 1)) continue;
            float x = CONCAT ? 0.f : s_s[h * LD + pos];
#pragma unroll
            for (int q = 0; q < HS; ++q) x += y_s[(q * HQ + h) * LD + pos];
            put_score(p, b, h, j0 + pos, x);
        }
    }
}

template <int HQ, bool CONCAT>
cudaError_t launch_fast(const ScoresParams& p, int dtype, cudaStream_t s) {
    // 128 positions to a CTA once that gives every SM one, else fewer
    int ch = 128;
    while (ch > 16 && (int64_t)p.B * ((p.L + ch - 1) / ch) < sm_count()) ch /= 2;
    auto kernel = ch == 128 ? paged_scores_kernel<HQ, 128, CONCAT> : ch == 64 ? paged_scores_kernel<HQ, 64, CONCAT>
                : ch == 32 ? paged_scores_kernel<HQ, 32, CONCAT> : paged_scores_kernel<HQ, 16, CONCAT>;
    const size_t smem = (size_t)scores_layout(HQ, ch, CONCAT, p.m).total;
    const cudaError_t e = allow_smem(kernel, smem);
    return e != cudaSuccess ? e : launch_chained(kernel, dim3((p.L + ch - 1) / ch, p.B), dim3(kScoresThreads), smem, s, p, dtype);
}

bool vec16(const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15u) == 0; }

}  // namespace

cudaError_t launch_paged_scores(const ScoresParams& p, int dtype, cudaStream_t s) {
    const bool fast = (p.Hq == 32 || p.Hq == 40) && p.integrate != LISA_INTEGRATE_PLUS && p.ffn_layers == 2 && p.w_dtype == LISA_BF16 && p.m % 8 == 0 &&
                      vec16(p.w1) && vec16(p.w2);
    cudaError_t e;
    if (fast) {
        const bool concat = p.integrate == LISA_INTEGRATE_CONCAT;
        if (p.Hq == 40) e = concat ? launch_fast<40, true>(p, dtype, s) : launch_fast<40, false>(p, dtype, s);
        else e = concat ? launch_fast<32, true>(p, dtype, s) : launch_fast<32, false>(p, dtype, s);
    } else {
        const size_t smem = general_smem(p);
        auto kernel = dtype == LISA_S8 ? paged_scores_general_kernel<LISA_S8> : paged_scores_general_kernel<LISA_E4M3>;
        if ((e = allow_smem(kernel, smem)) != cudaSuccess) return e;
        e = launch_chained(kernel, dim3((p.L + kGeneralThreads - 1) / kGeneralThreads, p.B), dim3(kGeneralThreads), smem, s, p);
    }
    count_launches(1);
    return e;
}

}  // namespace lisa
