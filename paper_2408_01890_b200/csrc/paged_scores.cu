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
constexpr int kRingHeads = 3;            // KV heads' K' of a warp on their way or in use

// Shared memory of a CTA (byte offsets): differences [HQ][CH + 4], partial FFN outputs [HS][HQ][CH + 4] (HS > 1), the two terms of q' [HQ][2][32] and its
// scales, weights, biases, and the warps' rings: a stage is [CH / 16 blocks][24 or 32 ranks][16 positions] and the blocks' scales
struct ScoresLayout {
    int y, qp, q_scale, w1, w2, b1, b2, ring, stage, scales, total;
};
__host__ __device__ inline ScoresLayout scores_layout(int HQ, int NW, int CH, bool concat, int m, int r) {
    ScoresLayout l;
    const int HS = NW * 16 / CH, mp = (m + 15) / 16 * 16, kp = concat ? 2 * HQ : (HQ + 15) / 16 * 16;
    int off = HQ * (CH + 4) * 4;
    l.y = off; off += HS > 1 ? HS * HQ * (CH + 4) * 4 : 0;
    l.qp = off; off += HQ * 2 * kMaxRank * 2;
    l.q_scale = off; off += HQ * 4;
    l.w1 = off; off += kp * (mp + 8) * 2;
    l.w2 = off; off += mp * (HQ + 8) * 2;
    l.b1 = off; off += mp * 4;
    l.b2 = off; off += HQ * 4;
    l.ring = off;
    l.scales = CH / kPageBlock * (r > 24 ? 32 : 24) * 16 + (r > 24 ? 0 : 128);      // (the load of a block of 24 ranks reaches 8 further)
    l.stage = l.scales + (CH / kPageBlock * 8 + 15) / 16 * 16;
    l.total = off + NW * kRingHeads * l.stage;
    return l;
}

// Differences of up to four query heads of one KV head, whose K' lies in a stage: positions 2g and 2g + 1 of a block are rows g and g + 8, ranks are k
template <int FMT, int NB>
__device__ __forceinline__ void delta_blocks(const uint8_t* stage, int scales, bool wide, const __half* q, const float* q_scale, int nh, float* s_s, int ld) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, ranks = wide ? 32 : 24;
    // column g: head g / 2's leading (even g) or second term
    uint32_t bf[4];
    const uint32_t* qr = reinterpret_cast<const uint32_t*>(q + (g >> 1) * 2 * kMaxRank + (g & 1) * kMaxRank) + t;
#pragma unroll
    for (int i = 0; i < 4; ++i) bf[i] = (g >> 1) < nh && (wide || i < 3) ? qr[4 * i] : 0u;
    const float qs = t < nh ? q_scale[t] : 0.f;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        uint32_t w[4];
        ldmatrix_trans(w, stage + (k * ranks + lane) * 16);
        float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = biased<FMT>(w[i]);
        mma_f16(c, across16<FMT>(w[0], false), across16<FMT>(w[0], true), across16<FMT>(w[1], false), across16<FMT>(w[1], true), bf[0], bf[1]);
        if (wide) mma_f16(c, across16<FMT>(w[2], false), across16<FMT>(w[2], true), across16<FMT>(w[3], false), across16<FMT>(w[3], true), bf[2], bf[3]);
        else mma_f16_k8(c, across16<FMT>(w[2], false), across16<FMT>(w[2], true), bf[2]);
        const float f = reinterpret_cast<const float2*>(stage + scales)[k].x * qs;
        if (t < nh) *reinterpret_cast<float2*>(s_s + t * ld + k * kPageBlock + 2 * g) = make_float2((c[0] + c[1]) * f, (c[2] + c[3]) * f);
    }
}

template <int HQ, int NW, int CH, bool CONCAT>
__global__ void __launch_bounds__(NW * 32, NW == 4 ? 4 : 2) paged_scores_kernel(const __grid_constant__ ScoresParams p, int dtype) {
    constexpr int THREADS = NW * 32, HS = NW * 16 / CH, LD = CH + 4, NB = CH / kPageBlock, NT2 = HQ / 8, KPH = (HQ + 15) / 16;
    constexpr int KS1 = CONCAT ? 2 * HQ / 16 : KPH, W2_LD = HQ + 8;
    extern __shared__ __align__(16) uint8_t smem_b[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int b = blockIdx.y, j0 = blockIdx.x * CH, m = p.m, mp = (m + 15) / 16 * 16, w1_ld = mp + 8, r = p.pool.r;
    const ScoresLayout lay = scores_layout(HQ, NW, CH, CONCAT, m, r);
    float* s_s = reinterpret_cast<float*>(smem_b);
    float* y_s = reinterpret_cast<float*>(smem_b + lay.y);
    __half* qp_s = reinterpret_cast<__half*>(smem_b + lay.qp);
    float* q_scale = reinterpret_cast<float*>(smem_b + lay.q_scale);
    __nv_bfloat16* w1_s = reinterpret_cast<__nv_bfloat16*>(smem_b + lay.w1);     // [inputs][mp + 8], zero rows and columns beyond the FFN's sizes
    __nv_bfloat16* w2_s = reinterpret_cast<__nv_bfloat16*>(smem_b + lay.w2);     // [mp][HQ + 8]
    float* b1_s = reinterpret_cast<float*>(smem_b + lay.b1);
    float* b2_s = reinterpret_cast<float*>(smem_b + lay.b2);
    uint8_t* ring = smem_b + lay.ring + warp * kRingHeads * lay.stage;
    chain_release();
    // the aligner's weights are constants of the model: staged while the kernel before this one may still be running
    const int c8 = mp / 8;
    for (int e = tid; e < KS1 * 16 * c8; e += THREADS) {
        const int k = e / c8, c = (e - k * c8) * 8;
        const bool in = k < (CONCAT ? 2 * HQ : HQ) && c < m;
        cp_async<16>((uint32_t)__cvta_generic_to_shared(w1_s + k * w1_ld + c), static_cast<const __nv_bfloat16*>(p.w1) + (in ? k * m + c : 0), in);
    }
    for (int e = tid; e < mp * NT2; e += THREADS) {
        const int k = e / NT2, c = e % NT2 * 8;
        cp_async<16>((uint32_t)__cvta_generic_to_shared(w2_s + k * W2_LD + c), static_cast<const __nv_bfloat16*>(p.w2) + (k < m ? k * HQ + c : 0), k < m);
    }
    cp_commit();
    for (int e = tid; e < mp; e += THREADS) b1_s[e] = e < m ? ldw(p.b1, e, p.w_dtype) : 0.f;
    for (int e = tid; e < HQ; e += THREADS) b2_s[e] = ldw(p.b2, e, p.w_dtype);
    for (int e = lane; e < kRingHeads * lay.stage / 16; e += 32) reinterpret_cast<uint4*>(ring)[e] = make_uint4(0u, 0u, 0u, 0u);   // ranks beyond r stay zero
    __syncwarp();
    chain_wait();
    const int L = length_of(p.seq_lens, b, p.L);
    if (j0 >= L) {
        cp_wait<0>();
        return;
    }

    // lane i: page of the chunk's block i
    const int id = lane < NB && j0 + lane * kPageBlock < L ? p.pool.page_of(b, j0 + lane * kPageBlock, warp == 0) : -1;
    const uint32_t there = __ballot_sync(0xffffffffu, id >= 0);
    const uint8_t* kp_at[NB];             // this lane's rank of KV head 0 in each block
#pragma unroll
    for (int k = 0; k < NB; ++k)
        kp_at[k] = p.pool.page(max(__shfl_sync(0xffffffffu, id, k), 0)) + p.pool.kp_block(0, j0 + k * kPageBlock) + lane * kPageBlock;
    const uint8_t* scale_at = reinterpret_cast<const uint8_t*>(p.pool.scales(p.pool.page(max(id, 0)), 0, j0 + lane * kPageBlock));
    const int blocks = 1 << (p.pool.shift - 4), passes = (p.G + 3) / 4, n_kv = p.pool.Hkv;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    auto ask = [&](int kvh, int stage) {
        if (kvh < n_kv) {
            const uint32_t to = ring_at + stage * lay.stage;
            const int64_t head = (int64_t)kvh * blocks;
#pragma unroll
            for (int k = 0; k < NB; ++k)
                if (lane < r) cp_async<16>(to + (k * (r > 24 ? 32 : 24) + lane) * 16, kp_at[k] + head * (r * kPageBlock), there >> k & 1);
            if (lane < NB) cp_async<8>(to + lay.scales + lane * 8, scale_at + head * 8, id >= 0);
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < kRingHeads - 1; ++i) ask(warp + i * NW, i);

    // the previous scores of the FFN phase: asked for now
    const int strip = warp % NB, hs = warp / NB, p0 = strip * 16 + g, p1 = p0 + 8;
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

    // q', each head brought to [2^13, 2^14) by a power of two, as two fp16 terms
    for (int h = warp; h < HQ; h += NW) {
        float x = lane < r ? ld_elem(p.qp.ptr, b * p.qp.sb + h * p.qp.sh + lane, p.qp.dtype) : 0.f;
        const int ex = exponent(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu)));
        x *= pow2(13 - ex);
        const __half hi = __float2half_rn(x);
        qp_s[h * 2 * kMaxRank + lane] = hi;
        qp_s[h * 2 * kMaxRank + kMaxRank + lane] = __float2half_rn(x - __half2float(hi));
        if (lane == 0) q_scale[h] = pow2(ex - 13) * rsqrtf((float)r);
    }
    __syncthreads();

    // phase 1
    for (int kvh = warp, stage = 0; kvh < n_kv; kvh += NW, stage = stage + 1 == kRingHeads ? 0 : stage + 1) {
        cp_wait<kRingHeads - 2>();
        __syncwarp();
        ask(kvh + (kRingHeads - 1) * NW, stage == 0 ? kRingHeads - 1 : stage - 1);
        for (int pass = 0; pass < passes; ++pass) {
            const int h0 = kvh * p.G + pass * 4, nh = min(4, p.G - pass * 4);
            if (dtype == LISA_S8) delta_blocks<LISA_S8, NB>(ring + stage * lay.stage, lay.scales, r > 24, qp_s + h0 * 2 * kMaxRank, q_scale + h0, nh, s_s + h0 * LD, LD);
            else delta_blocks<LISA_E4M3, NB>(ring + stage * lay.stage, lay.scales, r > 24, qp_s + h0 * 2 * kMaxRank, q_scale + h0, nh, s_s + h0 * LD, LD);
        }
    }
    cp_wait<0>();                         // (the weights; a warp without heads has not waited)
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
        if (!(there >> strip & 1)) return;
        const bool also = p.out_scores;
        float* to = p.scores + b * p.s_sb + 2 * t * p.s_sh + j0;
#pragma unroll
        for (int j = 0; j < NT2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = j * 8 + (e & 1), pos = e & 2 ? p1 : p0;
                const float v = yacc[j][e] + (CONCAT ? 0.f : s_s[(h + 2 * t) * LD + pos]);
                if (!(e & 2 ? ok1 : ok0)) continue;
                if (also) put_score(p, b, h + 2 * t, j0 + pos, v);
                else to[h * p.s_sh + pos] = v;
            }
    } else {
#pragma unroll
        for (int j = 0; j < NT2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) y_s[(hs * HQ + j * 8 + 2 * t + (e & 1)) * LD + (e & 2 ? p1 : p0)] = yacc[j][e];
        __syncthreads();
        for (int e = tid; e < HQ * CH; e += THREADS) {
            const int h = e / CH, pos = e % CH;
            if (j0 + pos >= L || !(there >> (pos / kPageBlock) & 1)) continue;
            float x = CONCAT ? 0.f : s_s[h * LD + pos];
#pragma unroll
            for (int q = 0; q < HS; ++q) x += y_s[(q * HQ + h) * LD + pos];
            put_score(p, b, h, j0 + pos, x);
        }
    }
}

template <int HQ, bool CONCAT>
cudaError_t launch_fast(const ScoresParams& p, int dtype, cudaStream_t s) {
    // Four warps to 64 positions; the concatenating form, whose weights are most of a CTA's shared memory, eight to 128.  Fewer positions where that
    // does not give every SM two CTAs.
    constexpr int NW = CONCAT ? 8 : 4;
    int ch = NW * 16;
    while (ch > 16 && (int64_t)p.B * ((p.L + ch - 1) / ch) < 2 * (int64_t)sm_count()) ch /= 2;
    void (*kernel)(ScoresParams, int) = ch == 64 ? paged_scores_kernel<HQ, NW, 64, CONCAT> : ch == 32 ? paged_scores_kernel<HQ, NW, 32, CONCAT>
                                                                                          : paged_scores_kernel<HQ, NW, 16, CONCAT>;
    if constexpr (CONCAT)
        if (ch == 128) kernel = paged_scores_kernel<HQ, NW, 128, CONCAT>;
    const size_t smem = (size_t)scores_layout(HQ, NW, ch, CONCAT, p.m, p.pool.r).total;
    const cudaError_t e = allow_smem(kernel, smem, true);
    return e != cudaSuccess ? e : launch_chained(kernel, dim3((p.L + ch - 1) / ch, p.B), dim3(NW * 32), smem, s, p, dtype);
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
