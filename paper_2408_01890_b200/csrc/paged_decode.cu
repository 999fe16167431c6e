// Decode step over a paged 8-bit cache: a standard layer (Eq. 1-2, last row) and a shared one (Sec. 5.2, decoding stage).
//
// o_h = softmax_j(a_hj) V_j with a_hj = q_h.K_j / sqrt(d), or, for a shared layer, scores that paged_scores.cu has left in a row.  One pass with a
// running maximum and sum: a warp streams its tiles of 16 positions (a tile never leaves a page) and keeps everything in registers; warps,
// and where a sequence is split CTAs, are joined at the end.
//
// Both products over codes run on mma.sync m16n8k16 with the codes as the A operand, as fp16, which holds them exactly; scales are applied to the
// fp32 results.  The other operand is q or the probabilities, brought to [2^13, 2^15) by a power of two and split into two fp16 terms (22 bits)
// that take two neighbouring columns of B, so that the eight columns are four query heads: with few heads to a KV head the columns
// are there anyway.  The sum of the two columns is what an fp32 product would give, up to 2^-22 of the largest term.
// The A operands come straight from global memory, without shared memory: the order of d in q.K, of d in the rows of the output, and of
// positions in P.V is free, so every lane's share of a fragment is 16 consecutive bytes of a row.
// Bound by HBM: a position and head are d bytes of K and d of V.
#include <algorithm>
#include <climits>

#include "paged_decode.cuh"

namespace lisa {
namespace {

struct AttendParams {
    PagedView pool;
    TView q, o;
    const int32_t* seq_lens;
    int B, Hq, G, L;
    int heads, passes;             // query heads of a KV head that one CTA takes, and CTAs that it takes for all of them
    int splits, tiles;             // CTAs a sequence's tiles are divided over, tiles of each
    void* out_scores;              // standard layer
    int64_t sc_sb, sc_sh;
    int row_bf16;
    const float* given;            // shared layer: its scores
    int64_t g_sb, g_sh;
    float *ws_m, *ws_l, *ws_o;     // [B][splits][Hq]( [d])
};

// W consecutive words
template <int W>
__device__ __forceinline__ void ld_words(uint32_t* w, const uint8_t* p) {
    if constexpr (W == 4) {
        const uint4 v = ld_stream16(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (W == 2) {
        asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    } else {
        asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    }
}

// ---------------------------------------------------------------------------------------------
// Attention of up to 4 NT query heads of one KV head.  Lane = (g, t) = (lane / 4, lane % 4) throughout.
// ---------------------------------------------------------------------------------------------
constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = kAttendWarps * 32;
constexpr int kUnit = 2;                                  // tiles that a warp takes at a time: its maximum is reduced once a unit
constexpr int kBatch = 32 / kUnit;                        // units whose pages and scales the lanes hold

template <int FMT, int D, int NT, bool GIVEN>
__global__ void __launch_bounds__(kAttendThreads) paged_attend_kernel(const __grid_constant__ AttendParams p) {
    constexpr int KW = D / 16, VW = D / 32, MT = D / 16;  // words of a lane per K row and per V row; tiles of 16 output columns
    constexpr int H = 4 * NT;
    __shared__ float s_m[kAttendWarps][H], s_l[kAttendWarps][H];
    __shared__ __align__(16) float s_o[kAttendWarps][H][D];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int b = blockIdx.z, split = blockIdx.x, kvh = blockIdx.y / p.passes, pass = blockIdx.y % p.passes;
    const int h0 = kvh * p.G + pass * p.heads, nh = min(p.heads, p.G - pass * p.heads);
    const PagedView& pool = p.pool;
    chain_release();
    chain_wait();
    const int L = length_of(p.seq_lens, b, p.L), all_tiles = (L + kPageBlock - 1) / kPageBlock;
    const int first = split * p.tiles, end = min(first + p.tiles, all_tiles), parts = (all_tiles + p.tiles - 1) / p.tiles;
    void* out = const_cast<void*>(p.o.ptr);
    if (first >= end) {
        if (L == 0 && split == 0)
            for (int e = tid; e < nh * D; e += kAttendThreads) st_elem(out, b * p.o.sb + (h0 + e / D) * p.o.sh + e % D, p.o.dtype, 0.f);
        return;
    }

    // q as B fragments: column g is head g / 2's leading (even g) or second term
    uint32_t qf[NT][KW][2];
    float q_scale[NT];                                    // of the head whose scores this lane gets: head t
    if constexpr (!GIVEN) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int j = nt * 4 + (g >> 1);
            float x[KW][4], amax = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const int d0 = D == 128 ? (w >> 2) * 64 + 16 * t + 4 * (w & 3) : 4 * KW * t + 4 * w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[w][e] = j < nh ? ld_elem(p.q.ptr, b * p.q.sb + (h0 + j) * p.q.sh + d0 + e, p.q.dtype) : 0.f;
                    amax = fmaxf(amax, fabsf(x[w][e]));
                }
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            const int ex = exponent(amax);
            const float up = pow2(13 - max(ex, -100));
#pragma unroll
            for (int w = 0; w < KW; ++w)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    qf[nt][w][e] = pack16(term_of(x[w][2 * e] * up, g & 1), term_of(x[w][2 * e + 1] * up, g & 1));
            q_scale[nt] = pow2(__shfl_sync(0xffffffffu, ex, 8 * t) - 13) * rsqrtf((float)D);
        }
    }

    const int units = (end - first + kUnit - 1) / kUnit, mine = units > warp ? (units - warp + kAttendWarps - 1) / kAttendWarps : 0;
    auto tile_of = [&](int k) { return first + (warp + kAttendWarps * (k / kUnit)) * kUnit + k % kUnit; };   // this warp's k-th tile
    auto id_of = [&](int k) {
        const int tile = tile_of(k);
        return k < mine * kUnit && tile < end ? pool.page_of(b, tile * kPageBlock, blockIdx.y == 0) : -1;
    };
    // lane i: page and scales of tile i of the batch; the next batch's pages are asked for a batch ahead
    int ids = id_of(lane), ids_next = id_of(32 + lane);
    float ks = 0.f, vs = 0.f;
    auto load_scales = [&](int k) {
        ks = vs = 0.f;
        if (ids >= 0) {
            const float2 v = *reinterpret_cast<const float2*>(pool.scales(pool.page(ids), kvh, tile_of(k) * kPageBlock));
            ks = v.x; vs = v.y;
        }
    };
    load_scales(lane);

    uint32_t kw[kUnit][2][KW], vw[kUnit][4][VW];
    int id[kUnit];                                        // pages of the unit whose rows are being loaded
    const uint32_t k_col = D == 128 ? 16 * t : 4 * KW * t, v_col = 4 * VW * g;
    auto load_k = [&](int i) {                            // K rows g and g + 8 of the unit's tiles, zeros past the end
#pragma unroll
        for (int u = 0; u < kUnit; ++u) {
            const int pos = tile_of(i * kUnit + u) * kPageBlock + g;
            const uint8_t* at = pool.page(max(id[u], 0)) + pool.row(kvh, pos) + k_col;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool ok = id[u] >= 0 && pos + 8 * e < L;
#pragma unroll
                for (int w = 0; w < KW; ++w) kw[u][e][w] = 0u;
                if (ok) {
                    constexpr int W = KW < 4 ? KW : 4;
#pragma unroll
                    for (int c = 0; c < KW / W; ++c) ld_words<W>(&kw[u][e][c * W], at + e * 8 * D + c * 64);
                }
            }
        }
    };
    auto load_v = [&](int i, const int* page_ids) {       // V rows 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
        for (int u = 0; u < kUnit; ++u) {
            const int pos = tile_of(i * kUnit + u) * kPageBlock + 2 * t;
            const uint8_t* at = pool.page(max(page_ids[u], 0)) + pool.v_off + pool.row(kvh, pos) + v_col;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int step = (e & 1) + (e >> 1) * 8;
                const bool ok = page_ids[u] >= 0 && pos + step < L;
#pragma unroll
                for (int w = 0; w < VW; ++w) vw[u][e][w] = 0u;
                if (ok) ld_words<VW>(vw[u][e], at + step * D);
            }
        }
    };

    float m[NT], l[NT], o[NT][MT][4], given[kUnit][NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = -INFINITY;
        l[nt] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][mt][e] = 0.f;
    }
    int r_exp = kLeastExp;                                // V enters as code * 2^13 scale / 2^r_exp

    auto load_given = [&](int i) {
#pragma unroll
        for (int u = 0; u < kUnit; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int pos = tile_of(i * kUnit + u) * kPageBlock + g + 8 * e;
                    given[u][nt][e] = pos < L && nt * 4 + t < nh ? p.given[b * p.g_sb + (h0 + nt * 4 + t) * p.g_sh + pos] : 0.f;
                }
    };

    if (mine > 0) {
#pragma unroll
        for (int u = 0; u < kUnit; ++u) id[u] = __shfl_sync(0xffffffffu, ids, u);
        if constexpr (GIVEN) load_given(0);
        else load_k(0);
        load_v(0, id);
    }
    for (int i = 0; i < mine; ++i) {
        const int at = i % kBatch * kUnit;
        float ks_u[kUnit], vs_u[kUnit], s[kUnit][NT][2];
        bool page_ok[kUnit];
#pragma unroll
        for (int u = 0; u < kUnit; ++u) {
            ks_u[u] = __shfl_sync(0xffffffffu, ks, at + u);
            vs_u[u] = __shfl_sync(0xffffffffu, vs, at + u);
            page_ok[u] = id[u] >= 0;
        }
        // scores
        if constexpr (!GIVEN) {
#pragma unroll
            for (int u = 0; u < kUnit; ++u) {
                float c[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0.f;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const uint32_t x0 = biased<FMT>(kw[u][0][w]), x1 = biased<FMT>(kw[u][1][w]);
                    const uint32_t a0 = pair16<FMT>(x0, false), a1 = pair16<FMT>(x1, false), a2 = pair16<FMT>(x0, true), a3 = pair16<FMT>(x1, true);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(c[nt], a0, a1, a2, a3, qf[nt][w][0], qf[nt][w][1]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float f = ks_u[u] * q_scale[nt];
                    s[u][nt][0] = (c[nt][0] + c[nt][1]) * f;
                    s[u][nt][1] = (c[nt][2] + c[nt][3]) * f;
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < kUnit; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) { s[u][nt][0] = given[u][nt][0]; s[u][nt][1] = given[u][nt][1]; }
        }
        // the next unit's K (or scores) are asked for as soon as the registers are free
        const bool more = i + 1 < mine;
        if (more) {
            if (i % kBatch == kBatch - 1) {
                ids = ids_next;
                load_scales((i + 1) * kUnit + lane);
                ids_next = id_of((i + 1) * kUnit + 32 + lane);
            }
            const int next = (i + 1) % kBatch * kUnit;
#pragma unroll
            for (int u = 0; u < kUnit; ++u) id[u] = __shfl_sync(0xffffffffu, ids, next + u);
            if constexpr (GIVEN) load_given(i + 1);
            else load_k(i + 1);
        }
        // running maximum
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx = m[nt];
#pragma unroll
            for (int u = 0; u < kUnit; ++u)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int pos = tile_of(i * kUnit + u) * kPageBlock + g + 8 * e;
                    const bool on = page_ok[u] && pos < L;
                    if (!GIVEN && p.out_scores && on && nt * 4 + t < nh) {
                        const int64_t to = b * p.sc_sb + (h0 + nt * 4 + t) * p.sc_sh + pos;
                        if (p.row_bf16) st_row<true>(p.out_scores, to, s[u][nt][e]);
                        else st_row<false>(p.out_scores, to, s[u][nt][e]);
                    }
                    if (!on) s[u][nt][e] = -INFINITY;
                    mx = fmaxf(mx, s[u][nt][e]);
                }
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            if (__any_sync(0xffffffffu, mx > m[nt])) {
                const float f = mx == -INFINITY ? 1.f : __expf(m[nt] - mx);
                l[nt] *= f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][mt][e] *= f;
                m[nt] = mx;
            }
        }
        // V's scales enter with the probabilities; their common power of two follows the largest so far
        int ex = r_exp;
#pragma unroll
        for (int u = 0; u < kUnit; ++u) ex = max(ex, exponent(vs_u[u]));
        if (ex > r_exp) {
            const float f = pow2(max(r_exp - ex, -126));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][mt][e] *= f;
            r_exp = ex;
        }
        const float up = pow2(min(13 - r_exp, 127));
#pragma unroll
        for (int u = 0; u < kUnit; ++u) {
            uint32_t bf[NT][2];
            const float f = vs_u[u] * up;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float ref = m[nt] == -INFINITY ? 0.f : m[nt];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float pj = __expf(s[u][nt][e] - ref);
                    l[nt] += pj;
                    bf[nt][e] = transpose8x8(two_terms(pj * f));
                }
            }
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                // pairs of positions for four columns of the output: rows g and g + 8 of two tiles
                const uint32_t y0 = biased<FMT>(vw[u][0][w]), y1 = biased<FMT>(vw[u][1][w]), y2 = biased<FMT>(vw[u][2][w]), y3 = biased<FMT>(vw[u][3][w]);
                const uint32_t lo01 = __byte_perm(y0, y1, 0x5140), hi01 = __byte_perm(y0, y1, 0x7362);
                const uint32_t lo23 = __byte_perm(y2, y3, 0x5140), hi23 = __byte_perm(y2, y3, 0x7362);
                const uint32_t a[2][4] = {{pair16<FMT>(lo01, false), pair16<FMT>(lo01, true), pair16<FMT>(lo23, false), pair16<FMT>(lo23, true)},
                                          {pair16<FMT>(hi01, false), pair16<FMT>(hi01, true), pair16<FMT>(hi23, false), pair16<FMT>(hi23, true)}};
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][2 * w + x], a[x][0], a[x][1], a[x][2], a[x][3], bf[nt][0], bf[nt][1]);
            }
        }
        if (more) load_v(i + 1, id);
    }

    // warps joined
    const float down = pow2(max(r_exp - 13, -126));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l[nt] += __shfl_xor_sync(0xffffffffu, l[nt], off);
        const int j = nt * 4 + t;
        if (g == 0) { s_m[warp][j] = m[nt]; s_l[warp][j] = l[nt]; }
#pragma unroll
        for (int w = 0; w < VW; ++w)
            *reinterpret_cast<float4*>(&s_o[warp][j][v_col + 4 * w]) =
                make_float4((o[nt][2 * w][0] + o[nt][2 * w][1]) * down, (o[nt][2 * w][2] + o[nt][2 * w][3]) * down,
                            (o[nt][2 * w + 1][0] + o[nt][2 * w + 1][1]) * down, (o[nt][2 * w + 1][2] + o[nt][2 * w + 1][3]) * down);
    }
    __syncthreads();
    for (int e = tid; e < nh * (D / 4); e += kAttendThreads) {
        const int j = e / (D / 4), x = e % (D / 4) * 4;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < kAttendWarps; ++w) mx = fmaxf(mx, s_m[w][j]);
        const float ref = mx == -INFINITY ? 0.f : mx;
        float den = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kAttendWarps; ++w) {
            const float f = __expf(s_m[w][j] - ref);
            const float4 v = *reinterpret_cast<const float4*>(&s_o[w][j][x]);
            den = fmaf(f, s_l[w][j], den);
            acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
        }
        if (parts == 1) {
            const float inv = den == 0.f ? 0.f : 1.f / den;      // (0: every position lies on a page that the table does not name)
            const int64_t to = b * p.o.sb + (h0 + j) * p.o.sh + x;
            st_elem(out, to, p.o.dtype, acc.x * inv); st_elem(out, to + 1, p.o.dtype, acc.y * inv);
            st_elem(out, to + 2, p.o.dtype, acc.z * inv); st_elem(out, to + 3, p.o.dtype, acc.w * inv);
        } else {
            const size_t part = ((size_t)b * p.splits + split) * p.Hq + h0 + j;
            if (x == 0) { p.ws_m[part] = mx; p.ws_l[part] = den; }
            *reinterpret_cast<float4*>(p.ws_o + part * D + x) = acc;
        }
    }
}

// Joins the parts of a sequence that was split: o = sum_c e^(m_c - M) o_c / sum_c e^(m_c - M) l_c.
__global__ void __launch_bounds__(128) paged_merge_kernel(const __grid_constant__ AttendParams p) {
    const int h = blockIdx.x, b = blockIdx.y, d = p.pool.d;
    chain_release();
    chain_wait();
    const int parts = ((length_of(p.seq_lens, b, p.L) + kPageBlock - 1) / kPageBlock + p.tiles - 1) / p.tiles;
    if (parts <= 1 || threadIdx.x >= d) return;
    const size_t base = (size_t)b * p.splits * p.Hq + h;
    float mx = -INFINITY;
    for (int c = 0; c < parts; ++c) mx = fmaxf(mx, p.ws_m[base + (size_t)c * p.Hq]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float den = 0.f, acc = 0.f;
#pragma unroll 4
    for (int c = 0; c < parts; ++c) {
        const size_t part = base + (size_t)c * p.Hq;
        const float f = __expf(p.ws_m[part] - ref);
        den = fmaf(f, p.ws_l[part], den);
        acc = fmaf(f, p.ws_o[part * d + threadIdx.x], acc);
    }
    st_elem(const_cast<void*>(p.o.ptr), b * p.o.sb + h * p.o.sh + threadIdx.x, p.o.dtype, den == 0.f ? 0.f : acc / den);
}

// ------------------------------------------------------------------ launches
constexpr int kMinTiles = kUnit * kAttendWarps;           // of a CTA: less would leave warps without work
constexpr int kSlots = 4;                                 // CTAs an SM is given at least, as long as there are tiles

int column_tiles(int G) { return G > 4 ? 2 : 1; }

int splits_for(int64_t ctas, int tiles) {
    const int64_t want = (int64_t)sm_count() * kSlots;
    if (ctas >= want) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>((want + ctas - 1) / ctas, (tiles + kMinTiles - 1) / kMinTiles));
}

int head_passes(int G) { return (G + 4 * column_tiles(G) - 1) / (4 * column_tiles(G)); }

// Parts that a step may produce, times heads: with B * Hkv * passes CTAs below `want`, fewer than twice as many after splitting.
size_t part_bytes(int B, int Hq, int Hkv, int d, int L) {
    const int G = Hq / Hkv;
    const int64_t tiles = (L + kPageBlock - 1) / kPageBlock;
    const int64_t most = 2 * (int64_t)sm_count() * kSlots * 4 * column_tiles(G), all = (int64_t)B * Hq * ((tiles + kMinTiles - 1) / kMinTiles);
    const size_t n = ((size_t)std::min(most, all) + 3) & ~(size_t)3;
    return (n * (2 + (size_t)d) * sizeof(float) + 255) & ~(size_t)255;
}

template <int FMT, bool GIVEN>
cudaError_t launch_attend(AttendParams& p, void* ws, cudaStream_t s) {
    const int nt = column_tiles(p.G), all_tiles = (p.L + kPageBlock - 1) / kPageBlock;
    p.heads = 4 * nt;
    p.passes = head_passes(p.G);
    const int64_t ctas = (int64_t)p.B * p.pool.Hkv * p.passes;
    const int splits = splits_for(ctas, all_tiles);
    p.tiles = ((all_tiles + splits - 1) / splits + kMinTiles - 1) / kMinTiles * kMinTiles;
    p.splits = (all_tiles + p.tiles - 1) / p.tiles;
    const size_t n = ((size_t)p.B * p.splits * p.Hq + 3) & ~(size_t)3;
    p.ws_m = static_cast<float*>(ws);
    p.ws_l = p.ws_m + n;
    p.ws_o = p.ws_l + n;
    void (*kernel)(AttendParams) = nullptr;
    switch (p.pool.d) {
        case 128: kernel = nt == 2 ? paged_attend_kernel<FMT, 128, 2, GIVEN> : paged_attend_kernel<FMT, 128, 1, GIVEN>; break;
        case 64: kernel = nt == 2 ? paged_attend_kernel<FMT, 64, 2, GIVEN> : paged_attend_kernel<FMT, 64, 1, GIVEN>; break;
        default: kernel = nt == 2 ? paged_attend_kernel<FMT, 32, 2, GIVEN> : paged_attend_kernel<FMT, 32, 1, GIVEN>; break;
    }
    cudaError_t e = launch_chained(kernel, dim3(p.splits, p.pool.Hkv * p.passes, p.B), dim3(kAttendThreads), 0, s, p);
    count_launches(1);
    if (e != cudaSuccess || p.splits == 1) return e;
    e = launch_chained(paged_merge_kernel, dim3(p.Hq, p.B), dim3(128), 0, s, p);
    count_launches(1);
    return e;
}

}  // namespace

size_t paged_anchor_workspace(int B, int Hq, int Hkv, int d, int L) { return part_bytes(B, Hq, Hkv, d, L); }

// A shared layer's scores lie in front of the parts, fp32.
static int64_t score_row(int L) { return (L + 7) / 8 * 8; }
static size_t score_bytes(int B, int Hq, int L) { return ((size_t)B * Hq * score_row(L) * sizeof(float) + 255) & ~(size_t)255; }
size_t paged_shared_workspace(int B, int Hq, int Hkv, int d, int L) { return score_bytes(B, Hq, L) + part_bytes(B, Hq, Hkv, d, L); }

cudaError_t launch_paged_anchor(const lisa_paged_anchor_args& a, cudaStream_t s) {
    AttendParams p{};
    p.pool = paged_view(*a.cache, a.table);
    if (!p.pool.status) return cudaErrorUnknown;
    p.q = make_view(a.q); p.o = make_view(a.o);
    p.seq_lens = a.seq_lens;
    p.B = a.B; p.Hq = a.Hq; p.G = a.Hq / a.cache->Hkv; p.L = a.L;
    p.out_scores = a.out_scores; p.sc_sb = a.scores_stride_b; p.sc_sh = a.scores_stride_h;
    p.row_bf16 = a.scores_dtype == LISA_BF16;
    return a.cache->dtype == LISA_S8 ? launch_attend<LISA_S8, false>(p, a.workspace, s) : launch_attend<LISA_E4M3, false>(p, a.workspace, s);
}

cudaError_t launch_paged_shared(const lisa_paged_shared_args& a, cudaStream_t s) {
    ScoresParams c{};
    c.pool = paged_view(*a.cache, a.table);
    if (!c.pool.status) return cudaErrorUnknown;
    c.qp = make_view(a.link.qp);
    c.seq_lens = a.seq_lens;
    c.B = a.B; c.Hq = a.Hq; c.G = a.Hq / a.cache->Hkv; c.L = a.L;
    c.prev = a.prev_scores; c.prev_sb = a.prev_stride_b; c.prev_sh = a.prev_stride_h;
    c.w1 = a.link.w1; c.b1 = a.link.b1; c.w2 = a.link.w2; c.b2 = a.link.b2;
    c.m = a.link.m; c.act = a.link.act; c.integrate = a.link.integrate; c.ffn_layers = a.link.ffn_layers; c.w_dtype = a.link.w_dtype;
    c.row_bf16 = a.scores_dtype == LISA_BF16;
    if (a.out_scores && !c.row_bf16) {      // the row for the next layer is where attention reads them
        c.scores = static_cast<float*>(a.out_scores);
        c.s_sb = a.scores_stride_b; c.s_sh = a.scores_stride_h;
    } else {
        c.scores = static_cast<float*>(a.workspace);
        c.s_sh = score_row(a.L); c.s_sb = c.s_sh * a.Hq;
        c.out_scores = a.out_scores; c.sc_sb = a.scores_stride_b; c.sc_sh = a.scores_stride_h;
    }
    const bool s8 = a.cache->dtype == LISA_S8;
    const cudaError_t e = launch_paged_scores(c, a.cache->dtype, s);
    if (e != cudaSuccess) return e;
    AttendParams p{};
    p.pool = c.pool;
    p.o = make_view(a.o);
    p.seq_lens = a.seq_lens;
    p.B = a.B; p.Hq = a.Hq; p.G = c.G; p.L = a.L;
    p.given = c.scores; p.g_sb = c.s_sb; p.g_sh = c.s_sh;
    void* parts = static_cast<char*>(a.workspace) + score_bytes(a.B, a.Hq, a.L);
    return s8 ? launch_attend<LISA_S8, true>(p, parts, s) : launch_attend<LISA_E4M3, true>(p, parts, s);
}

}  // namespace lisa
