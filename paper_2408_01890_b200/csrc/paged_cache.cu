// Rows into and out of a paged 8-bit cache layer.
//
// A warp owns one block: 16 positions of one head, of K (or K') or of V, i.e. one scale.  It reads the block's new rows with every load
// in flight at once, takes the largest magnitude (as unsigned bits, so that a NaN or an infinity is the largest of all), and writes the codes:
//   s = max(s_held, amax / top);  code = Q(x / s);  codes held from before are Q(code * (s_held / s)) where s has grown
// s_held counts only where the block holds positions in front of the new ones.  No block is touched by two warps, so nothing is atomic and the
// bytes do not depend on the order of threads.  The arithmetic is fp32 with IEEE division: the codes are those of the stated formula.
// Bytes: 2 in and 1 out per value.  8 x 2048 positions of 32 heads, d 128, bf16 (0.40 GB): in 78 us (5.2 TB/s of the bytes; the integer and logic units are at 70 %, the codes'
// arithmetic being what bounds it), out again 64 us (6.3 TB/s, HBM).  A token of each of 64 sequences is 7 us, latency.
#include <algorithm>

#include "decode_common.cuh"
#include "paged_common.cuh"

namespace lisa {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct RowsParams {
    PagedView pool;
    TView k, v;
    const int32_t *first, *counts;
    int B, n, blocks;      // blocks of a sequence that n rows can touch
    int64_t items;         // B * blocks * Hkv * 2
};

// Work item -> (sequence, block, head, K or V); false if the block has no rows of the call.  lo..hi: the block's positions of the call, relative
// to the block's start (base); rel0: row of the call at the block's start (negative where older positions come first).
struct Block {
    int b, h, base, rel0, lo, hi;
    bool is_v;
};
__device__ __forceinline__ bool block_of(const RowsParams& p, int64_t item, Block& x) {
    x.is_v = item & 1;
    uint32_t rest = (uint32_t)(item >> 1);
    x.h = rest % (uint32_t)p.pool.Hkv;
    rest /= (uint32_t)p.pool.Hkv;
    const uint32_t i = rest % (uint32_t)p.blocks;
    x.b = rest / (uint32_t)p.blocks;
    const int first = p.first ? p.first[x.b] : 0, count = p.counts ? max(0, min(p.counts[x.b], p.n)) : p.n;
    if (first < 0 || first > INT32_MAX - p.n - kPageBlock) {   // (a position that no table holds)
        if (count > 0 && i == 0 && x.h == 0 && x.is_v && (threadIdx.x & 31) == 0) atomicAdd(p.pool.status, 1);
        return false;
    }
    x.base = (first & ~(kPageBlock - 1)) + (int)i * kPageBlock;
    x.rel0 = x.base - first;
    x.lo = max(0, -x.rel0);
    x.hi = min(kPageBlock, count - x.rel0);
    return x.lo < x.hi;
}

// The block's page, or nullptr (counted once a block)
__device__ __forceinline__ uint8_t* page_at(const RowsParams& p, const Block& x) {
    const bool count = x.h == 0 && x.is_v && (threadIdx.x & 31) == 0;
    if (x.base >> p.pool.shift >= p.pool.max_pages) {
        if (count) atomicAdd(p.pool.status, 1);
        return nullptr;
    }
    const int id = p.pool.page_of(x.b, x.base, count);
    return id < 0 ? nullptr : p.pool.page(id);
}

template <typename T>
__device__ __forceinline__ float value_of(const uint32_t* raw, int i) {   // value i of a run of raw words
    if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? raw[i >> 1] & 0xffff0000u : raw[i >> 1] << 16);
    else return __uint_as_float(raw[i]);
}

// The block's scale from the largest magnitude of its new values (bits of this lane's) and what it holds
template <int FMT>
__device__ __forceinline__ float new_scale(uint32_t amax, float held) {
    const uint32_t all = __reduce_max_sync(0xffffffffu, amax);
    const float grown = __uint_as_float(all) / code_top<FMT>();
    return all >= 0x7f800000u || !(held == held) ? __uint_as_float(0x7fc00000u) : fmaxf(held, grown);
}

// Four values as codes by the formula: IEEE division, rounding to nearest even
template <int FMT>
__device__ __noinline__ uint32_t encode_exactly(float a, float b, float c, float d, float scale) {
    return to_code<FMT>(a / scale) | to_code<FMT>(b / scale) << 8 | to_code<FMT>(c / scale) << 16 | to_code<FMT>(d / scale) << 24;
}

// The same without the division where the reciprocal leaves no doubt: the rounded quotient lies between x lo and x hi, 2^-22 to either side of
// x / scale, so if both round to the same code that is the code (else, once in some ten thousand values, the division decides).  s8: x lo + 1.5 2^23
// in one fused multiply-add has the code in its low bits.  With a division for each value 8 x 2048 prompt rows of the 7B shape took 170 us.
template <int FMT>
struct Encoder {
    float scale, lo, hi;
    bool some, exact;
    __device__ __forceinline__ explicit Encoder(float s) : scale(s) {
        const float inv = __frcp_rn(s);
        lo = inv * (1.f - 0x1p-22f);
        hi = inv * (1.f + 0x1p-22f);
        some = s > 0.f;                                   // (false for NaN: codes 0 then)
        exact = !(s > 0x1p-100f && s < 0x1p100f);         // (a reciprocal out of range, a scale that is not exact to 2^-24)
    }
    __device__ __forceinline__ uint32_t operator()(float a, float b, float c, float d) const {
        uint32_t word, doubt;
        if constexpr (FMT == LISA_S8) {
            constexpr float kMagic = 12582912.f;
            const uint32_t a0 = __float_as_uint(fmaf(a, lo, kMagic)), b0 = __float_as_uint(fmaf(b, lo, kMagic)), c0 = __float_as_uint(fmaf(c, lo, kMagic)),
                           d0 = __float_as_uint(fmaf(d, lo, kMagic));
            doubt = (a0 ^ __float_as_uint(fmaf(a, hi, kMagic))) | (b0 ^ __float_as_uint(fmaf(b, hi, kMagic))) | (c0 ^ __float_as_uint(fmaf(c, hi, kMagic))) |
                    (d0 ^ __float_as_uint(fmaf(d, hi, kMagic)));
            word = __byte_perm(__byte_perm(a0, b0, 0x0040), __byte_perm(c0, d0, 0x0040), 0x5410);
        } else {
            auto pair = [](float x, float y) {            // (the second operand is the low byte)
                uint16_t v;
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(y), "f"(x));
                return (uint32_t)v;
            };
            word = pair(a * lo, b * lo) | pair(c * lo, d * lo) << 16;
            doubt = word ^ (pair(a * hi, b * hi) | pair(c * hi, d * hi) << 16);
        }
        if (doubt || exact) word = encode_exactly<FMT>(a, b, c, d, scale);
        return some ? word : 0u;
    }
};

// What a block holds, rescaled where its scale has grown
template <int FMT>
__device__ __forceinline__ uint32_t rescaled(uint32_t old, float f, bool some) {
    uint32_t out = 0;
    if (some)
#pragma unroll
        for (int t = 0; t < 4; ++t) out |= to_code<FMT>(__fmul_rn(code_value<FMT>(old, t), f)) << (8 * t);
    return out;
}

// D-wide rows (V, and K of a standard layer): 16 bytes per lane and load, all of the block's rows in flight
template <typename T, int D, int FMT>
__device__ __forceinline__ void append_rows_block(const RowsParams& p, const TView& src, const Block& x, uint8_t* page) {
    constexpr int VE = 16 / sizeof(T), LR = D / VE, RPI = 32 / LR, NI = kPageBlock / RPI;
    const int lane = threadIdx.x & 31, col = (lane % LR) * VE, r0 = lane / LR;
    const char* sp = reinterpret_cast<const char*>(src.ptr) + (x.b * src.sb + ((int64_t)x.rel0 + r0) * src.sn + x.h * src.sh + col) * (int64_t)sizeof(T);
    const int64_t step = src.sn * (int64_t)(RPI * sizeof(T));
    uint32_t raw[NI][4];
#pragma unroll
    for (int i = 0; i < NI; ++i, sp += step) {
        const int row = i * RPI + r0;
        const uint4 q = ld_stream16_or_zero(sp, row >= x.lo && row < x.hi);
        raw[i][0] = q.x; raw[i][1] = q.y; raw[i][2] = q.z; raw[i][3] = q.w;
    }
    float* scale_at = p.pool.scales(page, x.h, x.base) + x.is_v;
    const float held = x.lo > 0 ? *scale_at : 0.f;
    uint32_t amax = 0;
    // the larger magnitude of two, NaN if one is NaN, in one instruction (whose sign says nothing): bf16 two at a time
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(amax) : "r"(raw[i][e]));
            else asm("max.NaN.xorsign.abs.f32 %0, %0, %1;" : "+r"(amax) : "r"(raw[i][e]));
        }
    amax = sizeof(T) == 2 ? max(amax << 16 & 0x7fff0000u, amax & 0x7fff0000u) : amax & 0x7fffffffu;
    const float scale = new_scale<FMT>(amax, held);
    const Encoder<FMT> encode(scale);
    uint8_t* dst = page + (x.is_v ? p.pool.v_off : 0u) + p.pool.row(x.h, x.base) + col;
    if (x.lo > 0 && !(scale == held)) {
        const float f = held / scale;
        for (int e = lane * 4; e < x.lo * D; e += 128) {
            uint32_t* w = reinterpret_cast<uint32_t*>(dst - col + e);
            *w = rescaled<FMT>(*w, f, encode.some);
        }
    }
    if (lane == 0) *scale_at = scale;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int row = i * RPI + r0;
        uint32_t out[VE / 4];
#pragma unroll
        for (int w = 0; w < VE / 4; ++w)
            out[w] = encode(value_of<T>(raw[i], 4 * w), value_of<T>(raw[i], 4 * w + 1), value_of<T>(raw[i], 4 * w + 2), value_of<T>(raw[i], 4 * w + 3));
        if (row < x.lo || row >= x.hi) continue;
        if constexpr (VE == 8) *reinterpret_cast<uint2*>(dst + row * D) = make_uint2(out[0], out[1]);
        else *reinterpret_cast<uint32_t*>(dst + row * D) = out[0];
    }
}

// K' (r <= 32 values a row, any alignment): a lane is a rank, its 16 positions are 16 bytes of the block
template <typename T, int FMT>
__device__ __forceinline__ void append_kp_block(const RowsParams& p, const Block& x, uint8_t* page) {
    const int lane = threadIdx.x & 31;
    const bool on = lane < p.pool.r;
    const T* sp = reinterpret_cast<const T*>(p.k.ptr) + x.b * p.k.sb + (int64_t)x.rel0 * p.k.sn + x.h * p.k.sh + lane;
    float v[kPageBlock];
#pragma unroll
    for (int i = 0; i < kPageBlock; ++i, sp += p.k.sn) v[i] = on && i >= x.lo && i < x.hi ? (float)*sp : 0.f;
    uint4* dst = reinterpret_cast<uint4*>(page + p.pool.kp_block(x.h, x.base)) + lane;
    float* scale_at = p.pool.scales(page, x.h, x.base);
    const float held = x.lo > 0 ? *scale_at : 0.f;
    const bool partial = x.lo > 0 || x.hi < kPageBlock;
    uint32_t old[4] = {0u, 0u, 0u, 0u};
    if (on && partial) {
        const uint4 q = *dst;
        old[0] = q.x; old[1] = q.y; old[2] = q.z; old[3] = q.w;
    }
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kPageBlock; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
    const float scale = new_scale<FMT>(amax, held);
    const Encoder<FMT> encode(scale);
    const bool keep = x.lo == 0 || scale == held;
    const float f = held / scale;
    if (lane == 0) *scale_at = scale;
    uint32_t out[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        out[w] = encode(v[4 * w], v[4 * w + 1], v[4 * w + 2], v[4 * w + 3]);
        if (partial) {
            // bytes of positions before lo (what is held), lo .. hi - 1 (new), and from hi on (as they are)
            const int lo = min(max(x.lo - 4 * w, 0), 4), hi = min(max(x.hi - 4 * w, 0), 4);
            const uint32_t below = lo == 4 ? ~0u : (1u << (8 * lo)) - 1u, above = hi == 4 ? 0u : ~0u << (8 * hi);
            const uint32_t held_w = keep || lo == 0 ? old[w] : rescaled<FMT>(old[w], f, encode.some);
            out[w] = (out[w] & ~(below | above)) | (held_w & below) | (old[w] & above);
        }
    }
    if (on) *dst = make_uint4(out[0], out[1], out[2], out[3]);
}

// Four CTAs an SM (two where a block of fp32 rows is in flight): a block is a chain of loads (lengths, table, rows), which other warps have to hide.
template <typename T, int D, int FMT, bool SHARED>
__global__ void __launch_bounds__(kThreads, sizeof(T) * D > 256 ? 2 : 4) paged_append_kernel(const __grid_constant__ RowsParams p) {
    chain_release();
    chain_wait();
    for (int64_t item = blockIdx.x * (int64_t)kWarps + (threadIdx.x >> 5); item < p.items; item += (int64_t)gridDim.x * kWarps) {
        Block x;
        if (!block_of(p, item, x)) continue;
        uint8_t* page = page_at(p, x);
        if (!page) continue;
        if (SHARED && !x.is_v) append_kp_block<T, FMT>(p, x, page);
        else append_rows_block<T, D, FMT>(p, x.is_v ? p.v : p.k, x, page);
    }
}

template <typename T>
__device__ __forceinline__ T from_f32(float v) {
    if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(v);
    else return v;
}

template <typename T, int D, int FMT, bool SHARED>
__global__ void __launch_bounds__(kThreads) paged_read_kernel(const __grid_constant__ RowsParams p) {
    constexpr int VE = 16 / sizeof(T), LR = D / VE, RPI = 32 / LR, NI = kPageBlock / RPI;
    const int lane = threadIdx.x & 31;
    chain_release();
    chain_wait();
    for (int64_t item = blockIdx.x * (int64_t)kWarps + (threadIdx.x >> 5); item < p.items; item += (int64_t)gridDim.x * kWarps) {
        Block x;
        if (!block_of(p, item, x)) continue;
        uint8_t* page = page_at(p, x);
        if (!page) continue;
        const float scale = p.pool.scales(page, x.h, x.base)[x.is_v];
        const TView& dst = x.is_v ? p.v : p.k;
        T* out = reinterpret_cast<T*>(const_cast<void*>(dst.ptr)) + x.b * dst.sb + (int64_t)x.rel0 * dst.sn + x.h * dst.sh;
        if (SHARED && !x.is_v) {
            if (lane >= p.pool.r) continue;
            const uint4 q = reinterpret_cast<const uint4*>(page + p.pool.kp_block(x.h, x.base))[lane];
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < kPageBlock; ++i)
                if (i >= x.lo && i < x.hi) out[i * dst.sn + lane] = from_f32<T>(code_value<FMT>(w[i >> 2], i & 3) * scale);
            continue;
        }
        const int col = (lane % LR) * VE, r0 = lane / LR;
        const uint8_t* sp = page + (x.is_v ? p.pool.v_off : 0u) + p.pool.row(x.h, x.base) + col;
        uint32_t w[NI][VE / 4];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const uint8_t* q = sp + (i * RPI + r0) * D;
            if constexpr (VE == 8) {
                const uint2 u = *reinterpret_cast<const uint2*>(q);
                w[i][0] = u.x; w[i][1] = u.y;
            } else {
                w[i][0] = *reinterpret_cast<const uint32_t*>(q);
            }
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int row = i * RPI + r0;
            if (row < x.lo || row >= x.hi) continue;
            __align__(16) T v[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] = from_f32<T>(code_value<FMT>(w[i][e >> 2], e & 3) * scale);
            *reinterpret_cast<uint4*>(out + row * dst.sn + col) = *reinterpret_cast<const uint4*>(v);
        }
    }
}

template <bool READ, typename T, int D, int FMT>
cudaError_t launch_rows(const RowsParams& p, bool shared, cudaStream_t s) {
    void (*kernel)(RowsParams);
    if constexpr (READ) kernel = shared ? paged_read_kernel<T, D, FMT, true> : paged_read_kernel<T, D, FMT, false>;
    else kernel = shared ? paged_append_kernel<T, D, FMT, true> : paged_append_kernel<T, D, FMT, false>;
    const int64_t ctas = std::min<int64_t>((p.items + kWarps - 1) / kWarps, (int64_t)sm_count() * 32);
    const cudaError_t e = launch_chained(kernel, dim3((unsigned)ctas), dim3(kThreads), 0, s, p);
    count_launches(1);
    return e;
}

template <bool READ, typename T>
cudaError_t launch_typed(const RowsParams& p, const lisa_paged_layer& c, cudaStream_t s) {
    const bool shared = c.kind == LISA_CACHE_SHARED;
    if (c.dtype == LISA_S8) {
        if (c.d == 128) return launch_rows<READ, T, 128, LISA_S8>(p, shared, s);
        if (c.d == 64) return launch_rows<READ, T, 64, LISA_S8>(p, shared, s);
        return launch_rows<READ, T, 32, LISA_S8>(p, shared, s);
    }
    if (c.d == 128) return launch_rows<READ, T, 128, LISA_E4M3>(p, shared, s);
    if (c.d == 64) return launch_rows<READ, T, 64, LISA_E4M3>(p, shared, s);
    return launch_rows<READ, T, 32, LISA_E4M3>(p, shared, s);
}

template <bool READ>
cudaError_t launch(const lisa_paged_rows_args& a, cudaStream_t s) {
    RowsParams p{};
    p.pool = paged_view(*a.layer, a.table);
    if (!p.pool.status) return cudaErrorUnknown;
    p.k = make_view(a.k_or_kp); p.v = make_view(a.v);
    p.first = a.first; p.counts = a.counts;
    p.B = a.B; p.n = a.n;
    p.blocks = a.first ? (a.n + 2 * kPageBlock - 2) / kPageBlock : (a.n + kPageBlock - 1) / kPageBlock;
    p.items = (int64_t)a.B * p.blocks * a.layer->Hkv * 2;
    if (p.items >> 32) return cudaErrorInvalidValue;     // (item indexes are divided in 32 bits; 2^31 blocks are 34 billion rows)
    return a.v.dtype == LISA_BF16 ? launch_typed<READ, __nv_bfloat16>(p, *a.layer, s) : launch_typed<READ, float>(p, *a.layer, s);
}

}  // namespace

cudaError_t launch_paged_append(const lisa_paged_rows_args& a, cudaStream_t s) { return launch<false>(a, s); }
cudaError_t launch_paged_read(const lisa_paged_rows_args& a, cudaStream_t s) { return launch<true>(a, s); }

}  // namespace lisa
