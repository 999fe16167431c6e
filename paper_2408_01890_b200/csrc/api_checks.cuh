// Checks of arguments that the C-ABI entry points share (host code, before anything is launched).
#pragma once
#include "common.cuh"

namespace lisa {

// LISA_ERR_CUDA, the code kept for lisa_last_cuda_error()
lisa_status_t cuda_fail(cudaError_t e);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool dtype_ok(int dt) { return dt == LISA_F32 || dt == LISA_BF16; }
inline size_t esize(int dt) { return dt == LISA_BF16 ? 2 : 4; }

inline lisa_status_t check_tensor(const lisa_tensor& t) {
    if (!t.ptr || !dtype_ok(t.dtype) || !aligned16(t.ptr)) return LISA_ERR_INVALID_ARG;
    return LISA_OK;
}

inline lisa_status_t check_dims(int B, int N, int Hq, int Hkv, int d) {
    if (B < 1 || N < 1 || Hq < 1 || Hkv < 1 || d < 1) return LISA_ERR_INVALID_ARG;
    if (Hq % Hkv != 0) return LISA_ERR_INVALID_ARG;
    if (Hq > kMaxHeads) return LISA_ERR_UNSUPPORTED;
    if (d != 32 && d != 64 && d != 128) return LISA_ERR_UNSUPPORTED;
    return LISA_OK;
}

inline lisa_status_t check_link(const lisa_link& l, int Hq, bool prefill) {
    if (l.r < 1) return LISA_ERR_INVALID_ARG;
    if (l.r > kMaxRank) return LISA_ERR_UNSUPPORTED;
    if (l.integrate < LISA_INTEGRATE_ADD || l.integrate > LISA_INTEGRATE_PLUS) return LISA_ERR_INVALID_ARG;
    lisa_status_t st = check_tensor(l.qp);
    if (st != LISA_OK) return st;
    if (prefill && (st = check_tensor(l.kp)) != LISA_OK) return st;
    if (l.integrate == LISA_INTEGRATE_PLUS) return LISA_OK;
    if (l.act < LISA_ACT_NONE || l.act > LISA_ACT_SILU) return LISA_ERR_INVALID_ARG;
    if (l.ffn_layers != 1 && l.ffn_layers != 2) return LISA_ERR_INVALID_ARG;
    if (!dtype_ok(l.w_dtype) || !l.w1 || l.m < 1) return LISA_ERR_INVALID_ARG;
    if (l.m > kMaxHidden) return LISA_ERR_UNSUPPORTED;
    if (l.ffn_layers == 2 && !l.w2) return LISA_ERR_INVALID_ARG;
    if (l.ffn_layers == 1 && l.m != Hq) return LISA_ERR_INVALID_ARG;
    return LISA_OK;
}

inline lisa_status_t check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return LISA_OK;
    if (!ws || have < need || !aligned16(ws)) return LISA_ERR_WORKSPACE;
    return LISA_OK;
}

}  // namespace lisa
