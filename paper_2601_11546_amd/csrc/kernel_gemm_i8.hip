// int8 projections: out[t, n] = sum_k a[t, k] w[n, k] * (w_scale[n] * a_scale[t]) of 8-bit integers, summed exactly in 32 bits: the kernels of
// gemm_kernels.h on integers, with a factor for each token beside each feature's in their epilogues.
#define RELSERVE_GEMM_INT8 1
#include "gemm_kernels.h"

namespace relserve {

void gemm_force_plan_i8(int cand, int splits) {
    g_forced_plan.store(cand < 0 ? -1 : (cand | (splits << 8)), std::memory_order_relaxed);
}

// The kernels see rows of K / 2 two-byte units.
static hipError_t set_int8(GemmArgs& p, const float* t_scale, const float* w_scale) {
    if (p.K % 128) return hipErrorInvalidValue;
    p.f8 = 1;
    p.K /= 2;
    p.w_scale = w_scale;
    p.t_scale = t_scale;
    return hipSuccess;
}

hipError_t launch_linear_i8(const void* a, const float* a_scale, const void* w, const float* w_scale, int32_t T, int32_t N, int32_t K,
                            int32_t epilogue, const void* residual, void* out, hipStream_t s, float* accum, bool w_packed) {
    if (T == 0) return hipSuccess;
    if ((int64_t)T * K >= ((int64_t)1 << 31) || (int64_t)N * K >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    GemmArgs p{};
    set_linear(p, a, w, T, N, K, residual, out, accum, w_packed);
    if (hipError_t e = set_int8(p, a_scale, w_scale)) return e;
    return run_linear(p, epilogue, s, nullptr);
}

hipError_t launch_qkv_rope_append_i8(const BatchDev& b, const relserve_layer& L, const void* h, const float* h_scale, const void* w_qkv,
                                     const float* w_scale, void* q_out, void* k_pages, void* v_pages, hipStream_t s, float* accum,
                                     bool w_packed, KvFormat kv) {
    if (b.T == 0) return hipSuccess;
    if ((int64_t)b.T * L.cfg.hidden >= ((int64_t)1 << 31) || (int64_t)L.qkv_dim * L.cfg.hidden >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    GemmArgs p{};
    set_qkv(p, b, L, h, w_qkv, q_out, k_pages, v_pages, kv, accum, w_packed);
    if (hipError_t e = set_int8(p, h_scale, w_scale)) return e;
    return run_qkv(p, L.cfg.head_dim, s);
}

}  // namespace relserve
