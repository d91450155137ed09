// Host boundary of the int8 operators: argument checks, the layer and model steps built on them.
#include "relserve_host.h"

using namespace relserve;

namespace {

constexpr int32_t kMaxRowCodes = 1 << 30;   // rows are counted in 32 bits, a few past the last one too

// Sums of products of 8-bit integers stay inside 32 bits: 2^14 K < 2^31.
constexpr int32_t kMaxKInt8 = 131072 - 128;

// Codes [T, n] and, behind them, their scales [T] in a buffer of the workspace (n is a multiple of 128).
float* scales_behind(char* codes, int64_t T, int64_t n) { return reinterpret_cast<float*>(codes + T * n); }

// What is wrong with a layer's shape or weights for a step of T tokens.
int32_t check_int8(const relserve_layer* L, const relserve_layer_weights_i8* wt, int64_t T) {
    const relserve_layer_config& c = L->cfg;
    for (int64_t k : {(int64_t)c.hidden, (int64_t)L->q_dim, (int64_t)c.mlp_dim})
        if (k % 128 || k > kMaxKInt8) return RELSERVE_ERR_BAD_ARGUMENT;
    if ((int64_t)c.mlp_dim >= 2 * (int64_t)c.hidden + 4 * (int64_t)L->q_dim) return RELSERVE_ERR_BAD_ARGUMENT;   // where the step keeps codes
    if (T == 0) return RELSERVE_OK;
    if (!wt->w_in_norm || !wt->w_qkv || !wt->w_o || !wt->w_post_norm || !wt->w_gate_up || !wt->w_down || !wt->s_qkv || !wt->s_o ||
        !wt->s_gate_up || !wt->s_down)
        return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({wt->w_in_norm, wt->w_qkv, wt->w_o, wt->w_post_norm, wt->w_gate_up, wt->w_down, wt->s_qkv, wt->s_o, wt->s_gate_up, wt->s_down}))
        return RELSERVE_ERR_BAD_ARGUMENT;
    auto matrix = [&](int64_t rows, int64_t k) { return (wt->packed ? (rows + 255) / 256 * 256 : rows) * k; };
    const int64_t largest = std::max({T * std::max({c.hidden, L->q_dim, c.mlp_dim}), matrix(L->qkv_dim, c.hidden), matrix(c.hidden, L->q_dim),
                                      matrix(2 * (int64_t)c.mlp_dim, c.hidden), matrix(c.hidden, c.mlp_dim)});
    return largest >= ((int64_t)1 << 31) ? RELSERVE_ERR_TOO_LARGE : RELSERVE_OK;
}

int32_t layer_step_int8(const relserve_layer* L, const relserve_batch* b, const relserve_layer_weights_i8* wt, const void* x, void* y,
                        relserve_kv_cache cache, void* workspace, size_t workspace_bytes, void* stream) {
    if (int32_t rc = check_pair(L, b, stream)) return rc;
    if (!wt) return RELSERVE_ERR_NULL_POINTER;
    if (int32_t rc = check_cache(b, cache)) return rc;
    const relserve_layer_config& c = L->cfg;
    const int32_t T = b->dev.T;
    if (int32_t rc = check_int8(L, wt, T)) return rc;
    if (T == 0) return RELSERVE_OK;
    if (!x || !y) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({x, y})) return RELSERVE_ERR_BAD_ARGUMENT;
    const bool packed = wt->packed != 0;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) % kAlign)) return RELSERVE_ERR_WORKSPACE;
    Workspace w = carve(*L, T, workspace);
    if (w.total > workspace_bytes) return RELSERVE_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    relserve_layer* prof = L->profile ? const_cast<relserve_layer*>(L) : nullptr;
    hipError_t e = hipSuccess;
    auto run = [&](int slot, auto&& launch) {
        if (e != hipSuccess) return;
        profile_mark(prof, slot, s, true);
        e = launch();
        profile_mark(prof, slot, s, false);
    };
    // Codes live where the 16-bit step keeps what is over by then: of the norms in h, of the attention in q, of the SwiGLU product from h on
    // through q and attn (2 T H + 4 T q_dim bytes).
    char *h = w.h, *attn = w.q, *act = w.h;
    float *h_s = scales_behind(h, T, c.hidden), *attn_s = scales_behind(attn, T, L->q_dim), *act_s = scales_behind(act, T, c.mlp_dim);
    const BatchDev& batch = attention_batch(*b, cache);
    const PartialState part = partial_state(*L, batch, w);
    const KvFormat kv = kv_format(cache);
    run(S_NORM1, [&] { return launch_row_codes(x, false, nullptr, wt->w_in_norm, c.rms_eps, T, c.hidden, nullptr, h, h_s, s); });
    run(S_QKV, [&] {
        return launch_qkv_rope_append_i8(b->dev, *L, h, h_s, wt->w_qkv, wt->s_qkv, w.q, cache.k_pages, cache.v_pages, s, w.accum, packed, kv);
    });
    if (e == hipSuccess)
        e = launch_attention(batch, *L, w.q, L->q_dim, cache.k_pages, cache.v_pages, w.attn, part.o, part.ml, s, prof, kv);
    run(S_QUANTISE, [&] { return launch_row_codes(w.attn, false, nullptr, nullptr, 0.0f, T, L->q_dim, nullptr, attn, attn_s, s); });
    run(S_O, [&] { return launch_linear_i8(attn, attn_s, wt->w_o, wt->s_o, T, c.hidden, L->q_dim, 1, x, w.x1, s, w.accum, packed); });
    run(S_NORM2, [&] { return launch_row_codes(w.x1, true, nullptr, wt->w_post_norm, c.rms_eps, T, c.hidden, nullptr, h, h_s, s); });
    run(S_GU, [&] { return launch_linear_i8(h, h_s, wt->w_gate_up, wt->s_gate_up, T, 2 * c.mlp_dim, c.hidden, 3, nullptr, w.act, s, w.accum, packed); });
    run(S_DOWN, [&] {
        const hipError_t q = launch_row_codes(w.act, false, nullptr, nullptr, 0.0f, T, c.mlp_dim, nullptr, act, act_s, s);
        return q != hipSuccess ? q : launch_linear_i8(act, act_s, wt->w_down, wt->s_down, T, c.hidden, c.mlp_dim, 2, w.x1, y, s, w.accum, packed);
    });
    return e == hipSuccess ? RELSERVE_OK : RELSERVE_ERR_HIP;
}

}  // namespace

extern "C" {

int32_t relserve_quantise_rows_i8(const void* in, int32_t n_rows, int32_t n, void* codes, float* scales, void* stream) {
    drop_stale_hip_error();
    if (n_rows < 0 || n <= 0 || n % 8) return RELSERVE_ERR_BAD_ARGUMENT;
    if (n_rows > kMaxRowCodes) return RELSERVE_ERR_TOO_LARGE;
    if (n_rows == 0) return RELSERVE_OK;
    if (!in || !codes || !scales) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({in, codes})) return RELSERVE_ERR_BAD_ARGUMENT;
    return launch_row_codes(in, false, nullptr, nullptr, 0.0f, n_rows, n, nullptr, codes, scales, static_cast<hipStream_t>(stream)) == hipSuccess
               ? RELSERVE_OK
               : RELSERVE_ERR_HIP;
}

int32_t relserve_add_rmsnorm_i8(const void* x, int32_t x_is_f32, const void* delta, const void* w, float eps, int32_t n_rows,
                                int32_t hidden, void* sum, void* codes, float* scales, void* stream) {
    drop_stale_hip_error();
    if (n_rows < 0 || hidden <= 0 || hidden % 8) return RELSERVE_ERR_BAD_ARGUMENT;
    if (n_rows > kMaxRowCodes) return RELSERVE_ERR_TOO_LARGE;
    if (n_rows == 0) return RELSERVE_OK;
    if (!x || !w || !codes || !scales) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({x, delta, w, sum, codes})) return RELSERVE_ERR_BAD_ARGUMENT;
    return launch_row_codes(x, x_is_f32 != 0, delta, w, eps, n_rows, hidden, sum, codes, scales, static_cast<hipStream_t>(stream)) == hipSuccess
               ? RELSERVE_OK
               : RELSERVE_ERR_HIP;
}

int32_t relserve_linear_i8_workspace_bytes(int32_t T, int32_t N, size_t* out) {
    if (!out) return RELSERVE_ERR_NULL_POINTER;
    if (T < 0 || N <= 0) return RELSERVE_ERR_BAD_ARGUMENT;
    *out = (size_t)gemm_scratch_floats(T, N) * 4;
    return RELSERVE_OK;
}

int32_t relserve_linear_i8(const void* a, const float* a_scale, const void* w, const float* w_scale, int32_t T, int32_t N, int32_t K,
                           int32_t epilogue, const void* residual, void* out, int32_t packed, void* workspace, size_t workspace_bytes,
                           void* stream) {
    drop_stale_hip_error();
    if (T < 0 || N <= 0 || K <= 0 || K % 128 || epilogue < 0 || epilogue > 3) return RELSERVE_ERR_BAD_ARGUMENT;
    if (epilogue == 3 ? N % 16 : N % 4) return RELSERVE_ERR_BAD_ARGUMENT;
    const int64_t w_rows = packed ? ((int64_t)N + 255) / 256 * 256 : N;
    if (K > kMaxKInt8 || (int64_t)T * K >= ((int64_t)1 << 31) || w_rows * K >= ((int64_t)1 << 31)) return RELSERVE_ERR_TOO_LARGE;
    if (T == 0) return RELSERVE_OK;
    if (!a || !a_scale || !w || !w_scale || !out) return RELSERVE_ERR_NULL_POINTER;
    if (epilogue == 2 && !residual) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({a, w, w_scale, residual, out})) return RELSERVE_ERR_BAD_ARGUMENT;
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) % kAlign || workspace_bytes < (size_t)gemm_scratch_floats(T, N) * 4))
        return RELSERVE_ERR_WORKSPACE;
    return launch_linear_i8(a, a_scale, w, w_scale, T, N, K, epilogue, residual, out, static_cast<hipStream_t>(stream),
                            static_cast<float*>(workspace), packed != 0) == hipSuccess
               ? RELSERVE_OK
               : RELSERVE_ERR_HIP;
}

int32_t relserve_qkv_rope_append_i8(const relserve_layer* L, const relserve_batch* b, const void* h, const float* h_scale,
                                    const void* w_qkv, const float* s_qkv, void* q_out, relserve_kv_cache cache, int32_t packed,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    drop_stale_hip_error();
    if (int32_t rc = check_pair(L, b, stream)) return rc;
    if (int32_t rc = check_cache(b, cache)) return rc;
    const int32_t T = b->dev.T, H = L->cfg.hidden;
    if (H % 128) return RELSERVE_ERR_BAD_ARGUMENT;
    const int64_t w_rows = packed ? ((int64_t)L->qkv_dim + 255) / 256 * 256 : L->qkv_dim;
    if (H > kMaxKInt8 || (int64_t)T * H >= ((int64_t)1 << 31) || w_rows * H >= ((int64_t)1 << 31)) return RELSERVE_ERR_TOO_LARGE;
    if (T == 0) return RELSERVE_OK;
    if (!h || !h_scale || !w_qkv || !s_qkv || !q_out) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({h, w_qkv, s_qkv, q_out})) return RELSERVE_ERR_BAD_ARGUMENT;
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) % kAlign || workspace_bytes < (size_t)gemm_scratch_floats(T, L->qkv_dim) * 4))
        return RELSERVE_ERR_WORKSPACE;
    return launch_qkv_rope_append_i8(b->dev, *L, h, h_scale, w_qkv, s_qkv, q_out, cache.k_pages, cache.v_pages, static_cast<hipStream_t>(stream),
                                     static_cast<float*>(workspace), packed != 0, kv_format(cache)) == hipSuccess
               ? RELSERVE_OK
               : RELSERVE_ERR_HIP;
}

int32_t relserve_layer_step_i8(const relserve_layer* L, const relserve_batch* b, const relserve_layer_weights_i8* wt, const void* x, void* y,
                               relserve_kv_cache cache, void* workspace, size_t workspace_bytes, void* stream) {
    drop_stale_hip_error();
    return layer_step_int8(L, b, wt, x, y, cache, workspace, workspace_bytes, stream);
}

int32_t relserve_model_step_i8(const relserve_layer* L, const relserve_batch* b, const relserve_model* m,
                               const relserve_layer_weights_i8* layers, const int32_t* token_ids, void* logits,
                               void* workspace, size_t workspace_bytes, void* stream) {
    drop_stale_hip_error();
    if (!layers) return RELSERVE_ERR_NULL_POINTER;
    auto check = [&](int32_t l) { return check_int8(L, &layers[l], b->dev.T); };
    auto stack = [&](char* x, size_t layer_ws) -> int32_t {
        for (int32_t l = 0; l < m->n_layers; ++l)
            if (int32_t rc = layer_step_int8(L, b, &layers[l], x, x, m->caches[l], workspace, layer_ws, stream)) return rc;
        return RELSERVE_OK;
    };
    return model_around(L, b, m, layers, token_ids, logits, workspace, workspace_bytes, stream, check, stack);
}

}  // extern "C"
