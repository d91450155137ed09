// What the sources of the host boundary share: workspace carving, checks of handles and pools, the model step around its layers.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "relserve_internal.h"

namespace relserve {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

// the last slot is the int8 step's (its other pass over rows counts with the down projection); the attention kernels store the codes of
// relserve_layer_step_w8a8 themselves
enum { S_NORM1 = 0, S_QKV, S_ATTN_OWN, S_ATTN_PREFIX, S_ATTN_TILE, S_ATTN_SPLIT, S_O, S_NORM2, S_GU, S_DOWN, S_ATTN_MERGE, S_QUANTISE };

struct Workspace {
    char* h;         // [T, H] bf16 (normed activations; reused for the post norm)
    char* q;         // [T, q_dim] bf16 rotated queries
    char* attn;      // [T, q_dim] bf16
    char* x1;        // [T, H] fp32 residual stream after attention
    char* act;       // [T, I] bf16
    float* part_o;   // [T + split slots, n_q, d] fp32
    float* part_ml;  // [T + split slots, n_q, 2] fp32
    float* accum;    // fp32 split-K scratch of the GEMMs
    size_t accum_floats;
    size_t total;
};

inline Workspace carve(const relserve_layer& L, int64_t T, void* base) {
    Workspace w;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? static_cast<char*>(base) + off : nullptr;
        off += align_up(bytes);
        return p;
    };
    const relserve_layer_config& c = L.cfg;
    w.h = take((size_t)T * c.hidden * 2);
    w.q = take((size_t)T * L.q_dim * 2);
    w.attn = take((size_t)T * L.q_dim * 2);
    w.x1 = take((size_t)T * c.hidden * 4);
    w.act = take((size_t)T * c.mlp_dim * 2);
    const size_t part_rows = (size_t)(T + split_slot_cap(T));
    w.part_o = reinterpret_cast<float*>(take(part_rows * L.q_dim * 4));
    w.part_ml = reinterpret_cast<float*>(take(part_rows * c.n_q_heads * 2 * 4));
    w.accum_floats = (size_t)gemm_scratch_floats(T, std::max({L.qkv_dim, 2 * c.mlp_dim, c.hidden}));
    w.accum = reinterpret_cast<float*>(take(w.accum_floats * 4));
    w.total = off;
    return w;
}

// Where the attention passes of a batch keep partial state: the workspace's own rows, or (slot plans) the GEMM scratch.
struct PartialState { float* o; float* ml; };
inline PartialState partial_state(const relserve_layer& L, const BatchDev& b, const Workspace& w) {
    if (b.n_scratch_slots == 0) return {w.part_o, w.part_ml};
    return {w.accum, w.accum + (int64_t)b.n_scratch_slots * L.q_dim};
}

// The cut of the attention a step over these pools runs.  A 16-bit output that rounds the other way moves codes of the keys and
// values the next layer appends to its quantised pool, and those move the rest of the stack (3 % of the codes of a third 13B
// layer, 2e-2 of the logits after four), so over quantised pools every entry point takes the cut without slots, whose results
// stacks were recorded with.
inline const BatchDev& attention_batch(const relserve_batch& b, const relserve_kv_cache& cache) {
    return cache.dtype == RELSERVE_KV_FP8 ? b.dev_no_slots : b.dev;
}

inline KvFormat kv_format(const relserve_kv_cache& cache) {
    KvFormat f;
    f.fp8 = cache.dtype == RELSERVE_KV_FP8;
    if (f.fp8) f.k_scale = cache.k_scale, f.v_scale = cache.v_scale;
    return f;
}

inline int32_t check_cache(const relserve_batch* b, const relserve_kv_cache& cache, bool fp8_ok = true) {
    if (!cache.k_pages || !cache.v_pages) return RELSERVE_ERR_NULL_POINTER;
    if (cache.dtype != RELSERVE_KV_BF16 && cache.dtype != RELSERVE_KV_FP8) return RELSERVE_ERR_BAD_ARGUMENT;
    if (cache.dtype == RELSERVE_KV_FP8) {
        if (!fp8_ok) return RELSERVE_ERR_BAD_ARGUMENT;
        if (!(cache.k_scale > 0.0f) || !(cache.v_scale > 0.0f) || !std::isfinite(cache.k_scale) || !std::isfinite(cache.v_scale))
            return RELSERVE_ERR_BAD_ARGUMENT;
    }
    if (cache.num_pages < b->dev.num_pages) return RELSERVE_ERR_MISMATCH;
    return RELSERVE_OK;
}

// stream: where the caller submits work that reads the batch
inline int32_t check_pair(const relserve_layer* L, const relserve_batch* b, const void* stream) {
    if (!L || !b) return RELSERVE_ERR_NULL_POINTER;
    if (std::memcmp(&L->cfg, &b->cfg, sizeof(relserve_layer_config)) != 0) return RELSERVE_ERR_MISMATCH;
    if (stream) b->other_stream.store(true, std::memory_order_relaxed);
    return RELSERVE_OK;
}

// The launchers report hipGetLastError() after a launch; an error an earlier, unrelated HIP call of this thread left
// behind (the runtime keeps the last one until it is read) must not be taken for theirs.
inline void drop_stale_hip_error() { (void)hipGetLastError(); }

// Operands that kernels read and write 16 bytes at a time (null: not given).
inline bool aligned16(std::initializer_list<const void*> pointers) {
    for (const void* p : pointers)
        if (reinterpret_cast<uintptr_t>(p) % 16) return false;
    return true;
}

// A model step around its layers: check(l) is what is wrong with layer l's weights, layers(x, bytes of a layer's workspace) steps the stack on
// the residual stream x, rounded to bf16 between layers.
template <typename Check, typename Layers>
int32_t model_around(const relserve_layer* L, const relserve_batch* b, const relserve_model* m, const void* layer_weights, const int32_t* token_ids,
                     void* logits, void* workspace, size_t workspace_bytes, void* stream, Check check, Layers layers) {
    if (int32_t rc = check_pair(L, b, stream)) return rc;
    if (!m) return RELSERVE_ERR_NULL_POINTER;
    if (m->n_layers < 0 || m->vocab <= 0 || m->vocab % 4) return RELSERVE_ERR_BAD_ARGUMENT;
    const int32_t T = b->dev.T, B = b->dev.num_reqs, H = L->cfg.hidden;
    if (T == 0) return RELSERVE_OK;
    if (!token_ids || !logits || !m->embedding || !m->w_final_norm || !m->w_lm_head) return RELSERVE_ERR_NULL_POINTER;
    if (m->n_layers > 0 && (!layer_weights || !m->caches)) return RELSERVE_ERR_NULL_POINTER;
    for (int32_t l = 0; l < m->n_layers; ++l) {
        if (int32_t rc = check(l)) return rc;
        if (int32_t rc = check_cache(b, m->caches[l])) return rc;
    }
    if ((int64_t)m->vocab * H >= ((int64_t)1 << 31)) return RELSERVE_ERR_TOO_LARGE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) % kAlign)) return RELSERVE_ERR_WORKSPACE;
    const size_t layer_ws = carve(*L, T, nullptr).total;
    const size_t x_bytes = align_up((size_t)T * H * 2), last_bytes = align_up((size_t)B * H * 2);
    if (layer_ws + x_bytes + last_bytes > workspace_bytes) return RELSERVE_ERR_WORKSPACE;
    char* x = static_cast<char*>(workspace) + layer_ws;
    char* h_last = x + x_bytes;

    hipStream_t s = static_cast<hipStream_t>(stream);
    if (launch_embedding(token_ids, m->embedding, m->vocab, H, T, x, s) != hipSuccess) return RELSERVE_ERR_HIP;
    if (int32_t rc = layers(x, layer_ws)) return rc;
    if (launch_rmsnorm(x, false, m->w_final_norm, L->cfg.rms_eps, B, H, h_last, s, b->dev.last_tok) != hipSuccess)
        return RELSERVE_ERR_HIP;
    if (launch_linear(h_last, m->w_lm_head, B, m->vocab, H, 1, nullptr, logits, s) != hipSuccess)
        return RELSERVE_ERR_HIP;
    return RELSERVE_OK;
}

}  // namespace relserve
