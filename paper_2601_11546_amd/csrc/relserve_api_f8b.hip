// Host boundary of the block-scaled projections and of the log probabilities: argument checks.
#include "relserve_host.h"

using namespace relserve;

namespace {

constexpr int32_t kMaxRowBlocks = 1 << 30;    // rows are counted in 32 bits, a few past the last one too
constexpr int32_t kMaxRowLength = 1 << 22;    // its blocks are a dimension of a launch
constexpr int32_t kMaxLogitRows = 1 << 22;    // a workgroup's threads each, counted in 32 bits
constexpr int32_t kMaxVocab = 1 << 24;        // counted in fp32 too
constexpr int32_t kMaxTop = 32;

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

}  // namespace

extern "C" {

int32_t relserve_quantise_f8b(const void* in, int32_t n_rows, int32_t n, int32_t block_rows, void* codes, float* scales, void* stream) {
    drop_stale_hip_error();
    if (n_rows < 0 || n <= 0 || n % 128 || (block_rows != 1 && block_rows != 128)) return RELSERVE_ERR_BAD_ARGUMENT;
    if (n_rows > kMaxRowBlocks || n > kMaxRowLength) return RELSERVE_ERR_TOO_LARGE;
    if (n_rows == 0) return RELSERVE_OK;
    if (!in || !codes || !scales) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({in, codes}) || !aligned(scales, 4)) return RELSERVE_ERR_BAD_ARGUMENT;
    return launch_block_codes(in, n_rows, n, block_rows, codes, scales, static_cast<hipStream_t>(stream)) == hipSuccess ? RELSERVE_OK : RELSERVE_ERR_HIP;
}

int32_t relserve_add_rmsnorm_f8b(const void* x, int32_t x_is_f32, const void* delta, const void* w, float eps, int32_t n_rows, int32_t hidden,
                                 void* sum, void* codes, float* scales, void* stream) {
    drop_stale_hip_error();
    if (n_rows < 0 || hidden <= 0 || hidden % 128) return RELSERVE_ERR_BAD_ARGUMENT;
    if (n_rows > kMaxRowBlocks || hidden > kMaxRowLength) return RELSERVE_ERR_TOO_LARGE;
    if (n_rows == 0) return RELSERVE_OK;
    if (!x || !w || !codes || !scales) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({x, delta, w, sum, codes}) || !aligned(scales, 4)) return RELSERVE_ERR_BAD_ARGUMENT;
    return launch_add_rmsnorm_f8b(x, x_is_f32 != 0, delta, w, eps, n_rows, hidden, sum, codes, scales, static_cast<hipStream_t>(stream)) == hipSuccess
               ? RELSERVE_OK
               : RELSERVE_ERR_HIP;
}

int32_t relserve_linear_f8b_workspace_bytes(int32_t T, int32_t N, size_t* out) {
    if (!out) return RELSERVE_ERR_NULL_POINTER;
    if (T < 0 || N <= 0) return RELSERVE_ERR_BAD_ARGUMENT;
    *out = (size_t)gemm_f8b_scratch_floats(T, N) * 4;
    return RELSERVE_OK;
}

int32_t relserve_linear_f8b(const void* a, const float* a_scale, const void* w, const float* w_scale, int32_t T, int32_t N, int32_t K,
                            int32_t epilogue, const void* residual, void* out, int32_t packed, void* workspace, size_t workspace_bytes,
                            void* stream) {
    drop_stale_hip_error();
    if (T < 0 || N <= 0 || K <= 0 || K % 128 || epilogue < 0 || epilogue > 3) return RELSERVE_ERR_BAD_ARGUMENT;
    if (epilogue == 3 ? N % 16 : N % 4) return RELSERVE_ERR_BAD_ARGUMENT;
    const int64_t w_rows = packed ? ((int64_t)N + 255) / 256 * 256 : N;
    if ((int64_t)T * K >= ((int64_t)1 << 31) || w_rows * K >= ((int64_t)1 << 31)) return RELSERVE_ERR_TOO_LARGE;
    if (T == 0) return RELSERVE_OK;
    if (!a || !a_scale || !w || !w_scale || !out) return RELSERVE_ERR_NULL_POINTER;
    if (epilogue == 2 && !residual) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned16({a, w, residual, out}) || !aligned(a_scale, 4) || !aligned(w_scale, 4)) return RELSERVE_ERR_BAD_ARGUMENT;
    if (workspace && (!aligned(workspace, kAlign) || workspace_bytes < (size_t)gemm_f8b_scratch_floats(T, N) * 4)) return RELSERVE_ERR_WORKSPACE;
    return launch_linear_f8b(a, a_scale, w, w_scale, T, N, K, epilogue, residual, out, static_cast<hipStream_t>(stream), static_cast<float*>(workspace),
                             packed != 0) == hipSuccess
               ? RELSERVE_OK
               : RELSERVE_ERR_HIP;
}

int32_t relserve_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t n_top, size_t* out) {
    if (!out) return RELSERVE_ERR_NULL_POINTER;
    if (n_rows < 0 || vocab <= 0 || n_top < 0 || n_top > kMaxTop) return RELSERVE_ERR_BAD_ARGUMENT;
    *out = (size_t)logprobs_scratch_bytes(n_rows, n_top);
    return RELSERVE_OK;
}

int32_t relserve_logprobs(const void* logits, int32_t logits_are_f32, int32_t n_rows, int32_t vocab, int64_t pitch, const int32_t* ids, int32_t n_ids,
                          float* logprobs, float* entropy, int32_t n_top, int32_t* top_ids, float* top_logprobs, void* workspace,
                          size_t workspace_bytes, void* stream) {
    drop_stale_hip_error();
    if (n_rows < 0 || vocab <= 0 || pitch < vocab || n_ids < 0 || n_top < 0 || n_top > kMaxTop) return RELSERVE_ERR_BAD_ARGUMENT;
    if (n_rows > kMaxLogitRows || vocab > kMaxVocab) return RELSERVE_ERR_TOO_LARGE;
    if (n_rows == 0) return RELSERVE_OK;
    if (!logits || (n_ids && (!ids || !logprobs)) || (n_top && (!top_ids || !top_logprobs))) return RELSERVE_ERR_NULL_POINTER;
    if (!aligned(logits, logits_are_f32 ? 4 : 2) || !aligned(ids, 4) || !aligned(logprobs, 4) || !aligned(entropy, 4) || !aligned(top_ids, 4) ||
        !aligned(top_logprobs, 4))
        return RELSERVE_ERR_BAD_ARGUMENT;
    if (workspace && (!aligned(workspace, kAlign) || workspace_bytes < (size_t)logprobs_scratch_bytes(n_rows, n_top))) return RELSERVE_ERR_WORKSPACE;
    const LogprobsArgs args{logits, logits_are_f32 != 0, n_rows, vocab, pitch, ids, n_ids, logprobs, entropy, n_top, top_ids, top_logprobs, workspace};
    return launch_logprobs(args, static_cast<hipStream_t>(stream)) == hipSuccess ? RELSERVE_OK : RELSERVE_ERR_HIP;
}

}  // extern "C"
