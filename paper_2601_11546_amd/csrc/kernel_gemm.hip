// The projections on 16-bit operands and on 8-bit floating point codes: entry points of the kernels in gemm_kernels.h.
#define RELSERVE_GEMM_INT8 0
#include "gemm_kernels.h"

namespace relserve {

void gemm_force_plan(int cand, int splits) {
    g_forced_plan.store(cand < 0 || cand >= kTileCount ? -1 : (cand | (splits << 8)), std::memory_order_relaxed);
    gemm_force_plan_i8(cand, splits);
}

GemmPlan gemm_plan(int32_t T, int64_t features, int32_t K, bool qkv, bool swiglu, bool scratch) {
    const Plan p = plan_for(T, features, K, qkv, scratch, swiglu);
    GemmPlan g{kTiles[p.cand].bm, kTiles[p.cand].bn, p.tail_tiles, p.splits, p.cols1, 0, 0, false};
    if (p.cols1 > 0) g.rows1 = kTiles[p.cand1].bm, g.rows2 = kTiles[p.cand2].bm;
    g.halves = p.cand == 0 && p.tail_tiles > 0 && in_halves(tile_count(kTiles[0], T, features), p.tail_tiles, p.splits, K, false);
    return g;
}

int64_t gemm_scratch_floats(int64_t T, int64_t n_max) {
    // skinny: one slab per split, at most 256 units of 128 x 256 floats, or a single slab of T x N
    return T <= SKINNY_MAX_T ? std::max<int64_t>(T * n_max, GEMM_SKINNY_FLOATS) : kTailFloats;
}


// Tiled weight layout for streaming: out[n / 256][k / 64][n % 256][k % 64], rows past N are zeros.  One k
// slice of 256 rows is 32 KB of consecutive memory, so a stage of the GEMM reads whole DRAM pages
// instead of 128-byte pieces 2 K bytes apart.
__global__ void pack_weight_kernel(const uint4* w, uint4* out, int32_t N, int32_t K, int64_t n_chunks) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;   // 16-byte chunk of the output
    if (i >= n_chunks) return;
    const int c = (int)(i & 7), r = (int)((i >> 3) & 255);
    const int64_t slice = i >> 11;                                       // (block, k slice)
    const int ks = (int)(slice % (K / 64));
    const int64_t n = (slice / (K / 64)) * 256 + r;
    out[i] = n < N ? w[(n * K + ks * 64) / 8 + c] : make_uint4(0, 0, 0, 0);
}

hipError_t launch_pack_weight(const void* w, int32_t N, int32_t K, void* out, hipStream_t s) {
    const int64_t n_chunks = (int64_t)((N + 255) / 256) * 256 * K / 8;
    if (n_chunks == 0) return hipSuccess;
    pack_weight_kernel<<<dim3((unsigned)((n_chunks + 255) / 256)), dim3(256), 0, s>>>(
        static_cast<const uint4*>(w), static_cast<uint4*>(out), N, K, n_chunks);
    return hipGetLastError();
}


// 8-bit operands: the kernels see rows of K / 2 two-byte units (same bytes, same layouts) and the scales
static hipError_t set_codes(GemmArgs& p, const CodeScales* codes) {
    if (!codes || !codes->w_scale) return hipSuccess;
    if (p.K % 128 || !(codes->a_scale > 0.0f)) return hipErrorInvalidValue;
    p.f8 = 1;
    p.K /= 2;
    p.w_scale = codes->w_scale;
    p.a_scale = codes->a_scale;
    p.out_f8 = codes->out_scale > 0.0f ? 1 : 0;
    p.out_inv = p.out_f8 ? (float)(1.0 / (double)codes->out_scale) : 0.0f;   // reciprocal in double, rounded once
    return hipSuccess;
}

hipError_t launch_linear(const void* a, const void* w, int32_t T, int32_t N, int32_t K, int32_t epilogue,
                         const void* residual, void* out, hipStream_t s, float* accum, bool w_packed, const CodeScales* codes) {
    if (T == 0) return hipSuccess;
    if ((int64_t)T * K >= ((int64_t)1 << 31) || (int64_t)N * K >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    if (epilogue != EPI_SWIGLU && (N % 4)) return hipErrorInvalidValue;
    if (epilogue == EPI_SWIGLU && ((N / 2) % 8)) return hipErrorInvalidValue;
    if (w_packed && K % 64) return hipErrorInvalidValue;   // only the direct-to-LDS kernel reads it
    GemmArgs p{};
    set_linear(p, a, w, T, N, K, residual, out, accum, w_packed);
    if (hipError_t e = set_codes(p, codes)) return e;
    return run_linear(p, epilogue, s, codes ? codes->next : nullptr);
}

hipError_t launch_qkv_rope_append(const BatchDev& b, const relserve_layer& L, const void* h, const void* w_qkv,
                                  void* q_out, void* k_pages, void* v_pages, hipStream_t s, float* accum,
                                  bool w_packed, KvFormat kv, const CodeScales* codes) {
    if (b.T == 0) return hipSuccess;
    const int32_t K = L.cfg.hidden;
    if ((int64_t)b.T * K >= ((int64_t)1 << 31) || (int64_t)L.qkv_dim * K >= ((int64_t)1 << 31))
        return hipErrorInvalidValue;
    if (w_packed && K % 64) return hipErrorInvalidValue;
    GemmArgs p{};
    set_qkv(p, b, L, h, w_qkv, q_out, k_pages, v_pages, kv, accum, w_packed);
    if (hipError_t e = set_codes(p, codes)) return e;
    return run_qkv(p, L.cfg.head_dim, s);
}

}  // namespace relserve
