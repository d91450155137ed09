// int8 projections: out[t, n] = sum_k a[t, k] w[n, k] * (a_scale[t] * w_scale[n]) of 8-bit integers, summed exactly in 32 bits.
#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

typedef int i32x16_t __attribute__((ext_vector_type(16)));

struct LinearI8Args {
    const int8_t* a;
    const float* a_scale;
    const int8_t* w;
    const float* w_scale;
    const void* residual;
    void* out;
    int32_t w_packed, T, N, K, n_half;
    int32_t tiles_m;
};

// One wave per tile of 32 tokens x 32 features (two such feature tiles for SwiGLU: gate and up), operands straight from global memory.
// 32 x 32 products of k = 32: lane l holds 16 codes of row l % 32, half l / 32; result register r is feature 8 (r / 4) + 4 (l / 32) + r % 4
// of token l % 32.
template <int EPI>
__global__ void __launch_bounds__(64) linear_i8_wave_kernel(LinearI8Args p) {
    constexpr int NT = EPI == 3 ? 2 : 1, U = 4;
    const int lane = threadIdx.x, l32 = lane & 31, g = lane >> 5;
    const int unit = blockIdx.x / p.tiles_m, t = (int)(blockIdx.x % p.tiles_m) * 32 + l32, tc = min(t, p.T - 1);
    const int cols = EPI == 3 ? p.n_half : p.N, n0 = unit * 32, rows = min(32, cols - n0);
    const char* const ab = reinterpret_cast<const char*>(p.a) + (int64_t)tc * p.K + 16 * g;
    const char* wb[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = j * p.n_half + n0 + min(l32, rows - 1);   // rows past the end: the last one again, never stored
        wb[j] = reinterpret_cast<const char*>(p.w) + (p.w_packed ? (int64_t)(n >> 8) * p.K * 256 + (n & 255) * 128 : (int64_t)n * p.K) + 16 * g;
    }
    const int64_t slice = p.w_packed ? 32768 : 128;   // from one slice of 128 codes to the next
    i32x16_t acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] = 0;
    for (int s = 0; s < p.K / 128; ++s) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const i32x4_t av = *reinterpret_cast<const i32x4_t*>(ab + 128 * s + 32 * u);
#pragma unroll
            for (int j = 0; j < NT; ++j)
                acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4_t*>(wb[j] + s * slice + 32 * u), av, acc[j], 0, 0, 0);
        }
    }
    if (t >= p.T) return;
    const float at = p.a_scale[t];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int f = n0 + 8 * q + 4 * g;
        if (f >= cols) break;   // rows are a multiple of 4
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)acc[0][4 * q + i] * p.w_scale[f + i] * at;
        const int64_t o = (int64_t)t * cols + f;
        if constexpr (EPI == 3) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = silu_mul(v[i], (float)acc[NT - 1][4 * q + i] * p.w_scale[p.n_half + f + i] * at);
        }
        if constexpr (EPI == 1) {
            if (p.residual) {
                const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.residual) + o);
                v[0] += bf16_lo(r.x); v[1] += bf16_hi(r.x); v[2] += bf16_lo(r.y); v[3] += bf16_hi(r.y);
            }
            *reinterpret_cast<float4*>(static_cast<float*>(p.out) + o) = make_float4(v[0], v[1], v[2], v[3]);
            continue;
        }
        if constexpr (EPI == 2) {
            const float4 r = *reinterpret_cast<const float4*>(static_cast<const float*>(p.residual) + o);
            v[0] += r.x; v[1] += r.y; v[2] += r.z; v[3] += r.w;
        }
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
}

}  // namespace

hipError_t launch_linear_i8(const void* a, const float* a_scale, const void* w, const float* w_scale, int32_t T, int32_t N, int32_t K,
                            int32_t epilogue, const void* residual, void* out, hipStream_t s, float* accum, bool w_packed) {
    if (T == 0) return hipSuccess;
    LinearI8Args p{static_cast<const int8_t*>(a), a_scale, static_cast<const int8_t*>(w), w_scale, residual, out, w_packed, T, N, K, N / 2, (T + 31) / 32};
    const dim3 grid(p.tiles_m * (((epilogue == 3 ? N / 2 : N) + 31) / 32));
    switch (epilogue) {
        case 0: linear_i8_wave_kernel<0><<<grid, dim3(64), 0, s>>>(p); break;
        case 1: linear_i8_wave_kernel<1><<<grid, dim3(64), 0, s>>>(p); break;
        case 2: linear_i8_wave_kernel<2><<<grid, dim3(64), 0, s>>>(p); break;
        case 3: linear_i8_wave_kernel<3><<<grid, dim3(64), 0, s>>>(p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace relserve
