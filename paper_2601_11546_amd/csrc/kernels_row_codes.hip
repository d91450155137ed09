// Rows as 8-bit integers with one scale per row: what an int8 projection multiplies.
//   scale[t] = m / 127, m the row's largest magnitude;   code[t, i] = rint(value[t, i] * 127 / m)
// of the rows of a bf16 matrix, or of rmsnorm(x + delta) * w, whose sum with the addend is kept on the way.
#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

struct RowCodesArgs {
    const void* x;           // [rows, n] bf16 or fp32
    const uint16_t* delta;   // [rows, n] bf16 or null
    const uint16_t* w;       // [n] bf16, the norm's weights; null: the rows themselves
    float eps;
    int32_t n;
    void* sum;               // [rows, n] x + delta in x's type, or null
    uint8_t* codes;
    float* scales;
};

template <bool IN_F32>
__device__ __forceinline__ void load_values(const void* base, int64_t at, float (&v)[8]) {
    if (IN_F32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        const float4 a = p[0], b = p[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
        v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
        v[4] = bf16_lo(u.z); v[5] = bf16_hi(u.z); v[6] = bf16_lo(u.w); v[7] = bf16_hi(u.w);
    }
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// One workgroup per row, the row read twice.
template <bool IN_F32>
__global__ void __launch_bounds__(256) row_codes_kernel(RowCodesArgs p) {
    __shared__ float red_ss[4];
    __shared__ uint32_t red_m[4];
    const int64_t row = (int64_t)blockIdx.x * p.n;
    const int tid = threadIdx.x, chunks = p.n / 8;
    // the row's stream (as it is kept) and the values whose codes are taken, less the factor that a norm has for the whole row
    auto chunk = [&](int c, bool second, float (&s)[8], float (&v)[8]) {
        const int64_t at = row + 8 * (int64_t)c;
        load_values<IN_F32>(second && p.sum ? p.sum : p.x, at, s);
        if (p.delta && !(second && p.sum)) {
            float d[8];
            load_values<false>(p.delta, at, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[i] += d[i];
                if (!IN_F32) s[i] = bf16_to_f32((uint16_t)f32_to_bf16_bits(s[i]));
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = s[i];
        if (p.w) {
            float w[8];
            load_values<false>(p.w, 8 * (int64_t)c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= w[i];
        }
    };
    float ss = 0.f;
    uint32_t m = 0;   // magnitudes compare as integers, and a NaN is above all others
    for (int c = tid; c < chunks; c += 256) {
        float s[8], v[8];
        chunk(c, false, s, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(s[i], s[i], ss), m = max(m, magnitude_bits(v[i]));
        if (p.sum) {
            const int64_t at = row + 8 * (int64_t)c;
            if (IN_F32) {
                float4* o = reinterpret_cast<float4*>(static_cast<float*>(p.sum) + at);
                o[0] = make_float4(s[0], s[1], s[2], s[3]);
                o[1] = make_float4(s[4], s[5], s[6], s[7]);
            } else {
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.sum) + at) =
                    make_uint4(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]), pack_bf16x2(s[4], s[5]), pack_bf16x2(s[6], s[7]));
            }
        }
    }
    ss = wave_sum(ss);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if ((tid & 63) == 0) red_ss[tid >> 6] = ss, red_m[tid >> 6] = m;
    __syncthreads();
    ss = red_ss[0] + red_ss[1] + red_ss[2] + red_ss[3];
    m = max(max(red_m[0], red_m[1]), max(red_m[2], red_m[3]));
    const float top = __uint_as_float(m), inv = p.w ? 1.0f / sqrtf(ss / (float)p.n + p.eps) : 1.0f;
    if (tid == 0) p.scales[blockIdx.x] = top * inv / 127.0f;
    // 127 / top overflows for the smallest magnitudes: these are lifted by 2^100 first.  Nothing to scale by (0, infinite, NaN): codes of 0.
    const float lift = top < 0x1p-100f ? 0x1p100f : 1.0f;
    const bool none = m == 0 || m >= 0x7f800000u;
    const float per = none ? 0.0f : 127.0f / (top * lift);
    for (int c = tid; c < chunks; c += 256) {
        float s[8], v[8];
        chunk(c, true, s, v);
        uint32_t o[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i / 4] |= none ? 0u : ((uint32_t)(int)rintf(v[i] * lift * per) & 0xffu) << 8 * (i % 4);
        *reinterpret_cast<uint2*>(p.codes + row + 8 * (int64_t)c) = make_uint2(o[0], o[1]);
    }
}

}  // namespace

hipError_t launch_row_codes(const void* x, bool x_is_f32, const void* delta, const void* w, float eps, int32_t rows, int32_t n, void* sum,
                            void* codes, float* scales, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const RowCodesArgs p{x, static_cast<const uint16_t*>(delta), static_cast<const uint16_t*>(w), eps, n, sum, static_cast<uint8_t*>(codes), scales};
    if (x_is_f32)
        row_codes_kernel<true><<<dim3(rows), dim3(256), 0, s>>>(p);
    else
        row_codes_kernel<false><<<dim3(rows), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace relserve
