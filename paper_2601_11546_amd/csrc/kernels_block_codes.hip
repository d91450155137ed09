// Matrices as 8-bit floating point codes (1 sign, 4 exponent, 3 mantissa bits) with one fp32 scale per block: what a block-scaled projection
// multiplies.
//   scale = m / 448, m the block's largest magnitude;   code = the number of the format nearest to value * 448 / m, ties to even
// of the values of a bf16 matrix in blocks of 1 or 128 rows x 128 values, or of rmsnorm(x + delta) * w in blocks of 128 values of a row, whose
// sum with the addend is kept on the way.
//
// Sixteen lanes hold a block of a row, 16 bytes of bf16 each, and reduce its magnitude among themselves.  The norm's factor 1 / rms is the same
// for a whole row, so it cancels in value * 448 / m: codes are written before the row's sum of squares is known, which goes into the scales
// only.  Memory bound: every byte once.
#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

struct BlockCodesArgs {
    const void* x;           // [rows, n] bf16 or fp32
    const uint16_t* delta;   // [rows, n] bf16 or null
    const uint16_t* w;       // [n] bf16, the norm's weights
    float eps;
    int32_t rows, n;
    int32_t all_rows;        // of the whole matrix: distance of two blocks' scales of a row
    void* sum;               // [rows, n] x + delta in x's type, or null
    uint8_t* codes;
    float* scales;
};

// The larger magnitude, a NaN if either is one.
__device__ __forceinline__ float larger(float m, float v) { return __builtin_elementwise_maximum(m, __builtin_fabsf(v)); }

// The largest magnitude among the sixteen lanes of a block, by rotations inside a row of lanes.
__device__ __forceinline__ float block_largest(float m) {
    m = larger(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x128, 0xf, 0xf, true)));
    m = larger(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x124, 0xf, 0xf, true)));
    m = larger(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x122, 0xf, 0xf, true)));
    return larger(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x121, 0xf, 0xf, true)));
}

// m / 448, rounded once for normal results.
__device__ __forceinline__ float scale_of(float m) {
    if (!(m < INFINITY)) return m;
    const float q = m * (1.0f / 448.0f);
    return __builtin_fmaf(__builtin_fmaf(-q, 448.0f, m), 1.0f / 448.0f, q);
}

// Codes of eight values of a block whose largest magnitude is m.
// The quotient is the value times 448 / m and what that factor lacks: the product alone would put quotients halfway between two codes (in
// bf16 every |v| = m / 7 * 1.0625 is one) on either side.  It is within 2^-43 of its value before it is rounded to 24 bits, and no other
// quotient of two bf16 values, or of two products of such, is nearer than 2^-22 to one halfway: halfway is t / 448 of m with t of five bits, so
// that v * 448 - t * m is a whole multiple of the last place of t * m, a number of at most 21 bits.
// Nothing to scale by (0, infinite, NaN): codes of 0.  448 / m overflows for the smallest magnitudes, and what it lacks is no normal number for the
// largest: such blocks are moved by a power of two first.
__device__ __forceinline__ uint2 codes_of(const float (&u)[8], float m) {
    const bool some = m > 0.0f && m < INFINITY;
    const float move = m < 0x1p-90f ? 0x1p100f : m > 0x1p60f ? 0x1p-100f : 1.0f, top = m * move;
    const float per = some ? 448.0f * __builtin_amdgcn_rcpf(top) : 0.0f, lack = __builtin_fmaf(-per, top, 448.0f) * (per * (1.0f / 448.0f));
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = u[i];
    if (move != 1.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] *= move;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __builtin_fmaf(q[i], per, q[i] * lack);
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    return some ? make_uint2((uint32_t)lo, (uint32_t)hi) : make_uint2(0, 0);
}

__device__ __forceinline__ void widen8(const uint4& r, float (&v)[8]) {
    v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
    v[4] = bf16_lo(r.z); v[5] = bf16_hi(r.z); v[6] = bf16_lo(r.w); v[7] = bf16_hi(r.w);
}

// 8 values as they are loaded
template <bool F32>
struct Raw8 {
    uint4 lo, hi;   // hi: fp32 only
    template <bool FAR>
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const i32x4_t* p = reinterpret_cast<const i32x4_t*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
        if constexpr (FAR) {
            lo = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p));
            if (F32) hi = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p + 1));
        } else {
            lo = __builtin_bit_cast(uint4, p[0]);
            if (F32) hi = __builtin_bit_cast(uint4, p[1]);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if (F32) {
            v[0] = __uint_as_float(lo.x); v[1] = __uint_as_float(lo.y); v[2] = __uint_as_float(lo.z); v[3] = __uint_as_float(lo.w);
            v[4] = __uint_as_float(hi.x); v[5] = __uint_as_float(hi.y); v[6] = __uint_as_float(hi.z); v[7] = __uint_as_float(hi.w);
        } else {
            widen8(lo, v);
        }
    }
};

// ---- rows in blocks of 1 x 128 ----
// A workgroup takes 16 rows, sixteen lanes each, and U blocks of them, all loaded at once; the scales of its 16 rows are consecutive.
template <int U, bool FAR>
__global__ void __launch_bounds__(256) row_blocks_kernel(BlockCodesArgs p) {
    const int lane16 = threadIdx.x & 15, nb = p.n / 128;
    const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int b0 = blockIdx.y * U;
    if (row >= p.rows) return;
    const int64_t base = row * p.n + b0 * 128 + lane16 * 8;
    Raw8<false> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (b0 + u < nb) r[u].template load<FAR>(p.x, base + u * 128);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (b0 + u >= nb) break;
        float v[8], m = 0.f;
        r[u].values(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = larger(m, v[i]);
        m = block_largest(m);
        const uint2 c = codes_of(v, m);
        *reinterpret_cast<uint2*>(p.codes + base + u * 128) = c;
        if (lane16 == 0) p.scales[(int64_t)(b0 + u) * p.all_rows + row] = scale_of(m);
    }
}

// ---- blocks of 128 x 128: a workgroup each, 64 values a thread (27648 x 5120 67.6 .. 76 us, 6.3 .. 5.6 TB/s) ----
__global__ void __launch_bounds__(256) square_blocks_kernel(BlockCodesArgs p) {
    __shared__ float red[4];
    const int lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4, nb = p.n / 128;
    const int64_t first = (int64_t)blockIdx.y * 128;
    const int64_t base = (first + r0) * p.n + (int64_t)blockIdx.x * 128 + lane16 * 8;
    uint4 r[8];
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        r[j] = make_uint4(0, 0, 0, 0);
        if (first + r0 + 16 * j < p.rows)
            r[j] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const i32x4_t*>(static_cast<const uint16_t*>(p.x) + base + (int64_t)16 * j * p.n)));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float v[8];
        widen8(r[j], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = larger(m, v[i]);
    }
    m = block_largest(m);
    m = larger(m, __shfl_xor(m, 16, 64));
    m = larger(m, __shfl_xor(m, 32, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    m = larger(larger(red[0], red[1]), larger(red[2], red[3]));
    if (threadIdx.x == 0) p.scales[(int64_t)blockIdx.y * nb + blockIdx.x] = scale_of(m);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (first + r0 + 16 * j >= p.rows) break;
        float v[8];
        widen8(r[j], v);
        *reinterpret_cast<uint2*>(p.codes + base + (int64_t)16 * j * p.n) = codes_of(v, m);
    }
}

// ---- the norm of a row, or of its sum with an addend ----
// TPR threads per row (of one wave or of a whole workgroup), PER chunks of 8 values each; PER = 0 (longest rows): chunk after chunk, the
// scales less the norm's factor kept where they are written until it is known.  FAR: non-temporal accesses (see launch_norm).
template <bool F32, bool ADD, int TPR, int PER, bool FAR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_blocks_kernel(BlockCodesArgs p) {
    constexpr int WAVES = TPR / 64, BLOCK = TPR < 256 ? 256 : TPR;
    static_assert(TPR == 64 || TPR >= 256, "a wave or a workgroup per row");
    const int lane = threadIdx.x % TPR, chunks = p.n / 8;
    const int row = (int)blockIdx.x * (BLOCK / TPR) + (TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0);
    if (TPR == 64 && row >= p.rows) return;   // (one wave of its own: nothing waits for it)
    const int64_t base = (int64_t)row * p.n;
    float* const scales = p.scales + row;
    float ss = 0.f;
    auto take = [&](int c, const Raw8<F32>& rx, const uint4& rd, const uint4& rw) __attribute__((always_inline)) {   // -> the block's largest s * w
        float s[8], w[8];
        rx.values(s);
        if (ADD) {
            float d[8];
            widen8(rd, d);
            Raw8<F32> kept;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += d[i];
            if (F32) {
                kept.lo = make_uint4(__float_as_uint(s[0]), __float_as_uint(s[1]), __float_as_uint(s[2]), __float_as_uint(s[3]));
                kept.hi = make_uint4(__float_as_uint(s[4]), __float_as_uint(s[5]), __float_as_uint(s[6]), __float_as_uint(s[7]));
            } else {
                kept.lo = make_uint4(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]), pack_bf16x2(s[4], s[5]), pack_bf16x2(s[6], s[7]));
                kept.values(s);   // the norm reads the stream as it is kept
            }
            if (p.sum) {
                i32x4_t* o = reinterpret_cast<i32x4_t*>(static_cast<char*>(p.sum) + (base + 8 * (int64_t)c) * (F32 ? 4 : 2));
                if constexpr (FAR) {
                    __builtin_nontemporal_store(__builtin_bit_cast(i32x4_t, kept.lo), o);
                    if (F32) __builtin_nontemporal_store(__builtin_bit_cast(i32x4_t, kept.hi), o + 1);
                } else {
                    o[0] = __builtin_bit_cast(i32x4_t, kept.lo);
                    if (F32) o[1] = __builtin_bit_cast(i32x4_t, kept.hi);
                }
            }
        } else if (p.sum) {
            i32x4_t* o = reinterpret_cast<i32x4_t*>(static_cast<char*>(p.sum) + (base + 8 * (int64_t)c) * (F32 ? 4 : 2));
            o[0] = __builtin_bit_cast(i32x4_t, rx.lo);
            if (F32) o[1] = __builtin_bit_cast(i32x4_t, rx.hi);
        }
        widen8(rw, w);
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ss = __builtin_fmaf(s[i], s[i], ss);
            s[i] *= w[i];
            m = larger(m, s[i]);
        }
        m = block_largest(m);
        const uint2 code = codes_of(s, m);
        *reinterpret_cast<uint2*>(p.codes + base + 8 * (int64_t)c) = code;
        return m;
    };
    float m[PER > 0 ? PER : 1];
    if constexpr (PER > 0) {
        Raw8<F32> rx[PER];
        uint4 rd[PER], rw[PER];
        // everything the row reads is in flight at once; a block's sixteen lanes are all inside the row or all behind it
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int c = lane + TPR * j;
            if (c >= chunks) break;
            rx[j].template load<FAR>(p.x, base + 8 * (int64_t)c);
            if (ADD) {
                Raw8<false> d;
                d.template load<FAR>(p.delta, base + 8 * (int64_t)c);
                rd[j] = d.lo;
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane + TPR * j < chunks) rw[j] = reinterpret_cast<const uint4*>(p.w)[lane + TPR * j];
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane + TPR * j < chunks) m[j] = take(lane + TPR * j, rx[j], rd[j], rw[j]);
    } else {
        for (int c = lane; c < chunks; c += TPR) {
            Raw8<F32> rx;
            uint4 rd = make_uint4(0, 0, 0, 0);
            rx.template load<false>(p.x, base + 8 * (int64_t)c);
            if (ADD) rd = reinterpret_cast<const uint4*>(p.delta)[(base + 8 * (int64_t)c) / 8];
            const float most = take(c, rx, rd, reinterpret_cast<const uint4*>(p.w)[c]);
            if (lane % 16 == 0) scales[(int64_t)(c / 16) * p.all_rows] = most;
        }
    }
    ss = wave_sum(ss);
    if constexpr (WAVES > 1) {
        __shared__ float red[WAVES];
        if (lane % 64 == 0) red[lane / 64] = ss;
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) ss += red[i];
    }
    const float inv = 1.0f / sqrtf(ss / (float)p.n + p.eps);
    if (lane % 16 != 0) return;
    if constexpr (PER > 0) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane + TPR * j < chunks) scales[(int64_t)((lane + TPR * j) / 16) * p.all_rows] = scale_of(m[j] * inv);
    } else {
        for (int c = lane; c < chunks; c += TPR) {   // (this thread's own stores)
            float* at = scales + (int64_t)(c / 16) * p.all_rows;
            *at = scale_of(*at * inv);
        }
    }
}

// Threads per row, us: as many as hold it in two or three chunks each (norm 8192 x 5120 bf16 27.9, 4 x 5120 with an addend 3.6, of which a launch is 2);
// short rows a wave each, four to a workgroup and no barrier, where they fill the chip.
// Passes over more than the last-level cache (256 MB) holds stream past it, us without and with: add + norm 8192 x 8192 bf16 85.3, 76.5; 4099 x 8192
// fp32 70.5, 72.3; below that 8192 x 5120 bf16 27.9, 29.0, add + norm 640 x 5120 fp32 9.0, 10.5.
constexpr int64_t kFarBytes = (int64_t)256 << 20;

template <bool F32, bool ADD>
hipError_t launch_norm(const BlockCodesArgs& p, hipStream_t s) {
    const int chunks = p.n / 8;
    const int64_t bytes = (int64_t)p.rows * p.n * ((F32 ? 4 : 2) * (ADD && p.sum ? 2 : 1) + (ADD ? 2 : 0) + 1);
    // A launch counts its threads in 32 bits: at most 2^31 in one.
    auto go = [&](auto kernel, int tpr) {
        const int per_block = tpr < 256 ? 256 / tpr : 1, most = (int)(((int64_t)1 << 31) / (tpr < 256 ? 64 : tpr));
        for (int at = 0; at < p.rows; at += most) {
            BlockCodesArgs q = p;
            const int64_t skip = (int64_t)at * p.n;
            auto behind = [&](const void* base, int64_t bytes) { return base ? (void*)(static_cast<const char*>(base) + bytes) : nullptr; };
            q.rows = std::min(most, p.rows - at);
            q.x = behind(p.x, skip * (F32 ? 4 : 2));
            q.delta = static_cast<const uint16_t*>(behind(p.delta, skip * 2));
            q.sum = behind(p.sum, skip * (F32 ? 4 : 2));
            q.codes += skip;
            q.scales += at;
            kernel<<<dim3((q.rows + per_block - 1) / per_block), dim3(tpr < 256 ? 256 : tpr), 0, s>>>(q);
            if (hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    };
    if (chunks <= 64) return go(norm_blocks_kernel<F32, ADD, 64, 1, false>, 64);
    if (p.rows >= 1024) {   // one workgroup of four rows per CU
        if (chunks <= 128) return go(norm_blocks_kernel<F32, ADD, 64, 2, false>, 64);
        if (chunks <= 256) return go(norm_blocks_kernel<F32, ADD, 64, 4, false>, 64);
    }
    if (chunks <= 256) return go(norm_blocks_kernel<F32, ADD, 256, 1, false>, 256);
    auto long_rows = [&](auto far) {
        constexpr bool FAR = decltype(far)::value;
        if (chunks <= 512) return go(norm_blocks_kernel<F32, ADD, 256, 2, FAR>, 256);
        if (chunks <= 768) return go(norm_blocks_kernel<F32, ADD, 256, 3, FAR>, 256);
        if (chunks <= 1024) return go(norm_blocks_kernel<F32, ADD, 512, 2, FAR>, 512);
        if (chunks <= 2048) return go(norm_blocks_kernel<F32, ADD, 512, 4, FAR>, 512);
        if (chunks <= 4096) return go(norm_blocks_kernel<F32, ADD, 1024, 4, FAR>, 1024);
        return go(norm_blocks_kernel<F32, ADD, 1024, 0, false>, 1024);
    };
    return bytes > kFarBytes ? long_rows(std::true_type{}) : long_rows(std::false_type{});
}

}  // namespace

hipError_t launch_block_codes(const void* in, int32_t rows, int32_t n, int32_t block_rows, void* codes, float* scales, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    BlockCodesArgs p{in, nullptr, nullptr, 0.0f, rows, n, rows, nullptr, static_cast<uint8_t*>(codes), scales};
    const int nb = n / 128;
    // rows_per: rows of a row of workgroups, cols: workgroups of one.  A launch counts its threads in 32 bits and rows of workgroups in 16: at most 2^31
    // threads and 32768 rows of workgroups at once.
    auto go = [&](auto kernel, int rows_per, int cols, bool cols_first) {
        const int64_t most = std::min<int64_t>(((int64_t)1 << 23) / cols, 32768) * rows_per;
        for (int64_t at = 0; at < rows; at += most) {
            BlockCodesArgs q = p;
            q.x = static_cast<const uint16_t*>(in) + at * n;
            q.rows = (int32_t)std::min<int64_t>(most, rows - at);
            q.codes = p.codes + at * n;
            q.scales = scales + (block_rows == 128 ? at / 128 * nb : at);
            const unsigned groups = (unsigned)((q.rows + rows_per - 1) / rows_per);
            kernel<<<cols_first ? dim3(cols, groups) : dim3(groups, cols), dim3(256), 0, s>>>(q);
            if (hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    };
    if (block_rows == 128) return go(square_blocks_kernel, 128, nb, true);
    // Blocks that sixteen lanes take of a row, one or four, and whether accesses stream: rows 1282 x 5120 4.9 and 5.8 us, 1282 x 13824 9.8 and 10.1
    // (12.5 streamed), 4099 x 8192 17.3 and 19.1 (25.3); 4099 x 28672, more than the cache holds, 73 (two, not streamed), 61.2 (four, streamed).
    if ((int64_t)rows * n * 3 > kFarBytes) return go(row_blocks_kernel<4, true>, 16, (nb + 3) / 4, false);
    return go(row_blocks_kernel<1, false>, 16, nb, false);
}

hipError_t launch_add_rmsnorm_f8b(const void* x, bool x_is_f32, const void* delta, const void* w, float eps, int32_t rows, int32_t n, void* sum,
                                  void* codes, float* scales, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const BlockCodesArgs p{x, static_cast<const uint16_t*>(delta), static_cast<const uint16_t*>(w), eps, rows, n, rows, sum, static_cast<uint8_t*>(codes),
                           scales};
    if (!delta) return x_is_f32 ? launch_norm<true, false>(p, s) : launch_norm<false, false>(p, s);
    return x_is_f32 ? launch_norm<true, true>(p, s) : launch_norm<false, true>(p, s);
}

}  // namespace relserve
