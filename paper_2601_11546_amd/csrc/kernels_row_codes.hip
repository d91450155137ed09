// Rows as 8-bit integers with one scale per row: what an int8 projection multiplies.
//   scale[t] = m / 127, m the row's largest magnitude;   code[t, i] = rint(value[t, i] * 127 / m)
// of the rows of a bf16 matrix, or of rmsnorm(x + delta) * w, whose sum with the addend is kept on the way.
//
// The norm's factor 1 / rms is the same for the whole row, so it cancels in value * 127 / m: the codes come from s * w alone, and the sum of
// squares, which is done with the largest magnitude in one reduction, goes into the scale only.
// Memory bound: every byte once.  A row's values stay in registers between the reduction and the codes.
#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

struct RowCodesArgs {
    const void* x;           // [rows, n] bf16 or fp32
    const uint16_t* delta;   // [rows, n] bf16 or null
    const uint16_t* w;       // [n] bf16, the norm's weights
    float eps;
    int32_t rows, n;
    void* sum;               // [rows, n] x + delta in x's type, or null
    uint8_t* codes;
    float* scales;
};

// 8 values as they are loaded
template <bool F32>
struct Raw8 {
    uint4 lo, hi;   // hi: fp32 only
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
        lo = p[0];
        if (F32) hi = p[1];
    }
    __device__ __forceinline__ void load_far(const void* base, int64_t at) {
        const i32x4_t* p = reinterpret_cast<const i32x4_t*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
        lo = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p));
        if (F32) hi = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p + 1));
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if (F32) {
            v[0] = __uint_as_float(lo.x); v[1] = __uint_as_float(lo.y); v[2] = __uint_as_float(lo.z); v[3] = __uint_as_float(lo.w);
            v[4] = __uint_as_float(hi.x); v[5] = __uint_as_float(hi.y); v[6] = __uint_as_float(hi.z); v[7] = __uint_as_float(hi.w);
        } else {
            v[0] = bf16_lo(lo.x); v[1] = bf16_hi(lo.x); v[2] = bf16_lo(lo.y); v[3] = bf16_hi(lo.y);
            v[4] = bf16_lo(lo.z); v[5] = bf16_hi(lo.z); v[6] = bf16_lo(lo.w); v[7] = bf16_hi(lo.w);
        }
    }
};

// The larger magnitude, a NaN if either is one.
__device__ __forceinline__ float larger(float m, float v) { return __builtin_elementwise_maximum(m, __builtin_fabsf(v)); }

enum { ROWS_PLAIN = 0, ROWS_NORM = 1, ROWS_ADD_NORM = 2 };   // what the codes are of: the row, its norm, the norm of its sum with the addend

// TPR threads per row (of one wave or of a whole workgroup), PER chunks of 8 values each, held in registers; PER = 0 (longest rows): chunk
// after chunk, read again for the codes.  FAR: non-temporal accesses (see launch_rows; template arguments, since the compiler merges the two
// sides of a branch between them into plain ones).
template <bool F32, int OP, int TPR, int PER, bool FAR = false>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) row_codes_kernel(RowCodesArgs p) {
    constexpr int WAVES = TPR / 64, BLOCK = TPR < 256 ? 256 : TPR;
    static_assert(TPR == 64 || TPR >= 256, "a wave or a workgroup per row");
    const int lane = threadIdx.x % TPR, chunks = p.n / 8;
    const int row = (int)blockIdx.x * (BLOCK / TPR) + (TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0);
    if (TPR == 64 && row >= p.rows) return;   // (one wave of its own: nothing waits for it)
    const int64_t base = (int64_t)row * p.n;
    // values of chunk c whose codes are taken, less the norm's factor; the stream is kept as it is normed
    float ss = 0.f, m = 0.f;
    auto first = [&](int c, const Raw8<F32>& rx, const Raw8<false>& rd, const Raw8<false>& rw, bool mine, float (&v)[8]) {
        float s[8];
        rx.values(s);
        Raw8<F32> kept = rx;
        if (OP == ROWS_ADD_NORM) {
            float d[8];
            rd.values(d);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += d[i];
            if (F32) {
                kept.lo = make_uint4(__float_as_uint(s[0]), __float_as_uint(s[1]), __float_as_uint(s[2]), __float_as_uint(s[3]));
                kept.hi = make_uint4(__float_as_uint(s[4]), __float_as_uint(s[5]), __float_as_uint(s[6]), __float_as_uint(s[7]));
            } else {
                kept.lo = make_uint4(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]), pack_bf16x2(s[4], s[5]), pack_bf16x2(s[6], s[7]));
                kept.values(s);
            }
        }
        if (OP != ROWS_PLAIN && p.sum && mine) {
            i32x4_t* o = reinterpret_cast<i32x4_t*>(static_cast<char*>(p.sum) + (base + 8 * (int64_t)c) * (F32 ? 4 : 2));
            if constexpr (FAR) {
                __builtin_nontemporal_store(__builtin_bit_cast(i32x4_t, kept.lo), o);
                if (F32) __builtin_nontemporal_store(__builtin_bit_cast(i32x4_t, kept.hi), o + 1);
            } else {
                o[0] = __builtin_bit_cast(i32x4_t, kept.lo);
                if (F32) o[1] = __builtin_bit_cast(i32x4_t, kept.hi);
            }
        }
        if (OP == ROWS_PLAIN) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s[i];
        } else {
            float w[8];
            rw.values(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s[i] * w[i];
            if (mine) {   // a chunk past the end is the last one again, which would be counted twice
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(s[i], s[i], ss);
            }
        }
        if (OP != ROWS_ADD_NORM || mine) {   // (a sum in place may have reached that chunk before this read of it)
#pragma unroll
            for (int i = 0; i < 8; ++i) m = larger(m, v[i]);
        }
    };
    float v[PER > 0 ? PER : 1][8];
    if constexpr (PER > 0) {
        Raw8<F32> rx[PER];
        Raw8<false> rd[OP == ROWS_ADD_NORM ? PER : 1], rw[OP != ROWS_PLAIN ? PER : 1];
        // everything the row reads is in flight at once
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int64_t at = base + 8 * (int64_t)min(lane + TPR * j, chunks - 1);
            if constexpr (FAR) {
                rx[j].load_far(p.x, at);
                if (OP == ROWS_ADD_NORM) rd[j].load_far(p.delta, at);
            } else {
                rx[j].load(p.x, at);
                if (OP == ROWS_ADD_NORM) rd[j].load(p.delta, at);
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (OP != ROWS_PLAIN) rw[j].load(p.w, 8 * (int64_t)min(lane + TPR * j, chunks - 1));
#pragma unroll
        for (int j = 0; j < PER; ++j) first(lane + TPR * j, rx[j], rd[OP == ROWS_ADD_NORM ? j : 0], rw[OP != ROWS_PLAIN ? j : 0], lane + TPR * j < chunks, v[j]);
    } else {
        for (int c = lane; c < chunks; c += TPR) {
            Raw8<F32> rx;
            Raw8<false> rd, rw;
            rx.load(p.x, base + 8 * (int64_t)c);
            if (OP == ROWS_ADD_NORM) rd.load(p.delta, base + 8 * (int64_t)c);
            if (OP != ROWS_PLAIN) rw.load(p.w, 8 * (int64_t)c);
            first(c, rx, rd, rw, true, v[0]);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        if (OP != ROWS_PLAIN) ss += __shfl_xor(ss, o, 64);
        m = larger(m, __shfl_xor(m, o, 64));
    }
    if constexpr (WAVES > 1) {
        __shared__ float2 red[WAVES];
        if (lane % 64 == 0) red[lane / 64] = make_float2(ss, m);
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float2 r = red[i];
            ss += r.x;
            m = larger(m, r.y);
        }
    }
    const float inv = OP != ROWS_PLAIN ? 1.0f / sqrtf(ss / (float)p.n + p.eps) : 1.0f;
    if (lane == 0) p.scales[row] = m * inv / 127.0f;
    // Nothing to scale by (0, infinite, NaN): codes of 0.  127 / m overflows for the smallest magnitudes, and what it lacks is no normal
    // number for the largest: such rows are moved by a power of two first.
    const bool some = m > 0.0f && m < INFINITY;
    const float move = m < 0x1p-100f ? 0x1p100f : m > 0x1p60f ? 0x1p-100f : 1.0f, top = m * move;
    // The quotient from 127 / m and from what that lacks: its product alone would put quotients of an integer and a half (in bf16 rows every
    // |v| = m / 2 is 63.5) on either side.  It is rounded to 24 bits once, from within 2^-45 of its value, and no other quotient of two bf16
    // values, or of two products of such, is near enough to an integer and a half to become one by that.  (Two instructions a value more than
    // the product alone, us: rows 4099 x 28672 56.4 -> 56.9, 60 x 53248 5.7 -> 6.3; add + norm 8192 x 8192 71.0 -> 71.1, norm 4096 x 1024 3.8 -> 3.9.)
    const float per = some ? 127.0f / top : 0.0f, lack = __builtin_fmaf(-per, top, 127.0f) * (per * (1.0f / 127.0f));
    // quotient + 1.5 * 2^23 is the nearest integer, ties to even, and its low byte the code
    auto codes = [&](int c, float (&u)[8]) {
        uint32_t o[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = u[4 * h + i];
                if (move != 1.0f) v *= move;
                b[i] = __float_as_uint(__builtin_fmaf(v, per, v * lack) + 12582912.0f);
            }
            const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
            o[h] = some ? lo | hi : 0u;
        }
        uint64_t* at = reinterpret_cast<uint64_t*>(p.codes + base + 8 * (int64_t)c);
        const uint64_t bits = (uint64_t)o[1] << 32 | o[0];
        if constexpr (FAR && OP != ROWS_ADD_NORM) __builtin_nontemporal_store(bits, at);
        else *at = bits;
    };
    if constexpr (PER > 0) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane + TPR * j < chunks) codes(lane + TPR * j, v[j]);
    } else {
        const void* stream = OP == ROWS_ADD_NORM && p.sum ? p.sum : p.x;   // (x may have become the sum; this thread's own stores)
        for (int c = lane; c < chunks; c += TPR) {
            Raw8<F32> rx;
            Raw8<false> rd, rw;
            rx.load(stream, base + 8 * (int64_t)c);
            float s[8];
            rx.values(s);
            if (OP == ROWS_ADD_NORM && !p.sum) {
                rd.load(p.delta, base + 8 * (int64_t)c);
                float d[8];
                rd.values(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[i] += d[i];
                    if (!F32) s[i] = bf16_to_f32((uint16_t)f32_to_bf16_bits(s[i]));
                }
            }
            if (OP != ROWS_PLAIN) {
                rw.load(p.w, 8 * (int64_t)c);
                float w[8];
                rw.values(w);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] *= w[i];
            }
            codes(c, s);
        }
    }
}

// Threads per row.  A row's chunks go to as few threads as hold them in three registers' worth each (more threads: more of them idle at the
// end of a row; more chunks a thread: a longer chain of conversions per wave), us, here and below with codes of two instructions less than now (above):
//   rmsnorm 8192 x 5120 bf16     256 x 3: 23.2   64 x 10: 25.4   512 x 2: 27.5   1024 x 1: 37.7
//   add + norm 8192 x 8192       512 x 2: 80.5   256 x 4: 83.2   1024 x 1: 82.3
//   rows 1282 x 13824            512 x 4: 9.1    256 x 7: 8.9    1024 x 2: 9.1;    4099 x 28672   1024 x 4: 62.1   512 x 7: 63.2   read twice: 96
// Short rows take a wave each, without a barrier, four to a workgroup: norm 4096 x 1024 3.7 (a workgroup each 5.2), 4096 x 2048 6.6 (7.4); where
// those do not fill the chip the workgroup's shorter chain counts.  Four rows of 5120 take 2.8 us, of which a launch is 2.
//
// Passes over more than the last-level cache (256 MB) holds stream: loads, and stores of the sum, or where there is none of the codes.
// Add + norm 8192 x 8192 (470 MB) 80.7 -> 69.9 us (6.7 TB/s; loads alone 79.2, the sum alone 80.6, the codes too 77.4), rows 4099 x 28672 (350 MB)
// 62.8 -> 55.3 (6.4 TB/s; loads alone 58.8).  Smaller passes would lose what the cache still has of their input: norm 1282 x 5120 fp32 6.9 -> 8.8.
constexpr int64_t kFarBytes = (int64_t)256 << 20;

template <bool F32, int OP>
hipError_t launch_rows(const RowCodesArgs& p, hipStream_t s) {
    const int chunks = p.n / 8;
    const int64_t bytes = (int64_t)p.rows * p.n * ((F32 ? 4 : 2) * (OP == ROWS_ADD_NORM && p.sum ? 2 : 1) + (OP == ROWS_ADD_NORM ? 2 : 0) + 1);
    // A launch counts its threads in 32 bits, and one of more (2^26 + 5 rows of 8 values) leaves rows out without an error: at most 2^31 in one.
    auto go = [&](auto kernel, int tpr) {
        const int per_block = tpr < 256 ? 256 / tpr : 1, most = (int)(((int64_t)1 << 31) / tpr);
        auto behind = [&](const void* base, int64_t bytes) { return base ? (void*)(static_cast<const char*>(base) + bytes) : nullptr; };
        for (int at = 0; at < p.rows; at += most) {
            RowCodesArgs q = p;
            const int64_t skip = (int64_t)at * p.n;
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
    if (chunks <= 64) return go(row_codes_kernel<F32, OP, 64, 1>, 64);
    if (p.rows >= 1024) {   // one workgroup of four rows per CU
        if (chunks <= 128) return go(row_codes_kernel<F32, OP, 64, 2>, 64);
        if (chunks <= 192) return go(row_codes_kernel<F32, OP, 64, 3>, 64);
        if (chunks <= 256) return go(row_codes_kernel<F32, OP, 64, 4>, 64);
    }
    if (chunks <= 256) return go(row_codes_kernel<F32, OP, 256, 1>, 256);
    auto long_rows = [&](auto far) {
        constexpr bool FAR = decltype(far)::value;
        if (chunks <= 512) return go(row_codes_kernel<F32, OP, 256, 2, FAR>, 256);
        if (chunks <= 768) return go(row_codes_kernel<F32, OP, 256, 3, FAR>, 256);
        if (chunks <= 1024) return go(row_codes_kernel<F32, OP, 512, 2, FAR>, 512);
        if (chunks <= 1536) return go(row_codes_kernel<F32, OP, 512, 3, FAR>, 512);
        if (chunks <= 2048) return go(row_codes_kernel<F32, OP, 512, 4, FAR>, 512);
        if (chunks <= 3072) return go(row_codes_kernel<F32, OP, 1024, 3, FAR>, 1024);
        if (chunks <= 4096) return go(row_codes_kernel<F32, OP, 1024, 4, FAR>, 1024);
        return go(row_codes_kernel<F32, OP, 1024, 0>, 1024);
    };
    return bytes > kFarBytes ? long_rows(std::true_type{}) : long_rows(std::false_type{});
}

}  // namespace

hipError_t launch_row_codes(const void* x, bool x_is_f32, const void* delta, const void* w, float eps, int32_t rows, int32_t n, void* sum,
                            void* codes, float* scales, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const RowCodesArgs p{x, static_cast<const uint16_t*>(delta), static_cast<const uint16_t*>(w), eps, rows, n, sum, static_cast<uint8_t*>(codes), scales};
    if (!w) return launch_rows<false, ROWS_PLAIN>(p, s);
    if (!delta) return x_is_f32 ? launch_rows<true, ROWS_NORM>(p, s) : launch_rows<false, ROWS_NORM>(p, s);
    return x_is_f32 ? launch_rows<true, ROWS_ADD_NORM>(p, s) : launch_rows<false, ROWS_ADD_NORM>(p, s);
}

}  // namespace relserve
