// Projections on 8-bit floating point codes with a scale for each block of 128:
//   out[t, n] = sum over blocks b of k of (sum over k in b of a[t, k] w[n, k]) * (a_scale[b, t] * w_scale[block of n, b])
// A block's sum is one 16 x 16 x 128 matrix instruction from zero, and its four results a lane are added to the accumulators with one fused
// multiply-add each: half as many cycles of the vector units as the matrix instruction takes, which they spend beside it.  The accumulators
// therefore lie in the vector registers, where the other projections' stay in the matrix units'.
//
// The instruction on 8-bit codes adds groups of a few neighbouring products in a window of about 14 bits below the largest of them: its sums are
// off by 1.4e-5 of their norm on normal values, 2e-5 on activations with outliers.  Beside an output rounded to bf16 (2^-9 of each value on average) that is
// nothing.  Outputs of fp32 (epilogue 1: the residual stream, logits) are to be right to fp32, so there the codes are widened to bf16, which
// holds every code, and multiplied by the 16-bit instruction, whose sums are off by 1e-8: WIDE, at half the rate.
//
// The weights are the first operand: a lane's four results are four features of one token, so a token's scale is one register of a lane and a
// weight's is the same for a wave (a wave's features lie in one block, or of a SwiGLU projection in one of gate and one of up rows).
#include <algorithm>
#include <mutex>

#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

constexpr int KB = 128;        // codes of a k step: a block, a slice of the packed weights, a row of a stage in the LDS
constexpr int NUM_XCD = 8;
constexpr int GROUP_M = 8;

enum { EPI_BF16 = 0, EPI_RES_BF16_OUT_F32 = 1, EPI_RES_F32_OUT_BF16 = 2, EPI_SWIGLU = 3, EPI_SLAB = 4 };

struct Args {
    const uint8_t* a;        // [T, K]
    const float* a_scale;    // [K / 128, T]
    const uint8_t* w;        // [N, K], or packed: [N / 256][K / 128][256][128]
    const float* w_scale;    // [blocks of rows, K / 128]
    const void* residual;
    void* out;
    float* slabs;            // partial sums [split][T, N]
    int32_t T, N, K, packed;
    int32_t n_half;          // SwiGLU: gate rows [0, n_half), up rows [n_half, 2 n_half)
    int32_t tiles_m, tiles_n;
    int32_t per_split;       // k steps of a split (EPI_SLAB)
};

__device__ __forceinline__ const char* uniform_ptr(const char* ptr) {
    const uint64_t v = reinterpret_cast<uint64_t>(ptr);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}

// 64 lanes x 16 bytes from base + the lane's offset to 1 KB of LDS at lds_addr + at; one instruction has to stand between m0's write and the load.
template <bool NT = false>
__device__ __forceinline__ void dma16(const void* base, uint32_t voff, uint32_t lds_addr, int at) {
    if (NT)
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(base), "s"(lds_addr), "i"(at) : "memory", "scc");
    else
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(lds_addr), "i"(at) : "memory", "scc");
}
// 64 lanes x 4 bytes, each from an address of its own
__device__ __forceinline__ void dma4(const float* from, uint32_t lds_addr, int at) {
    asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(lds_addr), "i"(at) : "memory", "scc");
}

// sum of a block's products: of codes, or of the same codes widened to bf16 (32 codes a lane: four products of k = 32)
struct Wide { bf16x8_t v[4]; };
__device__ __forceinline__ Wide widen(const i32x8_t& c) {
    Wide w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        bf16x2_t h[4];
        h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[2 * q], 1.0f, false);
        h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[2 * q], 1.0f, true);
        h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[2 * q + 1], 1.0f, false);
        h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[2 * q + 1], 1.0f, true);
        w.v[q] = __builtin_shufflevector(__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3), __builtin_shufflevector(h[2], h[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return w;
}
template <bool WIDE>
__device__ __forceinline__ auto operand(const i32x8_t& c) {
    if constexpr (WIDE) return widen(c);
    else return c;
}
__device__ __forceinline__ f32x4_t block_sum(const i32x8_t& w, const i32x8_t& a) { return mfma_16x16x128_f8(w, a, f32x4_t{0.f, 0.f, 0.f, 0.f}); }
__device__ __forceinline__ f32x4_t block_sum(const Wide& w, const Wide& a) {
    f32x4_t v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) v = mfma_16x16x32(w.v[q], a.v[q], v);
    return v;
}

typedef const i32x4_t __attribute__((address_space(3))) * lds_chunk;
typedef const float __attribute__((address_space(3))) * lds_float;

// Consecutive workgroups go to different XCDs: each XCD's run of tiles is made contiguous, token tiles fastest within panels of GROUP_M.
__device__ __forceinline__ int remap_xcd(int bid, int num) {
    const int per = num / NUM_XCD, rem = num % NUM_XCD, xcd = bid % NUM_XCD, idx = bid / NUM_XCD;
    return xcd < rem ? xcd * (per + 1) + idx : rem * (per + 1) + (xcd - rem) * per + idx;
}
__device__ __forceinline__ void tile_coords(int t, int tiles_m, int tiles_n, int& tile_m, int& tile_n) {
    const int panels = (tiles_m + GROUP_M - 1) / GROUP_M, base = tiles_m / panels, extra = tiles_m % panels, big = (base + 1) * tiles_n;
    int first, size, in;
    if (t < extra * big) {
        size = base + 1;
        first = t / big * size;
        in = t % big;
    } else {
        const int u = t - extra * big, per = base * tiles_n;
        size = base;
        first = extra * (base + 1) + u / per * base;
        in = u % per;
    }
    tile_m = first + in % size;
    tile_n = in / size;
}

// Row of the weights' scales that feature n's block has.
__device__ __forceinline__ int scale_row(const Args& p, bool swiglu, int n, bool up) { return (swiglu && up ? (p.n_half + KB - 1) / KB : 0) + n / KB; }

// Eight consecutive features n .. of token t (lo, hi: four each; of a SwiGLU projection g and u are the gate's and the up's) to the output.
template <int EPI>
__device__ __forceinline__ void store8(const Args& p, int t, int n, int cols, const f32x4_t& lo, const f32x4_t& hi, const f32x4_t& ulo, const f32x4_t& uhi) {
    const bool second = n + 4 < cols;
    if constexpr (EPI == EPI_SWIGLU) {   // (whole eights: n_half % 8 == 0)
        const uint4 o = make_uint4(pack_bf16x2(silu_mul(lo[0], ulo[0]), silu_mul(lo[1], ulo[1])), pack_bf16x2(silu_mul(lo[2], ulo[2]), silu_mul(lo[3], ulo[3])),
                                   pack_bf16x2(silu_mul(hi[0], uhi[0]), silu_mul(hi[1], uhi[1])), pack_bf16x2(silu_mul(hi[2], uhi[2]), silu_mul(hi[3], uhi[3])));
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + (int64_t)t * p.n_half + n) = o;
        return;
    }
    const int64_t o = (int64_t)t * p.N + n;
    if constexpr (EPI == EPI_SLAB) {
        float* to = p.slabs + o;
        *reinterpret_cast<f32x4_t*>(to) = lo;
        if (second) *reinterpret_cast<f32x4_t*>(to + 4) = hi;
    } else if constexpr (EPI == EPI_RES_BF16_OUT_F32) {
        f32x4_t a = lo, b = hi;
        if (p.residual) {
            const uint16_t* r = static_cast<const uint16_t*>(p.residual) + o;
            const uint2 x = *reinterpret_cast<const uint2*>(r);
            a += f32x4_t{bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
            if (second) {
                const uint2 y = *reinterpret_cast<const uint2*>(r + 4);
                b += f32x4_t{bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
            }
        }
        float* to = static_cast<float*>(p.out) + o;
        *reinterpret_cast<f32x4_t*>(to) = a;
        if (second) *reinterpret_cast<f32x4_t*>(to + 4) = b;
    } else {
        f32x4_t a = lo, b = hi;
        if constexpr (EPI == EPI_RES_F32_OUT_BF16) {
            const float* r = static_cast<const float*>(p.residual) + o;
            a += *reinterpret_cast<const f32x4_t*>(r);
            if (second) b += *reinterpret_cast<const f32x4_t*>(r + 4);
        }
        uint16_t* to = static_cast<uint16_t*>(p.out) + o;
        const uint2 c = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3])), d = make_uint2(pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3]));
        if (second)
            *reinterpret_cast<uint4*>(to) = make_uint4(c.x, c.y, d.x, d.y);
        else
            *reinterpret_cast<uint2*>(to) = c;
    }
}

// ---- tiles ----
// WM x WN waves over BM tokens x BN features, NS stages of a k step each.  A stage's rows are 128 bytes, chunk c of row r in slot c ^ swizzle(r),
// so that the sixteen lanes that the LDS serves together cover all banks.  Two fragments share 32 features, so that a lane has eight
// consecutive ones: lane i of fragment f reads row 32 (f / 2) + 4 (f % 2) + 8 (i / 4) + i % 4.
template <int BM, int BN, int WM, int WN, int NS, int EPI, bool WIDE>
__global__ void __launch_bounds__(64 * WM * WN) tile_kernel(Args p) {
    constexpr int NW = WM * WN, TM = BM / (16 * WM), TN = BN / (16 * WN), FEAT = BN / WN;
    constexpr int A_IT = BM / (8 * NW), W_IT = BN / (8 * NW), LOADS = A_IT + W_IT + 1;
    constexpr int A_BYTES = BM * KB, W_BYTES = BN * KB, S_BYTES = (BM / 64 + 1) * 256, STAGE = A_BYTES + W_BYTES + S_BYTES;
    constexpr bool SWI = EPI == EPI_SWIGLU;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM / 64 < NW, "whole wave loads, a wave left for the weights' scales");
    static_assert(TN % (SWI ? 4 : 2) == 0 && FEAT <= 128, "pairs of fragments, features of one block");
    static_assert(NS * LOADS < 64, "vmcnt field");
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;

    const int n_tiles = p.tiles_m * p.tiles_n;
    const int split = EPI == EPI_SLAB ? blockIdx.x / n_tiles : 0;
    int tile_m, tile_n;
    tile_coords(remap_xcd(EPI == EPI_SLAB ? blockIdx.x % n_tiles : blockIdx.x, n_tiles), p.tiles_m, p.tiles_n, tile_m, tile_n);
    const int t0 = tile_m * BM, n0 = tile_n * (SWI ? BN / 2 : BN);
    const int cols = SWI ? p.n_half : p.N, nkb = p.K / KB;
    const int kbeg = EPI == EPI_SLAB ? split * p.per_split : 0, nk = EPI == EPI_SLAB ? min(p.per_split, nkb - kbeg) : nkb;

    // what a lane loads: slot lane % 8 of row lane / 8 of each wave load; rows past the end of a matrix are its last one again, never stored
    const int lrow = lane >> 3, r0 = wave * 8 + lrow;
    uint32_t a_off[A_IT], w_off[W_IT];
#pragma unroll
    for (int j = 0; j < A_IT; ++j) {
        const int r = NW * 8 * j + r0;
        a_off[j] = (uint32_t)min(t0 + r, p.T - 1) * (uint32_t)p.K + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
    }
    auto w_swz = [](int r) { return ((r >> 1) & 1) | ((r >> 2) & 6); };
#pragma unroll
    for (int j = 0; j < W_IT; ++j) {
        const int r = NW * 8 * j + r0;
        uint32_t n;
        if (SWI) n = (uint32_t)min(n0 + r % (BN / 2), p.n_half - 1) + (r >= BN / 2 ? p.n_half : 0);
        else n = (uint32_t)min(n0 + r, p.N - 1);
        w_off[j] = (p.packed ? (n >> 8) * (uint32_t)p.K * 256u + (n & 255) * 128u : n * (uint32_t)p.K) + (((lane & 7) ^ w_swz(r)) << 4);
    }
    // scales: the first waves' 64 tokens each, the others two rows of the weights' (two blocks, or the gate's and the up's)
    const float* s_from;
    int64_t s_step;
    if (wave < BM / 64) {
        s_from = p.a_scale + (int64_t)kbeg * p.T + min(t0 + wave * 64 + lane, p.T - 1);
        s_step = p.T;
    } else {
        const int row = SWI ? scale_row(p, true, n0, lane & 1) : min(n0 / KB + (lane & 1), (p.N - 1) / KB);
        s_from = p.w_scale + (int64_t)row * nkb + kbeg;
        s_step = 1;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const uint32_t lds_a = __builtin_amdgcn_readfirstlane(lds0 + wave * 1024), lds_s = __builtin_amdgcn_readfirstlane(lds0 + A_BYTES + W_BYTES + min(wave, BM / 64) * 256);
    const int w_step = p.packed ? 256 * KB : KB;
    const char* ab = uniform_ptr(reinterpret_cast<const char*>(p.a) + (int64_t)kbeg * KB);
    const char* wb = uniform_ptr(reinterpret_cast<const char*>(p.w) + (int64_t)kbeg * w_step);
    auto load = [&](int stage) __attribute__((always_inline)) {   // the next k step to load
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_a + stage * STAGE), to_s = __builtin_amdgcn_readfirstlane(lds_s + stage * STAGE);
#pragma unroll
        for (int j = 0; j < W_IT; ++j) dma16(wb, w_off[j], to, A_BYTES + j * (NW * 1024));
        dma4(s_from, to_s, 0);
#pragma unroll
        for (int j = 0; j < A_IT; ++j) dma16(ab, a_off[j], to, j * (NW * 1024));
        wb += w_step;
        ab += KB;
        s_from += s_step;
    };

    // operands in the LDS: chunks g and g + 4 of a row; which codes meet which is the same for both
    const uint32_t a_at = lds0 + (wm * (BM / WM) + l16) * KB + ((g ^ ((l16 >> 1) & 7)) << 4);
    const int wr = 8 * (l16 >> 2) + (l16 & 3);
    const uint32_t w_at = lds0 + A_BYTES + (wn * (SWI ? FEAT / 2 : FEAT) + wr) * KB + ((g ^ w_swz(wr)) << 4);
    const uint32_t ts_at = lds0 + A_BYTES + W_BYTES + (wm * (BM / WM) + l16) * 4;
    const uint32_t ws_at = lds0 + A_BYTES + W_BYTES + (BM / 64) * 256 + (SWI ? 0 : wn * FEAT / KB * 4);
    auto w_dist = [](int f) {   // of fragment f (SwiGLU: the second half are the up rows)
        const int up = SWI && f >= TN / 2 ? 1 : 0, i = f - up * (TN / 2);
        return (up * (BN / 2) + 32 * (i >> 1) + 4 * (i & 1)) * KB;
    };
    auto read = [](uint32_t at) __attribute__((always_inline)) {
        const i32x4_t lo = *(lds_chunk)(uintptr_t)at, hi = *(lds_chunk)(uintptr_t)(at ^ 64);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f32x4_t acc[TN][TM];
#pragma unroll
    for (int f = 0; f < TN; ++f)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[f][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

#pragma unroll
    for (int s = 0; s < NS - 1; ++s)
        if (s < nk) load(s);
    int stage = 0;
    for (int k = 0; k < nk; ++k) {
        if (k + NS - 1 <= nk) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (k + NS - 1 < nk) load(stage == 0 ? NS - 1 : stage - 1);
        const uint32_t off = stage * STAGE;
        using operand_t = decltype(operand<WIDE>(i32x8_t{}));
        operand_t af[TM];
        float ts[TM], us[SWI ? TM : 1];
        const float ws = *(lds_float)(uintptr_t)(ws_at + off), wu = SWI ? *(lds_float)(uintptr_t)(ws_at + 4 + off) : 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const float s = *(lds_float)(uintptr_t)(ts_at + off + 64 * i);
            af[i] = operand<WIDE>(read(a_at + off + 16 * KB * i));
            ts[i] = s * ws;
            if (SWI) us[i] = s * wu;
        }
#pragma unroll
        for (int f = 0; f < TN; ++f) {
            const operand_t wf = operand<WIDE>(read(w_at + off + w_dist(f)));
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const f32x4_t v = block_sum(wf, af[i]);
                const float s = SWI && f >= TN / 2 ? us[SWI ? i : 0] : ts[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[f][i][r] = __builtin_fmaf(v[r], s, acc[f][i][r]);
            }
        }
        stage = stage + 1 == NS ? 0 : stage + 1;
    }

    if (EPI == EPI_SLAB) p.slabs += (int64_t)split * p.T * p.N;
    const f32x4_t none{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int t = t0 + wm * (BM / WM) + 16 * i + l16;
        if (t >= p.T) continue;
#pragma unroll
        for (int f = 0; f < (SWI ? TN / 2 : TN); f += 2) {
            const int n = n0 + wn * (SWI ? FEAT / 2 : FEAT) + 16 * f + 8 * g;
            if (n >= cols) continue;
            if constexpr (SWI) store8<EPI>(p, t, n, cols, acc[f][i], acc[f + 1][i], acc[f + TN / 2][i], acc[f + 1 + TN / 2][i]);
            else store8<EPI>(p, t, n, cols, acc[f][i], acc[f + 1][i], none, none);
        }
    }
}

template <int BM, int BN, int WM, int WN, int NS, int EPI, bool WIDE>
hipError_t launch_tiles(Args p, int splits, hipStream_t s) {
    constexpr int smem = NS * ((BM + BN) * KB + (BM / 64 + 1) * 256);
    static_assert(smem <= 160 * 1024, "stages exceed the LDS");
    p.tiles_m = (p.T + BM - 1) / BM;
    p.tiles_n = EPI == EPI_SWIGLU ? (p.n_half + BN / 2 - 1) / (BN / 2) : (p.N + BN - 1) / BN;
    static std::once_flag once;
    static hipError_t st = hipSuccess;
    auto kernel = &tile_kernel<BM, BN, WM, WN, NS, EPI, WIDE>;
    std::call_once(once, [&] { st = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, smem); });
    if (st != hipSuccess) return st;
    kernel<<<dim3((unsigned)(p.tiles_m * p.tiles_n * splits)), dim3(64 * WM * WN), smem, s>>>(p);
    return hipGetLastError();
}

template <int EPI>
hipError_t run(const Args& p, hipStream_t s) {
    constexpr bool WIDE = EPI == EPI_RES_BF16_OUT_F32;
    if (p.T <= 128) return launch_tiles<128, 128, 2, 2, 2, EPI, WIDE>(p, 1, s);
    if constexpr (WIDE) return launch_tiles<128, 256, 2, 4, 3, EPI, WIDE>(p, 1, s);
    else return launch_tiles<256, 256, 4, 2, 2, EPI, WIDE>(p, 1, s);
}

}  // namespace

int64_t gemm_f8b_scratch_floats(int64_t T, int64_t N) { (void)T; (void)N; return 64; }

hipError_t launch_linear_f8b(const void* a, const float* a_scale, const void* w, const float* w_scale, int32_t T, int32_t N, int32_t K,
                             int32_t epilogue, const void* residual, void* out, hipStream_t s, float* scratch, bool w_packed) {
    if (T == 0) return hipSuccess;
    Args p{static_cast<const uint8_t*>(a), a_scale, static_cast<const uint8_t*>(w), w_scale, residual, out, scratch, T, N, K, w_packed, N / 2, 0, 0, 0};
    switch (epilogue) {
        case EPI_BF16: return run<EPI_BF16>(p, s);
        case EPI_RES_BF16_OUT_F32: return run<EPI_RES_BF16_OUT_F32>(p, s);
        case EPI_RES_F32_OUT_BF16: return run<EPI_RES_F32_OUT_BF16>(p, s);
        case EPI_SWIGLU: return run<EPI_SWIGLU>(p, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace relserve
