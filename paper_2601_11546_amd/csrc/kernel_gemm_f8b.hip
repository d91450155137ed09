// Projections on 8-bit floating point codes with a scale for each block of 128:
//   out[t, n] = sum over blocks b of k of (sum over k in b of a[t, k] w[n, k]) * (a_scale[b, t] * w_scale[block of n, b])
// A block's sum is one 16 x 16 x 128 matrix instruction from zero, and its four results a lane are added to the accumulators with one fused
// multiply-add each: half as many cycles of the vector units as the matrix instruction takes, which they spend beside it.  The accumulators
// therefore lie in the vector registers, where the other projections' stay in the matrix units'.
//
// The instruction on 8-bit codes takes the products of eight consecutive k together and cuts each one off, towards zero, at 2^-13 of 2^E, E the largest
// sum of two exponents among them (a subnormal code's is -6).  Products have three bits of mantissa a factor, so only those 2^7 below the largest lose any:
// sums are off by 1.4e-5 of their norm on normal values, 2.1e-5 with channels eight times as large, 6e-5 on magnitudes spread over orders, at most 7 / 2^13 of a
// group's largest product.  Outputs are rounded to bf16 behind it (1.65e-3 of the norm): their distance to 64-bit sums stays the same in three digits, and one
// in a hundred is the neighbouring number.  Outputs of fp32 (epilogue 1: the residual stream, logits) are to be right to fp32, so there the codes are widened
// to bf16, which holds every code, and multiplied by the 16-bit instruction, whose products are exact: WIDE, at half the rate, off by fp32's
// roundings (4e-8 of the norm at one block, 1.2e-7 at 108).
//
// The weights are the first operand: a lane's four results are four features of one token, so a token's scale is one register of a lane and a
// weight's is the same for a wave (a wave's features lie in one block, or of a SwiGLU projection in one of gate and one of up rows).
#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "device_utils.h"
#include "gemm_tiles.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

constexpr int KB = 128;        // codes of a k step: a block, a slice of the packed weights, a row of a stage in the LDS

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

// As dma16, 64 lanes x 4 bytes
__device__ __forceinline__ void dma4(const void* base, uint32_t voff, uint32_t lds_addr, int at) {
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(base), "s"(lds_addr), "i"(at) : "memory", "scc");
}
// the same, each from an address of its own
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
        // rows of N % 8 = 4 outputs: every other one begins 8 bytes further (as a uint4 it is also taken apart into four stores: 1282 x 15360 x 5120 114 us, 124)
        typedef uint32_t u32_quad __attribute__((ext_vector_type(4), aligned(8)));
        if (second)
            *reinterpret_cast<u32_quad*>(to) = u32_quad{c.x, c.y, d.x, d.y};
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
    const char* rf_s;
    uint32_t s_off;
    int64_t s_step;
    if (wave < BM / 64) {
        rf_s = uniform_ptr(reinterpret_cast<const char*>(p.a_scale + (int64_t)kbeg * p.T));
        s_off = (uint32_t)min(t0 + wave * 64 + lane, p.T - 1) * 4;
        s_step = (int64_t)p.T * 4;
    } else {
        const int row = SWI ? scale_row(p, true, n0, lane & 1) : min(n0 / KB + (lane & 1), (p.N - 1) / KB);
        rf_s = uniform_ptr(reinterpret_cast<const char*>(p.w_scale + kbeg));
        s_off = (uint32_t)row * (uint32_t)nkb * 4;
        s_step = 4;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const uint32_t lds_a = __builtin_amdgcn_readfirstlane(lds0 + wave * 1024), lds_s = __builtin_amdgcn_readfirstlane(lds0 + A_BYTES + W_BYTES + min(wave, BM / 64) * 256);
    const int w_step = p.packed ? 256 * KB : KB;
    const char* const ab = uniform_ptr(reinterpret_cast<const char*>(p.a) + (int64_t)kbeg * KB);
    const char* const wb = uniform_ptr(reinterpret_cast<const char*>(p.w) + (int64_t)kbeg * w_step);
    // the d-th of a stage's loads, of the step that rf_* stand at: weights first, which come from further away
    const char *rf_a = ab, *rf_w = wb;
    uint32_t to = 0;   // the stage's place
    auto load = [&](int d) __attribute__((always_inline)) {
        if (d < W_IT) dma16(rf_w, w_off[d], __builtin_amdgcn_readfirstlane(lds_a + to), A_BYTES + d * (NW * 1024));
        else if (d == W_IT) dma4(rf_s, s_off, __builtin_amdgcn_readfirstlane(lds_s + to), 0);
        else dma16(rf_a, a_off[d - W_IT - 1], __builtin_amdgcn_readfirstlane(lds_a + to), (d - W_IT - 1) * (NW * 1024));
    };
    auto next_step = [&]() __attribute__((always_inline)) { rf_w += w_step, rf_a += KB, rf_s += s_step; };

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
    struct At { uint32_t lo, hi; };
    auto read = [](At at, int dist) __attribute__((always_inline)) {
        const i32x4_t lo = *(lds_chunk)(uintptr_t)(at.lo + dist), hi = *(lds_chunk)(uintptr_t)(at.hi + dist);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    // One k step, issued in a fixed order: product j, then what is read and loaded and added behind it.  Fragments of features one after the other
    // against all tokens, the last two side by side token by token, so that a token's operand is free for the next step's behind its last pair.  The
    // stage's last operands are in registers ahead of that pair: there the wave waits for the next stage and hands this one over, reads the next
    // step's first operands beside the last products and refills the stage beside the next step's.  A product's results are added two products
    // later, those of a step's last two beside the next step's first.
    constexpr int NM = TN * TM, HAND = NM - 2 * TM, LAG = 2, NB = WIDE ? 2 : TN == 8 ? 3 : TN;
    static_assert(NM % 4 == 0 && (TN == 4 || TN == 8) && LAG <= TM, "a ring of four results, products for all tokens' scales behind the hand-over");
    constexpr auto frag_of = [](int j) { return j < HAND ? j / TM : TN - 2 + (j - HAND) % 2; };
    constexpr auto token_of = [](int j) { return j < HAND ? j % TM : (j - HAND) / 2; };
    // registers of fragment f: the last two and the first one of the next step are held together, and neighbours
    constexpr auto buffer_of = [](int f) { constexpr int of8[8] = {2, 0, 1, 0, 1, 2, 0, 1}; return WIDE ? f / 3 : TN == 8 ? of8[f] : f; };
    // Widening: the 16 conversions of a fragment behind one product, those of the next a product or two later, once the registers they go to are free and
    // BEHIND products after the fragment's read (all of them ahead of their first products: 2000 x 8192 x 8192 243 us, so 239; none at all, in a
    // build that leaves them out, 20 % less).  wide_of: fragment f's registers.
    static_assert(!WIDE || TN == 4, "widened fragments of features");
    constexpr int BEHIND = TM > 2 ? 2 : 1, NA = WIDE ? 2 : TM;
    constexpr auto wide_of = [](int f) { return f < 3 ? f : 1; };
    using operand_t = decltype(operand<WIDE>(i32x8_t{}));
    f32x4_t acc[TN][TM], sum[4];
#pragma unroll
    for (int f = 0; f < TN; ++f)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[f][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    i32x8_t w_raw[NB], a_raw[NA];          // as read
    operand_t wf[WIDE ? 3 : 1], af[WIDE ? TM : 1];   // widened
    float ts[TM], tn[TM], wn0 = 0.f, wn1 = 0.f;   // tokens' scales times the weights' of the features in turn; the tokens' and the weights' as read
#pragma unroll
    for (int i = 0; i < TM; ++i) ts[i] = tn[i] = 0.f;
    auto add = [&](int j) __attribute__((always_inline)) {
        const int f = frag_of(j), i = token_of(j);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[f][i][r] = __builtin_fmaf(sum[j % 4][r], ts[i], acc[f][i][r]);
    };
    // The loads of a refill: one behind every GAP-th product from the hand-over on.
    constexpr int GAP = NM / LOADS >= 2 ? 2 : 1;
    static_assert((LOADS - 1) * GAP < NM, "a refill is issued before the next hand-over");
    uint32_t cur = 0;   // the stage that is computed
    // What a step does of refills (REST: issues what is left of the one begun at the last hand-over, BEGIN: begins one at its own) and waits for.
    auto step = [&](auto rest, auto begin) __attribute__((always_inline)) {
        constexpr bool REST = decltype(rest)::value, BEGIN = decltype(begin)::value;
        const uint32_t next = cur + STAGE == NS * STAGE ? 0 : cur + STAGE;
        At wa{w_at + cur, (w_at ^ 64) + cur}, na{0, 0};
        asm("" : "+v"(wa.lo), "+v"(wa.hi));
#pragma unroll
        for (int j = 0; j < NM; ++j) {
            const int f = frag_of(j), i = token_of(j);
            __builtin_amdgcn_sched_barrier(0);
            if (j == HAND) {   // (stages behind the next one stay on their way)
                if (BEGIN) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * LOADS) : "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __syncthreads();
                next_step();
                to = cur;
            }
            const int since = j >= HAND ? j - HAND : j - HAND + NM;
            if ((j >= HAND ? BEGIN : REST) && since % GAP == 0 && since / GAP < LOADS) load(since / GAP);
            if constexpr (WIDE) {
                sum[j % 4] = block_sum(wf[wide_of(f)], af[i]);
            } else {
                sum[j % 4] = block_sum(w_raw[buffer_of(f)], a_raw[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (WIDE) {
                if (j == TM - (TM > 2 ? 2 : 1)) wf[1] = operand<WIDE>(w_raw[buffer_of(1)]);
                if (j == TM + BEHIND) wf[2] = operand<WIDE>(w_raw[buffer_of(2)]);
                if (j == HAND) wf[1] = operand<WIDE>(w_raw[buffer_of(3)]);
                if (j == HAND + 2) wf[0] = operand<WIDE>(w_raw[buffer_of(0)]);   // the next step's
#pragma unroll
                for (int q = 0; q < TM; ++q)
                    if (j == (HAND + 2 * q + 1 + BEHIND) % NM) af[q] = operand<WIDE>(a_raw[q % NA]);
            }
            if (j < HAND) {   // the next fragment of features; behind the last but two both that remain
                if (i == 0) w_raw[buffer_of(f + 1)] = read(wa, w_dist(f + 1));
                if (f == TN - 3 && i == TM / 2) w_raw[buffer_of(TN - 1)] = read(wa, w_dist(TN - 1));
            } else {
                if (j == HAND) {
                    na = At{a_at + next, (a_at ^ 64) + next};
                    asm("" : "+v"(na.lo), "+v"(na.hi));
                    w_raw[buffer_of(0)] = read(At{w_at + next, (w_at ^ 64) + next}, 0);
                }
                if ((j - HAND) % 2) a_raw[i % NA] = read(na, 16 * KB * i);
            }
            if (j == LAG || (SWI && j == TN / 2 * TM + LAG)) {
#pragma unroll
                for (int q = 0; q < TM; ++q) ts[q] = tn[q] * (j == LAG ? wn0 : wn1);
            }
            add(j >= LAG ? j - LAG : j - LAG + NM);
            // the next step's scales, behind the last use of this one's
            if (j == HAND + LAG) {
                wn0 = *(lds_float)(uintptr_t)(ws_at + next);
                if (SWI) wn1 = *(lds_float)(uintptr_t)(ws_at + 4 + next);
            }
            if (j >= HAND + LAG && j - HAND - LAG < TM) tn[j - HAND - LAG] = *(lds_float)(uintptr_t)(ts_at + next + 64 * (j - HAND - LAG));
        }
        cur = next;
    };

    // Fill the ring: all but the last stage, and of that what a hand-over ahead of the first step would have issued by now.  Fewer steps than
    // stages: the last step's operands again.
    constexpr int BEGUN = (2 * TM + GAP - 1) / GAP < LOADS ? (2 * TM + GAP - 1) / GAP : LOADS;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        to = s * STAGE;
        if (s > 0 && s < nk) next_step();
#pragma unroll
        for (int d = 0; d < (s + 1 < NS ? LOADS : BEGUN); ++d) load(d);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * LOADS + BEGUN) : "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        a_raw[i % NA] = read(At{a_at, a_at ^ 64}, 16 * KB * i);
        if constexpr (WIDE) af[i] = operand<WIDE>(a_raw[i % NA]);
        tn[i] = *(lds_float)(uintptr_t)(ts_at + 64 * i);
    }
    w_raw[buffer_of(0)] = read(At{w_at, w_at ^ 64}, 0);
    if constexpr (WIDE) wf[0] = operand<WIDE>(w_raw[buffer_of(0)]);
    wn0 = *(lds_float)(uintptr_t)ws_at;
    if (SWI) wn1 = *(lds_float)(uintptr_t)(ws_at + 4);
    const std::true_type yes;
    const std::false_type no;
    int kt = 0;
    if (nk >= NS) {
        for (; kt + NS < nk; ++kt) step(yes, yes);
        step(yes, no);
        ++kt;
    }
    for (; kt < nk; ++kt) step(no, no);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (fewer steps than stages: loads that no step has waited for)
#pragma unroll
    for (int j = NM - LAG; j < NM; ++j) add(j);

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
    if (hipError_t e = allow_smem_once(once, st, kernel, smem)) return e;
    kernel<<<dim3((unsigned)(p.tiles_m * p.tiles_n * splits)), dim3(64 * WM * WN), smem, s>>>(p);
    return hipGetLastError();
}

// ---- few tokens ----
// A workgroup of W waves owns FN x 16 features (of a SwiGLU projection half of the fragments are the up rows) of TM x 16 tokens, and its waves share
// out k.  A wave has a ring of S slices of its own in the LDS, which it fills and waits for by itself: nothing but the end of the loop needs the
// other waves.  The waves' sums meet in the LDS and are added in their order.  NT: weights that no other workgroup reads go past the caches.
template <int EPI, int FN, int TM, int W, int S, bool WIDE, bool NT>
__global__ void __launch_bounds__(64 * W) rows_kernel(Args p) {
    constexpr bool SWI = EPI == EPI_SWIGLU;
    constexpr int P = SWI ? FN / 2 : FN, PAIRS = P * TM, UPT = (PAIRS + W - 1) / W;   // (gate) fragments; a wave finishes UPT 16 x 16 results
    constexpr int SC = TM <= 2 ? 256 : 512, STAGE = (FN + TM) * 2048 + SC, L = 2 * (FN + TM) + SC / 256;   // bytes and loads of a slice
    static_assert(!SWI || FN % 2 == 0, "pairs");
    static_assert(S * L < 64 && TM <= 4, "vmcnt field, tokens whose scales one load brings");
    extern __shared__ __align__(16) unsigned char smem[];   // the rings, then the waves' sums
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n_tiles = p.tiles_m * p.tiles_n, unit = blockIdx.x % n_tiles, split = EPI == EPI_SLAB ? blockIdx.x / n_tiles : 0;
    const int n_lo = unit / p.tiles_m * (16 * P), t0 = unit % p.tiles_m * (16 * TM), cols = SWI ? p.n_half : p.N, nkb = p.K / KB;

    // what the epilogue reads besides the sums, as loaded
    float4 res[UPT];
#pragma unroll
    for (int q = 0; q < UPT; ++q) {
        const int pair = wave + W * q, n = n_lo + 16 * (pair / TM) + 4 * g, t = t0 + 16 * (pair % TM) + l16;
        res[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (pair >= PAIRS || t >= p.T || n >= cols) continue;
        const int64_t o = (int64_t)t * p.N + n;
        if (EPI == EPI_RES_BF16_OUT_F32 && p.residual) {
            const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.residual) + o);
            res[q].x = __uint_as_float(r.x);
            res[q].y = __uint_as_float(r.y);
        } else if (EPI == EPI_RES_F32_OUT_BF16) {
            res[q] = *reinterpret_cast<const float4*>(static_cast<const float*>(p.residual) + o);
        }
    }
    // the wave's slices; lane l loads slot l % 8 of row l / 8, which holds chunk slot ^ (row / 2 % 8).  Rows past the end are the last one again
    const int k_from = EPI == EPI_SLAB ? split * p.per_split : 0, k_many = EPI == EPI_SLAB ? min(p.per_split, nkb - k_from) : nkb;
    const int s_begin = k_from + k_many * wave / W, n_own = k_from + k_many * (wave + 1) / W - s_begin;
    const int w_step = p.packed ? 256 * KB : KB;
    const char* const ab = uniform_ptr(reinterpret_cast<const char*>(p.a) + (int64_t)s_begin * KB);
    const char* const wb = uniform_ptr(reinterpret_cast<const char*>(p.w) + (int64_t)s_begin * w_step);
    const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem + wave * (S * STAGE));
    uint32_t a_off[TM][2], w_off[FN][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = 8 * h + (lane >> 3);
        const uint32_t chunk = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
#pragma unroll
        for (int i = 0; i < TM; ++i) a_off[i][h] = (uint32_t)min(t0 + 16 * i + r, p.T - 1) * (uint32_t)p.K + chunk;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const bool up = SWI && j >= P;
            const uint32_t row = (uint32_t)(min(n_lo + 16 * (up ? j - P : j) + r, cols - 1) + (up ? p.n_half : 0));
            w_off[j][h] = (p.packed ? (row >> 8) * (uint32_t)p.K * 256u + (row & 255) * 128u : row * (uint32_t)p.K) + chunk;
        }
    }
    // scales: 64 tokens', or 32 tokens' and the weights' (gate, up)
    const float* const ws_from = p.w_scale + (int64_t)scale_row(p, SWI, n_lo, lane & 1) * nkb + s_begin;
    const float* const ts_from = p.a_scale + (int64_t)s_begin * p.T + min(t0 + lane, p.T - 1);
    const bool w_lane = TM <= 2 && lane >= 32;
    const float* const s_from = w_lane ? ws_from : ts_from;
    const int64_t s_step = w_lane ? 1 : p.T;
    auto load = [&](int stage, int k) __attribute__((always_inline)) {   // the wave's k-th slice; weights first, which come from further away
        const uint32_t to = __builtin_amdgcn_readfirstlane(ring + stage * STAGE);
        const char* ws = wb + (int64_t)k * w_step;
        const char* as = ab + (int64_t)k * KB;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) dma16<NT>(ws, w_off[j][h], to, j * 2048 + h * 1024);
        dma4(s_from + k * s_step, to, (FN + TM) * 2048);
        if (SC > 256) dma4(ws_from + k, to, (FN + TM) * 2048 + 256);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) dma16(as, a_off[i][h], to, (FN + i) * 2048 + h * 1024);
    };
    using operand_t = decltype(operand<WIDE>(i32x8_t{}));
    f32x4_t acc[FN][TM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const uint32_t frag = l16 * 128 + ((g ^ ((l16 >> 1) & 7)) << 4);
    auto slice = [&](int stage, int k) __attribute__((always_inline)) {
        const int behind = min(n_own - 1 - k, S - 1);   // slices that are on their way behind this one
        static_assert(S <= 4, "waits");
        if (behind >= S - 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * L) : "memory");
        else if (S > 3 && behind == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 3 ? 2 * L : 0) : "memory");
        else if (S > 2 && behind == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 2 ? L : 0) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint32_t at = ring + stage * STAGE, scales = at + (FN + TM) * 2048;
        auto read = [&](int i) __attribute__((always_inline)) {
            const i32x4_t lo = *(lds_chunk)(uintptr_t)(at + frag + i * 2048), hi = *(lds_chunk)(uintptr_t)((at + i * 2048) + (frag ^ 64));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        i32x8_t av[TM], wv[FN];
        float ts[TM];
        const float w0 = *(lds_float)(uintptr_t)(scales + (TM <= 2 ? 128 : 256)), w1 = SWI ? *(lds_float)(uintptr_t)(scales + (TM <= 2 ? 132 : 260)) : 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            av[i] = read(FN + i);
            ts[i] = *(lds_float)(uintptr_t)(scales + 64 * i + 4 * l16);
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) wv[j] = read(j);
        if (k + S < n_own) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the refill lands
            __builtin_amdgcn_sched_barrier(0);
            load(stage, k + S);
        }
        operand_t ao[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) ao[i] = operand<WIDE>(av[i]);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const operand_t wo = operand<WIDE>(wv[j]);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const f32x4_t v = block_sum(wo, ao[i]);
                const float f = ts[i] * (SWI && j >= P ? w1 : w0);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][i][r] = __builtin_fmaf(v[r], f, acc[j][i][r]);
            }
        }
    };
#pragma unroll
    for (int b = 0; b < S; ++b)
        if (b < n_own) load(b, b);
    for (int k = 0; k < n_own; k += S) {
#pragma unroll
        for (int b = 0; b < S; ++b)
            if (k + b < n_own) slice(b, k + b);
    }

    __syncthreads();   // the rings have been read
    f32x4_t* const red = reinterpret_cast<f32x4_t*>(smem);   // [wave][fragment pair][lane]
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) red[(wave * (FN * TM) + j * TM + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    auto total = [&](int pair) __attribute__((always_inline)) {
        f32x4_t v = red[pair * 64 + lane];
#pragma unroll
        for (int q = 1; q < W; ++q) v += red[(q * (FN * TM) + pair) * 64 + lane];
        return v;
    };
#pragma unroll
    for (int q = 0; q < UPT; ++q) {
        const int pair = wave + W * q, n = n_lo + 16 * (pair / TM) + 4 * g, t = t0 + 16 * (pair % TM) + l16;
        if (pair >= PAIRS || t >= p.T || n >= cols) continue;
        f32x4_t v = total(pair);
        const int64_t o = (int64_t)t * cols + n;
        if constexpr (EPI == EPI_SLAB) {
            *reinterpret_cast<f32x4_t*>(p.slabs + (int64_t)split * p.T * p.N + o) = v;
        } else if constexpr (EPI == EPI_RES_BF16_OUT_F32) {
            const uint32_t r0 = __float_as_uint(res[q].x), r1 = __float_as_uint(res[q].y);
            if (p.residual) v += f32x4_t{bf16_lo(r0), bf16_hi(r0), bf16_lo(r1), bf16_hi(r1)};
            *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + o) = v;
        } else {
            if constexpr (EPI == EPI_RES_F32_OUT_BF16) v += f32x4_t{res[q].x, res[q].y, res[q].z, res[q].w};
            if constexpr (SWI) {
                const f32x4_t u = total(PAIRS + pair);
                v = f32x4_t{silu_mul(v[0], u[0]), silu_mul(v[1], u[1]), silu_mul(v[2], u[2]), silu_mul(v[3], u[3])};
            }
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
    }
}

template <int EPI, int FN, int TM, int W, int S, bool WIDE, bool NT>
hipError_t launch_rows(Args p, int splits, hipStream_t s) {
    constexpr int P = EPI == EPI_SWIGLU ? FN / 2 : FN;
    constexpr int stage = (FN + TM) * 2048 + (TM <= 2 ? 256 : 512), smem = std::max(W * S * stage, W * FN * TM * 1024);
    static_assert(smem <= 160 * 1024, "rings exceed the LDS");
    p.tiles_m = (p.T + 16 * TM - 1) / (16 * TM);
    p.tiles_n = ((EPI == EPI_SWIGLU ? p.n_half : p.N) + 16 * P - 1) / (16 * P);
    static std::once_flag once;
    static hipError_t st = hipSuccess;
    auto kernel = &rows_kernel<EPI, FN, TM, W, S, WIDE, NT>;
    if (hipError_t e = allow_smem_once(once, st, kernel, smem)) return e;
    kernel<<<dim3((unsigned)(p.tiles_m * p.tiles_n * splits)), dim3(64 * W), smem, s>>>(p);
    return hipGetLastError();
}

// ---- partial sums of k ranges: added in their order, and the epilogue ----
template <int EPI>
__global__ void __launch_bounds__(256) finish_kernel(Args p, int splits) {
    const int64_t quads = (int64_t)p.T * (EPI == EPI_SWIGLU ? p.n_half : p.N) / 4, cols4 = (EPI == EPI_SWIGLU ? p.n_half : p.N) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= quads) return;
    const int64_t t = i / cols4, n = i % cols4 * 4, slab = (int64_t)p.T * p.N;
    const float* from = p.slabs + t * p.N + n;
    f32x4_t v = *reinterpret_cast<const f32x4_t*>(from), u{0.f, 0.f, 0.f, 0.f};
    if (EPI == EPI_SWIGLU) u = *reinterpret_cast<const f32x4_t*>(from + p.n_half);
    for (int s = 1; s < splits; ++s) {
        v += *reinterpret_cast<const f32x4_t*>(from + s * slab);
        if (EPI == EPI_SWIGLU) u += *reinterpret_cast<const f32x4_t*>(from + s * slab + p.n_half);
    }
    if constexpr (EPI == EPI_RES_BF16_OUT_F32) {
        if (p.residual) {
            const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.residual) + 4 * i);
            v += f32x4_t{bf16_lo(r.x), bf16_hi(r.x), bf16_lo(r.y), bf16_hi(r.y)};
        }
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + 4 * i) = v;
    } else {
        if constexpr (EPI == EPI_RES_F32_OUT_BF16) v += *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p.residual) + 4 * i);
        if constexpr (EPI == EPI_SWIGLU) v = f32x4_t{silu_mul(v[0], u[0]), silu_mul(v[1], u[1]), silu_mul(v[2], u[2]), silu_mul(v[3], u[3])};
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + 4 * i) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
}

template <int EPI>
hipError_t finish(const Args& p, int splits, hipStream_t s) {
    const int64_t quads = (int64_t)p.T * (EPI == EPI_SWIGLU ? p.n_half : p.N) / 4;
    finish_kernel<EPI><<<dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s>>>(p, splits);
    return hipGetLastError();
}

// How a projection runs: a tile, into how many ranges k is cut, and whether its weights go past the caches.
struct Plan { int tile, splits; bool streamed; };
enum { ROWS_16, ROWS_16_NARROW, ROWS_32, ROWS_32_NARROW, ROWS_64, TILE_64, TILE_128, TILE_128_WIDE, TILE_256, PLANS };

// What a tile takes, in us: a launch's base, then for each round of workgroups over the chip its begin and end and its k steps (of a wave's own slices
// for rows), both of codes and of codes widened to bf16; a step of a round that leaves CUs idle costs `alone` of that, the rest by how many work.
// Fitted to measured launches, weights from memory, fp32 outputs above 32 tokens apart from the rest.  Against the best plan of each of 325 shapes (6125 launches,
// weights from memory) the chosen one is slower by, on average and at worst: bf16 outputs and SwiGLU 2.4 %, 39 % (24 x 4096 x 14336: 21.7 us for 15.6 in
// ROWS_32_NARROW); fp32 outputs above 32 tokens 2.8 %, 26 % (2050 x 4096 x 4096: 113 for 90 in TILE_64), of 17..32 tokens 4.5 %, 27 %, of up to 16 tokens
// 12.3 %, 43 % (1 x 640 x 7552: 9.3 for 6.5).  The last is ROWS_16_NARROW's step_wide, which no launch stands behind: a step takes it 0.25 .. 0.35 us, and with 5.66 it is
// chosen at k = 128 alone, where fp32 outputs of up to 128 workgroups would gain by it (4 x 4096 x 4096 7.0 -> 6.1 us, 4 x 2560 x 5120 7.4 -> 5.8,
// 4 x 1024 x 4096 5.5 -> 4.7).
struct TileCost { int rows, features, at_once; double base, step, step_wide, round, round_wide, alone; };
constexpr TileCost kCost[PLANS] = {
    {16, 32, 512, 0.11, 1.17, 0.79, 1.63, 1.63, 0.19},  {16, 16, 768, 0.14, 0.53, 5.66, 1.29, 1.29, 0.18},  {32, 32, 512, 2.45, 1.52, 0.94, 1.22, 0.78, 0.10},
    {32, 16, 512, 0.15, 0.056, 0.45, 0.57, 0.57, 0.27}, {64, 32, 256, 2.08, 0.68, 0.66, 2.14, 1.12, 0.68},  {64, 128, 512, 1.62, 0.80, 0.93, 4.12, 3.40, 0.74},
    {128, 128, 512, 3.42, 1.50, 1.38, 4.50, 4.67, 2.37}, {128, 256, 256, 2.38, 0.91, 1.38, 12.0, 5.16, 0.53}, {256, 256, 256, 0.0, 1.70, 2.40, 16.2, 16.2, 0.72}};
constexpr int64_t kSlabFloats = (int64_t)1 << 24;   // of partial sums: 64 MB, which the last-level cache holds

double cost_of(const Args& p, bool wide, int tile, int splits) {
    const TileCost& c = kCost[tile];
    const double units = (double)((p.T + c.rows - 1) / c.rows) * ((p.N + c.features - 1) / c.features) * splits, rounds = units / c.at_once;
    const double steps = (double)((p.K / KB + splits - 1) / splits) / (tile <= ROWS_64 ? 4 : 1);
    const double busy = rounds > 1 ? 1.0 : c.alone + (1.0 - c.alone) * rounds;
    const double work = std::max(1.0, std::ceil(rounds)) * (wide ? c.round_wide + c.step_wide * steps * busy : c.round + c.step * steps * busy);
    // operands from memory and, for each column of tiles, from the caches
    const double bytes = (double)p.N * p.K + 0.02 * (double)p.T * p.K * ((p.N + c.features - 1) / c.features), out = (double)p.T * p.N;
    return c.base + std::max(work, bytes / 4.5e6) + (splits > 1 ? 2.0 + splits * out * 4 / 6e6 + out * 6 / 5e6 : out * 4 / 20e6);
}

// Up to 16 tokens weights of 32 MB and more are read with the non-temporal hint: two layers with such a matrix are more than the last-level cache holds, so
// that the next step finds them in memory.  us without -> with, from memory (from the cache): T = 1, 15360 x 5120 15.2 -> 14.2 (13.2, 13.2), SwiGLU 27648 x
// 5120 26.3 -> 24.1, T = 16, 12288 x 4096 12.7 -> 12.1 (9.8 -> 10.7).  At 24 tokens it loses more from the cache than it gains (15360 x 5120 18.1 -> 17.7, 14.0 -> 16.2).
constexpr int64_t kFarWeights = (int64_t)32 << 20;

Plan plan_for(const Args& p, int epi) {
    const bool swiglu = epi == EPI_SWIGLU, wide = epi == EPI_RES_BF16_OUT_F32;
    const int64_t out = (int64_t)p.T * p.N;
    auto fits = [&](int tile) {
        switch (tile) {
            case ROWS_16: return p.T <= 16;
            // 16 features each where that many more workgroups find idle CUs.  us in 32 and in 16, 4 tokens, bf16 outputs, weights from memory: 32 workgroups (of 32
            // features; k = 4096) 4.6, 4.0; 80 (5120) 7.0, 5.4; 128 (4096) 6.5, 5.8; 160 (5120) 7.6, 8.3, (13824) 14.2, 17.4; 192 (4096) 7.2, 7.7
            case ROWS_16_NARROW: return !swiglu && p.T <= 16 && (p.N + 31) / 32 < 160;
            case ROWS_32: return p.T <= 128;
            // the same, 24 tokens: 32 workgroups 5.5, 4.8; 80 9.2, 7.9; 160 9.8, 12.0 ((13824) 19.6, 24.1); 128, which it leaves out, 8.1, 6.9 ((14336) 19.5, 15.5)
            case ROWS_32_NARROW: return !swiglu && p.T > 16 && p.T <= 128 && (p.N + 31) / 32 * ((p.T + 31) / 32) < 128;
            case ROWS_64: return p.T > 32 && p.T <= 512;
            case TILE_64: return p.T > 32;
            case TILE_256: return p.T > 64 && !wide;
            default: return p.T > 64;
        }
    };
    Plan best{ROWS_32, 1, false};
    double least = 1e30;
    for (int tile = 0; tile < PLANS; ++tile) {
        if (!fits(tile)) continue;
        for (int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
            // (a range of gate rows and one of up rows in one tile of partial sums: where both end with a block)
            if (splits > 1 && (!p.slabs || splits * 2 > p.K / KB || splits * out > kSlabFloats || (swiglu && p.n_half % KB))) break;
            const double us = cost_of(p, wide, tile, splits);
            if (us < least) least = us, best = {tile, splits, tile == ROWS_16 && (int64_t)p.N * p.K >= kFarWeights};
        }
    }
    return best;
}

template <int EPI, bool WIDE>
hipError_t run_tile(const Args& p, Plan plan, hipStream_t s) {
    switch (plan.tile) {
        case ROWS_16:
            return plan.streamed ? launch_rows<EPI, 2, 1, 4, 3, WIDE, true>(p, plan.splits, s) : launch_rows<EPI, 2, 1, 4, 3, WIDE, false>(p, plan.splits, s);
        case ROWS_16_NARROW:
            if constexpr (EPI != EPI_SWIGLU) return launch_rows<EPI, 1, 1, 4, 4, WIDE, false>(p, plan.splits, s);
            else return hipErrorInvalidValue;
        case ROWS_32: return launch_rows<EPI, 2, 2, 4, 2, WIDE, false>(p, plan.splits, s);
        case ROWS_32_NARROW:
            if constexpr (EPI != EPI_SWIGLU) return launch_rows<EPI, 1, 2, 4, 3, WIDE, false>(p, plan.splits, s);
            else return hipErrorInvalidValue;
        case ROWS_64: return launch_rows<EPI, 2, 4, 4, 2, WIDE, false>(p, plan.splits, s);
        case TILE_64: return launch_tiles<64, 128, 2, 2, 3, EPI, WIDE>(p, plan.splits, s);
        case TILE_128: return launch_tiles<128, 128, 2, 2, 2, EPI, WIDE>(p, plan.splits, s);
        case TILE_128_WIDE: return launch_tiles<128, 256, 2, 4, 3, EPI, WIDE>(p, plan.splits, s);
        case TILE_256:
            if constexpr (!WIDE) return launch_tiles<256, 256, 4, 2, 2, EPI, WIDE>(p, plan.splits, s);
            else return hipErrorInvalidValue;
        default: return hipErrorInvalidValue;
    }
}

template <int EPI>
hipError_t run_plan(Args p, Plan plan, hipStream_t s) {
    constexpr bool WIDE = EPI == EPI_RES_BF16_OUT_F32;
    const int nkb = p.K / KB;
    p.per_split = (nkb + plan.splits - 1) / plan.splits;
    plan.splits = (nkb + p.per_split - 1) / p.per_split;
    if (plan.splits == 1) return run_tile<EPI, WIDE>(p, plan, s);
    if (hipError_t e = run_tile<EPI_SLAB, WIDE>(p, plan, s)) return e;
    return finish<EPI>(p, plan.splits, s);
}

template <int EPI>
hipError_t run(const Args& p, hipStream_t s) { return run_plan<EPI>(p, plan_for(p, EPI), s); }

}  // namespace

// (grows with either size, so that the largest call's serves all; any 32-bit sizes, whose product has up to 62 bits)
int64_t gemm_f8b_scratch_floats(int64_t T, int64_t N) { return std::max<int64_t>(64, 16 * std::min(T * N, kSlabFloats / 16)); }

GemmPlanF8b gemm_plan_f8b(int32_t T, int32_t N, int32_t K, int32_t epilogue, bool scratch) {
    float some_scratch;
    Args p{};
    p.T = T, p.N = N, p.K = K, p.n_half = N / 2;
    p.slabs = scratch ? &some_scratch : nullptr;
    const Plan plan = plan_for(p, epilogue);
    const int per_range = (K / KB + plan.splits - 1) / plan.splits;
    return {plan.tile, (K / KB + per_range - 1) / per_range, plan.streamed};
}

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
