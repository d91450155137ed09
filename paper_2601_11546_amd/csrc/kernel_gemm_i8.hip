// int8 projections: out[t, n] = sum_k a[t, k] w[n, k] * w_scale[n] * a_scale[t] of 8-bit integers, summed exactly in 32 bits: the kernels of
// gemm_kernels.h on integers, with a factor for each token beside each feature's in their epilogues.
#define RELSERVE_GEMM_INT8 1
#include "gemm_kernels.h"

namespace relserve {

void gemm_force_plan_i8(int cand, int splits) {
    g_forced_plan.store(cand < 0 ? -1 : (cand | (splits << 8)), std::memory_order_relaxed);
}

namespace {

// Few tokens, or a small problem: a workgroup of W waves owns FN x 16 features (of an epilogue that combines pairs half of the fragments
// are the partners: up rows, or the second halves of a head) of TM x 16 tokens, and its waves share out k.  A wave has a ring of S slices of
// 128 codes of its own in the LDS, which it fills and waits for by itself: nothing but the end of the loop needs the other waves.
// The waves' sums meet in the LDS, and one pass adds them up (exactly, being integers) and finishes: no second launch and no partial
// sums through memory.  What the epilogue reads besides is fetched ahead of the loop.
// (Fragments straight from memory to registers ask for 16 bytes of 16 rows with every 16 lanes, and a CU takes one line a cycle: no more than
// 5.4 TB/s of weights, less what the activations take.)
template <int EPI, int D, int FN, int TM, int W, int S, bool NT>
__global__ void __launch_bounds__(64 * W) linear_rows_kernel(GemmArgs p) {
    constexpr bool PAIRED = EPI == EPI_SWIGLU || EPI == EPI_QKV_ROPE;
    constexpr int P = PAIRED ? FN / 2 : FN, DH = D > 0 ? D : 64;   // fragments of first partners; of them a unit's quad comes
    constexpr int PAIRS = P * TM, UPT = (PAIRS + W - 1) / W;   // (first) fragment pairs: a wave finishes UPT of them, a lane 4 features of a token in each
    static_assert(!PAIRED || FN % 2 == 0, "pairs");
    constexpr int STAGE = (FN + TM) * 2048, L = 2 * (FN + TM);   // bytes and loads of a slice: 16 rows of 128 bytes each
    static_assert(S * L < 64, "vmcnt field");
    extern __shared__ __align__(16) unsigned char smem[];   // the rings, then the waves' sums
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile_n = blockIdx.x / p.tiles_m, t0 = (int)(blockIdx.x % p.tiles_m) * (16 * TM);
    // first feature of a fragment, and how many rows of the weight matrix there are from its partner group's start
    int head = 0, n_lo, cols;   // first partners: features n_lo .. of [.., cols)
    if (EPI == EPI_QKV_ROPE) {
        constexpr int PER = DH / 2 / (16 * P);   // workgroups per head
        head = tile_n / PER;
        n_lo = head * DH + tile_n % PER * (16 * P);
        cols = p.N;
    } else {
        n_lo = tile_n * (16 * P);
        cols = EPI == EPI_SWIGLU ? p.n_half : p.N;
    }
    const int partner = EPI == EPI_SWIGLU ? p.n_half : DH / 2;   // from a first partner to the second

    // what this thread's units read besides the sums
    float4 f_lo[UPT], f_hi[UPT], oa[UPT], ob[UPT];
    float ts[UPT];
    int slot[UPT];
#pragma unroll
    for (int q = 0; q < UPT; ++q) {
        const int pair = wave + W * q, n = n_lo + 16 * (pair / TM) + 4 * g, t = t0 + 16 * (pair % TM) + l16;
        f_lo[q] = f_hi[q] = oa[q] = ob[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        ts[q] = 0.f;
        slot[q] = 0;
        if (pair >= PAIRS || t >= p.T || n >= cols) continue;
        f_lo[q] = code_factor(p, n);
        if (PAIRED) f_hi[q] = code_factor(p, n + partner);
        ts[q] = p.t_scale[t];
        if constexpr (EPI == EPI_QKV_ROPE) {
            slot[q] = p.tok_slot[t];
            const float4* cs = reinterpret_cast<const float4*>(p.rope_cs + (int64_t)t * (DH / 2) + n - head * DH);
            oa[q] = cs[0];
            ob[q] = cs[1];
        } else if constexpr (EPI == EPI_RES_BF16_OUT_F32) {
            if (p.residual) {   // as loaded: widened when it is added, so that nothing waits for it here
                const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.residual) + (int64_t)t * p.N + n);
                oa[q].x = __uint_as_float(r.x);
                oa[q].y = __uint_as_float(r.y);
            }
        } else if constexpr (EPI == EPI_RES_F32_OUT_BF16) {
            oa[q] = *reinterpret_cast<const float4*>(static_cast<const float*>(p.residual) + (int64_t)t * p.N + n);
        }
    }
    // operands: rows past the end are the last one again, and nothing of them is stored.  Lane l loads slot l % 8 of row l / 8, which holds
    // chunk slot ^ (row >> 1 & 7): the 16 rows that a fragment's 16 lanes read lie in different banks
    const int slices = p.K / 64, s_begin = slices * wave / W, s_end = slices * (wave + 1) / W;   // (K counts pairs of codes)
    const int w_step = p.w_packed ? 32768 : 128;
    const char* const ab = uniform_ptr(reinterpret_cast<const char*>(p.a) + (int64_t)s_begin * 128);
    const char* const wb = uniform_ptr(reinterpret_cast<const char*>(p.w) + (int64_t)s_begin * w_step);
    const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem + wave * (S * STAGE));
    uint32_t a_off[TM][2], w_off[FN][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = 8 * h + (lane >> 3);
        const uint32_t chunk = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
#pragma unroll
        for (int i = 0; i < TM; ++i) a_off[i][h] = (uint32_t)min(t0 + 16 * i + r, p.T - 1) * (uint32_t)p.K * 2 + chunk;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const bool second = PAIRED && j >= P;
            const uint32_t row = (uint32_t)(min(n_lo + 16 * (second ? j - P : j) + r, cols - 1) + (second ? partner : 0));
            w_off[j][h] = (p.w_packed ? (row >> 8) * (uint32_t)p.K * 512u + (row & 255) * 128u : row * (uint32_t)p.K * 2u) + chunk;
        }
    }
    const uint32_t frag = ring + l16 * 128 + ((g ^ ((l16 >> 1) & 7)) << 4);   // of fragment 0 of stage 0; the second half's chunk is 4 further
    i32x4_t acc[FN][TM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = i32x4_t{};
    const int n_own = s_end - s_begin;
    auto load = [&](int stage, int k) __attribute__((always_inline)) {   // the wave's k-th slice; weights first, which come from further away
        const uint32_t to = __builtin_amdgcn_readfirstlane(ring + stage * STAGE);
        const char* ws = wb + (int64_t)k * w_step;
        const char* as = ab + (int64_t)k * 128;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) dma16<NT>(ws, w_off[j][h], to, j * 2048 + h * 1024);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) dma16(as, a_off[i][h], to, (FN + i) * 2048 + h * 1024);
    };
    typedef const i32x4_t __attribute__((address_space(3))) * lds_chunk;
    auto slice = [&](int stage, int k) __attribute__((always_inline)) {
        const int behind = min(n_own - 1 - k, S - 1);   // slices that are on their way behind this one
        static_assert(S <= 7, "waits");
        if (behind >= S - 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * L) : "memory");
        else if (S > 6 && behind == 5) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 6 ? 5 * L : 0) : "memory");
        else if (S > 5 && behind == 4) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 5 ? 4 * L : 0) : "memory");
        else if (S > 4 && behind == 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 4 ? 3 * L : 0) : "memory");
        else if (S > 3 && behind == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 3 ? 2 * L : 0) : "memory");
        else if (S > 2 && behind == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S > 2 ? L : 0) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint32_t at = frag + stage * STAGE;
        i32x4_t wv[FN][2], av[TM][2];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) av[i][h] = *(lds_chunk)(uintptr_t)((at ^ (64 * h)) + (FN + i) * 2048);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) wv[j][h] = *(lds_chunk)(uintptr_t)((at ^ (64 * h)) + j * 2048);
        if (k + S < n_own) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the refill lands
            __builtin_amdgcn_sched_barrier(0);
            load(stage, k + S);
        }
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j][h], av[i][h], acc[j][i], 0, 0, 0);
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
    i32x4_t* const red = reinterpret_cast<i32x4_t*>(smem);   // [wave][fragment pair][lane]
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) red[(wave * (FN * TM) + j * TM + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    auto total = [&](int pair) __attribute__((always_inline)) {
        i32x4_t v = red[pair * 64 + lane];
#pragma unroll
        for (int q = 1; q < W; ++q) v += red[(q * (FN * TM) + pair) * 64 + lane];
        return make_float4(__int_as_float(v[0]), __int_as_float(v[1]), __int_as_float(v[2]), __int_as_float(v[3]));
    };
#pragma unroll
    for (int q = 0; q < UPT; ++q) {
        const int pair = wave + W * q, n = n_lo + 16 * (pair / TM) + 4 * g, t = t0 + 16 * (pair % TM) + l16;
        if (pair >= PAIRS || t >= p.T || n >= cols) continue;
        float4 lo = total(pair), hi = make_float4(0.f, 0.f, 0.f, 0.f);
        const int64_t o = (int64_t)t * p.N + n;
        if constexpr (EPI == EPI_RES_BF16_OUT_F32) {
            const uint32_t r0 = __float_as_uint(oa[q].x), r1 = __float_as_uint(oa[q].y);
            if (p.residual) lo = code_scale_plus(lo, f_lo[q], ts[q], make_float4(bf16_lo(r0), bf16_hi(r0), bf16_lo(r1), bf16_hi(r1)));
            else code_scale(lo, p, f_lo[q], ts[q]);
            *reinterpret_cast<float4*>(static_cast<float*>(p.out) + o) = lo;
        } else if constexpr (EPI == EPI_RES_F32_OUT_BF16) {
            lo = code_scale_plus(lo, f_lo[q], ts[q], oa[q]);
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + o) = make_uint2(pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w));
        } else {
            code_scale(lo, p, f_lo[q], ts[q]);
            if constexpr (PAIRED) {
                hi = total(PAIRS + pair);
                code_scale(hi, p, f_hi[q], ts[q]);
            }
            store_unit<EPI, D>(p, t, n, head, lo, hi, oa[q], ob[q], slot[q]);
        }
    }
}

template <int EPI, int D, int FN, int TM, int W, int S, bool NT>
hipError_t launch_rows(GemmArgs p, hipStream_t s) {
    constexpr int P = EPI == EPI_SWIGLU || EPI == EPI_QKV_ROPE ? FN / 2 : FN;
    p.tiles_m = (p.T + 16 * TM - 1) / (16 * TM);
    const int cols = EPI == EPI_SWIGLU ? p.n_half : EPI == EPI_QKV_ROPE ? p.N / 2 : p.N;
    p.tiles_n = (cols + 16 * P - 1) / (16 * P);
    constexpr int smem = std::max(W * S * (FN + TM) * 2048, W * FN * TM * 1024);
    static_assert(smem <= 160 * 1024, "rings exceed the LDS");
    static std::once_flag once;
    static hipError_t st = hipSuccess;
    if (hipError_t e = allow_smem_once(once, st, &linear_rows_kernel<EPI, D, FN, TM, W, S, NT>, smem)) return e;
    linear_rows_kernel<EPI, D, FN, TM, W, S, NT><<<dim3(p.tiles_m * p.tiles_n), dim3(64 * W), smem, s>>>(p);
    return hipGetLastError();
}

// Up to 16 tokens weights of 32 MB and more are read with the non-temporal hint: two layers with such a matrix are more than the last-level cache
// (256 MB) holds, so that the next step finds them in memory.  us without -> with, from memory (from the cache): T = 1, 7168 x 5120 8.6 -> 7.7 (7.2 ->
// 7.1), 15360 x 5120 15.4 -> 13.9 (12.6 -> 13.2), SwiGLU 27648 x 5120 26.1 -> 23.7; T = 16, 12288 x 4096 12.6 -> 11.6 (9.2 -> 10.8).  Smaller ones gain 0.3 - 0.5 us
// from memory and lose up to 1.5 from the cache (5120 x 5120 at T = 16 8.2 -> 7.9, 5.9 -> 7.4).
constexpr int64_t kFarWeights = (int64_t)32 << 20;

// Which problems go this way, and on which tile.  Every workgroup loads its own activations beside its weights, so the time is a launch, two
// round trips and that traffic; the tiled kernels share both operands between more rows and columns, and win where the traffic gets long.
// Bytes are counted in MB of 10^6.
//
// In a step over a stack of layers the weights come from memory; those of a small stack stay in the last-level cache (256 MB).  us, tiled kernels with
// scratch -> this one, weights from memory (1.3 GB of sets in turn; three sets that the cache holds; outputs x k):
//   T = 1: 5120 x 5120 9.9 -> 7.0 (9.4 -> 5.8), 15360 x 5120 18.3 -> 13.9 (17.4 -> 13.2), 5120 x 13824 16.3 -> 13.1, SwiGLU 27648 x 5120 25.9 -> 23.7;
//   but 10240 x 8192 17.5 -> 17.6, at T = 16 18.6 -> 19.7
//   T = 24: 5120 x 5120 11.6 -> 9.5 (11.0 -> 6.5), 15360 x 5120 19.1 -> 18.0, 8192 x 8192 16.1 -> 14.5; 2560 x 8192 11.1 -> 12.0 (10.7 -> 7.4);
//   but 5120 x 13824 17.9 -> 19.3, 4096 x 14336 16.6 -> 18.9, 10240 x 8192 19.3 -> 22.8
//   T = 64: 15360 x 5120 22.5 -> 20.4, 6144 x 4096 14.4 -> 10.3; but 5120 x 13824 21.0 -> 26.0, 10240 x 8192 22.5 -> 25.8
//   T = 128: 15360 x 5120 29.4 -> 27.1, SwiGLU 11264 x 5120 25.8 -> 24.9, 7168 x 5120 21.3 -> 19.5, 4096 x 4096 19.7 -> 9.9;
//   but 5120 x 13824 26.3 -> 38.8 (26.1 -> 27.1), 8192 x 8192 22.1 -> 26.9, 10240 x 8192 29.4 -> 33.2
//   T = 256: 5120 x 5120 25.2 -> 22.1; 512: 4096 x 4096 27.4 -> 18.4 (19.5 -> 17.3), 2560 x 8192 30.3 -> 26.6; but 1000: 2048 x 2048 11.4 -> 12.6
//   T = 300: 2048 x 512 5.0 -> 4.5; but 1000: 5.5 -> 7.0, 2000: 9.6 -> 11.6, SwiGLU 2816 x 512 at 700 5.7 -> 7.3
// So with scratch, up to 64 tokens: what the fullest CU draws of the weights (k of 32 features for each of its workgroups) must not be long against
// what the tiled kernels take, which spread any matrix over all CUs and grow with its size.  From 65 tokens on: problems of short traffic, beyond
// 256 tokens on two workgroups per CU (the tiled kernels run whole tiles there), and tiles of 128 tokens in one round, counting the weights
// twice.  Against the tiled kernels, weights from memory: 18 % faster over 630 sizes of 26 shapes, 7 of them more than 5 % slower (12 at most);
// 16 % over 486 sizes of 26 other shapes, 6 % slower at most.  Without scratch the tiled kernels cannot cut k and are far slower on few
// tokens (5120 x 13824 at T = 24 85): there these limits do not hold.
//
// Tiles: as few fragments of tokens as they need up to 64 tokens.  With four, slices two deep where a CU gets one workgroup, else one deep and three
// workgroups (2000 x 2048 x 512 20.7, 12.2); four fragments of features for long k where they still fill the chip (64 x 10240 x 5120 17.0, 13.8).
enum { ROWS_NONE = 0, ROWS_16, ROWS_32, ROWS_64, ROWS_64_SHALLOW, ROWS_64_WIDE, ROWS_128, ROWS_128_WIDE };
int rows_tile(const GemmArgs& p, int epi) {
    if (forced_cand() >= 0) return ROWS_NONE;
    const bool paired = epi == EPI_SWIGLU || epi == EPI_QKV_ROPE, swiglu = epi == EPI_SWIGLU;
    const int64_t cols = swiglu ? 2 * (int64_t)p.n_half : p.N, k_bytes = 2 * (int64_t)p.K;
    const double weights_mb = 1e-6 * (double)(cols * k_bytes);
    auto tiles = [&](int fn, int tm) { return (int64_t)((p.T + 16 * tm - 1) / (16 * tm)) * (paired ? (cols / 2 + 8 * fn - 1) / (8 * fn) : (cols + 16 * fn - 1) / (16 * fn)); };
    auto traffic_mb = [&](int fn, int tm) { return 1e-6 * (double)(tiles(fn, tm) * 16 * (fn + tm) * k_bytes); };
    auto fills = [&](int fn, int tm) { return tiles(fn, tm) >= 150 && tiles(fn, tm) <= 256; };   // one round of workgroups, most CUs busy
    auto lean = [&](int fn, int tm) { return !p.accum || 1e-3 * (double)((tiles(fn, tm) + 255) / 256 * (fn / 2) * k_bytes) <= (p.T <= 16 ? 8.0 : 6.5) + 0.09 * weights_mb; };
    auto by_64 = [&] { return tiles(2, 4) > 256 ? ROWS_64_SHALLOW : tiles(2, 4) > 128 ? ROWS_64 : ROWS_32; };
    if (p.T <= 16) return traffic_mb(2, 1) <= (swiglu ? 268 : 420) && (weights_mb >= 100 || lean(2, 1)) ? ROWS_16 : ROWS_NONE;
    if (p.T <= 32) return traffic_mb(2, 2) <= 210 && lean(2, 2) ? ROWS_32 : ROWS_NONE;
    if (p.T <= 64) {
        if (k_bytes >= 4096 && tiles(4, 4) >= 160 && traffic_mb(4, 4) <= 210 && lean(4, 4)) return ROWS_64_WIDE;
        return traffic_mb(2, 4) <= 235 && lean(2, 4) ? by_64() : ROWS_NONE;
    }
    if (traffic_mb(2, 4) <= (swiglu ? 84 : 134) && (p.T <= 128 || tiles(2, 4) <= (p.T <= SKINNY_MAX_T ? 1280 : 512))) return by_64();
    if (k_bytes < 2048 || p.T > 768) return ROWS_NONE;
    const double weights_again = p.accum ? weights_mb : 0.0;
    if (fills(4, 8) && traffic_mb(4, 8) + weights_again <= (p.accum ? 320 : 252)) return ROWS_128_WIDE;
    if (fills(2, 8) && traffic_mb(2, 8) + weights_again <= (p.accum ? 270 : 357)) return ROWS_128;
    return ROWS_NONE;
}

template <int EPI, int D = 0>
hipError_t run_rows(const GemmArgs& p, hipStream_t s, int tile) {
    switch (tile) {
        case ROWS_16: return 2 * (int64_t)p.N * p.K >= kFarWeights ? launch_rows<EPI, D, 2, 1, 4, 3, true>(p, s) : launch_rows<EPI, D, 2, 1, 4, 3, false>(p, s);
        case ROWS_32: return launch_rows<EPI, D, 2, 2, 4, 2, false>(p, s);
        case ROWS_64: return launch_rows<EPI, D, 2, 4, 4, 2, false>(p, s);
        case ROWS_64_SHALLOW: return launch_rows<EPI, D, 2, 4, 4, 1, false>(p, s);
        case ROWS_64_WIDE: return launch_rows<EPI, D, 4, 4, 8, 1, false>(p, s);
        case ROWS_128: return launch_rows<EPI, D, 2, 8, 4, 1, false>(p, s);
        case ROWS_128_WIDE: return launch_rows<EPI, D, 4, 8, 4, 1, false>(p, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

GemmPlanI8 gemm_plan_i8(int32_t T, int64_t features, int32_t K, bool qkv, bool swiglu, bool scratch) {
    GemmArgs p{};
    float some_scratch;
    set_linear(p, nullptr, nullptr, T, (int32_t)features, K / 2, nullptr, nullptr, scratch ? &some_scratch : nullptr, false);
    if (const int tile = rows_tile(p, qkv ? EPI_QKV_ROPE : swiglu ? EPI_SWIGLU : EPI_BF16)) return {GemmPlanI8::WAVES, tile, 1, 0, 0};
    if (skinny_applies(p.T, p.N, p.K, p.accum)) {
        const int ranges = skinny_ranges(p.T, p.N, p.K, swiglu);
        return {ranges ? GemmPlanI8::FEW_RANGES : GemmPlanI8::FEW_WHOLE, 0, std::max(1, ranges), 0, 0};
    }
    const int bm = qkv ? 0 : split_rows(p.T, p.N, p.K, scratch, swiglu);
    if (bm && !one_range(p, bm)) return {GemmPlanI8::RANGES, bm, choose_splits(p.T, p.N, p.K, bm), 0, 0};
    const Plan plan = plan_for(p.T, p.N, p.K, qkv, scratch, swiglu);
    if (plan.cols1 > 0) return {GemmPlanI8::SHAPES, kTiles[plan.cand1].bm, 1, 0, plan.cols1};
    return {GemmPlanI8::TILES, kTiles[plan.cand].bm, plan.tail_tiles ? plan.splits : 1, plan.tail_tiles, 0};
}

// The kernels see rows of K / 2 two-byte units.
static hipError_t set_int8(GemmArgs& p, const float* t_scale, const float* w_scale) {
    if (p.K % 128) return hipErrorInvalidValue;
    p.f8 = 1;
    p.K /= 2;
    p.w_scale = w_scale;
    p.t_scale = t_scale;
    return hipSuccess;
}

hipError_t launch_linear_i8(const void* a, const float* a_scale, const void* w, const float* w_scale, int32_t T, int32_t N, int32_t K,
                            int32_t epilogue, const void* residual, void* out, hipStream_t s, float* accum, bool w_packed) {
    if (T == 0) return hipSuccess;
    if ((int64_t)T * K >= ((int64_t)1 << 31) || (int64_t)N * K >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    GemmArgs p{};
    set_linear(p, a, w, T, N, K, residual, out, accum, w_packed);
    if (hipError_t e = set_int8(p, a_scale, w_scale)) return e;
    if (const int tile = rows_tile(p, epilogue)) {
        switch (epilogue) {
            case EPI_BF16: return run_rows<EPI_BF16>(p, s, tile);
            case EPI_RES_BF16_OUT_F32: return run_rows<EPI_RES_BF16_OUT_F32>(p, s, tile);
            case EPI_RES_F32_OUT_BF16: return run_rows<EPI_RES_F32_OUT_BF16>(p, s, tile);
            case EPI_SWIGLU: return run_rows<EPI_SWIGLU>(p, s, tile);
            default: return hipErrorInvalidValue;
        }
    }
    return run_linear(p, epilogue, s, nullptr);
}

hipError_t launch_qkv_rope_append_i8(const BatchDev& b, const relserve_layer& L, const void* h, const float* h_scale, const void* w_qkv,
                                     const float* w_scale, void* q_out, void* k_pages, void* v_pages, hipStream_t s, float* accum,
                                     bool w_packed, KvFormat kv) {
    if (b.T == 0) return hipSuccess;
    if ((int64_t)b.T * L.cfg.hidden >= ((int64_t)1 << 31) || (int64_t)L.qkv_dim * L.cfg.hidden >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    GemmArgs p{};
    set_qkv(p, b, L, h, w_qkv, q_out, k_pages, v_pages, kv, accum, w_packed);
    if (hipError_t e = set_int8(p, h_scale, w_scale)) return e;
    if (const int tile = rows_tile(p, EPI_QKV_ROPE))
        return L.cfg.head_dim == 128 ? run_rows<EPI_QKV_ROPE, 128>(p, s, tile) : run_rows<EPI_QKV_ROPE, 64>(p, s, tile);
    return run_qkv(p, L.cfg.head_dim, s);
}

}  // namespace relserve
