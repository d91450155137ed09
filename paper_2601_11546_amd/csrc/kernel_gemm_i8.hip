// int8 projections: out[t, n] = sum_k a[t, k] w[n, k] * (w_scale[n] * a_scale[t]) of 8-bit integers, summed exactly in 32 bits: the kernels of
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

// Which problems go this way, and on which tile.  Every workgroup loads its own activations beside its weights, so the time is a launch, two
// round trips and that traffic; the tiled kernels share both operands between more rows and columns, and win where the traffic gets long.
// us, tiled kernels -> this one (three sets of operands in turn; outputs x k):
//   T = 1: 5120 x 5120 10.5 -> 6.7, 15360 x 5120 17.8 -> 13.3, 5120 x 13824 17.0 -> 12.4, SwiGLU 27648 x 5120 26.6 -> 24.5; T = 8: 8192 x 28672 42.6 -> 38.3
//   T = 24: 5120 x 5120 12.3 -> 7.3, 15360 x 5120 19.9 -> 14.0, 5120 x 13824 19.1 -> 13.2; but 5120 x 27648 (283 MB) 30.5 -> 39.3, SwiGLU 57344 x 8192 76 -> 86
//   T = 40: 5120 x 13824 19.9 -> 15.8; 56: 15360 x 5120 22.0 -> 16.7
//   T = 128: 15360 x 5120 27.6 -> 23.7, SwiGLU 11264 x 5120 27.2 -> 18.9, 8192 x 8192 24.3 -> 19.9; but 5120 x 13824 (354 MB) 25.4 -> 27.5;
//   100: 10240 x 8192 (252 MB) 24.8 -> 27.7; 256: 5120 x 5120 23.7 -> 19.2; 400: 4096 x 4096 22.7 -> 18.2; 520 (two rounds of tiles) 24.6 -> 30.2
//   T = 333: 1004 x 1152 12.2 -> 5.0; 500: 2048 x 2048 15.9 -> 9.4; 700: 2560 x 2560 21.5 -> 14.8; 2000: 2048 x 512 17.2 -> 12.2; but SwiGLU
//   2816 x 512 at 1500 (104 MB) 8.6 -> 11.8
// Tiles: as few fragments of tokens as they need up to 64 tokens.  With four, slices two deep where a CU gets one workgroup, else one deep and three
// workgroups (2000 x 2048 x 512 20.7, 12.2); four fragments of features for long k where they still fill the chip (64 x 10240 x 5120 17.0, 13.8).
// More tokens: those tiles while their traffic is short, else 128 tokens a tile, in one round.
enum { ROWS_NONE = 0, ROWS_16, ROWS_32, ROWS_64, ROWS_64_SHALLOW, ROWS_64_WIDE, ROWS_128, ROWS_128_WIDE };
int rows_tile(const GemmArgs& p, int epi) {
    if (forced_cand() >= 0) return ROWS_NONE;
    const bool paired = epi == EPI_SWIGLU || epi == EPI_QKV_ROPE, swiglu = epi == EPI_SWIGLU;
    const int64_t cols = swiglu ? 2 * (int64_t)p.n_half : p.N, k_bytes = 2 * (int64_t)p.K;
    auto tiles = [&](int fn, int tm) { return (int64_t)((p.T + 16 * tm - 1) / (16 * tm)) * (paired ? (cols / 2 + 8 * fn - 1) / (8 * fn) : (cols + 16 * fn - 1) / (16 * fn)); };
    auto traffic_mb = [&](int fn, int tm) { return tiles(fn, tm) * 16 * (fn + tm) * k_bytes >> 20; };
    auto fills = [&](int fn, int tm) { return tiles(fn, tm) >= 150 && tiles(fn, tm) <= 256; };   // one round of workgroups, most CUs busy
    auto by_64 = [&] { return tiles(2, 4) > 256 ? ROWS_64_SHALLOW : tiles(2, 4) > 128 ? ROWS_64 : ROWS_32; };
    if (p.T <= 16) return traffic_mb(2, 1) <= (swiglu ? 256 : 400) ? ROWS_16 : ROWS_NONE;
    if (p.T <= 32) return traffic_mb(2, 2) <= 200 ? ROWS_32 : ROWS_NONE;
    if (p.T <= 64) {
        if (k_bytes >= 4096 && tiles(4, 4) >= 160 && traffic_mb(4, 4) <= 200) return ROWS_64_WIDE;
        return traffic_mb(2, 4) <= 224 ? by_64() : ROWS_NONE;
    }
    if (traffic_mb(2, 4) <= (swiglu ? 80 : 128)) return by_64();
    if (k_bytes >= 2048 && fills(4, 8) && traffic_mb(4, 8) <= 240) return ROWS_128_WIDE;
    if (k_bytes >= 2048 && fills(2, 8) && traffic_mb(2, 8) <= 340) return ROWS_128;
    return ROWS_NONE;
}

// Weights that the last-level cache (256 MB) cannot hold beside others are read with the non-temporal hint: SwiGLU 27648 x 5120 (141 MB) 27.2 ->
// 24.5 us.  Smaller ones may still be there from the last call: 5120 x 13824 at T = 24 13.2 with three sets in turn, 21.2 with the hint; from memory
// (ten sets) 21.2 and 22.3, 15360 x 5120 at T = 1 15.6 and 14.6.  Only the tile of 16 tokens has the form with
// the hint: the others' rules end at weights of 100 MB.
constexpr int64_t kFarWeights = (int64_t)96 << 20;

template <int EPI, int D = 0>
hipError_t run_rows(const GemmArgs& p, hipStream_t s, int tile) {
    const bool far = 2 * (int64_t)p.N * p.K >= kFarWeights;
    switch (tile) {
        case ROWS_16: return far ? launch_rows<EPI, D, 2, 1, 4, 3, true>(p, s) : launch_rows<EPI, D, 2, 1, 4, 3, false>(p, s);
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
