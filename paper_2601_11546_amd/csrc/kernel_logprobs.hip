// Log probabilities of rows of logits: of given tokens, the row's entropy, and its top alternatives.
//   m = max x,  Z = sum e^(x - m),  log p(i) = (x[i] - m) - log Z,  H = log Z - (sum (x - m) e^(x - m)) / Z
// One pass: a thread keeps the running (m, c, s, E): how often it has met its largest value, the sum over the others, and sum (x - m) e^(x - m).
// Z = c + s and log Z = log1p((c - 1) + s), so that a nearly sure row keeps the digits of a log probability next to 0; both terms of H are
// positive, so nothing cancels in it.
//
// A workgroup of 256 threads holds 8192 values of a row at a time, 32 a thread, all loaded at once.  Its alternatives are kept as 64-bit keys,
// the value's bits in an order of whole numbers above the id's complement: larger value first, the lower id among equals, all keys different.
// Of a chunk only the values that can be among the first n_top are looked at: those from the n_top-th largest of its 256 threads' best on (found among
// the groups of four lanes first), so at most 32 n_top of them, whatever the row.
//
// Few rows are cut into parts of whole chunks for several workgroups, whose results a second launch joins in their order.
#include <algorithm>

#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

constexpr int THREADS = 256, PER = 32, CHUNK = THREADS * PER, MAX_TOP = 32;
constexpr float LOG2E = 1.4426950408889634f;

struct Sums {
    float m, c, s, e;   // largest value, how often, sum of e^(x - m) over the others, sum of (x - m) e^(x - m)
};

// What a sum of smaller values counts for at m: nothing if it holds none, a NaN if it holds one.
__device__ __forceinline__ void move_to(Sums& a, float m) {
    if (a.m == m) return;
    const float all = a.m == -INFINITY ? (a.s != a.s ? a.s : 0.0f) : a.c + a.s, d = a.m == -INFINITY ? 0.0f : a.m - m;
    const float f = a.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(d * LOG2E);
    a.e = (a.m == -INFINITY ? 0.0f : __builtin_fmaf(fmaxf(d, -200.0f), all, a.e)) * f;
    a.s = all * f;
    a.c = 0.0f;
    a.m = m;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m);
    move_to(a, m);
    move_to(b, m);
    return {m, a.c + b.c, a.s + b.s, a.e + b.e};
}
// log Z; a row with a NaN, an infinity or no finite value has no distribution
__device__ __forceinline__ float log_z(const Sums& a) { return a.m > -INFINITY && a.m < INFINITY ? log1pf((a.c - 1.0f) + a.s) : NAN; }

__device__ __forceinline__ uint32_t ordered(float v) {   // whole numbers in the order of the values, above 0 for every number
    const uint32_t b = __float_as_uint(v + 0.0f);          // (one zero)
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t id) { return v != v ? 0 : (uint64_t)ordered(v) << 32 | (uint32_t)~id; }

struct LogprobsLaunch {
    LogprobsArgs a;
    int32_t parts, chunks;   // parts of a row, chunks of all
    Sums* part_sums;         // [rows, parts]
    uint64_t* part_keys;     // [rows, parts, n_top]
};

// What is left to do when a row's sums and keys are known.
__device__ __forceinline__ void write_row(const LogprobsArgs& a, int64_t row, const Sums& z, const uint64_t* keys) {
    const float lz = log_z(z);
    const int tid = threadIdx.x;
    if (tid == 0 && a.entropy) a.entropy[row] = lz - z.e / (z.c + z.s);
    for (int j = tid; j < a.n_ids; j += THREADS) {
        const int32_t id = a.ids[row * a.n_ids + j];
        float lp = NAN;
        if (id >= 0 && id < a.vocab) {
            const int64_t at = row * a.pitch + id;
            const float x = a.is_f32 ? static_cast<const float*>(a.logits)[at] : bf16_to_f32(static_cast<const uint16_t*>(a.logits)[at]);
            lp = (x - z.m) - lz;
        }
        a.logprobs[row * a.n_ids + j] = lp;
    }
    if (tid < a.n_top) {
        const uint64_t k = keys[tid];
        a.top_ids[row * a.n_top + tid] = k ? (int32_t)~(uint32_t)k : -1;
        a.top_logprobs[row * a.n_top + tid] = lz != lz ? lz : k ? (value_of((uint32_t)(k >> 32)) - z.m) - lz : -INFINITY;
    }
}

// The sums of all threads, in every thread.
__device__ __forceinline__ Sums all_sums(Sums z, Sums* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) z = joined(z, Sums{__shfl_xor(z.m, o, 64), __shfl_xor(z.c, o, 64), __shfl_xor(z.s, o, 64), __shfl_xor(z.e, o, 64)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = z;
    __syncthreads();
    z = red[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) z = joined(z, red[w]);
    return z;
}

// The n largest of the keys in cand[0 .. count), in order, to list[0 .. n) (zeros behind them); all keys are different.
__device__ __forceinline__ void largest_keys(const uint64_t* cand, int count, uint64_t* list, int n) {
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const uint64_t k = cand[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += cand[j] > k;
        if (rank < n) list[rank] = k;
    }
}

template <bool F32, bool TOP>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(LogprobsLaunch p) {
    constexpr int V = F32 ? 4 : 8, LOADS = PER / V;   // values of a load
    typedef float f32_quad __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint16_t bf16_eight __attribute__((ext_vector_type(8), aligned(2)));
    __shared__ Sums red[THREADS / 64];
    __shared__ uint64_t list[TOP ? MAX_TOP : 1], best[TOP ? THREADS : 1], cand[TOP ? MAX_TOP * (PER + 1) : 1], floor_key;
    __shared__ uint32_t group[TOP ? 64 : 1];
    __shared__ int n_best, n_cand;
    const int tid = threadIdx.x, lane = tid & 63, vocab = p.a.vocab, n_top = p.a.n_top;
    const int64_t row = blockIdx.x / p.parts;
    const int part = blockIdx.x % p.parts, c0 = (int)((int64_t)p.chunks * part / p.parts), c1 = (int)((int64_t)p.chunks * (part + 1) / p.parts);
    const char* const base = static_cast<const char*>(p.a.logits) + row * p.a.pitch * (F32 ? 4 : 2);
    if (TOP && tid < MAX_TOP) list[tid] = 0;
    if (TOP && tid == 0) n_best = n_cand = 0;
    uint64_t last = 0;   // the n_top-th key so far
    Sums z{-INFINITY, 0.f, 0.f, 0.f};
    for (int c = c0; c < c1; ++c) {
        float x[PER];
        const int first = c * CHUNK + tid * V;   // of load l: first + l * THREADS * V
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
            const int at = first + l * (THREADS * V);
            if (at + V <= vocab) {
                if constexpr (F32) {
                    const f32_quad q = *reinterpret_cast<const f32_quad*>(base + (int64_t)at * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[l * V + i] = q[i];
                } else {
                    const bf16_eight q = *reinterpret_cast<const bf16_eight*>(base + (int64_t)at * 2);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[l * V + i] = bf16_to_f32(q[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    x[l * V + i] = -INFINITY;
                    if (at + i < vocab) x[l * V + i] = F32 ? reinterpret_cast<const float*>(base)[at + i] : bf16_to_f32(reinterpret_cast<const uint16_t*>(base)[at + i]);
                }
            }
        }
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i) m = fmaxf(m, x[i]);
        move_to(z, fmaxf(z.m, m));
        {
            const float from = z.m == -INFINITY ? 0.0f : z.m;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float d = x[i] - from, e = __builtin_amdgcn_exp2f(d * LOG2E);
                const bool top = x[i] == z.m;
                z.c += top ? 1.0f : 0.0f;
                z.s += top ? 0.0f : e;
                z.e = __builtin_fmaf(fmaxf(d, -200.0f), e, z.e);
            }
        }
        if constexpr (TOP) {
            // the thread's best key (elements of a thread are in the order of their ids)
            int at = -1;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i) at = x[i] == m ? i : at;
            const int id = first + at / V * (THREADS * V) + at % V;
            const uint64_t mine = at < 0 || id >= vocab ? 0 : key_of(m, id);
            // from which value on: the n_top-th largest of the groups of four lanes, by its upper half
            uint32_t g = mine > last ? (uint32_t)(mine >> 32) : 0;
            g = max(g, (uint32_t)__shfl_xor((int)g, 1, 64));
            g = max(g, (uint32_t)__shfl_xor((int)g, 2, 64));
            if ((lane & 3) == 0) group[tid >> 2] = g;
            __syncthreads();
            const uint32_t u = group[lane];
            uint32_t from = 0;
            for (int b = 31; b >= 16; --b)
                if (__popcll(__ballot(u >= (from | 1u << b))) >= n_top) from |= 1u << b;
            if (mine > last && (uint32_t)(mine >> 32) >= from) best[atomicAdd(&n_best, 1)] = mine;
            __syncthreads();
            const int count = n_best;
            if (count == 0) continue;   // (nothing was added: the counter stays 0; group is written again behind a barrier that follows its reads)
            uint64_t low = max(last + 1, (uint64_t)from << 32);   // (of at most n_top threads all that can count; from > 0 takes n_top groups)
            if (count > n_top) {
                if (tid < count) {
                    const uint64_t k = best[tid];
                    int rank = 0;
                    for (int j = 0; j < count; ++j) rank += best[j] > k;
                    if (rank == n_top - 1) floor_key = k;
                }
                __syncthreads();
                low = floor_key;
            }
            if (mine >= low) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int e = first + i / V * (THREADS * V) + i % V;
                    const uint64_t k = e < vocab ? key_of(x[i], e) : 0;
                    if (k >= low) cand[atomicAdd(&n_cand, 1)] = k;
                }
            }
            if (tid < n_top && list[tid]) cand[atomicAdd(&n_cand, 1)] = list[tid];
            __syncthreads();
            const int total = n_cand;
            if (tid < MAX_TOP) list[tid] = 0;
            __syncthreads();
            if (tid == 0) n_best = n_cand = 0;
            largest_keys(cand, total, list, n_top);
            __syncthreads();
            last = list[n_top - 1];
        }
    }
    z = all_sums(z, red);
    if (p.parts == 1) {
        write_row(p.a, row, z, list);
        return;
    }
    const int64_t slot = row * p.parts + part;
    if (tid == 0) p.part_sums[slot] = z;
    if (TOP && tid < n_top) p.part_keys[slot * n_top + tid] = list[tid];
}

// Joins the parts of a row.
__global__ void __launch_bounds__(THREADS) logprobs_join_kernel(LogprobsLaunch p) {
    extern __shared__ uint64_t keys[];   // [parts * n_top]
    __shared__ Sums red[THREADS / 64];
    __shared__ uint64_t list[MAX_TOP];
    const int tid = threadIdx.x, n = p.parts * p.a.n_top;
    const int64_t row = blockIdx.x;
    Sums z{-INFINITY, 0.f, 0.f, 0.f};
    for (int i = tid; i < p.parts; i += THREADS) z = joined(z, p.part_sums[row * p.parts + i]);
    for (int i = tid; i < n; i += THREADS) keys[i] = p.part_keys[row * n + i];
    if (tid < MAX_TOP) list[tid] = 0;
    z = all_sums(z, red);
    for (int i = tid; i < n; i += THREADS) {
        const uint64_t k = keys[i];
        if (!k) continue;
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += keys[j] > k;
        if (rank < p.a.n_top) list[rank] = k;
    }
    __syncthreads();
    write_row(p.a, row, z, list);
}

constexpr int kMaxParts = 64;   // of a row: their keys lie in the joining workgroup's LDS

int32_t parts_of(int64_t rows, int64_t vocab) {
    const int64_t chunks = (vocab + CHUNK - 1) / CHUNK;
    return (int32_t)std::min<int64_t>({chunks, kMaxParts, std::max<int64_t>(1, 512 / std::max<int64_t>(1, rows))});
}

}  // namespace

int64_t logprobs_scratch_bytes(int64_t rows, int64_t vocab, int64_t n_top) {
    const int64_t parts = parts_of(rows, vocab);
    return parts > 1 ? rows * parts * ((int64_t)sizeof(Sums) + 8 * n_top) : 0;
}

hipError_t launch_logprobs(const LogprobsArgs& args, hipStream_t s) {
    if (args.rows == 0) return hipSuccess;
    LogprobsLaunch p{args, args.scratch ? parts_of(args.rows, args.vocab) : 1, (int32_t)(((int64_t)args.vocab + CHUNK - 1) / CHUNK), nullptr, nullptr};
    p.part_sums = static_cast<Sums*>(args.scratch);
    p.part_keys = reinterpret_cast<uint64_t*>(p.part_sums + (int64_t)args.rows * p.parts);
    const dim3 grid((unsigned)(args.rows * p.parts));
    if (args.is_f32 && args.n_top) logprobs_kernel<true, true><<<grid, dim3(THREADS), 0, s>>>(p);
    else if (args.is_f32) logprobs_kernel<true, false><<<grid, dim3(THREADS), 0, s>>>(p);
    else if (args.n_top) logprobs_kernel<false, true><<<grid, dim3(THREADS), 0, s>>>(p);
    else logprobs_kernel<false, false><<<grid, dim3(THREADS), 0, s>>>(p);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.parts > 1) {
        logprobs_join_kernel<<<dim3((unsigned)args.rows), dim3(THREADS), (size_t)p.parts * args.n_top * 8, s>>>(p);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace relserve
