// Log probabilities of rows of logits: of given tokens, the row's entropy, and its top alternatives.
//   m = max x,  Z = sum e^(x - m),  log p(i) = (x[i] - m) - log Z,  H = log Z - (sum (x - m) e^(x - m)) / Z
// One pass: a thread keeps the running (m, c, s, E): how often it has met its wave's largest value, the sum over the others, and
// sum (x - m) e^(x - m).  Z = c + s and log Z = log1p((c - 1) + s), so that a nearly sure row keeps the digits of a log probability next to 0; both
// terms of H are positive, so nothing cancels in it.
//
// A workgroup holds 32 values a thread of a row at a time (8192 of 256 threads) while the next ones are on their way.  Nothing in that pass waits for
// another wave.  On bf16 the vector units issue in 88 % of the time that a CU holds waves, which is 74 % of the launch (2048 x 50257 without alternatives, 49 us,
// five or six workgroups a CU; 2560 rows the same), twelve instructions a value in all; on fp32 in 54 %, and the row's bytes come at 5.6 TB/s (73 us).  A chunk
// that does not reach its wave's largest value so far, most of a long row's, therefore takes seven instructions a value instead of ten, and loads behind the row's end
// take none: 2048 x 50257 bf16 57 -> 49 us, 600 x 1000000 285 -> 243.
// What a row's last loads have too early is shifted out where they are used, not where they are issued (4096 x 32000 bf16 with alternatives 74.0 -> 66.5).
//
// Alternatives are 64-bit keys, the value's bits in an order of whole numbers above the id's complement: larger value first, the lower id among
// equals, all keys different.  A thread remembers of up to sixteen stretches of its chunks the upper half of each one's largest value.  Behind the pass
// the largest values of 64 groups of lanes give a bound that n_top values reach at least; the loads of the stretches that reach it are dealt out
// to all threads once more, and what reaches the bound is gathered and ranked.  (All loads of a thread that reaches it, 16 bytes of a line each, were a
// second pass over the row's lines: 2048 x 50257 fp32 with 20 alternatives 102 us, 85 so; bf16 67, 64.)  Where ties let too much reach it, the bound
// is the n_top-th of the threads' best keys.
//
// Few rows are cut into parts of whole chunks for several workgroups, whose results a second launch joins in their order.
#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "relserve_internal.h"

namespace relserve {

namespace {

constexpr int PER = 32, MAX_TOP = 32;      // values a thread holds at a time; alternatives
constexpr int FEW = 256, MANY = 1024;      // threads of a workgroup
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float kPlainMost = 0x1p14f;      // largest values whose product with LOG2E lacks so little that exp2 of it is next to 1

struct Sums {
    float m, c, s, e;   // largest value, how often, sum of e^(x - m) over the others, sum of (x - m) e^(x - m)
};

// What a sum of smaller values counts for at m: nothing if it holds none, a NaN if it holds one.
__device__ __forceinline__ void move_to(Sums& a, float m) {
    if (a.m == m) return;
    const bool none = a.m == -INFINITY;
    const float all = none ? (a.s != a.s ? a.s : 0.0f) : a.c + a.s, d = none ? 0.0f : a.m - m;
    const float f = none ? 0.0f : __builtin_amdgcn_exp2f(d * LOG2E);
    a.e = (none ? 0.0f : __builtin_fmaf(fmaxf(d, -200.0f), all, a.e)) * f;
    a.s = all * f;
    a.c = 0.0f;
    a.m = m;
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

__device__ __forceinline__ float logit(const LogprobsArgs& a, int64_t at) {
    return a.is_f32 ? static_cast<const float*>(a.logits)[at] : bf16_to_f32(static_cast<const uint16_t*>(a.logits)[at]);
}

// The logit of the row's given token that this thread answers for first (fetched ahead of what it waits for).
struct Given { float x; bool valid; };
__device__ __forceinline__ Given given(const LogprobsArgs& a, int64_t row, int j) {
    if (j >= a.n_ids) return {0.0f, false};
    const int32_t id = a.ids[row * a.n_ids + j];
    const bool valid = id >= 0 && id < a.vocab;
    return {valid ? logit(a, row * a.pitch + id) : 0.0f, valid};
}

// What is left to do when a row's sums and keys are known.
template <int THREADS>
__device__ __forceinline__ void write_row(const LogprobsArgs& a, int64_t row, const Sums& z, const uint64_t* keys, Given first) {
    const float lz = log_z(z);
    const int tid = threadIdx.x;
    if (tid == 0 && a.entropy) a.entropy[row] = lz - z.e / (z.c + z.s);
    for (int j = tid; j < a.n_ids; j += THREADS) {
        const Given v = j == tid ? first : given(a, row, j);
        a.logprobs[row * a.n_ids + j] = v.valid ? (v.x - z.m) - lz : NAN;
    }
    if (tid < a.n_top) {
        const uint64_t k = keys[tid];
        a.top_ids[row * a.n_top + tid] = k ? (int32_t)~(uint32_t)k : -1;
        a.top_logprobs[row * a.n_top + tid] = lz != lz ? lz : k ? (value_of((uint32_t)(k >> 32)) - z.m) - lz : -INFINITY;
    }
}

// A value of another lane: 0x120 + n rotates rows of 16 lanes; 0x142 gives lane 15 of a row to the next one's lanes, 0x143 lane 31 to the upper half's;
// rows outside the mask get `old`.
template <int CTRL, int ROWS>
__device__ __forceinline__ float other_lane(float old, float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// The wave's largest value, the same scalar in every lane; all lanes call it.
__device__ __forceinline__ float wave_largest(float m) {
    m = fmaxf(m, other_lane<0x128, 0xf>(m, m));
    m = fmaxf(m, other_lane<0x124, 0xf>(m, m));
    m = fmaxf(m, other_lane<0x122, 0xf>(m, m));
    m = fmaxf(m, other_lane<0x121, 0xf>(m, m));
    m = fmaxf(m, other_lane<0x142, 0xa>(m, m));
    m = fmaxf(m, other_lane<0x143, 0xc>(m, m));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m), 63));
}
// The sum of all lanes, in the last one.
__device__ __forceinline__ float wave_total(float v) {
    v += other_lane<0x128, 0xf>(0.0f, v);
    v += other_lane<0x124, 0xf>(0.0f, v);
    v += other_lane<0x122, 0xf>(0.0f, v);
    v += other_lane<0x121, 0xf>(0.0f, v);
    v += other_lane<0x142, 0xa>(0.0f, v);
    v += other_lane<0x143, 0xc>(0.0f, v);
    return v;
}

// The sums of all threads, in every thread: moved to the largest value of all, then added.  A wave's own have one m.
template <int THREADS>
__device__ __forceinline__ Sums all_sums(Sums z, float4* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    z.c = wave_total(z.c);
    z.s = wave_total(z.s);
    z.e = wave_total(z.e);
    if (lane == 63) red[wave] = make_float4(z.m, z.c, z.s, z.e);
    __syncthreads();
    Sums part[THREADS / 64];
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const float4 r = red[w];
        part[w] = {r.x, r.y, r.z, r.w};
        m = fmaxf(m, r.x);
    }
    Sums all{m, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        move_to(part[w], m);
        all.c += part[w].c;
        all.s += part[w].s;
        all.e += part[w].e;
    }
    return all;
}

// How many of keys[0 .. count) are larger than k; zeros stand behind the last one up to a multiple of eight.
__device__ __forceinline__ int larger_keys(const uint64_t* keys, int count, uint64_t k) {
    int rank = 0;
    for (int j = 0; j < count; j += 8) {
#pragma unroll
        for (int q = 0; q < 8; ++q) rank += keys[j + q] > k;
    }
    return rank;
}

// 128 bits moved down by `bits`, with copies of fill behind them.
__device__ __forceinline__ uint4 behind(const uint4& q, int bits, uint32_t fill) {
    const uint64_t lo = (uint64_t)q.y << 32 | q.x, hi = (uint64_t)q.w << 32 | q.z, f = (uint64_t)fill << 32 | fill;
    const int b = bits & 63;
    const uint64_t a = bits < 64 ? lo : bits < 128 ? hi : f, c = bits < 64 ? hi : f;   // what lies b bits below the result
    const uint64_t x = b ? a >> b | c << (64 - b) : a, y = b ? c >> b | f << (64 - b) : c;
    return make_uint4((uint32_t)x, (uint32_t)(x >> 32), (uint32_t)y, (uint32_t)(y >> 32));
}

constexpr int kStretches = 16, kReaching = 1024;   // of a thread; stretches whose loads are dealt out at most
constexpr int kGathered = 2048;   // keys that a workgroup gathers at most: two chunks' of 32 alternatives

template <int THREADS, bool F32, bool TOP, bool ONE>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(LogprobsLaunch p) {
    constexpr int CHUNK = THREADS * PER, GROUP = THREADS / 64;   // values of a chunk; lanes of a group: 64 groups
    constexpr int V = F32 ? 4 : 8, LOADS = PER / V;   // values of a load
    typedef float f32_quad __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint16_t bf16_eight __attribute__((ext_vector_type(8), aligned(2)));
    __shared__ float4 red[THREADS / 64];
    __shared__ uint64_t list[TOP ? MAX_TOP : 1], best[TOP ? THREADS + 8 : 1], cand[TOP ? kGathered + MAX_TOP + 8 : 1], floor_key;
    __shared__ uint32_t group[TOP ? 64 : 1];
    __shared__ uint16_t stretch[TOP && !ONE ? kStretches * THREADS : 1], who[TOP && !ONE ? kReaching : 1];
    __shared__ int n_best, n_cand, n_who;
    const int tid = threadIdx.x, lane = tid & 63, vocab = p.a.vocab, n_top = p.a.n_top;
    const int64_t row = blockIdx.x / p.parts;
    const int part = blockIdx.x % p.parts, c0 = (int)((int64_t)p.chunks * part / p.parts), c1 = ONE ? c0 + 1 : (int)((int64_t)p.chunks * (part + 1) / p.parts);
    const char* const base = static_cast<const char*>(p.a.logits) + row * p.a.pitch * (F32 ? 4 : 2);
    // a chunk as it is loaded: quads of fp32, or eights of bf16; entries behind the vocabulary are -infinity
    struct Raw { uint4 q[LOADS]; };
    constexpr uint32_t FILL = F32 ? 0xff800000u : 0xff80ff80u;
    auto whole = [&](int from) __attribute__((always_inline)) {
        if constexpr (F32) return __builtin_bit_cast(uint4, *reinterpret_cast<const f32_quad*>(base + (int64_t)from * 4));
        else return __builtin_bit_cast(uint4, *reinterpret_cast<const bf16_eight*>(base + (int64_t)from * 2));
    };
    // how many of a chunk's loads lie in the row (an eighth of 50257 values is one load of a seventh chunk)
    auto loads_of = [&](int c) { return (int)min<int64_t>(LOADS, (vocab - (int64_t)c * CHUNK + THREADS * V - 1) / (THREADS * V)); };
    // (loads past the row's end are moved back to it)
    auto load = [&](int c, Raw& r) __attribute__((always_inline)) {
        const int at = c * CHUNK + tid * V;
        if (vocab >= V) {
#pragma unroll
            for (int l = 0; l < LOADS; ++l) r.q[l] = whole(min(at + l * (THREADS * V), vocab - V));
        } else {
            auto one = [&](int i) -> uint32_t {
                if (i >= vocab) return F32 ? 0xff800000u : 0xff80u;
                return F32 ? reinterpret_cast<const uint32_t*>(base)[i] : reinterpret_cast<const uint16_t*>(base)[i];
            };
            auto word = [&](int i) { return F32 ? one(at + i) : one(at + 2 * i) | one(at + 2 * i + 1) << 16; };
            r.q[0] = make_uint4(word(0), word(1), word(2), word(3));
#pragma unroll
            for (int l = 1; l < LOADS; ++l) r.q[l] = make_uint4(FILL, FILL, FILL, FILL);
        }
    };
    auto values = [&](int c, Raw& r, float (&x)[PER]) __attribute__((always_inline)) {
        if (vocab >= V && (c + 1) * (int64_t)CHUNK > vocab) {   // what moved loads have too early is shifted out
            const int at = c * CHUNK + tid * V, here = ONE ? LOADS : loads_of(c);
#pragma unroll
            for (int l = 0; l < LOADS; ++l)
                r.q[l] = l < here ? behind(r.q[l], max(at + l * (THREADS * V) + V - vocab, 0) * (128 / V), FILL) : make_uint4(FILL, FILL, FILL, FILL);
        }
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
            const uint32_t u[4] = {r.q[l].x, r.q[l].y, r.q[l].z, r.q[l].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (F32) x[4 * l + i] = __uint_as_float(u[i]);
                else x[8 * l + 2 * i] = bf16_lo(u[i]), x[8 * l + 2 * i + 1] = bf16_hi(u[i]);
            }
        }
    };
    auto id_of = [&](int c, int i) { return c * CHUNK + tid * V + i / V * (THREADS * V) + i % V; };

    const Given first = p.parts == 1 ? given(p.a, row, tid) : Given{0.f, false};
    Sums z{-INFINITY, 0.f, 0.f, 0.f};   // (m is the wave's, or, of a chunk alone, the thread's)
    float most_x = -INFINITY;           // the thread's largest value, and its chunk
    int best_chunk = c0, at_stretch = 0, left = 0;   // (left: chunks of the stretch behind this one)
    const int per_stretch = (c1 - c0 + kStretches - 1) / kStretches;
    float x[PER], stretch_most = -INFINITY;
    Raw next;
    load(c0, next);
    for (int c = c0; c < c1; ++c) {
        values(c, next, x);
        if (!ONE && c + 1 < c1) load(c + 1, next);
        const int here = ONE ? LOADS : loads_of(c);
        auto take = [&](auto whole_chunk) __attribute__((always_inline)) {
            auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
                for (int l = 0; l < LOADS; ++l)
                    if (decltype(whole_chunk)::value || l < here)
#pragma unroll
                        for (int i = l * V; i < (l + 1) * V; ++i) f(x[i]);
            };
            float m = -INFINITY;
            each([&](float v) __attribute__((always_inline)) { m = fmaxf(m, v); });
            if (m > most_x) most_x = m, best_chunk = c;
            if constexpr (TOP && !ONE) {
                stretch_most = left > 0 ? fmaxf(stretch_most, m) : m;
                left = left > 0 ? left - 1 : per_stretch - 1;
                stretch[at_stretch * THREADS + tid] = (uint16_t)(stretch_most > -INFINITY ? ordered(stretch_most) >> 16 : 0);
                at_stretch += left == 0;
            }
            if (!ONE && __builtin_fabsf(z.m) < kPlainMost && __ballot(m >= z.m) == 0) {
                // nothing reaches the wave's largest value: nothing is counted, and the exponent is one multiply-add
                const float high = z.m * LOG2E, low = __builtin_fmaf(z.m, LOG2E, -high), up = __builtin_amdgcn_exp2f(-low);
                float sum = 0.0f, sum_d = 0.0f;
                each([&](float v) __attribute__((always_inline)) {
                    const float d = __builtin_fmaf(v, LOG2E, -high), e = __builtin_amdgcn_exp2f(d);
                    sum += e;
                    sum_d = __builtin_fmaf(fmaxf(d, -200.0f), e, sum_d);
                });
                z.s = __builtin_fmaf(sum, up, z.s);
                z.e = __builtin_fmaf(__builtin_fmaf(-low, sum, sum_d) * LN2, up, z.e);
                return;
            }
            move_to(z, fmaxf(z.m, ONE ? m : wave_largest(m)));
            const float from = z.m == -INFINITY ? 0.0f : z.m;
            int others = 0;
            float sum = 0.0f, sum_e = 0.0f;   // of the chunk, as above: a chain through all of a thread's values drifts with equal ones
            each([&](float v) __attribute__((always_inline)) {
                const float d = v - from, e = __builtin_amdgcn_exp2f(d * LOG2E);
                const bool other = v != z.m;
                others += other;
                sum += other ? e : 0.0f;
                sum_e = __builtin_fmaf(fmaxf(d, -200.0f), e, sum_e);
            });
            z.s += sum;
            z.e += sum_e;
            z.c += (float)((decltype(whole_chunk)::value ? PER : here * V) - others);
        };
        if (here == LOADS) take(std::true_type{});
        else take(std::false_type{});
    }
    if constexpr (ONE) move_to(z, wave_largest(z.m));
    if constexpr (TOP) {
        if (tid < MAX_TOP) list[tid] = 0;
        best[tid] = 0;
        if (tid < 8) best[THREADS + tid] = 0;
        if (tid == 0) n_best = n_cand = n_who = 0;
        // From which value on: the n_top-th largest of the 64 groups of lanes, by its upper half (0: fewer groups have a number above -infinity).
        const uint32_t most = most_x > -INFINITY ? ordered(most_x) : 0;
        uint32_t g = most;
#pragma unroll
        for (int o = 1; o < GROUP; o *= 2) g = max(g, (uint32_t)__shfl_xor((int)g, o, 64));
        if (tid % GROUP == 0) group[tid / GROUP] = g;
        __syncthreads();
        const uint32_t u = group[lane];
        uint32_t from = 0;
#pragma unroll
        for (int b = 31; b >= 16; --b)
            if (__popcll(__ballot(u >= (from | 1u << b))) >= n_top) from |= 1u << b;
        auto gather = [&](float v, int id, uint64_t low) __attribute__((always_inline)) {
            const uint64_t key = key_of(v, id);
            if (id >= vocab || key < low) return;
            const int at = atomicAdd(&n_cand, 1);
            if (at < kGathered) cand[at] = key;
        };
        // cand[0 .. n_cand) to its n_top largest in list; all threads, behind a barrier that closes the gathering
        auto cut = [&]() __attribute__((always_inline)) {
            const int total = n_cand;
            if (tid < 8) cand[total + tid] = 0;
            if (tid < MAX_TOP) list[tid] = 0;
            __syncthreads();
            if (tid == 0) n_cand = 0;
            for (int i = tid; i < total; i += THREADS) {
                const uint64_t k = cand[i];
                const int rank = larger_keys(cand, total, k);
                if (rank < n_top) list[rank] = k;
            }
            __syncthreads();
        };
        bool done = false;
        if (from > 0) {   // gather all values from there on: some more than n_top, as a rule
            const float bound = value_of(from);
            const uint64_t low = (uint64_t)from << 32;
            if constexpr (ONE) {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (x[i] >= bound) gather(x[i], id_of(c0, i), low);
            } else {
                // the loads of the stretches that have such values, dealt out to all
                if (most >= from) {
#pragma unroll
                    for (int i = 0; i < kStretches; ++i)
                        if (i * per_stretch < c1 - c0 && stretch[i * THREADS + tid] >= from >> 16) {
                            const int slot = atomicAdd(&n_who, 1);
                            if (slot < kReaching) who[slot] = (uint16_t)(i * THREADS + tid);
                        }
                }
                __syncthreads();
                const int n = min(n_who, kReaching), loads = n * LOADS * per_stretch;
                constexpr int AT_ONCE = 4;
                const float one_nth = 1.0f / (float)n;
                for (int w0 = tid; w0 < loads; w0 += AT_ONCE * THREADS) {
                    uint4 q[AT_ONCE];
                    int ids[AT_ONCE];
#pragma unroll
                    for (int b = 0; b < AT_ONCE; ++b) {
                        const int w = min(w0 + b * THREADS, loads - 1);
                        int l = (int)((float)w * one_nth), rest = w - l * n;   // (the product may be next to the quotient)
                        if (rest < 0) --l, rest += n;
                        if (rest >= n) ++l, rest -= n;
                        const int at = who[rest], c = c0 + at / THREADS * per_stretch + l / LOADS;
                        ids[b] = c < c1 ? c * CHUNK + l % LOADS * (THREADS * V) + at % THREADS * V : vocab;
                        q[b] = whole(min(ids[b], vocab - V));   // (two chunks at least: more entries than V)
                    }
#pragma unroll
                    for (int b = 0; b < AT_ONCE; ++b) {
                        if (w0 + b * THREADS >= loads) break;
                        if (ids[b] + V > vocab) q[b] = behind(q[b], (ids[b] + V - vocab) * (128 / V), FILL);
                        const uint32_t words[4] = {q[b].x, q[b].y, q[b].z, q[b].w};
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float v = F32 ? __uint_as_float(words[i / (V / 4)]) : i % 2 ? bf16_hi(words[i / 2]) : bf16_lo(words[i / 2]);
                            if (v >= bound) gather(v, ids[b] + i, low);
                        }
                    }
                }
            }
            __syncthreads();
            done = n_cand <= kGathered && n_who <= kReaching;
            if (done) cut();
        }
        if (!done) {
            // Many equal values, or hardly any: the same from the n_top-th of the threads' best keys on, which at most 32 n_top keys of a chunk reach.
            __syncthreads();
            if (tid == 0) n_cand = 0;
            // the thread's best key (entries of a thread are in the order of their ids); one without a number above -infinity looks for the first -infinity
            int at = -1;
            for (int c = best_chunk; c < c1 && at < 0; ++c) {
                if constexpr (!ONE) {
                    load(c, next);
                    values(c, next, x);
                }
#pragma unroll
                for (int i = PER - 1; i >= 0; --i) at = x[i] == most_x ? i : at;
                best_chunk = c;
            }
            const int id = id_of(best_chunk, at);
            const uint64_t mine = at < 0 || id >= vocab ? 0 : key_of(most_x, id);
            if (mine && (uint32_t)(mine >> 32) >= from) best[atomicAdd(&n_best, 1)] = mine;
            __syncthreads();
            const int count = n_best;
            uint64_t low = max((uint64_t)1, (uint64_t)from << 32);   // (of at most n_top threads all that can count; from > 0 takes n_top groups)
            if (count > n_top) {
                if (tid < count) {
                    const uint64_t k = best[tid];
                    if (larger_keys(best, count, k) == n_top - 1) floor_key = k;
                }
                __syncthreads();
                low = floor_key;
            }
            const int at_once = ONE ? 1 : kGathered / (PER * n_top);   // chunks whose keys surely fit
            for (int c = c0; c < c1; c += at_once) {
                if (mine >= low) {
                    for (int k = c; k < min(c + at_once, c1); ++k) {
                        if constexpr (!ONE) {
                            load(k, next);
                            values(k, next, x);
                        }
#pragma unroll
                        for (int i = 0; i < PER; ++i) gather(x[i], id_of(k, i), low);
                    }
                }
                __syncthreads();
                if (c > c0 && tid < n_top && list[tid]) cand[atomicAdd(&n_cand, 1)] = list[tid];
                __syncthreads();
                cut();
                low = max(low, list[n_top - 1]);
            }
        }
    }
    z = all_sums<THREADS>(z, red);
    if (p.parts == 1) {
        write_row<THREADS>(p.a, row, z, list, first);
        return;
    }
    const int64_t slot = row * p.parts + part;
    if (tid == 0) p.part_sums[slot] = z;
    if (TOP && tid < n_top) p.part_keys[slot * n_top + tid] = list[tid];
}

// Joins the parts of a row.
__global__ void __launch_bounds__(FEW) logprobs_join_kernel(LogprobsLaunch p) {
    extern __shared__ uint64_t keys[];   // [parts * n_top], and zeros up to a multiple of eight
    __shared__ float4 red[FEW / 64];
    __shared__ uint64_t list[MAX_TOP];
    const int tid = threadIdx.x, n = p.parts * p.a.n_top;
    const int64_t row = blockIdx.x;
    Sums z{-INFINITY, 0.f, 0.f, 0.f};
    if (tid < p.parts) z = p.part_sums[row * p.parts + tid];
    for (int i = tid; i < n + 8; i += FEW) keys[i] = i < n ? p.part_keys[row * n + i] : 0;
    const Given first = given(p.a, row, tid);
    if (tid < MAX_TOP) list[tid] = 0;
    move_to(z, wave_largest(z.m));
    z = all_sums<FEW>(z, red);
    for (int i = tid; i < n; i += FEW) {
        const uint64_t k = keys[i];
        const int rank = k ? larger_keys(keys, n, k) : MAX_TOP;
        if (rank < p.a.n_top) list[rank] = k;
    }
    __syncthreads();
    write_row<FEW>(p.a, row, z, list, first);
}

constexpr int kMaxParts = 64;     // of a row: their keys lie in the joining workgroup's LDS
constexpr int kMostParts = 512;   // of all rows that are cut: two workgroups for each CU

// About as many rows as CUs, each of which a large workgroup holds at once: no second launch (200 x 32000, in parts and in one: fp32 13.7 -> 11.3 us, bf16
// with 20 alternatives 16.3 -> 13.3).  Fewer rows are faster in parts, a CU's vector units being what a row waits for (24 x 32000 with five
// alternatives 10.4 in parts, 11.9 in one), and so are shorter ones (256 x 16000 13.4, 13.8).
bool large_workgroups(int64_t rows, int64_t vocab) { return rows >= 64 && rows <= 256 && vocab > 2 * FEW * PER && vocab <= MANY * PER; }

int32_t parts_of(int64_t rows, int64_t vocab) {
    if (large_workgroups(rows, vocab)) return 1;
    const int64_t chunks = (vocab + FEW * PER - 1) / (FEW * PER);
    return (int32_t)std::min<int64_t>({chunks, kMaxParts, std::max<int64_t>(1, kMostParts / std::max<int64_t>(1, rows))});
}

template <int THREADS, bool ONE>
void launch_rows(const LogprobsLaunch& p, hipStream_t s) {
    auto go = [&](auto kernel) { kernel<<<dim3((unsigned)(p.a.rows * p.parts)), dim3(THREADS), 0, s>>>(p); };
    if (p.a.is_f32) p.a.n_top ? go(logprobs_kernel<THREADS, true, true, ONE>) : go(logprobs_kernel<THREADS, true, false, ONE>);
    else p.a.n_top ? go(logprobs_kernel<THREADS, false, true, ONE>) : go(logprobs_kernel<THREADS, false, false, ONE>);
}

}  // namespace

// (grows with the rows, so that the largest call's serves all: of whatever rows there are, at most kMostParts parts)
int64_t logprobs_scratch_bytes(int64_t rows, int64_t n_top) { return std::min<int64_t>(rows * kMaxParts, kMostParts) * ((int64_t)sizeof(Sums) + 8 * n_top); }

hipError_t launch_logprobs(const LogprobsArgs& args, hipStream_t s) {
    if (args.rows == 0) return hipSuccess;
    const bool large = large_workgroups(args.rows, args.vocab);
    const int32_t chunk = (large ? MANY : FEW) * PER;
    LogprobsLaunch p{args, args.scratch ? parts_of(args.rows, args.vocab) : 1, (int32_t)(((int64_t)args.vocab + chunk - 1) / chunk), nullptr, nullptr};
    p.part_sums = static_cast<Sums*>(args.scratch);
    p.part_keys = reinterpret_cast<uint64_t*>(p.part_sums + (int64_t)args.rows * p.parts);
    if (large) launch_rows<MANY, true>(p, s);
    else if (p.parts == p.chunks) launch_rows<FEW, true>(p, s);   // a chunk for each workgroup: it stays in registers
    else launch_rows<FEW, false>(p, s);
    if (hipError_t e = hipGetLastError()) return e;
    if (p.parts > 1) {
        logprobs_join_kernel<<<dim3((unsigned)args.rows), dim3(FEW), ((size_t)p.parts * args.n_top + 8) * 8, s>>>(p);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace relserve
