// What the tiled projections' sources share: the order of tiles, loads from global memory into the LDS, the LDS limit of a launch.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <mutex>

namespace relserve {

namespace {

// The dynamic-LDS limit of a kernel is raised once per process, whichever host thread launches it first.
template <typename Kernel>
hipError_t allow_smem_once(std::once_flag& once, hipError_t& status, Kernel kernel, int bytes) {
    std::call_once(once, [&] {
        status = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    });
    return status;
}

constexpr int NUM_XCD = 8;

// Consecutive workgroups go to different XCDs: each XCD's run of tiles is made contiguous.
__device__ __forceinline__ int remap_xcd(int bid, int num) {
    const int per = num / NUM_XCD, rem = num % NUM_XCD;
    const int xcd = bid % NUM_XCD, idx = bid / NUM_XCD;
    return xcd < rem ? xcd * (per + 1) + idx : rem * (per + 1) + (xcd - rem) * per + idx;
}

// Tile order inside an XCD's run: token tiles fastest within panels of about GROUP_M token tiles, then
// feature tiles, then the next panel.  The ~32 tiles an XCD works on at a time then cover about
// GROUP_M token tiles x 32 / GROUP_M feature tiles, so that its L2 serves ~12 distinct operand
// slices per k step instead of 33 when the batch has many token tiles.  The token tiles are divided
// evenly over the panels (9 token tiles: panels of 5 and 4, not of 8 and 1 -- a panel of one token tile
// shares nothing but its activation slice).
constexpr int GROUP_M = 8;
__device__ __forceinline__ void tile_coords(int t, int tiles_m, int tiles_n, int& tile_m, int& tile_n) {
    const int n_panels = (tiles_m + GROUP_M - 1) / GROUP_M;
    const int base = tiles_m / n_panels, extra = tiles_m % n_panels;   // the first `extra` panels hold base + 1 token tiles
    const int big = (base + 1) * tiles_n;
    int first_m, gsz, in_group;
    if (t < extra * big) {
        gsz = base + 1;
        first_m = (t / big) * gsz;
        in_group = t % big;
    } else {
        const int u = t - extra * big, per = base * tiles_n;
        gsz = base;
        first_m = extra * (base + 1) + (u / per) * base;
        in_group = u % per;
    }
    tile_m = first_m + in_group % gsz;
    tile_n = in_group / gsz;
}

// A pointer every lane holds the same value of, moved to scalar registers (the compiler cannot always prove it).
__device__ __forceinline__ const char* uniform_ptr(const char* ptr) {
    const uint64_t v = reinterpret_cast<uint64_t>(ptr);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}

// 64 lanes x 16 bytes from (base + per-lane byte offset) to 1 KB of LDS starting at lds_addr.
// NT = non-temporal: for bytes that are read once (the weights of a batch of one token tile).  A streaming read of
// HBM reaches 7.1-7.4 TB/s with the hint against 6.3-6.4 TB/s without (measured with 32 KB per workgroup in flight);
// operands that other workgroups read again keep the default policy, which lets the L2 hold them.
// In two halves: dma16_to names the LDS address lds_addr + at (the constant) in m0, dma16_from loads; one instruction at least has to
// stand between the two (a load reads m0 too early right behind the scalar instruction that writes it).
__device__ __forceinline__ void dma16_to(uint32_t lds_addr, int at) {
    asm volatile("s_add_u32 m0, %0, %1" ::"s"(lds_addr), "i"(at) : "memory", "scc");
}
template <bool NT = false>
__device__ __forceinline__ void dma16_from(const void* base, uint32_t voff) {
    if (NT)
        asm volatile("global_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(base) : "memory");
    else
        asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base) : "memory");
}
template <bool NT = false>
__device__ __forceinline__ void dma16(const void* base, uint32_t voff, uint32_t lds_addr, int at) {
    if (NT)
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(base), "s"(lds_addr), "i"(at) : "memory", "scc");
    else
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(lds_addr), "i"(at) : "memory", "scc");
}

}  // namespace

}  // namespace relserve
