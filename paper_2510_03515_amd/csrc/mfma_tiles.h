// What the tiled matrix kernels share: the geometry of a workgroup, barriers and loads written by hand, the order of the tiles.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rapid {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;

// Geometry of a workgroup: NWI x NWJ waves, each owning WI x WJ blocks of 32 x 32.
// 2 x 4 waves of 128 x 64 is the default (two waves per SIMD, which lets the hardware overlap one
// wave's LDS, barrier and memory-issue waits with the other's MFMAs at the price of 1.5x the LDS
// fragment reads); 2 x 2 waves of 128 x 128 (one wave per SIMD, 256 accumulator registers per lane)
// and 2 x 8 waves of 128 x 32 are selectable.
template <int NWI_, int NWJ_, int WI_, int WJ_>
struct Geo {
    static constexpr int NWI = NWI_, NWJ = NWJ_, WI = WI_, WJ = WJ_;
    static constexpr int NW = NWI * NWJ, NT = 64 * NW;
    static constexpr int BI = NWI * WI * 32, BJ = NWJ * WJ * 32;
    // A k-major operand of 192 (or 224) columns is loaded as 256 (a request then covers whole rows; the last columns are
    // not used), so an LDS stage has room for a power of two.
    static constexpr int LI = BI > 128 ? 256 : BI, LJ = BJ > 128 ? 256 : BJ;
    static constexpr int STAGE_BYTES = (LI + LJ) * 128;
    static constexpr int LDS_BYTES = 2 * STAGE_BYTES;
};

// Barrier without the memory fence of __syncthreads; the loops place their own waits before it.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// LDS fragment reads and their waits are issued by hand.  With direct memory -> LDS loads in the
// loop the compiler's wait insertion falls back to lgkmcnt(0) before every MFMA block, which also
// waits for the reads just issued for the NEXT sub-step and so undoes the software pipelining.
// LDS reads of a wave complete in order, so "at most n reads outstanding" after issuing the next
// sub-step's n reads means exactly "the current sub-step's fragments have arrived".
__device__ __forceinline__ uint32_t lds_addr(const char* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
__device__ __forceinline__ void load_to_lds_16(const char* gp, char* lp) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)gp,
                                     (__attribute__((address_space(3))) void*)lp, 16, 0, 0);
}

// Scheduling fence: nothing is moved across it.  The K step is written in the order that software-
// pipelines it (fragments of the next sub-step are requested before the MFMAs of the current one,
// tile requests sit between given MFMAs) and the fences keep that order.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// Workgroup id -> tile.  Hardware deals consecutive workgroup ids round-robin to the 8 XCDs (each
// with its own L2), so id % 8 picks the XCD and id / 8 the position in that XCD's contiguous share
// of a grouped order: GI tiles along i for one j, then the next j, ... so that workgroups resident
// together on an XCD re-use each other's operand panels out of L2.
struct TileId { int ti, tj; bool valid; };
// position `vid` of the grouped order -> tile
__device__ __forceinline__ TileId tile_of_vid(int vid, int tilesI, int tilesJ, int GI) {
    const int total = tilesI * tilesJ;
    TileId t;
    t.valid = vid < total;
    const int group_sz = GI * tilesJ;
    const int grp = vid / group_sz;
    const int first_i = grp * GI;
    const int gi = min(GI, tilesI - first_i);
    const int rem = vid - grp * group_sz;
    t.ti = first_i + rem % gi;
    t.tj = rem / gi;
    return t;
}
__host__ __device__ inline int ids_for(int tilesI, int tilesJ) { return (int)(((int64_t)tilesI * tilesJ + 7) / 8 * 8); }
template <class S>
struct Lane {
    int lane, wave, wave_i, wave_j, hi, lj;
    __device__ __forceinline__ Lane() {
        lane = threadIdx.x & 63;
        wave = threadIdx.x >> 6;
        wave_i = wave % S::NWI;
        wave_j = wave / S::NWI;
        hi = lane >> 5;
        lj = lane & 31;
    }
};

}  // namespace rapid
