// Shared by the tiled products (linear layers, in floating point and in 8-bit integers): order of tiles, copies to LDS.
#pragma once
#include "scnn_dense.h"

namespace scnn {

// Tiles of a launch in the order of its workgroups.  Workgroup i runs on XCD i % 8: each XCD takes one run of neighbouring
// tiles, and within a run eight rows of tiles go side by side, so that the tiles that an L2 works on share their operands.
__device__ __forceinline__ void tile_at(unsigned block, unsigned tiles_m, unsigned tiles_n, unsigned& tm, unsigned& tn) {
    const unsigned all = tiles_m * tiles_n, each = all / kXcds, more = all % kXcds;
    const unsigned xcd = block % kXcds, i = block / kXcds;
    const unsigned at = xcd * each + (xcd < more ? xcd : more) + i;
    constexpr unsigned kSide = 8;
    const unsigned group = at / (kSide * tiles_n), in = at % (kSide * tiles_n);
    const unsigned side = tiles_m - group * kSide < kSide ? tiles_m - group * kSide : kSide;
    // (divisions leave the vector unit: the addresses that follow from these are to be scalar)
    tm = (unsigned)__builtin_amdgcn_readfirstlane((int)(group * kSide + in % side));
    tn = (unsigned)__builtin_amdgcn_readfirstlane((int)(in / side));
}

// Sixteen bytes a lane straight from memory to LDS: lane l's to lds + 16 l.
__device__ __forceinline__ void copy_to_lds(const void* base, unsigned offset, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
// Waits until at most N of this wave's copies are on their way and its LDS reads have arrived, then for the workgroup's
// other waves.
template <int N>
__device__ __forceinline__ void copies_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

}  // namespace scnn
