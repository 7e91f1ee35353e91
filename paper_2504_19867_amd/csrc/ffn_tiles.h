// What the FFN's matrix products have in common: loads that go straight to LDS, and the order in which an XCD takes its tiles (device code).
#pragma once

#include "internal.h"

namespace spd {

// 16 bytes per lane from global memory to LDS: lane i's data lands at lds_byte_addr + 16 * i.
// The compiler does not see this write; completion is tracked by hand with vmcnt.
__device__ inline void dma16s(const void* sbase, uint32_t voff, uint32_t lds_byte_addr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_byte_addr), "v"(voff), "s"(sbase) : "memory");
}
#define SPD_WAIT_VMCNT(N) __builtin_amdgcn_s_waitcnt(((N) & 15) | (7 << 4) | (15 << 8) | (((N) >> 4) << 14))
// 4 bytes per lane, likewise: lane i's word lands at lds_byte_addr + 4 * i
__device__ inline void dma4s(const void* sbase, uint32_t voff, uint32_t lds_byte_addr) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_byte_addr), "v"(voff), "s"(sbase) : "memory");
}

// Which tile the workgroups of an XCD take, in the order in which they take them.  Workgroup b runs on XCD b % xcds, and the
// workgroups of an XCD start in the order of b.  Every XCD takes a contiguous range of weight tiles (columns) and all token tiles;
// inside it the tiles are ordered so that the 16 or so workgroups running together form a block of about 4 x 4 tiles:
// each slice of x and of the weights that misses the XCD's L2 then feeds four workgroups.
struct TileOrder {
  int tiles_m, start, cnt;                        // this XCD's weight tiles: cnt from `start` on
  __device__ TileOrder(int tiles_m_, int tiles_n, int xcds) : tiles_m(tiles_m_) {
    const int xcd = (int)blockIdx.x % xcds, base = tiles_n / xcds, rem = tiles_n % xcds;
    cnt = base + (xcd < rem ? 1 : 0);
    start = xcd * base + min(xcd, rem);
  }
  __device__ int slots() const { return cnt * tiles_m; }
  __device__ void tile(int slot, int& tm, int& tn) const {
    const int full = cnt / 4;                     // column blocks of four weight tiles; the last one narrower
    const bool in_full = slot < full * 4 * tiles_m;
    const int cb = in_full ? slot / (4 * tiles_m) : full, wb = in_full ? 4 : cnt - 4 * full;
    const int q = slot - cb * 4 * tiles_m;
    tm = q / wb;
    tn = start + 4 * cb + q % wb;
  }
};

}  // namespace spd
