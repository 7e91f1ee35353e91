// What the two GQA decode kernels (bf16 pages, and pages in 8 bits) have in common (device code and their launch arguments).
#pragma once

#include "internal.h"

namespace spd {

typedef unsigned short bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// two floats -> two bf16 (round to nearest even), packed low / high
__device__ inline uint32_t pack_bf16_rne(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// A 16-byte load of data that is read exactly once (KV pages in a decode step): marked non-temporal,
// so that the stream does not push the prefill partition's K/V tiles, which ARE re-read, out of the L2
// the two partitions share.
__device__ inline uint4 load_once(const uint4* p) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 r = __builtin_nontemporal_load((const u32x4*)p);
  return uint4{r.x, r.y, r.z, r.w};
}

// LDS written above by lanes of this wave is read below by other lanes of it (a wave's LDS accesses are served in order)
__device__ inline void lds_visible_in_wave() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Page ids of the tiles one wave streams, in its lanes: lane 2 i + u holds where tile u of the wave's i-th step lies.
struct TileWindow { uint32_t lo, hi; };

struct GqaArgs {
  char* pool;
  uint64_t page_bytes;
  uint32_t head_bytes, tile_bytes;
  int tiles_per_page;
  const bf16_t *q, *k_new, *v_new;
  bf16_t* out;
  const char* items;
  int item_stride, Hkv, H, G;
  float c;                      // scale * log2(e)
  int max_chunks;
  const double* w;
  int rot, off, interleaved;
  float *ws_o, *ws_ml;
  int32_t* put_chunks;
  uint32_t* counters;
  StepMark mark;
  uint64_t scale_off;           // of a page: its blocks' scales (pages in 8 bits)
};

inline GqaArgs gqa_args(const PoolGeom& g, char* pool_base, const DecodeLaunch& d) {
  GqaArgs a;
  a.pool = pool_base;
  a.page_bytes = g.page_bytes; a.head_bytes = g.head_bytes; a.tile_bytes = g.tile_bytes; a.tiles_per_page = g.tiles_per_page;
  a.q = (const bf16_t*)d.q; a.k_new = (const bf16_t*)d.k_new; a.v_new = (const bf16_t*)d.v_new; a.out = (bf16_t*)d.out;
  a.items = d.items; a.item_stride = d.item_stride;
  a.Hkv = g.Hkv; a.H = d.H; a.G = d.H / g.Hkv;
  a.c = d.scale * 1.4426950408889634f;
  a.max_chunks = d.max_chunks;
  a.w = d.w; a.rot = d.rot; a.off = d.off; a.interleaved = d.interleaved;
  a.ws_o = d.ws_o; a.ws_ml = d.ws_ml; a.put_chunks = d.put_chunks; a.counters = d.counters; a.mark = d.mark;
  a.scale_off = g.scale_off;
  return a;
}

}  // namespace spd
