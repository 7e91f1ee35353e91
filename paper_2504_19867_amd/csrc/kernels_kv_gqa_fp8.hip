// Rows into and out of the pages of a GQA pool in 8 bits.
//
// A block is 16 tokens of one KV head, keys and values each, with one power-of-two scale (mx.h).  Rows are written front to back: a write
// that begins at a block's first token begins the block anew; one that begins further on keeps the rows ahead of it, re-coded where the new ones
// need a larger scale.  Slots behind the last row written are zeros.
// A step whose attention reads dense rows wants a block's earlier rows as they were before the new ones came: the wave that writes the
// block hands them out too, since nobody else may read it meanwhile.
//
// One launch does what a call or a step does to rows: the page write of the new ones (with the rotation of the keys, and the rows as they are for
// a step whose attention reads dense rows), cached rows to dense ones, and the copy of the step's metadata.  A wave takes a block: its lane (t, c)
// has the token t and of every 32 entries of the head the eight from 8 c on, which for keys is the page's order.  Values lie in the page with four
// tokens of an entry together: the four lanes of a quad turn 4 x 4 bytes round among themselves, and the words cross LDS.
// Bound by memory (4 d + 2 d bytes per token and head either way).
#include "gqa_fp8_tile.h"
#include "rope_device.h"

#include <algorithm>
#include <type_traits>

namespace spd {

namespace {
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
__device__ inline void store_once(void* p, uint4 v) { __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, (u32x4*)p); }

// lane r of a quad has a word of four entries of token r: returns the word of the four tokens of entry r (and the other way round)
__device__ inline uint32_t turn_quad(uint32_t w, int r) {
  const uint32_t o1 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0xB1, 0xF, 0xF, true);   // lane ^ 1
  w = r & 1 ? __builtin_amdgcn_perm(o1, w, 0x03070105) : __builtin_amdgcn_perm(o1, w, 0x06020400);
  const uint32_t o2 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x4E, 0xF, 0xF, true);   // lane ^ 2
  return r & 2 ? __builtin_amdgcn_perm(o2, w, 0x03020706) : __builtin_amdgcn_perm(o2, w, 0x05040100);
}

// eight codes as eight bf16 under a scale
__device__ inline uint4 widen_row(uint32_t x, uint32_t y, float f) {
  auto two = [&](uint32_t c, auto hi) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, f, hi)); };
  return uint4{two(x, std::false_type{}), two(x, std::true_type{}), two(y, std::false_type{}), two(y, std::true_type{})};
}

struct Rows8Args {
  char* base;
  uint64_t page_bytes, scale_off;
  uint32_t head_bytes, tile_bytes;
  int tiles_per_page, Hkv;
  const TileDesc* descs;
  int n_tiles, HG, groups;       // HG: KV heads per workgroup
  const bf16_t *k, *v;
  bf16_t* k_rw;                  // k again, where the keys are rotated
  int n_copy;
  uint4* copy_dst;
  const uint4* copy_src;
  uint64_t copy_n16;
  const TileDesc* cached;
  int n_cached;
  bf16_t *k_all, *v_all;
  const double* w;
  int rot, off, interleaved;
  StepMark mark;
};
}  // namespace

template <int D, bool ROPE>
__global__ __launch_bounds__(256) void kv_rows_gqa_fp8_kernel(Rows8Args a) {
  int blk = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blk == 0 && tid == 0) store_mark(a.mark);
  if (blk < a.n_copy) {
    for (uint64_t j = (uint64_t)blk * 256 + tid; j < a.copy_n16; j += (uint64_t)a.n_copy * 256) a.copy_dst[j] = a.copy_src[j];
    return;
  }
  blk -= a.n_copy;
  constexpr int NP = D / 64, QUAD = 80;            // a token quad's 16 pieces of 16 bytes in LDS, in words, with room between
  __shared__ __attribute__((aligned(16))) uint32_t turn[4][NP * 4 * QUAD];
  __shared__ float cs[ROPE ? 16 * (D / 2 + 1) : 1], sn[ROPE ? 16 * (D / 2 + 1) : 1];
  const int col = lane & 15, c4 = lane >> 4;
  uint32_t* lds = turn[wave];
  // where in LDS this lane's words belong: after the turn, entry 64 p + 32 h + 8 c4 + 4 e + (col & 3) of the tokens 4 (col / 4) .. + 3
  auto word_at = [&](int p, int h, int e) -> int {
    const int d = 32 * h + 8 * c4 + 4 * e + (col & 3);
    return (p * 4 + (col >> 2)) * QUAD + (d & 15) * 4 + (d >> 4);
  };
  const bool write = blk < a.n_tiles * a.groups;
  if (!write) blk -= a.n_tiles * a.groups;
  const TileDesc d = (write ? a.descs : a.cached)[blk / a.groups];
  const int g_begin = blk % a.groups * a.HG, g_end = min(g_begin + a.HG, a.Hkv);
  const bool mine = col >= d.t_begin && col < d.t_end;
  char* page = a.base + (uint64_t)d.page * a.page_bytes;

  // the block k, v, as it lies in its page, to dense rows: token t to row row0 + t, where `wanted`
  auto hand_out = [&](const uint4 (&k)[NP], const uint4 (&v)[NP], uint32_t scales, int row0, int g, bool wanted) __attribute__((always_inline)) {
    const float ks = scale_of(scales & 255), vs = scale_of(scales >> 8);
#pragma unroll
    for (int p = 0; p < NP; ++p) *(uint4*)(lds + (p * 4 + c4) * QUAD + col * 4) = v[p];
    lds_visible_in_wave();
    const size_t row = ((size_t)(row0 + col) * a.Hkv + g) * D;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const uint32_t kw[4] = {k[p].x, k[p].y, k[p].z, k[p].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t x = turn_quad(lds[word_at(p, h, 0)], col & 3), y = turn_quad(lds[word_at(p, h, 1)], col & 3);
        if (wanted) {
          *(uint4*)(a.k_all + row + 64 * p + 32 * h + 8 * c4) = widen_row(kw[2 * h], kw[2 * h + 1], ks);
          *(uint4*)(a.v_all + row + 64 * p + 32 * h + 8 * c4) = widen_row(x, y, vs);
        }
      }
    }
    lds_visible_in_wave();
  };

  if (write) {
    if constexpr (ROPE) {
      const int half = a.rot >> 1;
      for (int i = tid; i < 16 * half; i += 256) {
        const int t = i / half, pair = i % half;
        const double turns = (double)(d.pad[0] + t) * a.w[pair] * 0.15915494309189535;   // angle / 2 pi
        const float r = (float)((turns - __builtin_rint(turns)) * 6.283185307179586);
        sincosf(r, &sn[t * (D / 2 + 1) + pair], &cs[t * (D / 2 + 1) + pair]);
      }
      __syncthreads();
    }
    for (int g = g_begin + wave; g < g_end; g += 4) {
      const size_t row = ((size_t)(d.src_row + col - d.t_begin) * a.Hkv + g) * D;
      char* tile = page + (uint64_t)g * a.head_bytes + (uint64_t)d.sub * a.tile_bytes;
      char* scale_at = page + a.scale_off + 2 * ((uint64_t)g * a.tiles_per_page + d.sub);
      uint4 k[2 * NP], v[2 * NP], oth[2 * NP], k_old[NP], v_old[NP];
      uint32_t scales = 0;
#pragma unroll
      for (int s = 0; s < 2 * NP; ++s) {
        k[s] = v[s] = oth[s] = uint4{0, 0, 0, 0};
        if (mine) {
          const int e0 = 32 * s + 8 * c4;
          k[s] = *(const uint4*)(a.k + row + e0);
          v[s] = *(const uint4*)(a.v + row + e0);
          if constexpr (ROPE) oth[s] = *(const uint4*)(a.k + row + rope_partner(e0, a.off, a.rot, a.interleaved != 0));
        }
      }
      if (d.t_begin > 0) {
        scales = *(const unsigned short*)scale_at;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          k_old[p] = *((const uint4*)tile + p * 64 + lane);
          v_old[p] = *((const uint4*)(tile + TILE_T * D) + p * 64 + lane);
        }
      }
      if constexpr (ROPE) {
        const float *c = cs + col * (D / 2 + 1), *si = sn + col * (D / 2 + 1);
#pragma unroll
        for (int s = 0; s < 2 * NP; ++s) k[s] = rope_rotate(k[s], oth[s], 32 * s + 8 * c4, a.off, a.rot, a.interleaved != 0, c, si);
      }
      uint32_t mk = 0, mv = 0;
#pragma unroll
      for (int s = 0; s < 2 * NP; ++s) {
        mk = max(max(mk, max(finite_magnitude_bf16x2(k[s].x), finite_magnitude_bf16x2(k[s].y))), max(finite_magnitude_bf16x2(k[s].z), finite_magnitude_bf16x2(k[s].w)));
        mv = max(max(mv, max(finite_magnitude_bf16x2(v[s].x), finite_magnitude_bf16x2(v[s].y))), max(finite_magnitude_bf16x2(v[s].z), finite_magnitude_bf16x2(v[s].w)));
      }
      uint32_t bk = scale_byte_e4m3(wave_max(mk)), bv = scale_byte_e4m3(wave_max(mv));
      const uint32_t ok = scales & 255, ov = scales >> 8;
      if (d.t_begin > 0) {
        bk = max(bk, ok);
        bv = max(bv, ov);
      }
      const float ik = inverse_scale_of(bk), iv = inverse_scale_of(bv);
      auto codes = [](uint32_t x, uint32_t y, float f) -> uint32_t {
        return e4m3_codes(rope_bf_lo(x) * f, rope_bf_hi(x) * f, rope_bf_lo(y) * f, rope_bf_hi(y) * f);
      };
      // rows as they are (rotated keys), where somebody wants them
      if (mine) {
        const size_t dense = ((size_t)(d.pad[1] + col - d.t_begin) * a.Hkv + g) * D;
#pragma unroll
        for (int s = 0; s < 2 * NP; ++s) {
          if constexpr (ROPE) *(uint4*)(a.k_rw + row + 32 * s + 8 * c4) = k[s];
          if (a.k_all) {
            *(uint4*)(a.k_all + dense + 32 * s + 8 * c4) = k[s];
            *(uint4*)(a.v_all + dense + 32 * s + 8 * c4) = v[s];
          }
        }
      }
      if (a.k_all && d.t_begin > 0) hand_out(k_old, v_old, scales, d.pad[1] - d.t_begin, g, col < d.t_begin);
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 x = v[2 * p + h];
          lds[word_at(p, h, 0)] = turn_quad(codes(x.x, x.y, iv), col & 3);
          lds[word_at(p, h, 1)] = turn_quad(codes(x.z, x.w, iv), col & 3);
        }
      lds_visible_in_wave();
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        uint32_t kw[4] = {codes(k[2 * p].x, k[2 * p].y, ik), codes(k[2 * p].z, k[2 * p].w, ik), codes(k[2 * p + 1].x, k[2 * p + 1].y, ik),
                          codes(k[2 * p + 1].z, k[2 * p + 1].w, ik)};
        const uint4 x = *(const uint4*)(lds + (p * 4 + c4) * QUAD + col * 4);
        uint32_t vw[4] = {x.x, x.y, x.z, x.w};
        if (d.t_begin > 0) {                       // the rows ahead stay, under the block's scale as it is now
          const uint32_t ko[4] = {k_old[p].x, k_old[p].y, k_old[p].z, k_old[p].w}, vo[4] = {v_old[p].x, v_old[p].y, v_old[p].z, v_old[p].w};
          const float fk = __builtin_bit_cast(float, (uint32_t)max(127 + (int)ok - (int)bk, 0) << 23);
          const float fv = __builtin_bit_cast(float, (uint32_t)max(127 + (int)ov - (int)bv, 0) << 23);
          const int in = d.t_begin - 4 * c4;       // bytes of a word of values that stay
          const uint32_t keep = in <= 0 ? 0 : in >= 4 ? ~0u : (1u << (8 * in)) - 1;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (col < d.t_begin) kw[i] = bk != ok ? recode(ko[i], fk) : ko[i];
            vw[i] = (vw[i] & ~keep) | ((bv != ov ? recode(vo[i], fv) : vo[i]) & keep);
          }
        }
        store_once((uint4*)tile + p * 64 + lane, uint4{kw[0], kw[1], kw[2], kw[3]});
        store_once((uint4*)(tile + TILE_T * D) + p * 64 + lane, uint4{vw[0], vw[1], vw[2], vw[3]});
      }
      if (lane == 0) *(unsigned short*)scale_at = (unsigned short)(bk | bv << 8);
      lds_visible_in_wave();                       // (the next head's words replace this one's)
    }
    return;
  }

  // cached rows: the values that codes and scales stand for, exact in bf16
  for (int g = g_begin + wave; g < g_end; g += 4) {
    const char* tile = page + (uint64_t)g * a.head_bytes + (uint64_t)d.sub * a.tile_bytes;
    const uint32_t scales = *(const unsigned short*)(page + a.scale_off + 2 * ((uint64_t)g * a.tiles_per_page + d.sub));
    uint4 k[NP], v[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      k[p] = load_once((const uint4*)tile + p * 64 + lane);
      v[p] = load_once((const uint4*)(tile + TILE_T * D) + p * 64 + lane);
    }
    hand_out(k, v, scales, d.src_row - d.t_begin, g, mine);
  }
}

hipError_t launch_kv_rows_gqa_fp8(const PoolGeom& g, char* pool_base, const TileDesc* d_tiles, int n_tiles, const void* k, const void* v,
                                  const KvRows& x, const StepMark& mark, hipStream_t stream) {
  if (x.q) return hipErrorInvalidValue;            // (the queries' rotation is a launch of its own)
  Rows8Args a{};
  a.base = pool_base;
  a.page_bytes = g.page_bytes; a.scale_off = g.scale_off; a.head_bytes = g.head_bytes; a.tile_bytes = g.tile_bytes;
  a.tiles_per_page = g.tiles_per_page; a.Hkv = g.Hkv;
  a.descs = d_tiles; a.n_tiles = n_tiles;
  a.HG = 4; a.groups = (g.Hkv + a.HG - 1) / a.HG;
  a.k = (const bf16_t*)k; a.v = (const bf16_t*)v; a.k_rw = (bf16_t*)const_cast<void*>(k);
  a.copy_dst = (uint4*)x.copy_dst; a.copy_src = (const uint4*)x.copy_src;
  a.copy_n16 = x.copy_dst ? (x.copy_bytes + 15) / 16 : 0;
  a.n_copy = (int)std::min<uint64_t>(128, (a.copy_n16 + 255) / 256);
  a.cached = x.d_cached; a.n_cached = x.n_cached; a.k_all = (bf16_t*)x.k_all; a.v_all = (bf16_t*)x.v_all;
  a.w = x.rope_w; a.rot = x.rot; a.off = x.off; a.interleaved = x.interleaved ? 1 : 0;
  a.mark = mark;
  const int64_t blocks = a.n_copy + ((int64_t)n_tiles + a.n_cached) * a.groups;
  if (blocks <= 0) return hipSuccess;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a); };
  if (g.dk == 128) {
    if (x.rope_w) launch(kv_rows_gqa_fp8_kernel<128, true>);
    else launch(kv_rows_gqa_fp8_kernel<128, false>);
  } else {
    if (x.rope_w) launch(kv_rows_gqa_fp8_kernel<64, true>);
    else launch(kv_rows_gqa_fp8_kernel<64, false>);
  }
  return hipGetLastError();
}

}  // namespace spd
