// A block of the 8-bit GQA cache (16 tokens of one KV head, keys or values) in a wave's registers, as it lies in its page (internal.h), and
// how a token is appended to it.
#pragma once

#include "decode_gqa.h"
#include "mx.h"

namespace spd {

// largest finite magnitude of two bf16 entries, as the bits of an fp32
__device__ inline uint32_t finite_magnitude_bf16x2(uint32_t w) {
  const uint32_t a = w << 16 & 0x7fffffff, b = w & 0x7fff0000;
  return max(a < 0x7f800000 ? a : 0, b < 0x7f800000 ? b : 0);
}
__device__ inline uint32_t wave_max(uint32_t m) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
  return m;
}
// four codes under another scale: their values times 2^(b_old - b_new), b_new >= b_old, rounded
__device__ inline uint32_t recode(uint32_t c, float f) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return e4m3_codes(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}

// Puts a token (krow, vrow: D bf16 entries each, in LDS, visible) into slot t of the block whose codes are k, v and whose scale bytes are
// `scales` (keys, values << 8), as the wave holds them: the slots ahead of t are re-coded where the scale grows, those behind are zeros.  With
// t = 0 the block begins anew.  Returns the new scale bytes.
template <int D>
__device__ inline uint32_t append_token(uint4 (&k)[D / 64], uint4 (&v)[D / 64], uint32_t scales, int t, const bf16_t* krow, const bf16_t* vrow, int lane) {
  const int col = lane & 15, c4 = lane >> 4;
  uint32_t mk, mv;
  if constexpr (D == 128) {
    mk = finite_magnitude_bf16x2(((const uint32_t*)krow)[lane]);
    mv = finite_magnitude_bf16x2(((const uint32_t*)vrow)[lane]);
  } else {
    mk = finite_magnitude_bf16x2(krow[lane]);
    mv = finite_magnitude_bf16x2(vrow[lane]);
  }
  uint32_t bk = scale_byte_e4m3(wave_max(mk)), bv = scale_byte_e4m3(wave_max(mv));
  const uint32_t ok = scales & 255, ov = scales >> 8 & 255;
  if (t) {
    bk = max(bk, ok);
    bv = max(bv, ov);
  }
  const bool again_k = t && bk != ok, again_v = t && bv != ov;
  const float fk = __builtin_bit_cast(float, (uint32_t)max(127 + (int)ok - (int)bk, 0) << 23), fv = __builtin_bit_cast(float, (uint32_t)max(127 + (int)ov - (int)bv, 0) << 23);
  const float ik = inverse_scale_of(bk), iv = inverse_scale_of(bv);
  auto value = [](bf16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); };
#pragma unroll
  for (int p = 0; p < D / 64; ++p) {
    uint32_t kw[4] = {k[p].x, k[p].y, k[p].z, k[p].w}, vw[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // keys: word i holds entries 64 p + 32 (i / 2) + 8 c4 + 4 (i % 2) .. + 3 of token `col`
      if (again_k) kw[i] = recode(kw[i], fk);
      const bf16_t* e = krow + 64 * p + 32 * (i >> 1) + 8 * c4 + 4 * (i & 1);
      const uint32_t mine = e4m3_codes(value(e[0]) * ik, value(e[1]) * ik, value(e[2]) * ik, value(e[3]) * ik);
      kw[i] = col < t ? kw[i] : col == t ? mine : 0;
      // values: word i holds entry 64 p + 16 i + col of tokens 4 c4 .. + 3
      if (again_v) vw[i] = recode(vw[i], fv);
      const int in = t - 4 * c4;                   // the token's byte of the word, if 0 .. 3
      const uint32_t keep = in <= 0 ? 0 : in >= 4 ? ~0u : (1u << (8 * in)) - 1;
      vw[i] &= keep;
      if (in >= 0 && in < 4) vw[i] |= (e4m3_codes(value(vrow[64 * p + 16 * i + col]) * iv, 0.f, 0.f, 0.f) & 255) << (8 * in);
    }
    k[p] = uint4{kw[0], kw[1], kw[2], kw[3]};
    v[p] = uint4{vw[0], vw[1], vw[2], vw[3]};
  }
  return bk | bv << 8;
}

// the block, and its scale bytes, back to its page
template <int D>
__device__ inline void store_block(char* tile, char* scale_at, const uint4 (&k)[D / 64], const uint4 (&v)[D / 64], uint32_t scales, int lane) {
#pragma unroll
  for (int p = 0; p < D / 64; ++p) {
    *((uint4*)tile + p * 64 + lane) = k[p];
    *((uint4*)(tile + TILE_T * D) + p * 64 + lane) = v[p];
  }
  if (lane == 0) *(unsigned short*)scale_at = (unsigned short)scales;
}

}  // namespace spd
