// Decode step, GQA, over pages in 8 bits: E4M3 codes with a power-of-two scale per block of 16 tokens and KV head, keys and values each.
//
// The same split of the work, the same records and the same merge as over bf16 pages (kernels_decode.hip); half the bytes per token.
// Codes are turned into bf16 under their scale by one conversion per two entries on their way into the matrix cores: E4M3 times a power of two is
// exact in bf16, so that the products are those of the values that codes and scales stand for, and the queries keep their bf16.
//   S^T[key, query] = K_tile[16 x d] . Q^T[d x 16]       v_mfma_f32_16x16x32_bf16, d/32 steps for each of two tiles
//   O^T[dim, query] += V^T[16 x 32] . P^T[32 x 16]       v_mfma_f32_16x16x32_bf16, d/16 blocks for both tiles together
// Bound by memory: 2 d + 1/8 bytes per token and KV head.  A wave streams its tiles through two steps' registers, the scales of its next 64
// tiles come by one load (one tile per lane) and from there by lane reads.  What is in registers bounds the workgroups of a compute unit, and
// three with two steps hide one another's starts and ends better than two with four (64 requests of 512 .. 4096 tokens, 8 KV heads of 128 dims, on
// 128 CUs 75.8 / 83.1 us, 128 lognormal ones of 64 query heads 139 / 147, six workgroups per compute unit dealt).  With two dealt (split_gqa) 69.4
// and 137: 4.4 and 4.8 TB/s inside the attention launch, where a plain read through registers has 5.5; over bf16 pages 122 and 234.
#include "decode_gqa.h"
#include "gqa_fp8_tile.h"
#include "internal.h"
#include "rope_device.h"
#include "split_merge.h"

namespace spd {

namespace {

template <int D>
struct Step8 {             // two tiles of 16 tokens, in operand order
  uint4 k[2][D / 64];
  uint4 v[2][D / 64];
};

template <int D>
__device__ inline void load_step8(Step8<D>& f, const char* __restrict__ base, const TileWindow& w, int i, int lane) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint64_t off = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)w.hi, 2 * i + u) << 32) |
                         (uint32_t)__builtin_amdgcn_readlane((int)w.lo, 2 * i + u);
    const uint4* p = (const uint4*)(base + off) + lane;
#pragma unroll
    for (int s = 0; s < D / 64; ++s) f.k[u][s] = load_once(p + s * 64);
#pragma unroll
    for (int s = 0; s < D / 64; ++s) f.v[u][s] = load_once(p + TILE_T * D / 16 + s * 64);
  }
}

// four codes as four bf16 under a scale
__device__ inline uint2 widen(uint32_t c, float scale) {
  return uint2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true))};
}

// sc[u]: the scale bytes of tile u (wave-uniform)
template <int D>
__device__ inline void compute_step8(const Step8<D>& f, const uint32_t (&sc)[2], const bf16x8 (&qf)[D / 32], f32x4 (&O)[D / 16], float& m, float& l,
                                     int tile, int n, float c, int c4) {
  f32x4 S[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    S[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float ks = scale_of(sc[u] & 255);
#pragma unroll
    for (int p = 0; p < D / 64; ++p) {
      const uint32_t w[4] = {f.k[u][p].x, f.k[u][p].y, f.k[u][p].z, f.k[u][p].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint2 a = widen(w[2 * h], ks), b = widen(w[2 * h + 1], ks);
        S[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, uint4{a.x, a.y, b.x, b.y}), qf[2 * p + h], S[u], 0, 0, 0);
      }
    }
  }
  // lane holds, for query (lane % 16), the keys tile*16 + 4*c4 + i of each tile
  const bool tail = (tile + 2) * TILE_T > n;
  if (tail) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((tile + u) * TILE_T + 4 * c4 + i >= n) S[u][i] = -INFINITY;
  }
  float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float m_new = fmaxf(m, mx);
  const float alpha = __builtin_amdgcn_exp2f((m - m_new) * c);
  const float mc = m_new * c;
  float psum = 0.f;
  uint2 pb[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] = __builtin_amdgcn_exp2f(S[u][i] * c - mc);
      psum += p[i];
    }
    pb[u].x = pack_bf16_rne(p[0], p[1]);
    pb[u].y = pack_bf16_rne(p[2], p[3]);
  }
  l = l * alpha + psum;
  m = m_new;
#pragma unroll
  for (int blk = 0; blk < D / 16; ++blk) O[blk] *= alpha;
  // entry j of a lane's eight along the 32 tokens: token 4 c4 + j of the first tile, 4 c4 + j - 4 of the second
  const bf16x8 pv = __builtin_bit_cast(bf16x8, uint4{pb[0].x, pb[0].y, pb[1].x, pb[1].y});
  const float vs[2] = {scale_of(sc[0] >> 8 & 255), scale_of(sc[1] >> 8 & 255)};
  uint32_t keep[2] = {~0u, ~0u};
  if (tail) {                                      // slots past the context: their bytes may be anything
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int in = n - (tile + u) * TILE_T - 4 * c4;   // bytes of a word that count
      keep[u] = in <= 0 ? 0 : in >= 4 ? ~0u : (1u << (8 * in)) - 1;
    }
  }
#pragma unroll
  for (int p = 0; p < D / 64; ++p) {
    const uint32_t w0[4] = {f.v[0][p].x, f.v[0][p].y, f.v[0][p].z, f.v[0][p].w}, w1[4] = {f.v[1][p].x, f.v[1][p].y, f.v[1][p].z, f.v[1][p].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 a = widen(tail ? w0[i] & keep[0] : w0[i], vs[0]), b = widen(tail ? w1[i] & keep[1] : w1[i], vs[1]);
      O[4 * p + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, uint4{a.x, a.y, b.x, b.y}), pv, O[4 * p + i], 0, 0, 0);
    }
  }
}

}  // namespace

// grid (n_items * n_kv_heads), block 256, as decode_gqa_kernel.  WHOLE: the launch rotates and appends too (the wave whose step holds the new
// token's block changes it in registers, on its way into the matrix cores, and puts it back); otherwise decode_prepare_fp8_kernel has.
template <int D, bool WHOLE>
__global__ __launch_bounds__(256, 3) void decode_gqa_fp8_kernel(GqaArgs a) {
  if constexpr (!WHOLE) {
    a.rot = 0;
    a.k_new = nullptr;
    a.mark.flag = nullptr;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(a.mark);
  const int g = blockIdx.x % a.Hkv;
  const char* rec = a.items + (size_t)(blockIdx.x / a.Hkv) * a.item_stride;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // wave-uniform
  const int col = lane & 15, c4 = lane >> 4;
  __shared__ __attribute__((aligned(16))) float sm_o[4][16][D + 4];
  __shared__ float sm_m[4][16], sm_l[4][16];
  __shared__ int32_t sm_rec[256];
  __shared__ uint32_t sm_last;
  // The record (header, page ids) is fetched once per workgroup: it may lie in pinned host memory.
  const int words = a.item_stride >> 2;
  if ((int)threadIdx.x < words) sm_rec[threadIdx.x] = ((const int32_t*)rec)[threadIdx.x];
  const double w_lane = a.rot ? a.w[min(lane, (a.rot >> 1) - 1)] : 0.0;
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(sm_rec[0]), chunk = __builtin_amdgcn_readfirstlane(sm_rec[1]);
  const int n_chunks = __builtin_amdgcn_readfirstlane(sm_rec[2]), n = __builtin_amdgcn_readfirstlane(sm_rec[3]);
  if (a.put_chunks && chunk == 0 && g == 0 && threadIdx.x == 0) a.put_chunks[b] = n_chunks;
  auto page_id = [&](int i) -> int {               // i-th page of the chunk
    const int wd = min(i + DECODE_ITEM_WORDS, words - 1);
    int id = sm_rec[min(wd, 255)];
    if (words > 256 && wd > 255) id = ((const int32_t*)rec)[wd];
    return id;
  };
  const int n_tiles = (n + TILE_T - 1) / TILE_T;
  const int tile0 = __builtin_amdgcn_readfirstlane(sm_rec[4]), tile1 = tile0 + __builtin_amdgcn_readfirstlane(sm_rec[5]);
  const int n_steps = (tile1 - tile0 + 1) >> 1;
  const int my_steps = (n_steps - wave + 3) >> 2;                      // this wave's steps: wave, wave + 4, ...
  const bool interleaved = a.interleaved != 0;

  // Each wave has a piece of LDS of its own, later used for its part of the merge: nothing in it needs a barrier.
  float* cs = &sm_o[wave][0][0];                   // [D / 2] cosines, sines, then the new token's key and value
  float* sn = cs + D / 2;
  bf16_t* krow = (bf16_t*)(sn + D / 2);
  bf16_t* vrow = krow + D;

  // where tile u of step i (of the 32 the window holds) lies, and its scale bytes: lane 2 i + u
  char* pool_g = a.pool + (uint64_t)g * a.head_bytes;
  char* scales_g = a.pool + a.scale_off + (uint64_t)2 * g * a.tiles_per_page;
  const int page0 = tile0 / a.tiles_per_page;
  uint32_t win_sc = 0;
  auto fill_window = [&](int s0) -> TileWindow {
    const int t = min(tile0 + 2 * (wave + 4 * (s0 + (lane >> 1))) + (lane & 1), n_tiles - 1);   // out of range: the last tile, masked later
    const int pg = t / a.tiles_per_page;
    const uint64_t page = (uint64_t)(uint32_t)page_id(pg - page0) * a.page_bytes;
    const uint64_t off = page + (uint64_t)(t - pg * a.tiles_per_page) * a.tile_bytes;
    win_sc = *(const unsigned short*)(scales_g + page + 2 * (t - pg * a.tiles_per_page));
    return TileWindow{(uint32_t)off, (uint32_t)(off >> 32)};
  };

  // ---- the loads that everything waits for first: query pieces, and in one wave the new token's key and value
  uint4 own[D / 32], oth[D / 32];
  const bf16_t* qrow = a.q + ((size_t)b * a.H + g * a.G + min(col, a.G - 1)) * D;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const int e0 = 8 * (4 * s + c4);
    own[s] = *(const uint4*)(qrow + e0);
    if (a.rot) oth[s] = *(const uint4*)(qrow + rope_partner(e0, a.off, a.rot, interleaved));
  }
  // the new token's tile is the last one of the request: the wave whose step holds it does the append
  const bool appends = a.k_new != nullptr && tile1 == n_tiles && ((n_steps - 1) & 3) == wave;
  constexpr int PCS = D / 8;                       // 16-byte pieces of a head
  uint4 kv_own = uint4{0, 0, 0, 0}, kv_oth = uint4{0, 0, 0, 0};
  if (appends) {                                   // lanes 0 .. PCS - 1: pieces of the key, the next PCS: of the value
    const int pc = lane % PCS, e0 = 8 * pc;
    const bf16_t* src = (lane / PCS & 1) ? a.v_new : a.k_new;
    src += ((size_t)b * a.Hkv + g) * D;
    kv_own = *(const uint4*)(src + e0);
    if (a.rot && lane < PCS) kv_oth = *(const uint4*)(src + rope_partner(e0, a.off, a.rot, interleaved));
  }

  constexpr int RING = 2;                          // steps in registers
  Step8<D> f[RING];
  TileWindow win = TileWindow{0, 0};
  // Where the steady state is reached its first loads are unconditional: the compiler then knows how many are on their way behind a
  // step's, and waits for that step's alone.
  constexpr int STEADY = 2 * RING - 1;
  const bool many_steps = my_steps >= STEADY;
  if (my_steps > 0) {
    win = fill_window(0);
    if (!many_steps) {
#pragma unroll
      for (int i = 0; i < RING - 1; ++i)
        if (i < my_steps) load_step8<D>(f[i], pool_g, win, i, lane);
    }
  }
  if (a.rot) {
    if (lane < (a.rot >> 1)) {
      const double turns = (double)(n - 1) * w_lane * 0.15915494309189535;
      const float ang = (float)((turns - __builtin_rint(turns)) * 6.283185307179586);
      sincosf(ang, &sn[lane], &cs[lane]);
    }
    lds_visible_in_wave();
  }
  bf16x8 qf[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    uint4 piece = own[s];
    if (a.rot) piece = rope_rotate(own[s], oth[s], 8 * (4 * s + c4), a.off, a.rot, interleaved, cs, sn);
    if (col >= a.G) piece = uint4{0, 0, 0, 0};
    qf[s] = __builtin_bit_cast(bf16x8, piece);
  }
  if (appends) {
    const int pc = lane % PCS;
    if (lane < PCS) *(uint4*)(krow + 8 * pc) = a.rot ? rope_rotate(kv_own, kv_oth, 8 * pc, a.off, a.rot, interleaved, cs, sn) : kv_own;
    else if (lane < 2 * PCS) *(uint4*)(vrow + 8 * pc) = kv_own;
    lds_visible_in_wave();
  }

  f32x4 O[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) O[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  // Software pipeline over this wave's steps: RING - 1 of them are on their way.  Only a request's last step can hold the new token's
  // block, which is the step's last tile that is not a repetition.
  auto compute = [&](Step8<D>& s, int i, int s0, bool last) __attribute__((always_inline)) {
    const int tile = tile0 + 2 * (wave + 4 * i);
    uint32_t sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) sc[u] = (uint32_t)__builtin_amdgcn_readlane((int)win_sc, 2 * (i - s0) + u);
    if (last && tile + 1 >= n_tiles) sc[1] = 0x7f7f;    // (a repetition, which weighs nothing: no scale of a block that is not there yet)
    if (last && appends) {
      const int u = n_tiles - 1 - tile;            // 0 or 1
      const int pg = (n_tiles - 1) / a.tiles_per_page, sub = n_tiles - 1 - pg * a.tiles_per_page;
      const uint64_t page = (uint64_t)(uint32_t)page_id(pg - page0) * a.page_bytes;
#pragma unroll
      for (int uu = 0; uu < 2; ++uu)
        if (uu == u) {
          sc[uu] = append_token<D>(s.k[uu], s.v[uu], sc[uu], (n - 1) % TILE_T, krow, vrow, lane);
          store_block<D>(pool_g + page + (uint64_t)sub * a.tile_bytes, scales_g + page + 2 * sub, s.k[uu], s.v[uu], sc[uu], lane);
        }
    }
    compute_step8<D>(s, sc, qf, O, m, l, tile, n, a.c, c4);
  };
  // steps i .. s1 - 1, fewer than 2 RING, their first RING - 1 on their way
  auto rest = [&](int i, int s0, int s1) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 2 * RING - 1; ++r) {
      if (i + r >= s1) break;
      if (i + r + RING - 1 < s1) load_step8<D>(f[(r + RING - 1) % RING], pool_g, win, i + r + RING - 1 - s0, lane);
      compute(f[r % RING], i + r, s0, i + r == my_steps - 1);
    }
  };
  if (!many_steps) {
    rest(0, 0, my_steps);
  } else {
    for (int s0 = 0; s0 < my_steps; s0 += 32) {    // 32 steps (of 128 tokens over the four waves) per window
      const int s1 = min(my_steps, s0 + 32);
      if (s0) win = fill_window(s0);
      // (steps past the request's end are its last tile again)
#pragma unroll
      for (int i = 0; i < RING - 1; ++i) load_step8<D>(f[i], pool_g, win, i, lane);
      int i = s0;
      while (i + STEADY <= s1) {
#pragma unroll
        for (int r = 0; r < RING; ++r) {
          load_step8<D>(f[(r + RING - 1) % RING], pool_g, win, i + r + RING - 1 - s0, lane);
          __builtin_amdgcn_sched_barrier(0);
          compute(f[r], i + r, s0, false);
        }
        i += RING;
      }
      rest(i, s0, s1);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // merge the four waves' (m, l, O) through LDS
#pragma unroll
  for (int blk = 0; blk < D / 16; ++blk)
    *(f32x4*)&sm_o[wave][col][16 * blk + 4 * c4] = O[blk];
  if (c4 == 0) { sm_m[wave][col] = m; sm_l[wave][col] = l; }
  __syncthreads();
  const size_t head0 = (size_t)b * a.H + g * a.G;
  // two output dims per thread
  for (int idx = threadIdx.x; idx < a.G * (D / 2); idx += 256) {
    const int qh = idx / (D / 2), d = 2 * (idx % (D / 2));
    const float m_tot = fmaxf(fmaxf(sm_m[0][qh], sm_m[1][qh]), fmaxf(sm_m[2][qh], sm_m[3][qh]));
    float l_tot = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float wgt = __builtin_amdgcn_exp2f((sm_m[w][qh] - m_tot) * a.c);
      l_tot += sm_l[w][qh] * wgt;
      o0 += sm_o[w][qh][d] * wgt;
      o1 += sm_o[w][qh][d + 1] * wgt;
    }
    const size_t head = head0 + qh;
    if (n_chunks == 1) {
      *(uint32_t*)(a.out + head * D + d) = pack_bf16_rne(o0 / l_tot, o1 / l_tot);
    } else {
      const size_t slot = head * a.max_chunks + chunk;
      store_partial(a.ws_o + slot * D + d, o0, o1, a.counters != nullptr);
      if (d == 0) store_partial(a.ws_ml + slot * 2, m_tot * a.c, l_tot, a.counters != nullptr);
    }
  }
  if (n_chunks == 1 || a.counters == nullptr) return;
  // ---- few chunks: the workgroup that finds itself to be the last of its (request, KV head) merges them
  if (!last_of(a.counters + (size_t)b * a.Hkv + g, (uint32_t)n_chunks, &sm_last)) return;
  const size_t slot0 = head0 * a.max_chunks;
  merge_in_launch<D, 256>(a.ws_o + slot0 * D, a.ws_ml + slot0 * 2, a.G, a.max_chunks, n_chunks, &sm_o[0][0][0], a.out + head0 * D);
}

// Rotation of the queries into q_rot and the append of the new tokens, ahead of an attention launch of many workgroups (as
// decode_prepare_kernel).  grid (n_items, 1 + n_kv_heads / 4), block 256: the workgroups of a request's last chunk do the request, the first the
// queries, each of the others four KV heads, a wave each.  Bound by latency (record, then rows and block): all a wave's loads go out together, and
// the angles are formed meanwhile.  200 requests, 32 query and 8 KV heads on 128 CUs: 7.0 us, with all of a request in one workgroup 10.3.
template <int D>
__global__ __launch_bounds__(256) void decode_prepare_fp8_kernel(GqaArgs a, bf16_t* __restrict__ q_rot) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* head = (const int32_t*)(a.items + (size_t)blockIdx.x * a.item_stride);
  __shared__ float cs[D / 2], sn[D / 2];
  __shared__ __attribute__((aligned(16))) bf16_t rows[4][2][D];
  const double w = tid < (a.rot >> 1) ? a.w[tid] : 0.0;
  const int last_page = head[(a.item_stride >> 2) - 1];          // (a record's end repeats the chunk's last page)
  const int b = head[0], n = head[3], n_tiles = (n + TILE_T - 1) / TILE_T;
  if (head[4] + head[5] != n_tiles) return;        // not the request's last chunk
  const bool interleaved = a.interleaved != 0;
  constexpr int PCS = D / 8, BATCH = 4;            // 16-byte pieces of a head; loads on their way per thread
  auto angles = [&]() __attribute__((always_inline)) {
    if (tid < (a.rot >> 1)) {
      const double turns = (double)(n - 1) * w * 0.15915494309189535;
      const float ang = (float)((turns - __builtin_rint(turns)) * 6.283185307179586);
      sincosf(ang, &sn[tid], &cs[tid]);
    }
    __syncthreads();
  };
  if (blockIdx.y == 0) {
    if (!a.rot) return;
    const bf16_t* q = a.q + (size_t)b * a.H * D;
    bf16_t* to = q_rot + (size_t)b * a.H * D;
    const int n_q = a.H * PCS;
    uint4 own[BATCH], oth[BATCH];
    auto load = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int i = min(i0 + 256 * j, n_q - 1);
        own[j] = *(const uint4*)(q + 8 * i);
        oth[j] = *(const uint4*)(q + i / PCS * D + rope_partner(8 * (i % PCS), a.off, a.rot, interleaved));
      }
    };
    load(tid);
    angles();
    for (int i0 = tid; i0 < n_q; i0 += 256 * BATCH) {
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int i = i0 + 256 * j;
        if (i < n_q) *(uint4*)(to + 8 * i) = rope_rotate(own[j], oth[j], 8 * (i % PCS), a.off, a.rot, interleaved, cs, sn);
      }
      load(i0 + 256 * BATCH);
    }
    return;
  }
  if (!a.k_new) return;
  const int g = 4 * ((int)blockIdx.y - 1) + wave, gc = min(g, a.Hkv - 1), sub = (n_tiles - 1) % a.tiles_per_page;   // (a wave without a head stores nothing)
  char* page = a.pool + (uint64_t)(uint32_t)last_page * a.page_bytes;
  char* tile = page + (uint64_t)gc * a.head_bytes + (uint64_t)sub * a.tile_bytes;
  char* scale_at = page + a.scale_off + 2 * ((uint64_t)gc * a.tiles_per_page + sub);
  bf16_t *krow = rows[wave][0], *vrow = rows[wave][1];
  const int pc = lane % PCS, e0 = 8 * pc;
  const bf16_t* src = (lane / PCS & 1 ? a.v_new : a.k_new) + ((size_t)b * a.Hkv + gc) * D;   // lanes 0 .. PCS - 1: pieces of the key, the next PCS: of the value
  uint4 piece = *(const uint4*)(src + e0), oth = uint4{0, 0, 0, 0};
  if (a.rot) oth = *(const uint4*)(src + rope_partner(e0, a.off, a.rot, interleaved));
  uint4 k[D / 64], v[D / 64];
#pragma unroll
  for (int p = 0; p < D / 64; ++p) {
    k[p] = *((const uint4*)tile + p * 64 + lane);
    v[p] = *((const uint4*)(tile + TILE_T * D) + p * 64 + lane);
  }
  const uint32_t sc = *(const unsigned short*)scale_at;
  if (a.rot) {
    angles();
    if (lane < PCS) piece = rope_rotate(piece, oth, e0, a.off, a.rot, interleaved, cs, sn);
  }
  if (lane < 2 * PCS) *(uint4*)((lane < PCS ? krow : vrow) + e0) = piece;
  lds_visible_in_wave();
  const uint32_t now = append_token<D>(k, v, sc, (n - 1) % TILE_T, krow, vrow, lane);
  if (g < a.Hkv) store_block<D>(tile, scale_at, k, v, now, lane);
}

template <int D>
static hipError_t launch_decode_gqa_fp8_t(const PoolGeom& g, char* pool_base, const DecodeLaunch& d, hipStream_t stream) {
  const dim3 grid((unsigned)d.n_wgs * g.Hkv);
  if (d.prepared) hipLaunchKernelGGL((decode_gqa_fp8_kernel<D, false>), grid, dim3(256), 0, stream, gqa_args(g, pool_base, d));
  else hipLaunchKernelGGL((decode_gqa_fp8_kernel<D, true>), grid, dim3(256), 0, stream, gqa_args(g, pool_base, d));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || d.max_chunks <= 1 || d.counters) return e;
  return launch_merge_chunks<D>(d, stream);
}

hipError_t launch_decode_gqa_fp8(const PoolGeom& g, char* pool_base, const DecodeLaunch& d, hipStream_t stream) {
  if (g.dk == 128) return launch_decode_gqa_fp8_t<128>(g, pool_base, d, stream);
  if (g.dk == 64) return launch_decode_gqa_fp8_t<64>(g, pool_base, d, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_decode_prepare_fp8(const PoolGeom& g, char* pool_base, const DecodeLaunch& d, int n_items, void* q_rot, hipStream_t stream) {
  const GqaArgs a = gqa_args(g, pool_base, d);
  const dim3 grid((unsigned)n_items, (unsigned)(1 + (d.k_new ? (g.Hkv + 3) / 4 : 0)));
  if (g.dk == 128) hipLaunchKernelGGL(decode_prepare_fp8_kernel<128>, grid, dim3(256), 0, stream, a, (bf16_t*)q_rot);
  else if (g.dk == 64) hipLaunchKernelGGL(decode_prepare_fp8_kernel<64>, grid, dim3(256), 0, stream, a, (bf16_t*)q_rot);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace spd
