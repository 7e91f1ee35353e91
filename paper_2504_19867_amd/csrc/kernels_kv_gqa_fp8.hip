// Rows into and out of the pages of a GQA pool in 8 bits.
//
// A block is 16 tokens of one KV head, keys and values each, with one power-of-two scale (mx.h).  Rows are written front to back: a write
// that begins at a block's first token begins the block anew; one that begins further on keeps the rows ahead of it, re-coded where the new ones
// need a larger scale.  Slots behind the last row written are zeros.
// A step whose attention reads dense rows wants a block's earlier rows as they were before the new ones came: the wave that writes the
// block hands them out too, since nobody else may read it meanwhile.
//
// A wave takes a block (of a few KV heads of a tile in turn).  Rows are moved in row order, 16 bytes per lane of whole rows; codes change between
// row order and page order in LDS, as rows of codes.  Values lie in the page with four tokens of an entry together: there the four lanes of
// a quad turn 4 x 4 bytes round among themselves.
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
  int HG, groups;                // KV heads per workgroup, workgroups per tile
  const bf16_t *k, *v;
  int n_copy;
  uint4* copy_dst;
  const uint4* copy_src;
  uint64_t copy_n16;
  bf16_t *k_all, *v_all;
  StepMark mark;
};
}  // namespace

// What a wave knows of its tile (one descriptor per workgroup) and of its place in it.
template <int D>
struct Place {
  static constexpr int NP = D / 64, PCS = D / 8, STEP = 64 / PCS, NR = 16 / STEP;   // pieces of a row; rows of one load instruction, instructions of a block
  static constexpr int PITCH = D + 8;              // bytes of a row of codes in LDS
  const Rows8Args& a;
  TileDesc d;
  int lane, col, c4;                               // page order: token (keys) or entry (values), quarter or token quad
  int piece, row0;                                 // row order: the lane's entries are 8 piece .. + 7 of the rows row0 + STEP r
  int g_begin, g_end;
  char *lds, *page;
  // Rows of [rows][Hkv][D] tensors: a wave-uniform address of the head's row `row` (of token slot 0, which may lie ahead of the tensor where
  // that slot is not touched) and of every STEP rows from there, and the lane's bytes behind it.
  uint32_t row_off;
  int64_t row_step;
  __device__ Place(const Rows8Args& args, int blk, char* codes_lds) : a(args), d(args.descs[blk / args.groups]) {
    d.src_row = __builtin_amdgcn_readfirstlane(d.src_row); d.page = __builtin_amdgcn_readfirstlane(d.page); d.sub = __builtin_amdgcn_readfirstlane(d.sub);
    d.t_begin = __builtin_amdgcn_readfirstlane(d.t_begin); d.t_end = __builtin_amdgcn_readfirstlane(d.t_end);
    d.pad[0] = __builtin_amdgcn_readfirstlane(d.pad[0]); d.pad[1] = __builtin_amdgcn_readfirstlane(d.pad[1]);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    lane = threadIdx.x & 63; col = lane & 15; c4 = lane >> 4; piece = lane % PCS; row0 = lane / PCS;
    g_begin = blk % a.groups * a.HG + wave; g_end = min(blk % a.groups * a.HG + a.HG, a.Hkv);   // (every fourth head: a wave's)
    lds = codes_lds + wave * (16 * PITCH);
    page = a.base + (uint64_t)d.page * a.page_bytes;
    row_off = (uint32_t)(row0 * a.Hkv * D + 8 * piece) * 2;
    row_step = (int64_t)STEP * a.Hkv * D * 2;
  }
  __device__ char* tile(int g) const { return page + (uint64_t)g * a.head_bytes + (uint64_t)d.sub * a.tile_bytes; }
  __device__ char* scales(int g) const { return page + a.scale_off + 2 * ((uint64_t)g * a.tiles_per_page + d.sub); }
  __device__ char* rows(const void* p, int row, int g) const { return (char*)p + ((int64_t)row * a.Hkv + g) * (D * 2); }
  __device__ int token(int r) const { return row0 + STEP * r; }
  __device__ bool touched(int r) const { return token(r) >= d.t_begin && token(r) < d.t_end; }
  // the block of head g as bf16 to dense rows: token t to row dense0 + t, for first <= t < last
  __device__ __attribute__((always_inline)) void hand_out(int dense0, int g, int first, int last) const {
    uint4 b[2][NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      b[0][p] = load_once((const uint4*)tile(g) + p * 64 + lane);
      b[1][p] = load_once((const uint4*)(tile(g) + TILE_T * D) + p * 64 + lane);
    }
    const uint32_t sc = *(const unsigned short*)scales(g);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
#pragma unroll
      for (int p = 0; p < NP; ++p) {               // rows of codes in LDS
        const uint32_t w[4] = {b[side][p].x, b[side][p].y, b[side][p].z, b[side][p].w};
        if (side == 0) {
          *(uint2*)(lds + col * PITCH + 64 * p + 8 * c4) = uint2{w[0], w[1]};
          *(uint2*)(lds + col * PITCH + 64 * p + 32 + 8 * c4) = uint2{w[2], w[3]};
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) *(uint32_t*)(lds + (4 * c4 + (col & 3)) * PITCH + 64 * p + 16 * i + (col & ~3)) = turn_quad(w[i], col & 3);
        }
      }
      lds_visible_in_wave();
      const float f = scale_of(side == 0 ? sc & 255 : sc >> 8);
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int t = token(r);
        const uint2 c = *(const uint2*)(lds + t * PITCH + 8 * piece);
        if (t >= first && t < last) *(uint4*)(rows(side == 0 ? a.k_all : a.v_all, dense0, g) + r * row_step + row_off) = widen_row(c.x, c.y, f);
      }
      lds_visible_in_wave();
    }
  }
};

// grid (n_tiles * groups), block 256: cached rows to dense ones, the values that codes and scales stand for, exact in bf16.  A kernel of its own: it
// needs a quarter of the registers of the page write, and what its workgroups wait for (descriptor, then block) is hidden by their number: 16001
// rows of 8 heads of 128 dims 28 us on 128 CUs (3.5 TB/s), in one kernel with the page write 40.
template <int D>
__global__ __launch_bounds__(256, 8) void kv_read_gqa_fp8_kernel(Rows8Args a) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(a.mark);
  __shared__ __attribute__((aligned(16))) char codes_lds[4 * 16 * Place<D>::PITCH];
  const Place<D> at(a, blockIdx.x, codes_lds);
  for (int g = at.g_begin; g < at.g_end; g += 4) at.hand_out(at.d.src_row - at.d.t_begin, g, at.d.t_begin, at.d.t_end);
}

// grid (n_copy + n_tiles * groups), block 256: the page write, the rows as they are to dense ones, and the copy of the step's metadata.  9000 rows of 8
// heads of 128 dims 19 us on 128 CUs (2.9 TB/s).  Rotating the keys on the way as the bf16 page write does was slower than the rotation's own launch
// (2500 rows: 26 us instead of 9, which that launch, busy with the queries anyway, takes 3 us longer): the angles' code holds the registers.
template <int D>
__global__ __launch_bounds__(256, 4) void kv_write_gqa_fp8_kernel(Rows8Args a) {
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && tid == 0) store_mark(a.mark);
  if ((int)blockIdx.x < a.n_copy) {
    for (uint64_t j = (uint64_t)blockIdx.x * 256 + tid; j < a.copy_n16; j += (uint64_t)a.n_copy * 256) a.copy_dst[j] = a.copy_src[j];
    return;
  }
  using P = Place<D>;
  constexpr int NP = P::NP, NR = P::NR, PITCH = P::PITCH;
  __shared__ __attribute__((aligned(16))) char codes_lds[4 * 16 * PITCH];
  const P at(a, (int)blockIdx.x - a.n_copy, codes_lds);
  const TileDesc& d = at.d;
  const int e0 = 8 * at.piece, col = at.col, c4 = at.c4;
  char* const lds = at.lds;
  for (int g = at.g_begin; g < at.g_end; g += 4) {
    uint4 k[NR], v[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      k[r] = v[r] = uint4{0, 0, 0, 0};
      if (at.touched(r)) {
        k[r] = load_once((const uint4*)(at.rows(a.k, d.src_row - d.t_begin, g) + r * at.row_step + at.row_off));
        v[r] = load_once((const uint4*)(at.rows(a.v, d.src_row - d.t_begin, g) + r * at.row_step + at.row_off));
      }
    }
    uint32_t mk = 0, mv = 0, before = 0;
    if (d.t_begin > 0) before = *(const unsigned short*)at.scales(g);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      mk = max(max(mk, max(finite_magnitude_bf16x2(k[r].x), finite_magnitude_bf16x2(k[r].y))), max(finite_magnitude_bf16x2(k[r].z), finite_magnitude_bf16x2(k[r].w)));
      mv = max(max(mv, max(finite_magnitude_bf16x2(v[r].x), finite_magnitude_bf16x2(v[r].y))), max(finite_magnitude_bf16x2(v[r].z), finite_magnitude_bf16x2(v[r].w)));
    }
    uint32_t bk = scale_byte_e4m3(wave_max(mk)), bv = scale_byte_e4m3(wave_max(mv));
    const uint32_t ok = before & 255, ov = before >> 8;
    if (d.t_begin > 0) {
      bk = max(bk, ok);
      bv = max(bv, ov);
    }
    if (a.k_all) {                                 // rows as they are, where somebody wants them
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        if (at.touched(r)) {
          *(uint4*)(at.rows(a.k_all, d.pad[1] - d.t_begin, g) + r * at.row_step + at.row_off) = k[r];
          *(uint4*)(at.rows(a.v_all, d.pad[1] - d.t_begin, g) + r * at.row_step + at.row_off) = v[r];
        }
      }
    }
    if (a.k_all && d.t_begin > 0) at.hand_out(d.pad[1] - d.t_begin, g, 0, d.t_begin);
    char* tile = at.tile(g);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      __builtin_amdgcn_sched_barrier(0);
      const float f = inverse_scale_of(side == 0 ? bk : bv);
#pragma unroll
      for (int r = 0; r < NR; ++r) {               // rows of codes in LDS
        const uint4 y = side == 0 ? k[r] : v[r];
        *(uint2*)(lds + at.token(r) * PITCH + e0) =
            uint2{e4m3_codes(rope_bf_lo(y.x) * f, rope_bf_hi(y.x) * f, rope_bf_lo(y.y) * f, rope_bf_hi(y.y) * f),
                  e4m3_codes(rope_bf_lo(y.z) * f, rope_bf_hi(y.z) * f, rope_bf_lo(y.w) * f, rope_bf_hi(y.w) * f)};
      }
      lds_visible_in_wave();
      const uint32_t was = side == 0 ? ok : ov, now = side == 0 ? bk : bv;
      const float grown = __builtin_bit_cast(float, (uint32_t)max(127 + (int)was - (int)now, 0) << 23);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        uint32_t w[4];
        if (side == 0) {
          const uint2 lo = *(const uint2*)(lds + col * PITCH + 64 * p + 8 * c4), hi = *(const uint2*)(lds + col * PITCH + 64 * p + 32 + 8 * c4);
          w[0] = lo.x; w[1] = lo.y; w[2] = hi.x; w[3] = hi.y;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = turn_quad(*(const uint32_t*)(lds + (4 * c4 + (col & 3)) * PITCH + 64 * p + 16 * i + (col & ~3)), col & 3);
        }
        if (d.t_begin > 0) {                       // the rows ahead stay, under the block's scale as it is now
          const uint4 o = *((const uint4*)(tile + side * TILE_T * D) + p * 64 + at.lane);
          const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
          const int in = d.t_begin - 4 * c4;       // bytes of a word of values that stay
          const uint32_t keep = side == 0 ? (col < d.t_begin ? ~0u : 0) : in <= 0 ? 0 : in >= 4 ? ~0u : (1u << (8 * in)) - 1;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (w[i] & ~keep) | ((now != was ? recode(ow[i], grown) : ow[i]) & keep);
        }
        store_once((uint4*)(tile + side * TILE_T * D) + p * 64 + at.lane, uint4{w[0], w[1], w[2], w[3]});
      }
      lds_visible_in_wave();
    }
    if (at.lane == 0) *(unsigned short*)at.scales(g) = (unsigned short)(bk | bv << 8);
  }
}

// KV heads per workgroup: one per wave, unless there are so many tiles that workgroups queue for compute units; then the reads of the descriptors, which
// may lie in pinned host memory, are worth halving.  Rows read back, in us with two heads per wave / one: 16 of 8 heads 5.4 / 4.8 on 128 CUs, 1000 6.0 / 5.6,
// 3000 7.8 / 7.1; of 32 heads on 256 CUs 250 6.4 / 5.1, 2000 12.5 / 11.3, on 128 CUs 1000 9.3 / 8.2.  The read, whose workgroups wait for little else than
// descriptors, stops at 200 tiles: 3500 rows of 8 heads 8.2 / 8.7 on 128 CUs, 7.6 / 8.2 on 256, 4000 8.7 / 9.4 and 8.0 / 8.6 (the write 9.8 / 9.6).
constexpr int MOST_TILES_READ_BY_HEAD = 200;
static int heads_per_workgroup(int n_tiles, int Hkv, int cus) { return (int64_t)n_tiles * ((Hkv + 3) / 4) <= 4 * (int64_t)cus ? 4 : 8; }

hipError_t launch_kv_rows_gqa_fp8(const PoolGeom& g, char* pool_base, const TileDesc* d_tiles, int n_tiles, const void* k, const void* v,
                                  const KvRows& x, const StepMark& mark, hipStream_t stream) {
  if (x.rope_w) return hipErrorInvalidValue;       // (the rotation is a launch of its own)
  Rows8Args a{};
  a.base = pool_base;
  a.page_bytes = g.page_bytes; a.scale_off = g.scale_off; a.head_bytes = g.head_bytes; a.tile_bytes = g.tile_bytes;
  a.tiles_per_page = g.tiles_per_page; a.Hkv = g.Hkv;
  a.k = (const bf16_t*)k; a.v = (const bf16_t*)v;
  a.copy_dst = (uint4*)x.copy_dst; a.copy_src = (const uint4*)x.copy_src;
  a.copy_n16 = x.copy_dst ? (x.copy_bytes + 15) / 16 : 0;
  a.n_copy = (int)std::min<uint64_t>(128, (a.copy_n16 + 255) / 256);
  a.k_all = (bf16_t*)x.k_all; a.v_all = (bf16_t*)x.v_all;
  a.mark = mark;
  // what is done to `tiles` tiles, `heads` KV heads per workgroup, `copying` workgroups ahead of them
  auto launch = [&](auto kernel, int tiles, int copying, int heads) -> hipError_t {
    a.HG = heads; a.groups = (g.Hkv + a.HG - 1) / a.HG;
    const int64_t blocks = copying + (int64_t)tiles * a.groups;
    if (blocks <= 0) return hipSuccess;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a);
    a.mark.flag = nullptr;
    return hipGetLastError();
  };
  a.descs = d_tiles;
  int heads = heads_per_workgroup(n_tiles, g.Hkv, x.cus);
  hipError_t e;
  if (g.dk == 128) e = launch(kv_write_gqa_fp8_kernel<128>, n_tiles, a.n_copy, heads);
  else e = launch(kv_write_gqa_fp8_kernel<64>, n_tiles, a.n_copy, heads);
  if (e != hipSuccess) return e;
  a.descs = x.d_cached;
  heads = x.n_cached > MOST_TILES_READ_BY_HEAD ? 8 : heads_per_workgroup(x.n_cached, g.Hkv, x.cus);
  return g.dk == 128 ? launch(kv_read_gqa_fp8_kernel<128>, x.n_cached, 0, heads) : launch(kv_read_gqa_fp8_kernel<64>, x.n_cached, 0, heads);
}

}  // namespace spd
