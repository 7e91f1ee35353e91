// First step of the gated FFN over MXFP4 weights and MX E4M3 rows:
//     out[t, i] = silu(g) u,   g = sum_k x[t, k] W_gate[i, k],  u = sum_k x[t, k] W_up[i, k]
// on the values that codes and scales stand for, fp32 sums, one rounding to bf16.  silu(z) = z / (1 + exp(-z)).
//
// The scaled matrix instructions take both formats as they are: a lane holds 32 codes of one row (16 bytes of E2M1, 32 of E4M3) and the
// scale byte of its 32 entries.  Weights are the A operand, so that a lane has consecutive outputs of one token.  Where the E2M1 lane of row r
// and quarter c of a step of 128 entries holds the entries 32 c .. 32 c + 31, the E4M3 lane holds 16 c .. 16 c + 15 and 64 + 16 c ..
// 64 + 16 c + 15: that is the order in which the instruction multiplies; the scales go by quarters in both.
//
// Of eight neighbouring entries' products the instruction cuts each, towards zero, to 2^-13 of the largest sum of a pair's exponents ahead of the fp32
// sums (tried on the instructions: products of 2688 and -2688 leave multiples of 1/8 of their six neighbours, and of all others everything).  No instruction
// takes these formats without; codes widened to bf16 would be exact, at a quarter of the rate.  Over random rows the sums are off by 4e-6 of their size
// where the rounding to bf16 takes 1e-3.
#include "ffn_stream.h"
#include "ffn_tiles.h"
#include "mx.h"

#include <algorithm>
#include <type_traits>

namespace spd {

namespace {
typedef unsigned short bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2_any __attribute__((ext_vector_type(2), aligned(2)));   // `out` is only promised to be aligned to its entries

__device__ inline uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ inline float bf_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ inline float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g)); }
__device__ inline i32x8 e2m1_operand(u32x4 a) { return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}; }
__device__ inline i32x8 e4m3_operand(u32x4 a, u32x4 b) { return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w}; }
constexpr int E4M3 = 0, E2M1 = 4;                  // the instructions' names of the formats
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));   // `out` is only promised to be aligned to its entries
}  // namespace

// ---- the packed weights.  A tile is 128 outputs x 128 hidden entries; unit u of it (16 outputs) keeps, from byte 2048 u on, the codes of its
// gate rows, then of its up rows, [quarter of 32 entries][row][16 bytes], and from byte 16384 + 128 u on the scales, [row][gate, up][quarter].
// Four lanes per (row, quarter), eight entries each: 16 lanes have the 256 bytes of a row that lie in the tile.  Bound by memory: hidden 4096, inter
// 14336 (235 MB of bf16, 62 MB packed) 54 us packed and 52 unpacked on 256 CUs (5.5 and 5.7 TB/s; event times of single
// calls, which hold a launch each: back to back both together take 97), 77 and 73 on 128 (4 TB/s), 132 and 134 on 64.  A workgroup has
// four groups of 256 pieces on their way, and finds its tile once for all its threads; with one piece per thread, each dividing for itself, 62 and 80, 103 and
// 119, 178 and 225.  With a lane per (row, quarter), whose 64 bytes of bf16 are four accesses of its own: 80 and 97 on 256 CUs.
constexpr int SCALES_AT = 16384;
constexpr int PACK_GROUPS = 4;                     // groups whose loads a workgroup has on their way together: of one tile, which has 16
// The 256 threads' place in a group: 16 rows of one side of a unit.  What differs from group to group is uniform.
struct PackGroup {
  size_t tile, src;                                // byte of the tile, first entry of the weight matrix
  int up, unit;
  __device__ PackGroup(uint32_t tile_no, int group, int n_kt, int hidden) {
    const uint32_t tn = tile_no / (uint32_t)n_kt, kt = tile_no % (uint32_t)n_kt;
    up = group & 1; unit = group >> 1;
    tile = (size_t)tile_no * FFN_MX_TILE_BYTES;
    src = (size_t)(tn * 128 + unit * 16) * hidden + kt * 128;
  }
};
struct PackLane {
  int part, quarter, row;                          // part: which eight of the quarter's 32 entries
  __device__ PackLane() : part(threadIdx.x & 3), quarter(threadIdx.x >> 2 & 3), row((int)threadIdx.x >> 4) {}
  __device__ uint32_t src(int hidden) const { return (uint32_t)row * hidden + quarter * 32 + part * 8; }
  __device__ uint32_t codes() const { return quarter * 256 + row * 16 + part * 4; }
  __device__ uint32_t scales() const { return row * 8; }
};

// grid-stride over n_loads times PACK_GROUPS groups, block 256
__global__ __launch_bounds__(256) void ffn_pack_mx_kernel(const bf16_t* __restrict__ wg, const bf16_t* __restrict__ wu, char* __restrict__ dst,
                                                          int n_kt, int hidden, uint32_t n_loads, StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  const PackLane lane;
  for (uint32_t l = blockIdx.x; l < n_loads; l += gridDim.x) {
    u32x4 in[PACK_GROUPS];
#pragma unroll
    for (int g = 0; g < PACK_GROUPS; ++g) {
      const PackGroup p(l / (16 / PACK_GROUPS), l % (16 / PACK_GROUPS) * PACK_GROUPS + g, n_kt, hidden);
      in[g] = __builtin_nontemporal_load((const u32x4*)((p.up ? wu : wg) + p.src + lane.src(hidden)));
    }
#pragma unroll
    for (int g = 0; g < PACK_GROUPS; ++g) {
      const PackGroup p(l / (16 / PACK_GROUPS), l % (16 / PACK_GROUPS) * PACK_GROUPS + g, n_kt, hidden);
      const u32x4 w = in[g];
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) m = max(m, max(w[j] << 16 & 0x7fffffff, w[j] & 0x7fff0000));
      m = max(m, (uint32_t)__shfl_xor((int)m, 1));   // (a quarter's four lanes)
      m = max(m, (uint32_t)__shfl_xor((int)m, 2));
      const bool finite = m < 0x7f800000;          // (E2M1 has neither infinities nor NaN: such a block is NaN as a whole)
      const uint32_t b = finite ? scale_byte_e2m1(m) : MX_NAN_SCALE;
      const float f = finite ? scale_of(b) : 1.f;
      uint32_t c = 0;                              // (the conversion divides by the scale)
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, bf_lo(w[0]), bf_hi(w[0]), f, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, bf_lo(w[1]), bf_hi(w[1]), f, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, bf_lo(w[2]), bf_hi(w[2]), f, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, bf_lo(w[3]), bf_hi(w[3]), f, 3);
      *(uint32_t*)(dst + p.tile + p.unit * 2048 + p.up * 1024 + lane.codes()) = c;
      uint32_t four = b << (8 * lane.quarter);     // the quarters of a row are 4 lanes apart
      four |= (uint32_t)__shfl_xor((int)four, 4);
      four |= (uint32_t)__shfl_xor((int)four, 8);
      if (lane.quarter == 0 && lane.part == 0) *(uint32_t*)(dst + p.tile + SCALES_AT + p.unit * 128 + p.up * 4 + lane.scales()) = four;
    }
  }
}

// The values that the packed weights stand for (exact in bf16).
__global__ __launch_bounds__(256) void ffn_unpack_mx_kernel(const char* __restrict__ w, bf16_t* __restrict__ wg, bf16_t* __restrict__ wu, int n_kt,
                                                            int hidden, uint32_t n_loads, StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  const PackLane lane;
  for (uint32_t l = blockIdx.x; l < n_loads; l += gridDim.x) {
    uint32_t codes[PACK_GROUPS], scales[PACK_GROUPS];
#pragma unroll
    for (int g = 0; g < PACK_GROUPS; ++g) {
      const PackGroup p(l / (16 / PACK_GROUPS), l % (16 / PACK_GROUPS) * PACK_GROUPS + g, n_kt, hidden);
      codes[g] = *(const uint32_t*)(w + p.tile + p.unit * 2048 + p.up * 1024 + lane.codes());
      scales[g] = *(const uint8_t*)(w + p.tile + SCALES_AT + p.unit * 128 + p.up * 4 + lane.scales() + lane.quarter);
    }
#pragma unroll
    for (int g = 0; g < PACK_GROUPS; ++g) {
      const PackGroup p(l / (16 / PACK_GROUPS), l % (16 / PACK_GROUPS) * PACK_GROUPS + g, n_kt, hidden);
      const uint32_t c = codes[g];
      const float f = scales[g] == MX_NAN_SCALE ? __builtin_nanf("") : scale_of(scales[g]);
      auto value = [&](uint32_t code) -> float {
        const uint32_t e = code >> 1 & 3, man = code & 1;
        const float v = e ? __builtin_bit_cast(float, (e + 126) << 23 | man << 22) : 0.5f * (float)man;
        return (code & 8 ? -v : v) * f;
      };
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = pack_bf16(value(c >> (8 * e) & 15), value(c >> (8 * e + 4) & 15));
      __builtin_nontemporal_store(o, (u32x4*)((p.up ? wu : wg) + p.src + lane.src(hidden)));
    }
  }
}

// Up to 128 tokens: bound by reading the weights once.  They go straight from memory into operand registers (a load is 1 KiB of consecutive
// bytes, 16 rows x 128 entries, and 128 bytes of scales), every wave streaming the gate and up rows of 16 outputs, or a part of their entries,
// through a ring of RING slices of 128 entries that no barrier touches.  All 16 NB tokens' rows, which the waves share, go through LDS, XS slices
// at a time in two stages, loaded a stage ahead: a barrier per XS slices.  A workgroup has UNITS x SPLIT waves: UNITS of 16 outputs, the entries of
// each in SPLIT parts, whose sums meet in LDS at the end (ffn_mx_stream_units says which).
// 1 token of hidden 4096, inter 14336 takes 12.4 us on 128 CUs and 9.8 on 256 (5.0 and 6.4 TB/s, weights from HBM), 64 tokens 16 and 14, 128 tokens
// 27 and 19: from there on operand reads from LDS and the matrix instructions take as long as the weights.  Weights through a ring in LDS,
// filled by loads that go straight there: 12.4, at 64 tokens 19 us on 128 CUs.  Rings of eight slices, or x pieces in smaller stages: slower.
template <int NB, int UNITS, int SPLIT, int RING, int XS>
__global__ __launch_bounds__(64 * UNITS * SPLIT, 1) void ffn_gate_up_mx_stream_kernel(const char* __restrict__ x, const uint32_t* __restrict__ xs,
                                                                                    const char* __restrict__ w, bf16_t* __restrict__ out, int T, int K,
                                                                                    int I, StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  constexpr int WAVES = UNITS * SPLIT, THREADS = 64 * WAVES, ROWS = 16 * NB;
  constexpr int PIECES = SPLIT * XS * ROWS * 8, XL = (PIECES + THREADS - 1) / THREADS;   // 16-byte pieces of a stage, per thread
  constexpr int WORDS = SPLIT * XS * ROWS, SL = (WORDS + THREADS - 1) / THREADS;         // scale words of a stage
  constexpr int SLICE = ROWS * 128, X_STAGE = SPLIT * XS * SLICE, STAGE = X_STAGE + WORDS * 4;
  static_assert(RING % XS == 0, "whole stages per ring");
  static_assert((SPLIT - 1) * UNITS * 2 * NB * 1024 <= 2 * STAGE, "room for the parts' sums");
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, c4 = lane >> 4;
  const int n_slices = K / 128, per_part = (n_slices + SPLIT - 1) / SPLIT;
  const int part = wave / UNITS, first = part * per_part, mine = min(per_part, n_slices - first);
  // (waves of the last workgroup without outputs of their own repeat the last ones and store nothing)
  const int n_units = I / 16, unit = (int)blockIdx.x * UNITS + wave % UNITS, u = min(unit, n_units - 1);
  const char* wt = w + (size_t)(u >> 3) * n_slices * FFN_MX_TILE_BYTES;
  const uint32_t code_off = (uint32_t)((u & 7) * 2048 + lane * 16), scale_off = (uint32_t)(SCALES_AT + (u & 7) * 128 + n16 * 8);
  struct Slice { u32x4 g, u; u32x2 s; };
  auto load_w = [&](int s) __attribute__((always_inline)) -> Slice {
    const char* t = wt + (size_t)min(first + s, n_slices - 1) * FFN_MX_TILE_BYTES;
    return Slice{__builtin_nontemporal_load((const u32x4*)(t + code_off)), __builtin_nontemporal_load((const u32x4*)(t + code_off + 1024)),
                 __builtin_nontemporal_load((const u32x2*)(t + scale_off))};
  };
  // piece i of a stage: chunk i % 8 of row i / 8 % ROWS of slice i / (8 ROWS) % XS of part i / (8 ROWS XS); rows past T re-read row T - 1, slices
  // past the last one that one.  Slot s of a row of 128 bytes holds the row's chunk s ^ ((row >> 1) & 7): 16 rows then lie in all banks.
  u32x4 xr[XL];
  uint32_t sr[SL];
  auto slice_of = [&](int st, int q) __attribute__((always_inline)) -> int { return min(q / XS * per_part + st * XS + q % XS, n_slices - 1); };
  auto load_x = [&](int st) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < XL; ++j) {
      const int i = min(tid + THREADS * j, PIECES - 1), row = i / 8 % ROWS;
      xr[j] = *(const u32x4*)(x + (uint32_t)(min(row, T - 1) * K + slice_of(st, i / (8 * ROWS)) * 128 + i % 8 * 16));
    }
#pragma unroll
    for (int j = 0; j < SL; ++j) {
      const int i = min(tid + THREADS * j, WORDS - 1);
      sr[j] = xs[(uint32_t)(slice_of(st, i / ROWS) * T + min(i % ROWS, T - 1))];
    }
  };
  auto store_x = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < XL; ++j) {
      const int i = tid + THREADS * j, row = i / 8 % ROWS;
      if (PIECES % THREADS == 0 || i < PIECES) *(u32x4*)(smem + buf * STAGE + i / 8 * 128 + ((i % 8) ^ ((row >> 1) & 7)) * 16) = xr[j];
    }
#pragma unroll
    for (int j = 0; j < SL; ++j) {
      const int i = tid + THREADS * j;
      if (WORDS % THREADS == 0 || i < WORDS) *(uint32_t*)(smem + buf * STAGE + X_STAGE + i * 4) = sr[j];
    }
  };
  f32x4 acc[2][NB];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  Slice wr[RING];
  load_x(0);
  store_x(0);
  // the next x pieces before the weights, as inside the loop: the compiler then waits for them with the weights still on their way
  load_x(1);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < RING; ++s) wr[s] = load_w(s);
  int buf = 0;
  const int sw = (n16 >> 1) & 7, x0 = part * XS * SLICE + n16 * 128 + (c4 ^ sw) * 16, x1 = part * XS * SLICE + n16 * 128 + ((4 + c4) ^ sw) * 16;
  const int s_at = X_STAGE + part * XS * ROWS * 4 + n16 * 4 + c4;
  const int n_stages = (per_part + XS - 1) / XS;
  // RING slices from s0 on, with the loads of the next RING; `tail`: of both, those that there are
  auto round = [&](int s0, auto tail) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < RING; ++r) {
      if (r % XS == 0) {
        // everyone's pieces of this stage are there, and everyone is done with the one before, which the next pieces replace
        __syncthreads();
        store_x(buf ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        if (!tail || (s0 + r) / XS + 2 < n_stages) load_x((s0 + r) / XS + 2);
        __builtin_amdgcn_sched_barrier(0);
      }
      const char* st = smem + buf * STAGE;
      if (!tail || s0 + r < mine) {
        const int sg = (int)(wr[r].s.x >> (8 * c4)), su = (int)(wr[r].s.y >> (8 * c4));
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const i32x8 xv = e4m3_operand(*(const u32x4*)(st + x0 + r % XS * SLICE + b * 2048), *(const u32x4*)(st + x1 + r % XS * SLICE + b * 2048));
          const int sx = *(const uint8_t*)(st + s_at + r % XS * ROWS * 4 + b * 64);
          acc[0][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(e2m1_operand(wr[r].g), xv, acc[0][b], E2M1, E4M3, 0, sg, 0, sx);
          acc[1][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(e2m1_operand(wr[r].u), xv, acc[1][b], E2M1, E4M3, 0, su, 0, sx);
          if (b == 3) __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (!tail || s0 + r + RING < mine) wr[r] = load_w(s0 + r + RING);
      __builtin_amdgcn_sched_barrier(0);
      if (r % XS == XS - 1) buf ^= 1;
    }
  };
  int s0 = 0;
  const int whole = n_slices - (SPLIT - 1) * per_part;            // slices that every part has: fewer than some
  for (; s0 + 2 * RING <= whole; s0 += RING) round(s0, std::false_type{});
  for (; s0 < per_part; s0 += RING) round(s0, std::true_type{});
  if constexpr (SPLIT > 1) {                      // the parts' sums, through LDS, to the first, which adds them up in order
    __syncthreads();
    f32x4* const sums = (f32x4*)smem + lane;
    if (part > 0) {
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) sums[(((part - 1) * UNITS + wave % UNITS) * 2 * NB + i) * 64] = acc[i / NB][i % NB];
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 0; p < SPLIT - 1; ++p)
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) acc[i / NB][i % NB] += sums[((p * UNITS + wave) * 2 * NB + i) * 64];
  }
  // element i of lane (n16, c4) is output 4 c4 + i of token n16 of its block
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int t = 16 * b + n16;
    const uint32_t y0 = pack_bf16(silu(acc[0][b][0]) * acc[1][b][0], silu(acc[0][b][1]) * acc[1][b][1]);
    const uint32_t y1 = pack_bf16(silu(acc[0][b][2]) * acc[1][b][2], silu(acc[0][b][3]) * acc[1][b][3]);
    if (t < T && unit < n_units) *(u32x2_any*)(out + (size_t)t * I + unit * 16 + 4 * c4) = u32x2_any{y0, y1};
  }
}

// 64 MB tokens x 128 outputs (256 rows of weights).  As ffn_gate_up_large_kernel: eight waves in two groups that run half a step apart, one group's
// matrix instructions beside the other group's loads and operand reads, an s_barrier at every change; a workgroup walks the tiles slot, slot +
// gridDim / xcds, .. with its loads running ahead across tiles.  A step is 64 hidden entries, 2 MB v_mfma_scale_f32_32x32x64 per wave, 128 MB cycles at the
// rate of the 8-bit operand; both operands' bytes come in pairs of steps (128 entries: whole cache lines of x, a tile of the packed weights), three
// pairs in LDS: 3 x (8 MB KiB x, 16 KiB codes of weights, 1 KiB of scales of either).
// MB is 4, or 2 where half as many tokens per tile fill the share better (low_tiles_pay).
// Bound by the matrix instructions: 8192 tokens of hidden 4096, inter 14336 on 128 compute units 892 us, 2.16 PFLOP/s, 86% of what 64 cycles per
// instruction allow at 2.4 GHz; 4096 tokens 475 us, on 256 compute units 312 (3.1 PFLOP/s).
template <int MB>
__global__ __launch_bounds__(512, 2) void ffn_gate_up_mx_large_kernel(const char* __restrict__ x, const uint32_t* __restrict__ xs, const char* __restrict__ w,
                                                                      bf16_t* __restrict__ out, int T, int K, int I, int tiles_m, int tiles_n, int xcds,
                                                                      StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  constexpr int BM = 64 * MB, JX = MB / 2, X_PAIR = BM * 128, W_PAIR = SCALES_AT, S_PAIR = 2048, NP = 3;   // bytes of a pair, pairs in LDS
  constexpr int W_LDS = NP * X_PAIR, S_LDS = W_LDS + NP * W_PAIR;
  __shared__ __attribute__((aligned(1024))) char smem[S_LDS + NP * S_PAIR];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, hh = lane >> 5;
  const int wm = wave >> 2, wn = wave & 3;        // wm: also the wave's group
  const TileOrder order(tiles_m, tiles_n, xcds);
  const int n_slots = order.slots(), slot_step = (int)gridDim.x / xcds;
  int slot = (int)blockIdx.x / xcds;
  if (slot >= n_slots) return;
  const uint32_t smem_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int n_pairs = K / 128, n_steps = 2 * n_pairs;
  int left = ((n_slots - 1 - slot) / slot_step + 1) * n_steps;   // steps of all tiles of this workgroup from the current one on

  // ---- loads, in two halves of a pair: half the rows of x (JX instructions per wave; slot s of a row of 128 bytes holds the row's chunk
  // s ^ ((row >> 1) & 7)) and four units of the weights (one); with the first half the scales (one: waves 0 .. 3 the tokens', of 128 tokens twice,
  // 4 .. 7 the weights').  Token rows past T re-read row T - 1.
  const int x_chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
  uint32_t x_voff[2][JX], s_voff;                  // [half][j]
  const uint32_t w_voff = (uint32_t)lane * 16;
  const char *x_ptr, *w_ptr, *s_ptr;              // the next pair's
  size_t s_step;                                  // of s_ptr, from pair to pair
  int l_slot = slot, l_left = n_pairs;            // its tile, and pairs until that tile's end
  auto l_tile = [&]() __attribute__((always_inline)) {
    int tm, tn;
    order.tile(l_slot, tm, tn);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < JX; ++j)
        x_voff[hf][j] = (uint32_t)min(BM / 2 * hf + 8 * (wave + 8 * j) + (lane >> 3), T - 1 - tm * BM) * (uint32_t)K + (uint32_t)x_chunk * 16;
    x_ptr = x + (size_t)(tm * BM) * K;
    w_ptr = w + (size_t)tn * n_pairs * FFN_MX_TILE_BYTES + wave * 1024;
    if (wave < 4) {
      s_ptr = (const char*)(xs + tm * BM);
      s_step = (size_t)T * 4;
      s_voff = (uint32_t)min(64 * (wave % MB) + lane, T - 1 - tm * BM) * 4;
    } else {
      s_ptr = w + (size_t)tn * n_pairs * FFN_MX_TILE_BYTES + SCALES_AT;
      s_step = FFN_MX_TILE_BYTES;
      s_voff = (uint32_t)(64 * (wave - 4) + lane) * 4;
    }
  };
  l_tile();
  auto load = [&](int stage, int hf) __attribute__((always_inline)) {
    const uint32_t lds = smem_base + stage * X_PAIR + hf * (X_PAIR / 2) + wave * 1024;
#pragma unroll
    for (int j = 0; j < JX; ++j) dma16s(x_ptr, x_voff[hf][j], lds + j * 8192);
    dma16s(w_ptr + hf * 8192, w_voff, smem_base + W_LDS + stage * W_PAIR + hf * 8192 + wave * 1024);
    if (hf == 0) {
      dma4s(s_ptr, s_voff, smem_base + S_LDS + stage * S_PAIR + (wave < 4 ? wave % MB : wave) * 256);
    } else {
      x_ptr += 128;
      w_ptr += FFN_MX_TILE_BYTES;
      s_ptr += s_step;
      if (--l_left == 0) {
        l_left = n_pairs;
        l_slot += slot_step;
        if (l_slot < n_slots) l_tile();
      }
    }
  };

  // ---- LDS operand addresses.  Of a step's 64 entries the lane half hh has, of the weights, the quarter 2 sl + hh (32 entries, 16 bytes); of x the
  // chunks 4 sl + hh and 4 sl + 2 + hh; and of both the scale of that quarter.  The stage is part of a read's 16-bit immediate; the third
  // pair of x lies beyond its reach and gets lane addresses of its own.
  int x_off[2][2][2];                             // [third stage][step of the pair][chunk]
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int sl = 0; sl < 2; ++sl) {
      x_off[0][sl][j] = (wm * (BM / 2) + n32) * 128 + ((4 * sl + 2 * j + hh) ^ ((n32 >> 1) & 7)) * 16;
      x_off[1][sl][j] = x_off[0][sl][j] + 2 * X_PAIR;
      asm volatile("" : "+v"(x_off[1][sl][j]));   // a value of its own, not "x_off + constant" to be recomputed
    }
  const int unit = 2 * wn + (n32 >> 4), row = n32 & 15;
  int w_off = W_LDS + unit * 2048 + hh * 256 + row * 16, ws_off = S_LDS + 1024 + unit * 128 + row * 8, xs_off = S_LDS + (wm * (BM / 2) + n32) * 4;
  asm volatile("" : "+v"(w_off), "+v"(ws_off), "+v"(xs_off));
  u32x4 ox[MB][2], ow[2];
  uint32_t sx[MB], sw[2];                         // scale bytes: of the pair's first step in byte 0, of its second in byte 2
  // acc[mb][0] = gate, acc[mb][1] = up: element i of lane (n32, hh) is output 8 (i / 4) + 4 hh + i % 4 of token 32 mb + n32
  f32x16 acc[MB][2];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[mb][nb][e] = 0.f;
  };
  clear();
  auto barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // ahead of the first step: pairs 0 and 1, as the steps -4 .. -1 would load them
  load(0, 0);
  load(0, 1);
  if (left > 2) {
    load(1, 0);
    load(1, 1);
    SPD_WAIT_VMCNT(2 * JX + 3);
  } else {
    SPD_WAIT_VMCNT(0);
  }
  barrier();                                      // pair 0 is there
  if (wm) barrier();                              // the second group starts half a step later

  int ct = 0;                                     // step of the tile
  int ready = 0;                                  // steps that need not wait: the end of a tile has awaited all loads up to it
  auto step = [&](auto stc) __attribute__((always_inline)) {
    constexpr int ST = stc, SL = ST & 1, P = ST / 2;   // step modulo the ring's period; step of the pair
    // Loading and reading half of step u, of pair p.  The stage being loaded held pair p - 1, whose reads both groups had behind them at the
    // last barrier.  At this half's end the wave's own reads are done, and so is what it loaded up to step u - 2: its part of the pair that
    // the other group may read a whole step from now, this one in one and a half.
    if (left > 4) load((P + 2) % NP, SL);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (SL == 0) {
      const uint2 two = *(const uint2*)(smem + ws_off + P * S_PAIR);
      sw[0] = two.x; sw[1] = two.y;
#pragma unroll
      for (int r = 0; r < MB; ++r) sx[r] = *(const uint32_t*)(smem + xs_off + P * S_PAIR + r * 128);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) ow[r] = *(const u32x4*)(smem + w_off + P * W_PAIR + SL * 512 + r * 1024);
#pragma unroll
    for (int r = 0; r < MB; ++r)
#pragma unroll
      for (int j = 0; j < 2; ++j) ox[r][j] = *(const u32x4*)(smem + x_off[P == 2][SL][j] + (P == 1 ? X_PAIR : 0) + r * (32 * 128));
    __builtin_amdgcn_sched_barrier(0);
    if (ready > 0) --ready;
    else if (left >= 5) SPD_WAIT_VMCNT(2 * JX + 3);   // this step's loads and those of the one before
    else if (left == 4) SPD_WAIT_VMCNT(JX + 1);
    else SPD_WAIT_VMCNT(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);           // lgkmcnt(0)
    if constexpr (SL == 0) {
#pragma unroll
      for (int r = 0; r < 2; ++r) sw[r] >>= 8 * hh;
#pragma unroll
      for (int r = 0; r < MB; ++r) sx[r] >>= 8 * hh;
    }
    barrier();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
        acc[mb][nb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(e2m1_operand(ow[nb]), e4m3_operand(ox[mb][0], ox[mb][1]), acc[mb][nb], E2M1, E4M3,
                                                                      2 * SL, (int)sw[nb], 2 * SL, (int)sx[mb]);
    // (the products belong here: without side effects of their own they would be moved past the barriers to where their sums are used)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) asm volatile("" : "+v"(acc[mb][0]), "+v"(acc[mb][1]));
    __builtin_amdgcn_s_setprio(0);
    barrier();
    --left;
    ++ct;
  };
  // ---- the tile's end, as in ffn_gate_up_large_kernel: the halves of the wave exchange four outputs each, so that a lane stores eight consecutive
  // ones.  All loads so far are awaited ahead of the first store: the next two steps then have nothing to wait for, and do not wait for the
  // stores either.
  auto finish_tile = [&]() __attribute__((always_inline)) {
    int tm, tn;
    order.tile(slot, tm, tn);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      uint32_t y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        y[i] = pack_bf16(silu(acc[mb][0][2 * i]) * acc[mb][1][2 * i], silu(acc[mb][0][2 * i + 1]) * acc[mb][1][2 * i + 1]);
      if (mb == 0) SPD_WAIT_VMCNT(0);
      const int t = tm * BM + wm * (BM / 2) + mb * 32 + n32;
      bf16_t* o = out + (size_t)t * I + tn * 128 + wn * 32 + 8 * hh;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        // (machine code: the compiler's builtin for the swap loses the second result)
        asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\tv_permlane32_swap_b32 %2, %3\n\ts_nop 1"
                     : "+v"(y[4 * p]), "+v"(y[4 * p + 2]), "+v"(y[4 * p + 1]), "+v"(y[4 * p + 3]));
        if (t < T) *(u32x4_any*)(o + 16 * p) = u32x4_any{y[4 * p], y[4 * p + 1], y[4 * p + 2], y[4 * p + 3]};
      }
    }
  };
  // a pair of steps and, behind a tile's last one, its end; false behind the last tile
  auto pair = [&](auto pc) __attribute__((always_inline)) -> bool {
    constexpr int P = pc;
    step(std::integral_constant<int, 2 * P>{});
    step(std::integral_constant<int, 2 * P + 1>{});
    if (ct == n_steps) {
      finish_tile();
      if (left == 0) return false;
      slot += slot_step;
      clear();
      ct = 0;
      ready = 2;
    }
    return true;
  };
  for (;;) {
    if (!pair(std::integral_constant<int, 0>{})) break;
    if (!pair(std::integral_constant<int, 1>{})) break;
    if (!pair(std::integral_constant<int, 2>{})) break;
  }
  if (!wm) barrier();                             // as many as the second group
}

template <int NB>
static hipError_t launch_mx_stream(const void* x, const void* x_scales, const void* w_mx, void* out, int T, int K, int I, int cus, const StepMark& mark,
                                   hipStream_t stream) {
  auto launch = [&](auto kernel, int units, int split) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((I / 16 + units - 1) / units)), dim3((unsigned)(64 * units * split)), 0, stream, (const char*)x,
                       (const uint32_t*)x_scales, (const char*)w_mx, (bf16_t*)out, T, K, I, mark);
  };
  const int units = ffn_mx_stream_units(NB, I / 16, cus);
  if constexpr (NB <= 4) {
    if (units == 7) launch(ffn_gate_up_mx_stream_kernel<NB, 7, 1, 4, 4>, 7, 1);
    if (units == 6) launch(ffn_gate_up_mx_stream_kernel<NB, 6, 1, 4, 4>, 6, 1);
    if (units == 5) launch(ffn_gate_up_mx_stream_kernel<NB, 5, 1, 4, 4>, 5, 1);
    if (units == 4) launch(ffn_gate_up_mx_stream_kernel<NB, 4, 1, 4, 4>, 4, 1);
    if (units == 3) launch(ffn_gate_up_mx_stream_kernel<NB, 3, 2, 4, 4>, 3, 2);
    if (units == 2) launch(ffn_gate_up_mx_stream_kernel<NB, 2, 2, 4, 4>, 2, 2);
  } else {
    if (units == 4) launch(ffn_gate_up_mx_stream_kernel<NB, 4, 2, 4, 2>, 4, 2);
    if (units == 2) launch(ffn_gate_up_mx_stream_kernel<NB, 2, 2, 4, 2>, 2, 2);
  }
  if (units == 8) launch(ffn_gate_up_mx_stream_kernel<NB, 8, 1, 4, 4>, 8, 1);
  return hipGetLastError();
}

template <int MB>
static hipError_t launch_mx_tiles(const void* x, const void* x_scales, const void* w_mx, void* out, int T, int K, int I, int xcds, int cus, bool exclusive,
                                  const StepMark& mark, hipStream_t stream) {
  const int tiles_m = (int)(((int64_t)T + 64 * MB - 1) / (64 * MB)), tiles_n = I / 128;
  const int persistent = exclusive ? cus : 0;      // workgroups, one per compute unit of a share that has them to itself; 0: one per tile
  if (tiles_n < xcds || persistent % xcds) xcds = 1;
  int64_t n = xcds > 1 ? (int64_t)((tiles_n + xcds - 1) / xcds) * tiles_m * xcds : (int64_t)tiles_m * tiles_n;
  if (n > INT32_MAX) return hipErrorInvalidValue;
  if (persistent) n = std::min<int64_t>(n, persistent);
  hipLaunchKernelGGL(ffn_gate_up_mx_large_kernel<MB>, dim3((unsigned)n), dim3(512), 0, stream, (const char*)x, (const uint32_t*)x_scales, (const char*)w_mx,
                     (bf16_t*)out, T, K, I, tiles_m, tiles_n, xcds, mark);
  return hipGetLastError();
}

// Whether tiles of 128 tokens are to be taken instead of 256.  One round of them, a tile per compute unit, takes 0.70 .. 0.75 of the time of one of the larger
// ones, which are fed from LDS once for twice the products, and every further round 0.65; three rounds for two are a tie.  256 / 128 tokens
// per tile: hidden 4096, inter 14336 on 256 CUs, 256 tokens (1 round either) 43.3 / 32.4 us, 512 (1, 2) 47.2 / 59.2, 700 (2, 3) 82.9 / 80.5, 8192 on 128 CUs (28, 56)
// 892 / 1200; 300 on 96 CUs (3, 4) 105 / 94; hidden 4096, inter 3584 on 128 CUs, 512 (1, 1) 38.3 / 28.4.
static bool low_tiles_pay(int T, int I, int cus) {
  const int64_t columns = I / 128, high = (((int64_t)T + 255) / 256 * columns + cus - 1) / cus, low = (((int64_t)T + 127) / 128 * columns + cus - 1) / cus;
  return 2 * low < 3 * high;
}

hipError_t launch_ffn_gate_up_mx(const void* x, const void* x_scales, const void* w_mx, void* out, int T, int K, int I, int xcds, int cus, bool exclusive,
                                 const StepMark& mark, hipStream_t stream) {
  if (T > 128)
    return low_tiles_pay(T, I, cus) ? launch_mx_tiles<2>(x, x_scales, w_mx, out, T, K, I, xcds, cus, exclusive, mark, stream)
                                    : launch_mx_tiles<4>(x, x_scales, w_mx, out, T, K, I, xcds, cus, exclusive, mark, stream);
  if (T <= 16) return launch_mx_stream<1>(x, x_scales, w_mx, out, T, K, I, cus, mark, stream);
  if (T <= 32) return launch_mx_stream<2>(x, x_scales, w_mx, out, T, K, I, cus, mark, stream);
  if (T <= 64) return launch_mx_stream<4>(x, x_scales, w_mx, out, T, K, I, cus, mark, stream);
  return launch_mx_stream<8>(x, x_scales, w_mx, out, T, K, I, cus, mark, stream);
}

// pack and unpack: rounds of PACK_GROUPS groups (a matrix pair that fits the card has fewer than 2^32), and workgroups
static uint32_t pack_loads(int K, int I) { return (uint32_t)((int64_t)(I / 128) * (K / 128) * (16 / PACK_GROUPS)); }

hipError_t launch_ffn_pack_mx(const void* w_gate, const void* w_up, void* w_mx, int K, int I, const StepMark& mark, hipStream_t stream) {
  const uint32_t n = pack_loads(K, I);
  hipLaunchKernelGGL(ffn_pack_mx_kernel, dim3(std::min(n, 8192u)), dim3(256), 0, stream, (const bf16_t*)w_gate, (const bf16_t*)w_up, (char*)w_mx, K / 128, K, n, mark);
  return hipGetLastError();
}

hipError_t launch_ffn_unpack_mx(const void* w_mx, void* w_gate, void* w_up, int K, int I, const StepMark& mark, hipStream_t stream) {
  const uint32_t n = pack_loads(K, I);
  hipLaunchKernelGGL(ffn_unpack_mx_kernel, dim3(std::min(n, 8192u)), dim3(256), 0, stream, (const char*)w_mx, (bf16_t*)w_gate, (bf16_t*)w_up, K / 128, K, n, mark);
  return hipGetLastError();
}

}  // namespace spd
