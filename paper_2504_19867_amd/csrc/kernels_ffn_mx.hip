// First step of the gated FFN over MXFP4 weights and MX E4M3 rows:
//     out[t, i] = silu(g) u,   g = sum_k x[t, k] W_gate[i, k],  u = sum_k x[t, k] W_up[i, k]
// on the values that codes and scales stand for, fp32 sums, one rounding to bf16.  silu(z) = z / (1 + exp(-z)).
//
// The scaled matrix instructions take both formats as they are: a lane holds 32 codes of one row (16 bytes of E2M1, 32 of E4M3) and the
// scale byte of its 32 entries.  Weights are the A operand, so that a lane has consecutive outputs of one token.  Where the E2M1 lane of row r
// and quarter c of a step of 128 entries holds the entries 32 c .. 32 c + 31, the E4M3 lane holds 16 c .. 16 c + 15 and 64 + 16 c ..
// 64 + 16 c + 15: that is the order in which the instruction multiplies; the scales go by quarters in both.
#include "mx.h"

#include <algorithm>

namespace spd {

namespace {
typedef unsigned short bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ inline float bf_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ inline float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g)); }
__device__ inline i32x8 e2m1_operand(u32x4 a) { return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}; }
__device__ inline i32x8 e4m3_operand(u32x4 a, u32x4 b) { return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w}; }
constexpr int E4M3 = 0, E2M1 = 4;                  // the instructions' names of the formats
}  // namespace

// ---- the packed weights.  A tile is 128 outputs x 128 hidden entries; unit u of it (16 outputs) keeps, from byte 2048 u on, the codes of its
// gate rows, then of its up rows, [quarter of 32 entries][row][16 bytes], and from byte 16384 + 128 u on the scales, [row][gate, up][quarter].
// One thread per (row, quarter): piece i of a tile is piece i of the codes, so that reads are 256 consecutive bytes of 16 rows per wave and
// writes 1 KiB.  Bound by memory.
constexpr int SCALES_AT = 16384;
struct PackPlace {
  size_t tile;                                     // byte of the tile
  size_t src;                                      // entry of the weight matrix
  int piece, up, quarter, row, unit;
  __device__ PackPlace(long i, int n_kt, int hidden) {
    const long t = i >> 10;
    piece = (int)(i & 1023);
    unit = piece >> 7; up = (piece >> 6) & 1; quarter = (piece >> 4) & 3; row = piece & 15;
    const long tn = t / n_kt, kt = t % n_kt;
    tile = (size_t)t * FFN_MX_TILE_BYTES;
    src = (size_t)(tn * 128 + unit * 16 + row) * hidden + kt * 128 + quarter * 32;
  }
  __device__ size_t scale_word() const { return tile + SCALES_AT + unit * 128 + row * 8 + up * 4; }
};

// E2M1 code of a magnitude up to 6: nearest of 0, .5, 1, 1.5, 2, 3, 4, 6, halfway to the even code
__device__ inline uint32_t e2m1_code(float x) {
  const float a = fabsf(x);
  const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
  return c | (__builtin_bit_cast(uint32_t, x) >> 28 & 8);
}

// grid-stride over 1024 n_tiles pieces, block 256 (whole waves)
__global__ __launch_bounds__(256) void ffn_pack_mx_kernel(const bf16_t* __restrict__ wg, const bf16_t* __restrict__ wu, char* __restrict__ dst,
                                                          int n_kt, int hidden, long n_pieces, StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  const long stride = (long)gridDim.x * blockDim.x;
  for (long i = (long)blockIdx.x * blockDim.x + threadIdx.x; i < n_pieces; i += stride) {
    const PackPlace p(i, n_kt, hidden);
    const uint4* src = (const uint4*)((p.up ? wu : wg) + p.src);
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 v = src[j];
      w[4 * j] = v.x; w[4 * j + 1] = v.y; w[4 * j + 2] = v.z; w[4 * j + 3] = v.w;
    }
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) m = max(m, max(w[j] << 16 & 0x7fffffff, w[j] & 0x7fff0000));
    const bool finite = m < 0x7f800000;            // (E2M1 has neither infinities nor NaN: such a block is NaN as a whole)
    const uint32_t b = finite ? scale_byte_e2m1(m) : MX_NAN_SCALE;
    const float f = finite ? inverse_scale_of(b) : 0.f;
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c[j] |= (e2m1_code(bf_lo(w[4 * j + e]) * f) | e2m1_code(bf_hi(w[4 * j + e]) * f) << 4) << (8 * e);
    }
    *(uint4*)(dst + p.tile + p.piece * 16) = uint4{c[0], c[1], c[2], c[3]};
    uint32_t four = b << (8 * p.quarter);          // the quarters of a row are 16 lanes apart
    four |= (uint32_t)__shfl_xor((int)four, 16);
    four |= (uint32_t)__shfl_xor((int)four, 32);
    if (p.quarter == 0) *(uint32_t*)(dst + p.scale_word()) = four;
  }
}

// The values that the packed weights stand for (exact in bf16).
__global__ __launch_bounds__(256) void ffn_unpack_mx_kernel(const char* __restrict__ w, bf16_t* __restrict__ wg, bf16_t* __restrict__ wu, int n_kt,
                                                            int hidden, long n_pieces, StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  const long stride = (long)gridDim.x * blockDim.x;
  for (long i = (long)blockIdx.x * blockDim.x + threadIdx.x; i < n_pieces; i += stride) {
    const PackPlace p(i, n_kt, hidden);
    const uint4 v = *(const uint4*)(w + p.tile + p.piece * 16);
    const uint32_t c[4] = {v.x, v.y, v.z, v.w};
    const uint32_t b = *(const uint8_t*)(w + p.scale_word() + p.quarter);
    const float f = b == MX_NAN_SCALE ? __builtin_nanf("") : scale_of(b);
    auto value = [&](uint32_t code) -> float {
      const uint32_t e = code >> 1 & 3, man = code & 1;
      const float v = e ? __builtin_bit_cast(float, (e + 126) << 23 | man << 22) : 0.5f * (float)man;
      return (code & 8 ? -v : v) * f;
    };
    uint4* out = (uint4*)((p.up ? wu : wg) + p.src);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = pack_bf16(value(c[j] >> (8 * e) & 15), value(c[j] >> (8 * e + 4) & 15));
      out[j] = uint4{o[0], o[1], o[2], o[3]};
    }
  }
}

// grid (inter / 16 * token blocks of 16), block 64: a wave computes 16 outputs of 16 tokens, operands straight from memory.
__global__ __launch_bounds__(64) void ffn_gate_up_mx_kernel(const char* __restrict__ x, const uint32_t* __restrict__ xs, const char* __restrict__ w,
                                                            bf16_t* __restrict__ out, int T, int K, int I, StepMark mark) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(mark);
  const int lane = threadIdx.x, n16 = lane & 15, c4 = lane >> 4, n_kt = K / 128;
  const int unit = blockIdx.x % (I / 16), t = blockIdx.x / (I / 16) * 16 + n16, tc = min(t, T - 1);
  const char* wt = w + (size_t)(unit >> 3) * n_kt * FFN_MX_TILE_BYTES;
  const char* codes = wt + (unit & 7) * 2048 + lane * 16;
  const char* scales = wt + SCALES_AT + (unit & 7) * 128 + n16 * 8;
  const char* xr = x + (size_t)tc * K + 16 * c4;
  f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = g;
  for (int kt = 0; kt < n_kt; ++kt) {
    const size_t at = (size_t)kt * FFN_MX_TILE_BYTES;
    const u32x4 wg = *(const u32x4*)(codes + at), wu = *(const u32x4*)(codes + at + 1024);
    const uint2 s = *(const uint2*)(scales + at);
    const uint32_t sx = xs[(size_t)kt * T + tc] >> (8 * c4);
    const i32x8 xv = e4m3_operand(*(const u32x4*)(xr + kt * 128), *(const u32x4*)(xr + kt * 128 + 64));
    g = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(e2m1_operand(wg), xv, g, E2M1, E4M3, 0, (int)(s.x >> (8 * c4)), 0, (int)sx);
    u = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(e2m1_operand(wu), xv, u, E2M1, E4M3, 0, (int)(s.y >> (8 * c4)), 0, (int)sx);
  }
  // element i of lane (n16, c4) is output 4 c4 + i of token n16
  if (t >= T) return;
  const uint32_t y0 = pack_bf16(silu(g[0]) * u[0], silu(g[1]) * u[1]), y1 = pack_bf16(silu(g[2]) * u[2], silu(g[3]) * u[3]);
  bf16_t* o = out + (size_t)t * I + unit * 16 + 4 * c4;
  o[0] = (bf16_t)y0; o[1] = (bf16_t)(y0 >> 16); o[2] = (bf16_t)y1; o[3] = (bf16_t)(y1 >> 16);
}

hipError_t launch_ffn_gate_up_mx(const void* x, const void* x_scales, const void* w_mx, void* out, int T, int K, int I, int xcds, int cus, bool exclusive,
                                 const StepMark& mark, hipStream_t stream) {
  (void)xcds; (void)cus; (void)exclusive;
  const int64_t wgs = (int64_t)(I / 16) * ((T + (int64_t)15) / 16);
  if (wgs > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL(ffn_gate_up_mx_kernel, dim3((unsigned)wgs), dim3(64), 0, stream, (const char*)x, (const uint32_t*)x_scales, (const char*)w_mx,
                     (bf16_t*)out, T, K, I, mark);
  return hipGetLastError();
}

static unsigned pack_grid(long n_pieces) { return (unsigned)std::min<long>((n_pieces + 255) / 256, 8192); }

hipError_t launch_ffn_pack_mx(const void* w_gate, const void* w_up, void* w_mx, int K, int I, const StepMark& mark, hipStream_t stream) {
  const long n_pieces = (long)(I / 128) * (K / 128) * 1024;
  hipLaunchKernelGGL(ffn_pack_mx_kernel, dim3(pack_grid(n_pieces)), dim3(256), 0, stream, (const bf16_t*)w_gate, (const bf16_t*)w_up, (char*)w_mx, K / 128,
                     K, n_pieces, mark);
  return hipGetLastError();
}

hipError_t launch_ffn_unpack_mx(const void* w_mx, void* w_gate, void* w_up, int K, int I, const StepMark& mark, hipStream_t stream) {
  const long n_pieces = (long)(I / 128) * (K / 128) * 1024;
  hipLaunchKernelGGL(ffn_unpack_mx_kernel, dim3(pack_grid(n_pieces)), dim3(256), 0, stream, (const char*)w_mx, (bf16_t*)w_gate, (bf16_t*)w_up, K / 128, K,
                     n_pieces, mark);
  return hipGetLastError();
}

}  // namespace spd
