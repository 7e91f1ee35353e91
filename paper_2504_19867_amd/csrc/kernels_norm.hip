// RMS norm with the residual's addition, and an output in bf16 or in 8 bits with scales.
//
// For a row x of `hidden` entries (and the residual stream's row r, where there is one):
//     h = bf16(x + r),  r <- h,      y_i = h_i w_i / sqrt(mean_j h_j^2 + eps)
// rounded once to fp32 and from there to bf16, or to MX E4M3 (mx.h: blocks of 32 entries under one power-of-two scale).  Squares are summed in fp64, and
// the root's inverse is carried in two fp32 numbers: a scale byte turns on whether a block's largest y passes a border, and an error of the sum's moves
// all of a row's entries to the same side of theirs.  fp64 products: 4 % longer on prompt batches, the two numbers nothing.
//
// Bound by memory: every row is read once and written once.  A workgroup takes a row and keeps it in registers between the sum of squares
// and the output; the block maxima of the 8-bit form are formed over the four lanes that hold a block.
//
// Two pieces of 8 entries per thread: one leaves half the loads on the way when the sum is waited for, four or more make few rows slow.  8-bit output with
// the residual, by a phase of 128 compute units (7 bytes per entry; event times, which hold 4 us of launch): 8192 rows of hidden 4096, two / one / four pieces
// 62.4 / 67.7 / 65.0 us (3.8 TB/s, where a copy reaches 4.3), 8192 rows of 8192 127 / 143 / 129, of 2048 25.0 / 27.6 / 24.8; one row of 8192
// 6.0 / 6.0 / 7.1, of 16384 6.7 (1024 threads at most) and with four 6.8.
#include "mx.h"

#include <algorithm>

namespace spd {

namespace {
typedef unsigned short bf16_t;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ inline float bf_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

struct NormArgs {
  const bf16_t* x;
  bf16_t* residual;
  const bf16_t* w;
  void* out;
  uint32_t* scales;                                // [hidden / 128][T]: the four scale bytes of 128 entries
  float eps;
  double per_entry;                                // 1 / hidden
  int T, hidden, first;                            // rows of all launches; this one's first
  StepMark mark;
};
}  // namespace

// grid (rows), block THREADS: a row of up to THREADS * PIECES pieces of 8 entries
template <int THREADS, int PIECES, bool MX>
__global__ __launch_bounds__(THREADS) void rmsnorm_kernel(NormArgs a) {
  if (blockIdx.x == 0 && threadIdx.x == 0) store_mark(a.mark);
  const int tid = threadIdx.x, n = a.hidden >> 3, t = a.first + blockIdx.x;
  const size_t row = (size_t)t * a.hidden;
  uint4 h[PIECES];
  double sum = 0.;
#pragma unroll
  for (int j = 0; j < PIECES; ++j) {
    const int p = tid + THREADS * j;
    h[j] = uint4{0, 0, 0, 0};
    if (p < n) {
      h[j] = *(const uint4*)(a.x + row + 8 * p);
      if (a.residual) {
        const uint4 r = *(const uint4*)(a.residual + row + 8 * p);
        uint32_t hw[4] = {h[j].x, h[j].y, h[j].z, h[j].w};
        const uint32_t rw[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) hw[i] = pack_bf16(bf_lo(hw[i]) + bf_lo(rw[i]), bf_hi(hw[i]) + bf_hi(rw[i]));
        h[j] = uint4{hw[0], hw[1], hw[2], hw[3]};
        *(uint4*)(a.residual + row + 8 * p) = h[j];
      }
    }
    const uint32_t hw[4] = {h[j].x, h[j].y, h[j].z, h[j].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double lo = bf_lo(hw[i]), hi = bf_hi(hw[i]);
      sum = __builtin_fma(lo, lo, sum);
      sum = __builtin_fma(hi, hi, sum);
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
  if constexpr (THREADS > 64) {
    __shared__ double part[THREADS / 64];
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    sum = 0.;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) sum += part[i];
  }
  // 1 / root: one Newton step takes the instruction's to 2^-40 and less (of an infinite mean it is 0, and stays).  Used as (high + low) 2^e, 1 <= high + low < 2:
  // h 2^e is exact and passes the row's root by hidden^(1/2) at most, h 2^e w has 16 bits, and a product is rounded once.  (low is positive: an
  // infinite product stays what it is.)
  const double mean = __builtin_fma(sum, a.per_entry, (double)a.eps), r0 = __builtin_amdgcn_rsq(mean);
  const double inv = r0 > 0. ? __builtin_fma(0.5 * r0, __builtin_fma(-mean * r0, r0, 1.), r0) : r0;
  const int e = inv > 0. ? (int)(__builtin_bit_cast(uint64_t, inv) >> 52) - 1023 : 0;
  const double step = __builtin_ldexp(inv, -e);
  const float power = inv == 0. ? 0.f : __builtin_ldexpf(1.f, e), high = (float)(step * (1. - 0x1p-23)), low = (float)(step - (double)high);
  auto product = [&](float hv, float wv) -> float {
    const float q = hv * power * wv;
    return __builtin_fmaf(q, high, q * low);
  };
#pragma unroll
  for (int j = 0; j < PIECES; ++j) {
    const int p = tid + THREADS * j;
    if (p >= n) break;                             // (in the 8-bit form whole groups of 16 lanes leave together)
    const uint4 wv = *(const uint4*)(a.w + 8 * p);
    const uint32_t hw[4] = {h[j].x, h[j].y, h[j].z, h[j].w}, ww[4] = {wv.x, wv.y, wv.z, wv.w};
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = product(bf_lo(hw[i]), bf_lo(ww[i]));
      y[2 * i + 1] = product(bf_hi(hw[i]), bf_hi(ww[i]));
    }
    if constexpr (!MX) {
      *(uint4*)((bf16_t*)a.out + row + 8 * p) = uint4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, finite_magnitude(y[i]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 1));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2));
      const uint32_t b = scale_byte_e4m3(m);
      const float f = inverse_scale_of(b);
      *(uint2*)((char*)a.out + row + 8 * p) = uint2{e4m3_codes(y[0] * f, y[1] * f, y[2] * f, y[3] * f), e4m3_codes(y[4] * f, y[5] * f, y[6] * f, y[7] * f)};
      uint32_t four = b << (8 * ((tid >> 2) & 3));
      four |= (uint32_t)__shfl_xor((int)four, 4);
      four |= (uint32_t)__shfl_xor((int)four, 8);
      if ((tid & 15) == 0) a.scales[(size_t)(p >> 4) * a.T + t] = four;
    }
  }
}

hipError_t launch_rmsnorm(const void* x, void* residual, const void* weight, float eps, void* out, void* out_scales, int T, int hidden, const StepMark& mark,
                          hipStream_t stream) {
  NormArgs a{(const bf16_t*)x, (bf16_t*)residual, (const bf16_t*)weight, out, (uint32_t*)out_scales, eps, 1. / hidden, T, hidden, 0, mark};
  constexpr int MOST_ROWS = 1 << 21;               // of a launch: a grid has fewer than 2^32 threads
  auto launch = [&](auto mx, auto bf, int threads) {
    for (a.first = 0; a.first < T; a.mark.flag = nullptr) {
      const int rows = std::min(T - a.first, MOST_ROWS);
      hipLaunchKernelGGL(out_scales ? mx : bf, dim3((unsigned)rows), dim3((unsigned)threads), 0, stream, a);
      if (T - a.first <= MOST_ROWS) break;
      a.first += MOST_ROWS;
    }
  };
  const int n = hidden / 8;
  if (n <= 64) launch(rmsnorm_kernel<64, 1, true>, rmsnorm_kernel<64, 1, false>, 64);
  else if (n <= 128) launch(rmsnorm_kernel<64, 2, true>, rmsnorm_kernel<64, 2, false>, 64);
  else if (n <= 256) launch(rmsnorm_kernel<128, 2, true>, rmsnorm_kernel<128, 2, false>, 128);
  else if (n <= 512) launch(rmsnorm_kernel<256, 2, true>, rmsnorm_kernel<256, 2, false>, 256);
  else if (n <= 1024) launch(rmsnorm_kernel<512, 2, true>, rmsnorm_kernel<512, 2, false>, 512);
  else if (n <= 2048) launch(rmsnorm_kernel<1024, 2, true>, rmsnorm_kernel<1024, 2, false>, 1024);
  else launch(rmsnorm_kernel<1024, 4, true>, rmsnorm_kernel<1024, 4, false>, 1024);
  return hipGetLastError();
}

}  // namespace spd
