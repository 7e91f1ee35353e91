// Entry point of the RMS norm.
#include <cmath>
#include <cstdint>

#include "internal.h"

using namespace spd;

extern "C" int spd_rmsnorm(spd_ctx* ctx, int phase, const void* x, void* residual, const void* weight, float eps, void* out,
                           void* out_scales, int32_t n_tokens, int32_t hidden) {
  if (!ctx || (phase != SPD_PHASE_PREFILL && phase != SPD_PHASE_DECODE)) return SPD_EINVAL;
  if (n_tokens < 0 || hidden <= 0 || hidden > NORM_MOST_HIDDEN || hidden % (out_scales ? 128 : 8)) return SPD_EINVAL;
  if (!(eps > 0.f) || !std::isfinite(eps)) return SPD_EINVAL;
  if (n_tokens > 0 && (!x || !weight || !out)) return SPD_EINVAL;
  if ((((uintptr_t)x | (uintptr_t)residual | (uintptr_t)weight | (uintptr_t)out) & 15) || ((uintptr_t)out_scales & 3)) return SPD_EINVAL;
  // a row's workgroup has read it before it writes, but not the others' rows, nor the weights
  const uint64_t n = (uint64_t)n_tokens * hidden, out_bytes = out_scales ? n : 2 * n, scale_bytes = n / 32;
  if (overlap(residual, 2 * n, x, 2 * n) || overlap(residual, 2 * n, weight, 2ull * hidden) || overlap(out, out_bytes, residual, 2 * n) ||
      overlap(out, out_bytes, weight, 2ull * hidden) || (overlap(out, out_bytes, x, 2 * n) && (out != x || out_scales)))
    return SPD_EINVAL;
  if (overlap(out_scales, scale_bytes, x, 2 * n) || overlap(out_scales, scale_bytes, residual, 2 * n) || overlap(out_scales, scale_bytes, out, out_bytes) ||
      overlap(out_scales, scale_bytes, weight, 2ull * hidden))
    return SPD_EINVAL;
  if (ctx->device < 0) return SPD_ESTATE;
  if (n_tokens == 0) return SPD_OK;
  hipStream_t stream;
  int rc = phase_enter(ctx, phase, &stream);
  if (rc != SPD_OK) return rc;
  if ((rc = kernel_timing_mark(ctx, phase, 0, stream)) != SPD_OK) return rc;
  SPD_HIP(launch_rmsnorm(x, residual, weight, eps, out, out_scales, n_tokens, hidden, step_mark(ctx, phase, stream_capturing(ctx, stream)),
                         stream));
  return kernel_timing_mark(ctx, phase, 1, stream);
}
