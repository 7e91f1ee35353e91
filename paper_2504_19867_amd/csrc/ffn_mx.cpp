// Entry points of the gated FFN's first step over MXFP4 weights and MX E4M3 rows.
#include <cstdint>

#include "internal.h"

using namespace spd;

static int shape_check(int32_t hidden, int32_t inter) {
  // tiles of 128 outputs x 128 hidden entries
  if (hidden <= 0 || inter <= 0 || hidden % 128 || inter % 128) return SPD_EINVAL;
  if ((int64_t)hidden * 255 > INT32_MAX) return SPD_EINVAL;   // per-lane row offsets are 32-bit
  return SPD_OK;
}
static uint64_t packed_bytes(int32_t hidden, int32_t inter) { return (uint64_t)(inter / 128) * (uint64_t)(hidden / 128) * FFN_MX_TILE_BYTES; }
static bool phase_ok(int phase) { return phase == SPD_PHASE_PREFILL || phase == SPD_PHASE_DECODE; }

extern "C" int spd_ffn_mx_bytes(int32_t hidden, int32_t inter, uint64_t* bytes_out) {
  if (shape_check(hidden, inter) != SPD_OK || !bytes_out) return SPD_EINVAL;
  *bytes_out = packed_bytes(hidden, inter);
  return SPD_OK;
}

static int repack(spd_ctx* ctx, int phase, const void* w_gate, const void* w_up, const void* w_mx, int32_t hidden, int32_t inter, bool pack) {
  if (!ctx || !phase_ok(phase)) return SPD_EINVAL;
  int rc = shape_check(hidden, inter);
  if (rc != SPD_OK) return rc;
  if (!w_gate || !w_up || !w_mx || (((uintptr_t)w_gate | (uintptr_t)w_up | (uintptr_t)w_mx) & 15)) return SPD_EINVAL;
  const uint64_t bf16_bytes = 2ull * hidden * inter, mx_bytes = packed_bytes(hidden, inter);
  if (overlap(w_mx, mx_bytes, w_gate, bf16_bytes) || overlap(w_mx, mx_bytes, w_up, bf16_bytes) || (!pack && overlap(w_gate, bf16_bytes, w_up, bf16_bytes)))
    return SPD_EINVAL;
  if (ctx->device < 0) return SPD_ESTATE;
  hipStream_t stream;
  if ((rc = phase_enter(ctx, phase, &stream)) != SPD_OK) return rc;
  const StepMark mark = step_mark(ctx, phase, stream_capturing(ctx, stream));
  if (pack) SPD_HIP(launch_ffn_pack_mx(w_gate, w_up, (void*)w_mx, hidden, inter, mark, stream));
  else SPD_HIP(launch_ffn_unpack_mx(w_mx, (void*)w_gate, (void*)w_up, hidden, inter, mark, stream));
  return SPD_OK;
}

extern "C" int spd_ffn_pack_gate_up_mx(spd_ctx* ctx, int phase, const void* w_gate, const void* w_up, void* w_mx, int32_t hidden, int32_t inter) {
  return repack(ctx, phase, w_gate, w_up, w_mx, hidden, inter, true);
}

extern "C" int spd_ffn_unpack_gate_up_mx(spd_ctx* ctx, int phase, const void* w_mx, void* w_gate, void* w_up, int32_t hidden, int32_t inter) {
  return repack(ctx, phase, w_gate, w_up, w_mx, hidden, inter, false);
}

extern "C" int spd_ffn_gate_up_mx(spd_ctx* ctx, int phase, const void* x, const void* x_scales, const void* w_mx, void* out, int32_t n_tokens,
                                  int32_t hidden, int32_t inter) {
  if (!ctx || !phase_ok(phase)) return SPD_EINVAL;
  int rc = shape_check(hidden, inter);
  if (rc != SPD_OK) return rc;
  if (n_tokens < 0) return SPD_EINVAL;
  if (n_tokens > 0 && (!x || !x_scales || !w_mx || !out || (((uintptr_t)x | (uintptr_t)w_mx) & 15) || ((uintptr_t)x_scales & 3) || ((uintptr_t)out & 1)))
    return SPD_EINVAL;
  const uint64_t n = (uint64_t)n_tokens * hidden, out_bytes = 2ull * n_tokens * inter;
  if (overlap(out, out_bytes, x, n) || overlap(out, out_bytes, x_scales, n / 32) || overlap(out, out_bytes, w_mx, packed_bytes(hidden, inter)))
    return SPD_EINVAL;
  if (ctx->device < 0) return SPD_ESTATE;
  if (n_tokens == 0) return SPD_OK;
  int share;
  const bool exclusive = phase_exclusive(ctx, phase, &share);
  hipStream_t stream;
  if ((rc = phase_enter(ctx, phase, &stream)) != SPD_OK) return rc;
  if ((rc = kernel_timing_mark(ctx, phase, 0, stream)) != SPD_OK) return rc;
  SPD_HIP(launch_ffn_gate_up_mx(x, x_scales, w_mx, out, n_tokens, hidden, inter, ctx->xcds, share, exclusive,
                                step_mark(ctx, phase, stream_capturing(ctx, stream)), stream));
  return kernel_timing_mark(ctx, phase, 1, stream);
}
