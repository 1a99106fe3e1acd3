// C ABI entry points of the feed-forward operators (declared and documented in
// include/cattn.h): argument validation on the host, then dispatch to the
// kernel launchers on the caller's stream.
#include <math.h>

#include "../../include/cattn.h"
#include "api_util.h"
#include "ffn_launch.h"

using namespace cattn;

namespace {

bool valid_dtype(int dtype) { return dtype == CATTN_F32 || dtype == CATTN_BF16; }
size_t size_of(int dtype) { return dtype == CATTN_BF16 ? 2 : 4; }

// Of a shape without a 0.
bool gated_supported(int T, int C, int F) {
  return C % 8 == 0 && F % 8 == 0 && C <= kFfnMaxW && F <= kFfnMaxW && (int64_t)T * C <= kFfnMaxElements &&
         (int64_t)T * F <= kFfnMaxElements && (int64_t)F * C <= kFfnMaxElements;
}

cattn_status check_gated(int T, int C, int F, int activation, int dtype) {
  g_last_error[0] = '\0';
  if (T < 0 || C < 0 || F < 0) return fail(CATTN_ERR_INVALID_ARG, "negative T, C or F");
  if (!valid_dtype(dtype)) return fail(CATTN_ERR_INVALID_ARG, "dtype must be CATTN_F32 or CATTN_BF16");
  if (activation != CATTN_SILU && activation != CATTN_GELU)
    return fail(CATTN_ERR_INVALID_ARG, "activation must be CATTN_SILU or CATTN_GELU");
  if (T == 0 || C == 0 || F == 0 || gated_supported(T, C, F)) return CATTN_OK;
  return fail(CATTN_ERR_UNSUPPORTED, "C and F must be multiples of 8 and at most 2^18, T * C, T * F and F * C at most 2^33");
}

cattn_status check_tensors(const void* const* p, int n) {
  for (int i = 0; i < n; ++i) {
    if (!p[i]) return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
    if (!aligned16(p[i])) return fail(CATTN_ERR_INVALID_ARG, "tensors and the workspace must be 16-byte aligned");
  }
  return CATTN_OK;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------
// Gated projections
// ---------------------------------------------------------------------------
cattn_status cattn_gated_fwd(const void* x, const void* w_gate, const void* w_up, void* h, void* gate, void* up, int T,
                             int C, int F, int activation, int dtype, void* stream) {
  const cattn_status st = check_gated(T, C, F, activation, dtype);
  if (st != CATTN_OK || T == 0 || C == 0 || F == 0) return st;
  if (!gate != !up) return fail(CATTN_ERR_INVALID_ARG, "gate and up are stored both or neither");
  const void* tensors[6] = {x, w_gate, w_up, h, gate, up};
  if (const cattn_status e = check_tensors(tensors, gate ? 6 : 4)) return e;
  const size_t e = size_of(dtype), xn = (size_t)T * C * e, wn = (size_t)F * C * e, hn = (size_t)T * F * e;
  const Range ins[3] = {range_of(x, xn), range_of(w_gate, wn), range_of(w_up, wn)};
  const Range outs[3] = {range_of(h, hn), range_of(gate, gate ? hn : 0), range_of(up, up ? hn : 0)};
  if (any_overlap(ins, 3, outs, 3)) return fail(CATTN_ERR_INVALID_ARG, "outputs overlap inputs or each other");
  const GatedFwd a{x, w_gate, w_up, h, gate, up, T, C, F, activation == CATTN_GELU, dtype == CATTN_BF16};
  (void)hipGetLastError();
  return hip_status(launch_gated_fwd(a, (hipStream_t)stream));
}

size_t cattn_gated_bwd_workspace_bytes(int T, int C, int F, int dtype) {
  if (T <= 0 || C <= 0 || F <= 0 || !valid_dtype(dtype) || !gated_supported(T, C, F)) return 0;
  return gated_bwd_bytes(T, C, F, dtype == CATTN_BF16);
}

cattn_status cattn_gated_bwd(const void* x, const void* w_gate, const void* w_up, const void* gate, const void* up,
                             const void* dh, void* dx, void* dw_gate, void* dw_up, void* workspace, int T, int C, int F,
                             int activation, int dtype, void* stream) {
  const cattn_status st = check_gated(T, C, F, activation, dtype);
  if (st != CATTN_OK || T == 0 || C == 0 || F == 0) return st;
  const void* tensors[10] = {x, w_gate, w_up, gate, up, dh, dx, dw_gate, dw_up, workspace};
  if (const cattn_status e = check_tensors(tensors, 10)) return e;
  const size_t e = size_of(dtype), xn = (size_t)T * C * e, wn = (size_t)F * C * e, hn = (size_t)T * F * e;
  const Range ins[6] = {range_of(x, xn),    range_of(w_gate, wn), range_of(w_up, wn),
                        range_of(gate, hn), range_of(up, hn),     range_of(dh, hn)};
  const Range outs[4] = {range_of(dx, xn), range_of(dw_gate, wn), range_of(dw_up, wn),
                         range_of(workspace, cattn_gated_bwd_workspace_bytes(T, C, F, dtype))};
  if (any_overlap(ins, 6, outs, 4)) return fail(CATTN_ERR_INVALID_ARG, "outputs overlap inputs or each other");
  const GatedBwd a{x,  w_gate,  w_up,  gate,      up, dh, dx, dw_gate, dw_up, workspace, T, C, F, activation == CATTN_GELU,
                   dtype == CATTN_BF16};
  (void)hipGetLastError();
  return hip_status(launch_gated_bwd(a, (hipStream_t)stream));
}

// ---------------------------------------------------------------------------
// Dropout
// ---------------------------------------------------------------------------
static cattn_status dropout(const void* x, const void* residual, void* y, long long n, double p, unsigned long long seed,
                            unsigned site, unsigned long long step, const long long* step_at, int dtype, void* stream) {
  g_last_error[0] = '\0';
  if (n < 0) return fail(CATTN_ERR_INVALID_ARG, "negative n");
  if (!valid_dtype(dtype)) return fail(CATTN_ERR_INVALID_ARG, "dtype must be CATTN_F32 or CATTN_BF16");
  if (!(p >= 0.0) || !(p <= 1.0 - 0x1p-32)) return fail(CATTN_ERR_INVALID_ARG, "p must be in [0, 1 - 2^-32]");
  if (n == 0) return CATTN_OK;
  if (n > kFfnMaxElements) return fail(CATTN_ERR_UNSUPPORTED, "n exceeds 2^33");
  if (!x || !y) return fail(CATTN_ERR_INVALID_ARG, "NULL tensor pointer");
  if (!aligned16(x) || !aligned16(residual) || !aligned16(y))
    return fail(CATTN_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if ((uintptr_t)step_at & 7) return fail(CATTN_ERR_INVALID_ARG, "step_at must be 8-byte aligned");
  const size_t bytes = (size_t)n * size_of(dtype);
  const Range out = range_of(y, bytes);
  if ((y != x && overlap(out, range_of(x, bytes))) || (residual && y != residual && overlap(out, range_of(residual, bytes))))
    return fail(CATTN_ERR_INVALID_ARG, "y overlaps an input and is not the same tensor");
  if (step_at && overlap(out, range_of(step_at, 8))) return fail(CATTN_ERR_INVALID_ARG, "y overlaps step_at");
  const Dropout a{x, residual, y, step_at, seed, step, n, site, (unsigned)nearbyint(p * 0x1p32), (float)(1.0 / (1.0 - p)),
                  dtype == CATTN_BF16};
  (void)hipGetLastError();
  return hip_status(launch_dropout(a, (hipStream_t)stream));
}

cattn_status cattn_dropout_fwd(const void* x, const void* residual, void* y, long long n, double p,
                               unsigned long long seed, unsigned site, unsigned long long step, const long long* step_at,
                               int dtype, void* stream) {
  return dropout(x, residual, y, n, p, seed, site, step, step_at, dtype, stream);
}

cattn_status cattn_dropout_bwd(const void* dy, void* dx, long long n, double p, unsigned long long seed, unsigned site,
                               unsigned long long step, const long long* step_at, int dtype, void* stream) {
  return dropout(dy, nullptr, dx, n, p, seed, site, step, step_at, dtype, stream);
}

}  // extern "C"
