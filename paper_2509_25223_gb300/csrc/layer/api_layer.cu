// api_layer.cu -- the C ABI of the operators around the recurrence (convolution,
// selective scan, norms; include/rdn.h): argument validation and dispatch to
// the launchers.  No exception or abort crosses this boundary.
#include <math.h>

#include "common.cuh"
#include "entry.cuh"

namespace rdn {
size_t conv_bwd_bytes(const rdn_conv_args &a);
cudaError_t launch_conv(const rdn_conv_args &a, bool bwd, cudaStream_t s);
cudaError_t launch_conv_step(const rdn_conv_step_args &a, cudaStream_t s);
long long scan_slots(const rdn_scan_args &a);
size_t scan_fwd_bytes(const rdn_scan_args &a);
size_t scan_bwd_bytes(const rdn_scan_args &a);
cudaError_t launch_scan_fwd(const rdn_scan_args &a, cudaStream_t s);
cudaError_t launch_scan_bwd(const rdn_scan_args &a, cudaStream_t s);
cudaError_t launch_scan_step(const rdn_scan_step_args &a, cudaStream_t s);
size_t norm_bwd_bytes(const rdn_norm_args &a);
cudaError_t launch_norm(const rdn_norm_args &a, bool bwd, cudaStream_t s);
}  // namespace rdn

using rdn::CallRange;
using rdn::entry_cuda;
using rdn::entry_fail;
using rdn::entry_injected;
using rdn::entry_ok;

namespace {

bool dtype_ok(int d) { return d == RDN_F32 || d == RDN_BF16; }
size_t dtype_size(int d) { return d == RDN_BF16 ? 2 : 4; }

// `size`: the element's bytes, the alignment every data pointer needs
rdn_status_t check_ptr(const char *fn, const char *name, const void *p, size_t size, bool required) {
  if (!p) return required ? entry_fail(RDN_ERR_INVALID_ARG, "%s: %s is NULL", fn, name) : RDN_OK;
  if ((uintptr_t)p & (size - 1))
    return entry_fail(RDN_ERR_MISALIGNED, "%s: %s is not %zu-byte aligned", fn, name, size);
  return RDN_OK;
}
// A state's or a parameter's rows may be read 16 bytes at a time.
rdn_status_t check_ptr16(const char *fn, const char *name, const void *p, bool required) {
  return check_ptr(fn, name, p, 16, required);
}
// A state that is written against one that other CTAs of the call may still read.
rdn_status_t check_apart(const char *fn, const char *name, const void *out, size_t bytes, const char *in_name,
                         const void *in, size_t in_bytes) {
  const uintptr_t o = (uintptr_t)out, i = (uintptr_t)in;
  if (out && in && (o < i ? i - o < bytes : o - i < in_bytes))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, name, in_name);
  return RDN_OK;
}
// A row stride: 0 stands for contiguous.
rdn_status_t check_ld(const char *fn, const char *name, long long *ld, long long row) {
  if (*ld == 0) *ld = row;
  if (*ld < row || *ld > (1ll << 40))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: %s = %lld is shorter than the row (%lld) or too long", fn, name, *ld, row);
  return RDN_OK;
}
rdn_status_t check_seqs(const char *fn, int B, int T, const int *cu, int num_seqs) {
  if (B < 1 || T < 0) return entry_fail(RDN_ERR_INVALID_ARG, "%s: need B >= 1, T >= 0 (got B=%d T=%d)", fn, B, T);
  // (token rows, and units and slots that are at most a few more, in 31 bits)
  if ((long long)B * T > (1ll << 30))
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: B*T = %lld too large", fn, (long long)B * T);
  if (B > (1 << 24)) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: B = %d too large", fn, B);
  if (!cu) return RDN_OK;
  if (B != 1) return entry_fail(RDN_ERR_INVALID_ARG, "%s: cu_seqlens needs B = 1 (got B=%d)", fn, B);
  if (num_seqs < 1 || num_seqs > (1 << 24))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= num_seqs <= 2^24 (got %d)", fn, num_seqs);
  return check_ptr(fn, "cu_seqlens", cu, 4, true);
}
rdn_status_t check_dtype(const char *fn, int dtype) {
  return dtype_ok(dtype) ? RDN_OK : entry_fail(RDN_ERR_UNSUPPORTED, "%s: dtype %d unsupported", fn, dtype);
}
rdn_status_t check_flag(const char *fn, const char *name, int v) {
  return v == 0 || v == 1 ? RDN_OK : entry_fail(RDN_ERR_INVALID_ARG, "%s: %s must be 0 or 1 (got %d)", fn, name, v);
}
rdn_status_t check_ws(const char *fn, const void *ws, size_t got, size_t need) {
  if (!need) return RDN_OK;
  if (!ws || got < need)
    return entry_fail(RDN_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need, ws ? got : (size_t)0);
  if ((uintptr_t)ws & 15) return entry_fail(RDN_ERR_WORKSPACE, "%s: workspace is not 16-byte aligned", fn);
  return RDN_OK;
}

#define TRY(expr)                                    \
  do {                                               \
    const rdn_status_t st_ = (expr);                 \
    if (st_ != RDN_OK) return st_;                   \
  } while (0)

// ---- convolution

rdn_status_t conv_shapes(const char *fn, rdn_conv_args *a) {
  TRY(check_seqs(fn, a->B, a->T, a->cu_seqlens, a->num_seqs));
  if (a->C < 1 || a->C > (1 << 20))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= C <= 2^20 (got %d)", fn, a->C);
  if (a->W < 2 || a->W > 4) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: supported widths are W in {2, 3, 4} (got %d)", fn, a->W);
  TRY(check_dtype(fn, a->dtype));
  TRY(check_flag(fn, "silu", a->silu));
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->C));
  TRY(check_ld(fn, "y_ld", &a->y_ld, a->C));
  TRY(check_ld(fn, "dy_ld", &a->dy_ld, a->C));
  return check_ld(fn, "dx_ld", &a->dx_ld, a->C);
}

rdn_status_t conv_common(const char *fn, const rdn_conv_args *args, bool bwd, cudaStream_t s) {
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_conv_args copy = *args, *a = &copy;
  TRY(conv_shapes(fn, a));
  const size_t e = dtype_size(a->dtype);
  const size_t states = (size_t)(a->cu_seqlens ? a->num_seqs : a->B) * (a->W - 1) * a->C * e;
  const bool any = a->T > 0;
  TRY(check_ptr(fn, "x", a->x, e, any));
  TRY(check_ptr(fn, "w", a->w, 4, true));
  TRY(check_ptr(fn, "bias", a->bias, 4, false));
  TRY(check_ptr(fn, "state0", a->state0, e, false));
  if (!bwd) {
    TRY(check_ptr(fn, "y", a->y, e, any));
    TRY(check_ptr(fn, "stateT", a->stateT, e, false));
    TRY(check_apart(fn, "stateT", a->stateT, states, "state0", a->state0, states));
    if (a->y && a->y == a->x) return entry_fail(RDN_ERR_INVALID_ARG, "%s: y aliases x", fn);
  } else {
    TRY(check_ptr(fn, "dy", a->dy, e, any));
    TRY(check_ptr(fn, "dx", a->dx, e, any));
    TRY(check_ptr(fn, "dw", a->dw, 4, true));
    TRY(check_ptr(fn, "dbias", a->dbias, 4, false));
    TRY(check_ptr(fn, "dstateT", a->dstateT, e, false));
    TRY(check_ptr(fn, "dstate0", a->dstate0, e, false));
    TRY(check_apart(fn, "dstate0", a->dstate0, states, "dstateT", a->dstateT, states));
    TRY(check_apart(fn, "dstate0", a->dstate0, states, "state0", a->state0, states));
    if (a->dx && (a->dx == a->x || a->dx == a->dy))
      return entry_fail(RDN_ERR_INVALID_ARG, "%s: dx aliases x or dy", fn);
    TRY(check_ws(fn, a->workspace, a->workspace_bytes, rdn::conv_bwd_bytes(*a)));
  }
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_conv(*a, bwd, s));
}

// ---- selective scan

rdn_status_t scan_shapes(const char *fn, rdn_scan_args *a) {
  TRY(check_seqs(fn, a->B, a->T, a->cu_seqlens, a->num_seqs));
  if (a->D < 1 || a->D > (1 << 19) || a->G < 1 || a->D % a->G)
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= D <= 2^19 and G dividing D (got D=%d G=%d)", fn, a->D, a->G);
  if (a->G > 4096) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: at most 4096 groups (got %d)", fn, a->G);
  if (a->S < 1) return entry_fail(RDN_ERR_INVALID_ARG, "%s: need S >= 1 (got %d)", fn, a->S);
  if (a->S > 64) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: at most 64 states (got %d)", fn, a->S);
  TRY(check_dtype(fn, a->dtype));
  TRY(check_flag(fn, "dt_softplus", a->dt_softplus));
  const long long gs = (long long)a->G * a->S;
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->D));
  TRY(check_ld(fn, "dt_ld", &a->dt_ld, a->D));
  TRY(check_ld(fn, "z_ld", &a->z_ld, a->D));
  TRY(check_ld(fn, "b_ld", &a->b_ld, gs));
  TRY(check_ld(fn, "c_ld", &a->c_ld, gs));
  TRY(check_ld(fn, "out_ld", &a->out_ld, a->D));
  TRY(check_ld(fn, "dout_ld", &a->dout_ld, a->D));
  TRY(check_ld(fn, "dx_ld", &a->dx_ld, a->D));
  TRY(check_ld(fn, "ddt_ld", &a->ddt_ld, a->D));
  return check_ld(fn, "dz_ld", &a->dz_ld, a->D);
}

rdn_status_t scan_common(const char *fn, const rdn_scan_args *args, bool bwd, cudaStream_t s) {
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_scan_args copy = *args, *a = &copy;
  TRY(scan_shapes(fn, a));
  const size_t e = dtype_size(a->dtype), row = (size_t)a->D * a->S * 4;
  const size_t states = (a->cu_seqlens ? a->num_seqs : a->B) * row;
  const bool any = a->T > 0;
  TRY(check_ptr(fn, "x", a->x, e, any));
  TRY(check_ptr(fn, "dt", a->dt, e, any));
  TRY(check_ptr(fn, "z", a->z, e, false));
  TRY(check_ptr(fn, "Bm", a->Bm, e, any));
  TRY(check_ptr(fn, "Cm", a->Cm, e, any));
  TRY(check_ptr16(fn, "A", a->A, true));
  TRY(check_ptr(fn, "Dskip", a->Dskip, 4, false));
  TRY(check_ptr(fn, "dt_bias", a->dt_bias, 4, false));
  TRY(check_ptr16(fn, "h0", a->h0, false));
  TRY(check_ptr16(fn, "h_chunks", a->h_chunks, false));
  if (!bwd) {
    TRY(check_ptr(fn, "out", a->out, e, any));
    TRY(check_ptr16(fn, "hT", a->hT, false));
    TRY(check_apart(fn, "hT", a->hT, states, "h0", a->h0, states));
    TRY(check_apart(fn, "h_chunks", a->h_chunks, (size_t)rdn::scan_slots(*a) * row, "h0", a->h0, states));
    TRY(check_ws(fn, a->workspace, a->workspace_bytes, rdn::scan_fwd_bytes(*a)));
    TRY(entry_injected(fn));
    return entry_cuda(fn, rdn::launch_scan_fwd(*a, s));
  }
  TRY(check_ptr(fn, "dout", a->dout, e, any));
  TRY(check_ptr16(fn, "dhT", a->dhT, false));
  TRY(check_ptr(fn, "dx", a->dx, e, any));
  TRY(check_ptr(fn, "ddt", a->ddt, e, any));
  TRY(check_ptr(fn, "dz", a->dz, e, any && a->z));
  TRY(check_ptr(fn, "dB", a->dB, e, any));
  TRY(check_ptr(fn, "dC", a->dC, e, any));
  TRY(check_ptr(fn, "dA", a->dA, 4, true));
  TRY(check_ptr(fn, "dD", a->dD, 4, false));
  TRY(check_ptr(fn, "ddt_bias", a->ddt_bias, 4, false));
  TRY(check_ptr16(fn, "dh0", a->dh0, false));
  TRY(check_apart(fn, "dh0", a->dh0, states, "dhT", a->dhT, states));
  TRY(check_ws(fn, a->workspace, a->workspace_bytes, rdn::scan_bwd_bytes(*a)));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_scan_bwd(*a, s));
}

// ---- norms

rdn_status_t norm_shapes(const char *fn, rdn_norm_args *a) {
  if (a->rows < 1 || a->rows > (1ll << 30))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: rows must be in [1, 2^30] (got %lld)", fn, a->rows);
  if (a->D < 1) return entry_fail(RDN_ERR_INVALID_ARG, "%s: need D >= 2 (got %d)", fn, a->D);
  if (a->D < 2 || a->D > 16384)
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: rows of 2 to 16384 elements (got %d)", fn, a->D);
  if (a->heads < 1 || a->rows % a->heads || a->heads > 65535)
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: heads must be in [1, 65535] and divide rows (got %d)", fn, a->heads);
  if (a->heads > 1 && (a->x || a->w_next))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: heads > 1 takes neither x nor w_next", fn);
  TRY(check_dtype(fn, a->dtype));
  if (!a->x) a->x_dtype = a->dtype;
  if (!dtype_ok(a->x_dtype)) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: x_dtype %d unsupported", fn, a->x_dtype);
  TRY(check_flag(fn, "gate", a->gate));
  if (!(a->eps >= 0.f) || isinf(a->eps)) return entry_fail(RDN_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  if (!a->f && (!a->x || !a->w_next))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: without f, x and w_next are required", fn);
  if (a->f && a->x && !a->scale && (isnan(a->scale_const) || isinf(a->scale_const)))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: scale_const must be finite", fn);
  TRY(check_ld(fn, "f_ld", &a->f_ld, a->D));
  TRY(check_ld(fn, "z_ld", &a->z_ld, a->D));
  return check_ld(fn, "x_ld", &a->x_ld, a->D);
}

rdn_status_t norm_common(const char *fn, const rdn_norm_args *args, bool bwd, cudaStream_t s) {
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_norm_args copy = *args, *a = &copy;
  TRY(norm_shapes(fn, a));
  const size_t e = dtype_size(a->dtype), xe = dtype_size(a->x_dtype);
  TRY(check_ptr(fn, "f", a->f, e, false));
  TRY(check_ptr(fn, "z", a->z, e, false));
  TRY(check_ptr(fn, "x", a->x, xe, false));
  TRY(check_ptr(fn, "w", a->w, 4, a->f));
  TRY(check_ptr(fn, "scale", a->scale, 4, false));
  TRY(check_ptr(fn, "w_next", a->w_next, 4, false));
  if (!bwd) {
    // (with x and h both given the caller may do without r itself)
    TRY(check_ptr(fn, "r_out", a->r_out, xe, a->f && !(a->x && a->w_next)));
    TRY(check_ptr(fn, "h", a->h, e, a->w_next));
  } else {
    TRY(check_ptr(fn, "dr", a->dr, xe, !a->w_next));
    TRY(check_ptr(fn, "dh", a->dh, e, a->w_next));
    TRY(check_ptr(fn, "df", a->df, e, a->f));
    TRY(check_ptr(fn, "dz", a->dz, e, a->f && a->z));
    TRY(check_ptr(fn, "dx", a->dx, xe, a->x));
    TRY(check_ptr(fn, "dw", a->dw, 4, a->f));
    TRY(check_ptr(fn, "dscale", a->dscale, 4, a->f && a->x && a->scale));
    TRY(check_ptr(fn, "dw_next", a->dw_next, 4, a->w_next));
    TRY(check_ws(fn, a->workspace, a->workspace_bytes, rdn::norm_bwd_bytes(*a)));
  }
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_norm(*a, bwd, s));
}

rdn_status_t check_step(const char *fn, int N, int num_slots, const int *slots) {
  if (N < 1) return entry_fail(RDN_ERR_INVALID_ARG, "%s: need N >= 1 (got %d)", fn, N);
  if (num_slots < 1 || (!slots && num_slots < N))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: num_slots = %d is too small", fn, num_slots);
  return check_ptr(fn, "slots", slots, 4, false);
}

}  // namespace

extern "C" {

rdn_status_t rdn_conv_fwd(const rdn_conv_args *a, rdn_stream_t stream) {
  return conv_common("rdn_conv_fwd", a, false, (cudaStream_t)stream);
}
rdn_status_t rdn_conv_bwd(const rdn_conv_args *a, rdn_stream_t stream) {
  return conv_common("rdn_conv_bwd", a, true, (cudaStream_t)stream);
}
rdn_status_t rdn_conv_bwd_workspace_size(const rdn_conv_args *args, size_t *bytes) {
  const char *fn = "rdn_conv_bwd_workspace_size";
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_conv_args a = *args;
  TRY(conv_shapes(fn, &a));
  if (!bytes) return entry_fail(RDN_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
  *bytes = rdn::conv_bwd_bytes(a);
  return entry_ok();
}

rdn_status_t rdn_conv_step(const rdn_conv_step_args *args, rdn_stream_t stream) {
  const char *fn = "rdn_conv_step";
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_conv_step_args copy = *args, *a = &copy;
  TRY(check_step(fn, a->N, a->num_slots, a->slots));
  if (a->C < 1 || a->C > (1 << 20))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= C <= 2^20 (got %d)", fn, a->C);
  if (a->W < 2 || a->W > 4) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: supported widths are W in {2, 3, 4} (got %d)", fn, a->W);
  TRY(check_dtype(fn, a->dtype));
  TRY(check_flag(fn, "silu", a->silu));
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->C));
  TRY(check_ld(fn, "y_ld", &a->y_ld, a->C));
  const size_t e = dtype_size(a->dtype);
  TRY(check_ptr(fn, "x", a->x, e, true));
  TRY(check_ptr(fn, "w", a->w, 4, true));
  TRY(check_ptr(fn, "bias", a->bias, 4, false));
  TRY(check_ptr(fn, "state", a->state, e, true));
  TRY(check_ptr(fn, "y", a->y, e, true));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_conv_step(*a, (cudaStream_t)stream));
}

rdn_status_t rdn_scan_fwd(const rdn_scan_args *a, rdn_stream_t stream) {
  return scan_common("rdn_scan_fwd", a, false, (cudaStream_t)stream);
}
rdn_status_t rdn_scan_bwd(const rdn_scan_args *a, rdn_stream_t stream) {
  return scan_common("rdn_scan_bwd", a, true, (cudaStream_t)stream);
}
namespace {
rdn_status_t scan_size(const char *fn, const rdn_scan_args *args, bool bwd, size_t *bytes) {
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_scan_args a = *args;
  TRY(scan_shapes(fn, &a));
  if (!bytes) return entry_fail(RDN_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
  *bytes = bwd ? rdn::scan_bwd_bytes(a) : rdn::scan_fwd_bytes(a);
  return entry_ok();
}
}  // namespace
rdn_status_t rdn_scan_fwd_workspace_size(const rdn_scan_args *a, size_t *bytes) {
  return scan_size("rdn_scan_fwd_workspace_size", a, false, bytes);
}
rdn_status_t rdn_scan_bwd_workspace_size(const rdn_scan_args *a, size_t *bytes) {
  return scan_size("rdn_scan_bwd_workspace_size", a, true, bytes);
}
rdn_status_t rdn_scan_chunk_slots(const rdn_scan_args *args, long long *slots) {
  const char *fn = "rdn_scan_chunk_slots";
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_scan_args a = *args;
  TRY(scan_shapes(fn, &a));
  if (!slots) return entry_fail(RDN_ERR_INVALID_ARG, "%s: slots is NULL", fn);
  *slots = rdn::scan_slots(a);
  return entry_ok();
}

rdn_status_t rdn_scan_step(const rdn_scan_step_args *args, rdn_stream_t stream) {
  const char *fn = "rdn_scan_step";
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_scan_step_args copy = *args, *a = &copy;
  TRY(check_step(fn, a->N, a->num_slots, a->slots));
  if (a->D < 1 || a->D > (1 << 19) || a->G < 1 || a->D % a->G)
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= D <= 2^19 and G dividing D (got D=%d G=%d)", fn, a->D, a->G);
  if (a->G > 4096) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: at most 4096 groups (got %d)", fn, a->G);
  if (a->S < 1) return entry_fail(RDN_ERR_INVALID_ARG, "%s: need S >= 1 (got %d)", fn, a->S);
  if (a->S > 64) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: at most 64 states (got %d)", fn, a->S);
  TRY(check_dtype(fn, a->dtype));
  TRY(check_flag(fn, "dt_softplus", a->dt_softplus));
  const long long gs = (long long)a->G * a->S;
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->D));
  TRY(check_ld(fn, "dt_ld", &a->dt_ld, a->D));
  TRY(check_ld(fn, "z_ld", &a->z_ld, a->D));
  TRY(check_ld(fn, "b_ld", &a->b_ld, gs));
  TRY(check_ld(fn, "c_ld", &a->c_ld, gs));
  TRY(check_ld(fn, "out_ld", &a->out_ld, a->D));
  const size_t e = dtype_size(a->dtype);
  TRY(check_ptr(fn, "x", a->x, e, true));
  TRY(check_ptr(fn, "dt", a->dt, e, true));
  TRY(check_ptr(fn, "z", a->z, e, false));
  TRY(check_ptr(fn, "Bm", a->Bm, e, true));
  TRY(check_ptr(fn, "Cm", a->Cm, e, true));
  TRY(check_ptr16(fn, "A", a->A, true));
  TRY(check_ptr(fn, "Dskip", a->Dskip, 4, false));
  TRY(check_ptr(fn, "dt_bias", a->dt_bias, 4, false));
  TRY(check_ptr16(fn, "h", a->h, true));
  TRY(check_ptr(fn, "out", a->out, e, true));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_scan_step(*a, (cudaStream_t)stream));
}

rdn_status_t rdn_norm_fwd(const rdn_norm_args *a, rdn_stream_t stream) {
  return norm_common("rdn_norm_fwd", a, false, (cudaStream_t)stream);
}
rdn_status_t rdn_norm_bwd(const rdn_norm_args *a, rdn_stream_t stream) {
  return norm_common("rdn_norm_bwd", a, true, (cudaStream_t)stream);
}
rdn_status_t rdn_norm_bwd_workspace_size(const rdn_norm_args *args, size_t *bytes) {
  const char *fn = "rdn_norm_bwd_workspace_size";
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_norm_args a = *args;
  TRY(norm_shapes(fn, &a));
  if (!bytes) return entry_fail(RDN_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
  *bytes = rdn::norm_bwd_bytes(a);
  return entry_ok();
}

}  // extern "C"
