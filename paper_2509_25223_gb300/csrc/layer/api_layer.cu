// api_layer.cu -- the C ABI of the operators around the recurrence (convolution,
// selective scan, norms, gated recurrence, matrix products; include/rdn.h): argument
// validation and dispatch to the launchers.  No exception or abort crosses this boundary.
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
long long gscan_slots(const rdn_gscan_args &a);
long long gscan_ctas(const rdn_gscan_args &a);
size_t gscan_bwd_bytes(const rdn_gscan_args &a);
cudaError_t launch_gscan_fwd(const rdn_gscan_args &a, cudaStream_t s);
cudaError_t launch_gscan_bwd(const rdn_gscan_args &a, cudaStream_t s);
cudaError_t launch_gscan_step(const rdn_gscan_step_args &a, cudaStream_t s);
cudaError_t launch_norm_q8(const rdn_norm_q8_args &a, cudaStream_t s);
size_t linear_bwd_bytes(const rdn_linear_args &a, bool dbias);
cudaError_t launch_linear_fwd(const rdn_linear_args &a, cudaStream_t s);
cudaError_t launch_linear_bwd(const rdn_linear_args &a, cudaStream_t s);
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
// Rows of an operand, in bytes: `rows` of them, `width` each, `ld` from one to the next.
struct Bytes {
  const char *name;
  const void *p;
  long long rows, ld, width;
  bool dense() const { return rows == 1 || ld == width; }
  long long size() const {  // (no tensor is as long as 2^60: products of the largest rows and distances pass 63 bits)
    return rows > 1 && ld > (1ll << 60) / rows ? 1ll << 60 : (rows - 1) * ld + width;
  }
};
// Whether two operands share a byte.  Slices of the columns of one wider tensor do not, though each lies between
// the other's rows.  (Rows of two distances, both with gaps: by the ranges from their first to their last byte.)
bool share(const Bytes &a, const Bytes &b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
  const long long d = (long long)((uintptr_t)b.p - (uintptr_t)a.p);  // from a's first byte to b's
  if (d >= a.size() || -d >= b.size()) return false;
  if (a.dense() && b.dense()) return true;
  if (b.dense()) return share(b, a);
  if (a.dense()) {  // the last row of b that starts before a's end
    long long k = (a.size() - 1 - d) / b.ld;
    if (k > b.rows - 1) k = b.rows - 1;
    return d + k * b.ld + b.width > 0;
  }
  if (a.ld != b.ld) return true;
  // b's row j starts `at` behind a's row j + k
  const long long k = d >= 0 ? d / a.ld : -((-d + a.ld - 1) / a.ld), at = d - k * a.ld;
  return (at < a.width && k < a.rows && k > -b.rows) || (at + b.width > a.ld && k + 1 < a.rows && k + 1 > -b.rows);
}
// A result against what other CTAs of the call may still read, or write.
template <size_t N>
rdn_status_t check_alone(const char *fn, const Bytes &out, const Bytes (&others)[N]) {
  for (const Bytes &o : others)
    if (share(out, o)) return entry_fail(RDN_ERR_INVALID_ARG, "%s: %s aliases %s", fn, out.name, o.name);
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

// ---- gated linear recurrence

rdn_status_t gscan_shapes(const char *fn, rdn_gscan_args *a) {
  TRY(check_seqs(fn, a->B, a->T, a->cu_seqlens, a->num_seqs));
  if (a->D < 1 || a->D > (1 << 19))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= D <= 2^19 (got %d)", fn, a->D);
  TRY(check_dtype(fn, a->dtype));
  if (!(a->c > 0.f) || isinf(a->c)) return entry_fail(RDN_ERR_INVALID_ARG, "%s: c must be finite and > 0", fn);
  if (rdn::gscan_ctas(*a) > 0x7fffffffll)
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: B = %d rows of D = %d channels are too many", fn, a->B, a->D);
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->D));
  TRY(check_ld(fn, "r_ld", &a->r_ld, a->D));
  TRY(check_ld(fn, "i_ld", &a->i_ld, a->D));
  TRY(check_ld(fn, "y_ld", &a->y_ld, a->D));
  TRY(check_ld(fn, "dy_ld", &a->dy_ld, a->D));
  TRY(check_ld(fn, "dx_ld", &a->dx_ld, a->D));
  TRY(check_ld(fn, "dr_ld", &a->dr_ld, a->D));
  TRY(check_ld(fn, "di_ld", &a->di_ld, a->D));
  const long long lds[7] = {a->x_ld, a->r_ld, a->i_ld, a->y_ld, a->dy_ld, a->dx_ld, a->dr_ld};
  bool far = a->di_ld >= (1 << 24);
  for (long long ld : lds) far = far || ld >= (1 << 24);
  return far ? entry_fail(RDN_ERR_UNSUPPORTED, "%s: rows 2^24 elements and more apart", fn) : RDN_OK;
}

rdn_status_t gscan_common(const char *fn, const rdn_gscan_args *args, bool bwd, cudaStream_t s) {
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_gscan_args copy = *args, *a = &copy;
  TRY(gscan_shapes(fn, a));
  const size_t e = dtype_size(a->dtype), row = (size_t)a->D * 4;
  const size_t states = (a->cu_seqlens ? a->num_seqs : a->B) * row, kept = (size_t)rdn::gscan_slots(*a) * row;
  const bool any = a->T > 0;
  TRY(check_ptr(fn, "x", a->x, e, any));
  TRY(check_ptr(fn, "r", a->r, e, any));
  TRY(check_ptr(fn, "i", a->i, e, any));
  TRY(check_ptr(fn, "lam", a->lam, 4, true));
  TRY(check_ptr(fn, "h0", a->h0, 4, false));
  TRY(check_ptr(fn, "h_chunks", a->h_chunks, 4, false));
  if (!bwd) {
    TRY(check_ptr(fn, "y", a->y, e, any));
    TRY(check_ptr(fn, "hT", a->hT, 4, false));
    TRY(check_apart(fn, "hT", a->hT, states, "h0", a->h0, states));
    TRY(check_apart(fn, "h_chunks", a->h_chunks, kept, "h0", a->h0, states));
    TRY(check_apart(fn, "h_chunks", a->h_chunks, kept, "hT", a->hT, states));
    if (a->y && (a->y == a->x || a->y == a->r || a->y == a->i))
      return entry_fail(RDN_ERR_INVALID_ARG, "%s: y aliases an input", fn);
    TRY(entry_injected(fn));
    return entry_cuda(fn, rdn::launch_gscan_fwd(*a, s));
  }
  TRY(check_ptr(fn, "dy", a->dy, e, any));
  TRY(check_ptr(fn, "dhT", a->dhT, 4, false));
  TRY(check_ptr(fn, "dlam", a->dlam, 4, true));
  TRY(check_ptr(fn, "dh0", a->dh0, 4, false));
  const void *outs[3] = {a->dx, a->dr, a->di}, *ins[4] = {a->x, a->r, a->i, a->dy};
  const char *names[3] = {"dx", "dr", "di"};
  for (int k = 0; k < 3; ++k) {
    TRY(check_ptr(fn, names[k], outs[k], e, any));
    for (const void *in : ins)
      if (any && outs[k] == in) return entry_fail(RDN_ERR_INVALID_ARG, "%s: %s aliases an input", fn, names[k]);
    for (int q = 0; q < k; ++q)
      if (any && outs[k] == outs[q])
        return entry_fail(RDN_ERR_INVALID_ARG, "%s: %s aliases %s", fn, names[k], names[q]);
  }
  TRY(check_apart(fn, "dh0", a->dh0, states, "dhT", a->dhT, states));
  TRY(check_apart(fn, "dh0", a->dh0, states, "h0", a->h0, states));
  TRY(check_apart(fn, "dh0", a->dh0, states, "h_chunks", a->h_chunks, kept));
  TRY(check_ws(fn, a->workspace, a->workspace_bytes, rdn::gscan_bwd_bytes(*a)));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_gscan_bwd(*a, s));
}

// ---- matrix products

rdn_status_t check_on16(const char *fn, const char *name, const void *p, long long ld, size_t e, bool required) {
  TRY(check_ptr16(fn, name, p, required));
  if (p && (ld * e) & 15)
    return entry_fail(RDN_ERR_MISALIGNED, "%s: rows of %s (%lld elements apart) do not start on 16 bytes", fn, name, ld);
  return RDN_OK;
}

rdn_status_t linear_shapes(const char *fn, rdn_linear_args *a, bool bwd) {
  if (a->M < 0 || a->N < 1 || a->K < 1)
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need M >= 0, N, K >= 1 (got M=%lld N=%d K=%d)", fn, a->M, a->N, a->K);
  if (a->dtype != RDN_BF16 && (bwd || a->dtype != RDN_E4M3))
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: dtype %d unsupported (bf16%s)", fn, a->dtype, bwd ? "" : " or e4m3");
  const int by = a->dtype == RDN_E4M3 ? 16 : 8;
  if (a->K % by || a->N % 8)
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: K must be a multiple of %d and N of 8 (got N=%d K=%d)", fn, by, a->N, a->K);
  const long long wide = a->N > a->K ? a->N : a->K;
  if (a->M > (1ll << 30) || wide > (1 << 20) || a->M * wide > (1ll << 40))
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: M=%lld N=%d K=%d are too large", fn, a->M, a->N, a->K);
  if (!dtype_ok(a->y_dtype) || !dtype_ok(a->bias_dtype) || !dtype_ok(a->dw_dtype))
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: y_dtype, bias_dtype and dw_dtype are bf16 or fp32", fn);
  if (a->act < 0 || a->act > 3) return entry_fail(RDN_ERR_INVALID_ARG, "%s: act must be 0 to 3 (got %d)", fn, a->act);
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->K));
  TRY(check_ld(fn, "w_ld", &a->w_ld, a->K));
  TRY(check_ld(fn, "res_ld", &a->res_ld, a->N));
  TRY(check_ld(fn, "y_ld", &a->y_ld, a->N));
  // (the tensor maps hold strides below 2^40 bytes)
  if (a->x_ld >= (1ll << 38) || a->w_ld >= (1ll << 38) || a->dy_ld >= (1ll << 38))
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: rows of x, w or dy are too far apart", fn);
  return check_ld(fn, "dy_ld", &a->dy_ld, a->N);
}

rdn_status_t linear_common(const char *fn, const rdn_linear_args *args, bool bwd, cudaStream_t s) {
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_linear_args copy = *args, *a = &copy;
  TRY(linear_shapes(fn, a, bwd));
  const bool any = a->M > 0, q8 = a->dtype == RDN_E4M3;
  const size_t e = q8 ? 1 : 2, ye = dtype_size(a->y_dtype), be = dtype_size(a->bias_dtype);
  TRY(check_on16(fn, "x", a->x, a->x_ld, e, any));
  TRY(check_on16(fn, "w", a->w, a->w_ld, e, true));
  if (!bwd) {
    TRY(check_ptr(fn, "x_scale", a->x_scale, 4, q8 && any));
    TRY(check_ptr(fn, "w_scale", a->w_scale, 4, q8));
    if (!q8 && (a->x_scale || a->w_scale))
      return entry_fail(RDN_ERR_INVALID_ARG, "%s: scales go with e4m3 operands", fn);
    TRY(check_ptr(fn, "bias", a->bias, be, false));
    TRY(check_ptr(fn, "res", a->res, ye, false));
    TRY(check_ptr(fn, "y", a->y, ye, any));
    TRY(check_ptr16(fn, "pre", a->pre, false));
    const Bytes x{"x", a->x, a->M, a->x_ld * (long long)e, a->K * (long long)e};
    const Bytes w{"w", a->w, a->N, a->w_ld * (long long)e, a->K * (long long)e};
    const Bytes xs{"x_scale", a->x_scale, 1, 0, a->M * 4}, ws{"w_scale", a->w_scale, 1, 0, a->N * 4ll};
    const Bytes bias{"bias", a->bias, 1, 0, a->N * (long long)be};
    const Bytes res{"res", a->res, a->M, a->res_ld * (long long)ye, a->N * (long long)ye};
    const Bytes y{"y", a->y, a->M, a->y_ld * (long long)ye, a->N * (long long)ye};
    TRY(check_alone(fn, y, {x, w, xs, ws, bias}));
    if (any && !(a->y == a->res && a->y_ld == a->res_ld) && share(y, res))
      return entry_fail(RDN_ERR_INVALID_ARG, "%s: y may be res only with the same rows", fn);
    TRY(check_alone(fn, {"pre", a->pre, a->M, a->N * 2ll, a->N * 2ll}, {x, w, xs, ws, bias, res, y}));
    TRY(entry_injected(fn));
    return entry_cuda(fn, rdn::launch_linear_fwd(*a, s));
  }
  TRY(check_on16(fn, "dy", a->dy, a->dy_ld, 2, any));
  TRY(check_ptr16(fn, "pre", a->pre, any && a->act));
  TRY(check_ptr16(fn, "dx", a->dx, false));
  TRY(check_ptr(fn, "dw", a->dw, dtype_size(a->dw_dtype), false));
  TRY(check_ptr(fn, "dbias", a->dbias, be, false));
  TRY(check_ws(fn, a->workspace, a->workspace_bytes, rdn::linear_bwd_bytes(*a, a->dbias != nullptr)));
  const Bytes x{"x", a->x, a->M, a->x_ld * 2, a->K * 2ll}, w{"w", a->w, a->N, a->w_ld * 2, a->K * 2ll};
  const Bytes dy{"dy", a->dy, a->M, a->dy_ld * 2, a->N * 2ll};
  const Bytes pre{"pre", a->act ? a->pre : nullptr, a->M, a->N * 2ll, a->N * 2ll};
  const long long wide = a->K * (long long)dtype_size(a->dw_dtype);
  const Bytes dx{"dx", a->dx, a->M, a->K * 2ll, a->K * 2ll}, dw{"dw", a->dw, a->N, wide, wide};
  TRY(check_alone(fn, dx, {x, w, dy, pre}));
  TRY(check_alone(fn, dw, {x, w, dy, pre, dx}));
  TRY(check_alone(fn, {"dbias", a->dbias, 1, 0, a->N * (long long)be}, {x, w, dy, pre, dx, dw}));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_linear_bwd(*a, s));
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

rdn_status_t rdn_gscan_fwd(const rdn_gscan_args *a, rdn_stream_t stream) {
  return gscan_common("rdn_gscan_fwd", a, false, (cudaStream_t)stream);
}
rdn_status_t rdn_gscan_bwd(const rdn_gscan_args *a, rdn_stream_t stream) {
  return gscan_common("rdn_gscan_bwd", a, true, (cudaStream_t)stream);
}
rdn_status_t rdn_gscan_bwd_workspace_size(const rdn_gscan_args *args, size_t *bytes) {
  const char *fn = "rdn_gscan_bwd_workspace_size";
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_gscan_args a = *args;
  TRY(gscan_shapes(fn, &a));
  if (!bytes) return entry_fail(RDN_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
  *bytes = rdn::gscan_bwd_bytes(a);
  return entry_ok();
}

rdn_status_t rdn_gscan_step(const rdn_gscan_step_args *args, rdn_stream_t stream) {
  const char *fn = "rdn_gscan_step";
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_gscan_step_args copy = *args, *a = &copy;
  TRY(check_step(fn, a->N, a->num_slots, a->slots));
  if (a->D < 1 || a->D > (1 << 19))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: need 1 <= D <= 2^19 (got %d)", fn, a->D);
  TRY(check_dtype(fn, a->dtype));
  if (!(a->c > 0.f) || isinf(a->c)) return entry_fail(RDN_ERR_INVALID_ARG, "%s: c must be finite and > 0", fn);
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->D));
  TRY(check_ld(fn, "r_ld", &a->r_ld, a->D));
  TRY(check_ld(fn, "i_ld", &a->i_ld, a->D));
  TRY(check_ld(fn, "y_ld", &a->y_ld, a->D));
  const size_t e = dtype_size(a->dtype);
  TRY(check_ptr(fn, "x", a->x, e, true));
  TRY(check_ptr(fn, "r", a->r, e, true));
  TRY(check_ptr(fn, "i", a->i, e, true));
  TRY(check_ptr(fn, "lam", a->lam, 4, true));
  TRY(check_ptr(fn, "h", a->h, 4, true));
  TRY(check_ptr(fn, "y", a->y, e, true));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_gscan_step(*a, (cudaStream_t)stream));
}

rdn_status_t rdn_norm_q8(const rdn_norm_q8_args *args, rdn_stream_t stream) {
  const char *fn = "rdn_norm_q8";
  CallRange range(fn);
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_norm_q8_args copy = *args, *a = &copy;
  if (a->rows < 0 || a->rows > (1ll << 30))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: rows must be in [0, 2^30] (got %lld)", fn, a->rows);
  if (a->D < 1) return entry_fail(RDN_ERR_INVALID_ARG, "%s: need D >= 1 (got %d)", fn, a->D);
  if (a->D > 16384) return entry_fail(RDN_ERR_UNSUPPORTED, "%s: rows of at most 16384 elements (got %d)", fn, a->D);
  if (!dtype_ok(a->x_dtype) || (a->f && !dtype_ok(a->f_dtype)))
    return entry_fail(RDN_ERR_UNSUPPORTED, "%s: x_dtype %d or f_dtype %d unsupported", fn, a->x_dtype, a->f_dtype);
  if (!(a->eps >= 0.f) || isinf(a->eps)) return entry_fail(RDN_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  TRY(check_ld(fn, "x_ld", &a->x_ld, a->D));
  TRY(check_ld(fn, "f_ld", &a->f_ld, a->D));
  const bool any = a->rows > 0;
  const size_t xe = dtype_size(a->x_dtype);
  TRY(check_ptr(fn, "x", a->x, xe, any));
  TRY(check_ptr(fn, "f", a->f, a->f ? dtype_size(a->f_dtype) : 1, false));
  TRY(check_ptr(fn, "w", a->w, 4, false));
  TRY(check_ptr(fn, "r_out", a->r_out, xe, false));
  TRY(check_ptr(fn, "q", a->q, 1, any));
  TRY(check_ptr(fn, "scale", a->scale, 4, any));
  const long long fe = a->f ? (long long)dtype_size(a->f_dtype) : 1, wide = a->D * (long long)xe;
  const Bytes x{"x", a->x, a->rows, a->x_ld * (long long)xe, wide}, f{"f", a->f, a->rows, a->f_ld * fe, a->D * fe};
  const Bytes w{"w", a->w, 1, 0, a->D * 4ll}, r{"r_out", a->r_out, a->rows, wide, wide};
  if (share(r, f) || (share(r, x) && !(a->r_out == a->x && a->x_ld == a->D)))
    return entry_fail(RDN_ERR_INVALID_ARG, "%s: r_out may be x only where x is contiguous, and not f", fn);
  TRY(check_alone(fn, {"q", a->q, a->rows, a->D, a->D}, {x, f, w, r}));
  TRY(entry_injected(fn));
  return entry_cuda(fn, rdn::launch_norm_q8(*a, (cudaStream_t)stream));
}

rdn_status_t rdn_linear_fwd(const rdn_linear_args *a, rdn_stream_t stream) {
  return linear_common("rdn_linear_fwd", a, false, (cudaStream_t)stream);
}
rdn_status_t rdn_linear_bwd(const rdn_linear_args *a, rdn_stream_t stream) {
  return linear_common("rdn_linear_bwd", a, true, (cudaStream_t)stream);
}
rdn_status_t rdn_linear_bwd_workspace_size(const rdn_linear_args *args, size_t *bytes) {
  const char *fn = "rdn_linear_bwd_workspace_size";
  if (!args) return entry_fail(RDN_ERR_INVALID_ARG, "%s: args is NULL", fn);
  rdn_linear_args a = *args;
  TRY(linear_shapes(fn, &a, true));
  if (!bytes) return entry_fail(RDN_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
  *bytes = rdn::linear_bwd_bytes(a, true);
  return entry_ok();
}

}  // extern "C"
