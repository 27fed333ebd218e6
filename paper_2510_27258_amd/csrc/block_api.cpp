// C ABI of the operators of a block: argument validation, workspace checks and
// dispatch.  No call allocates, synchronises or throws across the boundary.
#include <cmath>

#include "block.h"
#include "checks.h"

namespace {

int check_eps(float eps) {
  if (!std::isfinite(eps) || eps < 0.f) return fail(HLA_ERR_INVALID, "eps must be finite and >= 0");
  return HLA_OK;
}

// Tokens are counted in 31 bits.
int check_tokens(int B, int n) {
  if (B < 1 || n < 1) return fail(HLA_ERR_INVALID, "B and n must be >= 1 (got B=%d n=%d)", B, n);
  if ((long long)B * n >= (1LL << 31)) return fail(HLA_ERR_UNSUPPORTED, "B*n=%lld must stay below 2^31", (long long)B * n);
  return HLA_OK;
}

// The type of a mixer's output or residual stream beside that of the rest: the same, or fp32 beside bf16.
int check_pair(int first, int rest, const char* name) {
  int rc;
  if ((rc = check_type(first, name)) || (rc = check_type(rest, "dtype"))) return rc;
  if (first == HLA_BF16 && rest == HLA_FP32)
    return fail(HLA_ERR_UNSUPPORTED, "%s must be dtype or HLA_FP32: bf16 beside fp32 is not covered", name);
  return HLA_OK;
}

// ---------------------------------------------------------------------------
int gn_sizes(int B, int n, int G, int d, int per_group) {
  int rc;
  if ((rc = check_tokens(B, n)) || (rc = check_flag(per_group, "per_group"))) return rc;
  if (G < 1 || d < 1) return fail(HLA_ERR_INVALID, "G and d must be >= 1 (got G=%d d=%d)", G, d);
  if (d > hla::kNormMax) return fail(HLA_ERR_UNSUPPORTED, "d=%d exceeds %d", d, hla::kNormMax);
  if (G > 65535) return fail(HLA_ERR_UNSUPPORTED, "G=%d exceeds 65535", G);
  return HLA_OK;
}

int check_rows3(hla::Rows3& r, int B, int n, int G, int dtype, const char* name, bool need = true) {
  if (B == 1) r.bs = 0;
  if (n == 1) r.ts = 0;
  if (G == 1) r.gs = 0;
  const int rc = check_own(r.p, esize(dtype), name, need);
  if (rc || !r.p) return rc;
  if (r.bs < 0 || r.ts < 0 || r.gs < 0)
    return fail(HLA_ERR_INVALID, "%s: strides must be >= 0 (got %lld, %lld, %lld)", name, r.bs, r.ts, r.gs);
  return HLA_OK;
}

int gn_check(hla::GatedNorm& a) {
  int rc;
  if ((rc = gn_sizes(a.B, a.n, a.G, a.d, a.per_group)) || (rc = check_flag(a.norm_first, "norm_first")) ||
      (rc = check_eps(a.eps)) || (rc = check_pair(a.y_dtype, a.dtype, "y_dtype")) || (rc = check_type(a.w_dtype, "w_dtype")) ||
      (rc = check_rows3(a.y, a.B, a.n, a.G, a.y_dtype, "y")) || (rc = check_rows3(a.z, a.B, a.n, a.G, a.dtype, "z", false)) ||
      (rc = check_own(a.w, esize(a.w_dtype), "weight", false)))
    return rc;
  return HLA_OK;
}

// ---------------------------------------------------------------------------
int rn_sizes(int B, int n, int D) {
  const int rc = check_tokens(B, n);
  if (rc) return rc;
  if (D < 1) return fail(HLA_ERR_INVALID, "D must be >= 1 (got D=%d)", D);
  if (D > hla::kNormMax) return fail(HLA_ERR_UNSUPPORTED, "D=%d exceeds %d", D, hla::kNormMax);
  return HLA_OK;
}

int rn_check(hla::ResidualNorm& a) {
  int rc;
  drop_unused(a.x, a.B, a.n);
  drop_unused(a.y, a.B, a.n);
  if ((rc = rn_sizes(a.B, a.n, a.D)) || (rc = check_eps(a.eps)) || (rc = check_pair(a.x_dtype, a.dtype, "x_dtype")) ||
      (rc = check_type(a.w_dtype, "w_dtype")))
    return rc;
  if (!std::isfinite(a.alpha)) return fail(HLA_ERR_INVALID, "alpha must be finite");
  const unsigned ws = esize(a.w_dtype);
  if ((rc = check_own(a.x.p, esize(a.x_dtype), "x")) || (rc = check_stride(a.x.bs, a.x.ts, "x")) ||
      (rc = check_own(a.y.p, esize(a.dtype), "y")) || (rc = check_stride(a.y.bs, a.y.ts, "y")) ||
      (rc = check_own(a.w, ws, "weight", false)) || (rc = check_own(a.post, ws, "post_weight", false)) ||
      (rc = check_own(a.scale, ws, "scale", false)))
    return rc;
  return HLA_OK;
}

// ---------------------------------------------------------------------------
// Outputs and inputs of a wave's tokens, 128 at most, are addressed with 31-bit byte offsets.
constexpr int kGlrWide = 1 << 21;

int glr_sizes(int B, int n, int D) {
  const int rc = check_tokens(B, n);
  if (rc) return rc;
  if (D < 1) return fail(HLA_ERR_INVALID, "D must be >= 1 (got D=%d)", D);
  if (D > kGlrWide) return fail(HLA_ERR_UNSUPPORTED, "D=%d exceeds 2^21", D);
  if (hla::glr_threads(B, n, D) >= 4294967296.0)
    return fail(HLA_ERR_UNSUPPORTED, "B=%d D=%d: too many channels for a launch", B, D);
  return HLA_OK;
}

int glr_check(hla::Glr& p) {
  int rc;
  if ((rc = glr_sizes(p.B, p.n, p.D)) || (rc = check_type(p.dtype, "dtype"))) return rc;
  if (!std::isfinite(p.c) || p.c < 0.f) return fail(HLA_ERR_INVALID, "c must be finite and >= 0");
  const unsigned es = esize(p.dtype);
  hla::Rows* rows[] = {&p.x, &p.f, &p.g};
  const char* names[] = {"x", "f", "g"};
  for (int i = 0; i < 3; ++i) {
    drop_unused(*rows[i], p.B, p.n);
    if ((rc = check_own(rows[i]->p, es, names[i])) || (rc = check_stride(rows[i]->bs, rows[i]->ts, names[i]))) return rc;
    if (rows[i]->ts > kGlrWide)
      return fail(HLA_ERR_UNSUPPORTED, "%s: a token stride of %lld elements is too long", names[i], rows[i]->ts);
  }
  if ((rc = check_own(p.decay, 4, "decay")) || (rc = check_own(p.fb, 4, "f_bias", false)) ||
      (rc = check_own(p.gb, 4, "g_bias", false)))
    return rc;
  return HLA_OK;
}

// ---------------------------------------------------------------------------
// Whether tiles of 512 threads over rows x cols exceed a launch.
bool glu_over(double rows, double tall, double cols, double wide, double times = 1.) {
  return times * std::ceil(rows / tall) * std::ceil(cols / wide) * 512 >= 4294967296.0;
}

int glu_sizes(int B, int n, int D, int F) {
  const int rc = check_tokens(B, n);
  if (rc) return rc;
  if (D < 1 || F < 1) return fail(HLA_ERR_INVALID, "D and F must be >= 1 (got D=%d F=%d)", D, F);
  if (D % 8 || F % 8) return fail(HLA_ERR_UNSUPPORTED, "D and F must be multiples of 8 (got D=%d F=%d)", D, F);
  if (D > 1 << 20 || F > 1 << 20) return fail(HLA_ERR_UNSUPPORTED, "D and F must be at most 2^20 (got D=%d F=%d)", D, F);
  // A launch has less than 2^32 threads: 512 a tile of 128 tokens and 64 outputs, or 256 x 256 of a gradient.
  const double M = (double)B * n;
  if (glu_over(M, 128, F, 64) || glu_over(M, 256, D, 256) || glu_over(D, 256, 2. * F, 256) || M + 256 >= 2147483648.0)
    return fail(HLA_ERR_UNSUPPORTED, "B=%d n=%d D=%d F=%d: too many tiles for a launch", B, n, D, F);
  return HLA_OK;
}

int glu_check(hla::Glu& p, int act, int dtype) {
  int rc;
  if ((rc = glu_sizes(p.B, p.n, p.D, p.F))) return rc;
  if (act != HLA_ACT_SILU && act != HLA_ACT_GELU)
    return fail(HLA_ERR_INVALID, "act must be HLA_ACT_SILU or HLA_ACT_GELU");
  if ((rc = check_type(dtype, "dtype"))) return rc;
  if (dtype != HLA_BF16) return fail(HLA_ERR_UNSUPPORTED, "the gated projections cover bf16");
  drop_unused(p.x, p.B, p.n);
  if ((rc = check_rows(p.x, dtype, "x")) || (rc = check_16(p.wg, "w_gate")) || (rc = check_16(p.wu, "w_up"))) return rc;
  // a tile's 256 rows are addressed with 31-bit byte offsets (of single tokens the stride between sequences)
  const long long far = p.n == 1 ? p.x.bs : p.x.ts;
  if (far > (1LL << 22) - 8192) return fail(HLA_ERR_UNSUPPORTED, "x: a token stride of %lld elements is too long", far);
  // a tile lies in one sequence, unless they lie one behind the other
  auto apart = [&](const hla::Rows& r) { return r.p && r.bs != p.n * r.ts; };
  if (p.B > 1 && p.n > 1 && (apart(p.x) || apart(p.dh)) && glu_over(p.n, 128, p.F, 64, p.B))
    return fail(HLA_ERR_UNSUPPORTED, "B=%d n=%d F=%d: too many tiles for a launch of sequences laid apart", p.B, p.n, p.F);
  p.gelu = act == HLA_ACT_GELU;
  return HLA_OK;
}

hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int hla_gated_norm(const void* y, long long y_bs, long long y_ts, long long y_gs, const void* z, long long z_bs,
                   long long z_ts, long long z_gs, const void* weight, void* out, int B, int n, int G, int d,
                   int per_group, int norm_first, float eps, int y_dtype, int dtype, int w_dtype, void* stream) {
  hla::GatedNorm a{};
  a.y = {y, y_bs, y_ts, y_gs};
  a.z = {z, z_bs, z_ts, z_gs};
  a.w = weight; a.out = out;
  a.B = B; a.n = n; a.G = G; a.d = d; a.per_group = per_group; a.norm_first = norm_first; a.eps = eps;
  a.y_dtype = y_dtype; a.dtype = dtype; a.w_dtype = w_dtype;
  int rc;
  if ((rc = gn_check(a)) || (rc = check_own(out, esize(dtype), "out"))) return rc;
  return done(hla::launch_gated_norm(a, stream_of(stream)), "gated norm");
}

size_t hla_gated_norm_backward_workspace_bytes(int B, int n, int G, int d, int per_group) {
  return gn_sizes(B, n, G, d, per_group) == HLA_OK ? hla::gated_norm_backward_ws(B, n, G, d, per_group) : 0;
}

int hla_gated_norm_backward(const void* y, long long y_bs, long long y_ts, long long y_gs, const void* z, long long z_bs,
                            long long z_ts, long long z_gs, const void* weight, const void* dout, void* dy,
                            long long dy_bs, long long dy_ts, long long dy_gs, void* dz, void* dweight, int B, int n,
                            int G, int d, int per_group, int norm_first, float eps, int y_dtype, int dtype, int w_dtype,
                            void* workspace, size_t workspace_bytes, void* stream) {
  hla::GatedNorm a{};
  a.y = {y, y_bs, y_ts, y_gs};
  a.z = {z, z_bs, z_ts, z_gs};
  a.dy = {dy, dy_bs, dy_ts, dy_gs};
  a.w = weight; a.dout = dout; a.dz = dz; a.dw = dweight;
  a.B = B; a.n = n; a.G = G; a.d = d; a.per_group = per_group; a.norm_first = norm_first; a.eps = eps;
  a.y_dtype = y_dtype; a.dtype = dtype; a.w_dtype = w_dtype;
  int rc;
  if ((rc = gn_check(a)) || (rc = check_own(dout, esize(dtype), "dout")) ||
      (rc = check_rows3(a.dy, B, n, G, y_dtype, "dy")) || (rc = check_own(dz, esize(dtype), "dz", z != nullptr)) ||
      (rc = check_own(dweight, esize(w_dtype), "dweight", false)))
    return rc;
  // rows of dy are written: they must not overlap
  if ((G > 1 && a.dy.gs < d) || (n > 1 && a.dy.ts < d) || (B > 1 && a.dy.bs < d))
    return fail(HLA_ERR_INVALID, "dy: strides of %lld, %lld, %lld elements make rows of %d overlap", a.dy.bs, a.dy.ts,
                a.dy.gs, d);
  if ((rc = check_ws(workspace, workspace_bytes, hla::gated_norm_backward_ws(B, n, G, d, per_group)))) return rc;
  return done(hla::launch_gated_norm_backward(a, workspace, stream_of(stream)), "gradients of the gated norm");
}

int hla_residual_norm(const void* x, long long x_bs, long long x_ts, const void* y, long long y_bs, long long y_ts,
                      const void* weight, const void* post_weight, const void* scale, void* out, void* r, int B, int n,
                      int D, float alpha, float eps, int x_dtype, int dtype, int w_dtype, void* stream) {
  hla::ResidualNorm a{};
  a.x = {x, x_bs, x_ts};
  a.y = {y, y_bs, y_ts};
  a.w = weight; a.post = post_weight; a.scale = scale; a.out = out; a.r = r;
  a.B = B; a.n = n; a.D = D; a.alpha = alpha; a.eps = eps; a.x_dtype = x_dtype; a.dtype = dtype; a.w_dtype = w_dtype;
  int rc;
  if ((rc = rn_check(a)) || (rc = check_own(out, esize(dtype), "out")) || (rc = check_own(r, esize(x_dtype), "r"))) return rc;
  return done(hla::launch_residual_norm(a, stream_of(stream)), "residual norm");
}

size_t hla_residual_norm_backward_workspace_bytes(int B, int n, int D) {
  return rn_sizes(B, n, D) == HLA_OK ? hla::residual_norm_backward_ws(B, n, D) : 0;
}

int hla_residual_norm_backward(const void* x, long long x_bs, long long x_ts, const void* y, long long y_bs,
                               long long y_ts, const void* weight, const void* post_weight, const void* scale,
                               const void* dout, const void* dr, void* dx, void* dy, void* dweight, void* dpost_weight,
                               void* dscale, int B, int n, int D, float alpha, float eps, int x_dtype, int dtype,
                               int w_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  hla::ResidualNorm a{};
  a.x = {x, x_bs, x_ts};
  a.y = {y, y_bs, y_ts};
  a.w = weight; a.post = post_weight; a.scale = scale; a.dout = dout; a.dr = dr; a.dx = dx; a.dy = dy;
  a.dw = dweight; a.dpost = dpost_weight; a.dscale = dscale;
  a.B = B; a.n = n; a.D = D; a.alpha = alpha; a.eps = eps; a.x_dtype = x_dtype; a.dtype = dtype; a.w_dtype = w_dtype;
  int rc;
  const unsigned xs = esize(x_dtype), es = esize(dtype), wes = esize(w_dtype);
  if ((rc = rn_check(a)) || (rc = check_own(dout, es, "dout", dr == nullptr)) || (rc = check_own(dr, xs, "dr", false)) ||
      (rc = check_own(dx, xs, "dx")) || (rc = check_own(dy, es, "dy")) || (rc = check_own(dweight, wes, "dweight", false)) ||
      (rc = check_own(dpost_weight, wes, "dpost_weight", false)) || (rc = check_own(dscale, wes, "dscale", false)))
    return rc;
  if (dpost_weight && !post_weight) return fail(HLA_ERR_INVALID, "dpost_weight without a post_weight");
  if ((rc = check_ws(workspace, workspace_bytes, hla::residual_norm_backward_ws(B, n, D)))) return rc;
  return done(hla::launch_residual_norm_backward(a, workspace, stream_of(stream)), "gradients of the residual norm");
}

size_t hla_glr_workspace_bytes(int B, int n, int D) {
  return glr_sizes(B, n, D) == HLA_OK ? hla::glr_forward_ws(B, n, D) : 0;
}

size_t hla_glr_kept_bytes(int B, int n, int D) {
  if (glr_sizes(B, n, D) != HLA_OK) return 0;
  return sizeof(float) * (size_t)B * D * (((size_t)n + hla::kGlrTile - 1) / hla::kGlrTile);
}

int hla_glr_forward(const void* x, long long x_bs, long long x_ts, const void* f, long long f_bs, long long f_ts,
                    const void* g, long long g_bs, long long g_ts, const float* decay, const float* f_bias,
                    const float* g_bias, float* state, void* y, float* kept, int B, int n, int D, float c, int dtype,
                    void* workspace, size_t workspace_bytes, void* stream) {
  hla::Glr p{};
  p.x = {x, x_bs, x_ts};
  p.f = {f, f_bs, f_ts};
  p.g = {g, g_bs, g_ts};
  p.decay = decay; p.fb = f_bias; p.gb = g_bias; p.state = state; p.y = y; p.kept = kept;
  p.B = B; p.n = n; p.D = D; p.c = c; p.dtype = dtype;
  int rc;
  if ((rc = glr_check(p)) || (rc = check_own(y, esize(dtype), "y")) || (rc = check_own(state, 4, "state", false)) ||
      (rc = check_own(kept, 4, "kept", false)) || (rc = check_ws(workspace, workspace_bytes, hla::glr_forward_ws(B, n, D))))
    return rc;
  return done(hla::launch_glr_forward(p, workspace, stream_of(stream)), "gated linear recurrence");
}

int hla_glr_step(float* state, const void* x, long long x_bs, const void* f, long long f_bs, const void* g,
                 long long g_bs, const float* decay, const float* f_bias, const float* g_bias, void* y, int B, int D,
                 float c, int dtype, void* stream) {
  hla::Glr p{};
  p.x = {x, x_bs, 0};
  p.f = {f, f_bs, 0};
  p.g = {g, g_bs, 0};
  p.decay = decay; p.fb = f_bias; p.gb = g_bias; p.state = state; p.y = y;
  p.B = B; p.n = 1; p.D = D; p.c = c; p.dtype = dtype;
  int rc;
  if ((rc = glr_check(p)) || (rc = check_own(y, esize(dtype), "y")) || (rc = check_own(state, 4, "state"))) return rc;
  return done(hla::launch_glr_step(p, stream_of(stream)), "step of the gated linear recurrence");
}

size_t hla_glr_backward_workspace_bytes(int B, int n, int D) {
  return glr_sizes(B, n, D) == HLA_OK ? hla::glr_backward_ws(B, n, D) : 0;
}

int hla_glr_backward(const void* x, long long x_bs, long long x_ts, const void* f, long long f_bs, long long f_ts,
                     const void* g, long long g_bs, long long g_ts, const float* decay, const float* f_bias,
                     const float* g_bias, const float* kept, const void* dy, long long dy_bs, long long dy_ts, void* dx,
                     void* df, void* dg, float* ddecay, float* df_bias, float* dg_bias, int B, int n, int D, float c,
                     int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  hla::Glr p{};
  p.x = {x, x_bs, x_ts};
  p.f = {f, f_bs, f_ts};
  p.g = {g, g_bs, g_ts};
  p.dy = {dy, dy_bs, dy_ts};
  p.decay = decay; p.fb = f_bias; p.gb = g_bias; p.kept = const_cast<float*>(kept);
  p.dx = dx; p.df = df; p.dg = dg; p.ddecay = ddecay; p.dfb = df_bias; p.dgb = dg_bias;
  p.B = B; p.n = n; p.D = D; p.c = c; p.dtype = dtype;
  int rc;
  if ((rc = glr_check(p))) return rc;
  drop_unused(p.dy, B, n);
  const unsigned es = esize(dtype);
  if ((rc = check_own(kept, 4, "kept")) || (rc = check_own(dy, es, "dy")) || (rc = check_stride(p.dy.bs, p.dy.ts, "dy")) ||
      (rc = p.dy.ts > kGlrWide ? fail(HLA_ERR_UNSUPPORTED, "dy: a token stride of %lld elements is too long", p.dy.ts) : HLA_OK) ||
      (rc = check_own(dx, es, "dx")) || (rc = check_own(df, es, "df")) || (rc = check_own(dg, es, "dg")) ||
      (rc = check_own(ddecay, 4, "ddecay")) || (rc = check_own(df_bias, 4, "df_bias", false)) ||
      (rc = check_own(dg_bias, 4, "dg_bias", false)) ||
      (rc = check_ws(workspace, workspace_bytes, hla::glr_backward_ws(B, n, D))))
    return rc;
  return done(hla::launch_glr_backward(p, workspace, stream_of(stream)), "gradients of the gated linear recurrence");
}

int hla_glu_forward(const void* x, long long x_bs, long long x_ts, const void* w_gate, const void* w_up, void* h, int B,
                    int n, int D, int F, int act, int dtype, void* stream) {
  hla::Glu p{};
  p.x = {x, x_bs, x_ts};
  p.wg = w_gate; p.wu = w_up; p.h = h;
  p.B = B; p.n = n; p.D = D; p.F = F;
  int rc;
  if ((rc = glu_check(p, act, dtype)) || (rc = check_16(h, "h"))) return rc;
  return done(hla::launch_glu(p, stream_of(stream)), "gated projections");
}

size_t hla_glu_backward_workspace_bytes(int B, int n, int D, int F) {
  return glu_sizes(B, n, D, F) == HLA_OK ? hla::glu_backward_ws(B, n, D, F) : 0;
}

int hla_glu_backward(const void* x, long long x_bs, long long x_ts, const void* w_gate, const void* w_up, const void* dh,
                     long long dh_bs, long long dh_ts, void* dx, void* dw_gate, void* dw_up, int B, int n, int D, int F,
                     int act, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  hla::Glu p{};
  p.x = {x, x_bs, x_ts};
  p.dh = {dh, dh_bs, dh_ts};
  p.wg = w_gate; p.wu = w_up; p.dx = dx; p.dwg = dw_gate; p.dwu = dw_up;
  p.B = B; p.n = n; p.D = D; p.F = F;
  int rc;
  if ((rc = glu_check(p, act, dtype))) return rc;
  drop_unused(p.dh, B, n);
  if ((rc = check_rows(p.dh, dtype, "dh")) || (rc = check_16(dx, "dx")) || (rc = check_16(dw_gate, "dw_gate")) ||
      (rc = check_16(dw_up, "dw_up")) || (rc = check_ws(workspace, workspace_bytes, hla::glu_backward_ws(B, n, D, F))))
    return rc;
  return done(hla::launch_glu_backward(p, workspace, stream_of(stream)), "gradients of the gated projections");
}

}  // extern "C"
