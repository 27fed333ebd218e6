// C ABI of the operators around the attention: argument validation, workspace
// checks and dispatch.  No call allocates, synchronises or throws across the
// boundary.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/hla.h"
#include "common.h"
#include "mixer.h"

namespace hla {
int api_fail(int code, const char* msg);
}

namespace {

int fail(int code, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  return hla::api_fail(code, msg);
}

int done(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(HLA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return hla::api_fail(HLA_OK, "");
}

int esize(int dtype) { return dtype == HLA_BF16 ? 2 : 4; }

int check_type(int dtype, const char* name) {
  if (dtype != HLA_FP32 && dtype != HLA_BF16) return fail(HLA_ERR_INVALID, "%s must be HLA_FP32 or HLA_BF16", name);
  return HLA_OK;
}

int check_flag(int f, const char* name) {
  if (f != 0 && f != 1) return fail(HLA_ERR_INVALID, "%s must be 0 or 1", name);
  return HLA_OK;
}

bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// A tensor whose elements are read one by one (weights, tables): its own alignment.
int check_own(const void* p, unsigned a, const char* name, bool need = true) {
  if (!p) return need ? fail(HLA_ERR_INVALID, "%s is NULL", name) : HLA_OK;
  if (!aligned(p, a)) return fail(HLA_ERR_INVALID, "%s is not %u-byte aligned", name, a);
  return HLA_OK;
}
int check_16(const void* p, const char* name, bool need = true) { return check_own(p, 16, name, need); }

// The strides of dimensions of size one are not used, whatever they are.
void drop_unused(hla::Rows& r, int B, int n) {
  if (B == 1) r.bs = 0;
  if (n == 1) r.ts = 0;
}

int check_stride(long long bs, long long ts, const char* name) {
  if (bs < 0 || ts < 0) return fail(HLA_ERR_INVALID, "%s: strides must be >= 0 (got %lld, %lld)", name, bs, ts);
  return HLA_OK;
}

// Rows read in 16-byte pieces: the base and both strides in whole pieces.
int check_rows(const hla::Rows& r, int dtype, const char* name) {
  int rc;
  if ((rc = check_16(r.p, name)) || (rc = check_stride(r.bs, r.ts, name))) return rc;
  const int v = 16 / esize(dtype);
  if (r.bs % v || r.ts % v)
    return fail(HLA_ERR_INVALID, "%s: strides must be whole 16-byte pieces (got %lld, %lld elements)", name, r.bs, r.ts);
  return HLA_OK;
}

int check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return fail(HLA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, have);
  return check_16(ws, "workspace");
}

// ---------------------------------------------------------------------------
int conv_sizes(int B, int n, int D, int K) {
  if (B < 1 || n < 1 || D < 1) return fail(HLA_ERR_INVALID, "B, n and D must be >= 1 (got B=%d n=%d D=%d)", B, n, D);
  if (K < 2 || K > 4) return fail(HLA_ERR_UNSUPPORTED, "K must be 2, 3 or 4 (got %d)", K);
  if (B > 65535) return fail(HLA_ERR_UNSUPPORTED, "B=%d exceeds 65535", B);
  if (n > 1 << 22) return fail(HLA_ERR_UNSUPPORTED, "n=%d exceeds 2^22", n);
  if ((long long)D * ((n + 3) / 4) >= (1LL << 31))
    return fail(HLA_ERR_UNSUPPORTED, "n=%d of D=%d is too long: D n / 4 must stay below 2^31", n, D);
  return HLA_OK;
}

// The gradients' sums over the tokens: 16 threads a weight or bias, in whole blocks of 64 of these, less than 2^32.
int conv_back_sizes(int D, int K) {
  if ((long long)D * (K + 1) > (1LL << 28) - 64)
    return fail(HLA_ERR_UNSUPPORTED, "D=%d of K=%d is too wide for the gradients: D (K + 1) must stay below 2^28 - 63", D, K);
  return HLA_OK;
}

int conv_check(hla::Conv& c) {
  int rc;
  drop_unused(c.x, c.B, c.n);
  drop_unused(c.dy, c.B, c.n);
  if ((rc = conv_sizes(c.B, c.n, c.D, c.K)) || (rc = check_flag(c.silu, "silu")) ||
      (rc = check_type(c.dtype, "dtype")) || (rc = check_type(c.w_dtype, "w_dtype")))
    return rc;
  const unsigned es = esize(c.dtype), ws = esize(c.w_dtype);
  if ((rc = check_own(c.x.p, es, "x")) || (rc = check_stride(c.x.bs, c.x.ts, "x")) ||
      (rc = check_own(c.w, ws, "weight")) || (rc = check_own(c.bias, ws, "bias", false)))
    return rc;
  return HLA_OK;
}

// ---------------------------------------------------------------------------
int qk_check(hla::QkRope& a) {
  int rc;
  drop_unused(a.q, a.B, a.n);
  drop_unused(a.k, a.B, a.n);
  if (a.B < 1 || a.n < 1 || a.H < 1 || a.Hk < 1)
    return fail(HLA_ERR_INVALID, "B, n, H and Hk must be >= 1 (got B=%d n=%d H=%d Hk=%d)", a.B, a.n, a.H, a.Hk);
  if (a.d < 16 || a.d > 256 || a.d % 8)
    return fail(HLA_ERR_UNSUPPORTED, "d must be a multiple of 8 from 16 to 256 (got %d)", a.d);
  if (a.rot < 0 || a.rot > a.d || a.rot % 2)
    return fail(HLA_ERR_INVALID, "rot must be even, from 0 to d (got %d, d=%d)", a.rot, a.d);
  if (a.positions < 0 || (a.rot && a.positions < 1))
    return fail(HLA_ERR_INVALID, "positions must be >= 1 (got %d)", a.positions);
  if ((rc = check_flag(a.interleaved, "interleaved")) || (rc = check_type(a.dtype, "dtype")) ||
      (rc = check_type(a.w_dtype, "w_dtype")) || (rc = check_flag(a.pos64, "pos64")))
    return rc;
  if (!std::isfinite(a.eps) || a.eps < 0.f) return fail(HLA_ERR_INVALID, "eps must be finite and >= 0");
  // a launch has less than 2^32 threads (the gradients' own has few: they cover what the forward does)
  if (hla::qk_rope_threads(a) >= 4294967296.0)
    return fail(HLA_ERR_UNSUPPORTED, "B=%d n=%d H=%d Hk=%d: too many rows for a launch", a.B, a.n, a.H, a.Hk);
  const unsigned ws = esize(a.w_dtype);
  if ((rc = check_rows(a.q, a.dtype, "q")) || (rc = check_rows(a.k, a.dtype, "k")) ||
      (rc = check_own(a.qw, ws, "q_weight", false)) || (rc = check_own(a.kw, ws, "k_weight", false)) ||
      (rc = check_own(a.cs, 4, "cos", a.rot > 0)) || (rc = check_own(a.sn, 4, "sin", a.rot > 0)) ||
      (rc = check_own(a.pos, a.pos64 ? 8 : 4, "pos", false)))
    return rc;
  if (a.pos_bs < 0) return fail(HLA_ERR_INVALID, "pos_bs must be >= 0 (got %lld)", a.pos_bs);
  return HLA_OK;
}

// ---------------------------------------------------------------------------
// A launch of the scan has the heads in its second dimension, the step a workgroup of 256 threads for each.
constexpr long long kScanHeads = 65535, kStepHeads = (1LL << 24) - 1;

int ssm_sizes(int B, int n, int H, int P, int G, int N, long long most = kScanHeads) {
  if (B < 1 || n < 1 || H < 1 || G < 1)
    return fail(HLA_ERR_INVALID, "B, n, H and G must be >= 1 (got B=%d n=%d H=%d G=%d)", B, n, H, G);
  if (H % G) return fail(HLA_ERR_INVALID, "H=%d must be a multiple of G=%d", H, G);
  if ((long long)B * H > most)
    return fail(HLA_ERR_UNSUPPORTED, "B*H=%lld exceeds %lld", (long long)B * H, most);
  if (!hla::ssm_sizes_ok(P, N))
    return fail(HLA_ERR_UNSUPPORTED, "P and N must be multiples of 16 from 16 to 128 (got P=%d N=%d)", P, N);
  if ((long long)B * H * n >= (1LL << 31) || n > (1LL << 31) - 64)   // tokens are counted in whole blocks of 64
    return fail(HLA_ERR_UNSUPPORTED, "n=%d is too long: B*H*n must stay below 2^31, n at most 2^31 - 64", n);
  return HLA_OK;
}

// What the gradients ask for beyond the scan itself: a launch has less than 2^32 threads.
int ssm_back_sizes(int B, int n, int H, int G, int dtype) {
  if (dtype != HLA_BF16) return fail(HLA_ERR_UNSUPPORTED, "the scan's gradients cover bf16 inputs");
  if (hla::ssm_backward_threads(B, n, H, G) >= 4294967296.0)
    return fail(HLA_ERR_UNSUPPORTED, "n=%d is too long for the gradients of B=%d G=%d", n, B, G);
  return HLA_OK;
}

// Rows of w elements, n of them a sequence.  The kernels' tiles end where the
// next row would begin, so rows must not overlap; the stride of a single row
// is set to one that does not.
int ssm_rows(hla::Rows& r, int B, int n, int w, int dtype, const char* name) {
  drop_unused(r, B, n);
  if (n == 1) r.ts = w;
  const int rc = check_rows(r, dtype, name);
  if (rc) return rc;
  if (r.ts < w)
    return fail(HLA_ERR_INVALID, "%s: a token stride of %lld elements makes rows of %d overlap", name, r.ts, w);
  // a tile's rows are addressed with 32-bit byte offsets
  if (r.ts * 64 * esize(dtype) >= (1LL << 30))
    return fail(HLA_ERR_UNSUPPORTED, "%s: a token stride of %lld elements is too long", name, r.ts);
  return HLA_OK;
}

int ssm_check(hla::Ssm& a, long long most = kScanHeads) {
  int rc;
  if ((rc = ssm_sizes(a.B, a.n, a.H, a.P, a.G, a.N, most)) || (rc = check_flag(a.softplus, "softplus")) ||
      (rc = check_type(a.dtype, "dtype")) || (rc = check_type(a.dt_dtype, "dt_dtype")))
    return rc;
  drop_unused(a.dt, a.B, a.n);
  if ((rc = ssm_rows(a.x, a.B, a.n, a.H * a.P, a.dtype, "x")) ||
      (rc = ssm_rows(a.Bm, a.B, a.n, a.G * a.N, a.dtype, "Bm")) ||
      (rc = ssm_rows(a.Cm, a.B, a.n, a.G * a.N, a.dtype, "Cm")) || (rc = check_own(a.dt.p, esize(a.dt_dtype), "dt")) ||
      (rc = check_stride(a.dt.bs, a.dt.ts, "dt")) || (rc = check_own(a.A, 4, "A")) ||
      (rc = check_own(a.D, 4, "D", false)) || (rc = check_own(a.dt_bias, 4, "dt_bias", false)))
    return rc;
  return HLA_OK;
}

}  // namespace

extern "C" {

int hla_conv_forward(const void* x, long long x_bs, long long x_ts, const void* weight, const void* bias, void* state,
                     void* y, int B, int n, int D, int K, int silu, int dtype, int w_dtype, void* stream) {
  hla::Conv c{};
  c.x = {x, x_bs, x_ts};
  c.w = weight; c.bias = bias; c.state = state; c.y = y;
  c.B = B; c.n = n; c.D = D; c.K = K; c.silu = silu; c.dtype = dtype; c.w_dtype = w_dtype;
  int rc;
  if ((rc = conv_check(c)) != HLA_OK) return rc;
  if ((rc = check_own(y, esize(dtype), "y")) || (rc = check_own(state, esize(dtype), "state", false))) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(hla::launch_conv_forward(c, s), "convolution");
}

size_t hla_conv_backward_workspace_bytes(int B, int n, int D, int K) {
  if (conv_sizes(B, n, D, K) != HLA_OK || conv_back_sizes(D, K) != HLA_OK) return 0;
  return hla::conv_backward_ws(B, n, D, K);
}

int hla_conv_backward(const void* x, long long x_bs, long long x_ts, const void* weight, const void* bias,
                      const void* dy, long long dy_bs, long long dy_ts, void* dx, void* dweight, void* dbias, int B,
                      int n, int D, int K, int silu, int dtype, int w_dtype, void* workspace, size_t workspace_bytes,
                      void* stream) {
  hla::Conv c{};
  c.x = {x, x_bs, x_ts};
  c.dy = {dy, dy_bs, dy_ts};
  c.w = weight; c.bias = bias; c.dx = dx; c.dw = dweight; c.dbias = dbias;
  c.B = B; c.n = n; c.D = D; c.K = K; c.silu = silu; c.dtype = dtype; c.w_dtype = w_dtype;
  int rc;
  if ((rc = conv_check(c)) || (rc = conv_back_sizes(D, K))) return rc;
  const unsigned es = esize(dtype), wes = esize(w_dtype);
  if ((rc = check_own(dy, es, "dy")) || (rc = check_stride(c.dy.bs, c.dy.ts, "dy")) || (rc = check_own(dx, es, "dx")) ||
      (rc = check_own(dweight, wes, "dweight")) || (rc = check_own(dbias, wes, "dbias", false)) ||
      (rc = check_ws(workspace, workspace_bytes, hla::conv_backward_ws(B, n, D, K))))
    return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(hla::launch_conv_backward(c, workspace, s), "convolution's gradients");
}

int hla_qk_norm_rope(const void* q, long long q_bs, long long q_ts, const void* k, long long k_bs, long long k_ts,
                     const void* q_weight, const void* k_weight, const float* cos, const float* sin, const void* pos,
                     long long pos_bs, void* q_out, void* k_out, int B, int n, int H, int Hk, int d, int rot,
                     int positions, int interleaved, float eps, int dtype, int w_dtype, int pos64, void* stream) {
  hla::QkRope a{};
  a.q = {q, q_bs, q_ts};
  a.k = {k, k_bs, k_ts};
  a.qw = q_weight; a.kw = k_weight; a.cs = cos; a.sn = sin; a.pos = pos; a.pos_bs = pos_bs;
  a.qo = q_out; a.ko = k_out;
  a.B = B; a.n = n; a.H = H; a.Hk = Hk; a.d = d; a.rot = rot; a.positions = positions; a.interleaved = interleaved;
  a.eps = eps; a.dtype = dtype; a.w_dtype = w_dtype; a.pos64 = pos64;
  int rc;
  if ((rc = qk_check(a)) || (rc = check_16(q_out, "q_out")) || (rc = check_16(k_out, "k_out"))) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(hla::launch_qk_rope(a, s), "norm and rotation");
}

size_t hla_qk_norm_rope_backward_workspace_bytes(int d) {
  if (d < 16 || d > 256 || d % 8) {
    fail(HLA_ERR_UNSUPPORTED, "d must be a multiple of 8 from 16 to 256 (got %d)", d);
    return 0;
  }
  return hla::qk_rope_backward_ws(d);
}

int hla_qk_norm_rope_backward(const void* q, long long q_bs, long long q_ts, const void* k, long long k_bs,
                              long long k_ts, const void* q_weight, const void* k_weight, const float* cos,
                              const float* sin, const void* pos, long long pos_bs, const void* dq_out,
                              const void* dk_out, void* dq, void* dk, void* dq_weight, void* dk_weight, int B, int n,
                              int H, int Hk, int d, int rot, int positions, int interleaved, float eps, int dtype,
                              int w_dtype, int pos64, void* workspace, size_t workspace_bytes, void* stream) {
  hla::QkRope a{};
  a.q = {q, q_bs, q_ts};
  a.k = {k, k_bs, k_ts};
  a.qw = q_weight; a.kw = k_weight; a.cs = cos; a.sn = sin; a.pos = pos; a.pos_bs = pos_bs;
  a.gq = dq_out; a.gk = dk_out; a.dq = dq; a.dk = dk; a.dqw = dq_weight; a.dkw = dk_weight;
  a.B = B; a.n = n; a.H = H; a.Hk = Hk; a.d = d; a.rot = rot; a.positions = positions; a.interleaved = interleaved;
  a.eps = eps; a.dtype = dtype; a.w_dtype = w_dtype; a.pos64 = pos64;
  int rc;
  const unsigned wes = esize(w_dtype);
  if ((rc = qk_check(a)) || (rc = check_16(dq_out, "dq_out")) || (rc = check_16(dk_out, "dk_out")) ||
      (rc = check_16(dq, "dq")) || (rc = check_16(dk, "dk")) || (rc = check_own(dq_weight, wes, "dq_weight", false)) ||
      (rc = check_own(dk_weight, wes, "dk_weight", false)) ||
      (rc = check_ws(workspace, workspace_bytes, hla::qk_rope_backward_ws(d))))
    return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(hla::launch_qk_rope_backward(a, workspace, s),
              "gradients of norm and rotation");
}

size_t hla_ssm_workspace_bytes(int B, int n, int H, int P, int G, int N, int dtype) {
  if (ssm_sizes(B, n, H, P, G, N) != HLA_OK || check_type(dtype, "dtype") != HLA_OK) return 0;
  return hla::ssm_forward_ws(B, n, H, P, N, dtype);
}

int hla_ssm_forward(const void* x, long long x_bs, long long x_ts, const void* dt, long long dt_bs, long long dt_ts,
                    const float* A, const void* Bm, long long b_bs, long long b_ts, const void* Cm, long long c_bs,
                    long long c_ts, const float* D, const float* dt_bias, float* state, void* y, int B, int n, int H,
                    int P, int G, int N, int softplus, int dtype, int dt_dtype, void* workspace,
                    size_t workspace_bytes, void* stream) {
  hla::Ssm a{};
  a.x = {x, x_bs, x_ts};
  a.dt = {dt, dt_bs, dt_ts};
  a.Bm = {Bm, b_bs, b_ts};
  a.Cm = {Cm, c_bs, c_ts};
  a.A = A; a.D = D; a.dt_bias = dt_bias; a.state = state; a.y = y;
  a.B = B; a.n = n; a.H = H; a.P = P; a.G = G; a.N = N; a.softplus = softplus; a.dtype = dtype; a.dt_dtype = dt_dtype;
  int rc;
  if ((rc = ssm_check(a)) || (rc = check_16(y, "y")) || (rc = check_16(state, "state", false)) ||
      (rc = check_ws(workspace, workspace_bytes, hla::ssm_forward_ws(B, n, H, P, N, dtype))))
    return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(hla::launch_ssm_forward(a, workspace, s), "state space scan");
}

int hla_ssm_step(float* state, const void* x, long long x_bs, const void* dt, long long dt_bs, const float* A,
                 const void* Bm, long long b_bs, const void* Cm, long long c_bs, const float* D, const float* dt_bias,
                 void* y, int B, int H, int P, int G, int N, int softplus, int dtype, int dt_dtype, void* stream) {
  hla::Ssm a{};
  a.x = {x, x_bs, 0};
  a.dt = {dt, dt_bs, 0};
  a.Bm = {Bm, b_bs, 0};
  a.Cm = {Cm, c_bs, 0};
  a.A = A; a.D = D; a.dt_bias = dt_bias; a.state = state; a.y = y;
  a.B = B; a.n = 1; a.H = H; a.P = P; a.G = G; a.N = N; a.softplus = softplus; a.dtype = dtype; a.dt_dtype = dt_dtype;
  int rc;
  if ((rc = ssm_check(a, kStepHeads)) || (rc = check_16(y, "y")) || (rc = check_16(state, "state"))) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return done(hla::launch_ssm_step(a, s), "state space step");
}

size_t hla_ssm_backward_workspace_bytes(int B, int n, int H, int P, int G, int N, int dtype) {
  if (ssm_sizes(B, n, H, P, G, N) != HLA_OK || check_type(dtype, "dtype") != HLA_OK ||
      ssm_back_sizes(B, n, H, G, dtype) != HLA_OK)
    return 0;
  return hla::ssm_backward_ws(B, n, H, P, G, N);
}

int hla_ssm_backward(const void* x, long long x_bs, long long x_ts, const void* dt, long long dt_bs, long long dt_ts,
                     const float* A, const void* Bm, long long b_bs, long long b_ts, const void* Cm, long long c_bs,
                     long long c_ts, const float* D, const float* dt_bias, const void* dy, long long dy_bs,
                     long long dy_ts, void* dx, void* ddt, float* dA, void* dBm, void* dCm, float* dD,
                     float* ddt_bias, int B, int n, int H, int P, int G, int N, int softplus, int dtype, int dt_dtype,
                     void* workspace, size_t workspace_bytes, void* stream) {
  hla::Ssm a{};
  a.x = {x, x_bs, x_ts};
  a.dt = {dt, dt_bs, dt_ts};
  a.Bm = {Bm, b_bs, b_ts};
  a.Cm = {Cm, c_bs, c_ts};
  a.dy = {dy, dy_bs, dy_ts};
  a.A = A; a.D = D; a.dt_bias = dt_bias;
  a.dx = dx; a.ddt = ddt; a.dA = dA; a.dBm = dBm; a.dCm = dCm; a.dD = dD; a.ddt_bias = ddt_bias;
  a.B = B; a.n = n; a.H = H; a.P = P; a.G = G; a.N = N; a.softplus = softplus; a.dtype = dtype; a.dt_dtype = dt_dtype;
  int rc;
  if ((rc = ssm_check(a)) || (rc = ssm_back_sizes(B, n, H, G, dtype))) return rc;
  if ((rc = ssm_rows(a.dy, B, n, H * P, dtype, "dy")) || (rc = check_16(dx, "dx")) ||
      (rc = check_own(ddt, esize(dt_dtype), "ddt")) || (rc = check_own(dA, 4, "dA")) || (rc = check_16(dBm, "dBm")) ||
      (rc = check_16(dCm, "dCm")) || (rc = check_own(dD, 4, "dD", false)) ||
      (rc = check_own(ddt_bias, 4, "ddt_bias", false)) ||
      (rc = check_ws(workspace, workspace_bytes, hla::ssm_backward_ws(B, n, H, P, G, N))))
    return rc;
  return done(hla::launch_ssm_backward(a, workspace, reinterpret_cast<hipStream_t>(stream)),
              "state space scan's gradients");
}

}  // extern "C"
