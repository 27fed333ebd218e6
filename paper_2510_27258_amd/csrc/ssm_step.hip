// Decode step of the selective state space scan, one token a head, the state
// updated in place:
//   dt = softplus(raw + bias),  h <- exp(dt A) h + dt B x^T,  y = h^T C + D x
//
// Bound by the state's bytes: each fp32 element is read once and written once.
// A workgroup takes a head; a thread holds 16-byte pieces of every RG-th row
// of [N][P], all of them loading before the token's vectors are needed, and
// the rows' sums meet in LDS in a fixed order.  The stores are non-temporal
// (the state is not read again within the step).
// Measured: 64 sequences of 32 heads of 128 x 128 (269 MB) 45 us, 6.0 TB/s,
// more than a copy of 1 GiB reaches (5.1): the last-level cache may hold part.
#include "common.h"
#include "mixer.h"
#include "vec.h"

namespace hla {
namespace {

constexpr int kSsmStepThreads = 256;
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int CNT>
__global__ __launch_bounds__(kSsmStepThreads) void k_ssm_step(Ssm a, int P4, int RG) {
  const int bh = blockIdx.x, b = bh / a.H, head = bh - b * a.H, grp = head / (a.H / a.G), tid = threadIdx.x;
  const int rg = tid / P4, c4 = tid - rg * P4;
  const bool mine = rg < RG;
  f32x4* st = reinterpret_cast<f32x4*>(a.state + (size_t)bh * a.N * a.P) + c4;
  f32x4 h[CNT];
#pragma unroll
  for (int k = 0; k < CNT; ++k) {
    const int n = rg + RG * k;
    if (mine && n < a.N) h[k] = st[(size_t)n * P4];
  }
  __shared__ float Bs[128], Cs[128], xs[128];
  __shared__ f32x4 red[kSsmStepThreads];
  if (tid < 128) {
    if (tid < a.N) {
      Bs[tid] = load_any(a.Bm.p, a.dtype, (size_t)(b * a.Bm.bs + (long long)grp * a.N + tid));
      Cs[tid] = load_any(a.Cm.p, a.dtype, (size_t)(b * a.Cm.bs + (long long)grp * a.N + tid));
    }
  } else if (tid - 128 < a.P) {
    xs[tid - 128] = load_any(a.x.p, a.dtype, (size_t)(b * a.x.bs + (long long)head * a.P + tid - 128));
  }
  float dt = load_any(a.dt.p, a.dt_dtype, (size_t)(b * a.dt.bs + head));
  if (a.dt_bias) dt += a.dt_bias[head];
  if (a.softplus) dt = dt > 20.f ? dt : log1pf(expf(dt));
  const float decay = expf(dt * a.A[head]);
  lds_barrier();
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (mine) {
    const f32x4 u = f32x4{xs[4 * c4], xs[4 * c4 + 1], xs[4 * c4 + 2], xs[4 * c4 + 3]} * dt;
#pragma unroll
    for (int k = 0; k < CNT; ++k) {
      const int n = rg + RG * k;
      if (n < a.N) {
        const f32x4 v = h[k] * decay + u * Bs[n];
        __builtin_nontemporal_store(v, st + (size_t)n * P4);
        acc += v * Cs[n];
      }
    }
  }
  red[tid] = acc;
  lds_barrier();
  if (tid < a.P) {
    const float* f = reinterpret_cast<const float*>(red);
    float y = 0.f;
    for (int k = 0; k < RG; ++k) y += f[k * a.P + tid];
    if (a.D) y += a.D[head] * xs[tid];
    store_any(a.y, a.dtype, (size_t)bh * a.P + tid, y);
  }
}

}  // namespace

hipError_t launch_ssm_step(const Ssm& a, hipStream_t s) {
  const int P4 = a.P / 4, RG = kSsmStepThreads / P4 < a.N ? kSsmStepThreads / P4 : a.N, cnt = (a.N + RG - 1) / RG;
  const dim3 grid(a.B * a.H), block(kSsmStepThreads);
  if (cnt <= 2) return HLA_TIMED("ssm_step", k_ssm_step<2>, grid, block, 0, s, a, P4, RG);
  if (cnt <= 4) return HLA_TIMED("ssm_step", k_ssm_step<4>, grid, block, 0, s, a, P4, RG);
  if (cnt <= 8) return HLA_TIMED("ssm_step", k_ssm_step<8>, grid, block, 0, s, a, P4, RG);
  return HLA_TIMED("ssm_step", k_ssm_step<16>, grid, block, 0, s, a, P4, RG);
}

}  // namespace hla
