// The operators around the attention (csrc/mixer_api.cpp is their C ABI): the
// short causal convolution, the norm and rotation of queries and keys, and
// the selective state space scan.  Host-side argument records and launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "profile.h"

namespace hla {

// Row-strided view of a [B, n, ...] tensor: elements between batches and tokens.
struct Rows {
  const void* p;
  long long bs, ts;
};

struct Conv {
  Rows x;                       // [B, n, D]
  const void* w;                // [D, K]
  const void* bias;             // [D] or null
  void* state;                  // [B, K-1, D] of x's type, or null
  void* y;                      // [B, n, D] contiguous
  int B, n, D, K, silu, dtype, w_dtype;
  Rows dy;                      // backward: [B, n, D]
  void* dx;                     // [B, n, D] contiguous
  void* dw;                     // [D, K] of w's type
  void* dbias;                  // [D] of w's type, or null
};
hipError_t launch_conv_forward(const Conv& c, hipStream_t s);
size_t conv_backward_ws(int B, int n, int D, int K);
hipError_t launch_conv_backward(const Conv& c, void* ws, hipStream_t s);

struct QkRope {
  Rows q, k;                    // [B, n, H, d], [B, n, Hk, d], heads contiguous
  const void *qw, *kw;          // [d] or null
  const float *cs, *sn;         // [positions, rot/2]
  const void* pos;              // [B, n] int32 or int64, or null: 0, 1, ...
  long long pos_bs;             // elements between batches of pos (0: one row for all)
  void *qo, *ko;                // [B, H, n, d], [B, Hk, n, d]
  int B, n, H, Hk, d, rot, positions, interleaved, dtype, w_dtype, pos64;
  float eps;
  const void *gq, *gk;          // backward: gradients of qo and ko
  void *dq, *dk;                // [B, n, H, d], [B, n, Hk, d] contiguous
  void *dqw, *dkw;              // [d] of the weights' type, or null
};
hipError_t launch_qk_rope(const QkRope& a, hipStream_t s);
double qk_rope_threads(const QkRope& a);   // of the forward's launch
size_t qk_rope_backward_ws(int d);
hipError_t launch_qk_rope_backward(const QkRope& a, void* ws, hipStream_t s);

struct Ssm {
  Rows x;                       // [B, n, H, P]
  Rows dt;                      // [B, n, H]
  Rows Bm, Cm;                  // [B, n, G, N]
  const float *A, *D, *dt_bias; // [H]; D and dt_bias may be null
  float* state;                 // [B, H, N, P] or null; read and written
  void* y;                      // [B, n, H, P] contiguous
  int B, n, H, P, G, N, softplus, dtype, dt_dtype;
  Rows dy;                      // backward: [B, n, H, P]
  void *dx, *ddt, *dBm, *dCm;   // contiguous, of x's, dt's and x's type
  float *dA, *dD, *ddt_bias;    // [H]; dD and ddt_bias may be null
};
bool ssm_sizes_ok(int P, int N);
size_t ssm_forward_ws(int B, int n, int H, int P, int N, int dtype);
hipError_t launch_ssm_forward(const Ssm& a, void* ws, hipStream_t s);
hipError_t launch_ssm_step(const Ssm& a, hipStream_t s);
double ssm_backward_threads(int B, int n, int H, int G);   // of its largest launch
size_t ssm_backward_ws(int B, int n, int H, int P, int G, int N);
hipError_t launch_ssm_backward(const Ssm& a, void* ws, hipStream_t s);

// One kernel as a bracket of its own; its launch status.
#define HLA_TIMED(name, kernel, grid, block, lds, stream, ...)       \
  HLA_PROF(name, stream, [&]() {                                     \
    HLA_LAUNCH(kernel, grid, block, lds, stream, __VA_ARGS__);       \
    return hipGetLastError();                                        \
  }())
}  // namespace hla
