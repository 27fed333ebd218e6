// The operators of a block around its mixer (csrc/block_api.cpp is their C
// ABI): the norm of a mixer's output with its gate, the residual addition
// with the norms on both sides of it, the gated linear recurrence, and the
// gated feed-forward projections.  Host-side argument records and launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mixer.h"

namespace hla {

// View of a [B, n, G, d] tensor: elements between batches, tokens and groups.
struct Rows3 {
  const void* p;
  long long bs, ts, gs;
};

struct GatedNorm {
  Rows3 y, z;                   // [B, n, G, d] of y_dtype and dtype; z.p may be null
  const void* w;                // [d] or (per_group) [G, d], or null
  void* out;                    // [B, n, G, d] contiguous, of dtype
  int B, n, G, d, per_group, norm_first, y_dtype, dtype, w_dtype;
  float eps;
  const void* dout;             // backward: contiguous, of dtype
  Rows3 dy;                     // of y_dtype
  void *dz, *dw;                // dz contiguous or null, dw like w or null
};
hipError_t launch_gated_norm(const GatedNorm& a, hipStream_t s);
size_t gated_norm_backward_ws(int B, int n, int G, int d, int per_group);
hipError_t launch_gated_norm_backward(const GatedNorm& a, void* ws, hipStream_t s);

struct ResidualNorm {
  Rows x, y;                    // [B, n, D] of x_dtype and dtype
  const void *w, *post, *scale; // [D] of w_dtype, each may be null
  void *out, *r;                // [B, n, D] contiguous, of dtype and x_dtype
  int B, n, D, x_dtype, dtype, w_dtype;
  float alpha, eps;
  const void *dout, *dr;        // backward: contiguous, of dtype and x_dtype; each may be null
  void *dx, *dy;                // contiguous, of x_dtype and dtype
  void *dw, *dpost, *dscale;    // [D] of w_dtype, each may be null
};
hipError_t launch_residual_norm(const ResidualNorm& a, hipStream_t s);
size_t residual_norm_backward_ws(int B, int n, int D);
hipError_t launch_residual_norm_backward(const ResidualNorm& a, void* ws, hipStream_t s);

// part [rows][cols] per sum, summed over the rows in a fixed order: up to three sums a call
// (a null `to` is left out); sum k's part starts at part + k * rows * cols.
struct ColumnSums {
  const float* part;
  void* to[3];
  int rows, cols, dtype;
};
hipError_t launch_column_sums(const ColumnSums& c, hipStream_t s);

constexpr int kNormMax = 16384;  // elements of a normed row, at most

constexpr int kGlrTile = 128;    // tokens between two states that a forward keeps for its gradients
struct Glr {
  Rows x, f, g;                 // [B, n, D]
  const float *decay, *fb, *gb; // [D]; the biases may be null
  float* state;                 // [B, D] or null; read and written
  void* y;                      // [B, n, D] contiguous
  float* kept;                  // the state before every kGlrTile tokens [B, tiles, D], or null
  int B, n, D, dtype;
  float c;
  Rows dy;                      // backward
  void *dx, *df, *dg;           // [B, n, D] contiguous
  float *ddecay, *dfb, *dgb;    // [D]; the biases' may be null
};
double glr_threads(int B, int n, int D);
size_t glr_forward_ws(int B, int n, int D);
hipError_t launch_glr_forward(const Glr& a, void* ws, hipStream_t s);
hipError_t launch_glr_step(const Glr& a, hipStream_t s);
size_t glr_backward_ws(int B, int n, int D);
hipError_t launch_glr_backward(const Glr& a, void* ws, hipStream_t s);

struct Glu {
  Rows x;                       // [B, n, D]
  const void *wg, *wu;          // [F, D]
  void* h;                      // [B, n, F] contiguous
  int B, n, D, F, gelu;
  Rows dh;                      // backward: [B, n, F]
  void *dx, *dwg, *dwu;         // [B, n, D], [F, D] contiguous
};
hipError_t launch_glu(const Glu& a, hipStream_t s);
size_t glu_backward_ws(int B, int n, int D, int F);
hipError_t launch_glu_backward(const Glu& a, void* ws, hipStream_t s);

}  // namespace hla
