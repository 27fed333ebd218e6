// The residual addition with the norms on both sides of it:
//   u = y, or post y / sqrt(mean y^2 + eps)      (the norm after a block)
//   r = x + alpha scale u                        (the residual stream)
//   out = w r / sqrt(mean r^2 + eps)             (the norm before the next)
// and its gradients, with hat_v = v / rms(v), g of out and gr of r:
//   dr = gr + (g w - hat_r mean(g w hat_r)) / rms(r) = dx,  du = alpha scale dr,
//   dy = du or (du post - hat_y mean(du post hat_y)) / rms(y),
//   dw = sum g hat_r,  dpost = sum du hat_y,  dscale = sum alpha u dr.
// out is made from the fp32 r, not from the rounded one that goes on, and the
// gradients form r again from x and y: a bf16 r would cost the weight's
// gradient up to 2^-8 of every term.
//
// Bound by memory: every input is read once and every output written once: 32768
// rows of 4096 in bf16 197 us, 5.4 TB/s; 16384 rows of 1024 of an fp32 stream with
// both norms 39 us, 5.1 TB/s, their gradients 61 us, 5.0.  A thread keeps its
// elements of a row while its block goes over the rows, so the weights are loaded
// once and their gradients summed in registers.
#include "block.h"
#include "rows.h"

namespace hla {
namespace {

constexpr int kBlocks = 4096;       // of a forward, at most

// The row's place in memory: sequences laid apart cost a division.
__device__ __forceinline__ size_t at(const Rows& r, const ResidualNorm& a, unsigned row) {
  if (a.B == 1) return (size_t)row * r.ts;
  const unsigned b = row / a.n;
  return (size_t)b * r.bs + (size_t)(row - b * a.n) * r.ts;
}

template <typename TX, typename T, typename S, bool WHOLE>
__global__ __launch_bounds__(S::THREADS) void k_residual_norm(ResidualNorm a) {
  __shared__ float red[2][2][1][S::WAVES];
  const int lane = threadIdx.x % S::LANES;
  const unsigned rows = (unsigned)a.B * a.n;
  float w[S::E], step[S::E], post[S::E];
  load_weight<S, WHOLE>(a.w, a.w_dtype, 0, a.D, lane, w);
  load_weight<S, WHOLE>(a.scale, a.w_dtype, 0, a.D, lane, step);
  if (a.post) load_weight<S, WHOLE>(a.post, a.w_dtype, 0, a.D, lane, post);
  int turn = 0;
  for (unsigned long long r0 = (unsigned long long)blockIdx.x * S::ROWS; r0 < rows;
       r0 += (unsigned long long)gridDim.x * S::ROWS, turn ^= 1) {
    const unsigned row = (unsigned)r0 + threadIdx.x / S::LANES;
    const bool there = row < rows;
    const int d = there ? a.D : 0;
    RowRaw<TX, S, WHOLE> x;
    RowRaw<T, S, WHOLE> y;
    x.load(static_cast<const TX*>(a.x.p) + (there ? at(a.x, a, row) : 0), d, lane);
    y.load(static_cast<const T*>(a.y.p) + (there ? at(a.y, a, row) : 0), d, lane);
    float ry = 1.f;
    if (a.post) {
      float ss[1] = {0.f};
#pragma unroll
      for (int e = 0; e < S::E; ++e) ss[0] += y.at(e) * y.at(e);
      row_sums<S, 1>(ss, red[turn][0]);
      ry = 1.f / sqrtf(ss[0] / a.D + a.eps);
    }
    float r[S::E], ss[1] = {0.f};
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float u = a.post ? y.at(e) * ry * post[e] : y.at(e);
      r[e] = x.at(e) + a.alpha * step[e] * u;
      ss[0] += r[e] * r[e];
    }
    row_sums<S, 1>(ss, red[turn][1]);
    const float rr = 1.f / sqrtf(ss[0] / a.D + a.eps);
    const size_t here = there ? (size_t)row * a.D : 0;
    store_row<TX, S, WHOLE>(static_cast<TX*>(a.r) + here, d, lane, r);
#pragma unroll
    for (int e = 0; e < S::E; ++e) r[e] *= rr * w[e];
    store_row<T, S, WHOLE>(static_cast<T*>(a.out) + here, d, lane, r);
  }
}

// Partial sums of the three weights' gradients: [3][blocks][D], the block's
// rows summed in a fixed order.  Rows of several waves wait for each other three
// times: where a thread has one piece of each, the next rows are loaded meanwhile
// (8192 rows of 4096 in bf16 92 us, 118 without; of 2048 53 and 58).
template <typename TX, typename T, typename S, bool WHOLE>
__global__ __launch_bounds__(S::THREADS) void k_residual_norm_back(ResidualNorm a, float* __restrict__ part,
                                                                  float4* __restrict__ stats) {
  constexpr bool kSums = !sums_apart<S>();
  __shared__ float red[2][4][S::WAVES];
  const int lane = threadIdx.x % S::LANES;
  const unsigned rows = (unsigned)a.B * a.n;
  float w[S::E], step[S::E], post[S::E], dw[S::E], dscale[S::E], dpost[S::E];
  load_weight<S, WHOLE>(a.w, a.w_dtype, 0, a.D, lane, w);
  load_weight<S, WHOLE>(a.scale, a.w_dtype, 0, a.D, lane, step);
  if (a.post) load_weight<S, WHOLE>(a.post, a.w_dtype, 0, a.D, lane, post);
#pragma unroll
  for (int e = 0; e < S::E; ++e) dw[e] = dscale[e] = dpost[e] = 0.f;
  constexpr bool kAhead = S::CH == 1 && S::WAVES > 1;
  RowRaw<TX, S, WHOLE> x1, gr1;
  RowRaw<T, S, WHOLE> y1, go1;
  auto load = [&](unsigned long long r0) {
    const unsigned long long row = r0 + threadIdx.x / S::LANES;
    const bool there = row < rows;
    const int d = there ? a.D : 0;
    const size_t here = there ? (size_t)row * a.D : 0;
    x1.load(static_cast<const TX*>(a.x.p) + (there ? at(a.x, a, (unsigned)row) : 0), d, lane);
    y1.load(static_cast<const T*>(a.y.p) + (there ? at(a.y, a, (unsigned)row) : 0), d, lane);
    go1.load(static_cast<const T*>(a.dout) + here, a.dout ? d : 0, lane);
    gr1.load(static_cast<const TX*>(a.dr) + here, a.dr ? d : 0, lane);
  };
  if constexpr (kAhead) load((unsigned long long)blockIdx.x * S::ROWS);
  int turn = 0;
  for (unsigned long long r0 = (unsigned long long)blockIdx.x * S::ROWS; r0 < rows;
       r0 += (unsigned long long)gridDim.x * S::ROWS, turn ^= 1) {
    const unsigned long long row = r0 + threadIdx.x / S::LANES;
    const bool there = row < rows;
    const int d = there ? a.D : 0;
    const size_t here = there ? (size_t)row * a.D : 0;
    if constexpr (!kAhead) load(r0);
    const RowRaw<TX, S, WHOLE> x = x1, gr = gr1;
    const RowRaw<T, S, WHOLE> y = y1, go = go1;
    if constexpr (kAhead) load(r0 + (unsigned long long)gridDim.x * S::ROWS);
    // behind the last row both inverse roots are 0: those rows are zeros, and with eps = 0 infinite roots would make NaN
    // of the weights' sums
    float ry = 1.f;
    if (a.post) {
      float ss[1] = {0.f};
#pragma unroll
      for (int e = 0; e < S::E; ++e) ss[0] += y.at(e) * y.at(e);
      row_sums<S, 1>(ss, red[turn]);
      ry = there ? 1.f / sqrtf(ss[0] / a.D + a.eps) : 0.f;
    }
    float r[S::E], dr[S::E], two[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float u = a.post ? y.at(e) * ry * post[e] : y.at(e);
      r[e] = x.at(e) + a.alpha * step[e] * u;
      two[0] += r[e] * r[e];
      two[1] += go.at(e) * w[e] * r[e];
    }
    row_sums<S, 2>(two, red[turn] + 1);
    const float rr = there ? 1.f / sqrtf(two[0] / a.D + a.eps) : 0.f, mean = two[1] / a.D * rr;
    float dot[1] = {0.f};
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float hat = r[e] * rr;
      dr[e] = gr.at(e) + rr * (go.at(e) * w[e] - hat * mean);
      const float yhat = y.at(e) * ry, u = a.post ? yhat * post[e] : y.at(e);
      if constexpr (kSums) {
        dw[e] += go.at(e) * hat;
        dscale[e] += a.alpha * u * dr[e];
      }
      if (a.post) {
        const float du = a.alpha * step[e] * dr[e];
        if constexpr (kSums) dpost[e] += du * yhat;
        dot[0] += du * post[e] * yhat;
      }
    }
    if constexpr (!kSums) {
      if (lane == 0 && there) stats[row] = make_float4(ry, rr, mean, 0.f);
    }
    store_row<TX, S, WHOLE>(static_cast<TX*>(a.dx) + here, d, lane, dr);
    if (a.post) row_sums<S, 1>(dot, red[turn] + 3);
    const float mean_y = dot[0] / a.D;
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float du = a.alpha * step[e] * dr[e];
      r[e] = a.post ? ry * (du * post[e] - y.at(e) * ry * mean_y) : du;
    }
    store_row<T, S, WHOLE>(static_cast<T*>(a.dy) + here, d, lane, r);
  }
  if constexpr (!kSums) return;
  __shared__ float sums[S::ROWS > 1 ? S::ROWS : 1][S::ROWS > 1 ? S::LANES * S::E + 1 : 1];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (!(k == 0 ? a.dw : k == 1 ? a.dpost : a.dscale)) continue;
    const float(&mine)[S::E] = k == 0 ? dw : k == 1 ? dpost : dscale;
    float* to = part + ((size_t)k * gridDim.x + blockIdx.x) * a.D;
    if constexpr (S::ROWS > 1) __syncthreads();
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = (ch * S::LANES + lane) * 8 + i;
        if constexpr (S::ROWS > 1)
          sums[threadIdx.x / S::LANES][c] = mine[ch * 8 + i];
        else if (c < a.D)
          to[c] = mine[ch * 8 + i];
      }
    if constexpr (S::ROWS > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += S::THREADS) {
        float s = 0.f;
        for (int o = 0; o < S::ROWS; ++o) s += sums[o][c];
        to[c] = s;
      }
    }
  }
}

// The weights' sums of wide rows, from the statistics 1 / rms(y), 1 / rms(r) and
// mean(g w hat_r) of each: [3][kShares][D].
template <typename TX, typename T, bool WHOLE>
__global__ __launch_bounds__(256) void k_residual_norm_sums(ResidualNorm a, float* __restrict__ part,
                                                            const float4* __restrict__ stats) {
  using S = Columns;
  const int lane = blockIdx.x * 256 + threadIdx.x;
  const unsigned rows = (unsigned)a.B * a.n;
  float w[S::E], step[S::E], post[S::E], dw[S::E], dscale[S::E], dpost[S::E];
  load_weight<S, WHOLE>(a.w, a.w_dtype, 0, a.D, lane, w);
  load_weight<S, WHOLE>(a.scale, a.w_dtype, 0, a.D, lane, step);
  load_weight<S, WHOLE>(a.post, a.w_dtype, 0, a.D, lane, post);
#pragma unroll
  for (int e = 0; e < S::E; ++e) dw[e] = dscale[e] = dpost[e] = 0.f;
#pragma unroll 2
  for (unsigned row = blockIdx.y; row < rows; row += kShares) {
    const float4 st = stats[row];
    const size_t here = (size_t)row * a.D;
    RowRaw<TX, S, WHOLE> x, gr;
    RowRaw<T, S, WHOLE> y, go;
    x.load(static_cast<const TX*>(a.x.p) + at(a.x, a, row), a.D, lane);
    y.load(static_cast<const T*>(a.y.p) + at(a.y, a, row), a.D, lane);
    go.load(static_cast<const T*>(a.dout) + here, a.dout ? a.D : 0, lane);
    gr.load(static_cast<const TX*>(a.dr) + here, a.dr ? a.D : 0, lane);
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float yhat = y.at(e) * st.x, u = a.post ? yhat * post[e] : y.at(e);
      const float hat = (x.at(e) + a.alpha * step[e] * u) * st.y;
      const float dr = gr.at(e) + st.y * (go.at(e) * w[e] - hat * st.z);
      dw[e] += go.at(e) * hat;
      dscale[e] += a.alpha * u * dr;
      dpost[e] += a.alpha * step[e] * dr * yhat;
    }
  }
#pragma unroll
  for (int e = 0; e < S::E; ++e) {
    const int c = lane * 8 + e;
    if (c >= a.D) continue;
    float* to = part + (size_t)blockIdx.y * a.D + c;
    const size_t apart = (size_t)kShares * a.D;
    to[0] = dw[e];
    to[apart] = dpost[e];
    to[2 * apart] = dscale[e];
  }
}

// Sequences laid one behind the other are one long one.
void flatten(ResidualNorm& a) {
  if (a.B == 1) return;
  if (a.n == 1) {
    a.x.ts = a.x.bs;
    a.y.ts = a.y.bs;
  } else if (a.x.bs != a.n * a.x.ts || a.y.bs != a.n * a.y.ts) {
    return;
  }
  a.n *= a.B;
  a.B = 1;
}

template <typename S>
int blocks_of(int B, int n, int most) {
  const long long need = ((long long)B * n + S::ROWS - 1) / S::ROWS;
  return (int)(need < most ? need : most);
}

template <typename TX, typename T, bool WHOLE>
hipError_t forward(const ResidualNorm& a, hipStream_t s) {
  return by_row<false>(a.D, [&](auto shape) {
    using S = decltype(shape);
    return HLA_TIMED("residual_norm", (k_residual_norm<TX, T, S, WHOLE>), dim3(blocks_of<S>(a.B, a.n, kBlocks)),
                     dim3(S::THREADS), 0, s, a);
  });
}

template <typename TX, typename T, bool WHOLE>
hipError_t backward(const ResidualNorm& a, float* part, hipStream_t s) {
  int blocks = 0;
  const hipError_t e = by_row<true>(a.D, [&](auto shape) {
    using S = decltype(shape);
    float4* stats = reinterpret_cast<float4*>(part);
    blocks = blocks_of<S>(a.B, a.n, sums_apart<S>() ? kBlocks : back_blocks<S>());
    const hipError_t e = HLA_TIMED("residual_norm_back", (k_residual_norm_back<TX, T, S, WHOLE>), dim3(blocks),
                                   dim3(S::THREADS), 0, s, a, part, stats);
    if (e != hipSuccess || !sums_apart<S>() || !(a.dw || a.dpost || a.dscale)) return e;
    part += 4 * (size_t)a.B * a.n;
    blocks = kShares;
    return HLA_TIMED("residual_norm_sums", (k_residual_norm_sums<TX, T, WHOLE>), dim3((a.D + 2047) / 2048, kShares),
                     dim3(256), 0, s, a, part, stats);
  });
  if (e != hipSuccess || !(a.dw || a.dpost || a.dscale)) return e;
  return launch_column_sums({part, {a.dw, a.dpost, a.dscale}, blocks, a.D, a.w_dtype}, s);
}

template <typename TX, typename T>
hipError_t by_width(ResidualNorm a, bool back, float* part, hipStream_t s) {
  flatten(a);
  const bool whole = a.D % 8 == 0;
  if (back) return whole ? backward<TX, T, true>(a, part, s) : backward<TX, T, false>(a, part, s);
  return whole ? forward<TX, T, true>(a, s) : forward<TX, T, false>(a, s);
}

hipError_t by_type(const ResidualNorm& a, bool back, float* part, hipStream_t s) {
  if (a.dtype == 0) return by_width<float, float>(a, back, part, s);
  return a.x_dtype == 0 ? by_width<float, bf16>(a, back, part, s) : by_width<bf16, bf16>(a, back, part, s);
}

}  // namespace

hipError_t launch_residual_norm(const ResidualNorm& a, hipStream_t s) { return by_type(a, false, nullptr, s); }
size_t residual_norm_backward_ws(int B, int n, int D) {
  return by_row<true>(D, [&](auto shape) {
    using S = decltype(shape);
    if (sums_apart<S>()) return sizeof(float) * (4 * (size_t)B * n + 3 * (size_t)kShares * D);
    return sizeof(float) * 3 * (size_t)blocks_of<S>(B, n, back_blocks<S>()) * D;
  });
}
hipError_t launch_residual_norm_backward(const ResidualNorm& a, void* ws, hipStream_t s) {
  return by_type(a, true, static_cast<float*>(ws), s);
}

}  // namespace hla
