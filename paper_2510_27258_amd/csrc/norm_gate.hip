// The norm of a mixer's output with its gate, over the d elements of a group
// (a head, or the whole token):
//   gate = z sigmoid(z),  v = y gate,  out = w v r         (the gate first)
//                         v = y,       out = w v r gate    (norm_first)
//   r = 1 / sqrt(mean v^2 + eps)
// and its gradients, with hat = v r and g the incoming one (times the gate
// where the norm comes first):
//   dv = r (g w - hat mean(g w hat)),  dw = sum g hat,
//   dz = (dv y or dout w hat) sigmoid(z) (1 + z (1 - sigmoid(z))).
//
// Bound by memory: every input is read once and every output written once: 16384
// tokens of 16 heads of 64, fp32 beside bf16 gates, 35 us, 3.8 TB/s where heads lie
// apart, their gradients 47 us, 5.0 TB/s.  A thread keeps its group and its elements
// of a row while its block goes over the tokens, so the weight is loaded once and
// its gradient summed in registers.
#include "block.h"
#include "rows.h"

namespace hla {
namespace {

constexpr int kBlocks = 2048;       // of a forward, at most, a block of groups

// A thread's place: slots of LANES threads take the block's groups, then its tokens.
template <typename S>
struct Place {
  int lane, g, off, tokens;  // off: its token among the block's `tokens`
  bool there;
  __device__ __forceinline__ Place(int G) {
    const int slot = threadIdx.x / S::LANES, per = min(G, S::ROWS);
    lane = threadIdx.x % S::LANES;
    tokens = S::ROWS / per;
    off = slot / per;
    g = blockIdx.y * per + slot % per;
    there = off < tokens && g < G;
  }
};

__device__ __forceinline__ size_t at(const Rows3& r, unsigned b, unsigned t, int g) {
  return (size_t)b * r.bs + (size_t)t * r.ts + (size_t)g * r.gs;
}

template <typename TY, typename T, typename S, bool WHOLE>
__global__ __launch_bounds__(S::THREADS) void k_gated_norm(GatedNorm a) {
  __shared__ float red[2][1][S::WAVES];
  constexpr bool kExact = sizeof(T) == 4;
  const Place<S> p(a.G);
  const unsigned toks = (unsigned)a.B * a.n;
  float w[S::E];
  load_weight<S, WHOLE>(a.w, a.w_dtype, a.per_group ? (size_t)p.g * a.d : 0, p.there ? a.d : 0, p.lane, w);
  int turn = 0;
  for (unsigned t0 = blockIdx.x; t0 * (unsigned long long)p.tokens < toks; t0 += gridDim.x, turn ^= 1) {
    const unsigned long long tok = (unsigned long long)t0 * p.tokens + p.off;
    const bool there = p.there && tok < toks;
    const unsigned b = a.B > 1 ? (unsigned)tok / a.n : 0, t = (unsigned)tok - b * a.n;
    const int d = there ? a.d : 0;
    RowRaw<TY, S, WHOLE> y;
    RowRaw<T, S, WHOLE> z;
    y.load(static_cast<const TY*>(a.y.p) + (there ? at(a.y, b, t, p.g) : 0), d, p.lane);
    if (a.z.p) z.load(static_cast<const T*>(a.z.p) + (there ? at(a.z, b, t, p.g) : 0), d, p.lane);
    float v[S::E], gate[S::E], ss[1] = {0.f};
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      v[e] = y.at(e);
      if (a.z.p) {
        gate[e] = z.at(e) * sigmoid<kExact>(z.at(e));
        if (!a.norm_first) v[e] *= gate[e];
      }
      ss[0] += v[e] * v[e];
    }
    row_sums<S, 1>(ss, red[turn]);
    const float r = 1.f / sqrtf(ss[0] / a.d + a.eps);
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      v[e] *= r * w[e];
      if (a.z.p && a.norm_first) v[e] *= gate[e];
    }
    store_row<T, S, WHOLE>(static_cast<T*>(a.out) + (there ? ((size_t)tok * a.G + p.g) * a.d : 0), d, p.lane, v);
  }
}

// Blocks keep their groups and take every gridDim.x-th share of the tokens; the
// weight's partial sums: [grid.x][G][d] with a weight for each group, else
// [grid.x grid.y][d], the block's rows summed in a fixed order.
template <typename TY, typename T, typename S, bool WHOLE>
__global__ __launch_bounds__(S::THREADS) void k_gated_norm_back(GatedNorm a, float* __restrict__ part,
                                                               float* __restrict__ stats) {
  constexpr bool kSums = !sums_apart<S>();
  __shared__ float red[2][2][1][S::WAVES];
  constexpr bool kExact = sizeof(TY) == 4;
  const Place<S> p(a.G);
  const unsigned toks = (unsigned)a.B * a.n;
  float w[S::E], dw[S::E];
  load_weight<S, WHOLE>(a.w, a.w_dtype, a.per_group ? (size_t)p.g * a.d : 0, p.there ? a.d : 0, p.lane, w);
#pragma unroll
  for (int e = 0; e < S::E; ++e) dw[e] = 0.f;
  int turn = 0;
  for (unsigned t0 = blockIdx.x; t0 * (unsigned long long)p.tokens < toks; t0 += gridDim.x, turn ^= 1) {
    const unsigned long long tok = (unsigned long long)t0 * p.tokens + p.off;
    const bool there = p.there && tok < toks;
    const unsigned b = a.B > 1 ? (unsigned)tok / a.n : 0, t = (unsigned)tok - b * a.n;
    const int d = there ? a.d : 0;
    const size_t here = there ? ((size_t)tok * a.G + p.g) * a.d : 0;
    RowRaw<TY, S, WHOLE> y;
    RowRaw<T, S, WHOLE> z, go;
    y.load(static_cast<const TY*>(a.y.p) + (there ? at(a.y, b, t, p.g) : 0), d, p.lane);
    go.load(static_cast<const T*>(a.dout) + here, d, p.lane);
    if (a.z.p) z.load(static_cast<const T*>(a.z.p) + (there ? at(a.z, b, t, p.g) : 0), d, p.lane);
    float v[S::E], sig[S::E], ss[1] = {0.f};
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      v[e] = y.at(e);
      if (a.z.p) {
        sig[e] = sigmoid<kExact>(z.at(e));
        if (!a.norm_first) v[e] *= z.at(e) * sig[e];
      }
      ss[0] += v[e] * v[e];
    }
    row_sums<S, 1>(ss, red[turn][0]);
    // behind the last token 0: the rows there are zeros, and with eps = 0 an infinite r would make NaN of the weight's sums
    const float r = there ? 1.f / sqrtf(ss[0] / a.d + a.eps) : 0.f;
    float dot[1] = {0.f};
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      v[e] *= r;                                   // hat from here on
      const float g = a.z.p && a.norm_first ? go.at(e) * (z.at(e) * sig[e]) : go.at(e);
      dot[0] += g * w[e] * v[e];
      if constexpr (kSums) dw[e] += g * v[e];
    }
    if constexpr (!kSums) {
      if (p.lane == 0 && there) stats[(size_t)tok * a.G + p.g] = r;
    }
    row_sums<S, 1>(dot, red[turn][1]);
    const float mean = dot[0] / a.d;
    float dy[S::E], dz[S::E];
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float zz = a.z.p ? z.at(e) : 0.f, s = a.z.p ? sig[e] : 0.f, gate = a.z.p ? zz * s : 1.f;
      const float g = a.norm_first ? go.at(e) * gate : go.at(e);
      const float dv = r * (g * w[e] - v[e] * mean);
      dy[e] = a.norm_first ? dv : dv * gate;
      dz[e] = (a.norm_first ? go.at(e) * w[e] * v[e] : dv * y.at(e)) * (s * (1.f + zz * (1.f - s)));
    }
    store_row<TY, S, WHOLE>(static_cast<TY*>(const_cast<void*>(a.dy.p)) + (there ? at(a.dy, b, t, p.g) : 0), d, p.lane, dy);
    if (a.z.p) store_row<T, S, WHOLE>(static_cast<T*>(a.dz) + here, d, p.lane, dz);
  }
  if (!kSums || !a.dw) return;
  if constexpr (S::ROWS == 1) {
    float* to = part + (a.per_group ? (size_t)blockIdx.x * a.G + p.g : (size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.d;
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = (ch * S::LANES + p.lane) * 8 + i;
        if (c < a.d) to[c] = dw[ch * 8 + i];
      }
  } else {
    __shared__ float sums[S::ROWS][S::LANES * S::E + 1];
    const int per = min(a.G, S::ROWS), slot = threadIdx.x / S::LANES;
#pragma unroll
    for (int ch = 0; ch < S::CH; ++ch)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        sums[slot][(ch * S::LANES + p.lane) * 8 + i] = p.there ? dw[ch * 8 + i] : 0.f;
    __syncthreads();
    if (a.per_group) {
      for (int e = threadIdx.x; e < per * a.d; e += S::THREADS) {
        const int k = e / a.d, c = e - k * a.d, g = blockIdx.y * per + k;
        if (g >= a.G) continue;
        float s = 0.f;
        for (int o = 0; o < p.tokens; ++o) s += sums[o * per + k][c];
        part[((size_t)blockIdx.x * a.G + g) * a.d + c] = s;
      }
    } else {
      for (int c = threadIdx.x; c < a.d; c += S::THREADS) {
        float s = 0.f;
        for (int o = 0; o < S::ROWS; ++o) s += sums[o][c];
        part[((size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.d + c] = s;
      }
    }
  }
}

// The weight's sums of wide rows, from each one's 1 / rms(v): with a weight for each
// group [kShares][G][d], blockIdx.z the group, else [kShares][d].
template <typename TY, typename T, bool WHOLE>
__global__ __launch_bounds__(256) void k_gated_norm_sums(GatedNorm a, float* __restrict__ part,
                                                         const float* __restrict__ stats) {
  using S = Columns;
  constexpr bool kExact = sizeof(TY) == 4;
  const int lane = blockIdx.x * 256 + threadIdx.x;
  const unsigned toks = (unsigned)a.B * a.n, groups = a.per_group ? 1 : a.G;
  float dw[S::E];
#pragma unroll
  for (int e = 0; e < S::E; ++e) dw[e] = 0.f;
#pragma unroll 2
  for (unsigned long long row = blockIdx.y; row < (unsigned long long)toks * groups; row += kShares) {
    const unsigned tok = (unsigned)(row / groups), b = tok / a.n, t = tok - b * a.n;
    const int g = a.per_group ? blockIdx.z : (int)(row - (unsigned long long)tok * groups);
    const size_t at_row = (size_t)tok * a.G + g;
    const float r = stats[at_row];
    RowRaw<TY, S, WHOLE> y;
    RowRaw<T, S, WHOLE> z, go;
    y.load(static_cast<const TY*>(a.y.p) + at(a.y, b, t, g), a.d, lane);
    go.load(static_cast<const T*>(a.dout) + at_row * a.d, a.d, lane);
    if (a.z.p) z.load(static_cast<const T*>(a.z.p) + at(a.z, b, t, g), a.d, lane);
#pragma unroll
    for (int e = 0; e < S::E; ++e) {
      const float gate = a.z.p ? z.at(e) * sigmoid<kExact>(z.at(e)) : 1.f;
      dw[e] += go.at(e) * gate * (y.at(e) * r);      // the gate belongs to the one or the other
    }
  }
#pragma unroll
  for (int e = 0; e < S::E; ++e)
    if (lane * 8 + e < a.d) part[((size_t)blockIdx.y * gridDim.z + blockIdx.z) * a.d + lane * 8 + e] = dw[e];
}

constexpr int kSumRows = 64, kSumCols = 16;
// Workgroups of a sum, at most: a launch has less than 2^32 threads a dimension, and one with more runs a part of them
// without an error.  Wider sums take several turns of the same workgroups.
constexpr int kSumBlocks = 65536;
__global__ __launch_bounds__(kSumRows * kSumCols) void k_column_sums(ColumnSums c) {
  __shared__ float red[kSumRows][kSumCols];
  const int cl = threadIdx.x % kSumCols, rg = threadIdx.x / kSumCols, apart = gridDim.x * kSumCols;
  void* to = c.to[blockIdx.y];
  if (!to) return;
  const float* part = c.part + (size_t)blockIdx.y * c.rows * c.cols;
  for (int c0 = blockIdx.x * kSumCols; c0 < c.cols; c0 += apart) {
    const int col = c0 + cl;
    float s = 0.f;
    if (col < c.cols) {
      constexpr int kAtOnce = 8;      // loads on their way together
      for (int r0 = rg; r0 < c.rows; r0 += kSumRows * kAtOnce) {
        float v[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
          v[k] = r0 + k * kSumRows < c.rows ? part[(size_t)(r0 + k * kSumRows) * c.cols + col] : 0.f;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) s += v[k];
      }
    }
    red[rg][cl] = s;
    __syncthreads();
    if (rg == 0 && col < c.cols) {
      for (int r = 1; r < kSumRows; ++r) s += red[r][cl];
      store_any(to, c.dtype, col, s);
    }
    if (c.cols - c0 > apart) __syncthreads();      // another turn writes red again
  }
}

// Sequences laid one behind the other are one long one: no division by n.
void flatten(GatedNorm& a) {
  auto joined = [&](const Rows3& r) { return !r.p || a.n == 1 || r.bs == (long long)a.n * r.ts; };
  if (a.B == 1) return;
  if (a.n == 1) {   // a batch of single tokens is a sequence
    auto turn = [](Rows3& r) { r.ts = r.bs; };
    turn(a.y), turn(a.z), turn(a.dy);
  } else if (!joined(a.y) || !joined(a.z) || !joined(a.dy)) {
    return;
  }
  a.n *= a.B;
  a.B = 1;
}

struct Grid {
  int x, y;
};
template <typename S>
Grid grid_of(int B, int n, int G, int most) {
  const int per = G < S::ROWS ? G : S::ROWS, tokens = S::ROWS / per, gy = (G + per - 1) / per;
  const long long shares = ((long long)B * n + tokens - 1) / tokens, x = most / gy > 1 ? most / gy : 1;
  return {(int)(shares < x ? shares : x), gy};
}

template <typename TY, typename T, bool WHOLE>
hipError_t forward(const GatedNorm& a, hipStream_t s) {
  return by_row<false>(a.d, [&](auto shape) {
    using S = decltype(shape);
    const Grid g = grid_of<S>(a.B, a.n, a.G, kBlocks * ((a.G + S::ROWS - 1) / S::ROWS));
    return HLA_TIMED("gated_norm", (k_gated_norm<TY, T, S, WHOLE>), dim3(g.x, g.y), dim3(S::THREADS), 0, s, a);
  });
}

template <typename TY, typename T, bool WHOLE>
hipError_t backward(const GatedNorm& a, float* part, hipStream_t s) {
  Grid g{};
  const hipError_t e = by_row<true>(a.d, [&](auto shape) {
    using S = decltype(shape);
    float* stats = part;
    g = grid_of<S>(a.B, a.n, a.G, sums_apart<S>() ? kBlocks : back_blocks<S>());
    const hipError_t e = HLA_TIMED("gated_norm_back", (k_gated_norm_back<TY, T, S, WHOLE>), dim3(g.x, g.y), dim3(S::THREADS),
                                   0, s, a, part, stats);
    if (e != hipSuccess || !sums_apart<S>() || !a.dw) return e;
    part += ((size_t)a.B * a.n * a.G + 3) & ~(size_t)3;
    g = {kShares, 1};
    return HLA_TIMED("gated_norm_sums", (k_gated_norm_sums<TY, T, WHOLE>),
                     dim3((a.d + 2047) / 2048, kShares, a.per_group ? a.G : 1), dim3(256), 0, s, a, part, stats);
  });
  if (e != hipSuccess || !a.dw) return e;
  ColumnSums c{part, {a.dw, nullptr, nullptr}, a.per_group ? g.x : g.x * g.y, a.per_group ? a.G * a.d : a.d, a.w_dtype};
  return launch_column_sums(c, s);
}

template <typename TY, typename T>
hipError_t by_width(GatedNorm a, bool back, float* part, hipStream_t s) {
  flatten(a);
  const bool whole = a.d % 8 == 0;
  if (back) return whole ? backward<TY, T, true>(a, part, s) : backward<TY, T, false>(a, part, s);
  return whole ? forward<TY, T, true>(a, s) : forward<TY, T, false>(a, s);
}

hipError_t by_type(const GatedNorm& a, bool back, float* part, hipStream_t s) {
  if (a.dtype == 0) return by_width<float, float>(a, back, part, s);
  return a.y_dtype == 0 ? by_width<float, bf16>(a, back, part, s) : by_width<bf16, bf16>(a, back, part, s);
}

}  // namespace

hipError_t launch_column_sums(const ColumnSums& c, hipStream_t s) {
  const int blocks = (c.cols + kSumCols - 1) / kSumCols;
  return HLA_TIMED("column_sums", k_column_sums, dim3(blocks < kSumBlocks ? blocks : kSumBlocks, 3),
                   dim3(kSumRows * kSumCols), 0, s, c);
}

hipError_t launch_gated_norm(const GatedNorm& a, hipStream_t s) { return by_type(a, false, nullptr, s); }
size_t gated_norm_backward_ws(int B, int n, int G, int d, int per_group) {
  return by_row<true>(d, [&](auto shape) {
    using S = decltype(shape);
    if (sums_apart<S>())
      return sizeof(float) * ((((size_t)B * n * G + 3) & ~(size_t)3) + (size_t)kShares * (per_group ? G : 1) * d);
    const Grid g = grid_of<S>(B, n, G, back_blocks<S>());
    return sizeof(float) * g.x * (size_t)(per_group ? G : g.y) * d;
  });
}
hipError_t launch_gated_norm_backward(const GatedNorm& a, void* ws, hipStream_t s) {
  return by_type(a, true, static_cast<float*>(ws), s);
}

}  // namespace hla
