// Norm and position rotation of queries and keys, head by head, from the
// projection's [B, n, H, d] to the attention's [B, H, n, d] in one pass:
//   u = w x r,  r = 1 / sqrt(mean x^2 + eps)
//   (u_i, u_j) -> (u_i c - u_j s, u_j c + u_i s)  for the pairs (i, j) of the
//   first rot dimensions: (i, i + rot/2), or (2i, 2i + 1) interleaved;
// and its gradients, with g the incoming one rotated back:
//   dx = r (g w - xhat mean(g w xhat)),  dw = sum g xhat,  xhat = x r.
//
// Bound by memory: every row is read once and written once.  LP lanes hold a
// head's row, 16 bytes each, the mean square goes over them by shuffles, and
// the other half of a rotation pair comes from its lane.  A thread takes
// several heads of one token, so that cos and sin are read once for them and
// the heads' loads are in flight together; queries and keys share the launch.
#include "common.h"
#include "mixer.h"
#include "profile.h"
#include "vec.h"

namespace hla {
namespace {

constexpr int kQkThreads = 256;

// Where the row of virtual head v (queries, then keys) of token (b, t) is.
template <typename T>
struct Head {
  const T* x;
  size_t out;      // row index in the [B, H, n, d] output of its kind
  bool key;
};
template <typename T>
__device__ __forceinline__ Head<T> head_at(const QkRope& a, int b, int t, int v) {
  Head<T> h;
  h.key = v >= a.H;
  const Rows& r = h.key ? a.k : a.q;
  const int i = h.key ? v - a.H : v;
  h.x = static_cast<const T*>(r.p) + b * r.bs + t * r.ts + (size_t)i * a.d;
  h.out = ((size_t)b * (h.key ? a.Hk : a.H) + i) * a.n + t;
  return h;
}

// cos and sin of the lane's V dimensions (1 and 0 past rot).  A position
// outside the tables rotates by NaN: nothing is read there.
template <int V>
__device__ __forceinline__ void angles(const QkRope& a, int b, int t, int c, float (&cs)[V], float (&sn)[V]) {
  long long pos = t;
  if (a.pos)
    pos = a.pos64 ? static_cast<const long long*>(a.pos)[b * a.pos_bs + t]
                  : static_cast<const int*>(a.pos)[b * a.pos_bs + t];
  const bool in = pos >= 0 && pos < a.positions;
  const int half = a.rot / 2;
  const size_t at = in ? (size_t)pos * half : 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = c + i;
    if (e < a.rot) {
      const int p = a.interleaved ? e / 2 : (e < half ? e : e - half);
      cs[i] = in ? a.cs[at + p] : __builtin_nanf("");
      sn[i] = in ? a.sn[at + p] : __builtin_nanf("");
    } else {
      cs[i] = 1.f;
      sn[i] = 0.f;
    }
  }
}

// out = u rotated by (cs, sign sn), u the lane's V dimensions from c on.  The
// pair's other element is in the lane itself (interleaved), or `hop` lanes
// on or back (hop > 0: rot/2 is a whole number of lanes), or, where a pair
// straddles lanes, fetched element by element from its lane.
template <int V>
__device__ __forceinline__ void rotate(const QkRope& a, int c, int hop, float sign, const float (&u)[V],
                                       const float (&cs)[V], const float (&sn)[V], float (&out)[V]) {
  const int half = a.rot / 2, lane = threadIdx.x & 63;
  if (a.interleaved || a.rot == 0) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float s0 = sign * sn[i], s1 = sign * sn[i + 1];
      out[i] = u[i] * cs[i] - u[i + 1] * s0;
      out[i + 1] = u[i + 1] * cs[i + 1] + u[i] * s1;
    }
    return;
  }
  const bool first = c < half;
  if (hop > 0) {
    const int from = c >= a.rot ? lane : first ? lane + hop : lane - hop;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float o = __shfl(u[i], from);
      const float s = first ? -sign * sn[i] : sign * sn[i];
      out[i] = c < a.rot ? u[i] * cs[i] + o * s : u[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = c + i;
    const int pe = e < half ? e + half : e - half;       // the pair's other element, for e < rot
    const int from = lane + (e < a.rot ? pe / V - c / V : 0), slot = pe % V;
    float o = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float w = __shfl(u[j], from);
      if (j == slot) o = w;
    }
    const float s = e < half ? -sign * sn[i] : sign * sn[i];
    out[i] = e < a.rot ? u[i] * cs[i] + o * s : u[i];
  }
}

template <int LP>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int m = 1; m < LP; m *= 2) v += __shfl_xor(v, m);
  return v;
}

template <int V>
__device__ __forceinline__ void weight(const void* w, int dtype, int c, bool there, float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = !there ? 0.f : w ? load_any(w, dtype, c + i) : 1.f;
}

// A row's lanes past d hold zeros.  Unit: HP virtual heads of one token.
template <typename T, int V, int LP, int HP>
__global__ __launch_bounds__(kQkThreads) void k_qk_rope(QkRope a, int groups, long long units) {
  const int lane = threadIdx.x % LP, c = lane * V;
  const long long unit = (long long)blockIdx.x * (kQkThreads / LP) + threadIdx.x / LP;
  if (unit >= units) return;                      // the LP lanes of a row leave together
  const int gr = (int)(unit % groups);
  const long long tok = unit / groups;
  const int b = (int)(tok / a.n), t = (int)(tok - (long long)b * a.n);
  const bool there = c < a.d;
  const int hop = (a.rot / 2) % V == 0 ? a.rot / 2 / V : 0;
  float x[HP][V];
#pragma unroll
  for (int k = 0; k < HP; ++k) {
    const int v = min(gr * HP + k, a.H + a.Hk - 1);
    if (there) {
      load_vec<T, V>(head_at<T>(a, b, t, v).x + c, x[k]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[k][i] = 0.f;
    }
  }
  float cs[V], sn[V];
  angles<V>(a, b, t, c, cs, sn);
#pragma unroll
  for (int k = 0; k < HP; ++k) {
    const int v = min(gr * HP + k, a.H + a.Hk - 1);
    const Head<T> h = head_at<T>(a, b, t, v);
    float w[V], u[V], o[V], ss = 0.f;
    weight<V>(h.key ? a.kw : a.qw, a.w_dtype, c, there, w);
#pragma unroll
    for (int i = 0; i < V; ++i) ss += x[k][i] * x[k][i];
    const float r = 1.f / sqrtf(row_sum<LP>(ss) / a.d + a.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) u[i] = x[k][i] * r * w[i];
    rotate<V>(a, c, hop, 1.f, u, cs, sn, o);
    if (there && gr * HP + k < a.H + a.Hk)
      store_vec<T, V>(static_cast<T*>(h.key ? a.ko : a.qo) + h.out * a.d + c, o);
  }
}

// Gradients.  Blocks walk units by the grid's stride; a thread keeps its lane's
// dimensions through all of them, so the two weights' gradients are summed in
// registers, then over the block's rows in a fixed order, a row of partials
// [2][d] a block; k_qk_sum adds the rows.
constexpr int kQkBackBlocks = 2048;

template <typename T, int V, int LP, int HP>
__global__ __launch_bounds__(kQkThreads) void k_qk_rope_back(QkRope a, int groups, long long units,
                                                             float* __restrict__ part) {
  constexpr int RB = kQkThreads / LP;
  const int lane = threadIdx.x % LP, c = lane * V;
  const bool there = c < a.d;
  const int hop = (a.rot / 2) % V == 0 ? a.rot / 2 / V : 0;
  float dw[2][V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[0][i] = dw[1][i] = 0.f;
  for (long long unit = (long long)blockIdx.x * RB + threadIdx.x / LP; unit < units;
       unit += (long long)gridDim.x * RB) {
    const int gr = (int)(unit % groups);
    const long long tok = unit / groups;
    const int b = (int)(tok / a.n), t = (int)(tok - (long long)b * a.n);
    float x[HP][V], g[HP][V];
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      const int v = min(gr * HP + k, a.H + a.Hk - 1);
      const Head<T> h = head_at<T>(a, b, t, v);
      if (there) {
        load_vec<T, V>(h.x + c, x[k]);
        load_vec<T, V>(static_cast<const T*>(h.key ? a.gk : a.gq) + h.out * a.d + c, g[k]);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[k][i] = g[k][i] = 0.f;
      }
    }
    float cs[V], sn[V];
    angles<V>(a, b, t, c, cs, sn);
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      const int v = min(gr * HP + k, a.H + a.Hk - 1);
      const Head<T> h = head_at<T>(a, b, t, v);
      float w[V], du[V], ss = 0.f, dot = 0.f;
      weight<V>(h.key ? a.kw : a.qw, a.w_dtype, c, there, w);
      rotate<V>(a, c, hop, -1.f, g[k], cs, sn, du);
#pragma unroll
      for (int i = 0; i < V; ++i) ss += x[k][i] * x[k][i];
      const float r = 1.f / sqrtf(row_sum<LP>(ss) / a.d + a.eps);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] *= r;
        dot += du[i] * w[i] * x[k][i];
      }
      const float mean = row_sum<LP>(dot) / a.d;
      if (there && gr * HP + k < a.H + a.Hk) {
        float dx[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dx[i] = r * (du[i] * w[i] - x[k][i] * mean);
          dw[0][i] += h.key ? 0.f : du[i] * x[k][i];
          dw[1][i] += h.key ? du[i] * x[k][i] : 0.f;
        }
        const int i = h.key ? v - a.H : v, heads = h.key ? a.Hk : a.H;
        store_vec<T, V>(static_cast<T*>(h.key ? a.dk : a.dq) + (((size_t)b * a.n + t) * heads + i) * a.d + c, dx);
      }
    }
  }
  __shared__ float red[RB][LP * V + 1];
#pragma unroll
  for (int z = 0; z < 2; ++z) {
#pragma unroll
    for (int i = 0; i < V; ++i) red[threadIdx.x / LP][c + i] = dw[z][i];
    __syncthreads();
    for (int e = threadIdx.x; e < a.d; e += kQkThreads) {
      float s = 0.f;
      for (int r = 0; r < RB; ++r) s += red[r][e];
      part[((size_t)blockIdx.x * 2 + z) * a.d + e] = s;
    }
    __syncthreads();
  }
}

constexpr int kQkSumRows = 64, kQkSumCols = 16;
__global__ __launch_bounds__(kQkSumRows * kQkSumCols) void k_qk_sum(QkRope a, const float* __restrict__ part,
                                                                    int rows) {
  __shared__ float red[kQkSumRows][kQkSumCols];
  const int cl = threadIdx.x % kQkSumCols, rg = threadIdx.x / kQkSumCols, col = blockIdx.x * kQkSumCols + cl;
  float s = 0.f;
  if (col < 2 * a.d)
    for (int r = rg; r < rows; r += kQkSumRows) s += part[(size_t)r * 2 * a.d + col];
  red[rg][cl] = s;
  __syncthreads();
  if (rg != 0 || col >= 2 * a.d) return;
  for (int r = 1; r < kQkSumRows; ++r) s += red[r][cl];
  void* to = col < a.d ? a.dqw : a.dkw;
  if (to) store_any(to, a.w_dtype, col % a.d, s);
}

template <typename T, int V, int LP, int HP>
hipError_t launch(const QkRope& a, float* part, hipStream_t s) {
  const int groups = (a.H + a.Hk + HP - 1) / HP;
  const long long units = (long long)a.B * a.n * groups, per = kQkThreads / LP;
  const long long blocks = (units + per - 1) / per;
  if (!part)
    return HLA_TIMED("qk_norm_rope", (k_qk_rope<T, V, LP, HP>), dim3((unsigned)blocks), dim3(kQkThreads), 0, s, a,
                     groups, units);
  const int nb = (int)(blocks < kQkBackBlocks ? blocks : kQkBackBlocks);
  const hipError_t e = HLA_TIMED("qk_norm_rope_back", (k_qk_rope_back<T, V, LP, HP>), dim3(nb), dim3(kQkThreads), 0, s,
                                 a, groups, units, part);
  if (e != hipSuccess || (!a.dqw && !a.dkw)) return e;
  return HLA_TIMED("qk_sum", k_qk_sum, dim3((2 * a.d + kQkSumCols - 1) / kQkSumCols), dim3(kQkSumRows * kQkSumCols), 0, s,
                   a, part, nb);
}

// four heads a thread where that still leaves every CU eight waves, one otherwise (a few tokens)
template <typename T, int V, int LP>
hipError_t by_heads(const QkRope& a, float* part, hipStream_t s) {
  const long long rows = (long long)a.B * a.n * (a.H + a.Hk);
  if (rows * LP / 4 >= 256LL * 8 * 64) return launch<T, V, LP, 4>(a, part, s);
  return launch<T, V, LP, 1>(a, part, s);
}

template <typename T, int V>
hipError_t by_width(const QkRope& a, float* part, hipStream_t s) {
  const int pieces = a.d / V;
  if (pieces <= 4) return by_heads<T, V, 4>(a, part, s);
  if (pieces <= 8) return by_heads<T, V, 8>(a, part, s);
  if (pieces <= 16) return by_heads<T, V, 16>(a, part, s);
  if (pieces <= 32) return by_heads<T, V, 32>(a, part, s);
  return by_heads<T, V, 64>(a, part, s);
}

hipError_t by_type(const QkRope& a, float* part, hipStream_t s) {
  return a.dtype == 1 ? by_width<bf16, 8>(a, part, s) : by_width<float, 4>(a, part, s);
}

}  // namespace

hipError_t launch_qk_rope(const QkRope& a, hipStream_t s) { return by_type(a, nullptr, s); }
size_t qk_rope_backward_ws(int d) { return sizeof(float) * kQkBackBlocks * 2 * (size_t)d; }
hipError_t launch_qk_rope_backward(const QkRope& a, void* ws, hipStream_t s) {
  return by_type(a, static_cast<float*>(ws), s);
}

}  // namespace hla
