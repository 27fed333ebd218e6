// Norm and position rotation of queries and keys, head by head, from the
// projection's [B, n, H, d] to the attention's [B, H, n, d] in one pass:
//   u = w x r,  r = 1 / sqrt(mean x^2 + eps)
//   (u_i, u_j) -> (u_i c - u_j s, u_j c + u_i s)  for the pairs (i, j) of the
//   first rot dimensions: (i, i + rot/2), or (2i, 2i + 1) interleaved;
// and its gradients, with g the incoming one rotated back:
//   dx = r (g w - xhat mean(g w xhat)),  dw = sum g xhat,  xhat = x r.
//
// Bound by memory: every row is read once and written once.  LP lanes hold a
// head's row, 16 bytes each; the mean square goes over them by lane moves, and
// the other half of a rotation pair comes, as it was loaded, from its lane.
// A thread takes HP heads of one token and kind: cos, sin and the weight,
// folded into one factor for the element itself and one for its pair's other
// element, are made once for them, and the heads' loads are in flight
// together.  A block takes 256 / LP neighbouring tokens of the same heads, so
// that both its reads (HP rows of a token) and its writes (its tokens' rows of
// a head) are contiguous; queries and keys share the launch.
// Measured: 2 x 16384 tokens of 32 + 32 heads of 128 in bf16 (1.07 GB) 278 us,
// 3.9 TB/s; 4 x 4096 of 16 + 16 heads of 64 40 us, their gradients (201 MB) 53
// us, 3.8 TB/s, and 4 us for the weights' sums.
#include <cmath>

#include "common.h"
#include "mixer.h"
#include "vec.h"

namespace hla {
namespace {

constexpr int kQkThreads = 256;

// A block's share: tokens [tok0, tok0 + 256 / LP) of all B n, heads [h0, h0 + HP) of one kind.
struct Share {
  long long tok0;
  int h0, heads;
  bool key;
};
__device__ __forceinline__ Share share_of(const QkRope& a, long long unit, int HP, int tokens) {
  const int gq = (a.H + HP - 1) / HP, gk = (a.Hk + HP - 1) / HP;
  const int gr = (int)(unit % (gq + gk));
  Share s;
  s.tok0 = unit / (gq + gk) * tokens;
  s.key = gr >= gq;
  s.h0 = (s.key ? gr - gq : gr) * HP;
  s.heads = min(HP, (s.key ? a.Hk : a.H) - s.h0);
  return s;
}

// cos and sin of the lane's V dimensions (1 and 0 past rot), sin with the sign
// it has for the pair's other element (- in the first half).  A position
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
  // 16 bytes of a table at once, where its rows and its own address allow (it needs an fp32's alignment only)
  const bool wide = ((reinterpret_cast<uintptr_t>(a.cs) | reinterpret_cast<uintptr_t>(a.sn)) & 15) == 0;
  if (!a.interleaved && half % V == 0 && wide) {
    if (c < a.rot) {
      const int p = c < half ? c : c - half;
      load_many<float, 4, V>(a.cs, at + p, cs);
      load_many<float, 4, V>(a.sn, at + p, sn);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float s = c < half ? -sn[i] : sn[i];
      cs[i] = c >= a.rot ? 1.f : in ? cs[i] : __builtin_nanf("");
      sn[i] = c >= a.rot ? 0.f : in ? s : __builtin_nanf("");
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = c + i;
    cs[i] = 1.f;
    sn[i] = 0.f;
    if (e < a.rot) {
      const int p = a.interleaved ? e / 2 : (e < half ? e : e - half);
      const bool first = a.interleaved ? e % 2 == 0 : e < half;
      cs[i] = in ? a.cs[at + p] : __builtin_nanf("");
      sn[i] = in ? (first ? -a.sn[at + p] : a.sn[at + p]) : __builtin_nanf("");
    }
  }
}

// The other elements of the lane's pairs, v their own: from the lane itself
// (interleaved), from the lane hop on or back (rot/2 a whole number of lanes),
// or, where a pair straddles lanes, element by element.  Past rot: anything
// finite times the 0 of angles() - the lane's own elements.
template <typename T, int V>
__device__ __forceinline__ void others(const QkRope& a, int c, int hop, const Raw<T, V>& v, float (&o)[V]) {
  const int half = a.rot / 2, lane = threadIdx.x & 63;
  if (a.interleaved || a.rot == 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = v.at(i ^ 1);
    return;
  }
  if (hop > 0) {
    const int from = c >= a.rot ? lane : c < half ? lane + hop : lane - hop;
    Raw<T, V> w;
#pragma unroll
    for (int i = 0; i < Raw<T, V>::N; ++i) w.w[i] = __shfl((int)v.w[i], from);
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = w.at(i);
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = c + i;
    const int pe = e >= a.rot ? e : e < half ? e + half : e - half;
    const int from = lane + pe / V - c / V, slot = pe % V;
    o[i] = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float w = __shfl(v.at(j), from);
      if (j == slot) o[i] = w;
    }
  }
}

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}
// Sum over the LP lanes of a row, in each of them: neighbours, pairs of
// neighbours, then mirrored halves of 8, 16, 32 and 64 lanes.
template <int LP>
__device__ __forceinline__ float row_sum(float v) {
  v += moved<0xb1>(v);                       // quad_perm 1 0 3 2
  v += moved<0x4e>(v);                       // quad_perm 2 3 0 1
  if (LP >= 8) v += moved<0x141>(v);         // row_half_mirror
  if (LP >= 16) v += moved<0x140>(v);        // row_mirror
  if (LP >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if (LP >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return v;
}

template <int V>
__device__ __forceinline__ void weight(const QkRope& a, bool key, int c, bool there, float (&v)[V]) {
  const void* w = key ? a.kw : a.qw;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = !there ? 0.f : w ? load_any(w, a.w_dtype, c + i) : 1.f;
}

// A row's lanes past d hold zeros.
template <typename T, int V, int LP, int HP>
__global__ __launch_bounds__(kQkThreads) void k_qk_rope(QkRope a) {
  const int c = threadIdx.x % LP * V;
  const Share s = share_of(a, blockIdx.x, HP, kQkThreads / LP);
  const long long tok = s.tok0 + threadIdx.x / LP;
  if (tok >= (long long)a.B * a.n) return;        // the LP lanes of a row leave together
  const int b = (int)(tok / a.n), t = (int)(tok - (long long)b * a.n);
  const bool there = c < a.d;
  const int hop = (a.rot / 2) % V == 0 ? a.rot / 2 / V : 0;
  const Rows& rows = s.key ? a.k : a.q;
  const T* x = static_cast<const T*>(rows.p) + b * rows.bs + t * rows.ts + (size_t)s.h0 * a.d + c;
  T* y = static_cast<T*>(s.key ? a.ko : a.qo) + (((size_t)b * (s.key ? a.Hk : a.H) + s.h0) * a.n + t) * a.d + c;
  Raw<T, V> in[HP];
#pragma unroll
  for (int k = 0; k < HP; ++k) {
    in[k].zero();
    if (there) in[k].load(x + (size_t)min(k, s.heads - 1) * a.d);
  }
  // out_i = r (x_i w_i c_i + x_j w_j s_i), j the pair's other element
  float own[V], pair[V];
  {
    float w[V], wo[V];
    weight<V>(a, s.key, c, there, w);
    angles<V>(a, b, t, c, own, pair);
    Raw<float, V> wr;
#pragma unroll
    for (int i = 0; i < V; ++i) wr.w[i] = __float_as_uint(w[i]);
    others<float, V>(a, c, hop, wr, wo);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      own[i] *= w[i];
      pair[i] *= wo[i];
    }
  }
#pragma unroll
  for (int k = 0; k < HP; ++k) {
    float o[V], ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) ss += in[k].at(i) * in[k].at(i);
    const float r = 1.f / sqrtf(row_sum<LP>(ss) / a.d + a.eps);
    others<T, V>(a, c, hop, in[k], o);
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = r * (in[k].at(i) * own[i] + (c + i < a.rot ? o[i] * pair[i] : 0.f));
    if (there && k < s.heads) store_vec<T, V>(y + (size_t)k * a.n * a.d, o);
  }
}

// Gradients.  Blocks walk the shares of one kind by the grid's stride; a
// thread keeps its lane's dimensions through all of them, so the weight's
// gradient is summed in registers, then over the block's rows in a fixed
// order, a row of partials [d] a block; k_qk_sum adds the rows of each kind.
constexpr int kQkBackBlocks = 1024;   // at most, of the two kinds together

template <typename T, int V, int LP, int HP>
__global__ __launch_bounds__(kQkThreads) void k_qk_rope_back(QkRope a, int qblocks, float* __restrict__ part) {
  constexpr int RB = kQkThreads / LP;
  const int c = threadIdx.x % LP * V;
  const bool there = c < a.d, key = (int)blockIdx.x >= qblocks;
  const int hop = (a.rot / 2) % V == 0 ? a.rot / 2 / V : 0;
  const int nb = key ? gridDim.x - qblocks : qblocks, me = key ? blockIdx.x - qblocks : blockIdx.x;
  const int heads = key ? a.Hk : a.H, groups = (heads + HP - 1) / HP;
  const long long toks = (long long)a.B * a.n, units = (toks + RB - 1) / RB * groups;
  const Rows& rows = key ? a.k : a.q;
  float dw[V], w[V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = 0.f;
  weight<V>(a, key, c, there, w);
  for (long long unit = me; unit < units; unit += nb) {
    const int h0 = (int)(unit % groups) * HP;
    const long long tok = unit / groups * RB + threadIdx.x / LP;
    if (tok >= toks) continue;
    const int b = (int)(tok / a.n), t = (int)(tok - (long long)b * a.n), last = min(HP, heads - h0) - 1;
    const T* x = static_cast<const T*>(rows.p) + b * rows.bs + t * rows.ts + (size_t)h0 * a.d + c;
    const T* g = static_cast<const T*>(key ? a.gk : a.gq) + (((size_t)b * heads + h0) * a.n + t) * a.d + c;
    T* dx = static_cast<T*>(key ? a.dk : a.dq) + (((size_t)b * a.n + t) * heads + h0) * a.d + c;
    Raw<T, V> in[HP], up[HP];
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      in[k].zero();
      up[k].zero();
      if (there) {
        in[k].load(x + (size_t)min(k, last) * a.d);
        up[k].load(g + (size_t)min(k, last) * a.n * a.d);
      }
    }
    float cs[V], sn[V];
    angles<V>(a, b, t, c, cs, sn);
#pragma unroll
    for (int k = 0; k < HP; ++k) {
      // u: the gradient turned back, by the negative angle
      float u[V], ss = 0.f, dot = 0.f;
      others<T, V>(a, c, hop, up[k], u);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u[i] = up[k].at(i) * cs[i] - (c + i < a.rot ? u[i] * sn[i] : 0.f);
        ss += in[k].at(i) * in[k].at(i);
        dot += u[i] * w[i] * in[k].at(i);
      }
      const float r = 1.f / sqrtf(row_sum<LP>(ss) / a.d + a.eps);
      const float mean = row_sum<LP>(dot) / a.d * r;      // r^3 would overflow for rows below 1e-12
      if (there && k <= last) {
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float xhat = in[k].at(i) * r;
          o[i] = r * (u[i] * w[i] - xhat * mean);
          dw[i] += u[i] * xhat;
        }
        store_vec<T, V>(dx + (size_t)k * a.d, o);
      }
    }
  }
  __shared__ float red[RB][LP * V + 1];
#pragma unroll
  for (int i = 0; i < V; ++i) red[threadIdx.x / LP][c + i] = dw[i];
  __syncthreads();
  for (int e = threadIdx.x; e < a.d; e += kQkThreads) {
    float s = 0.f;
    for (int r = 0; r < RB; ++r) s += red[r][e];
    part[(size_t)blockIdx.x * a.d + e] = s;
  }
}

// part [blocks][d], the queries' qblocks first -> the weights' gradients.  grid (columns, kinds).
constexpr int kQkSumRows = 64, kQkSumCols = 16;
__global__ __launch_bounds__(kQkSumRows * kQkSumCols) void k_qk_sum(QkRope a, const float* __restrict__ part, int qblocks,
                                                                    int blocks) {
  __shared__ float red[kQkSumRows][kQkSumCols];
  const int cl = threadIdx.x % kQkSumCols, rg = threadIdx.x / kQkSumCols, col = blockIdx.x * kQkSumCols + cl;
  const bool key = blockIdx.y != 0;
  float s = 0.f;
  if (col < a.d)
    for (int r = (key ? qblocks : 0) + rg; r < (key ? blocks : qblocks); r += kQkSumRows) s += part[(size_t)r * a.d + col];
  red[rg][cl] = s;
  __syncthreads();
  if (rg != 0 || col >= a.d) return;
  for (int r = 1; r < kQkSumRows; ++r) s += red[r][cl];
  void* to = key ? a.dkw : a.dqw;
  if (to) store_any(to, a.w_dtype, col, s);
}

template <typename T, int V, int LP, int HP>
hipError_t launch(const QkRope& a, hipStream_t s) {
  constexpr int RB = kQkThreads / LP;
  const long long tb = ((long long)a.B * a.n + RB - 1) / RB;
  const int gq = (a.H + HP - 1) / HP, gk = (a.Hk + HP - 1) / HP;
  return HLA_TIMED("qk_norm_rope", (k_qk_rope<T, V, LP, HP>), dim3((unsigned)(tb * (gq + gk))), dim3(kQkThreads), 0, s, a);
}

template <typename T, int V, int LP, int HP>
hipError_t launch_back(const QkRope& a, float* part, hipStream_t s) {
  constexpr int RB = kQkThreads / LP;
  const long long tb = ((long long)a.B * a.n + RB - 1) / RB;
  const int gq = (a.H + HP - 1) / HP, gk = (a.Hk + HP - 1) / HP;
  // each kind the blocks of its share of the rows
  auto some = [&](int mine) {
    const long long most = (long long)kQkBackBlocks * mine / (gq + gk), units = tb * mine;
    return (int)(units < 1 || most < 1 ? 1 : units < most ? units : most);
  };
  const int qb = some(gq), kb = some(gk);
  const hipError_t e = HLA_TIMED("qk_norm_rope_back", (k_qk_rope_back<T, V, LP, HP>), dim3(qb + kb), dim3(kQkThreads), 0, s,
                                 a, qb, part);
  if (e != hipSuccess || (!a.dqw && !a.dkw)) return e;
  return HLA_TIMED("qk_sum", k_qk_sum, dim3((a.d + kQkSumCols - 1) / kQkSumCols, 2), dim3(kQkSumRows * kQkSumCols), 0, s, a,
                   part, qb, qb + kb);
}

// HP heads a thread where that still leaves every CU eight waves, one otherwise (a few tokens).
// Forward eight (a load each), gradients four (two loads each).  Measured, several
// heads against one: 276 and 639 us (2 x 16384 tokens of 64 heads of 128), 97 and 130
// (4 x 4096 of 32 of 64 with gradients); the other way 7.1 and 4.5 us (64 tokens).
constexpr int kQkHeads = 8, kQkBackHeads = 4;
bool several_heads(const QkRope& a, int LP, int HP) {      // in doubles: any sizes may be asked for
  return (double)a.B * a.n * ((double)a.H + a.Hk) * LP / HP >= 256. * 8 * 64;
}
template <typename T, int V, int LP>
hipError_t by_heads(const QkRope& a, float* part, hipStream_t s) {
  if (part)
    return several_heads(a, LP, kQkBackHeads) ? launch_back<T, V, LP, kQkBackHeads>(a, part, s)
                                              : launch_back<T, V, LP, 1>(a, part, s);
  return several_heads(a, LP, kQkHeads) ? launch<T, V, LP, kQkHeads>(a, s) : launch<T, V, LP, 1>(a, s);
}

template <typename T, int V>
hipError_t by_width(const QkRope& a, float* part, hipStream_t s) {
  const int pieces = a.d / V;
  if (pieces <= 4) return by_heads<T, V, 4>(a, part, s);
  if (pieces <= 8) return by_heads<T, V, 8>(a, part, s);
  if (pieces <= 16) return by_heads<T, V, 16>(a, part, s);
  if constexpr (V == 4) {  // d <= 256: at most 32 pieces of eight
    if (pieces > 32) return by_heads<T, V, 64>(a, part, s);
  }
  return by_heads<T, V, 32>(a, part, s);
}

hipError_t by_type(const QkRope& a, float* part, hipStream_t s) {
  return a.dtype == 1 ? by_width<bf16, 8>(a, part, s) : by_width<float, 4>(a, part, s);
}

}  // namespace

hipError_t launch_qk_rope(const QkRope& a, hipStream_t s) { return by_type(a, nullptr, s); }
double qk_rope_threads(const QkRope& a) {
  const int pieces = a.d / (a.dtype == 1 ? 8 : 4);
  int LP = 4;
  while (LP < pieces) LP *= 2;
  const double HP = several_heads(a, LP, kQkHeads) ? kQkHeads : 1, RB = kQkThreads / LP;
  return std::ceil((double)a.B * a.n / RB) * (std::ceil(a.H / HP) + std::ceil(a.Hk / HP)) * kQkThreads;
}
size_t qk_rope_backward_ws(int d) { return sizeof(float) * (kQkBackBlocks + 2) * (size_t)d; }
hipError_t launch_qk_rope_backward(const QkRope& a, void* ws, hipStream_t s) {
  return by_type(a, static_cast<float*>(ws), s);
}

}  // namespace hla
