// Gated linear recurrence, channel by channel:
//   r = sigmoid(f + fb), i = sigmoid(g + gb), L = -c softplus(decay) r, a = e^L
//   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) i_t x_t,  y_t = h_t
// and its gradients, with l_t = dy_t + a_{t+1} l_{t+1} that of h_t:
//   dL = l (a h_{t-1} - i x a^2 / sqrt(1 - a^2)),  dx = l sqrt(1 - a^2) i,
//   dg = l sqrt(1 - a^2) x i (1 - i),  df = dL L (1 - r),
//   ddecay = sum dL (-c) r sigmoid(decay).
//
// A span of tokens acts on the state as h -> A h + H, and spans join: a thread
// takes S neighbouring tokens of V channels, a wave 64 / LPR such runs below
// one another (LPR lanes a token's CB = V LPR channels), W waves a tile.  Runs
// join by lane moves within a wave and through LDS between waves, then every
// thread goes over its tokens again from its true state, all from registers:
// inputs are read once.  The next tile's loads are in flight meanwhile.  Where
// the channel blocks of all sequences leave CUs empty, sequences are cut into
// segments: a first launch brings each segment's A and H (or, backwards, its
// effect on l), and every segment of the second joins what lies before it.
// Bound by vector instructions (six exponentials, roots and quotients a value, at a
// quarter of the rate) and by the loads in flight of one workgroup a CU, two waves a
// SIMD: 4 x 4096 x 2048 in bf16 82 us, 3.3 TB/s, vector instructions 63 % of the
// time; gradients 128 us, 3.7 TB/s, 75 %.  In fp32 125 and 214 us.
// 1 - a^2 is taken as -expm1(2 L): a state that keeps 0.999 of itself a token
// would lose ten bits of it to the difference.
#include <cmath>
#include <type_traits>

#include "block.h"
#include "lanes.h"
#include "vec.h"

namespace hla {
namespace {

// V values of one token as they lie in memory.
template <typename T, int V>
struct Few {
  static constexpr int N = V * sizeof(T) / 4 ? V * sizeof(T) / 4 : 1;
  uint32_t w[N];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (N == 2) {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      w[0] = u.x;
      w[1] = u.y;
    } else if constexpr (sizeof(T) * V == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = (uint32_t) reinterpret_cast<const uint16_t*>(p)[0] << 16;
    }
  }
  // `off` bytes into a view; zeros outside of it
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t view, uint32_t off) {
    if constexpr (N == 2) {
      const auto u = __builtin_amdgcn_raw_buffer_load_b64(view, off, 0, 0);
      w[0] = u[0];
      w[1] = u[1];
    } else if constexpr (sizeof(T) * V == 4) {
      w[0] = __builtin_amdgcn_raw_buffer_load_b32(view, off, 0, 0);
    } else {
      w[0] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(view, off, 0, 0) << 16;
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4 || V == 1)
      return __uint_as_float(w[i]);
    else
      return __uint_as_float(i ? w[0] & 0xffff0000u : w[0] << 16);
  }
};
template <typename T, int V>
__device__ __forceinline__ Few<T, V> rounded(const float (&v)[V]) {
  Few<T, V> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) r.w[i] = __float_as_uint(v[i]);
  } else if constexpr (V == 2) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    r.w[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[0], v[1]}, b2));
  } else {
    r.w[0] = to_bf16(v[0]);
  }
  return r;
}
template <typename T, int V>
__device__ __forceinline__ void store_few(T* p, const float (&v)[V]) {
  const Few<T, V> r = rounded<T, V>(v);
  if constexpr (sizeof(T) * V == 8)
    *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
  else if constexpr (sizeof(T) * V == 4)
    *reinterpret_cast<uint32_t*>(p) = r.w[0];
  else
    p->bits = (uint16_t)r.w[0];
}
// `off` bytes into a view; nothing outside of it
template <typename T, int V>
__device__ __forceinline__ void store_few(__amdgpu_buffer_rsrc_t view, uint32_t off, const float (&v)[V]) {
  const Few<T, V> r = rounded<T, V>(v);
  if constexpr (sizeof(T) * V == 8) {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64((u2){r.w[0], r.w[1]}, view, off, 0, 0);
  } else if constexpr (sizeof(T) * V == 4) {
    __builtin_amdgcn_raw_buffer_store_b32(r.w[0], view, off, 0, 0);
  } else {
    __builtin_amdgcn_raw_buffer_store_b16((short)r.w[0], view, off, 0, 0);
  }
}

constexpr float kLog2e = 1.44269504f;

// A channel's constants: the gates' arguments in powers of two, -f log2 e - fb log2 e.
struct Channel {
  float k2, k3;   // -c softplus(decay) times log2 e, and times -2
  float fb, gb;   // -bias log2 e
};
__device__ __forceinline__ float softplus(float d) { return fmaxf(d, 0.f) + log1pf(expf(-fabsf(d))); }
__device__ __forceinline__ Channel channel(const Glr& p, int c) {
  const float k = -p.c * softplus(p.decay[c]);
  return {k * kLog2e, -2.f * k, p.fb ? -kLog2e * p.fb[c] : 0.f, p.gb ? -kLog2e * p.gb[c] : 0.f};
}

// sigmoid(v + bias), bias folded in as above
__device__ __forceinline__ float sigm(float v, float bias) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(fmaf(v, -kLog2e, bias)));
}

// 1 - e^-u for 0 <= u <= 1/2: u times the polynomial of degree 5 that meets (1 -
// e^-u) / u at the six Chebyshev points of [0, 1/2], off by at most 3e-9 of it.
__device__ __forceinline__ float one_minus_exp(float u) {
  float s = fmaf(u, -0.00112340425f, 0.00818961393f);
  s = fmaf(u, s, -0.0416300744f);
  s = fmaf(u, s, 0.166662425f);
  s = fmaf(u, s, -0.499999821f);
  return u * fmaf(u, s, 1.f);
}

struct Gates {
  float r, i, a, om;   // om: 1 - a^2
};
__device__ __forceinline__ Gates gates(const Channel& ch, float f, float g) {
  Gates o;
  o.r = sigm(f, ch.fb);
  o.i = sigm(g, ch.gb);
  o.a = __builtin_amdgcn_exp2f(ch.k2 * o.r);
  const float u = ch.k3 * o.r;
  // both are formed and one selected: left to itself the compiler branches
  float series = one_minus_exp(u), difference = fmaf(-o.a, o.a, 1.f);
  asm volatile("" : "+v"(series), "+v"(difference));
  o.om = u <= 0.5f ? series : difference;
  return o;
}

// How a launch is cut: channel blocks, sequences, segments of `tiles` tiles.
struct Cut {
  int blocks, segs, tiles;
};

// A workgroup's place.  Workgroups go to the 8 XCDs in turn; neighbouring
// channel blocks, which share cache lines, are given to one XCD.
struct Spot {
  int c0, b, seg;
};
__device__ __forceinline__ Spot spot(const Cut& cut, int B, int CB) {
  const unsigned total = gridDim.x, x = blockIdx.x & 7, k = blockIdx.x >> 3;
  const unsigned per = total >> 3, more = total & 7;
  const unsigned id = x * per + min(x, more) + k;
  const unsigned rest = id / cut.blocks;
  return {(int)(id - rest * cut.blocks) * CB, (int)(rest % B), (int)(rest / B)};
}

// The maps v -> A v + M of a wave's runs joined: ex* = what the runs before
// (UP) or behind (!UP) this lane's do, all* = the whole wave's, in the lanes of
// its last run in that direction.
template <int LPR, int V, bool UP>
__device__ __forceinline__ void join_wave(const float (&A)[V], const float (&M)[V], float (&exA)[V], float (&exM)[V],
                                          float (&allA)[V], float (&allM)[V]) {
  constexpr int RW = 64 / LPR;
  const int row = (threadIdx.x & 63) / LPR, at = UP ? row : RW - 1 - row;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float a = A[v], m = M[v];
#pragma unroll
    for (int k = 1; k < RW; k *= 2) {
      const float pa = UP ? __shfl_up(a, k * LPR) : __shfl_down(a, k * LPR);
      const float pm = UP ? __shfl_up(m, k * LPR) : __shfl_down(m, k * LPR);
      if (at >= k) {
        m = fmaf(a, pm, m);
        a *= pa;
      }
    }
    allA[v] = a;
    allM[v] = m;
    const float pa = UP ? __shfl_up(a, LPR) : __shfl_down(a, LPR);
    const float pm = UP ? __shfl_up(m, LPR) : __shfl_down(m, LPR);
    exA[v] = at ? pa : 1.f;
    exM[v] = at ? pm : 0.f;
  }
}

// v after the maps of segments [from, to), or backwards from the last one on: eight at a time are loaded together.
template <bool BACK>
__device__ __forceinline__ float joined(const float2* __restrict__ sums, size_t apart, int from, int to, float v) {
  for (int s = 0; s < to - from; s += 8) {
    float2 m[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      m[k] = s + k < to - from ? sums[(size_t)(BACK ? to - 1 - s - k : from + s + k) * apart] : make_float2(1.f, 0.f);
#pragma unroll
    for (int k = 0; k < 8; ++k) v = fmaf(m[k].x, v, m[k].y);
  }
  return v;
}

// [p, p + bytes) from a uniform address on, the bytes cut at 2^31 - 1: no offset here is larger.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t view_of(const void* from, long long bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(from);
  const uint64_t u = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) << 32 |
                     (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p);
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u), (short)0,
                                           __builtin_amdgcn_readfirstlane((int)min(bytes, 0x7fffffffLL)), 0x00020000);
}
constexpr uint32_t kOutside = 1u << 31;

// A thread's S tokens of an input in the tile that is loaded ahead.  A wave's
// tokens are a view from its first one on, which ends with the sequence: tokens
// behind it load as zeros, or as other values of the input where rows overlap.
template <typename T, int V, int S>
struct Ahead {
  Few<T, V> raw[S];
  const T* seq;           // the sequence's token 0
  uint32_t ts, off;       // bytes between tokens; this thread's first token and channel in the view
  __amdgpu_buffer_rsrc_t view;
  __device__ __forceinline__ Ahead(const Rows& r, int b, int c, int row)
      : seq(static_cast<const T*>(r.p) + (size_t)b * r.bs), ts((uint32_t)(r.ts * sizeof(T))),
        off((uint32_t)(row * S * r.ts + c) * (uint32_t)sizeof(T)) {}
  // the wave's tokens from t (uniform) on are next; with !there none
  __device__ __forceinline__ void aim(long long t, int n, int D, bool there) {
    asm volatile("" : "+v"(off));   // the tokens' offsets are formed at their loads, not kept in registers
    const long long tokens = ts / sizeof(T);
    const bool some = there && t < n;
    view = view_of(seq + (some ? t * tokens : 0), some ? ((n - 1 - t) * tokens + D) * (long long)sizeof(T) : 0);
  }
  __device__ __forceinline__ void load(int s) { raw[s].load(view, off + s * ts); }
};

// ---------------------------------------------------------------------------
// Forward.  ENDS: only a segment's A and H, to sums [seg][B][D] (A, H); the
// first segment's launch also keeps the state at `first` [B][D], which the
// last segment of the second launch replaces.
template <typename T, int V, int LPR, int S, int W, bool ENDS>
__global__ __launch_bounds__(64 * W) void k_glr(Glr p, Cut cut, float2* __restrict__ sums, float* __restrict__ first) {
  constexpr int CB = V * LPR, RW = 64 / LPR, TILE = S * RW * W;
  __shared__ float2 join[2][W][CB];
  const Spot at = spot(cut, p.B, CB);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane / LPR, q = lane % LPR * V;
  const bool mine = at.c0 + q < p.D;
  const int c = mine ? at.c0 + q : 0;
  Channel ch[V];
#pragma unroll
  for (int v = 0; v < V; ++v) ch[v] = channel(p, c + v);

  // the state before this segment
  float carry[V], through[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const size_t s0 = (size_t)at.b * p.D + c + v;
    through[v] = 1.f;
    carry[v] = 0.f;
    if constexpr (ENDS) {
      if (at.seg == 0 && wave == 0 && row == 0 && mine) first[s0] = p.state ? p.state[s0] : 0.f;
    } else {
      carry[v] = cut.segs > 1 ? first[s0] : p.state ? p.state[s0] : 0.f;
      carry[v] = joined<false>(sums + s0, (size_t)p.B * p.D, 0, at.seg, carry[v]);
    }
  }

  const long long t_first = (long long)at.seg * cut.tiles * TILE, own = (wave * RW + row) * S;
  const int tiles = (int)min((long long)cut.tiles, (p.n - t_first + TILE - 1) / TILE);
  Ahead<T, V, S> x(p.x, at.b, c, row), f(p.f, at.b, c, row), g(p.g, at.b, c, row);
  auto aim = [&](long long t0, bool there) {
    const long long t = t0 + __builtin_amdgcn_readfirstlane(wave) * RW * S;
    x.aim(t, p.n, p.D, there);
    f.aim(t, p.n, p.D, there);
    g.aim(t, p.n, p.D, there);
  };
  uint32_t out = mine ? (uint32_t)((row * S * p.D + c) * sizeof(T)) : kOutside;   // this thread's first output in its wave's
  aim(t_first, true);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    f.load(s);
    g.load(s);
    x.load(s);
  }
  for (int k = 0; k < tiles; ++k) {
    const long long t0 = t_first + (long long)k * TILE, t = t0 + own, tw = t0 + __builtin_amdgcn_readfirstlane(wave) * RW * S;
    float a[S][V], b[S][V], A[V], H[V];
    asm volatile("" : "+v"(out));
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      H[v] = 0.f;
    }
    // each token's registers take the next tile's token as soon as they are free
    aim(t0 + TILE, k + 1 < tiles);
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates o = gates(ch[v], f.raw[s].at(v), g.raw[s].at(v));
        a[s][v] = o.a;
        b[s][v] = __builtin_amdgcn_sqrtf(o.om) * o.i * x.raw[s].at(v);
        A[v] *= a[s][v];
        H[v] = fmaf(a[s][v], H[v], b[s][v]);
      }
      f.load(s);
      g.load(s);
      x.load(s);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (t0 + TILE > p.n) {       // tokens past the end change nothing
#pragma unroll
      for (int v = 0; v < V; ++v) {
        A[v] = 1.f;
        H[v] = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
          a[s][v] = t + s < p.n ? a[s][v] : 1.f;
          b[s][v] = t + s < p.n ? b[s][v] : 0.f;
          A[v] *= a[s][v];
          H[v] = fmaf(a[s][v], H[v], b[s][v]);
        }
      }
    }
    float exA[V], exH[V], allA[V], allH[V];
    join_wave<LPR, V, true>(A, H, exA, exH, allA, allH);
    if (row == RW - 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) join[k & 1][wave][q + v] = make_float2(allA[v], allH[v]);
    }
    lds_barrier();
    float h[V];
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float2 m = join[k & 1][w][q + v];
        if (w == wave) h[v] = fmaf(exA[v], carry[v], exH[v]);
        carry[v] = fmaf(m.x, carry[v], m.y);
        if constexpr (ENDS) through[v] *= m.x;
      }
    if constexpr (!ENDS) {
      if (p.kept && mine && t < p.n && t % kGlrTile == 0) {
        float* to = p.kept + ((size_t)at.b * ((p.n + kGlrTile - 1) / kGlrTile) + t / kGlrTile) * p.D + c;
#pragma unroll
        for (int v = 0; v < V; ++v) to[v] = h[v];
      }
      // behind the sequence's end, and for lanes behind the last channel, nothing is written
      const auto y = view_of(static_cast<T*>(p.y) + ((size_t)at.b * p.n + min(tw, (long long)p.n)) * p.D,
                             max((p.n - tw) * p.D, 0LL) * (long long)sizeof(T));
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = fmaf(a[s][v], h[v], b[s][v]);
        store_few<T, V>(y, out + s * (uint32_t)(p.D * sizeof(T)), h);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (wave != 0 || row != 0 || !mine) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const size_t s0 = (size_t)at.b * p.D + c + v;
    if constexpr (ENDS)
      sums[(size_t)at.seg * p.B * p.D + s0] = make_float2(through[v], carry[v]);
    else if (p.state && at.seg == cut.segs - 1)
      p.state[s0] = carry[v];
  }
}

// ---------------------------------------------------------------------------
// Gradients.  The walk goes from the last tile to the first; the states before
// its tiles were kept by the forward.  m_t = a_t l_t is what token t hands to
// the one before it: a span acts on it as m -> A m + M.  ENDS: only a
// segment's A and M.  part: the sums of the parameters' gradients over this
// segment, [3][B segs][D], formed in fp64 across a thread's runs.
template <typename T, int V, int LPR, int S, int W, bool ENDS>
__global__ __launch_bounds__(64 * W, 2) void k_glr_back(Glr p, Cut cut, float2* __restrict__ sums, float* __restrict__ part) {
  constexpr int CB = V * LPR, RW = 64 / LPR, TILE = S * RW * W;
  static_assert(TILE % kGlrTile == 0, "a tile begins where a state is kept");
  __shared__ float2 join[2][2][W][CB];
  __shared__ double total[ENDS ? 1 : 3][W][CB];
  const Spot at = spot(cut, p.B, CB);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane / LPR, q = lane % LPR * V;
  const bool mine = at.c0 + q < p.D;
  const int c = mine ? at.c0 + q : 0;
  Channel ch[V];
  float carry[V], through[V];
  double sum[3][V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    ch[v] = channel(p, c + v);
    through[v] = 1.f;
    carry[v] = 0.f;
    sum[0][v] = sum[1][v] = sum[2][v] = 0.;
    if constexpr (!ENDS) {
      carry[v] = joined<true>(sums + (size_t)at.b * p.D + c + v, (size_t)p.B * p.D, at.seg + 1, cut.segs, 0.f);
    }
  }
  const int kept = (p.n + kGlrTile - 1) / kGlrTile;
  const long long t_first = (long long)at.seg * cut.tiles * TILE, own = (wave * RW + row) * S;
  const int tiles = (int)min((long long)cut.tiles, (p.n - t_first + TILE - 1) / TILE);
  const long long t_last = t_first + (long long)(tiles - 1) * TILE;
  Ahead<T, V, S> x(p.x, at.b, c, row), f(p.f, at.b, c, row), g(p.g, at.b, c, row), dy(p.dy, at.b, c, row);
  auto aim = [&](long long t0, bool there) {
    const long long t = t0 + __builtin_amdgcn_readfirstlane(wave) * RW * S;
    f.aim(t, p.n, p.D, there);
    dy.aim(t, p.n, p.D, there);
    if constexpr (!ENDS) {
      x.aim(t, p.n, p.D, there);
      g.aim(t, p.n, p.D, there);
    }
  };
  float start[V];
  auto load_start = [&](long long t0) {
    if constexpr (!ENDS) {
#pragma unroll
      for (int v = 0; v < V; ++v) start[v] = p.kept[((size_t)at.b * kept + t0 / kGlrTile) * p.D + c + v];
    }
  };
  auto load = [&](int s) {
    f.load(s);
    dy.load(s);
    if constexpr (!ENDS) {
      x.load(s);
      g.load(s);
    }
  };
  uint32_t out = mine ? (uint32_t)((row * S * p.D + c) * sizeof(T)) : kOutside;   // this thread's first output in its wave's
  aim(t_last, true);
#pragma unroll
  for (int s = 0; s < S; ++s) load(s);
  load_start(t_last);
  for (int k = tiles - 1; k >= 0; --k) {
    const long long t0 = t_first + (long long)k * TILE, t = t0 + own, tw = t0 + __builtin_amdgcn_readfirstlane(wave) * RW * S;
    const bool whole = t0 + TILE <= p.n;
    asm volatile("" : "+v"(out));
    float a[S][V], r[S][V], in[S][V], inv[S][V], root[S][V], ix[S][V], dys[S][V], A[V], H[V], M[V], st[V];
    // each token's registers take the tile before as soon as they are free
    aim(t0 - TILE, k > 0);
#pragma unroll
    for (int v = 0; v < V; ++v) st[v] = start[v];
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates o = gates(ch[v], f.raw[s].at(v), ENDS ? 0.f : g.raw[s].at(v));
        a[s][v] = o.a;
        dys[s][v] = dy.raw[s].at(v);
        if constexpr (!ENDS) {
          r[s][v] = o.r;
          in[s][v] = o.i;
          // where r = 0 the root is too, and log a / root has the limit 0
          inv[s][v] = __builtin_amdgcn_rsqf(fmaxf(o.om, 1e-36f));
          root[s][v] = o.om * inv[s][v];
          ix[s][v] = o.i * x.raw[s].at(v);
        }
      }
      load(s);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (k > 0) load_start(t0 - TILE);
    if (!whole) {               // tokens past the end change nothing, whatever was loaded for them
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (t + s >= p.n) {
            a[s][v] = 1.f;
            dys[s][v] = 0.f;
            if constexpr (!ENDS) root[s][v] = ix[s][v] = r[s][v] = in[s][v] = 0.f;
          }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      H[v] = M[v] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        A[v] *= a[s][v];
        if constexpr (!ENDS) H[v] = fmaf(a[s][v], H[v], root[s][v] * ix[s][v]);
      }
#pragma unroll
      for (int s = S - 1; s >= 0; --s) M[v] = a[s][v] * (dys[s][v] + M[v]);
    }
    float exA[V], exH[V], bkA[V], bkM[V], all[V], allH[V], allM[V];
    join_wave<LPR, V, false>(A, M, bkA, bkM, all, allM);
    if (row == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) join[k & 1][1][wave][q + v] = make_float2(all[v], allM[v]);
    }
    if constexpr (!ENDS) {
      join_wave<LPR, V, true>(A, H, exA, exH, all, allH);
      if (row == RW - 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) join[k & 1][0][wave][q + v] = make_float2(all[v], allH[v]);
      }
    }
    lds_barrier();
    float h[V], m[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int w = W - 1; w >= 0; --w) {
        const float2 o = join[k & 1][1][w][q + v];
        if (w == wave) m[v] = fmaf(bkA[v], carry[v], bkM[v]);
        carry[v] = fmaf(o.x, carry[v], o.y);
        if constexpr (ENDS) through[v] *= o.x;
      }
      if constexpr (!ENDS) {
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float2 o = join[k & 1][0][w][q + v];
          if (w == wave) h[v] = fmaf(exA[v], st[v], exH[v]);
          st[v] = fmaf(o.x, st[v], o.y);
        }
      }
    }
    if constexpr (!ENDS) {
      float before[S][V], run[3][V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        run[0][v] = run[1][v] = run[2][v] = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
          before[s][v] = h[v];
          h[v] = fmaf(a[s][v], h[v], root[s][v] * ix[s][v]);
        }
      }
      // behind the sequence's end, and for lanes behind the last channel, nothing is written
      auto output = [&](void* to) {
        return view_of(static_cast<T*>(to) + ((size_t)at.b * p.n + min(tw, (long long)p.n)) * p.D,
                       max((p.n - tw) * p.D, 0LL) * (long long)sizeof(T));
      };
      const auto dxs = output(p.dx), dfs = output(p.df), dgs = output(p.dg);
#pragma unroll
      for (int s = S - 1; s >= 0; --s) {
        float dx[V], df[V], dg[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float l = dys[s][v] + m[v], lr = l * root[s][v];
          m[v] = a[s][v] * l;
          // r times the gradient of log a
          const float rL = r[s][v] * m[v] * fmaf(-a[s][v], ix[s][v] * inv[s][v], before[s][v]);
          dx[v] = lr * in[s][v];
          dg[v] = lr * ix[s][v] * (1.f - in[s][v]);
          df[v] = rL * (-0.5f * ch[v].k3) * (1.f - r[s][v]);
          run[0][v] += rL;
          run[1][v] += df[v];
          run[2][v] += dg[v];
        }
        const uint32_t off = out + s * (uint32_t)(p.D * sizeof(T));
        store_few<T, V>(dxs, off, dx);
        store_few<T, V>(dfs, off, df);
        store_few<T, V>(dgs, off, dg);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 3; ++j) sum[j][v] += (double)run[j][v];
    }
  }
  if constexpr (ENDS) {
    if (wave == 0 && row == 0 && mine) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        sums[((size_t)at.seg * p.B + at.b) * p.D + c + v] = make_float2(through[v], carry[v]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int k = LPR; k < 64; k *= 2) sum[j][v] += __shfl_xor(sum[j][v], k);
        if (row == 0) total[j][wave][q + v] = sum[j][v];
      }
    __syncthreads();
    if (wave != 0 || row != 0 || !mine) return;
    const size_t rows = (size_t)p.B * cut.segs, mr = (size_t)at.b * cut.segs + at.seg;
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        double s = 0.;
        for (int w = 0; w < W; ++w) s += total[j][w][q + v];
        if (j == 0) s *= -p.c / (1. + exp(-(double)p.decay[c + v]));
        part[((size_t)j * rows + mr) * p.D + c + v] = (float)s;
      }
  }
}

// ---------------------------------------------------------------------------
// One token a sequence: a thread takes V channels.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_glr_step(Glr p) {
  const unsigned per = (p.D + V - 1) / V;
  for (unsigned long long id = blockIdx.x * 256ull + threadIdx.x; id < (unsigned long long)p.B * per;
       id += gridDim.x * 256ull) {
    const unsigned b = (unsigned)(id / per), c = (unsigned)(id - (unsigned long long)b * per) * V;
    Few<T, V> x, f, g;
    x.load(static_cast<const T*>(p.x.p) + (size_t)b * p.x.bs + c);
    f.load(static_cast<const T*>(p.f.p) + (size_t)b * p.f.bs + c);
    g.load(static_cast<const T*>(p.g.p) + (size_t)b * p.g.bs + c);
    float* state = p.state + (size_t)b * p.D + c;
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Gates o = gates(channel(p, c + v), f.at(v), g.at(v));
      h[v] = fmaf(o.a, state[v], __builtin_amdgcn_sqrtf(o.om) * o.i * x.at(v));
      state[v] = h[v];
    }
    store_few<T, V>(static_cast<T*>(p.y) + (size_t)b * p.D + c, h);
  }
}

// Pairs of channels where every row allows them.
bool pairs(const Glr& p) {
  const unsigned es = p.dtype == 1 ? 2 : 4, mask = 2 * es - 1;
  auto fits = [&](const Rows& r) {
    return !r.p || ((reinterpret_cast<uintptr_t>(r.p) & mask) == 0 && r.bs % 2 == 0 && r.ts % 2 == 0);
  };
  bool ok = p.D % 2 == 0 && fits(p.x) && fits(p.f) && fits(p.g) && fits(p.dy);
  for (const void* q : {(const void*)p.y, (const void*)p.dx, (const void*)p.df, (const void*)p.dg})
    ok = ok && (reinterpret_cast<uintptr_t>(q) & mask) == 0;
  return ok;
}

// Runs and waves of the two walks, and segments at most.  Measured: the backward walk of 4 x 4096 x 2048 with runs of
// 4 in 8 waves 127 us, of 8 in 4 waves 142, of 8 in 8 waves 215 (registers).  The forward's were not compared by figures.
constexpr int kFwdS = 16, kFwdW = 8, kBackS = 4, kBackW = 8, kBackLpr = 16;
constexpr int kMostSegs = 32;

// One launch of `groups` workgroups of `per` tiles each, in us: in rounds of one
// workgroup a CU, a tile `empty` on an empty chip and `full` where every CU has one;
// a launch takes 2 and a round's start 2.  So it is for pairs of channels, which the
// constants were measured with.  Single channels (118 registers at most) fit two
// workgroups a CU and are cut by the same rule, without figures of their own.
float launch_time(long long groups, int per, float empty, float full) {
  const float load = groups < 256 ? groups / 256.f : 1.f;
  return 2.f + (float)((groups + 255) / 256) * (2.f + per * (empty + (full - empty) * load));
}
// f(segments' count, tiles each) of uncut sequences, and of those cut so as to fill the CUs, or half or twice of that.
template <typename F>
void each_cut(long long have, int tiles, F f) {
  f(1, tiles);
  if (have >= 256) return;
  const int fill = (int)(256 / have), more = (int)((255 + have) / have);
  for (int want : {fill, more, 2 * more, more / 2, tiles}) {
    if (want < 2 || want > kMostSegs || want > tiles) continue;
    const int per = (tiles + want - 1) / want;
    f((tiles + per - 1) / per, per);
  }
}

// The forward's lanes a row, 32, 16 or 8 (128, 64 or 32 bytes of bf16), and its cut:
// what promises the shortest time: a tile is 16384 values.
// Measured at 32, 16 and 8 lanes (cut where that fills CUs): 4 x 4096 x 2048 88, 71,
// 92; 8 x 4096 x 4096 253, 282, 347; 1 x 8000 x 4096 100, 128, 95; 1 x 16384 x 1024
// 59, 70, 92; 2 x 12000 x 3000 264, 159, 245; 1 x 2500 x 512 27, 38, 20 (by
// this rule 18); 4 x 2500 x 512 30, 41, 26.
struct Plan {
  int lanes;
  Cut cut;
};
template <int V>
Plan forward_plan(int B, int n, int D) {
  Plan best{};
  float least = 0.f;
  auto consider = [&](int lanes, float full) {
    const int cb = V * lanes, blocks = (D + cb - 1) / cb, tile = kFwdS * (64 / lanes) * kFwdW;
    const int tiles = (int)(((long long)n + tile - 1) / tile);
    const long long have = (long long)blocks * B;
    each_cut(have, tiles, [&](int segs, int per) {
      const float t = launch_time(have * segs, per, 5.f, full) +
                      (segs > 1 ? launch_time(have * (segs - 1), per, 5.f, full) : 0.f);
      if (best.lanes && t >= least) return;
      least = t;
      best = {lanes, {blocks, segs, per}};
    });
  };
  consider(16, 9.f);
  consider(32, 8.f);
  consider(8, 12.f);
  return best;
}
// The gradients' cut: a tile of 128 tokens takes 2.7 to 4, of the ends alone 0.9 to
// 1.3.  Uncut, and cut into 4, 8 and 32: 4 x 12000 x 512 301, 131, 131 and 173; 1 x
// 12000 x 1000 266, -, 67 and 91; 2 x 12000 x 3000 316 uncut, 431 in two.
template <int V>
Cut backward_cut(int B, int n, int D) {
  constexpr int CB = V * kBackLpr, TILE = kBackS * (64 / kBackLpr) * kBackW;
  const int blocks = (D + CB - 1) / CB, tiles = (int)(((long long)n + TILE - 1) / TILE);
  const long long have = (long long)blocks * B;
  Cut best{};
  float least = 0.f;
  each_cut(have, tiles, [&](int segs, int per) {
    const float t = launch_time(have * segs, per, 2.7f, 4.f) +
                    (segs > 1 ? launch_time(have * segs, per, 0.9f, 1.3f) : 0.f);
    if (best.segs && t >= least) return;
    least = t;
    best = {blocks, segs, per};
  });
  return best;
}

template <typename T, int V>
hipError_t forward(const Glr& p, void* ws, hipStream_t s) {
  const Plan plan = forward_plan<V>(p.B, p.n, p.D);
  const Cut cut = plan.cut;
  float* first = static_cast<float*>(ws);
  float2* sums = reinterpret_cast<float2*>(first + (((size_t)p.B * p.D + 3) & ~(size_t)3));
  const unsigned one = (unsigned)cut.blocks * p.B;
  auto run = [&](auto l) {
    constexpr int LPR = decltype(l)::value;
    if (cut.segs > 1) {
      const hipError_t e = HLA_TIMED("glr_ends", (k_glr<T, V, LPR, kFwdS, kFwdW, true>), dim3(one * (cut.segs - 1)),
                                     dim3(64 * kFwdW), 0, s, p, cut, sums, first);
      if (e != hipSuccess) return e;
    }
    return HLA_TIMED("glr", (k_glr<T, V, LPR, kFwdS, kFwdW, false>), dim3(one * cut.segs), dim3(64 * kFwdW), 0, s, p, cut,
                     sums, first);
  };
  return plan.lanes == 32   ? run(std::integral_constant<int, 32>{})
         : plan.lanes == 16 ? run(std::integral_constant<int, 16>{})
                            : run(std::integral_constant<int, 8>{});
}

template <typename T, int V>
hipError_t backward(const Glr& p, void* ws, hipStream_t s) {
  const Cut cut = backward_cut<V>(p.B, p.n, p.D);
  const size_t rows = (size_t)p.B * cut.segs;
  float* part = static_cast<float*>(ws);
  float2* sums = reinterpret_cast<float2*>(part + ((3 * rows * p.D + 3) & ~(size_t)3));
  const unsigned one = (unsigned)cut.blocks * p.B;
  if (cut.segs > 1) {
    const hipError_t e = HLA_TIMED("glr_back_ends", (k_glr_back<T, V, kBackLpr, kBackS, kBackW, true>), dim3(one * cut.segs),
                                   dim3(64 * kBackW), 0, s, p, cut, sums, part);
    if (e != hipSuccess) return e;
  }
  const hipError_t e = HLA_TIMED("glr_back", (k_glr_back<T, V, kBackLpr, kBackS, kBackW, false>), dim3(one * cut.segs),
                                 dim3(64 * kBackW), 0, s, p, cut, sums, part);
  if (e != hipSuccess) return e;
  return launch_column_sums({part, {p.ddecay, p.dfb, p.dgb}, (int)rows, p.D, 0}, s);
}

}  // namespace

size_t glr_forward_ws(int B, int n, int D) {
  const int a = forward_plan<1>(B, n, D).cut.segs, b = forward_plan<2>(B, n, D).cut.segs;
  return sizeof(float) * (size_t)B * D * (2 * (a > b ? a : b) + 1) + 64;
}
size_t glr_backward_ws(int B, int n, int D) {
  const int a = backward_cut<1>(B, n, D).segs, b = backward_cut<2>(B, n, D).segs;
  return sizeof(float) * (size_t)B * D * 5 * (a > b ? a : b) + 64;
}
double glr_threads(int B, int n, int D) {   // of the largest launch: single channels
  const Cut f = forward_plan<1>(B, n, D).cut, b = backward_cut<1>(B, n, D);
  return std::fmax((double)f.blocks * f.segs * kFwdW, (double)b.blocks * b.segs * kBackW) * 64. * B;
}

hipError_t launch_glr_forward(const Glr& p, void* ws, hipStream_t s) {
  if (p.dtype == 1) return pairs(p) ? forward<bf16, 2>(p, ws, s) : forward<bf16, 1>(p, ws, s);
  return pairs(p) ? forward<float, 2>(p, ws, s) : forward<float, 1>(p, ws, s);
}
hipError_t launch_glr_backward(const Glr& p, void* ws, hipStream_t s) {
  if (p.dtype == 1) return pairs(p) ? backward<bf16, 2>(p, ws, s) : backward<bf16, 1>(p, ws, s);
  return pairs(p) ? backward<float, 2>(p, ws, s) : backward<float, 1>(p, ws, s);
}
hipError_t launch_glr_step(const Glr& p, hipStream_t s) {
  const bool two = pairs(p);
  const long long threads = (long long)p.B * ((p.D + two) / (1 + two)), blocks = (threads + 255) / 256;
  const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
  if (p.dtype == 1)
    return two ? HLA_TIMED("glr_step", (k_glr_step<bf16, 2>), grid, block, 0, s, p)
               : HLA_TIMED("glr_step", (k_glr_step<bf16, 1>), grid, block, 0, s, p);
  return two ? HLA_TIMED("glr_step", (k_glr_step<float, 2>), grid, block, 0, s, p)
             : HLA_TIMED("glr_step", (k_glr_step<float, 1>), grid, block, 0, s, p);
}

}  // namespace hla
