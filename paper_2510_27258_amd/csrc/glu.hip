// Gated feed-forward projections: p = x Wg^T, u = x Wu^T, h = act(p) u, both
// products and the gate in one kernel, and their gradients:
//   dp = dh u act'(p), du = dh act(p)       (p and u formed again)
//   dx = dp Wg + du Wu,  dWg = dp^T x,  dWu = du^T x.
// act: SiLU, or GELU by the error function.
#include <cmath>

#include "block.h"
#include "glu_tiles.h"

namespace hla {
namespace {

// The normal distribution up to p and its density.  Its tail, 1/2 erfc(x) with x =
// |p| / sqrt 2, is e^(-x^2) times a function that is close to t = 1 / (1 + 0.375 x):
// taken as t times the polynomial of degree 6 in t that is nearest to it relatively
// over 0 <= x <= 9.3, off by at most 6.4e-7 of it.  Relatively, because far below
// zero GELU is p times the tail itself.  The rounding of x^2 = p^2 / 2 moves e^(-x^2)
// by up to 2e-5 of it at p = -13, where the tail stops being a normal number.
__device__ __forceinline__ void normal(float p, float& below, float& density) {
  const float x = fabsf(p) * 0.70710678f, t = __builtin_amdgcn_rcpf(fmaf(0.375f, x, 1.f)), e = __expf(-x * x);
  float s = fmaf(t, -0.0675478354f, 0.193968460f);
  s = fmaf(t, s, -0.0647979081f);
  s = fmaf(t, s, 0.141530156f);
  s = fmaf(t, s, 0.0833325610f);
  s = fmaf(t, s, 0.107844524f);
  const float tail = e * (t * fmaf(t, s, 0.105669729f));
  below = p < 0.f ? tail : 1.f - tail;
  density = 0.39894228f * e;
}

template <bool GELU>
__device__ __forceinline__ float act(float p) {
  if constexpr (GELU) {
    float below, density;
    normal(p, below, density);
    return p * below;
  } else {
    return p * __builtin_amdgcn_rcpf(1.f + __expf(-p));
  }
}
// act(p) and its derivative
template <bool GELU>
__device__ __forceinline__ void act_both(float p, float& f, float& d) {
  if constexpr (GELU) {
    float below, density;
    normal(p, below, density);
    f = p * below;
    d = fmaf(p, density, below);
  } else {
    const float s = __builtin_amdgcn_rcpf(1.f + __expf(-p));
    f = p * s;
    d = s * (1.f + p * (1.f - s));
  }
}

// Workgroups go to the 8 XCDs in turn: each XCD gets neighbouring tiles, in
// groups of kGroup tiles of rows j that pass over the same rows i.
constexpr int kGroup = 4;
__device__ __forceinline__ void tile_of(unsigned block, int ni, int nj, int& i, int& j) {
  const unsigned total = (unsigned)ni * nj, x = block & 7, k = block >> 3;
  const unsigned per = total >> 3, more = total & 7, id = x * per + min(x, more) + k;
  const unsigned group = id / (kGroup * ni), rest = id - group * kGroup * ni, high = min((unsigned)(nj - group * kGroup), (unsigned)kGroup);
  j = group * kGroup + rest % high;
  i = rest / high;
}

// 4 HALF values of a lane as 16-byte pieces; columns from `at` on, those below `end`.
template <int N>
__device__ __forceinline__ void store_pieces(bf16* row, int at, int end, const float (&v)[N]) {
#pragma unroll
  for (int p = 0; p < N; p += 8) {
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = v[p + e];
    if (at + p < end) store_vec<bf16, 8>(row + at + p, o);
  }
}

// h, or with BACK dp and du, side by side in rows of 2 F at `both`.  A workgroup
// takes every gridDim.x-th tile.  Products and gate in one kernel leave p and u in
// registers: two products by themselves would write and read 8 bytes of each
// output, 0.5 GB or 107 us at 16384 x 4096.
template <typename S, bool GELU, bool BACK>
__global__ __launch_bounds__(S::THREADS) void k_glu(Glu p, bf16* __restrict__ both) {
  extern __shared__ __align__(1024) char lds[];
  const int ni = (p.F + S::OUT - 1) / S::OUT, per = (p.n + S::BJ - 1) / S::BJ;
  const unsigned tiles = (unsigned)ni * p.B * per;
  struct Spot {
    int f0, b, t0;
  };
  auto spot = [&](int n) {
    int ti, tj;
    tile_of(blockIdx.x + n * gridDim.x, ni, p.B * per, ti, tj);
    const int b = tj / per;
    return Spot{ti * S::OUT, b, (tj - b * per) * S::BJ};
  };
  auto at = [&](int n, auto take) {
    const Spot o = spot(n);
    const bf16* x = static_cast<const bf16*>(p.x.p) + (size_t)o.b * p.x.bs + (size_t)o.t0 * p.x.ts;
    const size_t w = (size_t)o.f0 * p.D;
    take(Operand{static_cast<const bf16*>(p.wg) + w, static_cast<const bf16*>(p.wu) + w, p.D, p.F - o.f0},
         Operand{x, nullptr, p.x.ts, p.n - o.t0}, 0, p.D);
  };
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto done = [&](int n, f32x4(&acc)[S::TI][S::TJ]) {
    const int lane = lane_here(), wi = wave % S::WI, wj = wave / S::WI;
    const Spot at = spot(n);
    const int f = at.f0 + wi * 16 * S::HALF + (lane >> 4) * 4 * S::HALF;
    // dh, asked for three rows ahead (4096 x 1024 x 4096 75 us, 79 with a wait a row)
    Raw<bf16, 8> up[3][S::HALF / 2];
    auto ask = [&](int j) {
      const int t = at.t0 + (wj * S::TJ + j) * 16 + (lane & 15);
      const bf16* dh = static_cast<const bf16*>(p.dh.p) + (size_t)at.b * p.dh.bs + (size_t)t * p.dh.ts + f;
#pragma unroll
      for (int q = 0; q < S::HALF / 2; ++q) {
        up[j % 3][q].zero();
        if (t < p.n && f + 8 * q < p.F) up[j % 3][q].load(dh + 8 * q);
      }
    };
    if constexpr (BACK) ask(0), ask(1), ask(2);
#pragma unroll
    for (int j = 0; j < S::TJ; ++j) {
      const int t = at.t0 + (wj * S::TJ + j) * 16 + (lane & 15);
      if (t < p.n) {
        const size_t m = (size_t)at.b * p.n + t;
        float o[4 * S::HALF], o2[4 * S::HALF];
        if constexpr (!BACK) {
#pragma unroll
          for (int e = 0; e < 4 * S::HALF; ++e) o[e] = act<GELU>(acc[e / 4][j][e % 4]) * acc[S::HALF + e / 4][j][e % 4];
          store_pieces(static_cast<bf16*>(p.h) + m * p.F, f, p.F, o);
        } else {
#pragma unroll
          for (int q = 0; q < 4 * S::HALF; q += 8) {
            const Raw<bf16, 8> g = up[j % 3][q / 8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float a, d;
              act_both<GELU>(acc[(q + e) / 4][j][e % 4], a, d);
              o[q + e] = g.at(e) * acc[S::HALF + (q + e) / 4][j][e % 4] * d;
              o2[q + e] = g.at(e) * a;
            }
          }
          if (j + 3 < S::TJ) ask(j + 3);
          bf16* to = both + m * 2 * p.F;
          store_pieces(to, f, p.F, o);
          store_pieces(to + p.F, f, p.F, o2);
        }
      }
    }
  };
  tile_products<S, false>(lds, (int)((tiles - blockIdx.x + gridDim.x - 1) / gridDim.x), at, done);
}

// Up to 16 tokens: the weights' bytes bound it.  A workgroup takes 16 outputs (16
// rows of both weights); its eight waves share out k, read their operands from
// memory to registers, four steps of 32 k at a time, and join in LDS.  16 tokens of
// 2048 x 8192 (67 MB of weights): 15.3 us, 4.4 TB/s; the 128-token tiles 17.4.
constexpr int kFew = 16, kFewWaves = 8, kFewSteps = 4;
template <bool GELU>
__global__ __launch_bounds__(64 * kFewWaves) void k_glu_few(Glu p) {
  __shared__ float sums[kFewWaves][2][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int f0 = blockIdx.x * 16, M = p.B * p.n, token = min(m, M - 1), seq = token / p.n;
  const size_t row = (size_t)min(f0 + m, p.F - 1) * p.D;
  const bf16 *wg = static_cast<const bf16*>(p.wg) + row, *wu = static_cast<const bf16*>(p.wu) + row;
  const bf16* x = static_cast<const bf16*>(p.x.p) + (size_t)seq * p.x.bs + (size_t)(token - seq * p.n) * p.x.ts;
  f32x4 acc[2] = {};
  const int steps = (p.D + 31) / 32, per = (steps + kFewWaves - 1) / kFewWaves, last = min(steps, (wave + 1) * per);
  for (int s = wave * per; s < last; s += kFewSteps) {
    Raw<bf16, 8> a[kFewSteps][2], b[kFewSteps];
#pragma unroll
    for (int i = 0; i < kFewSteps; ++i) {
      const int k = (s + i) * 32 + 8 * g;
      a[i][0].zero();
      a[i][1].zero();
      b[i].zero();
      if (s + i < last && k < p.D) {
        a[i][0].load(wg + k);
        a[i][1].load(wu + k);
        b[i].load(x + k);
      }
    }
#pragma unroll
    for (int i = 0; i < kFewSteps; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i][h]),
                                                         __builtin_bit_cast(bf16x8, b[i]), acc[h], 0, 0, 0);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][h][e][lane] = acc[h][e];
  __syncthreads();
  const int f = threadIdx.x & 15, t = threadIdx.x >> 4, l = (f >> 2) * 16 + t;
  if (t >= M || f0 + f >= p.F) return;
  float v[2] = {0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
    for (int h = 0; h < 2; ++h) v[h] += sums[w][h][f & 3][l];
  static_cast<bf16*>(p.h)[(size_t)t * p.F + f0 + f].bits = to_bf16(act<GELU>(v[0]) * v[1]);
}

// The gradients' products, C[j][i] = sum over one or two spans of k of A[i][k]
// B[j][k].  A has its rows i contiguous, B its rows j (TRJ) or its k.  The spans
// are cut into `cuts` parts of `per` k each (a multiple of 64); a workgroup takes
// one part of a tile, or with one cut all spans of it.  Rows j of C from `split`
// on lie at c2.  With several cuts, sums go to `part` [cuts spans][J][I].
struct Product {
  const bf16 *a[2], *b[2];
  long long lda, ldb;
  bf16 *c, *c2;
  float* part;
  int I, J, K, spans, cuts, per, split;
};
template <typename S>
__global__ __launch_bounds__(S::THREADS) void k_product(Product p) {
  extern __shared__ __align__(1024) char lds[];
  const int ni = (p.I + S::BI - 1) / S::BI, nj = (p.J + S::BJ - 1) / S::BJ;
  int ti, tj;
  tile_of(blockIdx.x, ni, nj, ti, tj);
  const int i0 = ti * S::BI, j0 = tj * S::BJ, z = blockIdx.y, runs = !S::TRJ && p.cuts == 1 && !p.part ? p.spans : 1;
  auto at = [&](int n, auto take) {
    const int span = runs == 2 ? n : z % p.spans, k = z / p.spans * p.per;
    take(Operand{p.a[span] + i0, nullptr, p.lda, p.I - i0},
         Operand{p.b[span] + (S::TRJ ? j0 : (size_t)j0 * p.ldb), nullptr, p.ldb, p.J - j0}, k, min(k + p.per, p.K));
  };
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto done = [&](int n, f32x4(&acc)[S::TI][S::TJ]) {
    const int lane = lane_here(), wi = wave % S::WI, wj = wave / S::WI;
    const int i = i0 + wi * 16 * S::TI + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < S::TJ; ++j) {
      const int row = j0 + (wj * S::TJ + j) * 16 + (lane & 15);
      if (row >= p.J) continue;
      bf16* c = row < p.split ? p.c + (size_t)row * p.I : p.c2 + (size_t)(row - p.split) * p.I;
#pragma unroll
      for (int t = 0; t < S::TI; ++t) {
        const float o[4] = {acc[t][j][0], acc[t][j][1], acc[t][j][2], acc[t][j][3]};
        if (i + 16 * t >= p.I) continue;
        if (p.part)
          store_vec<float, 4>(p.part + ((size_t)z * p.J + row) * p.I + i + 16 * t, o);
        else
          store_vec<bf16, 4>(c + i + 16 * t, o);
      }
    }
  };
  tile_products<S, true>(lds, runs, at, done);
}

// The parts joined in their order: eight values a thread.
__global__ __launch_bounds__(256) void k_joined(Product p) {
  const size_t all = (size_t)p.J * p.I / 8, e = blockIdx.x * 256ull + threadIdx.x;
  if (e >= all) return;
  float s[8] = {};
  const int slabs = p.cuts * p.spans;
  for (int z0 = 0; z0 < slabs; z0 += 4) {
    float v[4][8] = {};
#pragma unroll
    for (int z = 0; z < 4; ++z)
      if (z0 + z < slabs) load_vec<float, 8>(p.part + ((size_t)(z0 + z) * all + e) * 8, v[z]);
#pragma unroll
    for (int z = 0; z < 4; ++z)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += v[z][i];
  }
  const size_t half = (size_t)p.split * p.I / 8;
  store_vec<bf16, 8>(e < half ? p.c + e * 8 : p.c2 + (e - half) * 8, s);
}

// x [B, n, D] with sequences apart -> [B n, D] without gaps, 16 bytes a thread.
__global__ __launch_bounds__(256) void k_packed(Rows x, int B, int n, int D, bf16* __restrict__ to) {
  const size_t all = (size_t)B * n * (D / 8);
  for (size_t e = blockIdx.x * 256ull + threadIdx.x; e < all; e += gridDim.x * 256ull) {
    const size_t m = e / (D / 8);
    const int c = (int)(e - m * (D / 8)) * 8, b = (int)(m / n), t = (int)(m - (size_t)b * n);
    *reinterpret_cast<uint4*>(to + m * D + c) =
        *reinterpret_cast<const uint4*>(static_cast<const bf16*>(x.p) + (size_t)b * x.bs + (size_t)t * x.ts + c);
  }
}

template <typename K>
hipError_t allow_lds(K kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

// Sequences laid one behind the other are one long one: a tile lies in one sequence.
Glu joined(Glu p) {
  auto fits = [&](const Rows& r) { return !r.p || r.bs == (long long)p.n * r.ts; };
  if (p.B == 1) return p;
  if (p.n == 1) {
    p.x.ts = p.x.bs;
    p.dh.ts = p.dh.bs;
  } else if (!fits(p.x) || !fits(p.dh)) {
    return p;
  }
  p.n *= p.B;
  p.B = 1;
  return p;
}

template <typename S>
unsigned tiles_of(const Glu& p) {
  return (unsigned)((p.F + S::OUT - 1) / S::OUT) * (unsigned)p.B * (unsigned)((p.n + S::BJ - 1) / S::BJ);
}

template <typename S, bool GELU, bool BACK>
hipError_t tiled(const Glu& p, bf16* both, hipStream_t s) {
  auto kernel = k_glu<S, GELU, BACK>;
  const hipError_t e = allow_lds(kernel, S::LDS);
  if (e != hipSuccess) return e;
  const unsigned tiles = tiles_of<S>(p), most = 256 * (S::LDS > 81920 ? 1 : 2);
  return HLA_TIMED(BACK ? "glu_gates_back" : "glu", kernel, dim3(tiles < most ? tiles : most), dim3(S::THREADS), S::LDS, s, p,
                   both);
}

// Tiles of 256, 192 and 128 tokens; the last one half as wide, two workgroups a
// CU.  Taken is what promises the shortest time: rounds of one tile a CU times what
// a round took, and what the first one's start and the last one's end took beside
// it, in one unit (16384 x 1024 x 4096: 251, 265 and 299 us; 2001 x 2048 x 5464: 96,
// 85, 95; 2048 x 1024 x 4096: 32, 42, 36; 512 x 2048 x 8192: 46, 41, 34; 128: 42,
// 36, 18).
template <bool GELU, bool BACK>
hipError_t projections(const Glu& given, bf16* both, hipStream_t s) {
  const Glu p = joined(given);
  if constexpr (!BACK) {
    if ((long long)p.B * p.n <= kFew)
      return HLA_TIMED("glu_few", k_glu_few<GELU>, dim3((p.F + 15) / 16), dim3(64 * kFewWaves), 0, s, p);
  }
  using S256 = Tile<8, 4, 2, 4, true, false, false>;
  using S192 = Tile<8, 3, 2, 4, true, false, false>;
  using S128 = Tile<4, 2, 2, 4, true, false, false>;
  auto time = [](unsigned tiles, float round, float rest) { return (tiles + 255) / 256 * round + rest; };
  const float t256 = time(tiles_of<S256>(p), 31.5f, 12), t192 = time(tiles_of<S192>(p), 23, 14),
              t128 = time(tiles_of<S128>(p), 8.65f, 10);
  if (t128 < t192 && t128 < t256) return tiled<S128, GELU, BACK>(p, both, s);
  return t192 < t256 ? tiled<S192, GELU, BACK>(p, both, s) : tiled<S256, GELU, BACK>(p, both, s);
}

using DxTile = Tile<8, 4, 2, 4, false, true, false>;
using DwTile = Tile<8, 4, 2, 4, false, true, true>;

// How a product's sums over `spans` spans of K are cut: `cuts` parts of `per` k of
// each, in slabs of their own that are joined behind, or (slabs = 0) one workgroup
// a tile for all.  Taken is what promises the shortest time, in us: rounds of one
// workgroup a CU, at 1.5 a step of 64 k and 6 for its start and end; the join takes
// 4, 0.3 a slab and their bytes written and read at 6 TB/s.  Measured with parts of
// 512 k at least, cut over idle CUs alone, and by this rule, the join with it: 22 x
// 200 from 696 outputs 31.7 and 12.1 us, 1124 x 176 from 720 35.5 and 17.9, 512 x
// 2048 from 8192 52.2 and 52.1.
struct Cuts {
  int cuts, per, slabs;
};
template <typename S>
Cuts cuts_of(long long I, long long J, int K, int spans) {
  const long long tiles = ((I + S::BI - 1) / S::BI) * ((J + S::BJ - 1) / S::BJ);
  auto time = [&](long long groups, long long k) {
    const long long steps = (k + 63) / 64;
    return (double)((groups + 255) / 256) * (1.5 * (steps > 2 ? steps : 2) + 6);
  };
  Cuts best{1, K, 0};
  double least = time(tiles, (long long)spans * K);
  for (int c = spans > 1 ? 1 : 2; c <= 64 && (c == 1 || K / c >= 128); ++c) {
    const int per = (int)((((long long)K + c - 1) / c + 63) / 64 * 64), cuts = (int)(((long long)K + per - 1) / per);
    const double t = time(tiles * spans * cuts, per) + 4 + cuts * spans * (0.3 + (double)I * (double)J * 8 / 6e6);
    if (t < least) {
      least = t;
      best = {cuts, per, cuts * spans};
    }
  }
  return best;
}

template <typename S>
hipError_t product(Product p, float* part, const char* name, hipStream_t s) {
  const Cuts c = cuts_of<S>(p.I, p.J, p.K, p.spans);
  p.cuts = c.cuts;
  p.per = c.per;
  p.part = c.slabs ? part : nullptr;
  const unsigned tiles = (unsigned)((p.I + S::BI - 1) / S::BI) * (unsigned)((p.J + S::BJ - 1) / S::BJ);
  hipError_t e = allow_lds(k_product<S>, S::LDS);
  if (e != hipSuccess) return e;
  e = HLA_TIMED(name, k_product<S>, dim3(tiles, c.slabs ? c.slabs : 1), dim3(S::THREADS), S::LDS, s, p);
  if (e != hipSuccess || !p.part) return e;
  return HLA_TIMED("glu_joined", k_joined, dim3((unsigned)(((size_t)p.I * p.J / 8 + 255) / 256)), dim3(256), 0, s, p);
}

struct Space {
  size_t both, x, part, bytes;
};
Space space(int B, int n, int D, int F) {
  Space a;
  const size_t M = (size_t)B * n;
  const Cuts dx = cuts_of<DxTile>(D, M, F, 2), dw = cuts_of<DwTile>(D, 2LL * F, (int)M, 1);
  const size_t px = M * D * 4 * dx.slabs, pw = (size_t)2 * F * D * 4 * dw.slabs;
  a.both = 0;
  a.x = a.both + M * 2 * F * 2;
  a.part = a.x + (B > 1 && n > 1 ? M * D * 2 : 0);
  a.bytes = a.part + (px > pw ? px : pw);
  return a;
}

}  // namespace

hipError_t launch_glu(const Glu& p, hipStream_t s) {
  return p.gelu ? projections<true, false>(p, nullptr, s) : projections<false, false>(p, nullptr, s);
}

size_t glu_backward_ws(int B, int n, int D, int F) { return space(B, n, D, F).bytes; }
hipError_t launch_glu_backward(const Glu& p, void* ws, hipStream_t s) {
  const Space sp = space(p.B, p.n, p.D, p.F);
  char* w = static_cast<char*>(ws);
  bf16* both = reinterpret_cast<bf16*>(w + sp.both);
  float* part = reinterpret_cast<float*>(w + sp.part);
  const int M = p.B * p.n, F2 = 2 * p.F;
  hipError_t e = p.gelu ? projections<true, true>(p, both, s) : projections<false, true>(p, both, s);
  if (e != hipSuccess) return e;
  const bf16 *wg = static_cast<const bf16*>(p.wg), *wu = static_cast<const bf16*>(p.wu);
  Product dx{};
  dx.a[0] = wg, dx.a[1] = wu, dx.lda = p.D;
  dx.b[0] = both, dx.b[1] = both + p.F, dx.ldb = F2;
  dx.c = static_cast<bf16*>(p.dx);
  dx.I = p.D, dx.J = dx.split = M, dx.K = p.F, dx.spans = 2;
  if ((e = product<DxTile>(dx, part, "glu_dx", s))) return e;
  // the tokens as one sequence
  Rows x = joined(p).x;
  if (joined(p).B > 1) {
    bf16* packed = reinterpret_cast<bf16*>(w + sp.x);
    if ((e = HLA_TIMED("glu_packed", k_packed, dim3(2048), dim3(256), 0, s, p.x, p.B, p.n, p.D, packed))) return e;
    x = {packed, 0, p.D};
  }
  Product dw{};
  dw.a[0] = static_cast<const bf16*>(x.p), dw.lda = x.ts;
  dw.b[0] = both, dw.ldb = F2;
  dw.c = static_cast<bf16*>(p.dwg), dw.c2 = static_cast<bf16*>(p.dwu);
  dw.I = p.D, dw.J = F2, dw.split = p.F, dw.K = M, dw.spans = 1;
  return product<DwTile>(dw, part, "glu_dw", s);
}

}  // namespace hla
