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

template <bool GELU>
__device__ __forceinline__ float act(float p) {
  if constexpr (GELU)
    return 0.5f * p * (1.f + erff(p * 0.70710678f));
  else
    return p * __builtin_amdgcn_rcpf(1.f + __expf(-p));
}
// act(p) and its derivative
template <bool GELU>
__device__ __forceinline__ void act_both(float p, float& f, float& d) {
  if constexpr (GELU) {
    const float phi = 0.5f * (1.f + erff(p * 0.70710678f));
    f = p * phi;
    d = phi + p * (0.39894228f * __expf(-0.5f * p * p));
  } else {
    const float s = __builtin_amdgcn_rcpf(1.f + __expf(-p));
    f = p * s;
    d = s * (1.f + p * (1.f - s));
  }
}

__device__ __forceinline__ const bf16* token(const Rows& r, int n, long long m) {
  const unsigned b = (unsigned)m / (unsigned)n;
  return static_cast<const bf16*>(r.p) + (size_t)b * r.bs + (size_t)((unsigned)m - b * n) * r.ts;
}

// Workgroups go to the 8 XCDs in turn: each XCD gets neighbouring tiles, in
// groups of kGroup tiles of rows j that pass over the same rows i.
constexpr int kGroup = 4;
__device__ __forceinline__ void tile_of(int ni, int nj, int& i, int& j) {
  const unsigned total = (unsigned)ni * nj, x = blockIdx.x & 7, k = blockIdx.x >> 3;
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

// h, or with BACK dp and du, side by side in rows of 2 F at `both`.
template <typename S, bool GELU, bool BACK>
__global__ __launch_bounds__(S::THREADS) void k_glu(Glu p, bf16* __restrict__ both) {
  extern __shared__ __align__(1024) char lds[];
  const int ni = (p.F + S::OUT - 1) / S::OUT, per = (p.n + S::BJ - 1) / S::BJ;
  int ti, tj;
  tile_of(ni, p.B * per, ti, tj);
  const int f0 = ti * S::OUT, b = tj / per, t0 = (tj - b * per) * S::BJ;
  const bf16* x = static_cast<const bf16*>(p.x.p) + (size_t)b * p.x.bs + (size_t)t0 * p.x.ts;
  f32x4 acc[S::TI][S::TJ] = {};
  tile_products<S>(acc, lds, 0, p.D, [&](int r) {
    if (r >= S::BI) return RowAt{x, (uint32_t)(min(r - S::BI, p.n - 1 - t0) * p.x.ts * 2)};
    const int wi = r / (16 * S::TI), q = r % (16 * S::TI), c = q % (16 * S::HALF);
    const bf16* w = static_cast<const bf16*>(q < 16 * S::HALF ? p.wg : p.wu) + (size_t)f0 * p.D;
    return RowAt{w, (uint32_t)(min(wi * 16 * S::HALF + c, p.F - 1 - f0) * p.D * 2)};
  });
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave % S::WI, wj = wave / S::WI;
  const int f = f0 + wi * 16 * S::HALF + (lane >> 4) * 4 * S::HALF;
#pragma unroll
  for (int j = 0; j < S::TJ; ++j) {
    const int t = t0 + (wj * S::TJ + j) * 16 + (lane & 15);
    if (t >= p.n) continue;
    const size_t m = (size_t)b * p.n + t;
    float o[4 * S::HALF], o2[4 * S::HALF];
    if constexpr (!BACK) {
#pragma unroll
      for (int e = 0; e < 4 * S::HALF; ++e) o[e] = act<GELU>(acc[e / 4][j][e % 4]) * acc[S::HALF + e / 4][j][e % 4];
      store_pieces(static_cast<bf16*>(p.h) + m * p.F, f, p.F, o);
    } else {
      const bf16* dh = static_cast<const bf16*>(p.dh.p) + (size_t)b * p.dh.bs + (size_t)t * p.dh.ts;
#pragma unroll
      for (int q = 0; q < 4 * S::HALF; q += 8) {
        Raw<bf16, 8> g;
        g.zero();
        if (f + q < p.F) g.load(dh + f + q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float a, d;
          act_both<GELU>(acc[(q + e) / 4][j][e % 4], a, d);
          o[q + e] = g.at(e) * acc[S::HALF + (q + e) / 4][j][e % 4] * d;
          o2[q + e] = g.at(e) * a;
        }
      }
      bf16* to = both + m * 2 * p.F;
      store_pieces(to, f, p.F, o);
      store_pieces(to + p.F, f, p.F, o2);
    }
  }
}

// C[j][i] = sum_k A[i][k] B[j][k], a [ni][lda], b [nj][ldb]; rows j of C from `split` on lie at c2.
struct Product {
  const bf16 *a, *b;
  bf16 *c, *c2;
  long long lda, ldb, ldc;
  int I, J, K, split;
};
template <typename S>
__global__ __launch_bounds__(S::THREADS) void k_product(Product p) {
  extern __shared__ __align__(1024) char lds[];
  const int ni = (p.I + S::BI - 1) / S::BI, nj = (p.J + S::BJ - 1) / S::BJ;
  int ti, tj;
  tile_of(ni, nj, ti, tj);
  const int i0 = ti * S::BI, j0 = tj * S::BJ;
  f32x4 acc[S::TI][S::TJ] = {};
  tile_products<S>(acc, lds, 0, p.K, [&](int r) {
    return r < S::BI ? RowAt{p.a + (size_t)i0 * p.lda, (uint32_t)(min(r, p.I - 1 - i0) * p.lda * 2)}
                     : RowAt{p.b + (size_t)j0 * p.ldb, (uint32_t)(min(r - S::BI, p.J - 1 - j0) * p.ldb * 2)};
  });
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave % S::WI, wj = wave / S::WI;
  const int i = i0 + wi * 16 * S::TI + (lane >> 4) * 4 * S::TI;
#pragma unroll
  for (int j = 0; j < S::TJ; ++j) {
    const int row = j0 + (wj * S::TJ + j) * 16 + (lane & 15);
    if (row >= p.J) continue;
    float o[4 * S::TI];
#pragma unroll
    for (int e = 0; e < 4 * S::TI; ++e) o[e] = acc[e / 4][j][e % 4];
    store_pieces(row < p.split ? p.c + (size_t)row * p.ldc : p.c2 + (size_t)(row - p.split) * p.ldc, i, p.I, o);
  }
}

// to[c][at + r] = row(r)[c] for r < R, zeros for r in [R, rows); blocks of 64 x 64.
constexpr int kTr = 64;
__global__ __launch_bounds__(256) void k_transposed(Rows x, int n, int R, int C, int rows, bf16* __restrict__ to,
                                                    long long pitch, long long at) {
  __shared__ uint16_t tile[kTr][kTr + 2];
  const int r0 = blockIdx.x * kTr, c0 = blockIdx.y * kTr;
  for (int e = threadIdx.x; e < kTr * kTr / 8; e += 256) {
    const int r = e / (kTr / 8), c = e % (kTr / 8) * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r0 + r < R && c0 + c < C) v = *reinterpret_cast<const uint4*>(token(x, n, r0 + r) + c0 + c);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) tile[c + i][r] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
  }
  __syncthreads();
  for (int e = threadIdx.x; e < kTr * kTr / 8; e += 256) {
    const int c = e / (kTr / 8), r = e % (kTr / 8) * 8;
    if (c0 + c >= C || r0 + r >= rows) continue;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = tile[c][r + 2 * i] | (uint32_t)tile[c][r + 2 * i + 1] << 16;
    *reinterpret_cast<uint4*>(to + (size_t)(c0 + c) * pitch + at + r0 + r) = make_uint4(w[0], w[1], w[2], w[3]);
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

template <bool GELU, bool BACK>
hipError_t projections(const Glu& given, bf16* both, hipStream_t s) {
  const Glu p = joined(given);
  using S = Tile<8, 4, 2, 4, true>;
  const unsigned tiles = (unsigned)((p.F + S::OUT - 1) / S::OUT) * (unsigned)p.B * (unsigned)((p.n + S::BJ - 1) / S::BJ);
  auto kernel = k_glu<S, GELU, BACK>;
  const hipError_t e = allow_lds(kernel, S::LDS);
  if (e != hipSuccess) return e;
  return HLA_TIMED(BACK ? "glu_gates_back" : "glu", kernel, dim3(tiles), dim3(S::THREADS), S::LDS, s, p, both);
}

hipError_t product(const Product& p, const char* name, hipStream_t s) {
  using S = Tile<8, 4, 2, 4, false>;
  const unsigned tiles = (unsigned)((p.I + S::BI - 1) / S::BI) * (unsigned)((p.J + S::BJ - 1) / S::BJ);
  const hipError_t e = allow_lds(k_product<S>, S::LDS);
  if (e != hipSuccess) return e;
  return HLA_TIMED(name, k_product<S>, dim3(tiles), dim3(S::THREADS), S::LDS, s, p);
}

hipError_t transposed(const Rows& x, int n, int R, int C, int rows, bf16* to, long long pitch, long long at, hipStream_t s) {
  return HLA_TIMED("glu_transposed", k_transposed, dim3((rows + kTr - 1) / kTr, (C + kTr - 1) / kTr), dim3(256), 0, s, x, n, R,
                   C, rows, to, pitch, at);
}

struct Space {
  size_t both, turned, xt, wt, bytes;
  long long pitch;
};
Space space(int B, int n, int D, int F) {
  Space a;
  const size_t M = (size_t)B * n;
  a.pitch = (long long)((M + 7) / 8 * 8);
  a.both = 0;
  a.turned = a.both + M * 2 * F * 2;
  a.xt = a.turned + (size_t)a.pitch * 2 * F * 2;
  a.wt = a.xt + (size_t)a.pitch * D * 2;
  a.bytes = a.wt + (size_t)D * 2 * F * 2;
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
  bf16 *both = reinterpret_cast<bf16*>(w + sp.both), *turned = reinterpret_cast<bf16*>(w + sp.turned);
  bf16 *xt = reinterpret_cast<bf16*>(w + sp.xt), *wt = reinterpret_cast<bf16*>(w + sp.wt);
  const int M = p.B * p.n, F2 = 2 * p.F;
  hipError_t e = p.gelu ? projections<true, true>(p, both, s) : projections<false, true>(p, both, s);
  if (e != hipSuccess) return e;
  const Rows wg{p.wg, 0, p.D}, wu{p.wu, 0, p.D}, b{both, 0, F2};
  if ((e = transposed(wg, p.F, p.F, p.D, p.F, wt, F2, 0, s)) || (e = transposed(wu, p.F, p.F, p.D, p.F, wt, F2, p.F, s)) ||
      (e = product({wt, both, static_cast<bf16*>(p.dx), nullptr, F2, F2, p.D, p.D, M, F2, M}, "glu_dx", s)) ||
      (e = transposed(b, M, M, F2, (int)sp.pitch, turned, sp.pitch, 0, s)) || (e = transposed(p.x, p.n, M, p.D, (int)sp.pitch, xt, sp.pitch, 0, s)))
    return e;
  return product({xt, turned, static_cast<bf16*>(p.dwg), static_cast<bf16*>(p.dwu), sp.pitch, sp.pitch, p.D, p.D, F2,
                  (int)sp.pitch, p.F}, "glu_dw", s);
}

}  // namespace hla
