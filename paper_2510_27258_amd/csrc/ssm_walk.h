// The tile walk of the selective state space scan (ssm_scan.hip has the
// mathematics and the plan), shared by the outputs and the gradients' states.
#pragma once
#include "ssm_tiles.h"

namespace hla {
namespace {

// What a walk does: the end state of a segment from zero, the outputs, or the
// state before every tile (after every tile, backwards).
// For the gradients' states the accumulators hold the state transposed, four
// neighbours of a row of [N][P] a lane, so that its stores are 16 bytes wide;
// the readout needs it as it is.
enum WalkMode { kEnds = 0, kOutputs = 1, kStates = 2, kEndsOfStates = 3 };
constexpr bool transposed(int mode) { return mode == kStates || mode == kEndsOfStates; }

struct WalkArgs {
  Rows x, k, q;               // x [B, n, H, P]; k, q [B, n, G, N] (backwards: dy and C in x's and k's place)
  const float* D;             // [H] or null
  const Step* tab;            // [B H][tok]
  float* ends;                // [B H][segs] end states in the walk's own order; slot segs - 1: the first state
  float* segdec;              // [B H][segs] decay over a segment
  float* state;               // [B, H, N, P] or null
  void* y;                    // outputs
  float* carry;               // kStates: [B H][tiles][N][P]
  int n, H, P, G, N, tok;
  SsmPlan plan;
  int segs_run;               // segments of this launch
  int summed;                 // ends[s] is the state after segment s
  int rev;                    // from the last tile to the first, weights 2^L
};

// Up to two walks of the same sizes in a launch (the gradients' states, both ways).
struct WalkPair {
  WalkArgs a[2];
};

template <int PP>
struct Waves {
  static constexpr int NW = PP / 16, THR = 64 * NW, CB = PP / 16 / NW;
};

template <typename T, int PP, int NN, int MODE>
struct WalkLds {
  static constexpr int NX = Kind<T>::NX, Q = Kind<T>::Q;
  static constexpr int LDK = ld_of(NN), LDX = ld_of(PP), LDS_ = ld_of(Q);
  uint16_t k[NX * Q * LDK], x[NX * Q * LDX];
  // q in the order of accumulator pairs: the readout takes it with the state's
  // accumulators in 16-byte reads (as two 8-byte ones they met in the banks)
  uint16_t q[MODE == kOutputs ? NX * Q * LDK : 8], s[MODE == kOutputs ? NX * Q * LDS_ : 8];
  float Lh[Q], Ll[Q], dt[Q], w[Q];
  int firstx[PP], firstk[NN], first_all, bad[2];
};

// ends[s] += decay ends[s - 1], s = 1 .. segs - 2: the state after each segment.
// Beyond kOwnSums earlier segments, so that no walk reads more than one; V:
// float4s a slot.  Each walk summing for itself costs the reads of all earlier
// ends.  A call with this launch against one without (us): 111 and 141 with 16
// segments of 32 heads of 128 x 128, 323 and 326 with 8 of 64; at 8 of 64 heads
// of 64 x 128 337 and 331, 36 and 35 with 16 of 8 fp32 heads of 64 x 64: the
// gain where the ends are large is worth the loss where they are small.
constexpr int kOwnSums = 3;
__global__ __launch_bounds__(256) void k_ssm_carry(WalkPair pair, int V) {
  const WalkArgs& a = pair.a[blockIdx.z];
  const int i = blockIdx.x * 256 + threadIdx.x, bh = blockIdx.y, segs = a.plan.segs;
  if (i >= V) return;
  f32x4* e = reinterpret_cast<f32x4*>(a.ends) + (size_t)bh * segs * V + i;
  const float* d = a.segdec + (size_t)bh * segs;
  f32x4 sum = e[0];
  constexpr int U = 8;
  for (int s = 1; s < segs - 1; s += U) {
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < segs - 1) x[u] = e[(size_t)(s + u) * V];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < segs - 1) {
        sum = sum * d[s + u] + x[u];
        e[(size_t)(s + u) * V] = sum;
      }
  }
}

// One workgroup walks one segment of one head; wave w owns 16 CB columns of
// the state, h[n = 16 nb + 4g + i][p = 16 (w CB + cb) + r], in accumulators
// (transposed: h[n = 16 nb + r][p = 16 (w CB + cb) + 4g + i]).
// NU pieces carry the scaled inputs into the state; the readout's rounding
// (one piece of the state and of the scores for bf16 outputs, 2^-8 of each
// term, as large as the output's own rounding; three for fp32) is NX.  Outputs
// are 0.0017 to 0.0018 off 64 bits so; with two pieces of both 0.00166, their
// own rounding alone, for 376 us instead of 341 (2 x 16384 tokens of 32 heads of
// 128 x 128), 125 instead of 120 (8000 tokens) and 335 instead of 329 (4 x 4096
// of 16 of 64 x 128 with gradients).
template <typename T, int PP, int NN, int MODE, int NU>
__global__ __launch_bounds__(Waves<PP>::THR, sizeof(T) == 2 ? (PP == 128 ? 4 : 2) : 1) void k_ssm_walk(WalkPair pair) {
  const WalkArgs& a = pair.a[blockIdx.y];
  const bool REV = a.rev;
  using W = Waves<PP>;
  using L_ = WalkLds<T, PP, NN, MODE>;
  constexpr int NW = W::NW, THR = W::THR, CB = W::CB, NX = L_::NX, Q = L_::Q, NB = NN / 16, KN = NN / 32;
  constexpr int TB = Q / 16, KS = Q / 32, LDK = L_::LDK, LDX = L_::LDX, LDQ = L_::LDS_;
  constexpr int PK = Q * LDK, PX = Q * LDX, PS = Q * LDQ;
  extern __shared__ __align__(16) char smem[];
  L_& S = *reinterpret_cast<L_*>(smem);
  const int tid = threadIdx.x, l = tid & 63, r = l & 15, g = l >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

  // heads of one sequence and segment share k and q: neighbours on one XCD
  const int total = gridDim.x;
  const int lin = total % 8 ? blockIdx.x : (blockIdx.x % 8) * (total / 8) + blockIdx.x / 8;
  const int head = lin % a.H, seg = (lin / a.H) % a.segs_run, b = lin / a.H / a.segs_run;
  const int bh = b * a.H + head, M = a.plan.tiles;
  const int i0 = seg * a.plan.per, i1 = min(M, i0 + a.plan.per);
  const int pw = 16 * CB * w;
  const T* xp = static_cast<const T*>(a.x.p) + b * a.x.bs + (long long)head * a.P;
  const T* kp = static_cast<const T*>(a.k.p) + b * a.k.bs + (long long)(head / (a.H / a.G)) * a.N;
  const T* qp = MODE == kOutputs ? static_cast<const T*>(a.q.p) + b * a.q.bs + (long long)(head / (a.H / a.G)) * a.N
                                 : nullptr;
  const Step* tab = a.tab + (size_t)bh * a.tok;
  // outputs: row r of a 16-token block, columns pw + 4g .. + 3 of a column block
  const int ybytes = a.H * a.P * (int)sizeof(T), ystep = 16 * ybytes;
  char* yp = MODE == kOutputs ? static_cast<char*>(a.y) + ((size_t)b * a.n + (size_t)i0 * Q) * ybytes : nullptr;
  const uint32_t yoff = (uint32_t)((r * a.H * a.P + head * a.P + pw + 4 * g) * (int)sizeof(T));

  Tile<T, NN, THR> tk, tq;
  Tile<T, PP, THR> tx;
  Step st{};
  // bytes of a token's row, and the tile that fetch() will load next
  const int kbytes = (int)a.k.ts * (int)sizeof(T), xbytes = (int)a.x.ts * (int)sizeof(T);
  const int qbytes = MODE == kOutputs ? (int)a.q.ts * (int)sizeof(T) : 0;
  const uint32_t k1 = Tile<T, NN, THR>::first(a.k.ts, a.N, tid), kby = Tile<T, NN, THR>::step(a.k.ts);
  const uint32_t x1 = Tile<T, PP, THR>::first(a.x.ts, a.P, tid), xby = Tile<T, PP, THR>::step(a.x.ts);
  const uint32_t q1 = Tile<T, NN, THR>::first(a.q.ts, a.N, tid), qby = Tile<T, NN, THR>::step(a.q.ts);
  const int first_tile = REV ? M - 1 - i0 : i0, ahead = REV ? -1 : 1;
  const char* knext = reinterpret_cast<const char*>(kp + (long long)first_tile * Q * a.k.ts);
  const char* xnext = reinterpret_cast<const char*>(xp + (long long)first_tile * Q * a.x.ts);
  const char* qnext = reinterpret_cast<const char*>(qp) + (long long)first_tile * Q * qbytes;
  const Step* tnext = tab + (long long)first_tile * Q;
  // no branches here: a wait after one would be for every load in flight
  auto fetch = [&](int i) {
    const int rows = min(Q, a.n - (REV ? M - 1 - i : i) * Q);
    st = tnext[tid & (Q - 1)];
    tk.load(knext, rows, kbytes, a.N, k1, kby);
    tx.load(xnext, rows, xbytes, a.P, x1, xby);
    if (MODE == kOutputs) tq.load(qnext, rows, qbytes, a.N, q1, qby);
    knext += ahead * (long long)(Q * kbytes);
    xnext += ahead * (long long)(Q * xbytes);
    qnext += Q * qbytes;
    tnext += ahead * Q;
  };
  fetch(i0);
  f32x4 h[NB][CB];
  // the [N][P] record of a head
  auto load_state = [&](const float* p) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = 16 * nb + 4 * g + i, c = pw + 16 * cb + r;
          h[nb][cb][i] = n < a.N && c < a.P ? p[n * a.P + c] : 0.f;
        }
  };
  auto store_state = [&](float* p) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = 16 * nb + 4 * g + i, c = pw + 16 * cb + r;
          if (n < a.N && c < a.P) p[n * a.P + c] = h[nb][cb][i];
        }
  };
  auto slot = [&](int s) { return reinterpret_cast<f32x4*>(a.ends) + ((size_t)bh * a.plan.segs + s) * NB * CB * THR; };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) h[nb][cb] = zero4();
  if (MODE == kEnds || MODE == kEndsOfStates) {
    if (MODE == kEnds && seg == 0 && a.state) {
      load_state(a.state + (size_t)bh * a.N * a.P);
      f32x4* to = slot(a.plan.segs - 1);          // the outputs' last segment overwrites a.state
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) to[(nb * CB + cb) * THR + tid] = h[nb][cb];
    }
  } else if (seg == 0) {
    if (MODE == kOutputs && a.state) {
      if (a.plan.segs == 1) {
        load_state(a.state + (size_t)bh * a.N * a.P);
      } else {
        const f32x4* from = slot(a.plan.segs - 1);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) h[nb][cb] = from[(nb * CB + cb) * THR + tid];
      }
    }
  } else {
    // segment 0's end state holds the first state; summed slots (k_ssm_carry) hold all before them
    for (int s = a.summed ? seg - 1 : 0; s < seg; ++s) {
      const float d = a.summed ? 0.f : a.segdec[(size_t)bh * a.plan.segs + s];
      const f32x4* from = slot(s);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) h[nb][cb] = h[nb][cb] * d + from[(nb * CB + cb) * THR + tid];
    }
  }

  auto forget = [&]() {
    for (int c = tid; c < PP; c += THR) S.firstx[c] = Q;
    for (int c = tid; c < NN; c += THR) S.firstk[c] = Q;
    if (tid == 0) S.first_all = Q;
  };
  if (MODE == kOutputs) {
    forget();
    if (tid == 0) S.bad[0] = S.bad[1] = 0;
    __syncthreads();
  }

  const float Dh = MODE == kOutputs && a.D ? a.D[head] : 0.f;
  float segL = 0.f;
  // Everything loaded so far is here: were the state's loads still open where
  // the loop begins, the wait before their first use in it would, on every
  // turn, be one for the tile on its way.
  __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
  for (int i = i0; i < i1; ++i) {
    const int tile = REV ? M - 1 - i : i, t0 = tile * Q, par = i & 1;
    const int tid = opaque(threadIdx.x), l = tid & 63, r = l & 15, g = l >> 4;
    bool bad = tk.template store<MODE == kOutputs>(S.k, tid);
    bad |= tx.template store<MODE == kOutputs>(S.x, tid);
    if (MODE == kOutputs) tq.template store<false, true>(S.q, tid);
    if (tid < Q) {
      S.Lh[tid] = st.Lh;
      S.Ll[tid] = st.Ll;
      S.dt[tid] = st.dt;
      S.w[tid] = REV ? exp2_(st.Lh + st.Ll) : st.w;
    }
    if (MODE == kOutputs && bad) S.bad[par] = 1;
    lds_barrier();
    // An infinite or NaN input spoils the state by itself, its column (x) or
    // its row (k).  The outputs of the tile's earlier tokens it must not reach
    // through a zero weight: it is taken out of the tile, and the outputs and
    // the state that depend on it are set to NaN.
    bool flagged = false;
    if (MODE == kOutputs) {
      flagged = __builtin_amdgcn_readfirstlane(S.bad[par]) != 0;
      if (tid == 0) S.bad[par ^ 1] = 0;
      if (flagged) {
        Tile<T, NN, THR>::mend(S.k, S.firstk, &S.first_all, tid);
        Tile<T, PP, THR>::mend(S.x, S.firstx, nullptr, tid);
        lds_barrier();
      }
    }
    if (i + 1 < i1) fetch(i + 1);

    if (MODE == kStates) {
      const rsrc_t to = tile_rsrc(a.carry + ((size_t)bh * M + tile) * a.N * a.P, a.N * a.P * 4);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const int c = pw + 16 * cb + 4 * g;                    // rows past N lie past the end
          const float v[4] = {h[nb][cb][0], h[nb][cb][1], h[nb][cb][2], h[nb][cb][3]};
          store16(to, c < a.P ? (uint32_t)((16 * nb + r) * a.P + c) * 4 : 0x80000000u, v);
        }
    }

    bf16x8 xf[KS][CB][NX];
    if (MODE == kOutputs) {
      // scores, transposed (rows s, columns t), weighted and stored as s[t][s];
      // blocks above the diagonal ones as far as the products over 32 tokens
      // read them (all of their weights are zeros).  No branches: a wave's
      // loads and products of all its blocks are in flight together.
      auto rows_of = [&](int tb, bf16x8 (&cf)[KN][NX]) {
#pragma unroll
        for (int k = 0; k < KN; ++k) load_frags_plain<NX>(S.q, PK, LDK, 16 * tb, 32 * k, l, cf[k]);
      };
      auto product = [&](int sb, const bf16x8 (&cf)[KN][NX]) {
        f32x4 acc = zero4();
#pragma unroll
        for (int k = 0; k < KN; ++k) {
          bf16x8 bf[NX];
          load_frags<NX>(S.k, PK, LDK, 16 * sb, 32 * k, l, bf);
          mma_pieces<NX, NX>(bf, cf[k], acc);
        }
        return acc;
      };
      auto weigh = [&](int tb, int sb, const f32x4& acc) {
        const int t = 16 * tb + r, s0 = 16 * sb + 4 * g;
        const f32x4 lh = *reinterpret_cast<const f32x4*>(S.Lh + s0), dd = *reinterpret_cast<const f32x4*>(S.dt + s0);
        // both parts for every type: behind one very large step the high parts alone are 2^-24 of L apart
        const f32x4 d = (S.Lh[t] - lh) + (S.Ll[t] - *reinterpret_cast<const f32x4*>(S.Ll + s0));
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = s0 + e <= t ? acc[e] * (exp2_(d[e]) * dd[e]) : 0.f;
        uint2 p[NX];
        pieces4<NX>(v, p);
#pragma unroll
        for (int k = 0; k < NX; ++k) *reinterpret_cast<uint2*>(S.s + k * PS + t * LDQ + s0) = p[k];
      };
      if constexpr (TB == 4 && NW == 4) {
        // twelve blocks over four waves: (3; 0 1) (0; 0), (3; 2 3) (1; 0), (2; 0 1) (1; 1), (2; 2 3) (0; 1)
        const int ta = w < 2 ? 3 : 2, sa = 2 * (w & 1), tb = w == 1 || w == 2 ? 1 : 0, sb = w >> 1;
        bf16x8 ca[KN][NX], cb[KN][NX];
        rows_of(ta, ca);
        rows_of(tb, cb);
        const f32x4 x0 = product(sa, ca), x1 = product(sa + 1, ca), x2 = product(sb, cb);
        weigh(ta, sa, x0);
        weigh(ta, sa + 1, x1);
        weigh(tb, sb, x2);
      } else if constexpr (TB == 4 && NW == 8) {
        // eight waves: the blocks of w's parity of the 16 tokens w / 2
        const int tb = w / 2, sb = w & 1;
        bf16x8 cf[KN][NX];
        rows_of(tb, cf);
        weigh(tb, sb, product(sb, cf));
        if (tb >= 2) weigh(tb, sb + 2, product(sb + 2, cf));
      } else {
        constexpr int WPT = NW > TB ? NW / TB : 1;
        bf16x8 cf[KN][NX];
#pragma unroll
        for (int u0 = 0; u0 < TB * WPT; u0 += NW) {
          const int u = u0 + w, tb = u / WPT;
          if (u < TB * WPT) {
            rows_of(tb, cf);
            for (int sb = u % WPT; sb <= (tb | 1); sb += WPT) weigh(tb, sb, product(sb, cf));
          }
        }
      }
      // the state's part, y^T[p][t] = 2^L_t sum_n h[n][p] q[t][n]
      f32x4 y[TB][CB];
#pragma unroll
      for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) y[tb][cb] = zero4();
#pragma unroll
      for (int k = 0; k < KN; ++k) {
        bf16x8 hf[CB][NX];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) frag_from_acc<NX>(h[2 * k][cb], h[2 * k + 1][cb], hf[cb]);
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
          bf16x8 cf[NX];
          load_frags<NX>(S.q, PK, LDK, 16 * tb, 32 * k, l, cf);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) mma_pieces<NX, NX>(hf[cb], cf, y[tb][cb]);
        }
      }
#pragma unroll
      for (int tb = 0; tb < TB; ++tb) {
        const float e = exp2_(S.Lh[16 * tb + r] + S.Ll[16 * tb + r]);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) y[tb][cb] *= e;
      }
      lds_barrier();
      // the tile's own part, and the outputs
      const int l = opaque(tid) & 63, r = l & 15, g = l >> 4;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) load_frags_tr<NX>(S.x, PX, LDX, pw + 16 * cb, 32 * ks, l, xf[ks][cb]);
      const rsrc_t yr = tile_rsrc(yp, min(Q, a.n - t0) * ybytes);
      yp += Q * ybytes;
#pragma unroll
      for (int tb = 0; tb < TB; ++tb) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          if (2 * ks <= tb) {
            bf16x8 pf[NX];
            load_frags<NX>(S.s, PS, LDQ, 16 * tb, 32 * ks, l, pf);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) mma_pieces<NX, NX>(xf[ks][cb], pf, y[tb][cb]);
          }
        const int t = 16 * tb + r;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const int c = pw + 16 * cb + 4 * g;
#pragma unroll
          for (int k = NX - 1; k >= 0; --k) {
            const uint2 u = *reinterpret_cast<const uint2*>(S.x + k * PX + t * LDX + c);
            y[tb][cb][0] += Dh * __uint_as_float(u.x << 16);
            y[tb][cb][1] += Dh * __uint_as_float(u.x & 0xffff0000u);
            y[tb][cb][2] += Dh * __uint_as_float(u.y << 16);
            y[tb][cb][3] += Dh * __uint_as_float(u.y & 0xffff0000u);
          }
        }
      }
      if (flagged) {
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (16 * tb + r >= min(S.firstx[pw + 16 * cb + 4 * g + e], S.first_all)) y[tb][cb][e] = nan_();
      }
#pragma unroll
      for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const float v[4] = {y[tb][cb][0], y[tb][cb][1], y[tb][cb][2], y[tb][cb][3]};
          const uint32_t off = pw + 16 * cb + 4 * g < a.P ? yoff + (uint32_t)(tb * ystep) + 16 * cb * sizeof(T) : 0x80000000u;
          if constexpr (NX == 1) {
            uint2 p[1];
            pieces4<1>(v, p);
            store8(yr, off, p[0]);
          } else {
            store16(yr, off, v);
          }
        }
    } else {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) load_frags_tr<NX>(S.x, PX, LDX, pw + 16 * cb, 32 * ks, l, xf[ks][cb]);
    }

    // h <- 2^Ltile h + sum_s k_s (w_s x_s)^T
    const float Ltile = S.Lh[Q - 1] + S.Ll[Q - 1], dec = exp2_(Ltile);
    segL += Ltile;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 u[CB][NU];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) scaled<NX, NU>(xf[ks][cb], S.w + 32 * ks + 8 * g, u[cb]);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        bf16x8 bt[NX];
        load_frags_tr<NX>(S.k, PK, LDK, 16 * nb, 32 * ks, l, bt);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          if (ks == 0) h[nb][cb] *= dec;
          if constexpr (transposed(MODE))
            mma_pieces<NU, NX>(u[cb], bt, h[nb][cb]);
          else
            mma_pieces<NX, NU>(bt, u[cb], h[nb][cb]);
        }
      }
    }
    if constexpr (NX == 1) interleave<KS * NB * CB * NU, 3>();
    if (flagged) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (min(S.firstx[pw + 16 * cb + r], S.firstk[16 * nb + 4 * g + e]) < Q) h[nb][cb][e] = nan_();
      lds_barrier();
      forget();
    }
    lds_barrier();
  }

  if (MODE == kEnds || MODE == kEndsOfStates) {
    f32x4* to = slot(seg);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) to[(nb * CB + cb) * THR + tid] = h[nb][cb];
    if (tid == 0) a.segdec[(size_t)bh * a.plan.segs + seg] = exp2_(segL);
  } else if (MODE == kOutputs && a.state && seg == a.plan.segs - 1) {
    store_state(a.state + (size_t)bh * a.N * a.P);
  }
}

template <typename T, int PP, int NN, int MODE, int NU>
hipError_t walk(const WalkPair& a, int count, int B, hipStream_t s) {
  constexpr size_t lds = sizeof(WalkLds<T, PP, NN, MODE>);
  static_assert(lds <= 160 * 1024, "fits a CU's LDS");
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_ssm_walk<T, PP, NN, MODE, NU>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  constexpr const char* name = MODE == kEnds || MODE == kEndsOfStates ? "ssm_ends" : MODE == kOutputs ? "ssm_outputs" : "ssm_states";
  return HLA_TIMED(name, (k_ssm_walk<T, PP, NN, MODE, NU>), dim3((unsigned)(B * a.a[0].H * a.a[0].segs_run), count),
                   dim3(Waves<PP>::THR), lds, s, a);
}

template <typename T, int PP, int MODE, int NU>
hipError_t walk_n(const WalkPair& a, int count, int B, hipStream_t s) {
  if (a.a[0].N <= 32) return walk<T, PP, 32, MODE, NU>(a, count, B, s);
  if (a.a[0].N <= 64) return walk<T, PP, 64, MODE, NU>(a, count, B, s);
  return walk<T, PP, 128, MODE, NU>(a, count, B, s);
}
template <typename T, int MODE, int NU>
hipError_t walk_pn(const WalkPair& a, int count, int B, hipStream_t s) {
  if (a.a[0].P <= 32) return walk_n<T, 32, MODE, NU>(a, count, B, s);
  if (a.a[0].P <= 64) return walk_n<T, 64, MODE, NU>(a, count, B, s);
  return walk_n<T, 128, MODE, NU>(a, count, B, s);
}

// A wave: 64 tokens of one (sequence, head).  Sums in fp64: L reaches the
// hundreds, where fp32 sums would put 1e-5 into the weights of neighbours.
// Measured: 11 us for 2 x 16384 tokens of 32 heads (16.8 MB written), 5.6 for
// 8000 tokens of 32: bound by latency, a wave does one block of 64.
template <int Q>
__global__ __launch_bounds__(256) void k_ssm_steps(Ssm a, Step* __restrict__ tab, int tok) {
  const int wv = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  const int head = wv % a.H, blk = (wv / a.H) % (tok / 64), b = wv / a.H / (tok / 64);
  if (b >= a.B) return;
  const int t = blk * 64 + lane, bh = b * a.H + head;
  float dt = 0.f;
  double la = 0.0;
  if (t < a.n) {
    dt = load_any(a.dt.p, a.dt_dtype, (size_t)(b * a.dt.bs + t * a.dt.ts + head));
    if (a.dt_bias) dt += a.dt_bias[head];
    if (a.softplus) dt = dt > 20.f ? dt : log1pf(expf(dt));
    la = (double)dt * (double)a.A[head] * 1.4426950408889634;
  }
  const double L = sums_to<Q>(la);
  double end = last_lane(L);
  if (Q == 32 && lane < 32) end = last_lane<31>(L);
  Step s;
  s.Lh = (float)L;
  s.Ll = (float)(L - (double)s.Lh);
  s.dt = dt;
  s.w = dt * exp2_((float)(end - L));
  tab[(size_t)bh * tok + t] = s;
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Segments a head: walks for two workgroups a CU, each of at least four tiles.
// 256, 512, 768 and 1024 workgroups (us): 415, 342, 377 and 363 on 2 x 16384
// tokens of 32 heads of 128 x 128; 127, 114, 134 and 141 on 8000 tokens.
inline SsmPlan ssm_plan(int BH, int n, int Q) {
  SsmPlan p;
  p.tiles = (n + Q - 1) / Q;
  int segs = BH >= 512 ? 1 : (512 + BH - 1) / BH;
  if (segs > p.tiles / 4) segs = p.tiles / 4;
  if (segs < 1) segs = 1;
  p.per = (p.tiles + segs - 1) / segs;
  p.segs = (p.tiles + p.per - 1) / p.per;
  return p;
}

inline hipError_t launch_steps(const Ssm& a, Step* tab, int Q, hipStream_t s) {
  const int tok = (a.n + 63) / 64 * 64;
  const long long waves = (long long)a.B * a.H * (tok / 64);
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (Q == 64) return HLA_TIMED("ssm_steps", k_ssm_steps<64>, grid, dim3(256), 0, s, a, tab, tok);
  return HLA_TIMED("ssm_steps", k_ssm_steps<32>, grid, dim3(256), 0, s, a, tab, tok);
}

constexpr int padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }


// The walks of `pair` in full: ends, their sums, then MODE.
template <typename T, int MODE, int NU>
hipError_t walk_all(WalkPair& pair, int count, int B, hipStream_t s) {
  const WalkArgs& a = pair.a[0];
  const int segs = a.plan.segs;
  if (segs > 1) {
    for (int i = 0; i < count; ++i) pair.a[i].segs_run = segs - 1;
    hipError_t e = walk_pn<T, MODE == kStates ? kEndsOfStates : kEnds, NU>(pair, count, B, s);
    if (e != hipSuccess) return e;
    if (segs - 1 > kOwnSums) {
      const int V = padded(a.P) * padded(a.N) / 4;
      e = HLA_TIMED("ssm_carry", k_ssm_carry, dim3((V + 255) / 256, B * a.H, count), dim3(256), 0, s, pair, V);
      if (e != hipSuccess) return e;
      for (int i = 0; i < count; ++i) pair.a[i].summed = 1;
    }
  }
  for (int i = 0; i < count; ++i) pair.a[i].segs_run = segs;
  return walk_pn<T, MODE, NU>(pair, count, B, s);
}

}  // namespace
}  // namespace hla
