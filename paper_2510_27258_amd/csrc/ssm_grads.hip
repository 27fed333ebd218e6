// Gradients of the selective state space scan (bf16 inputs), for the upstream
// gradient dy.  With h_t the state after token t, g_t its gradient and u_t =
// dt_t x_t, M_ts = 2^(L_t - L_s):
//   g_t = C_t dy_t^T + 2^(l_{t+1}) g_{t+1}
//   dC_t = h_t dy_t,  dB_t = g_t u_t,  du_t = g_t^T B_t,  dx_t = dt_t du_t + D dy_t
//   d(dt_t) = A da_t + x_t . du_t,     da_t = 2^(l_t) <g_t, h_{t-1}>.
// Over a tile with the state h before it and the gradient g after it:
//   dC_t = 2^(L_t) h dy_t            + sum_{s<=t} M_ts dt_s (dy_t . x_s) B_s
//   dB_s = 2^(Lend - L_s) dt_s g x_s + sum_{t>=s} M_ts dt_s (dy_t . x_s) C_t
//   du_s = 2^(Lend - L_s) g^T B_s    + sum_{t>=s} M_ts (C_t . B_s) dy_t
//   da_r = sum_{t>=r} (R_t - dt_t K_t + E_t) + sum_{s<r} dt_s F_s + 2^(Lend) <g, h>
// with R and K the row and column sums of q_ts = M_ts (C_t . B_s)(dy_t . x_s),
// s < t (R with dt_s), E_t = 2^(L_t) C_t . (h dy_t) and F_s = 2^(Lend - L_s) B_s .
// (g x_s).  All cancellation stays within a tile, between R and K, whose fp32
// terms (the same ones) are summed in fp64: the rounding of an fp32 sum counts
// for every token before it, and d dt_bias was 1.2e-6 off 64 bits instead of 4e-7.
//
// The states before and the gradients after every tile come from two walks
// (ssm_walk.h), one each way, into the workspace: 2 x 4 N P bytes a tile and
// head, which is what bounds the whole.  A workgroup here takes a tile and the
// heads that share its B and C: C B^T is formed once, the heads' M dt V are
// summed before they meet B and C, and dB and dC stay in accumulators over the
// heads.  h and g are kept and enter their products to 24 bits (three pieces):
// dA is a sum of either sign over every token, and with two pieces (2^-17) it
// was 2.6e-6 off 64 bits instead of 1.8e-6, for 1 % of the time.  What is left
// (1.7e-6 on 4 x 4096 tokens, 1.8e-7 with fp32 products on vector units) is an
// offset of one sign, 1e-7 of a tile's terms, that adds up over tokens where
// the terms themselves cancel.  It is there only where h and g take part; fp64
// sums of E, F and <g, h>, exact exponentials or another order of the pieces'
// products hardly change it.
// dx takes g and the weighted scores in one piece, 2^-8 of a term (0.0017 off).
//
// Measured on 4 x 4096 tokens of 16 heads of 64 x 128 (us): the walks both ways
// to the segments' ends 33, their states 89 (268 MB written, 3.0 TB/s), this
// kernel 117 (268 MB of states read; 113 with R and K in fp32; with four waves a
// workgroup of two row blocks each, before its loads were moved ahead, 253), the
// last sums 5.
#include "ssm_walk.h"

namespace hla {
namespace {

constexpr int kGQ = 64;   // Kind<bf16>::Q
constexpr int kGW = 8, kGThreads = 64 * kGW;   // waves

struct GradArgs {
  Rows x, dy, k, q;
  const Step* tab;
  const float *h0, *g1;       // [B H][tiles][N][P]
  const float *A, *D;
  void *dx, *ddt;
  void *dk, *dq;              // bf16 [B, n, G, N], or with hs > 1 fp32 [hs][B, n, G, N]
  float* par;                 // [B H][tiles][3]: dA, dD, d dt_bias
  int B, n, H, P, G, N, tok, tiles, hs, softplus, dt_dtype;
};

template <int PP, int NN>
struct GradLds {
  static constexpr int LDK = ld_of(NN), LDX = ld_of(PP), LDP = ld_of(kGQ);
  uint16_t k[kGQ * LDK], q[kGQ * LDK], g[NN * LDX];
  uint16_t x[kGQ * LDX], dy[kGQ * LDX], p[kGQ * LDP];
  float Lh[kGQ], Ll[kGQ], dt[kGQ], el[kGQ], wq[kGQ];
  double R[2][kGQ], K[4][kGQ];
  float own[kGQ], E[kGW][kGQ], F[kGW][kGQ], one[kGW][2];
};

__device__ __forceinline__ void unpack4(const uint2& u, float (&v)[4]) {
  v[0] = __uint_as_float(u.x << 16);
  v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16);
  v[3] = __uint_as_float(u.y & 0xffff0000u);
}

// Eight waves.  Scores: wave w takes the 16 tokens t of block w / 2 and the
// blocks s of w's parity.  h and g: NN / 16 blocks of 16 rows n, the four
// token blocks dealt to the waves that share one.  dx: PP / 16 blocks of
// columns, the token blocks dealt likewise.
template <int PP, int NN>
__global__ __launch_bounds__(kGThreads, 2) void k_ssm_grads(GradArgs a) {
  using L_ = GradLds<PP, NN>;
  constexpr int LDK = L_::LDK, LDX = L_::LDX, LDP = L_::LDP, KN = NN / 32, KP = PP / 32, TB = 4;
  constexpr int NBT = NN / 16, NT = TB * NBT / kGW;          // token blocks a wave takes of its n block
  constexpr int PBT = PP / 16, PT = TB * PBT / kGW;          // and of its p block
  static_assert(NT >= 1 && PT >= 1, "every wave has a block");
  extern __shared__ __align__(16) char smem[];
  L_& S = *reinterpret_cast<L_*>(smem);
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = 16 * (w % NBT), nt0 = NT * (w / NBT), p0 = 16 * (w % PBT), pt0 = PT * (w / PBT);

  int lin = blockIdx.x;
  const int hs = lin % a.hs; lin /= a.hs;
  const int grp = lin % a.G; lin /= a.G;
  const int tile = lin % a.tiles, b = lin / a.tiles;
  const int share = a.H / a.G, per = (share + a.hs - 1) / a.hs;
  const int head0 = grp * share + hs * per, heads = min(per, share - hs * per);
  const int t0 = tile * kGQ, rows = min(kGQ, a.n - t0);

  const uint16_t* kp = static_cast<const uint16_t*>(a.k.p) + b * a.k.bs + t0 * a.k.ts + (long long)grp * a.N;
  const uint16_t* qp = static_cast<const uint16_t*>(a.q.p) + b * a.q.bs + t0 * a.q.ts + (long long)grp * a.N;
  const uint16_t* xp = static_cast<const uint16_t*>(a.x.p) + b * a.x.bs + t0 * a.x.ts;
  const uint16_t* yp = static_cast<const uint16_t*>(a.dy.p) + b * a.dy.bs + t0 * a.dy.ts;

  using TN = Tile<bf16, NN, kGThreads>;
  using TP = Tile<bf16, PP, kGThreads>;
  TN tn;
  TP tx, ty;
  const uint32_t x1 = TP::first(a.x.ts, a.P, tid), xby = TP::step(a.x.ts);
  const uint32_t y1 = TP::first(a.dy.ts, a.P, tid), yby = TP::step(a.dy.ts);
  Step st{};
  float An = 0.f, Dn = 0.f;
  auto fetch = [&](int head) {
    An = a.A[head];
    Dn = (a.D ? a.D : a.A)[head];
    tx.load(reinterpret_cast<const bf16*>(xp + (long long)head * a.P), rows, (int)a.x.ts * 2, a.P, x1, xby);
    ty.load(reinterpret_cast<const bf16*>(yp + (long long)head * a.P), rows, (int)a.dy.ts * 2, a.P, y1, yby);
    st = a.tab[((size_t)b * a.H + head) * a.tok + t0 + (tid & (kGQ - 1))];
  };
  tn.load(reinterpret_cast<const bf16*>(kp), rows, (int)a.k.ts * 2, a.N, TN::first(a.k.ts, a.N, tid), TN::step(a.k.ts));
  tn.template store<false>(S.k, tid);
  tn.load(reinterpret_cast<const bf16*>(qp), rows, (int)a.q.ts * 2, a.N, TN::first(a.q.ts, a.N, tid), TN::step(a.q.ts));
  tn.template store<false>(S.q, tid);
  // rows n0 + r of the states; each is loaded anew, for the next head, as soon
  // as its pieces are made.  At P > 64 both do not fit the registers beside
  // the pieces: h comes with its head, g once h is in pieces.
  constexpr bool kAhead = PP <= 64;
  // The next head's tiles wait until the states' products are done where those
  // fill the registers (P = N = 128: 20 registers spilled instead of 37, 271 us
  // instead of 310 on 4 x 4096 tokens of 16 heads, 279 since R and K are fp64);
  // elsewhere nothing spills.
  constexpr bool kLate = PP > 64 && NN > 64;
  f32x4 hv[KP][2], gv[KP][2];
  auto rows_of = [&](const float* states, int head, f32x4 (&v)[KP][2]) {
    const int l = opaque(threadIdx.x) & 63;
    const rsrc_t rs = rows_rsrc(states + ((size_t)(b * a.H + head) * a.tiles + tile) * a.N * a.P, (long long)a.N * a.P * 4);
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int c = 32 * k + 8 * (l >> 4);
      const uint32_t off = c < a.P ? (uint32_t)((n0 + (l & 15)) * a.P + c) * 4 : 0x80000000u;   // rows past N lie past the end
#pragma unroll
      for (int i = 0; i < 2; ++i) v[k][i] = __builtin_bit_cast(f32x4, load16(rs, off + 16 * i));
    }
  };
  // the tile's rows of dx: the tokens past the sequence lie past the end
  const rsrc_t dxr = tile_rsrc(static_cast<uint16_t*>(a.dx) + ((size_t)b * a.n + t0) * a.H * a.P, rows * a.H * a.P * 2);
  fetch(head0);
  if (kAhead) {
    rows_of(a.h0, head0, hv);
    rows_of(a.g1, head0, gv);
  }
  lds_barrier();

  // (C B^T)^T of the wave's tokens t, its two blocks of rows s
  const int ts = w / 2, s1 = w & 1;
  f32x4 s_[2], z[2];
  {
    const int l = tid & 63;
    bf16x8 cf[KN];
#pragma unroll
    for (int k = 0; k < KN; ++k) cf[k] = frag(S.q, LDK, 16 * ts, 32 * k, l);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s_[i] = z[i] = zero4();
#pragma unroll
      for (int k = 0; k < KN; ++k) s_[i] = mma(frag(S.k, LDK, 16 * (s1 + 2 * i), 32 * k, l), cf[k], s_[i]);
    }
  }
  f32x4 dk[NT], dq[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) dk[j] = dq[j] = zero4();

#pragma unroll 1
  for (int hh = 0; hh < heads; ++hh) {
    const int head = head0 + hh, bh = b * a.H + head;
    const float Ah = An, Dh = a.D ? Dn : 0.f;
    const int tid = opaque(threadIdx.x), l = tid & 63, r = l & 15, g = l >> 4;
    tx.template store<false>(S.x, tid);
    ty.template store<false>(S.dy, tid);
    {
      const float eh = __shfl(st.Lh, kGQ - 1), el = __shfl(st.Ll, kGQ - 1);
      if (tid < kGQ) {
        S.Lh[tid] = st.Lh;
        S.Ll[tid] = st.Ll;
        S.dt[tid] = st.dt;
        S.el[tid] = exp2_(st.Lh + st.Ll);
        S.wq[tid] = exp2_((eh - st.Lh) + (el - st.Ll));
      }
    }
    if (!kAhead) rows_of(a.h0, head, hv);
    lds_barrier();
    if (!kLate) fetch(min(head + 1, head0 + heads - 1));

    // (dy x^T)^T, the weighted scores for dx, and their sums
    {
      const int t = 16 * ts + r;
      const float Lt = S.Lh[t], Ltl = S.Ll[t];
      bf16x8 yf[KP];
#pragma unroll
      for (int k = 0; k < KP; ++k) yf[k] = frag(S.dy, LDX, 16 * ts, 32 * k, l);
      double rsum = 0.0;
      float diag = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int s0 = 16 * (s1 + 2 * i) + 4 * g;
        f32x4 v = zero4();
#pragma unroll
        for (int k = 0; k < KP; ++k) v = mma(frag(S.x, LDX, 16 * (s1 + 2 * i), 32 * k, l), yf[k], v);
        const f32x4 lh = *reinterpret_cast<const f32x4*>(S.Lh + s0), ll = *reinterpret_cast<const f32x4*>(S.Ll + s0);
        const f32x4 dd = *reinterpret_cast<const f32x4*>(S.dt + s0);
        float p[4], q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = s0 + e <= t;
          const float m = exp2_((Lt - lh[e]) + (Ltl - ll[e]));
          p[e] = in ? m * s_[i][e] : 0.f;
          // q's diagonal has no part in da: left out of the sums that would cancel it
          q[e] = s0 + e < t ? p[e] * v[e] : 0.f;
          z[i][e] += in ? m * v[e] * dd[e] : 0.f;
          rsum += (double)q[e] * (double)dd[e];
          if (s0 + e == t) {
            diag = v[e];
            S.own[t] = p[e] * v[e];
          }
        }
        uint2 o[1];
        pieces4<1>(p, o);
        *reinterpret_cast<uint2*>(S.p + t * LDP + s0) = o[0];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double k = sum_row((double)q[e]);
          if (r == 0) S.K[ts][s0 + e] = k;
        }
      }
      rsum = sum_groups(rsum);
      if (g == 0) S.R[s1][t] = rsum;
      diag = sum_wave(diag);
      if (l == 0) S.one[w][0] = diag;
    }

    // h dy_t and g x_s for the wave's rows n and token blocks
    float zz = 0.f;
    {
      if (kAhead) {
#pragma unroll
        for (int k = 0; k < KP; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) zz += hv[k][i / 4][i % 4] * gv[k][i / 4][i % 4];
      }
      // one after the other, held apart: both operands' pieces at once do not fit the registers
      auto pieces = [&](const f32x4 (&v)[KP][2], bf16x8 (&f)[KP][3]) {
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          float q[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) q[i] = v[k][i / 4][i % 4];
          pieces8<3>(q, f[k]);
        }
      };
      auto times = [&](const bf16x8 (&f)[KP][3], const uint16_t* X, int j) {
        f32x4 c = zero4();
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          const bf16x8 xf = frag(X, LDX, 16 * (nt0 + j), 32 * k, l);
#pragma unroll
          for (int i = 2; i >= 0; --i) c = mma(f[k][i], xf, c);
        }
        return c;
      };
      __builtin_amdgcn_sched_barrier(0);
      bf16x8 hf[KP][3];
      pieces(hv, hf);
      if (kAhead)
        rows_of(a.h0, min(head + 1, head0 + heads - 1), hv);
      else
        rows_of(a.g1, head, gv);
      {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int t = 16 * (nt0 + j) + r;
          const f32x4 c0 = times(hf, S.dy, j);
          const float el = S.el[t];
          float qv[4], e_ = 0.f;
          unpack4(*reinterpret_cast<const uint2*>(S.q + t * LDK + n0 + 4 * g), qv);
#pragma unroll
          for (int i = 0; i < 4; ++i) e_ += qv[i] * c0[i];
          dq[j] += el * c0;
          e_ = sum_groups(el * e_);
          if (g == 0) S.E[w % NBT][t] = e_;
          if (j & 1) __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      {
        if (!kAhead) {
#pragma unroll
          for (int k = 0; k < KP; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              zz += (((float)hf[k][2][i] + (float)hf[k][1][i]) + (float)hf[k][0][i]) * gv[k][i / 4][i % 4];
          __builtin_amdgcn_sched_barrier(0);
        }
        if (nt0 != 0) zz = 0.f;
        bf16x8 gf[KP][3];
        pieces(gv, gf);
        if (kAhead) rows_of(a.g1, min(head + 1, head0 + heads - 1), gv);
#pragma unroll
        for (int k = 0; k < KP; ++k)
          if (nt0 == 0) *reinterpret_cast<uint4*>(S.g + (n0 + r) * LDX + 32 * k + 8 * g) = __builtin_bit_cast(uint4, gf[k][0]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int t = 16 * (nt0 + j) + r;
          const f32x4 b0 = times(gf, S.x, j);
          const float wq = S.wq[t], wd = wq * S.dt[t];
          float kv[4], f_ = 0.f;
          unpack4(*reinterpret_cast<const uint2*>(S.k + t * LDK + n0 + 4 * g), kv);
#pragma unroll
          for (int i = 0; i < 4; ++i) f_ += kv[i] * b0[i];
          dk[j] += wd * b0;
          f_ = sum_groups(wq * f_);
          if (g == 0) S.F[w % NBT][t] = f_;
          if (j & 1) __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (kLate) fetch(min(head + 1, head0 + heads - 1));
    zz = sum_wave(zz);
    if (l == 0) S.one[w][1] = zz;
    lds_barrier();

    // dx^T for the wave's columns p and token blocks
    {
      const int tid = opaque(threadIdx.x), l = tid & 63, r = l & 15, g = l >> 4;
      f32x4 acc[PT];
#pragma unroll
      for (int j = 0; j < PT; ++j) acc[j] = zero4();
#pragma unroll
      for (int k = 0; k < KN; ++k) {
        const bf16x8 gt = frag_tr(S.g, LDX, p0, 32 * k, l);
#pragma unroll
        for (int j = 0; j < PT; ++j) acc[j] = mma(gt, frag(S.k, LDK, 16 * (pt0 + j), 32 * k, l), acc[j]);
      }
#pragma unroll
      for (int j = 0; j < PT; ++j) acc[j] *= S.wq[16 * (pt0 + j) + r];
      // tokens s of block sb need t from 32 (sb / 2) on
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 yt = frag_tr(S.dy, LDX, p0, 32 * ks, l);
#pragma unroll
        for (int j = 0; j < PT; ++j)
          if (pt0 + j < 2 * ks + 2) acc[j] = mma(yt, frag_tr(S.p, LDP, 16 * (pt0 + j), 32 * ks, l), acc[j]);
      }
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        const int s = 16 * (pt0 + j) + r, c = p0 + 4 * g;
        float v[4];
        unpack4(*reinterpret_cast<const uint2*>(S.dy + s * LDX + c), v);
        const float dts = S.dt[s];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = dts * acc[j][e] + Dh * v[e];
        uint2 o[1];
        pieces4<1>(v, o);
        store8(dxr, c < a.P ? (uint32_t)((s * a.H + head) * a.P + c) * 2 : 0x80000000u, o[0]);
      }
    }
    // the gradients of dt and the per-head parameters: one wave, a token a lane
    if (w == (hh & (kGW - 1))) {
      const float dt = S.dt[l], Lend = S.Lh[kGQ - 1] + S.Ll[kGQ - 1];
      const double R = S.R[0][l] + S.R[1][l];
      double K = 0.0;
      float Et = 0.f, Fs = 0.f, hg = 0.f, dD = 0.f;
#pragma unroll
      for (int i = 0; i < TB; ++i) K += S.K[i][l];
#pragma unroll
      for (int i = 0; i < NBT; ++i) {
        Et += S.E[i][l];
        Fs += S.F[i][l];
      }
#pragma unroll
      for (int i = 0; i < kGW; ++i) {
        dD += S.one[i][0];
        hg += S.one[i][1];
      }
      const double back = R - (double)dt * K + Et, ahead = (double)dt * Fs;
      const double upto = sums_to(back), suf = last_lane(upto) - upto + back, pre = sums_to(ahead) - ahead;
      const double da = suf + pre + (double)exp2_(Lend) * hg;
      double d = (double)Ah * da + (K + S.own[l] + Fs);
      if (a.softplus) d *= -expm1f(-dt);
      if (l < rows) store_any(a.ddt, a.dt_dtype, ((size_t)b * a.n + t0 + l) * a.H + head, (float)d);
      const float dA = (float)last_lane(sums_to(l < rows ? dt * da : 0.0)), db = (float)last_lane(sums_to(l < rows ? d : 0.0));
      if (l == 0) {
        float* o = a.par + ((size_t)bh * a.tiles + tile) * 3;
        o[0] = dA;
        o[1] = dD;
        o[2] = db;
      }
    }
    lds_barrier();
  }

  // the tile's own part of dB and dC: the heads' sum z[t][s], in two pieces (16
  // bits; with one dB and dC were 0.0023 off 64 bits instead of the 0.0017 of
  // their own rounding), with C and B.  The second lies where x and dy were.
  static_assert(sizeof(S.x) + sizeof(S.dy) >= sizeof(S.p), "room for the second piece");
  uint16_t* const p2 = reinterpret_cast<uint16_t*>(smem + offsetof(L_, x));
  const int l = opaque(threadIdx.x) & 63, r = l & 15, g = l >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float v[4] = {z[i][0], z[i][1], z[i][2], z[i][3]};
    uint2 o[2];
    pieces4<2>(v, o);
    const int at = (16 * ts + r) * LDP + 16 * (s1 + 2 * i) + 4 * g;
    *reinterpret_cast<uint2*>(S.p + at) = o[0];
    *reinterpret_cast<uint2*>(p2 + at) = o[1];
  }
  lds_barrier();
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const bf16x8 kt = frag_tr(S.k, LDK, n0, 32 * ks, l), qt = frag_tr(S.q, LDK, n0, 32 * ks, l);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int tb = nt0 + j;
      if (tb >= 2 * ks) {
        dq[j] = mma(kt, frag(p2, LDP, 16 * tb, 32 * ks, l), dq[j]);
        dq[j] = mma(kt, frag(S.p, LDP, 16 * tb, 32 * ks, l), dq[j]);
      }
      if (tb < 2 * ks + 2) {
        dk[j] = mma(qt, frag_tr(p2, LDP, 16 * tb, 32 * ks, l), dk[j]);
        dk[j] = mma(qt, frag_tr(S.p, LDP, 16 * tb, 32 * ks, l), dk[j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int t = 16 * (nt0 + j) + r, n = n0 + 4 * g;
    if (t >= rows || n >= a.N) continue;
    const size_t at = (((size_t)b * a.n + t0 + t) * a.G + grp) * a.N + n;
    const float vk[4] = {dk[j][0], dk[j][1], dk[j][2], dk[j][3]}, vq[4] = {dq[j][0], dq[j][1], dq[j][2], dq[j][3]};
    if (a.hs == 1) {
      uint2 o[1];
      pieces4<1>(vk, o);
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.dk) + at) = o[0];
      pieces4<1>(vq, o);
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.dq) + at) = o[0];
    } else {
      const size_t all = (size_t)a.B * a.n * a.G * a.N;
      *reinterpret_cast<float4*>(static_cast<float*>(a.dk) + hs * all + at) = make_float4(vk[0], vk[1], vk[2], vk[3]);
      *reinterpret_cast<float4*>(static_cast<float*>(a.dq) + hs * all + at) = make_float4(vq[0], vq[1], vq[2], vq[3]);
    }
  }
}

// The first H blocks sum a head's parameters over sequences and tiles; the
// others the head subsets' dB and dC, four values a thread.
struct FinishArgs {
  const float* par;
  float *dA, *dD, *db;
  const float *dk, *dq;
  uint16_t *dBm, *dCm;
  size_t all;
  int B, H, tiles, hs;
};
__global__ __launch_bounds__(256) void k_ssm_finish(FinishArgs a) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < a.H) {
    const int head = blockIdx.x;
    double s[3] = {0.0, 0.0, 0.0};
    for (int i = tid; i < a.B * a.tiles; i += 256) {
      const int b = i / a.tiles, tile = i - b * a.tiles;
      const float* p = a.par + (((size_t)b * a.H + head) * a.tiles + tile) * 3;
#pragma unroll
      for (int j = 0; j < 3; ++j) s[j] += p[j];
    }
    __shared__ double red[3][256];
#pragma unroll
    for (int j = 0; j < 3; ++j) red[j][tid] = s[j];
    __syncthreads();
    for (int m = 128; m > 0; m /= 2) {
      if (tid < m)
#pragma unroll
        for (int j = 0; j < 3; ++j) red[j][tid] += red[j][tid + m];
      __syncthreads();
    }
    if (tid == 0) {
      a.dA[head] = (float)red[0][0];
      if (a.dD) a.dD[head] = (float)red[1][0];
      if (a.db) a.db[head] = (float)red[2][0];
    }
    return;
  }
  const size_t i = ((size_t)(blockIdx.x - a.H) * 256 + tid) * 4;
  if (i >= a.all) return;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float* p = j ? a.dq : a.dk;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int h = 0; h < a.hs; ++h) {
      const float4 u = *reinterpret_cast<const float4*>(p + h * a.all + i);
      v[0] += u.x;
      v[1] += u.y;
      v[2] += u.z;
      v[3] += u.w;
    }
    uint2 o[1];
    pieces4<1>(v, o);
    *reinterpret_cast<uint2*>((j ? a.dCm : a.dBm) + i) = o[0];
  }
}

template <int PP, int NN>
hipError_t grads(const GradArgs& a, hipStream_t s) {
  constexpr size_t lds = sizeof(GradLds<PP, NN>);
  static_assert(lds <= 160 * 1024, "fits a CU's LDS");
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_ssm_grads<PP, NN>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  return HLA_TIMED("ssm_grads", (k_ssm_grads<PP, NN>), dim3((unsigned)(a.B * a.tiles * a.G * a.hs)), dim3(kGThreads), lds, s,
                   a);
}
template <int PP>
hipError_t grads_n(const GradArgs& a, hipStream_t s) {
  if (a.N <= 32) return grads<PP, 32>(a, s);
  if (a.N <= 64) return grads<PP, 64>(a, s);
  return grads<PP, 128>(a, s);
}

// Head subsets a group: as many as keep all workgroups in one round, one a CU
// (its registers).  This kernel with subsets and without (us): 35 and 102 for
// 3864 tokens of 16 heads of 64 x 128, 17 and 54 for 2 x 517 of 8; the sums over
// the subsets add 0.3 and 1.5.  Calls: with two workgroups a CU as the aim 336,
// with one 317 (4 x 4096 of 16); 158 workgroups in two subsets 262, in one 248.
int head_subsets(int B, int tiles, int G, int share) {
  const long long wgs = (long long)B * tiles * G;
  long long hs = wgs >= 256 ? 1 : 256 / wgs;
  if (hs > share) hs = share;
  const int per = (int)((share + hs - 1) / hs);
  return (share + per - 1) / per;
}

struct GradWs {
  Step* tab;
  float *par, *ends[2], *segdec[2], *carry[2], *bc[2];
  size_t bytes;
};
GradWs carve(void* ws, int B, int n, int H, int P, int G, int N) {
  const int BH = B * H;
  const SsmPlan p = ssm_plan(BH, n, kGQ);
  const size_t tok = (size_t)(n + 63) / 64 * 64;
  char* c = static_cast<char*>(ws);
  size_t o = 0;
  GradWs r;
  auto take = [&](size_t floats) {
    float* q = reinterpret_cast<float*>(c + o);
    o += align256(sizeof(float) * floats);
    return q;
  };
  r.tab = reinterpret_cast<Step*>(take(4 * tok * BH));
  r.par = take((size_t)p.tiles * BH * 3);
  const int hs = head_subsets(B, p.tiles, G, H / G);
  for (int i = 0; i < 2; ++i) {
    r.segdec[i] = take((size_t)p.segs * BH);
    r.ends[i] = take(p.segs > 1 ? (size_t)p.segs * BH * padded(P) * padded(N) : 0);
    r.carry[i] = take((size_t)BH * p.tiles * N * P);
    r.bc[i] = take(hs > 1 ? (size_t)hs * B * n * G * N : 0);
  }
  r.bytes = o;
  return r;
}

}  // namespace

double ssm_backward_threads(int B, int n, int H, int G) {
  const int tiles = ssm_plan(B * H, n, kGQ).tiles;
  return (double)B * tiles * G * head_subsets(B, tiles, G, H / G) * kGThreads;
}
size_t ssm_backward_ws(int B, int n, int H, int P, int G, int N) { return carve(nullptr, B, n, H, P, G, N).bytes; }

hipError_t launch_ssm_backward(const Ssm& a, void* ws, hipStream_t s) {
  const GradWs c = carve(ws, a.B, a.n, a.H, a.P, a.G, a.N);
  hipError_t e = launch_steps(a, c.tab, kGQ, s);
  if (e != hipSuccess) return e;
  WalkPair pair{};
  for (int i = 0; i < 2; ++i) {
    WalkArgs& w = pair.a[i];
    w.x = i ? a.dy : a.x;
    w.k = i ? a.Cm : a.Bm;
    w.tab = c.tab; w.ends = c.ends[i]; w.segdec = c.segdec[i]; w.carry = c.carry[i];
    w.n = a.n; w.H = a.H; w.P = a.P; w.G = a.G; w.N = a.N; w.tok = (a.n + 63) / 64 * 64;
    w.plan = ssm_plan(a.B * a.H, a.n, kGQ);
    w.rev = i;
  }
  e = walk_all<bf16, kStates, 3>(pair, 2, a.B, s);
  if (e != hipSuccess) return e;

  GradArgs d{};
  d.x = a.x; d.dy = a.dy; d.k = a.Bm; d.q = a.Cm;
  d.tab = c.tab; d.h0 = c.carry[0]; d.g1 = c.carry[1];
  d.A = a.A; d.D = a.D; d.dx = a.dx; d.ddt = a.ddt; d.par = c.par;
  d.B = a.B; d.n = a.n; d.H = a.H; d.P = a.P; d.G = a.G; d.N = a.N; d.tok = (a.n + 63) / 64 * 64;
  d.tiles = pair.a[0].plan.tiles;
  d.hs = head_subsets(a.B, d.tiles, a.G, a.H / a.G);
  d.softplus = a.softplus; d.dt_dtype = a.dt_dtype;
  d.dk = d.hs > 1 ? c.bc[0] : a.dBm;
  d.dq = d.hs > 1 ? c.bc[1] : a.dCm;
  e = a.P <= 32 ? grads_n<32>(d, s) : a.P <= 64 ? grads_n<64>(d, s) : grads_n<128>(d, s);
  if (e != hipSuccess) return e;

  FinishArgs f{};
  f.par = c.par; f.dA = a.dA; f.dD = a.dD; f.db = a.ddt_bias;
  f.dk = c.bc[0]; f.dq = c.bc[1];
  f.dBm = static_cast<uint16_t*>(a.dBm); f.dCm = static_cast<uint16_t*>(a.dCm);
  f.all = d.hs > 1 ? (size_t)a.B * a.n * a.G * a.N : 0;
  f.B = a.B; f.H = a.H; f.tiles = d.tiles; f.hs = d.hs;
  return HLA_TIMED("ssm_finish", k_ssm_finish, dim3((unsigned)(a.H + (f.all / 4 + 255) / 256)), dim3(256), 0, s, f);
}

}  // namespace hla
