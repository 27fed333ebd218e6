// Selective state space scan, a scalar decay a head:
//   dt_t = softplus(raw_t + bias),  h_t = 2^(l_t) h_{t-1} + dt_t B_t x_t^T,
//   l_t = dt_t A log2 e,            y_t = h_t^T C_t + D x_t
// over tiles of Q tokens (64; fp32 inputs 32): with L_t the tile's running sum of l and h the state before the tile,
//   y_t = 2^(L_t) h^T C_t + sum_{s <= t} 2^(L_t - L_s) dt_s (C_t . B_s) x_s + D x_t
//   h  <- 2^(L_end) h + sum_s B_s (2^(L_end - L_s) dt_s x_s)^T.
// Every exponent is a difference within the tile, so nothing overflows for A <= 0.
//
// A head's tiles are cut into segments so that the walks fill the chip: the
// end state of each segment from zero, then one walk a segment from its true
// state, the decayed sum of the earlier ends (Fig. 1C's two levels with a
// scalar decay).  The state stays in MFMA accumulators for the whole walk;
// k_ssm_steps makes each token's dt, L and weights once for all walks.
//
// Measured in bf16 (us): a call over 2 x 16384 tokens of 32 heads of 128 x 128
// 333 to 350, over a prompt of 8000 tokens of 32 heads 113 to 123.  Floors by
// bytes: 108 and 27.  Kernel by kernel under the profiler, where each is slower
// than in the call (their sums exceed it): of the first the ends 95 (seven of
// eight segments), outputs 253, steps 11, sums of the ends 10; of the second 35,
// 75, 5 and 13.
// What bounds it: no one unit.  The outputs' walk of the first keeps vector
// instructions busy 53 % of the time, LDS 61 % (41 % of that conflicts) and the
// matrix cores 25 %; waves wait for memory or barriers 48 % of theirs.  In
// copies of a somewhat slower version (276 us) without loads and stores it took
// 212, without the products 197, without both 107 (staging, weights, barriers):
// two workgroups a CU overlap these only in part.
// Tried and not kept, on calls of the first: half as many waves with twice the columns
// 361 (against 347-353), two tiles of loads ahead for the shorter walks 340
// (340), the update at a higher wave priority 326-340 (332-350).
#include "ssm_walk.h"
#include "profile.h"

namespace hla {
namespace {

int tile_of(int dtype) { return dtype == 1 ? Kind<bf16>::Q : Kind<float>::Q; }

}  // namespace

bool ssm_sizes_ok(int P, int N) { return P >= 16 && P <= 128 && P % 16 == 0 && N >= 16 && N <= 128 && N % 16 == 0; }

struct SsmWs {
  Step* tab;
  float *ends, *segdec;
  size_t bytes;
};
static SsmWs carve(void* ws, int BH, int n, int P, int N, int Q) {
  const SsmPlan p = ssm_plan(BH, n, Q);
  const size_t tok = (size_t)(n + 63) / 64 * 64;
  char* c = static_cast<char*>(ws);
  SsmWs r;
  size_t o = 0;
  r.tab = reinterpret_cast<Step*>(c + o);
  o += align256(sizeof(Step) * tok * BH);
  r.segdec = reinterpret_cast<float*>(c + o);
  o += align256(sizeof(float) * (size_t)p.segs * BH);
  r.ends = reinterpret_cast<float*>(c + o);
  if (p.segs > 1) o += align256(sizeof(float) * (size_t)p.segs * BH * padded(P) * padded(N));
  r.bytes = o;
  return r;
}

size_t ssm_forward_ws(int B, int n, int H, int P, int N, int dtype) {
  return carve(nullptr, B * H, n, P, N, tile_of(dtype)).bytes;
}

template <typename T, int NU>
static hipError_t forward(const Ssm& a, void* ws, hipStream_t s) {
  constexpr int Q = Kind<T>::Q;
  const SsmWs c = carve(ws, a.B * a.H, a.n, a.P, a.N, Q);
  hipError_t e = launch_steps(a, c.tab, Q, s);
  if (e != hipSuccess) return e;
  WalkPair pair{};
  WalkArgs& w = pair.a[0];
  w.x = a.x; w.k = a.Bm; w.q = a.Cm;
  w.D = a.D; w.tab = c.tab; w.ends = c.ends; w.segdec = c.segdec;
  w.state = a.state; w.y = a.y;
  w.n = a.n; w.H = a.H; w.P = a.P; w.G = a.G; w.N = a.N; w.tok = (a.n + 63) / 64 * 64;
  w.plan = ssm_plan(a.B * a.H, a.n, Q);
  return walk_all<T, kOutputs, NU>(pair, 1, a.B, s);
}

// The scaled inputs go into the state in three pieces where the state is an
// output (24 bits: fp32's), in two where only bf16 outputs read it: 323 us for
// 2 x 16384 tokens of 32 heads of 128 x 128, with three pieces 359.
hipError_t launch_ssm_forward(const Ssm& a, void* ws, hipStream_t s) {
  if (a.dtype != 1) return forward<float, 3>(a, ws, s);
  return a.state ? forward<bf16, 3>(a, ws, s) : forward<bf16, 2>(a, ws, s);
}

}  // namespace hla
