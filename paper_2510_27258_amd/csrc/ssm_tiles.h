// Device building blocks of the selective state space scan: tiles staged in
// LDS as bf16 pieces, their MFMA fragments, and the step tables.  Included by
// the ssm_*.hip files only.
//
// An input tile is held as NX bf16 pieces a value: one for bf16 inputs (exact),
// three for fp32 ones (24 bits).  A product of operands of NA and NB pieces
// takes the pairs i + j < max(NA, NB), which keeps every product to the
// accuracy of the coarser operand's last piece.
#pragma once
#include "common.h"
#include "mixer.h"
#include "vec.h"

namespace hla {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr float kLog2e = 1.4426950408889634f;
// Row stride of an LDS tile of W bf16 values, a dwords: a/4 is odd modulo 16, so
// that 16 rows' 8- or 16-byte reads at one column fall into different banks
// (of 64), and 0, a, 2a, 3a are 8 banks apart or more, so that the four rows a
// transposed read takes do too: a = 28, 36, 76 for W = 32, 64, 128.
__host__ __device__ constexpr int ld_of(int W) { return W == 64 ? 72 : W + 24; }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float nan_() { return __builtin_nanf(""); }

__device__ __forceinline__ rsrc_t rows_rsrc(const void* p, long long bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)(bytes > 0 ? bytes : 0), 0x00020000);
}
__device__ __forceinline__ rsrc_t tile_rsrc(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, 0x00020000);
}
__device__ __forceinline__ uint4 load16(rsrc_t r, uint32_t off) {
  const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0);
  return make_uint4(x[0], x[1], x[2], x[3]);
}

__device__ __forceinline__ void store8(rsrc_t r, uint32_t off, const uint2& v) {
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  __builtin_amdgcn_raw_buffer_store_b64(u32x2{v.x, v.y}, r, (int)off, 0, 0);
}
__device__ __forceinline__ void store16(rsrc_t r, uint32_t off, const float (&v)[4]) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  __builtin_amdgcn_raw_buffer_store_b128(
      u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, r, (int)off, 0,
      0);
}

// x through an empty asm statement: what is computed from it is computed where
// it is used, not hoisted out of the walk and kept in registers (or spilled) through it.
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// v_mfma_f32_16x16x32_bf16, lane l = 16 g + r:
//   A: row r, k = 8g .. 8g+7;  B: column r, the same k (any k order that A and
//   B share);  D: element i is D[4g + i][r].
__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }

// The order of the instructions before it: N products, each with V vector
// operations and an LDS read.  A product occupies the matrix core four times
// as long as it takes to issue; what the wave issues behind it is free.
template <int N, int V>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  }
}

template <int NA, int NB>
__device__ __forceinline__ void mma_pieces(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4& c) {
  constexpr int M = NA > NB ? NA : NB;
#pragma unroll
  for (int s = M - 1; s >= 0; --s)        // the smallest products first
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s - i >= 0 && s - i < NB) c = mma(a[i], b[s - i], c);
}

// Sums across lanes without the LDS unit.  A swap of halves (rows 0 1 with 2 3,
// or 0 with 1 and 2 with 3) of a value with itself leaves both halves' sum in
// the two results' sum, in every lane.
__device__ __forceinline__ float sum_groups(float v) {        // over the four rows of 16 lanes
  auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  h = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}
__device__ __forceinline__ double sum_groups(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  v = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  lo = __builtin_amdgcn_permlane16_swap((uint32_t)w, (uint32_t)w, false, false);
  hi = __builtin_amdgcn_permlane16_swap((uint32_t)(w >> 32), (uint32_t)(w >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float v) {               // 0 where the lane has no source
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// over the 16 lanes of a row, in every one of them (rotations by 8, 4, 2, 1)
template <typename F>
__device__ __forceinline__ F sum_row(F v) {
  v += dpp<0x128, 0xf>(v);
  v += dpp<0x124, 0xf>(v);
  v += dpp<0x122, 0xf>(v);
  return v + dpp<0x121, 0xf>(v);
}
__device__ __forceinline__ float sum_wave(float v) { return sum_groups(sum_row(v)); }
// sums over the lanes up to and with this one: shifts by 1, 2, 4, 8 in a row, then a row's last lane to the rows behind
template <int LANES = 64>                                     // or within each 32
__device__ __forceinline__ double sums_to(double v) {
  v += dpp<0x111, 0xf>(v);
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);
  if (LANES == 64) v += dpp<0x143, 0xc>(v);
  return v;
}
template <int LANE = 63>
__device__ __forceinline__ double last_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, LANE);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), LANE);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Eight values in NP pieces, round to nearest.
template <int NP>
__device__ __forceinline__ void pieces8(const float (&v)[8], bf16x8 (&p)[NP]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  uint32_t w[NP][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x0 = v[2 * i], x1 = v[2 * i + 1];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      w[k][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){x0, x1}, b2));
      x0 -= __uint_as_float(w[k][i] << 16);
      x1 -= __uint_as_float(w[k][i] & 0xffff0000u);
    }
  }
#pragma unroll
  for (int k = 0; k < NP; ++k) p[k] = __builtin_bit_cast(bf16x8, make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]));
}
template <int NP>
__device__ __forceinline__ void pieces4(const float (&v)[4], uint2 (&p)[NP]) {
  float z[8] = {v[0], v[1], v[2], v[3], 0.f, 0.f, 0.f, 0.f};
  bf16x8 q[NP];
  pieces8<NP>(z, q);
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const uint4 u = __builtin_bit_cast(uint4, q[k]);
    p[k] = make_uint2(u.x, u.y);
  }
}

// Fragments of a row-major LDS tile X[row][k] of row stride ld.
// frag: row row0 + r, k0 + 8g .. + 7.
__device__ __forceinline__ bf16x8 frag(const uint16_t* X, int ld, int row0, int k0, int l) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(X + (row0 + (l & 15)) * ld + k0 + 8 * (l >> 4)));
}
// A tile whose rows are stored in the order of accumulator pairs: value 16 a +
// 4 b + i of each 32 sits at 8 b + 4 a + i, so that frag() takes k0 + 4g .. + 3
// and k0 + 16 + 4g .. + 3, the order of two accumulator blocks as one operand.
// frag_plain: the 8 values k0 + 8g .. + 7 of row row0 + r of such a tile.
__device__ __forceinline__ bf16x8 frag_plain(const uint16_t* X, int ld, int row0, int k0, int l) {
  const int g = l >> 4;
  const uint16_t* p = X + (row0 + (l & 15)) * ld + k0 + 16 * (g & 1) + 4 * (g >> 1);
  const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + 8);
  return __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y));
}
// frag_tr: column n0 + r, rows k0 + 8g .. + 7, through the LDS transpose unit:
// in a group of 16 lanes element m of lane j's result is element j % 4 of the
// 8 bytes read by lane 4m + j / 4.
__device__ __forceinline__ bf16x8 frag_tr(const uint16_t* Y, int ld, int n0, int k0, int l) {
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
  const int j = l & 15;
  const uint16_t* p = Y + (k0 + 8 * (l >> 4) + (j >> 2)) * ld + n0 + 4 * (j & 3);
  const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(p));
  const v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(p + 4 * ld));
  const uint2 ua = __builtin_bit_cast(uint2, a), ub = __builtin_bit_cast(uint2, b);
  return __builtin_bit_cast(bf16x8, make_uint4(ua.x, ua.y, ub.x, ub.y));
}

// Two accumulator blocks (rows 16 b + 4g + i of one column) as a fragment in the order of accumulator pairs.
template <int NP>
__device__ __forceinline__ void frag_from_acc(const f32x4& lo, const f32x4& hi, bf16x8 (&p)[NP]) {
  const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  pieces8<NP>(v, p);
}

// ---------------------------------------------------------------------------
// A tile of Q token rows of a [B, n, ...] tensor on its way to LDS: THR threads
// take 16-byte pieces, W values a row (the row's own width w <= W; the rest and
// the rows past the sequence are zeros, which add nothing).
template <typename T>
struct Kind;
template <>
struct Kind<bf16> {
  static constexpr int NX = 1, Q = 64, V = 8;
};
template <>
struct Kind<float> {
  static constexpr int NX = 3, Q = 32, V = 4;
};

template <typename T, int W, int THR>
struct Tile {
  static constexpr int Q = Kind<T>::Q, V = Kind<T>::V, NX = Kind<T>::NX;
  static constexpr int PR = W / V, TOT = Q * PR, CNT = (TOT + THR - 1) / THR;
  static_assert((TOT % THR == 0 || TOT < THR) && THR % PR == 0, "whole pieces a thread, all of one column");
  static constexpr bool kAll = TOT >= THR;         // else the threads past TOT have none
  static constexpr uint32_t kOut = 0x80000000u;    // past any tile: reads zeros
  static constexpr int LD = ld_of(W), PLANE = Q * LD;
  uint4 r[CNT];

  // This thread's first piece and the bytes between its pieces, for rows ts >= w elements apart, w values each.
  static __device__ __forceinline__ uint32_t first(long long ts, int w, int tid) {
    const int row = tid / PR, c = (tid % PR) * V;
    return c < w && (kAll || tid < TOT) ? (uint32_t)((row * (int)ts + c) * (int)sizeof(T)) : kOut;
  }
  static __device__ __forceinline__ uint32_t step(long long ts) { return (THR / PR) * (uint32_t)ts * sizeof(T); }
  // The tile from its first row on, of which `rows` are valid: the others lie
  // past the resource's end.  A tile's bytes fit 31 bits (checked on the host).
  __device__ __forceinline__ void load(const void* base, int rows, int row_bytes, int w, uint32_t off, uint32_t by) {
    const rsrc_t rs = tile_rsrc(base, (rows - 1) * row_bytes + w * (int)sizeof(T));
#pragma unroll
    for (int i = 0; i < CNT; ++i) r[i] = load16(rs, off + i * by);
  }

  // The largest magnitudes of the low and the high halves so far, as bit patterns.
  static __device__ __forceinline__ void note(uint32_t& most, uint32_t pair) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const u16x2 a = __builtin_bit_cast(u16x2, pair & 0x7fff7fffu), m = __builtin_bit_cast(u16x2, most);
    most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, m));
  }

  // The tile as NX planes of Q rows.  CHECK: returns whether a value of this
  // thread's is infinite or NaN.  PAIRS: rows in the order of accumulator pairs.
  template <bool CHECK, bool PAIRS = false>
  __device__ __forceinline__ bool store(uint16_t* X, int tid) const {
    uint32_t most = 0;
    if (!kAll && tid >= TOT) return false;
    const int row0 = tid / PR, c = (tid % PR) * V;
    // in the order of accumulator pairs the halves of 8 values are 8 apart
    const int c2 = PAIRS ? (c & ~31) + 2 * (c & (NX == 1 ? 8 : 12)) + ((c & 16) >> 2) : c;
    uint16_t* first = X + row0 * LD + c2;
#pragma unroll
    for (int i = 0; i < CNT; ++i) {
      uint16_t* to = first + i * (THR / PR) * LD;
      if constexpr (NX == 1) {
        if (CHECK) {
          note(most, r[i].x);
          note(most, r[i].y);
          note(most, r[i].z);
          note(most, r[i].w);
        }
        if constexpr (PAIRS) {
          *reinterpret_cast<uint2*>(to) = make_uint2(r[i].x, r[i].y);
          *reinterpret_cast<uint2*>(to + 8) = make_uint2(r[i].z, r[i].w);
        } else {
          *reinterpret_cast<uint4*>(to) = r[i];
        }
      } else {
        const float v[4] = {__uint_as_float(r[i].x), __uint_as_float(r[i].y), __uint_as_float(r[i].z),
                            __uint_as_float(r[i].w)};
        uint2 p[NX];
        pieces4<NX>(v, p);
        if (CHECK) {
          note(most, p[0].x);
          note(most, p[0].y);
        }
#pragma unroll
        for (int k = 0; k < NX; ++k) *reinterpret_cast<uint2*>(to + k * PLANE) = p[k];
      }
    }
    return (most & 0xffffu) >= 0x7f80u || most >= 0x7f800000u;
  }

  // After a store() found one: such values of the tile become zeros, and the
  // first token that held one goes to first[column] and, unless null, *any.
  static __device__ __forceinline__ void mend(uint16_t* X, int* first, int* any, int tid) {
#pragma unroll 1
    for (int e = tid; e < Q * W; e += THR) {
      const int row = e / W, c = e % W;
      uint16_t* x = X + row * LD + c;
      if ((*x & 0x7f80u) != 0x7f80u) continue;
#pragma unroll
      for (int k = 0; k < NX; ++k) x[k * PLANE] = 0;
      atomicMin(first + c, row);
      if (any) atomicMin(any, row);
    }
  }
};

// ---------------------------------------------------------------------------
// Step table: one entry a (sequence, head, token of whole tiles), made once a
// call by k_ssm_steps.  L: the sum of dt A over the tile's tokens so far, in
// log2, high and low part; dt after the softplus; w = dt 2^(Lend - L).
struct Step {
  float Lh, Ll, dt, w;
};
// and one a tile: its whole L.

struct SsmPlan {
  int tiles, segs, per;        // tiles a sequence, segments, tiles a segment
};

template <int NP>
__device__ __forceinline__ void load_frags(const uint16_t* X, int plane, int ld, int row0, int k0, int l,
                                           bf16x8 (&f)[NP]) {
#pragma unroll
  for (int k = 0; k < NP; ++k) f[k] = frag(X + k * plane, ld, row0, k0, l);
}
template <int NP>
__device__ __forceinline__ void load_frags_plain(const uint16_t* X, int plane, int ld, int row0, int k0, int l,
                                                 bf16x8 (&f)[NP]) {
#pragma unroll
  for (int k = 0; k < NP; ++k) f[k] = frag_plain(X + k * plane, ld, row0, k0, l);
}
template <int NP>
__device__ __forceinline__ void load_frags_tr(const uint16_t* X, int plane, int ld, int n0, int k0, int l,
                                              bf16x8 (&f)[NP]) {
#pragma unroll
  for (int k = 0; k < NP; ++k) f[k] = frag_tr(X + k * plane, ld, n0, k0, l);
}

// The fragment's eight values from all its pieces, scaled, in NU pieces.
template <int NX, int NU>
__device__ __forceinline__ void scaled(const bf16x8 (&x)[NX], const float* w, bf16x8 (&u)[NU]) {
  const float4 a = *reinterpret_cast<const float4*>(w), b = *reinterpret_cast<const float4*>(w + 4);
  const float ws[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float s = 0.f;
#pragma unroll
    for (int k = NX - 1; k >= 0; --k) s += (float)x[k][i];
    v[i] = s * ws[i];
  }
  pieces8<NU>(v, u);
}

}  // namespace
}  // namespace hla
