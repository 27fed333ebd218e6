// Short causal convolution of K = 2 .. 4 taps a channel, with bias and SiLU:
//   z_t = bias + sum_j w_j x_{t-K+1+j},  y_t = z_t or z_t sigmoid(z_t)
// and its gradients
//   dz_t = dy_t (1 or s (1 + z (1 - s))),  s = sigmoid(z_t)
//   dx_t = sum_j w_j dz_{t+K-1-j},  dw_j = sum_t dz_t x_{t-K+1+j},  dbias = sum_t dz_t
//
// 2K + a few operations an element: bound by memory.  A thread walks a run of
// tokens of four channels (one where the width, a stride or an address does
// not keep four together) with the last K - 1 inputs in registers, so each
// input is read once, plus K - 1 rows a run.  Four channels, 8 bytes of bf16,
// rather than 16 bytes: half the registers a thread, so that twice the waves
// hide the loads.  A chunk of rows loads while the one before it is
// computed.  Sums are fp32, rounded once on the store.
// Measured on 8000 x 4352 in bf16 with bias and SiLU (139 MB): 28.7 us, 4.8
// TB/s; one token for 64 sequences 4.3 us, the same with one channel a thread
// (latency).  Forward 18.5 us and gradients 36 us (126 MB, 3.5 TB/s; 86 as
// 16-byte threads without loads ahead) over 4 x 4096 x 1280, the sums over the
// blocks 4 us.  Calls with one channel a thread instead of four: the first 36
// us instead of 29.5, the last with its gradients 78 instead of 59.  fp32 8000 x
// 4352 with SiLU (279 MB) 59 us, 4.7 TB/s; gradients over 4 x 4096 x 1280 (252
// MB) 47 us, with the sums over the blocks (an accurate exponential and
// quotient: 55 and 43 us with the hardware's approximations).
#include "common.h"
#include "mixer.h"
#include "vec.h"

namespace hla {
namespace {

constexpr int kConvThreads = 256;
constexpr int kConvBackRun = 16;   // tokens a thread of the gradients walks

// sigmoid(z) for values of type T.  fp32: within 2 * 2^-23 of itself.  bf16: by
// the hardware's exponential and reciprocal, whose error, 2^-24 |z| and a
// little more, is nothing beside the output's 2^-8.
template <typename T>
__device__ __forceinline__ float sigmoid(float z) {
  if constexpr (sizeof(T) == 2)
    return __builtin_amdgcn_rcpf(1.f + __expf(-z));
  else
    return 1.f / (1.f + expf(-z));
}

template <int V, int K>
__device__ __forceinline__ void taps(const Conv& a, int c, float (&w)[K][V], float (&b)[V]) {
  float all[V * K];
  if (a.w_dtype == 1) {
    load_many<bf16, V, V * K>(a.w, (size_t)c * K, all);
    if (a.bias) load_many<bf16, V, V>(a.bias, c, b);
  } else {
    load_many<float, V, V * K>(a.w, (size_t)c * K, all);
    if (a.bias) load_many<float, V, V>(a.bias, c, b);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int j = 0; j < K; ++j) w[j][i] = all[i * K + j];
    if (!a.bias) b[i] = 0.f;
  }
}

// Thread (run, channels) of batch blockIdx.y.  run_len >= K - 1, so only run 0
// reaches back into the state; it alone reads and writes it, the last K - 1
// inputs of [state; x] after its own reads, whatever the length.
template <typename T, int V, int K>
__global__ __launch_bounds__(kConvThreads) void k_conv(Conv a, int CV, int runs, int run_len) {
  const long long idx = (long long)blockIdx.x * kConvThreads + threadIdx.x;
  if (idx >= (long long)CV * runs) return;
  const int run = (int)(idx / CV), c = (int)(idx - (long long)run * CV) * V, b = blockIdx.y;
  const T* x = static_cast<const T*>(a.x.p) + b * a.x.bs + c;
  T* y = static_cast<T*>(a.y) + (size_t)b * a.n * a.D + c;
  const int t0 = run * run_len, t1 = min(a.n, t0 + run_len);
  constexpr int U = 4;
  Raw<T, V> next[U];
  auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < U; ++u) next[u].load(x + min(t + u, a.n - 1) * a.x.ts);   // past the run: not used
  };
  fetch(t0);
  float w[K][V], bias[V], win[K - 1][V];
  if (run == 0) {
    if (a.state) {
      T* st = static_cast<T*>(a.state) + (size_t)b * (K - 1) * a.D + c;
      T last[K - 1][V];
#pragma unroll
      for (int j = 0; j < K - 1; ++j) {
        load_vec<T, V>(st + (size_t)j * a.D, win[j]);
        const int i = a.n + j - (K - 1);
        copy_vec<T, V>(i >= 0 ? x + i * a.x.ts : st + (size_t)(a.n + j) * a.D, last[j]);
      }
#pragma unroll
      for (int j = 0; j < K - 1; ++j) copy_vec<T, V>(last[j], st + (size_t)j * a.D);
    } else {
#pragma unroll
      for (int j = 0; j < K - 1; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) win[j][i] = 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < K - 1; ++j) load_vec<T, V>(x + (t0 - (K - 1) + j) * a.x.ts, win[j]);
  }
  taps<V, K>(a, c, w, bias);
  for (int t = t0; t < t1; t += U) {
    Raw<T, V> in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) in[u] = next[u];
    fetch(t + U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float z[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float x_t = in[u].at(i);
        z[i] = bias[i];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) z[i] += w[j][i] * win[j][i];
        z[i] += w[K - 1][i] * x_t;
        if (a.silu) z[i] *= sigmoid<T>(z[i]);
#pragma unroll
        for (int j = 0; j + 1 < K - 1; ++j) win[j][i] = win[j + 1][i];
        win[K - 2][i] = x_t;
      }
      if (t + u < t1) store_vec<T, V>(y + (size_t)(t + u) * a.D, z);
    }
  }
}

// Gradients.  A block is kConvCL channel pieces by kConvRL runs; a thread walks its run
// and K - 1 tokens past it with the last K inputs and the last K values of dz
// in registers, and sums its tokens' share of dw and dbias.  The runs of a
// block are summed in the wave and over the waves in a fixed order, a row of
// partials [D (K + 1)] a block, and k_conv_sum adds the rows: no atomics, so
// the same inputs give the same bits.
constexpr int kConvCL = 32, kConvRL = kConvThreads / kConvCL;

template <typename T, int V, int K>
__global__ __launch_bounds__(kConvThreads) void k_conv_back(Conv a, float* part) {
  const int cl = threadIdx.x % kConvCL, rl = threadIdx.x / kConvCL, b = blockIdx.z;
  const int c = (blockIdx.x * kConvCL + cl) * V;
  const int t0 = (blockIdx.y * kConvRL + rl) * kConvBackRun, t1 = min(a.n, t0 + kConvBackRun);
  float dw[K + 1][V];
#pragma unroll
  for (int j = 0; j <= K; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) dw[j][i] = 0.f;
  if (c < a.D && t0 < a.n) {
    const T* x = static_cast<const T*>(a.x.p) + b * a.x.bs + c;
    const T* dy = static_cast<const T*>(a.dy.p) + b * a.dy.bs + c;
    T* dx = static_cast<T*>(a.dx) + (size_t)b * a.n * a.D + c;
    constexpr int U = 4;
    Raw<T, V> nx[U], ng[U];
    // rows past the sequence: no part in anything (there is tested below)
    auto fetch = [&](int t) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        nx[u].load(x + min(t + u, a.n - 1) * a.x.ts);
        ng[u].load(dy + min(t + u, a.n - 1) * a.dy.ts);
      }
    };
    fetch(t0);
    float w[K][V], bias[V], win[K][V], dz[K][V];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int t = t0 - K + j;      // the first is shifted out at once
      if (j > 0 && t >= 0) {
        load_vec<T, V>(x + t * a.x.ts, win[j]);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) win[j][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) dz[j][i] = 0.f;
    }
    taps<V, K>(a, c, w, bias);
    for (int t = t0; t < t1 + K - 1; t += U) {
      Raw<T, V> in[U], g[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        in[u] = nx[u];
        g[u] = ng[u];
      }
      fetch(t + U);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool mine = t + u < t1;
        const bool there = t + u < t1 + K - 1 && t + u < a.n;
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
          for (int j = 0; j + 1 < K; ++j) {
            win[j][i] = win[j + 1][i];
            dz[j][i] = dz[j + 1][i];
          }
          win[K - 1][i] = in[u].at(i);
          float d = g[u].at(i);
          if (a.silu) {
            float z = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) z += w[j][i] * win[j][i];
            const float s = sigmoid<T>(z);
            d *= s * (1.f + z * (1.f - s));
          }
          dz[K - 1][i] = there ? d : 0.f;
          if (mine) {
#pragma unroll
            for (int j = 0; j < K; ++j) dw[j][i] += d * win[j][i];
            dw[K][i] += d;
          }
          out[i] = 0.f;
#pragma unroll
          for (int j = 0; j < K; ++j) out[i] += w[j][i] * dz[K - 1 - j][i];
        }
        const int to = t + u - (K - 1);
        if (to >= t0 && to < t1) store_vec<T, V>(dx + (size_t)to * a.D, out);
      }
    }
  }
  __shared__ float red[kConvThreads / 64][kConvCL * V];
  float* to = part + ((size_t)blockIdx.z * gridDim.y + blockIdx.y) * a.D * (K + 1);
#pragma unroll
  for (int j = 0; j <= K; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float v = dw[j][i] + __shfl_xor(dw[j][i], 32);
      if ((threadIdx.x & 63) < kConvCL) red[threadIdx.x / 64][cl * V + i] = v;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kConvCL * V; e += kConvThreads) {
      const int ch = blockIdx.x * kConvCL * V + e;
      if (ch < a.D) to[(size_t)j * a.D + ch] = red[0][e] + red[1][e] + red[2][e] + red[3][e];
    }
    __syncthreads();
  }
}

// part [rows][K + 1][D] -> dw [D, K], dbias [D]: 64 columns by 16 row groups a block.
constexpr int kSumRows = 16;
__global__ __launch_bounds__(64 * kSumRows) void k_conv_sum(Conv a, const float* __restrict__ part, int rows) {
  const int cols = a.D * (a.K + 1), col = blockIdx.x * 64 + threadIdx.x % 64, rg = threadIdx.x / 64;
  __shared__ float red[kSumRows][64];
  float s = 0.f;
  if (col < cols)
    for (int r = rg; r < rows; r += kSumRows) s += part[(size_t)r * cols + col];
  red[rg][threadIdx.x % 64] = s;
  __syncthreads();
  if (rg != 0 || col >= cols) return;
  for (int r = 1; r < kSumRows; ++r) s += red[r][threadIdx.x];
  const int j = col / a.D, c = col - j * a.D;
  if (j < a.K)
    store_any(a.dw, a.w_dtype, (size_t)c * a.K + j, s);
  else if (a.dbias)
    store_any(a.dbias, a.w_dtype, c, s);
}

// Blocks over the tokens of the gradients.
int conv_back_blocks(int n) { return (n + kConvBackRun * kConvRL - 1) / (kConvBackRun * kConvRL); }

// Whether four channels stay together: whole vectors of 4 values everywhere.
bool vec_ok(const Conv& c) {
  const int es = c.dtype == 1 ? 2 : 4, ws = c.w_dtype == 1 ? 2 : 4;
  auto whole = [](const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % (4 * size) == 0; };
  auto fits = [&](const Rows& r) { return whole(r.p, es) && r.bs % 4 == 0 && r.ts % 4 == 0; };
  return c.D % 4 == 0 && fits(c.x) && fits(c.dy) && whole(c.state, es) && whole(c.y, es) && whole(c.dx, es) &&
         whole(c.w, ws) && whole(c.bias, ws);
}

template <typename T, int V, int K>
hipError_t forward(const Conv& c, hipStream_t s) {
  const int CV = c.D / V;
  // runs of 4 (the shortest that keeps the state to run 0) up to 16 tokens: as long as all CUs still get eight waves
  int len = 4;
  while (len < 16 && (long long)CV * c.B * ((c.n + 2 * len - 1) / (2 * len)) >= 256LL * 8 * 64) len *= 2;
  const int runs = (c.n + len - 1) / len;
  const long long blocks = ((long long)CV * runs + kConvThreads - 1) / kConvThreads;
  return HLA_TIMED("conv", (k_conv<T, V, K>), dim3((unsigned)blocks, c.B), dim3(kConvThreads), 0, s, c, CV, runs, len);
}

template <typename T, int V, int K>
hipError_t backward(const Conv& c, float* part, hipStream_t s) {
  const int cb = (c.D / V + kConvCL - 1) / kConvCL, tb = conv_back_blocks(c.n);
  const hipError_t e = HLA_TIMED("conv_back", (k_conv_back<T, V, K>), dim3(cb, tb, c.B), dim3(kConvThreads), 0, s, c,
                                 part);
  if (e != hipSuccess) return e;
  const int cols = c.D * (K + 1);
  return HLA_TIMED("conv_sum", k_conv_sum, dim3((cols + 63) / 64), dim3(64 * kSumRows), 0, s, c, part, tb * c.B);
}

template <typename T, int V>
hipError_t by_k(const Conv& c, float* part, hipStream_t s) {
  switch (c.K) {
    case 2: return part ? backward<T, V, 2>(c, part, s) : forward<T, V, 2>(c, s);
    case 3: return part ? backward<T, V, 3>(c, part, s) : forward<T, V, 3>(c, s);
    default: return part ? backward<T, V, 4>(c, part, s) : forward<T, V, 4>(c, s);
  }
}

hipError_t by_type(const Conv& c, float* part, hipStream_t s) {
  const bool vec = vec_ok(c);
  if (c.dtype == 1) return vec ? by_k<bf16, 4>(c, part, s) : by_k<bf16, 1>(c, part, s);
  return vec ? by_k<float, 4>(c, part, s) : by_k<float, 1>(c, part, s);
}

}  // namespace

hipError_t launch_conv_forward(const Conv& c, hipStream_t s) { return by_type(c, nullptr, s); }

size_t conv_backward_ws(int B, int n, int D, int K) {
  return sizeof(float) * conv_back_blocks(n) * (size_t)B * D * (K + 1);
}

hipError_t launch_conv_backward(const Conv& c, void* ws, hipStream_t s) {
  return by_type(c, static_cast<float*>(ws), s);
}

}  // namespace hla
