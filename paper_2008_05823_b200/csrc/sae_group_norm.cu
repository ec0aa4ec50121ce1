// Group norm with an activation, channels last, forward and backward.  Declarations and contract: include/sae.h.
//
// x is [N][P][C] (P pixels, the channels of a pixel neighbours in memory); group j is the Cg channels from j * Cg on, over
// all P pixels of a sample, M = P * Cg values:
//   mean = sum x / M,  var = sum (x - mean)^2 / M,  rstd = 1 / sqrt(var + eps)
//   xhat = (x - mean) * rstd,  z = xhat * w_c + b_c (+ residual),  y = act(z)
//   dz = dy * act'(z),  db_c = sum dz,  dw_c = sum dz * xhat,  g = dz * w_c,
//   dx = rstd * (g - mean_group(g) - xhat * mean_group(g * xhat))
// z is computed by the same separately rounded operations in both directions, so that relu's mask in the backward pass is
// the forward pass's own.
//
// Everything is bound by HBM.  A group of neighbouring channels is a column of short runs, so a thread takes 16 bytes of a
// pixel, always the same channels, and walks down the pixels; the threads of a block stand side by side over the channels
// first, which makes a block's loads whole lines whatever the group size is.
#include "../../include/sae.h"
#include "sae_vec.cuh"

#include <algorithm>
#include <cooperative_groups.h>

using namespace sae;
namespace cg = cooperative_groups;

namespace {

constexpr int GN_THREADS = 256;
constexpr int GN_BATCH = 4;              // pixels a thread has in flight

struct Args {
  const void *x, *res, *dy, *w, *b;
  void *out, *dres;                      // y or dx; dense
  float *mean, *rstd;                    // [N][G]: written forwards, read backwards
  void *dw, *db;
  long long x_n, x_p, r_n, r_p, d_n, d_p;   // strides of a sample and of a pixel, in elements
  int N, P, C, G, Cg;
  int act, ptype;
  float eps;
  int slices, cvt;                       // runs of pixels a sample is cut into; vectors of a pixel a block takes
  float *part_a, *part_b;                // [N][slices][C] values of each channel's run (forwards: mean and squares about it;
                                         // backwards: sum dz and sum dz * xhat)
  float *mean_g, *mean_gx;               // [N][G] backwards: mean_group(g), mean_group(g * xhat)
};

__device__ __forceinline__ float param(const void* p, int type, int c, float none) {
  if (!p) return none;
  if (type == SAE_TYPE_FLOAT) return __ldg((const float*)p + c);
  if (type == SAE_TYPE_BFLOAT) return to_f(((const __nv_bfloat16*)p)[c]);
  return to_f(((const __half*)p)[c]);
}
__device__ __forceinline__ void put_param(void* p, int type, int c, float v) {
  if (type == SAE_TYPE_FLOAT) ((float*)p)[c] = v;
  else if (type == SAE_TYPE_BFLOAT) ((__nv_bfloat16*)p)[c] = from_f<__nv_bfloat16>(v);
  else ((__half*)p)[c] = from_f<__half>(v);
}

// ---- activations ------------------------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
// Exact enough for float32 results: expf and a true division.  (__expf's error grows with |z|.)
__device__ __forceinline__ float sigmoid_exact(float z) { return __fdiv_rn(1.0f, 1.0f + expf(-z)); }

template <typename T>
__device__ __forceinline__ float sigmoid_for(float z) { return sizeof(T) == 4 ? sigmoid_exact(z) : sigmoid(z); }

template <typename T, int V>
__device__ __forceinline__ void activate(float (&z)[V], int act) {
  if (act == SAE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(z[i]) : "f"(z[i]));
  } else if (act == SAE_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] *= sigmoid_for<T>(z[i]);
  } else if (act == SAE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] *= 0.5f * (1.0f + erff(z[i] * 0.70710678f));
  }
}

// dz[i] = dy[i] * act'(z[i])
template <typename T, int V>
__device__ __forceinline__ void slope(float (&dz)[V], const float (&z)[V], int act) {
  if (act == SAE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) dz[i] = z[i] > 0.0f ? dz[i] : 0.0f;
  } else if (act == SAE_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float s = sigmoid_for<T>(z[i]);
      dz[i] *= s * (1.0f + z[i] * (1.0f - s));
    }
  } else if (act == SAE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float cdf = 0.5f * (1.0f + erff(z[i] * 0.70710678f));
      dz[i] *= cdf + z[i] * (0.39894228f * expf(-0.5f * z[i] * z[i]));
    }
  }
}

// ---- what a thread stands for: V channels from c on, pixels p0 + row, p0 + row + rows, .. below p1 ----------------
struct Place {
  int n, slice, c, p, p1, rows, row, tid_in;
  bool on;
};
template <int V>
__device__ __forceinline__ Place place(const Args& a) {
  Place q;
  q.n = blockIdx.x / a.slices;
  q.slice = blockIdx.x - q.n * a.slices;
  q.rows = GN_THREADS / a.cvt;
  q.row = threadIdx.x / a.cvt;
  const int cv = threadIdx.x - q.row * a.cvt;
  q.c = (blockIdx.y * a.cvt + cv) * V;
  q.on = q.row < q.rows && q.c < a.C;
  const int p0 = (int)((long long)a.P * q.slice / a.slices);
  q.p1 = (int)((long long)a.P * (q.slice + 1) / a.slices);
  q.p = p0 + q.row;
  return q;
}

template <int V>
struct Channels {                        // a thread's channels: their group's statistics, weight and bias
  float mean[V], rstd[V], w[V], b[V];
  __device__ __forceinline__ void load(const Args& a, int n, int c) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int g = (c + i) / a.Cg;
      mean[i] = a.mean[(long long)n * a.G + g];
      rstd[i] = a.rstd[(long long)n * a.G + g];
      w[i] = param(a.w, a.ptype, c + i, 1.0f);
      b[i] = param(a.b, a.ptype, c + i, 0.0f);
    }
  }
  __device__ __forceinline__ float xhat(int i, float x) const { return __fmul_rn(__fsub_rn(x, mean[i]), rstd[i]); }
  __device__ __forceinline__ float z(int i, float xh) const { return __fadd_rn(__fmul_rn(xh, w[i]), b[i]); }
};

// ---- forward, two passes over x -----------------------------------------------------------------------------------
// A run's count, mean and squares about it; joining two runs by the update of Chan, Golub and LeVeque.
__device__ __forceinline__ void join(float& n, float& mean, float& m2, float on, float omean, float om2) {
  if (on == 0.0f) return;
  const float t = n + on, d = omean - mean, f = on / t;
  mean = __fmaf_rn(d, f, mean);
  m2 += om2 + d * d * (n * f);
  n = t;
}

template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS) k_gn_statistics(const Args a) {
  extern __shared__ float sh[];           // [2][V][GN_THREADS], then [GN_THREADS] counts
  const Place q = place<V>(a);
  float n = 0.0f, mean[V], m2[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { mean[i] = 0.0f; m2[i] = 0.0f; }
  if (q.on) {
    const T* x = (const T*)a.x + q.n * a.x_n + q.c;
    for (int p = q.p; p < q.p1; p += GN_BATCH * q.rows) {
      Raw<T, V> raw[GN_BATCH];
      float v[GN_BATCH][V];
      int m = 0;
#pragma unroll
      for (int k = 0; k < GN_BATCH; ++k)
        if (p + k * q.rows < q.p1) { raw[k].load(x + (long long)(p + k * q.rows) * a.x_p); m = k + 1; }
      // the batch's own mean and squares about it, then joined to what came before
      const float fm = (float)m, inv = 1.0f / fm, t = n + fm, f = fm / t, nf = n * f;
#pragma unroll
      for (int k = 0; k < GN_BATCH; ++k) {
        if (k < m) raw[k].widen(v[k]);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float s = v[0][i];
#pragma unroll
        for (int k = 1; k < GN_BATCH; ++k) if (k < m) s += v[k][i];
        const float bm = s * inv;
        float b2 = 0.0f;
#pragma unroll
        for (int k = 0; k < GN_BATCH; ++k) if (k < m) { const float d = v[k][i] - bm; b2 = __fmaf_rn(d, d, b2); }
        const float d = bm - mean[i];
        mean[i] = __fmaf_rn(d, f, mean[i]);
        m2[i] += __fmaf_rn(d * d, nf, b2);
      }
      n = t;
    }
  }
  float *sm = sh, *s2 = sh + V * GN_THREADS, *sn = sh + 2 * V * GN_THREADS;
#pragma unroll
  for (int i = 0; i < V; ++i) { sm[i * GN_THREADS + threadIdx.x] = mean[i]; s2[i * GN_THREADS + threadIdx.x] = m2[i]; }
  sn[threadIdx.x] = n;
  for (int w = q.rows; w > 1;) {          // rows join pairwise, always the same pairs
    const int half = (w + 1) / 2;
    __syncthreads();
    const bool take = q.on && q.row + half < w;
    if (take) {
      const int o = threadIdx.x + half * a.cvt;
      const float on = sn[o];
      float t = n;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        t = n;
        join(t, mean[i], m2[i], on, sm[i * GN_THREADS + o], s2[i * GN_THREADS + o]);
        sm[i * GN_THREADS + threadIdx.x] = mean[i]; s2[i * GN_THREADS + threadIdx.x] = m2[i];
      }
      n = t;
      sn[threadIdx.x] = n;
    }
    w = half;
  }
  if (q.on && q.row == 0) {
    const long long at = ((long long)q.n * a.slices + q.slice) * a.C + q.c;
#pragma unroll
    for (int i = 0; i < V; ++i) { a.part_a[at + i] = mean[i]; a.part_b[at + i] = m2[i]; }
  }
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ int slice_count(const Args& a, int s) {
  return (int)((long long)a.P * (s + 1) / a.slices) - (int)((long long)a.P * s / a.slices);
}

// One warp a group: its channels' runs joined about the group's own mean, in double.
__global__ void __launch_bounds__(GN_THREADS) k_gn_finish_statistics(const Args a) {
  const long long g = ((long long)blockIdx.x * GN_THREADS + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (g >= (long long)a.N * a.G) return;
  const int n = (int)(g / a.G), j = (int)(g - (long long)n * a.G);
  const long long base = (long long)n * a.slices * a.C + (long long)j * a.Cg;
  const int E = a.slices * a.Cg;
  double s = 0.0, q = 0.0;
  for (int e = lane; e < E; e += 32) {
    const int sl = e / a.Cg, c = e - sl * a.Cg;
    s += (double)slice_count(a, sl) * (double)a.part_a[base + (long long)sl * a.C + c];
  }
  const double M = (double)a.P * a.Cg, mean = warp_sum(s) / M;
  for (int e = lane; e < E; e += 32) {
    const int sl = e / a.Cg, c = e - sl * a.Cg;
    const double d = (double)a.part_a[base + (long long)sl * a.C + c] - mean;
    q += (double)a.part_b[base + (long long)sl * a.C + c] + (double)slice_count(a, sl) * d * d;
  }
  const double var = warp_sum(q) / M;
  if (lane == 0) {
    a.mean[g] = (float)mean;
    a.rstd[g] = (float)(1.0 / sqrt(var + (double)a.eps));
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS) k_gn_apply(const Args a) {
  const Place q = place<V>(a);
  if (!q.on) return;
  Channels<V> ch;
  ch.load(a, q.n, q.c);
  const T* x = (const T*)a.x + q.n * a.x_n + q.c;
  const T* r = a.res ? (const T*)a.res + q.n * a.r_n + q.c : nullptr;
  T* y = (T*)a.out + (long long)q.n * a.P * a.C + q.c;
  for (int p = q.p; p < q.p1; p += GN_BATCH * q.rows) {
    Raw<T, V> xr[GN_BATCH], rr[GN_BATCH];
#pragma unroll
    for (int k = 0; k < GN_BATCH; ++k) {
      const long long pk = p + (long long)k * q.rows;
      if (pk < q.p1) { xr[k].load(x + pk * a.x_p); if (r) rr[k].load(r + pk * a.r_p); }
    }
#pragma unroll
    for (int k = 0; k < GN_BATCH; ++k) {
      const long long pk = p + (long long)k * q.rows;
      if (pk < q.p1) {
        float v[V], z[V];
        xr[k].widen(v);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = ch.z(i, ch.xhat(i, v[i]));
        if (r) {
          rr[k].widen(v);
#pragma unroll
          for (int i = 0; i < V; ++i) z[i] = __fadd_rn(z[i], v[i]);
        }
        activate<T, V>(z, a.act);
        Raw<T, V> o;
        o.round(z);
        o.store(y + pk * a.C);
      }
    }
  }
}

// ---- backward, two passes over dy and x ----------------------------------------------------------------------------
template <typename T, int V>
__device__ __forceinline__ void grad_z(const Channels<V>& ch, const Raw<T, V>& xr, const Raw<T, V>& dr, const Raw<T, V>* rr, int act,
                                       float (&xh)[V], float (&dz)[V]) {
  float v[V], z[V];
  xr.widen(v);
  dr.widen(dz);
#pragma unroll
  for (int i = 0; i < V; ++i) { xh[i] = ch.xhat(i, v[i]); z[i] = ch.z(i, xh[i]); }
  if (rr) {
    rr->widen(v);
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = __fadd_rn(z[i], v[i]);
  }
  slope<T, V>(dz, z, act);
}

template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS) k_gn_grad_sums(const Args a) {
  extern __shared__ float sh[];           // [2][V][GN_THREADS]
  const Place q = place<V>(a);
  float s[V], sx[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { s[i] = 0.0f; sx[i] = 0.0f; }
  if (q.on) {
    Channels<V> ch;
    ch.load(a, q.n, q.c);
    const T* x = (const T*)a.x + q.n * a.x_n + q.c;
    const T* d = (const T*)a.dy + q.n * a.d_n + q.c;
    const T* r = a.res ? (const T*)a.res + q.n * a.r_n + q.c : nullptr;
    T* dres = a.dres ? (T*)a.dres + (long long)q.n * a.P * a.C + q.c : nullptr;
    for (int p = q.p; p < q.p1; p += GN_BATCH * q.rows) {
      Raw<T, V> xr[GN_BATCH], dr[GN_BATCH], rr[GN_BATCH];
#pragma unroll
      for (int k = 0; k < GN_BATCH; ++k) {
        const long long pk = p + (long long)k * q.rows;
        if (pk < q.p1) { xr[k].load(x + pk * a.x_p); dr[k].load(d + pk * a.d_p); if (r) rr[k].load(r + pk * a.r_p); }
      }
#pragma unroll
      for (int k = 0; k < GN_BATCH; ++k) {
        const long long pk = p + (long long)k * q.rows;
        if (pk < q.p1) {
          float xh[V], dz[V];
          grad_z<T, V>(ch, xr[k], dr[k], r ? &rr[k] : nullptr, a.act, xh, dz);
#pragma unroll
          for (int i = 0; i < V; ++i) { s[i] += dz[i]; sx[i] = __fmaf_rn(dz[i], xh[i], sx[i]); }
          if (dres) { Raw<T, V> o; o.round(dz); o.store(dres + pk * a.C); }
        }
      }
    }
  }
  float *s1 = sh, *s2 = sh + V * GN_THREADS;
#pragma unroll
  for (int i = 0; i < V; ++i) { s1[i * GN_THREADS + threadIdx.x] = s[i]; s2[i * GN_THREADS + threadIdx.x] = sx[i]; }
  for (int w = q.rows; w > 1;) {
    const int half = (w + 1) / 2;
    __syncthreads();
    if (q.on && q.row + half < w) {
      const int o = threadIdx.x + half * a.cvt;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s[i] += s1[i * GN_THREADS + o]; sx[i] += s2[i * GN_THREADS + o];
        s1[i * GN_THREADS + threadIdx.x] = s[i]; s2[i * GN_THREADS + threadIdx.x] = sx[i];
      }
    }
    w = half;
  }
  if (q.on && q.row == 0) {
    const long long at = ((long long)q.n * a.slices + q.slice) * a.C + q.c;
#pragma unroll
    for (int i = 0; i < V; ++i) { a.part_a[at + i] = s[i]; a.part_b[at + i] = sx[i]; }
  }
}

// One warp a group: mean_group(g) and mean_group(g * xhat) from the channels' sums.
__global__ void __launch_bounds__(GN_THREADS) k_gn_finish_grad(const Args a) {
  const long long g = ((long long)blockIdx.x * GN_THREADS + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (g >= (long long)a.N * a.G) return;
  const int n = (int)(g / a.G), j = (int)(g - (long long)n * a.G);
  const long long base = (long long)n * a.slices * a.C + (long long)j * a.Cg;
  const int E = a.slices * a.Cg;
  double s = 0.0, q = 0.0;
  for (int e = lane; e < E; e += 32) {
    const int sl = e / a.Cg, c = e - sl * a.Cg;
    const double w = (double)param(a.w, a.ptype, j * a.Cg + c, 1.0f);
    s += w * (double)a.part_a[base + (long long)sl * a.C + c];
    q += w * (double)a.part_b[base + (long long)sl * a.C + c];
  }
  s = warp_sum(s); q = warp_sum(q);
  if (lane == 0) {
    const double M = (double)a.P * a.Cg;
    a.mean_g[g] = (float)(s / M);
    a.mean_gx[g] = (float)(q / M);
  }
}

// dw and db: the channels' sums over samples and runs, 32 channels a block, in a fixed order.
__global__ void __launch_bounds__(1024) k_gn_param_grads(const Args a, int rows) {
  __shared__ float sa[32][33], sb[32][33];
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5, c = blockIdx.x * 32 + cx;
  float s = 0.0f, q = 0.0f;
  if (c < a.C)
    for (int r = ry; r < rows; r += 32) { s += a.part_a[(long long)r * a.C + c]; q += a.part_b[(long long)r * a.C + c]; }
  sa[ry][cx] = s; sb[ry][cx] = q;
  __syncthreads();
  s = sa[cx][ry]; q = sb[cx][ry];         // a warp now holds one channel's 32 sums
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { s += __shfl_xor_sync(0xffffffffu, s, o); q += __shfl_xor_sync(0xffffffffu, q, o); }
  const int cc = blockIdx.x * 32 + ry;
  if (cx == 0 && cc < a.C) {
    if (a.db) put_param(a.db, a.ptype, cc, s);
    if (a.dw) put_param(a.dw, a.ptype, cc, q);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(GN_THREADS) k_gn_grad_apply(const Args a) {
  const Place q = place<V>(a);
  if (!q.on) return;
  Channels<V> ch;
  ch.load(a, q.n, q.c);
  float mg[V], mx[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const long long g = (long long)q.n * a.G + (q.c + i) / a.Cg;
    mg[i] = a.mean_g[g]; mx[i] = a.mean_gx[g];
  }
  const T* x = (const T*)a.x + q.n * a.x_n + q.c;
  const T* d = (const T*)a.dy + q.n * a.d_n + q.c;
  const T* r = a.res ? (const T*)a.res + q.n * a.r_n + q.c : nullptr;
  T* dx = (T*)a.out + (long long)q.n * a.P * a.C + q.c;
  for (int p = q.p; p < q.p1; p += GN_BATCH * q.rows) {
    Raw<T, V> xr[GN_BATCH], dr[GN_BATCH], rr[GN_BATCH];
#pragma unroll
    for (int k = 0; k < GN_BATCH; ++k) {
      const long long pk = p + (long long)k * q.rows;
      if (pk < q.p1) { xr[k].load(x + pk * a.x_p); dr[k].load(d + pk * a.d_p); if (r) rr[k].load(r + pk * a.r_p); }
    }
#pragma unroll
    for (int k = 0; k < GN_BATCH; ++k) {
      const long long pk = p + (long long)k * q.rows;
      if (pk < q.p1) {
        float xh[V], dz[V];
        grad_z<T, V>(ch, xr[k], dr[k], r ? &rr[k] : nullptr, a.act, xh, dz);
#pragma unroll
        for (int i = 0; i < V; ++i) dz[i] = ch.rstd[i] * (__fmul_rn(dz[i], ch.w[i]) - mg[i] - xh[i] * mx[i]);
        Raw<T, V> o;
        o.round(dz);
        o.store(dx + pk * a.C);
      }
    }
  }
}

// ---- one pass: a unit (a sample's channels of one or more whole groups) stays in shared memory --------------------
// A cluster of S blocks takes a unit, each its run of pixels.  Every thread copies its own vectors into shared memory
// asynchronously (slots that nobody else reads: no barrier for the data), so the inputs are read from HBM once; the
// blocks' sums meet through distributed shared memory.
struct Unit {
  int log_cvt;                           // vectors of a pixel that stand side by side in a block: a power of two
  int cc, chunks;                        // channels of a unit (whole groups, whole vectors); units a sample has
  int px, S;                             // pixels a block takes; blocks of a cluster
  int slots;                             // vectors a thread holds of each tensor
};

template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const unsigned int s = (unsigned int)__cvta_generic_to_shared(to);
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from) : "memory");
  else if constexpr (BYTES >= 4) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(s), "l"(from), "n"(BYTES) : "memory");
  else *(unsigned short*)to = __ldg((const unsigned short*)from);
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's `turns` vectors, `step` elements apart, into its slots.
template <typename T, int V>
__device__ __forceinline__ void fetch(typename Raw<T, V>::B* to, const T* from, long long step, int pitch, int turns) {
#pragma unroll 4
  for (int k = 0; k < turns; ++k, from += step) copy_async<V * (int)sizeof(T)>(to + k * pitch, from);
}

// A thread's V channel sums as one, or as they are.
template <int V, int SL>
__device__ __forceinline__ void narrow(const float (&v)[V], float (&o)[SL]) {
  if constexpr (SL == V) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = v[i];
  } else {
    float t = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) t += v[i];
    o[0] = t;
  }
}

// Adds up v over the rows of a block, column by column: afterwards sh[r * pitch + column * SL + i] holds the sums of row r's
// warp (columns fewer than a warp's lanes: those are joined here) and `rows` such rows are left to add.  Ends with a barrier.
template <int SL>
__device__ __forceinline__ int fold_rows(float (&v)[SL], float* sh, int log_cvt) {
  const int cvt = 1 << log_cvt, tid = threadIdx.x;
  int rows = (int)blockDim.x >> log_cvt, row = tid >> log_cvt;
  bool write = true;
  if (log_cvt < 5) {
    for (int o = 16; o >= cvt; o >>= 1) {
#pragma unroll
      for (int i = 0; i < SL; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    rows = (int)blockDim.x >> 5;
    row = tid >> 5;
    write = (tid & 31) < cvt;
  }
  if (write) {
    float* to = sh + (row * cvt + (tid & (cvt - 1))) * SL;
#pragma unroll
    for (int i = 0; i < SL; ++i) to[i] = v[i];
  }
  __syncthreads();
  return rows;
}

// The folded values of each group: one warp a group, `per` neighbouring values of it in a row.  out[j] is written by lane 0.
template <typename F>
__device__ __forceinline__ void fold_groups(const float* sh, int rows, int pitch, int per, int groups, F out) {
  const int lane = threadIdx.x & 31;
  const float inv_per = 1.0f / (float)per;
  for (int j = threadIdx.x >> 5; j < groups; j += (int)blockDim.x >> 5) {
    float s = 0.0f;
    for (int e = lane; e < rows * per; e += 32) {
      const int r = (int)(((float)e + 0.5f) * inv_per);
      s += sh[r * pitch + j * per + (e - r * per)];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) out(j, s);
  }
}

// V neighbouring parameters at once: c is a multiple of V, and the parameters' own alignment is checked here.
template <int V>
__device__ __forceinline__ void params(const void* p, int type, int c, float none, float (&o)[V]) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = none;
  } else if (V >= 4 && type == SAE_TYPE_FLOAT && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i + 3 < V; i += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>((const float*)p + c + i));
      o[i] = f.x; o[i + 1] = f.y; o[i + 2] = f.z; o[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = param(p, type, c + i, none);
  }
}

// Small non-negative integers (below 2^20) over a divisor, by its reciprocal.
__device__ __forceinline__ int quotient(int a, float inv) { return (int)(((float)a + 0.5f) * inv); }

// A block's place: a cluster is one unit (chunk blockIdx.x / S of sample n), a block the rank-th run of its pixels.
struct Spot {
  int n, rank, cc, groups, c0, co, c, p0, all, row, rows, turns;
  bool on;                                // this thread's channels exist
};
template <int V>
__device__ __forceinline__ Spot spot(const Args& a, const Unit& u) {
  Spot q;
  q.n = blockIdx.y + gridDim.y * blockIdx.z;
  unsigned int rank, chunk;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(chunk));
  q.rank = (int)rank;
  q.c0 = (int)chunk * u.cc;
  q.cc = min(u.cc, a.C - q.c0);
  q.groups = q.cc / a.Cg;
  q.co = ((int)threadIdx.x & ((1 << u.log_cvt) - 1)) * V;
  q.c = q.c0 + q.co;
  q.row = (int)threadIdx.x >> u.log_cvt;
  q.rows = (int)blockDim.x >> u.log_cvt;
  q.p0 = q.rank * u.px;
  q.all = max(0, min(u.px, a.P - q.p0));
  q.on = q.co < q.cc;
  q.turns = q.on && q.all > q.row ? (q.all - q.row - 1) / q.rows + 1 : 0;
  return q;
}

// WHOLE: a vector lies within one group, so one value a thread is enough for a statistic; else one a channel.
// Statistics in one pass: a thread sums x - k and its square, k being its own first value (WHOLE: its first vector's mean).
// As k is one of the values, (mean - k)^2 is at most their squares' sum about the mean, so taking the squares about the mean
// from those about k loses at most the thread's count of values, in units of rounding: no large mean cancels.
template <typename T, int V, bool WHOLE>
__global__ void __launch_bounds__(GN_THREADS, 3) k_gn_unit(const Args a, const Unit u) {
  extern __shared__ __align__(16) unsigned char smem[];
  typedef typename Raw<T, V>::B B;
  constexpr int SL = WHOLE ? 1 : V;
  const Spot q = spot<V>(a, u);
  if (q.n >= a.N) return;                                                       // the whole cluster
  const int TH = blockDim.x, tid = threadIdx.x, cvt = 1 << u.log_cvt;
  const float inv_cg = 1.0f / (float)a.Cg;
  B* const xs = (B*)smem + tid;                                                 // slot k at k * TH
  B* const rs = xs + u.slots * TH;
  float* sh = (float*)((B*)smem + (size_t)u.slots * TH * (a.res ? 2 : 1));      // [rows or warps][cvt * SL]
  float2* stat = (float2*)(sh + (u.log_cvt < 5 ? TH >> 5 : q.rows) * cvt * SL); // [groups]: mean and squares, then mean and rstd
  float2* mine = stat + u.cc / a.Cg;                                            // [groups]: what the cluster's others read
  fetch<T, V>(xs, (const T*)a.x + q.n * a.x_n + (q.p0 + q.row) * a.x_p + q.c, q.rows * a.x_p, TH, q.turns);
  copies_commit();
  if (a.res) fetch<T, V>(rs, (const T*)a.res + q.n * a.r_n + (q.p0 + q.row) * a.r_p + q.c, q.rows * a.r_p, TH, q.turns);
  copies_commit();
  float w[V], b[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { w[i] = 0.0f; b[i] = 0.0f; }
  if (q.on) { params<V>(a.w, a.ptype, q.c, 1.0f, w); params<V>(a.b, a.ptype, q.c, 0.0f, b); }
  float s1[V], s2[V], less[V], fold[SL], k1[SL], k2[SL], shift[SL];
#pragma unroll
  for (int i = 0; i < V; ++i) { s1[i] = 0.0f; s2[i] = 0.0f; less[i] = 0.0f; }
  copies_wait<1>();
  if (q.turns > 0) {
    Raw<T, V> r;
    r.b = xs[0];
    r.widen(less);
    if constexpr (WHOLE) {
      float t = less[0];
#pragma unroll
      for (int i = 1; i < V; ++i) t += less[i];
#pragma unroll
      for (int i = 0; i < V; ++i) less[i] = t * (1.0f / V);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) less[i] = fabsf(less[i]) <= 3e38f ? -less[i] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < SL; ++i) shift[i] = -less[i];
#pragma unroll 4
  for (int k = 0; k < q.turns; ++k) {
    float v[V];
    Raw<T, V> r;
    r.b = xs[k * TH];
    r.widen(v);
    vadd<V>(v, v, less);
    vadd<V>(s1, s1, v);
    vfma<V>(s2, v, v, s2);
  }
  // k1: the thread's mean about its shift, k2: its squares about that mean; the block's mean of each group
  const int per = WHOLE ? a.Cg / V : a.Cg, pitch = cvt * SL;
  const float count = (float)(WHOLE ? q.turns * V : q.turns), inv_count = q.turns > 0 ? 1.0f / count : 0.0f;
  narrow<V, SL>(s1, k1);
  narrow<V, SL>(s2, k2);
#pragma unroll
  for (int i = 0; i < SL; ++i) {
    fold[i] = __fmaf_rn(count, shift[i], k1[i]);
    const float m = k1[i] * inv_count;
    k2[i] = __fmaf_rn(-m, k1[i], k2[i]);
    k1[i] = m;
  }
  int left = fold_rows<SL>(fold, sh, u.log_cvt);
  const float inv = q.all > 0 ? 1.0f / ((float)q.all * (float)a.Cg) : 0.0f;
  fold_groups(sh, left, pitch, per, q.groups, [&](int j, float s) { stat[j].x = s * inv; });
  __syncthreads();
  // the squares about it
#pragma unroll
  for (int i = 0; i < SL; ++i) {
    const float d = q.on ? (shift[i] - stat[quotient(q.co + i, inv_cg)].x) + k1[i] : 0.0f;
    fold[i] = __fmaf_rn(count * d, d, k2[i]);
  }
  left = fold_rows<SL>(fold, sh, u.log_cvt);
  fold_groups(sh, left, pitch, per, q.groups, [&](int j, float s) { mine[j] = make_float2(stat[j].x, s); });
  // joined over the cluster
  cg::cluster_group cluster = cg::this_cluster();
  if (u.S > 1) cluster.sync(); else __syncthreads();
  const float M = (float)a.P * (float)a.Cg;
  for (int j = tid; j < q.groups; j += TH) {
    float2 r = mine[j];
    if (u.S > 1) {
      float s = 0.0f;
      for (int k = 0; k < u.S; ++k) s += (float)max(0, min(u.px, a.P - k * u.px)) * cluster.map_shared_rank(mine, k)[j].x;
      const float m = s * (float)a.Cg / M;
      float m2 = 0.0f;
      for (int k = 0; k < u.S; ++k) {
        const float2 o = cluster.map_shared_rank(mine, k)[j];
        const float d = o.x - m;
        m2 += o.y + (float)max(0, min(u.px, a.P - k * u.px)) * (float)a.Cg * d * d;
      }
      r = make_float2(m, m2);
    }
    r.y = __fdiv_rn(1.0f, __fsqrt_rn(r.y / M + a.eps));
    stat[j] = r;
    if (q.rank == 0) { const long long g = (long long)q.n * a.G + q.c0 / a.Cg + j; a.mean[g] = r.x; a.rstd[g] = r.y; }
  }
  __syncthreads();
  if (u.S > 1) cluster.barrier_arrive();            // this block has read what it needs of the others
  copies_wait<0>();
  Per<V, WHOLE> mean, rstd;
  mean.set([&](int i) { return q.on ? stat[quotient(q.co + i, inv_cg)].x : 0.0f; });
  rstd.set([&](int i) { return q.on ? stat[quotient(q.co + i, inv_cg)].y : 0.0f; });
  float scale[V];
  mean.all(less);
  rstd.all(scale);
#pragma unroll
  for (int i = 0; i < V; ++i) less[i] = -less[i];
  T* y = (T*)a.out + ((long long)q.n * a.P + q.p0 + q.row) * a.C + q.c;
  const long long step = (long long)q.rows * a.C;
  const int act = a.act;
#pragma unroll 2
  for (int k = 0; k < q.turns; ++k, y += step) {
    float z[V];
    Raw<T, V> r;
    r.b = xs[k * TH];
    r.widen(z);
    vadd<V>(z, z, less);
    vmul<V>(z, z, scale);
    vmul<V>(z, z, w);
    vadd<V>(z, z, b);
    if (a.res) {
      float v[V];
      r.b = rs[k * TH];
      r.widen(v);
      vadd<V>(z, z, v);
    }
    activate<T, V>(z, act);
    r.round(z);
    r.store(y);
  }
  if (u.S > 1) cluster.barrier_wait();              // nobody leaves while another may still read its sums
}

// V floats of a 16-bit type's slots, half of their bytes in each of two.
template <typename T, int V>
__device__ __forceinline__ void hold(typename Raw<T, V>::B* lo, typename Raw<T, V>::B* hi, const float (&v)[V]) {
  if constexpr (sizeof(T) == 2) {
    typename Raw<T, V>::B b[2];
    if constexpr (V == 8) {
      b[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      b[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else if constexpr (V == 2) {
      b[0] = __float_as_uint(v[0]); b[1] = __float_as_uint(v[1]);
    } else {
      b[0] = (unsigned short)(__float_as_uint(v[0]) & 0xffffu); b[1] = (unsigned short)(__float_as_uint(v[0]) >> 16);
    }
    *lo = b[0]; *hi = b[1];
  }
}
template <typename T, int V>
__device__ __forceinline__ void held(const typename Raw<T, V>::B* lo, const typename Raw<T, V>::B* hi, float (&v)[V]) {
  if constexpr (sizeof(T) == 2) {
    const typename Raw<T, V>::B a = *lo, b = *hi;
    if constexpr (V == 8) {
      v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
      v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
    } else if constexpr (V == 2) {
      v[0] = __uint_as_float(a); v[1] = __uint_as_float(b);
    } else {
      v[0] = __uint_as_float((unsigned int)a | ((unsigned int)b << 16));
    }
  }
}

// xhat and dz of a vector.
template <typename T, int V>
__device__ __forceinline__ void unit_grad(Raw<T, V> x, Raw<T, V> d, const typename Raw<T, V>::B* res, const float (&less)[V], const float (&scale)[V],
                                          const float (&w)[V], const float (&b)[V], int act, float (&xh)[V], float (&dz)[V]) {
  float z[V];
  x.widen(xh);
  d.widen(dz);
  vadd<V>(xh, xh, less);
  vmul<V>(xh, xh, scale);
  if (act == SAE_ACT_NONE) return;
  vmul<V>(z, xh, w);
  vadd<V>(z, z, b);
  if (res) {
    Raw<T, V> r;
    float v[V];
    r.b = *res;
    r.widen(v);
    vadd<V>(z, z, v);
  }
  slope<T, V>(dz, z, act);
}

// Adds up 2 V values a lane over the lanes whose numbers differ in the bits above log_cvt: in each round a lane hands half of
// its values to the partner and takes the partner's other half, so the work halves from round to round.  Afterwards values
// v[0 .. left) of a lane are the sums of the values from `from` on; `left` is returned.  The order is fixed.
template <int W>
__device__ __forceinline__ int scatter_sum(float (&v)[W], int log_cvt, int& from) {
  const int lane = threadIdx.x & 31;
  int left = W;
  from = 0;
#pragma unroll
  for (int r = 0; r < 5; ++r) {
    const int o = 16 >> r;
    if (o < (1 << log_cvt)) break;
    const bool upper = (lane & o) != 0;
    if ((W >> r) >= 2) {
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        if (i < (W >> r) / 2) {
          const float keep = upper ? v[i + (W >> r) / 2] : v[i], give = upper ? v[i] : v[i + (W >> r) / 2];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
      left = (W >> r) / 2;
      if (upper) from += left;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
  return left;
}

// After the first pass a thread's dz stays in its slots: a 16-bit dz that rounding does not change (relu's, none's) in dy's
// place, else in float, which for 16-bit types takes a second slot (the residual's, if there is one).
template <typename T, int V, bool WHOLE>
__global__ void __launch_bounds__(GN_THREADS, WHOLE ? 3 : 2) k_gn_grad_unit(const Args a, const Unit u) {
  extern __shared__ __align__(16) unsigned char smem[];
  typedef typename Raw<T, V>::B B;
  const Spot q = spot<V>(a, u);
  if (q.n >= a.N) return;
  const int TH = blockDim.x, tid = threadIdx.x, cvt = 1 << u.log_cvt, groups = q.groups;
  const float inv_cg = 1.0f / (float)a.Cg;
  const int act = a.act;
  const bool wide = sizeof(T) == 2 && act >= SAE_ACT_SILU, second = wide || a.res != nullptr;
  B* const xs = (B*)smem + tid;
  B* const ds = xs + u.slots * TH;
  B* const rs = ds + u.slots * TH;
  float* sh = (float*)((B*)smem + (size_t)u.slots * TH * (second ? 3 : 2));     // [2][rows or warps][cvt * V]
  const int left = u.log_cvt < 5 ? TH >> 5 : q.rows, pitch = cvt * V, span = left * pitch;
  float2* mine = (float2*)(sh + 2 * span);                                      // [cc]: the block's sums of each channel
  float2* chan = mine + u.cc;                                                   // [cc]: the unit's, times the weight
  float2* grp = chan + u.cc;                                                    // [groups]: the two means
  fetch<T, V>(xs, (const T*)a.x + q.n * a.x_n + (q.p0 + q.row) * a.x_p + q.c, q.rows * a.x_p, TH, q.turns);
  fetch<T, V>(ds, (const T*)a.dy + q.n * a.d_n + (q.p0 + q.row) * a.d_p + q.c, q.rows * a.d_p, TH, q.turns);
  if (a.res) fetch<T, V>(rs, (const T*)a.res + q.n * a.r_n + (q.p0 + q.row) * a.r_p + q.c, q.rows * a.r_p, TH, q.turns);
  copies_commit();
  Per<V, WHOLE> mean, rstd;
  float w[V], b[V], less[V], scale[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { w[i] = 0.0f; b[i] = 0.0f; }
  if (q.on) { params<V>(a.w, a.ptype, q.c, 1.0f, w); params<V>(a.b, a.ptype, q.c, 0.0f, b); }
  const float* const gm = a.mean + (long long)q.n * a.G + q.c0 / a.Cg;
  const float* const gr = a.rstd + (long long)q.n * a.G + q.c0 / a.Cg;
  mean.set([&](int i) { return q.on ? __ldg(gm + quotient(q.co + i, inv_cg)) : 0.0f; });
  rstd.set([&](int i) { return q.on ? __ldg(gr + quotient(q.co + i, inv_cg)) : 0.0f; });
  mean.all(less);
  rstd.all(scale);
#pragma unroll
  for (int i = 0; i < V; ++i) less[i] = -less[i];
  float s[2 * V];                                   // sum dz, then sum dz * xhat
  {
    float s0[V], sx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { s0[i] = 0.0f; sx[i] = 0.0f; }
    T* dres = a.dres ? (T*)a.dres + ((long long)q.n * a.P + q.p0 + q.row) * a.C + q.c : nullptr;
    const long long step = (long long)q.rows * a.C;
    copies_wait<0>();
#pragma unroll 2
    for (int k = 0; k < q.turns; ++k) {
      float xh[V], dz[V];
      Raw<T, V> x, d;
      x.b = xs[k * TH];
      d.b = ds[k * TH];
      unit_grad<T, V>(x, d, a.res ? rs + k * TH : nullptr, less, scale, w, b, act, xh, dz);
      vadd<V>(s0, s0, dz);
      vfma<V>(sx, dz, xh, sx);
      if (act != SAE_ACT_NONE) {
        d.round(dz);
        if (wide) hold<T, V>(ds + k * TH, rs + k * TH, dz);
        else ds[k * TH] = d.b;
      }
      if (dres) { d.store(dres); dres += step; }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) { s[i] = s0[i]; s[V + i] = sx[i]; }
  }
  {
    int from, n = scatter_sum<2 * V>(s, u.log_cvt, from);
    const int at = (u.log_cvt < 5 ? tid >> 5 : q.row) * pitch + (tid & (cvt - 1)) * V;
#pragma unroll
    for (int i = 0; i < 2 * V; ++i)
      if (i < n) { const int j = from + i; sh[(j >= V ? span - V : 0) + at + j] = s[i]; }
  }
  __syncthreads();
  for (int i = tid; i < 2 * pitch; i += TH) {       // one thread a sum
    const bool x = i >= pitch;
    const int j = x ? i - pitch : i;
    const float* from = sh + (x ? span : 0) + j;
    float t = 0.0f;
#pragma unroll 4
    for (int r = 0; r < left; ++r) t += from[r * pitch];
    if (j < q.cc) ((float*)&mine[j])[x ? 1 : 0] = t;
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (u.S > 1) cluster.sync(); else __syncthreads();
  for (int i = tid; i < q.cc; i += TH) {
    float2 t = mine[i];
    if (u.S > 1) {
      t = make_float2(0.0f, 0.0f);
      for (int k = 0; k < u.S; ++k) { const float2 o = cluster.map_shared_rank(mine, k)[i]; t.x += o.x; t.y += o.y; }
    }
    if (q.rank == 0) { const long long at = (long long)q.n * a.C + q.c0 + i; a.part_a[at] = t.x; a.part_b[at] = t.y; }
    const float wi = param(a.w, a.ptype, q.c0 + i, 1.0f);
    chan[i] = make_float2(t.x * wi, t.y * wi);
  }
  __syncthreads();
  if (u.S > 1) cluster.barrier_arrive();
  const float M = (float)a.P * (float)a.Cg;
  for (int j = tid >> 5; j < groups; j += TH >> 5) {
    float p = 0.0f, t = 0.0f;
    for (int i = tid & 31; i < a.Cg; i += 32) { const float2 o = chan[j * a.Cg + i]; p += o.x; t += o.y; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { p += __shfl_xor_sync(0xffffffffu, p, o); t += __shfl_xor_sync(0xffffffffu, t, o); }
    if ((tid & 31) == 0) grp[j] = make_float2(-(p / M), -(t / M));
  }
  __syncthreads();
  // dx = rstd * (dz * w - mean(g) - xhat * mean(g * xhat)) = dz * (w rstd) + ((x - mean) * (-rstd^2 mean(g xhat)) - rstd mean(g))
  Per<V, WHOLE> m1, m2;
  m1.set([&](int i) { return q.on ? grp[quotient(q.co + i, inv_cg)].x * rstd.at(i) : 0.0f; });
  m2.set([&](int i) { return q.on ? grp[quotient(q.co + i, inv_cg)].y * rstd.at(i) * rstd.at(i) : 0.0f; });
  vmul<V>(w, w, scale);
  T* dx = (T*)a.out + ((long long)q.n * a.P + q.p0 + q.row) * a.C + q.c;
  const long long step = (long long)q.rows * a.C;
#pragma unroll 2
  for (int k = 0; k < q.turns; ++k, dx += step) {
    float v[V], dz[V], p[V], t[V];
    Raw<T, V> x, d;
    x.b = xs[k * TH];
    x.widen(v);
    if (wide) held<T, V>(ds + k * TH, rs + k * TH, dz);
    else { d.b = ds[k * TH]; d.widen(dz); }
    m2.all(p);
    m1.all(t);
    vadd<V>(v, v, less);
    vfma<V>(v, v, p, t);
    vfma<V>(dz, dz, w, v);
    x.round(dz);
    x.store(dx);
  }
  if (u.S > 1) cluster.barrier_wait();
}

// ---- host -----------------------------------------------------------------------------------------------------------
struct Plan {
  int vec, cvt, ctiles, slices;
  bool unit;                             // one pass: `u`, `threads` and `smem`; else two
  Unit u;
  int threads;
  size_t smem, bytes;
};

int elem(int type) { return type == SAE_TYPE_FLOAT ? 4 : 2; }
bool type_ok(int t) { return t == SAE_TYPE_FLOAT || t == SAE_TYPE_BFLOAT || t == SAE_TYPE_HALF; }

bool desc_ok(const sae_group_norm_desc* d) {
  if (!d || !type_ok(d->type) || !type_ok(d->param_type) || d->activation < SAE_ACT_NONE || d->activation > SAE_ACT_GELU) return false;
  if (d->samples < 0 || d->samples > (1 << 24) || d->pixels < 0 || d->pixels > (1ll << 30) || d->channels < 1 || d->channels > (1 << 20)) return false;
  if (d->groups < 1 || d->channels % d->groups || !(d->eps >= 0.0f) || d->samples * d->groups > 0x7fffffffll) return false;
  const long long s[6] = {d->x_sample, d->x_pixel, d->residual_sample, d->residual_pixel, d->dy_sample, d->dy_pixel};
  for (long long v : s) if (v < 0) return false;
  return true;
}

// Sixteen bytes at a time where every tensor of the call lets it (base, strides and the channel count), else four, else one element.
int vector_width(const sae_group_norm_desc* d, const void* const* ptrs, int n) {
  const int es = elem(d->type);
  uintptr_t m = 0;
  for (int i = 0; i < n; ++i) m |= reinterpret_cast<uintptr_t>(ptrs[i]);
  const long long s = d->x_sample | d->x_pixel | d->residual_sample | d->residual_pixel | d->dy_sample | d->dy_pixel | d->channels;
  m |= (uintptr_t)(s * es);
  return (m & 15) == 0 ? 16 / es : es == 2 && (m & 3) == 0 ? 2 : 1;
}

#ifdef SAE_GN_TUNE
#include <cstdlib>
int tune(const char* name, int otherwise) { const char* v = getenv(name); return v ? atoi(v) : otherwise; }
#else
int tune(const char*, int otherwise) { return otherwise; }
#endif

constexpr int SMEM_BLOCK = 227 * 1024;

// One pass over a unit of `seg` bytes a pixel or a little less (whole groups, whole vectors), in clusters of up to `most` blocks
// of up to `room` bytes; false if the unit does not fit.
bool unit_plan(const sae_group_norm_desc* d, int vec, int tensors, bool backward, int seg, int most, size_t room, int sms, Plan& p) {
  const int es = elem(d->type), VB = vec * es, cg_ = (int)(d->channels / d->groups);
  int step = cg_;
  while (step % vec) step += cg_;                                  // whole groups and whole vectors
  if (step > d->channels) return false;
  long long cc = std::max(1, seg / (step * es)) * (long long)step;
  cc = std::min<long long>(cc, d->channels);
  int log = 0;
  while ((1ll << log) * vec < cc) ++log;
  const int cvt = 1 << log;
  if (cvt > GN_THREADS) return false;
  cc = std::min<long long>(d->channels, (long long)cvt * vec / step * step);      // fill the lanes
  const long long vectors = d->pixels * cvt;
  int th = tune("GN_THREADS", 256);
  while (th > 64 && vectors < th * 2ll) th /= 2;
  th = std::max(th, cvt);
  if (th < 32) th = 32;
  const int rows = th >> log, SL = vec;
  const size_t fixed = (size_t)(log < 5 ? th / 32 : rows) * cvt * SL * 4 * (backward ? 2 : 1) + (size_t)cc * 8 * 3 + 64;
  if (fixed >= room) return false;
  const long long slots_most = (long long)((room - fixed) / ((size_t)th * VB * tensors));
  if (slots_most < 1) return false;
  long long S = (d->pixels + slots_most * rows - 1) / (slots_most * rows);
  if (S > most) return false;
  // few units: shorter runs over more blocks, as long as a thread keeps two vectors
  const int chunks = (int)((d->channels + cc - 1) / cc);
  const long long units = (long long)d->samples * chunks;
  while (S * 2 <= std::min(most, 8) && units * S * 2 <= sms * 2 && d->pixels >= S * 2 * rows * 2) S *= 2;
  Unit& u = p.u;
  u.log_cvt = log; u.cc = (int)cc; u.chunks = chunks; u.S = (int)S;
  u.px = (int)((d->pixels + S - 1) / S);
  u.slots = (u.px + rows - 1) / rows;
  p.unit = true;
  p.threads = th;
  p.smem = fixed + (size_t)u.slots * th * VB * tensors;
  return true;
}

Plan make_plan(const sae_group_norm_desc* d, int vec, bool backward, bool residual, int sms) {
  Plan p = {};
  p.vec = vec;
  // backward: a second slot for dz in float where its type cannot hold it
  const bool second = residual || (backward && elem(d->type) == 2 && d->activation >= SAE_ACT_SILU);
  const int tensors = (backward ? 2 : 1) + (second ? 1 : 0);
  const int segs[3] = {tune("GN_SEG", 128), 64, 32};
  for (int i = 0; i < 3 && !p.unit; ++i) unit_plan(d, vec, tensors, backward, segs[i], 8, (size_t)tune("GN_ROOM", 72) * 1024, sms, p);
  for (int i = 0; i < 3 && !p.unit; ++i) unit_plan(d, vec, tensors, backward, segs[i], 8, (size_t)SMEM_BLOCK / 2 - 1024, sms, p);
  if (tune("GN_SPLIT", 0)) p.unit = false;
  if (p.unit) {
    p.slices = 1;
    p.bytes = backward ? (size_t)2 * 4 * d->samples * d->channels : 0;
    return p;
  }
  const int cv = (int)((d->channels + vec - 1) / vec);
  p.ctiles = (cv + GN_THREADS - 1) / GN_THREADS;
  p.cvt = (cv + p.ctiles - 1) / p.ctiles;
  const int rows = GN_THREADS / p.cvt;
  const long long blocks = (long long)d->samples * p.ctiles;
  // enough blocks to fill the SMs, but at least four batches of pixels for a thread
  const long long want = std::max<long long>(1, ((long long)sms * 8 + blocks - 1) / std::max<long long>(1, blocks));
  const long long most = std::max<long long>(1, d->pixels / ((long long)rows * GN_BATCH * 4));
  p.slices = (int)std::min<long long>(1024, std::min(want, most));
  p.bytes = (size_t)2 * 4 * ((size_t)d->samples * p.slices * d->channels + (size_t)d->samples * d->groups);
  return p;
}

int device_sms() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return sms;
}

Args make_args(const sae_group_norm_desc* d, const Plan& p, void* ws) {
  Args a = {};
  a.x_n = d->x_sample; a.x_p = d->x_pixel; a.r_n = d->residual_sample; a.r_p = d->residual_pixel; a.d_n = d->dy_sample; a.d_p = d->dy_pixel;
  a.N = (int)d->samples; a.P = (int)d->pixels; a.C = (int)d->channels; a.G = d->groups; a.Cg = a.C / a.G;
  a.act = d->activation; a.ptype = d->param_type; a.eps = d->eps;
  a.slices = p.slices; a.cvt = p.cvt;
  float* f = (float*)ws;
  const size_t n = (size_t)a.N * a.slices * a.C, g = (size_t)a.N * a.G;
  a.part_a = f; a.part_b = f + n; a.mean_g = f + 2 * n; a.mean_gx = f + 2 * n + g;
  return a;
}

int launched() {
  return cudaGetLastError() == cudaSuccess ? SAE_OK : SAE_ERR_CUDA;
}

// A unit kernel in clusters of S blocks.  Its shared memory needs an opt-in above 48 KB, once a device and kernel.
template <void (*KERNEL)(const Args, const Unit)>
int launch_units(const Args& a, const Plan& p, cudaStream_t st) {
  static thread_local int opted = -1;               // one variable for each kernel
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
  if (opted != dev) {
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BLOCK) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
    opted = dev;
  }
  cudaLaunchConfig_t cfg = {};
  const int ny = std::min(a.N, 32768);
  cfg.gridDim = dim3((unsigned)(p.u.chunks * p.u.S), (unsigned)ny, (unsigned)((a.N + ny - 1) / ny));
  cfg.blockDim = dim3((unsigned)p.threads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)p.u.S, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, KERNEL, a, p.u) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
  return SAE_OK;
}

template <typename T, int V>
int forward(const Args& a, const Plan& p, cudaStream_t st) {
  if (p.unit) {
    if (V > 1 && a.Cg % V == 0) return launch_units<k_gn_unit<T, V, true>>(a, p, st);
    return launch_units<k_gn_unit<T, V, false>>(a, p, st);
  }
  const dim3 grid((unsigned)(a.N * p.slices), (unsigned)p.ctiles);
  const long long warps = (long long)a.N * a.G;
  k_gn_statistics<T, V><<<grid, GN_THREADS, (2 * V + 1) * GN_THREADS * sizeof(float), st>>>(a);
  k_gn_finish_statistics<<<(unsigned)((warps * 32 + GN_THREADS - 1) / GN_THREADS), GN_THREADS, 0, st>>>(a);
  k_gn_apply<T, V><<<grid, GN_THREADS, 0, st>>>(a);
  return launched();
}

template <typename T, int V>
int backward(const Args& a, const Plan& p, cudaStream_t st) {
  if (p.unit) {
    const int rc = V > 1 && a.Cg % V == 0 ? launch_units<k_gn_grad_unit<T, V, true>>(a, p, st) : launch_units<k_gn_grad_unit<T, V, false>>(a, p, st);
    if (rc != SAE_OK) return rc;
    if (a.dw || a.db) k_gn_param_grads<<<(unsigned)((a.C + 31) / 32), 1024, 0, st>>>(a, a.N);
    return launched();
  }
  const dim3 grid((unsigned)(a.N * p.slices), (unsigned)p.ctiles);
  const long long warps = (long long)a.N * a.G;
  k_gn_grad_sums<T, V><<<grid, GN_THREADS, 2 * V * GN_THREADS * sizeof(float), st>>>(a);
  k_gn_finish_grad<<<(unsigned)((warps * 32 + GN_THREADS - 1) / GN_THREADS), GN_THREADS, 0, st>>>(a);
  if (a.dw || a.db) k_gn_param_grads<<<(unsigned)((a.C + 31) / 32), 1024, 0, st>>>(a, a.N * a.slices);
  k_gn_grad_apply<T, V><<<grid, GN_THREADS, 0, st>>>(a);
  return launched();
}

// An element type and a vector width as template arguments.
#define GN_DISPATCH16(fn, T, vec, ...) ((vec) == 8 ? fn<T, 8>(__VA_ARGS__) : (vec) == 2 ? fn<T, 2>(__VA_ARGS__) : fn<T, 1>(__VA_ARGS__))
#define GN_DISPATCH(fn, type, vec, ...)                                                                  \
  ((type) == SAE_TYPE_FLOAT ? ((vec) == 4 ? fn<float, 4>(__VA_ARGS__) : fn<float, 1>(__VA_ARGS__))        \
   : (type) == SAE_TYPE_BFLOAT ? GN_DISPATCH16(fn, __nv_bfloat16, vec, __VA_ARGS__) : GN_DISPATCH16(fn, __half, vec, __VA_ARGS__))

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

extern "C" {

int64_t sae_group_norm_workspace(const sae_group_norm_desc* d, int32_t backward) {
  if (!desc_ok(d)) return -1;
  const int sms = device_sms();
  if (sms < 1) return -1;
  if (d->samples == 0 || d->pixels == 0) return 0;
  // the tensors' alignment and whether there is a residual are not known yet: the most that any form needs
  size_t most = 0;
  const int widths[3] = {16 / elem(d->type), 2, 1};
  for (int i = 0; i < 3; ++i) {
    if ((i == 1 && elem(d->type) == 4) || d->channels % widths[i]) continue;
    for (int r = 0; r < 2; ++r) most = std::max(most, make_plan(d, widths[i], backward != 0, r != 0, sms).bytes);
  }
  return (int64_t)most;
}

int sae_group_norm_forward(const sae_group_norm_desc* d, const void* x, const void* residual, const void* weight, const void* bias,
                           void* y, float* mean, float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc_ok(d)) return SAE_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->samples == 0) return SAE_OK;
  if (!mean || !rstd) return SAE_ERR_INVALID_ARG;
  if (d->pixels == 0) {                     // the mean of nothing
    const size_t g = (size_t)d->samples * d->groups * sizeof(float);
    return cudaMemsetAsync(mean, 0xff, g, st) == cudaSuccess && cudaMemsetAsync(rstd, 0xff, g, st) == cudaSuccess ? SAE_OK : SAE_ERR_CUDA;
  }
  const int es = elem(d->type);
  if (!x || !y || !aligned_to(x, es) || !aligned_to(y, es) || !aligned_to(residual, es) || !aligned_to(weight, elem(d->param_type)) ||
      !aligned_to(bias, elem(d->param_type))) return SAE_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms < 1) return SAE_ERR_CUDA;
  const void* ptrs[3] = {x, y, residual};
  const Plan p = make_plan(d, vector_width(d, ptrs, 3), false, residual != nullptr, sms);
  if ((p.bytes && !workspace) || !aligned_to(workspace, 16) || workspace_bytes < p.bytes || (long long)d->samples * p.slices > 0x7fffffffll) return SAE_ERR_INVALID_ARG;
  Args a = make_args(d, p, workspace);
  a.x = x; a.res = residual; a.w = weight; a.b = bias; a.out = y; a.mean = mean; a.rstd = rstd;
  return GN_DISPATCH(forward, d->type, p.vec, a, p, st);
}

int sae_group_norm_backward(const sae_group_norm_desc* d, const void* dy, const void* x, const void* residual, const float* mean,
                            const float* rstd, const void* weight, const void* bias, void* dx, void* dresidual, void* dweight,
                            void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc_ok(d)) return SAE_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->samples == 0 || d->pixels == 0) {  // sums of nothing
    const size_t c = (size_t)d->channels * elem(d->param_type);
    if (dweight && cudaMemsetAsync(dweight, 0, c, st) != cudaSuccess) return SAE_ERR_CUDA;
    if (dbias && cudaMemsetAsync(dbias, 0, c, st) != cudaSuccess) return SAE_ERR_CUDA;
    return SAE_OK;
  }
  const int es = elem(d->type), ps = elem(d->param_type);
  if (!dy || !x || !mean || !rstd || !dx || !aligned_to(dy, es) || !aligned_to(x, es) || !aligned_to(residual, es) || !aligned_to(dx, es) ||
      !aligned_to(dresidual, es) || !aligned_to(weight, ps) || !aligned_to(bias, ps) || !aligned_to(dweight, ps) || !aligned_to(dbias, ps))
    return SAE_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms < 1) return SAE_ERR_CUDA;
  const void* ptrs[5] = {dy, x, residual, dx, dresidual};
  const Plan p = make_plan(d, vector_width(d, ptrs, 5), true, residual != nullptr, sms);
  if ((p.bytes && !workspace) || !aligned_to(workspace, 16) || workspace_bytes < p.bytes || (long long)d->samples * p.slices > 0x7fffffffll) return SAE_ERR_INVALID_ARG;
  Args a = make_args(d, p, workspace);
  a.x = x; a.dy = dy; a.res = residual; a.w = weight; a.b = bias; a.out = dx; a.dres = dresidual; a.dw = dweight; a.db = dbias;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  return GN_DISPATCH(backward, d->type, p.vec, a, p, st);
}

}  // extern "C"
