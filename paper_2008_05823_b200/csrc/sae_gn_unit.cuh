// Group norm in one pass: thread block clusters that keep whole groups in shared memory.
#pragma once
#include "sae_gn_common.cuh"

#include <cooperative_groups.h>

namespace sae {

namespace cg = cooperative_groups;

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

// A thread's `turns` vectors, `step` elements apart, into its slots.
template <typename T, int V>
__device__ __forceinline__ void fetch(typename Raw<T, V>::B* to, const T* from, long long step, int pitch, int turns) {
  if constexpr (V * sizeof(T) >= 4) {
#pragma unroll 4
    for (int k = 0; k < turns; ++k, from += step) copy_async<V * (int)sizeof(T)>(to + k * pitch, from);
  } else {                                // no asynchronous copy of two bytes: eight loads, then eight stores
    for (int k = 0; k < turns; k += 8) {
      typename Raw<T, V>::B b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i, from += step)
        if (k + i < turns) b[i] = __ldg((const typename Raw<T, V>::B*)from);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < turns) to[(k + i) * pitch] = b[i];
    }
  }
}

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
// Bound by latency (load, reduce, store in turns; two or three blocks an SM overlap them in part), inputs in L2: 128x32x32x16
// float, 17 MB in 6.8 us; 16x14x14x1024 bf16 with a residual, 19 MB in 6.8.
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
    vmul_add<V>(z, z, w, b);
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

// After the first pass a thread's dz stays in its slots: a 16-bit dz that rounding does not change (relu's, none's) in dy's
// place, else in float, which for 16-bit types takes a second slot (the residual's, if there is one).
// Bound by latency as the forward kernel: 128x32x32x16 float, 25 MB in 8.0 us; 16x14x14x1024 bf16 with a residual, 32 MB in 10.
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
      Raw<T, V> x, d, r;
      x.b = xs[k * TH];
      d.b = ds[k * TH];
      if (a.res) r.b = rs[k * TH];
      vector_grad<T, V>(x, d, a.res ? &r : nullptr, less, scale, w, b, act, xh, dz);
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

}  // namespace sae
