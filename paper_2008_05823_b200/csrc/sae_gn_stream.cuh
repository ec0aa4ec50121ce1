// Group norm in two passes: streaming kernels for tensors too large to stay on chip.  The second pass runs backwards, so that
// it begins with what the first one read last and L2 still holds.
//
// Where the channel count is no multiple of a 16-byte vector but the tensors have no gaps, `rep` neighbouring pixels make one
// row of vectors: channel c of it is channel c mod C, and everything below works on rows of rep * C channels.
#pragma once
#include "sae_gn_common.cuh"

namespace sae {

struct Stream {
  int n0;                                // first sample of this launch
  int rep, vc;                           // pixels of a row (Args::P and the pixel strides count rows), its channels rep * C
  int slices, px;                        // runs of rows a sample is cut into, rows of one
  int cvt, tiles, tile_groups;           // vectors of a pixel a block takes, tiles of them in a pixel, groups a tile touches at most
  int param_z;                           // backward apply: leading layers of the grid that sum up dw and db
  bool held;                             // backward sums: the second pass reads dresidual instead of dy and the residual
};

// What a thread stands for: V channels from c on, pixels p, p + rows, .. below p1.  grid: (slices, tiles, samples).
struct Place {
  int n, slice, c, p, p1, rows, row;
  bool on;
};
template <int V>
__device__ __forceinline__ Place place(const Args& a, const Stream& s) {
  Place q;
  q.n = s.n0 + (int)blockIdx.z - s.param_z;
  q.slice = blockIdx.x;
  q.rows = GN_THREADS / s.cvt;
  q.row = threadIdx.x / s.cvt;
  q.c = (blockIdx.y * s.cvt + (threadIdx.x - q.row * s.cvt)) * V;
  q.on = q.row < q.rows && q.c < s.vc;
  q.p = q.slice * s.px + q.row;
  q.p1 = min(a.P, (q.slice + 1) * s.px);
  return q;
}
__device__ __forceinline__ int run_pixels(const Args& a, const Stream& s, int i) { return s.rep * min(s.px, a.P - i * s.px); }

// Channels of a row and their groups.
struct Channel {
  float inv_c, inv_cg;
  int C;
  bool rows;
  __device__ __forceinline__ Channel(const Args& a, const Stream& s) : inv_c(1.0f / (float)a.C), inv_cg(1.0f / (float)a.Cg), C(a.C), rows(s.rep > 1) {}
  __device__ __forceinline__ int of(int c) const { return rows ? c - C * quotient(c, inv_c) : c; }
  __device__ __forceinline__ int group(int c) const { return quotient(of(c), inv_cg); }
};
template <int V>
__device__ __forceinline__ void row_params(const Args& a, const Channel& ch, int c, float (&w)[V], float (&b)[V]) {
  if (!ch.rows) {
    params<V>(a.w, a.ptype, c, 1.0f, w);
    params<V>(a.b, a.ptype, c, 0.0f, b);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) { w[i] = param(a.w, a.ptype, ch.of(c + i), 1.0f); b[i] = param(a.b, a.ptype, ch.of(c + i), 0.0f); }
  }
}

// A stream kernel lets its successor start as soon as all its blocks run, and itself waits, before it touches what another
// kernel of the call has written, for all of its predecessor.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// How many of its pixels a thread has on their way: up to 64 KB of a block's shared memory, with the bytes that the thread keeps
// beside them 72 KB, three blocks an SM.
__host__ __device__ constexpr int ring_depth(int bytes, int tensors, int kept = 0) {
  const int most = bytes == 16 ? (tensors == 3 ? 5 : 8) : bytes == 4 ? 16 : 24 / tensors, fit = (288 - kept) / (tensors * bytes);
  return most < fit ? most : fit;
}
__host__ __device__ constexpr size_t ring_bytes(int bytes, int tensors, int kept = 0) {
  return bytes < 4 ? 0 : (size_t)ring_depth(bytes, tensors, kept) * tensors * bytes * GN_THREADS;
}

// A thread's walk over its pixels of NT tensors, first to last or (BACK) last to first: the second pass begins with what the
// first one read last.  Copies run ahead through a ring of slots of the thread's own in shared memory, so no barrier is
// needed and the loads in flight do not depend on registers; single 16-bit elements, which have no asynchronous copy, are
// loaded in batches instead, and not as constants: a backward apply that began early reads what the sums' kernel still wrote then.
template <typename T, int V, int NT, bool BACK, int KEPT = 0>
struct Walk {
  typedef typename Raw<T, V>::B B;
  static constexpr int D = ring_depth(sizeof(B), NT, KEPT);
  const T* next[NT];
  long long step[NT];
  B* slots;
  int turns, ahead;

  __device__ __forceinline__ void set(const Place& q, void* smem) {
    turns = q.on && q.p < q.p1 ? (q.p1 - q.p - 1) / q.rows + 1 : 0;
    ahead = 0;
    slots = (B*)smem + threadIdx.x;
  }
  __device__ __forceinline__ int first(const Place& q) const { return BACK ? q.p + (turns - 1) * q.rows : q.p; }
  // Tensor t: element (n, c) of it and the stride of a pixel.
  __device__ __forceinline__ void tensor(int t, const Place& q, const T* from, long long pixel) {
    next[t] = from + first(q) * pixel;
    step[t] = (BACK ? -q.rows : q.rows) * pixel;
  }
  __device__ __forceinline__ void fetch(int slot) {
    if constexpr (sizeof(B) >= 4) {
      if (ahead < turns) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          copy_async<sizeof(B)>(slots + (slot * NT + t) * GN_THREADS, next[t]);
          next[t] += step[t];
        }
      }
      ++ahead;
      copies_commit();
    }
  }
  __device__ __forceinline__ void start() {
    if constexpr (sizeof(B) >= 4) {
#pragma unroll
      for (int k = 0; k < D - 1; ++k) fetch(k);
    }
  }
  // use(the tensors' vectors, turn) for each pixel; after every D of them after(turns so far / D).
  template <typename F>
  __device__ __forceinline__ void run(F use) { run(use, [](int) {}); }
  template <typename F, typename G>
  __device__ __forceinline__ void run(F use, G after) {
    if constexpr (sizeof(B) >= 4) {
      int rounds = 0;
      for (int k = 0; k < turns; k += D) {
#pragma unroll
        for (int j = 0; j < D; ++j) {                       // slot j; the one before it has just been used
          if (k + j >= turns) break;
          fetch((j + D - 1) % D);
          copies_wait<D - 1>();
          Raw<T, V> r[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) r[t].b = slots[(j * NT + t) * GN_THREADS];
          use(r, k + j);
        }
        after(++rounds);
      }
      copies_wait<0>();
    } else {
      int rounds = 0;
      for (int k0 = 0; k0 < turns; k0 += D) {
        Raw<T, V> r[D][NT];
#pragma unroll
        for (int k = 0; k < D; ++k) {
          if (k0 + k < turns) {
#pragma unroll
            for (int t = 0; t < NT; ++t) { r[k][t].load_written(next[t]); next[t] += step[t]; }
          }
        }
#pragma unroll
        for (int k = 0; k < D; ++k)
          if (k0 + k < turns) use(r[k], k0 + k);
        after(++rounds);
      }
    }
  }
};

// ---- a tile's groups ----------------------------------------------------------------------------------------------
struct Tile {                            // the tile's channels [lo, hi), the groups they touch
  int lo, hi, g0, groups;
};
__device__ __forceinline__ Tile tile_of(const Args& a, const Stream& s, int tile, int vec) {
  Tile t;
  t.lo = tile * s.cvt * vec;
  t.hi = min(a.C, t.lo + s.cvt * vec);
  t.g0 = t.lo / a.Cg;
  t.groups = (t.hi - 1) / a.Cg - t.g0 + 1;
  return t;
}

// Few values a group: as many groups as fit share a warp.  The lanes a group gets: a power of two, 32 at most.
__device__ __forceinline__ int lanes_for(int entries) { return entries > 16 ? 32 : entries > 8 ? 16 : entries > 4 ? 8 : entries > 2 ? 4 : 2; }

// Calls f(j, lane, lanes) for each group j of a tile with the lanes that share it (j may be past the end: take part in shuffles).
template <typename F>
__device__ __forceinline__ void each_group(const Tile& t, int entries, F f) {
  const int lanes = lanes_for(entries), sub = threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
  for (int j0 = 0; j0 < t.groups; j0 += GN_THREADS / lanes) f(j0 + sub, lane, lanes);
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sums of each group's values in sh[rows][pitch], SL of them a vector of V channels: out(j, sum, channels).  Where there are
// more values than threads, columns are added up over the rows first.  Begins with a barrier.
template <int SL, int V, typename F>
__device__ __forceinline__ void fold_tile(const Args& a, const Tile& t, float* sh, int rows, int rep, int pitch, F out) {
  __syncthreads();
  if (rep > 1) {                          // a channel's places in the row too
    for (int i = threadIdx.x; i < a.C; i += GN_THREADS) {
      float s = 0.0f;
      for (int r = 0; r < rows; ++r)
        for (int e = i; e < rep * a.C; e += a.C) s += sh[r * pitch + e];
      sh[i] = s;
    }
    rows = 1;
    __syncthreads();
  }
  if (rows > 1 && rows * pitch > GN_THREADS) {
    for (int i = threadIdx.x; i < pitch; i += GN_THREADS) {
      float s = 0.0f;
#pragma unroll 4
      for (int r = 0; r < rows; ++r) s += sh[r * pitch + i];
      sh[i] = s;
    }
    rows = 1;
    __syncthreads();
  }
  each_group(t, rows * (a.Cg * SL / V), [&](int j, int lane, int lanes) {
    const int lo = max((t.g0 + j) * a.Cg, t.lo), hi = min((t.g0 + j + 1) * a.Cg, t.hi), len = (hi - lo) * SL / V;
    float s = 0.0f;
    if (j < t.groups) {
      const float* p = sh + (lo - t.lo) * SL / V;
      if (rows == 1) {
        for (int e = lane; e < len; e += lanes) s += p[e];
      } else if (len == 1) {
        for (int e = lane; e < rows; e += lanes) s += p[e * pitch];
      } else {
        const float inv = __frcp_rn((float)len);
        for (int e = lane; e < rows * len; e += lanes) {
          const int r = quotient(e, inv);
          s += p[r * pitch + (e - r * len)];
        }
      }
    }
    s = lanes_sum(s, lanes);
    if (j < t.groups && lane == 0) out(j, s, hi - lo);
  });
}

// The tile in which a group begins.
__device__ __forceinline__ int first_tile(const Args& a, const Stream& s, int g, int vec) { return s.tiles == 1 ? 0 : g * a.Cg / (s.cvt * vec); }

// Joins the runs' pairs of every group of a tile: the threads stand side by side over the groups and, as far as there are
// more threads, over the runs.  How many stand over the runs depends on the launch alone, not on the tile's own groups: tiles
// that share a group add in the same order and get the same bits.  add(sum, pixels * channels, pair, first pair) for each run;
// done(j, sum) for each group, from one thread, before a barrier.  `sums` holds a pair for each thread.
template <typename A, typename D>
__device__ __forceinline__ void join_runs(const Args& a, const Stream& s, const Tile& tile, int n, int vec, float2* sums, A add, D done) {
  const int tile_c = s.cvt * vec;
  const float2* part = a.part_s + (long long)n * s.slices * s.tiles * s.tile_groups;
  const int across = min(s.tile_groups, GN_THREADS), subs = GN_THREADS / across, sub = quotient(threadIdx.x, __frcp_rn((float)across));
  for (int j0 = 0; j0 < tile.groups; j0 += across) {
    const int j = j0 + (int)threadIdx.x - sub * across, g = tile.g0 + j;
    float2 t = make_float2(0.0f, 0.0f);
    if (sub < subs && j < tile.groups) {
      const int t0 = first_tile(a, s, g, vec);
      if (s.tiles == 1) {
        const float2 first = __ldcg(part + g);
#pragma unroll 4
        for (int i = sub; i < s.slices; i += subs) add(t, (float)run_pixels(a, s, i) * (float)a.Cg, __ldcg(part + i * s.tile_groups + g), first);
      } else {
        const int tiles = (g * a.Cg + a.Cg - 1) / tile_c - t0 + 1;
        const float2 first = __ldcg(part + t0 * s.tile_groups + g - t0 * tile_c / a.Cg);
        for (int e = sub; e < s.slices * tiles; e += subs) {
          const int i = tiles == 1 ? e : e / tiles, k = t0 + (e - i * tiles);
          const int lo = max(g * a.Cg, k * tile_c), hi = min(min((g + 1) * a.Cg, (k + 1) * tile_c), a.C);
          add(t, (float)run_pixels(a, s, i) * (float)(hi - lo), __ldcg(part + ((long long)i * s.tiles + k) * s.tile_groups + g - k * tile_c / a.Cg), first);
        }
      }
    }
    sums[threadIdx.x] = t;
    __syncthreads();
    if (sub == 0 && j < tile.groups) {
      for (int k = 1; k < subs; ++k) { const float2 o = sums[k * across + (int)threadIdx.x]; t.x += o.x; t.y += o.y; }
      done(j, t);
    }
    __syncthreads();
  }
}
__device__ __forceinline__ float2* run_out(const Args& a, const Stream& s, const Place& q) {
  return a.part_s + (((long long)q.n * s.slices + q.slice) * s.tiles + blockIdx.y) * s.tile_groups;
}

// ---- forward ------------------------------------------------------------------------------------------------------
// A thread sums x - k and its square over at most 32 vectors, k being the first one's value (WHOLE: mean), then joins count, mean
// and squares to what came before (Chan, Golub and LeVeque's update).
// Bound by HBM and, below 100 MB, by its start and end: 51 MB of bf16 in 15 us, 7 of them before and after the loads flow.
template <typename T, int V, bool WHOLE>
__global__ void __launch_bounds__(GN_THREADS, 3) k_gn_statistics(const Args a, const Stream st) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int SL = WHOLE ? 1 : V;
  float* const sh = (float*)smem;         // after the walk: [rows][cvt * SL], then [tile_groups]
  let_next_start();
  const Place q = place<V>(a, st);
  const Channel ch(a, st);
  float count = 0.0f, mean[SL], m2[SL], s1[V], s2[V], less[V];
#pragma unroll
  for (int i = 0; i < SL; ++i) { mean[i] = 0.0f; m2[i] = 0.0f; }
  Walk<T, V, 1, false> walk;
  walk.set(q, smem);
  walk.tensor(0, q, (const T*)a.x + q.n * a.x_n + q.c, a.x_p);
  walk.start();
  auto join = [&](int run) {
    float k1[SL], k2[SL];
    narrow<V, SL>(s1, k1);
    narrow<V, SL>(s2, k2);
    const float n = (float)(WHOLE ? run * V : run), inv = __frcp_rn(n), t = count + n, f = n * __frcp_rn(t);
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      const float m = k1[i] * inv, d = (m - less[i]) - mean[i];
      m2[i] += __fmaf_rn(-m, k1[i], k2[i]) + d * d * (count * f);
      mean[i] = __fmaf_rn(d, f, mean[i]);
    }
    count = t;
  };
  walk.run([&](const Raw<T, V> (&r)[1], int k) {
    float v[V];
    r[0].widen(v);
    if ((k & 31) == 0) {
      if (k) join(32);
#pragma unroll
      for (int i = 0; i < V; ++i) { s1[i] = 0.0f; s2[i] = 0.0f; less[i] = v[i]; }
      if constexpr (WHOLE && V > 1) {
        float t = v[0];
#pragma unroll
        for (int i = 1; i < V; ++i) t += v[i];
#pragma unroll
        for (int i = 0; i < V; ++i) less[i] = t * (1.0f / V);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) less[i] = fabsf(less[i]) <= 3e38f ? -less[i] : 0.0f;
    }
    vadd<V>(v, v, less);
    vadd<V>(s1, s1, v);
    vfma<V>(s2, v, v, s2);
  });
  if (walk.turns > 0) join(((walk.turns - 1) & 31) + 1);
  __syncthreads();                        // everybody is through with the ring
  // the block's mean of each group of its tile, then the squares about it
  const Tile tile = tile_of(a, st, blockIdx.y, V);
  const int pitch = st.cvt * SL, slot = q.row * pitch + (threadIdx.x - q.row * st.cvt) * SL;
  const float inv_pixels = 1.0f / (float)run_pixels(a, st, q.slice);
  float* const gmean = sh + q.rows * pitch;
  if (q.row < q.rows) {
#pragma unroll
    for (int i = 0; i < SL; ++i) sh[slot + i] = q.on ? count * mean[i] : 0.0f;
  }
  fold_tile<SL, V>(a, tile, sh, q.rows, st.rep, pitch, [&](int j, float s, int channels) { gmean[j] = s * inv_pixels * __frcp_rn((float)channels); });
  __syncthreads();
  if (q.row < q.rows) {
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      float v = 0.0f;
      if (q.on) { const float d = mean[i] - gmean[ch.group(q.c + i) - tile.g0]; v = __fmaf_rn(count * d, d, m2[i]); }
      sh[slot + i] = v;
    }
  }
  float2* const out = run_out(a, st, q);
  wait_for_previous();
  fold_tile<SL, V>(a, tile, sh, q.rows, st.rep, pitch, [&](int j, float s, int) { out[j] = make_float2(gmean[j], s); });
}

// act(z) with the tile's statistics joined first by every block (a launch of its own for that cost 4 to 6 us).  Bound by HBM:
// 32x56x56x256 bf16 with a residual, 154 MB in 24.5 us from a cold L2 (6.3 TB/s), about 20 behind the statistics.
template <typename T, int V, bool WHOLE, bool RES>
__global__ void __launch_bounds__(GN_THREADS, 3) k_gn_apply(const Args a, const Stream st) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NT = RES ? 2 : 1;
  float2* const stat = (float2*)(smem + ring_bytes(V * sizeof(T), NT));         // [tile_groups], then a pair for each thread
  let_next_start();
  const Place q = place<V>(a, st);
  Walk<T, V, NT, true> walk;
  walk.set(q, smem);
  walk.tensor(0, q, (const T*)a.x + q.n * a.x_n + q.c, a.x_p);
  if constexpr (RES) walk.tensor(1, q, (const T*)a.res + q.n * a.r_n + q.c, a.r_p);
  walk.start();                           // no kernel of the call has written these
  const Channel ch(a, st);
  float w[V], b[V], less[V], scale[V];
  if (q.on) row_params<V>(a, ch, q.c, w, b);
  wait_for_previous();
  // the tile's groups: their runs joined about the group's own mean
  const Tile tile = tile_of(a, st, blockIdx.y, V);
  const float inv_m = 1.0f / ((float)a.P * (float)(st.rep * a.Cg));
  // (sums about the first run's mean: it is off by no more than the runs' spread, which the squares contain)
  join_runs(a, st, tile, q.n, V, stat + st.tile_groups,
            [&](float2& t, float m, float2 v, float2 first) { const float d = v.x - first.x; t.x = __fmaf_rn(m, d, t.x); t.y += __fmaf_rn(m * d, d, v.y); },
            [&](int j, float2 t) {
              const int g = tile.g0 + j;
              const float d = t.x * inv_m;
              const float2* part = a.part_s + (long long)q.n * st.slices * st.tiles * st.tile_groups;
              const int t0 = first_tile(a, st, g, V);
              const float mean = __ldcg(part + t0 * st.tile_groups + g - (st.tiles == 1 ? 0 : t0 * (st.cvt * V) / a.Cg)).x + d;
              const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fmaf_rn(-d, t.x, t.y) * inv_m + a.eps));
              stat[j] = make_float2(mean, rstd);
              if (q.slice == 0 && (int)blockIdx.y == t0) { a.mean[(long long)q.n * a.G + g] = mean; a.rstd[(long long)q.n * a.G + g] = rstd; }
            });
  if (!q.on) return;
  {
    Per<V, WHOLE> mean, rstd;
    mean.set([&](int i) { return stat[ch.group(q.c + i) - tile.g0].x; });
    rstd.set([&](int i) { return stat[ch.group(q.c + i) - tile.g0].y; });
    mean.all(less);
    rstd.all(scale);
#pragma unroll
    for (int i = 0; i < V; ++i) less[i] = -less[i];
  }
  T* y = (T*)a.out + ((long long)q.n * a.P + walk.first(q)) * st.vc + q.c;
  const long long step = (long long)q.rows * st.vc;
  const int act = a.act;
  walk.run([&](const Raw<T, V> (&r)[NT], int) {
    float z[V];
    r[0].widen(z);
    vadd<V>(z, z, less);
    vmul<V>(z, z, scale);
    vmul_add<V>(z, z, w, b);
    if constexpr (RES) { float v[V]; r[1].widen(v); vadd<V>(z, z, v); }
    activate<T, V>(z, act);
    Raw<T, V> o;
    o.round(z);
    o.store_stream(y);
    y -= step;
  });
}

// ---- backward ------------------------------------------------------------------------------------------------------
// ACT: none, relu, or (2) the one that a.act names.  Backwards the residual only enters through act', so without an
// activation there is none.
template <int ACT>
__device__ __forceinline__ int act_of(const Args& a) { return ACT == 2 ? a.act : ACT == 1 ? SAE_ACT_RELU : SAE_ACT_NONE; }

// A thread's sums go to a second level, in shared memory, every eight rounds of its ring (32 to 128 pixels): no chain of additions is
// as long as a run (a constant of 0.1 over 16384 pixels: 2590 units off in one chain, 38 in two levels of 64 and 256).
__host__ __device__ constexpr int sums_kept(int vec) { return 2 * vec * (int)sizeof(float); }

// Each channel's sum dz and sum dz * xhat over a run, dresidual = dz on the way.  Bound by HBM: 32x56x56x256 bf16, relu with a
// residual, 206 MB in 36.7 us (5.6 TB/s); silu and gelu by the special-function unit (two operations an element):
// without a residual 103 MB in 32.5 and 39 us.
template <typename T, int V, bool WHOLE, int ACT, bool RES>
__global__ void __launch_bounds__(GN_THREADS, WHOLE ? 3 : 2) k_gn_grad_sums(const Args a, const Stream st) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NT = RES ? 3 : 2;
  constexpr int KEPT = sums_kept(V);
  float* const sh = (float*)smem;         // after the walk: [2][rows][cvt * V]; the first rows take the sums, times the weight
  float* const kept = (float*)(smem + ring_bytes(V * sizeof(T), NT, KEPT)) + threadIdx.x;     // [2 V][threads]
  let_next_start();
  const Place q = place<V>(a, st);
  const Channel ch(a, st);
  Walk<T, V, NT, false, KEPT> walk;
  walk.set(q, smem);
  walk.tensor(0, q, (const T*)a.x + q.n * a.x_n + q.c, a.x_p);
  walk.tensor(1, q, (const T*)a.dy + q.n * a.d_n + q.c, a.d_p);
  if constexpr (RES) walk.tensor(2, q, (const T*)a.res + q.n * a.r_n + q.c, a.r_p);
  walk.start();
  const int pitch = st.cvt * V, span = q.rows * pitch, slot = (threadIdx.x - q.row * st.cvt) * V;
  float s[V], sx[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { s[i] = 0.0f; sx[i] = 0.0f; kept[i * GN_THREADS] = 0.0f; kept[(V + i) * GN_THREADS] = 0.0f; }
  if (q.on) {
    float w[V], b[V], less[V], scale[V];
    row_params<V>(a, ch, q.c, w, b);
    Per<V, WHOLE> mean, rstd;
    const long long g = (long long)q.n * a.G;
    mean.set([&](int i) { return __ldg(a.mean + g + ch.group(q.c + i)); });
    rstd.set([&](int i) { return __ldg(a.rstd + g + ch.group(q.c + i)); });
    mean.all(less);
    rstd.all(scale);
#pragma unroll
    for (int i = 0; i < V; ++i) less[i] = -less[i];
    T* dres = a.dres ? (T*)a.dres + ((long long)q.n * a.P + q.p) * st.vc + q.c : nullptr;
    const long long step = (long long)q.rows * st.vc;
    const int act = act_of<ACT>(a);
    walk.run([&](const Raw<T, V> (&r)[NT], int) {
      float xh[V], dz[V];
      vector_grad<T, V>(r[0], r[1], RES ? &r[NT - 1] : nullptr, less, scale, w, b, act, xh, dz);
      vadd<V>(s, s, dz);
      vfma<V>(sx, dz, xh, sx);
      if (dres) { Raw<T, V> o; o.round(dz); o.store(dres); dres += step; }
    }, [&](int rounds) {
      if ((rounds & 7) == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          kept[i * GN_THREADS] += s[i]; kept[(V + i) * GN_THREADS] += sx[i];
          s[i] = 0.0f; sx[i] = 0.0f;
        }
      }
    });
  }
#pragma unroll
  for (int i = 0; i < V; ++i) { s[i] += kept[i * GN_THREADS]; sx[i] += kept[(V + i) * GN_THREADS]; }
  __syncthreads();                        // everybody is through with the ring
  if (q.row < q.rows) {
#pragma unroll
    for (int i = 0; i < V; ++i) { sh[q.row * pitch + slot + i] = s[i]; sh[span + q.row * pitch + slot + i] = sx[i]; }
  }
  __syncthreads();
  wait_for_previous();
  const Tile tile = tile_of(a, st, blockIdx.y, V);
  const long long at = ((long long)q.n * st.slices + q.slice) * a.C + tile.lo;
  for (int i = threadIdx.x; i < (st.rep > 1 ? a.C : pitch); i += GN_THREADS) {
    float s = 0.0f, sx = 0.0f, w = 0.0f;
    for (int r = 0; r < q.rows; ++r)
      for (int e = r * pitch + i, k = 0; k < st.rep; ++k, e += a.C) { s += sh[e]; sx += sh[span + e]; }
    if (tile.lo + i < tile.hi) { a.part_a[at + i] = s; a.part_b[at + i] = sx; w = param(a.w, a.ptype, tile.lo + i, 1.0f); }
    sh[i] = s * w;
    sh[span + i] = sx * w;
  }
  float2* const out = run_out(a, st, q);
  fold_tile<V, V>(a, tile, sh, 1, 1, pitch, [&](int j, float s, int) { out[j].x = s; });
  fold_tile<V, V>(a, tile, sh + span, 1, 1, pitch, [&](int j, float s, int) { out[j].y = s; });
}

// The channels' sums over `rows` runs, 32 channels a block of 256 threads, in a fixed order: dw and db.  In double: there may be
// millions of samples.
__device__ __forceinline__ void param_grads(const Args& a, int block, long long rows) {
  __shared__ double sa[8][33], sb[8][33];
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5, c = block * 32 + cx;
  double s = 0.0, q = 0.0;
  if (c < a.C) {
#pragma unroll 4
    for (long long r = ry; r < rows; r += 8) { s += (double)__ldcg(a.part_a + r * a.C + c); q += (double)__ldcg(a.part_b + r * a.C + c); }
  }
  sa[ry][cx] = s; sb[ry][cx] = q;
  __syncthreads();
  if (ry == 0 && c < a.C) {
    for (int i = 1; i < 8; ++i) { s += sa[i][cx]; q += sb[i][cx]; }
    if (a.db) put_param(a.db, a.ptype, c, (float)s);
    if (a.dw) put_param(a.dw, a.ptype, c, (float)q);
  }
}
__global__ void __launch_bounds__(GN_THREADS) k_gn_param_grads(const Args a, long long rows) {
  wait_for_previous();
  param_grads(a, blockIdx.x, rows);
}

// dx, and in leading layers of the grid dw and db.  Bound by HBM: the same tensors with dz read from dresidual, 154 MB in 24.5 us
// from a cold L2 (6.3 TB/s).
template <typename T, int V, bool WHOLE, int ACT, bool RES>
__global__ void __launch_bounds__(GN_THREADS, WHOLE ? 3 : 2) k_gn_grad_apply(const Args a, const Stream st) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NT = RES ? 3 : 2;
  float2* const stat = (float2*)(smem + ring_bytes(V * sizeof(T), NT));         // [tile_groups], then a pair for each thread
  let_next_start();
  if ((int)blockIdx.z < st.param_z) {     // dw and db, beside the rest
    wait_for_previous();
    const int block = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
    if (block * 32 < a.C) param_grads(a, block, (long long)a.N * st.slices);
    return;
  }
  const Place q = place<V>(a, st);
  const Channel ch(a, st);
  Walk<T, V, NT, true> walk;
  walk.set(q, smem);
  walk.tensor(0, q, (const T*)a.x + q.n * a.x_n + q.c, a.x_p);
  walk.tensor(1, q, (const T*)a.dy + q.n * a.d_n + q.c, a.d_p);
  if constexpr (RES) walk.tensor(2, q, (const T*)a.res + q.n * a.r_n + q.c, a.r_p);
  if (!st.held) walk.start();             // held: the first pass writes what is read here
  float w[V], b[V], less[V], scale[V], p1[V], p2[V], gw[V];
  if (q.on) {
    row_params<V>(a, ch, q.c, w, b);
    Per<V, WHOLE> mean, rstd;
    const long long g = (long long)q.n * a.G;
    mean.set([&](int i) { return __ldg(a.mean + g + ch.group(q.c + i)); });
    rstd.set([&](int i) { return __ldg(a.rstd + g + ch.group(q.c + i)); });
    mean.all(less);
    rstd.all(scale);
#pragma unroll
    for (int i = 0; i < V; ++i) less[i] = -less[i];
  }
  wait_for_previous();
  if (st.held) walk.start();
  // the tile's groups: mean(g) and mean(g * xhat), negated
  const Tile tile = tile_of(a, st, blockIdx.y, V);
  const float inv_m = 1.0f / ((float)a.P * (float)(st.rep * a.Cg));
  join_runs(a, st, tile, q.n, V, stat + st.tile_groups, [&](float2& t, float, float2 v, float2) { t.x += v.x; t.y += v.y; },
            [&](int j, float2 t) { stat[j] = make_float2(-t.x * inv_m, -t.y * inv_m); });
  if (!q.on) return;
  {
    // dx = rstd * (dz * w - mean(g) - xhat * mean(g * xhat)) = dz * (w rstd) + (xhat * (-rstd mean(g xhat)) - rstd mean(g))
    Per<V, WHOLE> m1, m2;
    m1.set([&](int i) { return scale[i] * stat[ch.group(q.c + i) - tile.g0].x; });
    m2.set([&](int i) { return scale[i] * stat[ch.group(q.c + i) - tile.g0].y; });
    m1.all(p1);
    m2.all(p2);
    vmul<V>(gw, w, scale);
  }
  T* dx = (T*)a.out + ((long long)q.n * a.P + walk.first(q)) * st.vc + q.c;
  const long long step = (long long)q.rows * st.vc;
  const int act = act_of<ACT>(a);
  walk.run([&](const Raw<T, V> (&r)[NT], int) {
    float xh[V], dz[V];
    vector_grad<T, V>(r[0], r[1], RES ? &r[NT - 1] : nullptr, less, scale, w, b, act, xh, dz);
    vfma<V>(xh, xh, p2, p1);
    vfma<V>(dz, dz, gw, xh);
    Raw<T, V> o;
    o.round(dz);
    o.store_stream(dx);
    dx -= step;
  });
}

}  // namespace sae
