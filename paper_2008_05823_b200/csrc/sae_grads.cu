// Gradient sets: the norm of a worker's gradients over many tensors, clipping by it, packing the tensors into
// the [K][d] buffer of sae_step and unpacking a vector into tensors.  Declarations and contract: include/sae.h.
//
//   norm_k = (sum_j sum_i |g_ji|^q)^(1/q), q = 1 or 2, or the largest |g_ji|;  coef_k = min(1, max_norm / (norm_k + 1e-6))
//
// Everything here is bound by HBM: a norm reads each element once; clipping and packing need the finished norm
// before the first store, so they are a second pass whose reads come from L2 as far as it still holds the row.
#include "../../include/sae.h"
#include "sae_vec.cuh"

#include <algorithm>
#include <new>
#include <type_traits>
#include <vector>

using namespace sae;

namespace {

typedef unsigned long long u64;
typedef unsigned int u32;

constexpr int GT_THREADS = 256;
constexpr int GT_TILE = 16384;           // bytes of one tensor that a block handles at a time
constexpr int GT_STAGES = 3;             // tiles on their way or in use: 48 KB of shared memory
constexpr int GT_BLOCKS_PER_SM = 4;
constexpr int GT_SMEM = GT_STAGES * GT_TILE;
constexpr int PTRS_SMALL = 64;           // tensor pointers that travel as kernel arguments
constexpr int PTRS_LARGE = 448;
constexpr int PTRS_UPLOAD = 3840;        // pointers one upload launch carries (30 KB of the 32 KB of arguments)
constexpr double COEF_EPS = 1e-6;

// One tile: elements of tensor `tensor` from element `start`, at element `at` of a packed row.
struct Tile {
  long long at;
  u32 tensor, start, count_type, pad;     // count * 4 + type
  __host__ __device__ u32 count() const { return count_type >> 2; }
  __host__ __device__ u32 type() const { return count_type & 3u; }
};

// The tensors' addresses, row-major [rows][T].  N > 0: in the kernel's arguments; N = 0: in device memory.
template <int N>
struct Ptrs {
  void* p[N];
  __device__ __forceinline__ void* get(int i) const { return p[i]; }
};
template <>
struct Ptrs<0> {
  void* const* p;
  __device__ __forceinline__ void* get(int i) const { return p[i]; }
};

struct UploadChunk { void* p[PTRS_UPLOAD]; };

__global__ void k_upload_ptrs(const __grid_constant__ UploadChunk c, void** table, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) table[i] = c.p[i];
}

// ---- the running value of a norm: a double (q = 1, 2), or the bits of the largest magnitude -------------------
// Eight elements are added in float first and the sum goes to the double accumulator: the float part rounds at most
// seven times and the row's length does not enter.  Where the float sum may have overflowed or lost its small terms
// (outside 1e-28 .. 1e37) the eight are added in double; q = 2 then covers every finite float.
template <int KIND>
struct Running {
  double s;
  __device__ __forceinline__ void zero() { s = 0.0; }
  __device__ __forceinline__ void one(float v) {
    const double a = (double)v;
    s += KIND == SAE_NORM_TWO ? a * a : fabs(a);
  }
  __device__ __forceinline__ void eight(const float (&v)[8]) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = KIND == SAE_NORM_TWO ? __fmaf_rn(v[i], v[i], t) : t + fabsf(v[i]);
    if (t >= 1e-28f && t <= 1e37f) {
      s += (double)t;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) one(v[i]);
    }
  }
  __device__ __forceinline__ void join(const Running& o) { s += o.s; }
  __device__ __forceinline__ Running shuffled(int o) const { Running r; r.s = __shfl_xor_sync(0xffffffffu, s, o); return r; }
  __device__ __forceinline__ u64 bits() const { return (u64)__double_as_longlong(s); }
  __device__ __forceinline__ void from_bits(u64 b) { s = __longlong_as_double((long long)b); }
  __device__ __forceinline__ double norm() const { return KIND == SAE_NORM_TWO ? sqrt(s) : s; }
};
// Magnitudes as unsigned integers order as their values do, infinity above all of them and NaN above infinity: a NaN stays.
template <>
struct Running<SAE_NORM_MAX> {
  u32 m;
  __device__ __forceinline__ void zero() { m = 0u; }
  __device__ __forceinline__ void one(float v) { m = max(m, __float_as_uint(v) & 0x7fffffffu); }
  __device__ __forceinline__ void eight(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) one(v[i]);
  }
  __device__ __forceinline__ void join(const Running& o) { m = max(m, o.m); }
  __device__ __forceinline__ Running shuffled(int o) const { Running r; r.m = __shfl_xor_sync(0xffffffffu, m, o); return r; }
  __device__ __forceinline__ u64 bits() const { return m; }
  __device__ __forceinline__ void from_bits(u64 b) { m = (u32)b; }
  __device__ __forceinline__ double norm() const { return (double)__uint_as_float(m); }
};

// The block's value in thread 0, joined in a fixed order: the same bits on every call.
template <int KIND>
__device__ __forceinline__ void block_join(Running<KIND>& r, u64* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.join(r.shuffled(o));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) sh[warp] = r.bits();
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < GT_THREADS / 32; ++w) { Running<KIND> o; o.from_bits(sh[w]); r.join(o); }
  }
}

// A block's tiles come through a ring of GT_STAGES shared-memory images, copied asynchronously in pieces of 16 bytes whatever
// the type: two tiles are on their way while one is used, so the loads in flight (128 KB an SM) do not depend on registers.
// A thread uses the pieces that it copied itself, so no barrier is needed.  A tensor that is not aligned to 16 bytes is not
// copied but read in place.
__device__ __forceinline__ int elem_size(u32 type) { return type == SAE_TYPE_FLOAT ? 4 : 2; }
template <int N>
struct Ring {
  static constexpr int PIECES = GT_TILE / (16 * GT_THREADS);
  unsigned char* smem;
  const Tile* tiles;
  const Ptrs<N>* ptrs;
  int first;                              // the row's first pointer

  __device__ __forceinline__ unsigned char* stage(int s) const { return smem + s * GT_TILE; }
  __device__ __forceinline__ unsigned char* address(const Tile& t) const {
    return (unsigned char*)ptrs->get(first + (int)t.tensor) + (size_t)t.start * elem_size(t.type());
  }
  __device__ __forceinline__ static bool copied(const unsigned char* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
  __device__ __forceinline__ void fetch(const Tile& t, int s) const {
    const unsigned char* const p = address(t);
    if (!copied(p)) return;
    const u32 n = t.count() * elem_size(t.type()) / 16;
    unsigned char* const to = stage(s);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const u32 e = i * GT_THREADS + threadIdx.x;
      if (e < n) copy_async<16>(to + e * 16, p + (size_t)e * 16);
    }
  }
  // use(tile, its address, its image) for count tiles from t0 on, dir = 1 or -1.
  template <typename F>
  __device__ __forceinline__ void run(int t0, int count, int dir, F use) const {
    // the tiles' entries wait in registers: w[0] in use, w[1] and w[2] on their way, w[3] next
    Tile w[GT_STAGES + 1] = {};
#pragma unroll
    for (int k = 0; k <= GT_STAGES; ++k)
      if (k < count) w[k] = tiles[t0 + dir * k];
#pragma unroll
    for (int k = 0; k < GT_STAGES - 1; ++k) {
      if (k < count) fetch(w[k], k);
      copies_commit();
    }
    int from = 0;
    for (int k = 0; k < count; ++k) {
      const int to = from == 0 ? GT_STAGES - 1 : from - 1;                      // (from + GT_STAGES - 1) % GT_STAGES
      if (k + GT_STAGES - 1 < count) fetch(w[GT_STAGES - 1], to);
      copies_commit();
      const Tile t = w[0];
#pragma unroll
      for (int i = 0; i < GT_STAGES; ++i) w[i] = w[i + 1];
      if (k + GT_STAGES + 1 < count) w[GT_STAGES] = tiles[t0 + dir * (k + GT_STAGES + 1)];
      copies_wait<GT_STAGES - 1>();
      use(t, address(t), stage(from));
      __syncwarp();                       // a warp's lanes may have used one another's pieces
      from = from + 1 == GT_STAGES ? 0 : from + 1;
    }
    copies_wait<0>();
  }
};

// Which eight values are added in float does not depend on the alignment: a tensor that is read in place is taken in the same pieces,
// element by element, so equal values give equal bits wherever they lie.
template <int KIND, typename T>
__device__ __forceinline__ void tile_norm(Running<KIND>& r, const T* p, const unsigned char* image, u32 cnt) {
  constexpr int V = 16 / (int)sizeof(T), N = GT_TILE / (GT_THREADS * 16), L = 16;
  const u32 tid = threadIdx.x, whole = cnt / V;
  if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8 / V) {
      float v[8];
#pragma unroll
      for (int h = 0; h < 8 / V; ++h) {
        const u32 e = (i + h) * GT_THREADS + tid;
        Raw<T, V> raw;
        raw.clear();
        if (e < whole) raw.b = *reinterpret_cast<const uint4*>(image + e * 16);
        raw.widen(*reinterpret_cast<float (*)[V]>(&v[h * V]));
      }
      r.eight(v);
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < N; i += L / V) {
      T t[L];
#pragma unroll
      for (int q = 0; q < L; ++q) {
        const u32 e = (i + q / V) * GT_THREADS + tid;
        t[q] = from_f<T>(0.0f);
        if (e < whole) t[q] = p[e * V + q % V];
      }
#pragma unroll
      for (int h = 0; h < L; h += 8) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = to_f(t[h + q]);
        r.eight(v);
      }
    }
  }
  const u32 e = whole * V + tid;
  if (e < cnt) r.one(to_f(p[e]));
}

// blockIdx.y: the row (worker).  The row's tiles are dealt out in runs of neighbours, one run a block.  The block
// that comes last (a ticket a row, back at zero after it) joins the runs' values in their order.  Bound by HBM: 1.75 GB of
// float in 276 us (6.3 TB/s), an encoder's 219 MB in 39 (5.6); 51 MB in 15, about 6 of them start, end and the join.
template <int KIND, int N>
__global__ void __launch_bounds__(GT_THREADS, GT_BLOCKS_PER_SM) k_grads_norm(const __grid_constant__ Ptrs<N> ptrs, const Tile* __restrict__ tiles,
                                                           int ntiles, int T, u64* partials, u32* tickets, float max_norm,
                                                           float* coefs, float* norms) {
  extern __shared__ __align__(16) unsigned char smem[];
  u64* const sh = (u64*)smem;             // after the ring: a value for each warp, then whether this block is the last
  int& sh_last = *(int*)(sh + GT_THREADS / 32);
  const int row = blockIdx.y, B = gridDim.x;
  const int t0 = (int)((long long)ntiles * blockIdx.x / B), t1 = (int)((long long)ntiles * (blockIdx.x + 1) / B);
  Running<KIND> r; r.zero();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Ring<N> ring = {smem, tiles, &ptrs, row * T};
  ring.run(t0, t1 - t0, 1, [&](const Tile& t, const unsigned char* p, const unsigned char* image) {
    if (t.type() == SAE_TYPE_FLOAT) tile_norm<KIND, float>(r, (const float*)p, image, t.count());
    else if (t.type() == SAE_TYPE_BFLOAT) tile_norm<KIND, __nv_bfloat16>(r, (const __nv_bfloat16*)p, image, t.count());
    else tile_norm<KIND, __half>(r, (const __half*)p, image, t.count());
  });
  __syncthreads();
  block_join<KIND>(r, sh);
  if (threadIdx.x == 0) {
    partials[(size_t)row * B + blockIdx.x] = r.bits();
    __threadfence();
    sh_last = atomicInc(tickets + row, (u32)B - 1u) == (u32)B - 1u;
  }
  __syncthreads();
  if (!sh_last) return;
  __threadfence();
  r.zero();
  for (int i = threadIdx.x; i < B; i += GT_THREADS) {
    Running<KIND> o; o.from_bits(__ldcg(partials + (size_t)row * B + i)); r.join(o);
  }
  __syncthreads();                 // sh is used again
  block_join<KIND>(r, sh);
  if (threadIdx.x == 0) {
    const double norm = r.norm(), c = (double)max_norm / (norm + COEF_EPS);
    coefs[row] = !(c >= 1.0) ? (float)c : 1.0f;       // a NaN stays
    if (norms) norms[row] = (float)norm;
  }
}

// ---- scaled copies --------------------------------------------------------------------------------------------
enum { MODE_CLIP, MODE_PACK };

// In place, a 16-bit tensor is scaled by the coefficient rounded to its own type, which is what torch's in-place product with
// a scalar tensor does: for the same coefficient both give the same bits.  Not below the type's normal numbers (a half's end at
// 2^-14), where the rounding would cost digits or leave zero.
template <typename T> __device__ __forceinline__ float coef_for(float c) { return c; }
template <> __device__ __forceinline__ float coef_for<__nv_bfloat16>(float c) { return c >= 1.17549435e-38f ? to_f(from_f<__nv_bfloat16>(c)) : c; }
template <> __device__ __forceinline__ float coef_for<__half>(float c) { return c >= 6.103515625e-5f ? to_f(from_f<__half>(c)) : c; }

// A warp's 32 neighbouring pieces (`left` of them exist), scaled, to D at 16-byte aligned addresses.  Between types of one
// size a lane stores its own piece.  16 bits to float doubles the bytes: lane after lane takes half a piece, so that a store
// of the warp is one run of 512 bytes (a lane storing both halves of its own piece leaves every sector to two stores:
// 35 against 25 us for a row of 25.6 M elements).
template <typename S, typename D>
__device__ __forceinline__ void store_pieces(const unsigned char* image, D* d, u32 left, float coef) {
  constexpr int V = 16 / (int)sizeof(D), P = 16 / (int)sizeof(S) / V;           // elements a store takes, stores a piece takes
  const u32 lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < P; ++h) {
    const u32 i = h * 32 + lane;
    if (i < left * P) {
      Raw<S, V> raw;
      raw.b = *reinterpret_cast<const typename Raw<S, V>::B*>(image + i * (V * sizeof(S)));
      float v[V];
      raw.widen(v);
#pragma unroll
      for (int q = 0; q < V; ++q) v[q] = __fmul_rn(v[q], coef);
      Raw<D, V> o;
      o.round(v);
      o.store_stream(d + i * V);
    }
  }
}

// coef * a tile of S (clip: D = S, in place; pack: D = float).  coef = 1 multiplies exactly.
template <typename S, typename D>
__device__ __forceinline__ void tile_scale(const S* s, const unsigned char* image, D* d, u32 cnt, float coef) {
  constexpr int V = 16 / (int)sizeof(S), N = GT_TILE / (GT_THREADS * 16);
  const u32 tid = threadIdx.x;
  if ((reinterpret_cast<uintptr_t>(s) & 15) != 0) {                             // not copied
    for (u32 e = tid; e < cnt; e += GT_THREADS) d[e] = from_f<D>(__fmul_rn(to_f(s[e]), coef));
    return;
  }
  const u32 whole = cnt / V;
  if ((reinterpret_cast<uintptr_t>(d) & 15) == 0) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const u32 e = i * GT_THREADS + (tid & ~31u);
      if (e < whole) store_pieces<S, D>(image + e * 16, d + e * V, min(32u, whole - e), coef);
    }
  } else {                                // neighbours by neighbouring threads, out of everybody's pieces
    __syncthreads();
    const S* const held = reinterpret_cast<const S*>(image);
#pragma unroll 4
    for (u32 e = tid; e < whole * V; e += GT_THREADS) d[e] = from_f<D>(__fmul_rn(to_f(held[e]), coef));
    __syncthreads();                      // the image is not overwritten before
  }
  const u32 e = whole * V + tid;
  if (e < cnt) d[e] = from_f<D>(__fmul_rn(to_f(s[e]), coef));
}

// The tiles run backwards: the norm's pass went forwards, and what it read last is what L2 still holds.  Bound by HBM's writes:
// ResNet-50 bf16 to float, 51 MB read and 102 written in 22 us behind the norm; in place with a coefficient below 1, 51 MB read and
// written in 14 (its copies wait for the norm), [8][858 868] float, 27 MB each way, in 10.
template <int MODE, int N>
__global__ void __launch_bounds__(GT_THREADS, GT_BLOCKS_PER_SM) k_grads_scale(const __grid_constant__ Ptrs<N> ptrs, const Tile* __restrict__ tiles,
                                                                              int ntiles, int T, const float* coefs, float* vec, long long stride) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int row = (int)(gridDim.y - 1 - blockIdx.y), B = gridDim.x, b = B - 1 - (int)blockIdx.x;
  const int t0 = (int)((long long)ntiles * b / B), t1 = (int)((long long)ntiles * (b + 1) / B);
  float coef = 1.0f;
  bool waited = false;
  if (MODE == MODE_CLIP) {
    cudaGridDependencySynchronize();
    coef = *(volatile const float*)(coefs + row);
    if (coef == 1.0f) return;             // nothing would change
  }
  float* const v = MODE == MODE_CLIP ? nullptr : vec + row * stride;
  const Ring<N> ring = {smem, tiles, &ptrs, row * T};
  ring.run(t1 - 1, t1 - t0, -1, [&](const Tile& t, unsigned char* p, const unsigned char* image) {
    if (MODE == MODE_PACK && !waited) {   // for the norm's kernel, with this one's first loads on their way
      cudaGridDependencySynchronize();
      if (coefs) coef = *(volatile const float*)(coefs + row);
      waited = true;
    }
    auto as = [&](auto* s) {
      typedef typename std::remove_pointer<decltype(s)>::type S;
      if (MODE == MODE_CLIP) tile_scale<S, S>(s, image, s, t.count(), coef_for<S>(coef));
      else tile_scale<S, float>(s, image, v + t.at, t.count(), coef);
    };
    if (t.type() == SAE_TYPE_FLOAT) as((float*)p);
    else if (t.type() == SAE_TYPE_BFLOAT) as((__nv_bfloat16*)p);
    else as((__half*)p);
  });
}

template <typename T>
__device__ __forceinline__ void tile_unpack(const float* s, T* d, u32 cnt) {
  if (((reinterpret_cast<uintptr_t>(s) & 15) | (reinterpret_cast<uintptr_t>(d) & (4 * sizeof(T) - 1))) == 0) {
    const u32 whole = cnt / 4;
#pragma unroll 4
    for (u32 i = threadIdx.x; i < whole; i += GT_THREADS) {
      Raw<float, 4> raw;
      raw.load(s + i * 4);
      float v[4];
      raw.widen(v);
      Raw<T, 4> o;
      o.round(v);
      o.store(d + i * 4);
    }
    const u32 e = whole * 4 + threadIdx.x;
    if (e < cnt) d[e] = from_f<T>(s[e]);
  } else {
#pragma unroll 8
    for (u32 e = threadIdx.x; e < cnt; e += GT_THREADS) d[e] = from_f<T>(s[e]);
  }
}

template <int N>
__global__ void __launch_bounds__(GT_THREADS) k_grads_unpack(const __grid_constant__ Ptrs<N> ptrs, const Tile* __restrict__ tiles, int ntiles,
                                                             int T, const float* vec, long long stride) {
  const int row = blockIdx.y;
  const int t0 = (int)((long long)ntiles * blockIdx.x / gridDim.x), t1 = (int)((long long)ntiles * (blockIdx.x + 1) / gridDim.x);
  for (int t = t0; t < t1; ++t) {
    const Tile ti = tiles[t];
    void* base = ptrs.get(row * T + (int)ti.tensor);
    const float* const s = vec + row * stride + ti.at;
    if (ti.type() == SAE_TYPE_FLOAT) tile_unpack(s, (float*)base + ti.start, ti.count());
    else if (ti.type() == SAE_TYPE_BFLOAT) tile_unpack(s, (__nv_bfloat16*)base + ti.start, ti.count());
    else tile_unpack(s, (__half*)base + ti.start, ti.count());
  }
}

thread_local int g_grads_cuda_error = 0;

struct DeviceGuard {
  int prev;
  bool ok;
  explicit DeviceGuard(int dev) : prev(-1), ok(false) {
    if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
    ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

}  // namespace

struct sae_grads {
  int K, T, device, num_sms, ntiles, last_cuda_error;
  long long d;
  cudaStream_t stream;
  std::vector<int64_t> sizes;
  std::vector<int> types;
  Tile* tiles;
  void** table;
  u64* partials;
  u32* tickets;
  float* coefs;
  int max_blocks;                 // blocks a row has at most: the length of its partial values
};

namespace {

int cuda_status(sae_grads* h, cudaError_t e) {
  h->last_cuda_error = (int)e;
  cudaGetLastError();
  return e == cudaErrorMemoryAllocation ? SAE_ERR_NOMEM : SAE_ERR_CUDA;
}

void release(sae_grads* h) {
  cudaFree(h->tiles); cudaFree(h->table); cudaFree(h->partials); cudaFree(h->tickets); cudaFree(h->coefs);
  delete h;
}

int elem_bytes(int type) { return type == SAE_TYPE_FLOAT ? 4 : 2; }

// Blocks of one row: every SM full once, one tile a block at least.
int row_blocks(const sae_grads* h) {
  const int want = (h->num_sms * GT_BLOCKS_PER_SM + h->K - 1) / h->K;
  return std::max(1, std::min(std::min(h->ntiles, h->max_blocks), want));
}

template <int N>
cudaError_t launch_norm(sae_grads* h, const Ptrs<N>& p, int kind, float max_norm, float* norms) {
  const dim3 grid((unsigned)row_blocks(h), (unsigned)h->K);
#define NORM(KIND) k_grads_norm<KIND, N><<<grid, GT_THREADS, GT_SMEM, h->stream>>>(p, h->tiles, h->ntiles, h->T, h->partials, h->tickets, \
                                                                              max_norm, h->coefs, norms)
  if (kind == SAE_NORM_TWO) NORM(SAE_NORM_TWO);
  else if (kind == SAE_NORM_ONE) NORM(SAE_NORM_ONE);
  else NORM(SAE_NORM_MAX);
#undef NORM
  return cudaGetLastError();
}

template <int MODE, int N>
cudaError_t launch_scale(sae_grads* h, const Ptrs<N>& p, bool scaled, float* vec, long long stride) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)row_blocks(h), (unsigned)h->K);
  cfg.blockDim = dim3(GT_THREADS);
  cfg.dynamicSmemBytes = GT_SMEM;
  cfg.stream = h->stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = scaled ? 1 : 0;           // only behind this call's own norm kernel
  return cudaLaunchKernelEx(&cfg, k_grads_scale<MODE, N>, p, (const Tile*)h->tiles, h->ntiles, h->T,
                            (const float*)(scaled ? h->coefs : nullptr), vec, stride);
}

enum { WITH_NORM = 1, WITH_CLIP = 2, WITH_PACK = 4, WITH_UNPACK = 8 };

// All rows at once: one by one, so that L2 keeps a row of up to 48 MB from the first pass to the second, costs more in launches
// than it saves (four ResNet-50 rows of 51 MB: 166 us against 152; four encoder rows of 219 MB: 635 against 620).
template <int N>
cudaError_t launch_all(sae_grads* h, const Ptrs<N>& p, int what, int kind, float max_norm, float* vec, long long stride, float* norms) {
  cudaError_t e = cudaSuccess;
  const bool scaled = (what & WITH_NORM) != 0;
  if (scaled) e = launch_norm<N>(h, p, kind, max_norm, norms);
  if (e != cudaSuccess || h->ntiles == 0) return e;
  if (what & WITH_CLIP) e = launch_scale<MODE_CLIP, N>(h, p, scaled, vec, stride);
  if (what & WITH_PACK) e = launch_scale<MODE_PACK, N>(h, p, scaled, vec, stride);
  if (what & WITH_UNPACK) {
    const int blocks = std::max(1, std::min(h->ntiles, h->num_sms * 8 / h->K));
    k_grads_unpack<N><<<dim3((unsigned)blocks, (unsigned)h->K), GT_THREADS, 0, h->stream>>>(p, h->tiles, h->ntiles, h->T, vec, stride);
    e = cudaGetLastError();
  }
  return e;
}

int run(sae_grads* h, const void* const* tensors, int what, int kind, float max_norm, float* vec, long long stride, float* norms) {
  const size_t n = (size_t)h->K * h->T;
  for (size_t i = 0; i < n; ++i) {
    const int j = (int)(i % (size_t)h->T);
    if (h->sizes[j] == 0) continue;
    if (!tensors[i] || (reinterpret_cast<uintptr_t>(tensors[i]) & (uintptr_t)(elem_bytes(h->types[j]) - 1))) return SAE_ERR_INVALID_ARG;
  }
  DeviceGuard guard(h->device);
  if (!guard.ok) return cuda_status(h, cudaGetLastError());
  cudaError_t e = cudaSuccess;
  if (n <= PTRS_SMALL) {
    Ptrs<PTRS_SMALL> p;
    for (size_t i = 0; i < n; ++i) p.p[i] = const_cast<void*>(tensors[i]);
    e = launch_all<PTRS_SMALL>(h, p, what, kind, max_norm, vec, stride, norms);
  } else if (n <= PTRS_LARGE) {
    Ptrs<PTRS_LARGE> p;
    for (size_t i = 0; i < n; ++i) p.p[i] = const_cast<void*>(tensors[i]);
    e = launch_all<PTRS_LARGE>(h, p, what, kind, max_norm, vec, stride, norms);
  } else {
    static thread_local UploadChunk chunk;
    for (size_t i = 0; i < n && e == cudaSuccess; i += PTRS_UPLOAD) {
      const int m = (int)std::min<size_t>(PTRS_UPLOAD, n - i);
      for (int q = 0; q < m; ++q) chunk.p[q] = const_cast<void*>(tensors[i + q]);
      k_upload_ptrs<<<(m + 255) / 256, 256, 0, h->stream>>>(chunk, h->table + i, m);
      e = cudaGetLastError();
    }
    Ptrs<0> p;
    p.p = h->table;
    if (e == cudaSuccess) e = launch_all<0>(h, p, what, kind, max_norm, vec, stride, norms);
  }
  return e == cudaSuccess ? SAE_OK : cuda_status(h, e);
}

bool norm_kind_ok(int32_t kind) { return kind == SAE_NORM_TWO || kind == SAE_NORM_ONE || kind == SAE_NORM_MAX; }

}  // namespace

extern "C" {

int sae_grads_init(const sae_grads_config* cfg, sae_grads** out) {
  if (!cfg || !out) return SAE_ERR_INVALID_ARG;
  *out = nullptr;
  if (cfg->abi_version != SAE_ABI_VERSION) return SAE_ERR_ABI;
  if (cfg->num_rows < 1 || cfg->num_rows > 1024 || cfg->num_tensors < 1 || !cfg->tensor_sizes || cfg->device < 0) return SAE_ERR_INVALID_ARG;
  const int K = cfg->num_rows, T = cfg->num_tensors;
  long long d = 0, nt = 0;
  for (int j = 0; j < T; ++j) {
    const int64_t n = cfg->tensor_sizes[j];
    const int32_t ty = cfg->tensor_types ? cfg->tensor_types[j] : SAE_TYPE_FLOAT;
    if (n < 0 || n > (1ll << 30) || (ty != SAE_TYPE_FLOAT && ty != SAE_TYPE_BFLOAT && ty != SAE_TYPE_HALF)) return SAE_ERR_INVALID_ARG;
    d += n;
    nt += (n * elem_bytes(ty) + GT_TILE - 1) / GT_TILE;
  }
  if (nt > (1ll << 30) || (long long)K * T > (1ll << 30)) return SAE_ERR_INVALID_ARG;
  sae_grads* h = new (std::nothrow) sae_grads();
  if (!h) return SAE_ERR_NOMEM;
  h->K = K; h->T = T; h->d = d; h->device = cfg->device; h->stream = (cudaStream_t)cfg->stream; h->ntiles = (int)nt;
  std::vector<Tile> tiles;
  try {
    h->sizes.assign(cfg->tensor_sizes, cfg->tensor_sizes + T);
    h->types.assign((size_t)T, SAE_TYPE_FLOAT);
    if (cfg->tensor_types) h->types.assign(cfg->tensor_types, cfg->tensor_types + T);
    tiles.reserve((size_t)nt);
    long long at = 0;
    for (int j = 0; j < T; ++j) {
      const int64_t step = GT_TILE / elem_bytes(h->types[j]);
      for (int64_t s = 0; s < h->sizes[j]; s += step) {
        Tile t = {};
        t.tensor = (u32)j; t.start = (u32)s; t.count_type = (u32)std::min<int64_t>(step, h->sizes[j] - s) * 4u + (u32)h->types[j];
        t.at = at + s;
        tiles.push_back(t);
      }
      at += h->sizes[j];
    }
  } catch (...) {
    delete h;
    return SAE_ERR_NOMEM;
  }
  DeviceGuard guard(cfg->device);
  cudaError_t e = guard.ok ? cudaSuccess : cudaGetLastError();
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, cfg->device);
  h->max_blocks = std::max(1, std::min(h->ntiles, h->num_sms * GT_BLOCKS_PER_SM));
  if (e == cudaSuccess) e = cudaMalloc(&h->tiles, std::max<size_t>(1, tiles.size()) * sizeof(Tile));
  if (e == cudaSuccess && (size_t)K * T > PTRS_LARGE) e = cudaMalloc(&h->table, (size_t)K * T * sizeof(void*));
  if (e == cudaSuccess) e = cudaMalloc(&h->partials, (size_t)K * h->max_blocks * sizeof(u64));
  if (e == cudaSuccess) e = cudaMalloc(&h->tickets, (size_t)K * sizeof(u32));
  if (e == cudaSuccess) e = cudaMalloc(&h->coefs, (size_t)K * sizeof(float));
  if (e == cudaSuccess) e = cudaMemsetAsync(h->tickets, 0, (size_t)K * sizeof(u32), h->stream);
  if (e == cudaSuccess && !tiles.empty()) e = cudaMemcpyAsync(h->tiles, tiles.data(), tiles.size() * sizeof(Tile), cudaMemcpyHostToDevice, h->stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
  if (e != cudaSuccess) {
    const int rc = cuda_status(h, e);
    g_grads_cuda_error = (int)e;
    release(h);
    return rc;
  }
  *out = h;
  return SAE_OK;
}

int sae_grads_norm(sae_grads* h, const void* const* tensors, int32_t norm_kind, float* norms) {
  if (!h || !tensors || !norms || !norm_kind_ok(norm_kind)) return SAE_ERR_INVALID_ARG;
  return run(h, tensors, WITH_NORM, norm_kind, 0.0f, nullptr, 0, norms);
}

int sae_grads_clip(sae_grads* h, void* const* tensors, int32_t norm_kind, float max_norm, float* norms) {
  if (!h || !tensors || !norm_kind_ok(norm_kind) || !(max_norm >= 0.0f)) return SAE_ERR_INVALID_ARG;
  return run(h, (const void* const*)tensors, WITH_NORM | WITH_CLIP, norm_kind, max_norm, nullptr, 0, norms);
}

int sae_grads_pack(sae_grads* h, const void* const* tensors, int32_t norm_kind, float max_norm, float* out, int64_t out_stride,
                   float* norms) {
  if (!h || !tensors || (!out && h->d) || (h->K > 1 && out_stride < h->d) || (reinterpret_cast<uintptr_t>(out) & 3)) return SAE_ERR_INVALID_ARG;
  if (norm_kind == SAE_NORM_NONE) {
    if (norms) return SAE_ERR_INVALID_ARG;
    return run(h, tensors, WITH_PACK, norm_kind, 0.0f, out, out_stride, nullptr);
  }
  if (!norm_kind_ok(norm_kind) || !(max_norm >= 0.0f)) return SAE_ERR_INVALID_ARG;
  return run(h, tensors, WITH_NORM | WITH_PACK, norm_kind, max_norm, out, out_stride, norms);
}

int sae_grads_unpack(sae_grads* h, const float* in, int64_t in_stride, void* const* tensors) {
  if (!h || !tensors || (!in && h->d) || (h->K > 1 && in_stride < 0) || (reinterpret_cast<uintptr_t>(in) & 3)) return SAE_ERR_INVALID_ARG;
  return run(h, (const void* const*)tensors, WITH_UNPACK, SAE_NORM_NONE, 0.0f, const_cast<float*>(in), in_stride, nullptr);
}

int sae_grads_last_cuda_error(const sae_grads* h) { return h ? h->last_cuda_error : g_grads_cuda_error; }

void sae_grads_destroy(sae_grads* h) {
  if (!h) return;
  DeviceGuard guard(h->device);
  if (guard.ok) cudaStreamSynchronize(h->stream);
  release(h);
}

}  // extern "C"
