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
#include <vector>

using namespace sae;

namespace {

typedef unsigned long long u64;
typedef unsigned int u32;

constexpr int GT_THREADS = 256;
constexpr int GT_TILE = 8192;            // elements of one tensor that a block handles at a time
constexpr int GT_BLOCKS_PER_SM = 8;      // 2048 resident threads
constexpr int PTRS_SMALL = 64;           // tensor pointers that travel as kernel arguments
constexpr int PTRS_LARGE = 448;
constexpr int PTRS_UPLOAD = 3840;        // pointers one upload launch carries (30 KB of the 32 KB of arguments)
constexpr double COEF_EPS = 1e-6;

// One tile: `count` elements of tensor `tensor` from element `start`, at element `at` of a packed row.
struct __align__(16) Tile {
  u32 tensor, start, count, type;
  long long at, pad;
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

// A thread's pieces are 16 bytes, neighbouring threads' pieces neighbours in memory.
template <int KIND, typename T>
__device__ __forceinline__ void tile_norm(Running<KIND>& r, const T* p, u32 cnt) {
  constexpr int V = 16 / (int)sizeof(T), N = GT_TILE / (GT_THREADS * V);
  const u32 tid = threadIdx.x;
  if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const u32 whole = cnt / V;
    Raw<T, V> raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (cnt == GT_TILE || i * GT_THREADS + tid < whole) raw[i].load(p + (i * GT_THREADS + tid) * V);
      else raw[i].clear();
    const u32 e = whole * V + tid;
    const float last = cnt != GT_TILE && e < cnt ? to_f(p[e]) : 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 8 / V) {
      float v[8];
      if constexpr (V == 8) {
        raw[i].widen(v);
      } else {
        raw[i].widen(*reinterpret_cast<float (*)[4]>(&v[0]));
        raw[i + 1].widen(*reinterpret_cast<float (*)[4]>(&v[4]));
      }
      r.eight(v);
    }
    r.one(last);
  } else {
    for (u32 e = tid; e < cnt; e += GT_THREADS) r.one(to_f(p[e]));
  }
}

// blockIdx.y: the row (worker).  The row's tiles are dealt out in runs of neighbours, one run a block.  The block
// that comes last (a ticket a row, back at zero after it) joins the runs' values in their order.
template <int KIND, int N>
__global__ void __launch_bounds__(GT_THREADS) k_grads_norm(const __grid_constant__ Ptrs<N> ptrs, const Tile* __restrict__ tiles,
                                                           int ntiles, int T, u64* partials, u32* tickets, float max_norm,
                                                           float* coefs, float* norms) {
  __shared__ u64 sh[GT_THREADS / 32];
  __shared__ int sh_last;
  const int row = blockIdx.y, B = gridDim.x;
  const int t0 = (int)((long long)ntiles * blockIdx.x / B), t1 = (int)((long long)ntiles * (blockIdx.x + 1) / B);
  Running<KIND> r; r.zero();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Tile next = t0 < t1 ? tiles[t0] : Tile{};
  for (int t = t0; t < t1; ++t) {
    const Tile ti = next;
    if (t + 1 < t1) next = tiles[t + 1];
    void* base = ptrs.get(row * T + (int)ti.tensor);
    if (ti.type == SAE_TYPE_FLOAT) tile_norm<KIND, float>(r, (const float*)base + ti.start, ti.count);
    else if (ti.type == SAE_TYPE_BFLOAT) tile_norm<KIND, __nv_bfloat16>(r, (const __nv_bfloat16*)base + ti.start, ti.count);
    else tile_norm<KIND, __half>(r, (const __half*)base + ti.start, ti.count);
  }
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
// coef = 1 multiplies exactly, so one form serves scaled and plain copies.  A piece is what makes the wider side 16 bytes, so
// that stores fill whole sectors; where the sides are not aligned for it, lane by lane, neighbours by neighbouring lanes,
// which any alignment coalesces.  In place each element is read and written by the same thread.
template <typename S, typename D>
struct Moved {
  static constexpr int V = 16 / (int)(sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D)), N = GT_TILE / (GT_THREADS * V);
  Raw<S, V> raw[N];
  bool aligned;
  __device__ __forceinline__ void load(const S* s, const D* d, u32 cnt) {
    aligned = (reinterpret_cast<uintptr_t>(s) & (V * sizeof(S) - 1)) == 0 && (reinterpret_cast<uintptr_t>(d) & (V * sizeof(D) - 1)) == 0;
    if (!aligned) return;
    const u32 whole = cnt / V;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (cnt == GT_TILE || i * GT_THREADS + threadIdx.x < whole) raw[i].load_once(s + (i * GT_THREADS + threadIdx.x) * V);
  }
  __device__ __forceinline__ void store(const S* s, D* d, u32 cnt, float coef) {
    if (aligned) {
      const u32 whole = cnt / V;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (cnt == GT_TILE || i * GT_THREADS + threadIdx.x < whole) {
          float v[V];
          raw[i].widen(v);
#pragma unroll
          for (int q = 0; q < V; ++q) v[q] = __fmul_rn(v[q], coef);
          Raw<D, V> o;
          o.round(v);
          o.store_stream(d + (i * GT_THREADS + threadIdx.x) * V);
        }
      }
      const u32 e = whole * V + threadIdx.x;
      if (e < cnt) d[e] = from_f<D>(__fmul_rn(to_f(s[e]), coef));
    } else {
      u32 e = threadIdx.x;
      for (; e + 7 * GT_THREADS < cnt; e += 8 * GT_THREADS) {
        S v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = s[e + q * GT_THREADS];
#pragma unroll
        for (int q = 0; q < 8; ++q) d[e + q * GT_THREADS] = from_f<D>(__fmul_rn(to_f(v[q]), coef));
      }
      for (; e < cnt; e += GT_THREADS) d[e] = from_f<D>(__fmul_rn(to_f(s[e]), coef));
    }
  }
};

enum { MODE_CLIP, MODE_PACK, MODE_UNPACK };

// In place, a 16-bit tensor is scaled by the coefficient rounded to its own type, which is what torch's in-place product with
// a scalar tensor does: replacing a torch clipping changes no bit.  Not below the type's normal numbers (a half's end at
// 2^-14), where the rounding would cost digits or leave zero.
template <typename T> __device__ __forceinline__ float coef_for(float c) { return c; }
template <> __device__ __forceinline__ float coef_for<__nv_bfloat16>(float c) { return c >= 1.17549435e-38f ? to_f(from_f<__nv_bfloat16>(c)) : c; }
template <> __device__ __forceinline__ float coef_for<__half>(float c) { return c >= 6.103515625e-5f ? to_f(from_f<__half>(c)) : c; }

template <int MODE, typename T>
__device__ __forceinline__ void tile_move(void* base, const Tile& ti, float* vec, const float* coefs, int row, bool& waited, float& coef) {
  T* const g = (T*)base + ti.start;
  auto wait = [&]() {                     // the norm's kernel, after this one's first loads are on their way
    if (waited) return;
    cudaGridDependencySynchronize();
    coef = coefs ? *(volatile const float*)(coefs + row) : 1.0f;
    waited = true;
  };
  if (MODE == MODE_PACK) {
    Moved<T, float> m;
    float* const d = vec + ti.at;
    m.load(g, d, ti.count);
    wait();
    m.store(g, d, ti.count, coef);
  } else if (MODE == MODE_CLIP) {
    wait();
    const float c = coef_for<T>(coef);
    if (c == 1.0f) return;                // nothing would change
    Moved<T, T> m;
    m.load(g, g, ti.count);
    m.store(g, g, ti.count, c);
  } else {
    Moved<float, T> m;
    const float* const s = vec + ti.at;
    m.load(s, g, ti.count);
    m.store(s, g, ti.count, 1.0f);
  }
}

// The tiles run backwards: the norm's pass went forwards, and what it read last is what L2 still holds.
template <int MODE, int N>
__global__ void __launch_bounds__(GT_THREADS) k_grads_move(const __grid_constant__ Ptrs<N> ptrs, const Tile* __restrict__ tiles,
                                                           int ntiles, int T, const float* coefs, float* vec, long long stride) {
  const int row = (int)(gridDim.y - 1 - blockIdx.y), B = gridDim.x, b = B - 1 - (int)blockIdx.x;
  const int t0 = (int)((long long)ntiles * b / B), t1 = (int)((long long)ntiles * (b + 1) / B);
  bool waited = false;
  float coef = 1.0f;
  float* const v = MODE == MODE_CLIP ? nullptr : vec + row * stride;
  Tile next = t0 < t1 ? tiles[t1 - 1] : Tile{};
  for (int t = t1 - 1; t >= t0; --t) {
    const Tile ti = next;
    if (t > t0) next = tiles[t - 1];
    void* base = ptrs.get(row * T + (int)ti.tensor);
    if (ti.type == SAE_TYPE_FLOAT) tile_move<MODE, float>(base, ti, v, coefs, row, waited, coef);
    else if (ti.type == SAE_TYPE_BFLOAT) tile_move<MODE, __nv_bfloat16>(base, ti, v, coefs, row, waited, coef);
    else tile_move<MODE, __half>(base, ti, v, coefs, row, waited, coef);
    if (MODE == MODE_CLIP && coef == 1.0f) return;
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

// Blocks of one row when `rows` rows share a launch: every SM full once, one tile a block at least.
int row_blocks(const sae_grads* h, int rows) {
  const int want = (h->num_sms * GT_BLOCKS_PER_SM + rows - 1) / rows;
  return std::max(1, std::min(std::min(h->ntiles, h->max_blocks), want));
}

template <int N>
cudaError_t launch_norm(sae_grads* h, const Ptrs<N>& p, int rows, int kind, float max_norm, float* norms) {
  const dim3 grid((unsigned)row_blocks(h, rows), (unsigned)rows);
#define NORM(KIND) k_grads_norm<KIND, N><<<grid, GT_THREADS, 0, h->stream>>>(p, h->tiles, h->ntiles, h->T, h->partials, h->tickets, \
                                                                              max_norm, h->coefs, norms)
  if (kind == SAE_NORM_TWO) NORM(SAE_NORM_TWO);
  else if (kind == SAE_NORM_ONE) NORM(SAE_NORM_ONE);
  else NORM(SAE_NORM_MAX);
#undef NORM
  return cudaGetLastError();
}

template <int MODE, int N>
cudaError_t launch_move(sae_grads* h, const Ptrs<N>& p, int rows, bool scaled, float* vec, long long stride) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)row_blocks(h, rows), (unsigned)rows);
  cfg.blockDim = dim3(GT_THREADS);
  cfg.stream = h->stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = scaled ? 1 : 0;           // only behind this call's own norm kernel
  return cudaLaunchKernelEx(&cfg, k_grads_move<MODE, N>, p, (const Tile*)h->tiles, h->ntiles, h->T,
                            (const float*)(scaled ? h->coefs : nullptr), vec, stride);
}

enum { WITH_NORM = 1, WITH_CLIP = 2, WITH_PACK = 4, WITH_UNPACK = 8 };

template <int N>
cudaError_t launch_all(sae_grads* h, const Ptrs<N>& p, int rows, int what, int kind, float max_norm, float* vec, long long stride, float* norms) {
  cudaError_t e = cudaSuccess;
  const bool scaled = (what & WITH_NORM) != 0;
  if (scaled) e = launch_norm<N>(h, p, rows, kind, max_norm, norms);
  if (e != cudaSuccess || h->ntiles == 0) return e;
  if (what & WITH_CLIP) e = launch_move<MODE_CLIP, N>(h, p, rows, scaled, vec, stride);
  if (what & WITH_PACK) e = launch_move<MODE_PACK, N>(h, p, rows, scaled, vec, stride);
  if (what & WITH_UNPACK) e = launch_move<MODE_UNPACK, N>(h, p, rows, scaled, vec, stride);
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
    e = launch_all<PTRS_SMALL>(h, p, h->K, what, kind, max_norm, vec, stride, norms);
  } else if (n <= PTRS_LARGE) {
    Ptrs<PTRS_LARGE> p;
    for (size_t i = 0; i < n; ++i) p.p[i] = const_cast<void*>(tensors[i]);
    e = launch_all<PTRS_LARGE>(h, p, h->K, what, kind, max_norm, vec, stride, norms);
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
    if (e == cudaSuccess) e = launch_all<0>(h, p, h->K, what, kind, max_norm, vec, stride, norms);
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
    nt += (n + GT_TILE - 1) / GT_TILE;
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
      for (int64_t s = 0; s < h->sizes[j]; s += GT_TILE) {
        Tile t = {};
        t.tensor = (u32)j; t.start = (u32)s; t.count = (u32)std::min<int64_t>(GT_TILE, h->sizes[j] - s);
        t.type = (u32)h->types[j]; t.at = at + s;
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
