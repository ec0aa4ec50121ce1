// Orthogonalisation of many matrices by Newton-Schulz products (sae_ortho_* of include/sae.h).
//
//   x <- g / (|g| + eps), then `steps` times  x <- a x + (b s + c s s) x  with s = x x' (x' x where a matrix is taller than wide)
//
// One call is a kernel for the norms, one that lays g out as two float16 parts, and three product kernels a step, each over
// the tiles of all matrices:  S = s;  B = b S + c S S;  x = a x + B x.
//
// Precision.  x is held as hi + lo, two float16 of a value scaled by a power of two (22 bits).  For results of 16 bits in bfloat16
// the products read hi alone (11 bits), and a x in the last product's epilogue reads both: a rounding of x itself to 11
// bits in every step would be multiplied by a^5 = 485 in the directions of small singular values (errors of 1.4e-2 for a gradient of a few
// strong directions over noise, 2e-4 this way).  Float32 and float16 results take hi and lo in all three products (hi lo + lo hi +
// hi hi): about the error of float32 products.
// Scales: singular values stay below a bound that follows from the coefficients, so no element of x, S or B leaves
// float16's range, and each is scaled up to near its top to keep small elements from becoming subnormal.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <map>
#include <new>
#include <tuple>
#include <vector>

#include "../../include/sae.h"
#include "sae_mma.cuh"
#include "sae_vec.cuh"

using namespace sae;

namespace {

constexpr int OT_THREADS = 256;
constexpr int OT_CHUNK = 2048;                // units of a row that a block takes
constexpr int OT_ARGS = 448;                  // matrices whose addresses travel as kernel arguments

// All matrices of one shape and precision.
struct Group {
  CUtensorMap x[2], s, b;
  __half *xp[2], *sp, *bp;
  long long x_plane, s_plane;                 // elements of a part
  int rows, cols, small, tall;
  int x_pitch, s_pitch;
  int s_parts;
  int x_tiles, x_tile_cols, s_tiles, s_tile_cols;   // tiles of one matrix
  int x_end, s_end;                           // tiles of all groups up to and with this one
  int first;                                  // its first matrix in the class's order
};

struct Matrix { const void* in; void* out; long long in_ld, out_ld; };
struct Place { int rows, cols, x_pitch, in_type, out_type, first_chunk, chunks; __half* x; long long x_plane; };
struct Chunk { int matrix, unit; };

struct Table { int n; Matrix m[OT_ARGS]; };

__device__ __forceinline__ void unit_of(const Matrix& m, int type, long long r, int c, int n, float (&v)[UNIT]) {
  const long long at = r * m.in_ld + c;
  if (type == SAE_TYPE_FLOAT) load_unit((const float*)m.in + at, n, v);
  else if (type == SAE_TYPE_BFLOAT) load_unit((const __nv_bfloat16*)m.in + at, n, v);
  else load_unit((const __half*)m.in + at, n, v);
}

// The sum of a value over the block, in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double v, double* scratch) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0;
  for (int i = 0; i < OT_THREADS / 32; ++i) s += scratch[i];
  return s;
}

__global__ void k_ortho_table(const __grid_constant__ Table t, Matrix* to) {
  for (int i = threadIdx.x; i < t.n; i += blockDim.x) to[i] = t.m[i];
}

// The sum of squares of every chunk, in double: squares of floats neither overflow nor vanish there.
__global__ void __launch_bounds__(OT_THREADS) k_ortho_norm(const Matrix* mats, const Place* places, const Chunk* chunks, double* sums) {
  __shared__ double scratch[OT_THREADS / 32];
  mma::let_next_start();
  mma::wait_for_previous();
  const Chunk ch = chunks[blockIdx.x];
  const Place p = places[ch.matrix];
  const Matrix m = mats[ch.matrix];
  const unsigned wide = (unsigned)(p.cols + UNIT - 1) / UNIT;
  double s = 0;
  for (int i = threadIdx.x; i < OT_CHUNK; i += OT_THREADS) {
    const unsigned u = (unsigned)ch.unit + (unsigned)i, r = u / wide, c = (u - r * wide) * UNIT;
    if (r >= (unsigned)p.rows) break;
    float v[UNIT];
    unit_of(m, p.in_type, r, (int)c, min(UNIT, p.cols - (int)c), v);
#pragma unroll
    for (int j = 0; j < UNIT; ++j) s += (double)v[j] * (double)v[j];
  }
  s = block_sum(s, scratch);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// x = g / (|g| + eps) as two float16 parts.
__global__ void __launch_bounds__(OT_THREADS) k_ortho_split(const Matrix* mats, const Place* places, const Chunk* chunks, const double* sums,
                                                            double eps, double scale) {
  __shared__ double scratch[OT_THREADS / 32];
  mma::let_next_start();
  const Chunk ch = chunks[blockIdx.x];
  const Place p = places[ch.matrix];
  mma::wait_for_previous();
  const Matrix m = mats[ch.matrix];
  double s = 0;
  for (int i = threadIdx.x; i < p.chunks; i += OT_THREADS) s += sums[p.first_chunk + i];
  const double factor = scale / (sqrt(block_sum(s, scratch)) + eps);
  const unsigned wide = (unsigned)(p.cols + UNIT - 1) / UNIT;
  for (int i = threadIdx.x; i < OT_CHUNK; i += OT_THREADS) {
    const unsigned u = (unsigned)ch.unit + (unsigned)i, r = u / wide, c = (u - r * wide) * UNIT;
    if (r >= (unsigned)p.rows) break;
    float v[UNIT];
    unit_of(m, p.in_type, r, (int)c, min(UNIT, p.cols - (int)c), v);
    u32 hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = (float)((double)v[2 * j] * factor), b = (float)((double)v[2 * j + 1] * factor);
      hi[j] = mma::pack_half(a, b);
      const float2 h = mma::unpack_half(hi[j]);
      lo[j] = mma::pack_half(a - h.x, b - h.y);
    }
    __half* const to = p.x + (long long)r * p.x_pitch + c;
    *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(to + p.x_plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// ---- products ---------------------------------------------------------------------------------------------------------
enum Phase { PHASE_S, PHASE_B, PHASE_X };

struct OrthoJob {
  int cols;
  bool bfloat;
  mma::Segments seg;
  const Group* groups;
  int phase, rows, total, from, last;
  float own, sum;                   // result = own * (the matrix's present value) + sum * acc
  const Matrix* mats;               // in the class's order, for the last step
  const Place* places;
  const int* order;

  struct Local { int first, step, g; };
  __device__ __forceinline__ Local begin(int cluster, int clusters) const { return {cluster, clusters, 0}; }
  __device__ __forceinline__ bool tile(Local& l, int i, mma::Tile& t) const {
    const int w = l.first + i * l.step;
    if (w >= total) return false;
    const bool px = phase == PHASE_X;
    while (w >= (px ? groups[l.g].x_end : groups[l.g].s_end)) ++l.g;
    const Group& g = groups[l.g];
    const int per = px ? g.x_tiles : g.s_tiles, wide = px ? g.x_tile_cols : g.s_tile_cols;
    const int before = l.g ? (px ? groups[l.g - 1].x_end : groups[l.g - 1].s_end) : 0;
    t.item = (w - before) / per;
    const int q = (w - before) % per;
    t.group = l.g;
    t.row = q / wide * rows;
    t.col = q % wide * cols;
    t.a_row = t.row;
    t.b_row = t.col;
    t.a_k = t.b_k = 0;
    const int zx = t.item * 2, zs = t.item * g.s_parts;
    int k;
    if (phase == PHASE_S) {
      t.a = t.b = &g.x[from];
      t.a_plane = t.b_plane = zx;
      t.a_rows_first = t.b_rows_first = g.tall;
      k = g.tall ? g.rows : g.cols;
    } else if (phase == PHASE_B) {
      t.a = t.b = &g.s;
      t.a_plane = t.b_plane = zs;
      t.a_rows_first = t.b_rows_first = false;
      k = g.small;
    } else {
      t.a = g.tall ? &g.x[from] : &g.b;
      t.b = g.tall ? &g.b : &g.x[from];
      t.a_plane = g.tall ? zx : zs;
      t.b_plane = g.tall ? zs : zx;
      t.a_rows_first = false;
      t.b_rows_first = !g.tall;
      k = g.small;
    }
    t.blocks = (k + mma::BLOCK_K - 1) / mma::BLOCK_K;
    return true;
  }

  struct Epilogue {
    const OrthoJob& job;
    int row, half;
    __device__ __forceinline__ Epilogue(const OrthoJob& j, const Local&, int r, int h) : job(j), row(r), half(h) {}
    __device__ __forceinline__ void finish() {}

    // own * (hi + lo of `from`) + sum * acc, `from` null: nothing of its own
    __device__ __forceinline__ void value(float (&v)[32], const __half* from, long long lo_at) const {
      if (from) {
        u32 w[16], u[16];
        mma::load_words(from, w);
        if (lo_at) mma::load_words(from + lo_at, u);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float2 h = mma::unpack_half(w[i]);
          if (lo_at) { const float2 l = mma::unpack_half(u[i]); h.x += l.x; h.y += l.y; }
          v[2 * i] = __fmaf_rn(job.own, h.x, job.sum * v[2 * i]);
          v[2 * i + 1] = __fmaf_rn(job.own, h.y, job.sum * v[2 * i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= job.sum;
      }
    }
    __device__ __forceinline__ void split(const float (&v)[32], __half* to, long long lo_at) const {
      u32 w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = mma::pack_half(v[2 * i], v[2 * i + 1]);
      mma::store_words(to, w);
      if (lo_at) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float2 h = mma::unpack_half(w[i]);
          w[i] = mma::pack_half(v[2 * i] - h.x, v[2 * i + 1] - h.y);
        }
        mma::store_words(to + lo_at, w);
      }
    }
    __device__ __forceinline__ void tile(const mma::Tile& t, const mma::Sums& sums) {
      const Group& g = job.groups[t.group];
      const bool px = job.phase == PHASE_X;
      const int r = t.row + row, rows = px ? g.rows : g.small, cols = px ? g.cols : g.small, pitch = px ? g.x_pitch : g.s_pitch;
      const int width = job.cols / 2;
      Matrix m = {};
      int type = 0;
      if (px && job.last) {
        const int i = job.order[g.first + t.item];
        m = job.mats[i];
        type = job.places[i].out_type;
      }
      for (int c = half * width; c < (half + 1) * width; c += 32) {
        const int col = t.col + c;
        if (col >= cols) break;                       // the same for the whole warp
        float v[32];
        mma::sums_of(sums, c, v);
        if (r >= rows) continue;
        const long long at = (long long)r * pitch + col;
        if (!px) {
          const long long plane = (long long)t.item * g.s_parts * g.s_plane, lo = g.s_parts == 2 ? g.s_plane : 0;
          value(v, job.phase == PHASE_B ? g.sp + plane + at : nullptr, lo);
          split(v, (job.phase == PHASE_B ? g.bp : g.sp) + plane + at, lo);
        } else {
          const long long plane = (long long)t.item * 2 * g.x_plane;
          value(v, g.xp[job.from] + plane + at, g.x_plane);
          if (!job.last) split(v, g.xp[job.from ^ 1] + plane + at, g.x_plane);
          else {
            const int n = min(32, cols - col);
            const long long to = r * m.out_ld + col;
            if (type == SAE_TYPE_FLOAT) mma::store_row((float*)m.out + to, v, n);
            else if (type == SAE_TYPE_BFLOAT) mma::store_row((__nv_bfloat16*)m.out + to, v, n);
            else mma::store_row((__half*)m.out + to, v, n);
          }
        }
      }
    }
  };
};

thread_local int g_ortho_cuda_error = 0;

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

int elem_bytes(int type) { return type == SAE_TYPE_FLOAT ? 4 : 2; }
bool type_ok(int type) { return type == SAE_TYPE_FLOAT || type == SAE_TYPE_BFLOAT || type == SAE_TYPE_HALF; }
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Groups whose products have the same number of parts: one launch a phase.
struct Class {
  int parts, cg, cols;
  int first, n;                  // groups
  int s_total, x_total;
};

// The largest |p(v)| and |b v^2 + c v^4| over 0 <= v <= top.
void bounds(const float* k, double top, double& p, double& q) {
  p = q = 0;
  for (int i = 0; i <= 4096; ++i) {
    const double v = top * i / 4096, s = v * v, e = k[1] * s + k[2] * s * s;
    p = std::max(p, std::fabs(v * (k[0] + e)));
    q = std::max(q, std::fabs(e));
  }
}

}  // namespace

struct sae_ortho {
  int K, T, device, num_sms, last_cuda_error, steps, chunks;
  double eps;
  cudaStream_t stream;
  std::vector<int64_t> rows, cols;
  std::vector<int> in_types, out_types;
  std::vector<float> coef;
  std::vector<double> s_scale, b_scale;          // of every step
  double x_scale;
  std::vector<Class> classes;
  char* arena;
  Group* groups;
  Matrix* mats;
  Place* places;
  Chunk* chunk_list;
  int* order;
  double* sums;
};

namespace {

int cuda_status(sae_ortho* h, cudaError_t e) {
  h->last_cuda_error = (int)e;
  cudaGetLastError();
  return e == cudaErrorMemoryAllocation ? SAE_ERR_NOMEM : SAE_ERR_CUDA;
}

void release(sae_ortho* h) {
  cudaFree(h->arena); cudaFree(h->groups); cudaFree(h->mats); cudaFree(h->places); cudaFree(h->chunk_list); cudaFree(h->order); cudaFree(h->sums);
  delete h;
}

template <typename T>
cudaError_t upload(T** to, const std::vector<T>& v, cudaStream_t st) {
  cudaError_t e = cudaMalloc((void**)to, std::max<size_t>(1, v.size()) * sizeof(T));
  if (e == cudaSuccess && !v.empty()) e = cudaMemcpyAsync(*to, v.data(), v.size() * sizeof(T), cudaMemcpyHostToDevice, st);
  return e;
}

// Tile shape of a class: time in units of a block's k loop, waves of tiles over the SMs (or pairs).
void choose_tiles(Class& c, const std::vector<Group>& groups, const std::vector<int>& count, int sms) {
  struct Shape { int cg, cols; double cost; };
  const Shape shapes[3] = {{2, c.parts == 1 ? 256 : 128, c.parts == 1 ? 2.0 : 1.2}, {1, 128, 1.3}, {1, 64, 1.0}};
  double best = 0;
  for (const Shape& s : shapes) {
    const int rows = 128 * s.cg, units = sms / s.cg;
    double work_s = 0, work_x = 0, longest_s = 0, longest_x = 0;
    for (int i = c.first; i < c.first + c.n; ++i) {
      const Group& g = groups[i];
      const auto tiles = [&](int r, int q) { return (double)((r + rows - 1) / rows) * ((q + s.cols - 1) / s.cols); };
      const int big = g.tall ? g.rows : g.cols;
      work_s += tiles(g.small, g.small) * big * count[i];
      work_x += (tiles(g.rows, g.cols) + tiles(g.small, g.small)) * g.small * count[i];
      longest_s = std::max(longest_s, (double)big);
      longest_x = std::max(longest_x, (double)g.small);
    }
    const double t = s.cost * (std::max(work_s / units, longest_s) + std::max(work_x / units, 2 * longest_x));
    if (best == 0 || t < best) { best = t; c.cg = s.cg; c.cols = s.cols; }
  }
}

cudaError_t products(const sae_ortho* h, const Class& c, const OrthoJob& job) {
  return mma::launch_products(job, c.cg, std::min(job.total, h->num_sms / c.cg), h->stream);
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), int blocks, cudaStream_t st, bool first, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(OT_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = first ? 0 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

extern "C" {

int sae_ortho_init(const sae_ortho_config* cfg, sae_ortho** out) {
  if (!cfg || !out) return SAE_ERR_INVALID_ARG;
  *out = nullptr;
  if (cfg->abi_version != SAE_ABI_VERSION) return SAE_ERR_ABI;
  const int K = cfg->num_rows, T = cfg->num_matrices;
  if (K < 1 || K > 1024 || T < 1 || !cfg->rows || !cfg->cols || !cfg->coefficients || cfg->device < 0 || cfg->steps < 1 || cfg->steps > 64 ||
      !(cfg->eps >= 0.0f) || !std::isfinite(cfg->eps) || (long long)K * T > (1 << 20)) return SAE_ERR_INVALID_ARG;
  for (int j = 0; j < T; ++j) {
    const int it = cfg->types ? cfg->types[j] : SAE_TYPE_FLOAT, ot = cfg->result_types ? cfg->result_types[j] : it;
    if (cfg->rows[j] < 0 || cfg->cols[j] < 0 || cfg->rows[j] > (1 << 20) || cfg->cols[j] > (1 << 20) || cfg->rows[j] * cfg->cols[j] > (1ll << 30) ||
        !type_ok(it) || !type_ok(ot)) return SAE_ERR_INVALID_ARG;
  }
  // Where the singular values can get to decides how far x, S and B may be scaled up in float16.
  std::vector<double> s_scale, b_scale;
  double top = 1.0, widest = 1.0;
  for (int i = 0; i < cfg->steps; ++i) {
    const float* k = cfg->coefficients + 3 * i;
    if (!std::isfinite(k[0]) || !std::isfinite(k[1]) || !std::isfinite(k[2])) return SAE_ERR_INVALID_ARG;
    double p, q;
    const double t = top * 1.01;                 // roundings
    bounds(k, t, p, q);
    if (!(p <= 16.0) || !(q <= 4096.0)) return SAE_ERR_INVALID_ARG;
    s_scale.push_back(std::exp2(std::floor(std::log2(32768.0 / (t * t)))));
    b_scale.push_back(std::exp2(std::min(14.0, std::floor(std::log2(32768.0 / std::max(q, 1e-6))))));
    top = std::max(p, 1e-3);
    widest = std::max(widest, top * 1.01);
  }
  sae_ortho* h = new (std::nothrow) sae_ortho();
  if (!h) return SAE_ERR_NOMEM;
  h->K = K; h->T = T; h->device = cfg->device; h->stream = (cudaStream_t)cfg->stream; h->steps = cfg->steps; h->eps = cfg->eps;
  h->x_scale = std::exp2(std::floor(std::log2(32768.0 / widest)));
  std::vector<Group> groups;
  std::vector<int> count, order;
  std::vector<Place> places;
  std::vector<Chunk> chunks;
  std::vector<std::vector<int>> members;
  DeviceGuard guard(cfg->device);
  cudaError_t e = guard.ok ? cudaSuccess : cudaGetLastError();
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, cfg->device);
  bool mapped = true;
  if (e == cudaSuccess) {
    try {
      h->rows.assign(cfg->rows, cfg->rows + T);
      h->cols.assign(cfg->cols, cfg->cols + T);
      h->coef.assign(cfg->coefficients, cfg->coefficients + 3 * cfg->steps);
      h->s_scale = s_scale; h->b_scale = b_scale;
      for (int j = 0; j < T; ++j) {
        h->in_types.push_back(cfg->types ? cfg->types[j] : SAE_TYPE_FLOAT);
        h->out_types.push_back(cfg->result_types ? cfg->result_types[j] : h->in_types[j]);
      }
      // groups: parts first (a class), then long sums before short ones
      std::map<std::tuple<int, int64_t, int64_t, int64_t>, std::vector<int>> by;
      for (int k = 0; k < K; ++k)
        for (int j = 0; j < T; ++j)
          if (h->rows[j] && h->cols[j]) {
            // bfloat16 results of a few rows or columns take both parts too: such products are short, and their roundings average out less
            const bool one = h->out_types[j] == SAE_TYPE_BFLOAT && std::min(h->rows[j], h->cols[j]) > 128;
            by[{one ? 1 : 2, -std::max(h->rows[j], h->cols[j]), h->rows[j], h->cols[j]}].push_back(k * T + j);
          }
      places.resize((size_t)K * T);
      int64_t bytes = 0;
      for (auto& kv : by) {
        Group g = {};
        g.s_parts = std::get<0>(kv.first);
        g.rows = (int)std::get<2>(kv.first); g.cols = (int)std::get<3>(kv.first);
        g.tall = g.rows > g.cols;
        g.small = std::min(g.rows, g.cols);
        g.x_pitch = (int)up(g.cols, 64); g.s_pitch = (int)up(g.small, 64);
        g.x_plane = (long long)g.rows * g.x_pitch; g.s_plane = (long long)g.small * g.s_pitch;
        g.first = (int)order.size();
        for (int i : kv.second) order.push_back(i);
        count.push_back((int)kv.second.size());
        members.push_back(kv.second);
        if (h->classes.empty() || h->classes.back().parts != g.s_parts) h->classes.push_back({g.s_parts, 1, 64, (int)groups.size(), 0, 0, 0});
        ++h->classes.back().n;
        groups.push_back(g);
        bytes += 2 * up(2 * g.x_plane * count.back() * 2, 1024) + 2 * up(g.s_parts * g.s_plane * count.back() * 2, 1024);
      }
      if (bytes) e = cudaMalloc((void**)&h->arena, (size_t)bytes);
      if (e == cudaSuccess) {
        char* at = h->arena;
        for (size_t i = 0; i < groups.size(); ++i) {
          Group& g = groups[i];
          const int n = count[i];
          const auto take = [&](int64_t elements) { __half* p = (__half*)at; at += up(elements * 2, 1024); return p; };
          for (int q = 0; q < 2; ++q) {
            g.xp[q] = take(2 * g.x_plane * n);
            mapped = mapped && mma::encode_map(&g.x[q], g.xp[q], false, g.cols, g.rows, 2ll * n, g.x_pitch, g.x_plane);
          }
          g.sp = take(g.s_parts * g.s_plane * n);
          g.bp = take(g.s_parts * g.s_plane * n);
          mapped = mapped && mma::encode_map(&g.s, g.sp, false, g.small, g.small, (int64_t)g.s_parts * n, g.s_pitch, g.s_plane);
          mapped = mapped && mma::encode_map(&g.b, g.bp, false, g.small, g.small, (int64_t)g.s_parts * n, g.s_pitch, g.s_plane);
          for (int q = 0; q < n; ++q) {
            const int i2 = members[i][q], j = i2 % T;
            Place& p = places[i2];
            p.rows = g.rows; p.cols = g.cols; p.x_pitch = g.x_pitch; p.in_type = h->in_types[j]; p.out_type = h->out_types[j];
            p.x = g.xp[0] + (long long)q * 2 * g.x_plane; p.x_plane = g.x_plane;
            p.first_chunk = (int)chunks.size();
            const int64_t units = (int64_t)g.rows * ((g.cols + UNIT - 1) / UNIT);
            for (int64_t u = 0; u < units; u += OT_CHUNK) chunks.push_back({i2, (int)u});
            p.chunks = (int)chunks.size() - p.first_chunk;
          }
        }
        for (Class& c : h->classes) {
          choose_tiles(c, groups, count, h->num_sms);
          for (int i = c.first; i < c.first + c.n; ++i) {
            Group& g = groups[i];
            const int r = 128 * c.cg;
            g.x_tile_cols = (g.cols + c.cols - 1) / c.cols; g.x_tiles = (g.rows + r - 1) / r * g.x_tile_cols;
            g.s_tile_cols = (g.small + c.cols - 1) / c.cols; g.s_tiles = (g.small + r - 1) / r * g.s_tile_cols;
            c.x_total += g.x_tiles * count[i]; c.s_total += g.s_tiles * count[i];
            g.x_end = c.x_total; g.s_end = c.s_total;
          }
        }
        h->chunks = (int)chunks.size();
      }
    } catch (...) {
      release(h);
      return SAE_ERR_NOMEM;
    }
  }
  if (e == cudaSuccess && !mapped) e = cudaErrorUnknown;
  if (e == cudaSuccess) e = upload(&h->groups, groups, h->stream);
  if (e == cudaSuccess) e = upload(&h->places, places, h->stream);
  if (e == cudaSuccess) e = upload(&h->chunk_list, chunks, h->stream);
  if (e == cudaSuccess) e = upload(&h->order, order, h->stream);
  if (e == cudaSuccess) e = cudaMalloc((void**)&h->mats, (size_t)K * T * sizeof(Matrix));
  if (e == cudaSuccess) e = cudaMalloc((void**)&h->sums, std::max<size_t>(1, chunks.size()) * sizeof(double));
  if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
  if (e != cudaSuccess) {
    const int rc = cuda_status(h, e);
    g_ortho_cuda_error = (int)e;
    release(h);
    return rc;
  }
  *out = h;
  return SAE_OK;
}

int sae_ortho_run(sae_ortho* h, const void* const* matrices, const int64_t* pitches, void* const* results, const int64_t* result_pitches) {
  if (!h || !matrices || !results) return SAE_ERR_INVALID_ARG;
  const int n = h->K * h->T;
  for (int i = 0; i < n; ++i) {
    const int j = i % h->T;
    if (!h->rows[j] || !h->cols[j]) continue;
    if (!matrices[i] || !results[i] || (reinterpret_cast<uintptr_t>(matrices[i]) & (uintptr_t)(elem_bytes(h->in_types[j]) - 1)) ||
        (reinterpret_cast<uintptr_t>(results[i]) & (uintptr_t)(elem_bytes(h->out_types[j]) - 1)) ||
        (pitches && h->rows[j] > 1 && pitches[i] < h->cols[j]) || (result_pitches && h->rows[j] > 1 && result_pitches[i] < h->cols[j]))
      return SAE_ERR_INVALID_ARG;
  }
  if (!h->chunks) return SAE_OK;
  DeviceGuard guard(h->device);
  if (!guard.ok) return cuda_status(h, cudaGetLastError());
  cudaError_t e = cudaSuccess;
  static thread_local Table table;
  bool first = true;
  for (int i = 0; i < n && e == cudaSuccess; i += OT_ARGS) {
    table.n = std::min(OT_ARGS, n - i);
    for (int q = 0; q < table.n; ++q) {
      const int64_t cols = h->cols[(i + q) % h->T];
      table.m[q] = {matrices[i + q], results[i + q], pitches ? pitches[i + q] : cols, result_pitches ? result_pitches[i + q] : cols};
    }
    e = launch(k_ortho_table, 1, h->stream, true, table, h->mats + i);
    first = false;
  }
  if (e == cudaSuccess) e = launch(k_ortho_norm, h->chunks, h->stream, first, (const Matrix*)h->mats, (const Place*)h->places, (const Chunk*)h->chunk_list, h->sums);
  if (e == cudaSuccess) e = launch(k_ortho_split, h->chunks, h->stream, false, (const Matrix*)h->mats, (const Place*)h->places, (const Chunk*)h->chunk_list, (const double*)h->sums, h->eps, h->x_scale);
  for (const Class& c : h->classes) {
    OrthoJob job = {};
    job.cols = c.cols;
    job.rows = 128 * c.cg;
    job.groups = h->groups + c.first;
    job.mats = h->mats;
    job.places = h->places;
    job.order = h->order;
    if (c.parts == 2) job.seg = {3, {0, 1, 0}, {1, 0, 0}};
    else job.seg = {1, {0}, {0}};
    for (int i = 0; i < h->steps && e == cudaSuccess; ++i) {
      const float* k = h->coef.data() + 3 * i;
      const double sx = h->x_scale, ss = h->s_scale[i], sb = h->b_scale[i];
      job.from = i & 1;
      job.phase = PHASE_S; job.total = c.s_total; job.own = 0; job.sum = (float)(ss / (sx * sx));
      e = products(h, c, job);
      job.phase = PHASE_B; job.own = (float)(k[1] * sb / ss); job.sum = (float)(k[2] * sb / (ss * ss));
      if (e == cudaSuccess) e = products(h, c, job);
      job.last = i + 1 == h->steps;
      job.phase = PHASE_X; job.total = c.x_total;
      const double to = job.last ? 1.0 / sx : 1.0;
      job.own = (float)(k[0] * to); job.sum = (float)(to / sb);
      if (e == cudaSuccess) e = products(h, c, job);
    }
  }
  return e == cudaSuccess ? SAE_OK : cuda_status(h, e);
}

int sae_ortho_last_cuda_error(const sae_ortho* h) { return h ? h->last_cuda_error : g_ortho_cuda_error; }

void sae_ortho_destroy(sae_ortho* h) {
  if (!h) return;
  DeviceGuard guard(h->device);
  if (guard.ok) cudaStreamSynchronize(h->stream);
  release(h);
}

}  // extern "C"
