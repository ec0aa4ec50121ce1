// Linear cross entropy (sae_linear_ce_* of include/sae.h): the loss of a linear output layer and its gradients, no logits kept.
//
// forward   rows that take part are gathered (k_ce_rows), then one product kernel makes z = x w' tile by tile and keeps of each row
//           the running maximum, the sum of exp(z - maximum) and the target's z; the runs are joined (k_ce_join).
// backward  z is made again, to the last bit as it was, piece by piece of the classes, and leaves the tensor cores as p = (exp(z - lse) - [target]) g
//           in 16 bits; lse is a float and what its rounding left out, so that p of a row adds up to 0 however large its logits are;
//           p w is added to dx's float sums, p' x is the piece's dweight.  8 N D V operations in all, against 6 with all of z kept.
//
// A row without a target costs nothing: the gathered rows are counted on the device, and every kernel goes by that count.  Gathering is
// also where rows get the 16-byte pitch that TMA wants and float rows become three bfloat16 parts.
#include <cuda_runtime.h>

#include <algorithm>

#include "../../include/sae.h"
#include "sae_mma.cuh"
#include "sae_vec.cuh"

using namespace sae;

namespace {

constexpr int CE_THREADS = 256;
constexpr int CE_ROWS = 32;                   // rows of a block of k_ce_rows
constexpr int CE_COUNT_ROWS = 4096;           // rows counted by a block of k_ce_count
constexpr int CE_SCAN_ROWS = 16384;           // up to here every block counts the rows before its own by itself
constexpr int CE_CHUNK = 1024;                // units that a block copies
constexpr int64_t CE_PIECE_BYTES = 256ll << 20;
constexpr float LOG2E = 1.44269504088896340736f;

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int elem_bytes(int type) { return type == SAE_TYPE_FLOAT ? 4 : 2; }
bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// log(sum) + maximum as a float and what that leaves out (the sum's error, exactly).  Behind a logit of 30000 a float's last bit is 0.2 % of p.
__device__ __forceinline__ float lse_of(float m, float s, float& rest) {
  const float l = logf(s), lse = m + l, back = lse - m;
  rest = (m - (lse - back)) + (l - back);
  return lse;
}
// exp(z - lse), the exponent for base 2: both subtractions before they are rounded to much.
__device__ __forceinline__ float log2_p(float z, float lse, float rest_log2e) { return __fmaf_rn(z - lse, LOG2E, -rest_log2e); }

// ---- pieces and splits ----------------------------------------------------------------------------------------------------
// Pieces of the classes.  p has room for all rows times `piece` classes; where fewer rows take part, a piece has as many times more classes, up
// to CE_WIDER, and the launches for the last pieces find nothing to do (16384 x 768 x 30522, 15 % of the targets: one piece in place of five).
constexpr int CE_WIDER = 8;
struct Pieces {
  int piece, number, classes, most;     // most: times wider at most
  int64_t rows;
  __device__ __host__ __forceinline__ int times(int count) const {
    const int64_t taken = ((int64_t)count + 255) / 256 * 256;
    const int can = (int)(taken ? (rows / taken < most ? rows / taken : most) : most);
    const int left = (number + can - 1) / can;                       // pieces
    return (number + left - 1) / left;
  }
};

// Time of a list of tiles that the clusters take in turn: n1 of them, then n2, in units of a tile's k.
__device__ __host__ inline float list_time(u32 n1, float t1, u32 n2, float t2, u32 clusters) {
  const u32 whole1 = n1 / clusters, left1 = n1 - whole1 * clusters, whole = (n1 + n2) / clusters, left = n1 + n2 - whole * clusters;
  float most = 0;
  for (int i = 0; i < 3; ++i) {                   // the loads are the same between these clusters
    const u32 at = i == 0 ? 0 : i == 1 ? left1 : left, a = whole1 + (at < left1), b = whole + (at < left) - a;
    const float t = (float)a * t1 + (float)b * t2;
    most = t > most ? t : most;
  }
  return most;
}
// How often the classes of a piece are split for dx, where there are too few tiles for the clusters, or tiles of dweight beside them.  A tile's
// own sums, read and written in float, are about 500 k (2458 x 768 and 6144 classes: 2 splits 25 us, 7 splits, which fill three waves
// to 95 %, 44 us).
struct Product {
  int dx_blocks, across, clusters, depth, room;   // blocks of rows, tiles across the features; classes of a whole piece; row blocks that the sums have place for
  int dw_tiles, count;
  __device__ __host__ inline float time(int s) const {
    const u32 n = (u32)(dx_blocks * across * s);
    const float dx = (float)depth / (float)s + 500.0f, dw = (float)count;
    return dx > dw ? list_time(n, dx, dw_tiles, dw, clusters) : list_time(dw_tiles, dw, n, dx, clusters);
  }
  __device__ __host__ inline int splits() const {
    int best = 1;
    float least = 0;
    for (int s = 1; s <= 8 && (s == 1 || (int64_t)s * dx_blocks <= room); ++s) {
      const float t = time(s);
      if (s == 1 || t < least) { least = t; best = s; }
    }
    return best;
  }
};

// What the gathering kernel leaves for those behind it: the rows that take part, a ticket of the forward pass, and what their number decides.
enum Counted { COUNT_ROWS, COUNT_TICKET, COUNT_TIMES, COUNT_SPLITS, COUNT_WORDS };      // how much wider pieces are; splits of dx

// ---- gathering ----------------------------------------------------------------------------------------------------------
struct RowsArgs {
  const void* x;
  const int64_t* target;
  int64_t x_pitch, rows, ignore;
  int type, parts, features, classes, pitch;      // pitch of the gathered rows
  unsigned short* xg;
  int64_t xg_plane;
  const int* before;                              // rows that take part in each CE_COUNT_ROWS, where there are many
  int* index;                                     // of every gathered row: where it came from,
  int* at;                                        // its target (-1: out of range),
  int* counted;                                   // and how many there are: [COUNT_WORDS]
  int64_t* count;                                 // forward: the caller's
  float *loss, *lse, *rest;                       // forward: 0 for rows that take no part (loss NULL: reduced; rest NULL: not wanted)
  // backward
  Pieces pieces;
  Product product;                                // of a piece, but for what the count gives
  bool both;                                      // dx and dweight in one list
  int product_rows;                               // rows of a tile of it
  const float *lse_in, *rest_in, *dloss;
  const int64_t* count_in;
  int reduction;
  float p_scale;
  float *lse_g, *rest_g, *g, *alpha;              // of every gathered row: lse and the rest of it, its factor in p;  the factor behind the sums
  const float* g_top;                             // the largest |dloss|, for float16 p
  void* dx;
  // copies beside it
  const void* w;
  int64_t w_pitch, wg_plane;
  unsigned short* wg;
  const void* bias;
  int bias_type, bias_room;
  float* bias_out;
  int row_blocks, w_blocks;
};

// A float as the exact sum of three bfloat16: each takes the leading 8 bits of what is left.
__device__ __forceinline__ void three_parts(float v, float (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = __bfloat162float(__float2bfloat16_rz(v));
    v = isfinite(p[i]) ? v - p[i] : 0.0f;
  }
}

// One unit of a row to its place in every part.
__device__ __forceinline__ void put_unit(const void* from, int type, int parts, int n, unsigned short* to, int64_t plane) {
  u32 w[4];
  if (parts == 1) {                     // 16 bits stay as they are
    const unsigned short* p = (const unsigned short*)from;
    if (n == UNIT && (reinterpret_cast<uintptr_t>(p) & 15) == 0) *reinterpret_cast<uint4*>(to) = __ldg(reinterpret_cast<const uint4*>(p));
    else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? p[2 * i] : 0u) | (2 * i + 1 < n ? (u32)p[2 * i + 1] << 16 : 0u);
      *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return;
  }
  float v[UNIT], p[UNIT][3];
  load_unit((const float*)from, n, v);
#pragma unroll
  for (int i = 0; i < UNIT; ++i) three_parts(v[i], p[i]);
#pragma unroll
  for (int q = 0; q < 3; ++q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = mma::pack_bfloat(p[2 * i][q], p[2 * i + 1][q]);
    *reinterpret_cast<uint4*>(to + q * plane) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

__device__ __forceinline__ int block_total(int v, int* scratch) {
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  int s = 0;
  for (int i = 0; i < CE_THREADS / 32; ++i) s += scratch[i];
  return s;
}
__device__ __forceinline__ int rows_with_target(const RowsArgs& a, int64_t from, int64_t to, int* scratch) {
  int n = 0;
  for (int64_t i = from + threadIdx.x; i < to; i += CE_THREADS) n += __ldg(a.target + i) != a.ignore;
  return block_total(n, scratch);
}

__global__ void __launch_bounds__(CE_THREADS) k_ce_count(const __grid_constant__ RowsArgs a, int* before) {
  __shared__ int scratch[CE_THREADS / 32];
  const int64_t from = (int64_t)blockIdx.x * CE_COUNT_ROWS;
  const int n = rows_with_target(a, from, min(from + CE_COUNT_ROWS, a.rows), scratch);
  if (threadIdx.x == 0) before[blockIdx.x] = n;
}

// The largest |dloss| of the rows that take part, or 1 where that is 0 or not finite.
__global__ void __launch_bounds__(1024) k_ce_top(const __grid_constant__ RowsArgs a, float* top) {
  __shared__ float scratch[32];
  mma::wait_for_previous();             // the gathering kernel waits for this one alone, and reads what k_ce_count wrote before it
  float m = 0;
  for (int64_t i = threadIdx.x; i < a.rows; i += 1024)
    if (a.target[i] != a.ignore) { const float v = fabsf(a.dloss[i]); if (v <= 3.0e38f) m = fmaxf(m, v); }
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 32; ++i) m = fmaxf(m, scratch[i]);
    *top = m > 0 ? m : 1.0f;
  }
}

template <bool BACKWARD>
__global__ void __launch_bounds__(CE_THREADS) k_ce_rows(const __grid_constant__ RowsArgs a) {
  __shared__ int scratch[CE_THREADS / 32], place[CE_ROWS];
  mma::let_next_start();
  mma::wait_for_previous();
  int b = blockIdx.x;
  if (b >= a.row_blocks) {              // copies of the weights' rows and of the bias
    b -= a.row_blocks;
    if (b < a.w_blocks) {
      const unsigned wide = (unsigned)a.pitch / UNIT;
      for (int i = threadIdx.x; i < CE_CHUNK; i += CE_THREADS) {
        const int64_t u = (int64_t)b * CE_CHUNK + i, r = u / wide;
        const int c = (int)(u - r * wide) * UNIT;
        if (r >= a.classes) break;
        put_unit((const char*)a.w + (r * a.w_pitch + c) * (a.type == SAE_TYPE_FLOAT ? 4 : 2), a.type, a.parts, min(UNIT, a.features - c),
                 a.wg + r * a.pitch + c, a.wg_plane);
      }
    } else {
      const int j = (b - a.w_blocks) * CE_THREADS + threadIdx.x;
      if (j < a.bias_room) {
        float v = __int_as_float(0xff800000);                  // classes that there are not
        if (j < a.classes)
          v = a.bias_type == SAE_TYPE_FLOAT ? ((const float*)a.bias)[j]
              : a.bias_type == SAE_TYPE_BFLOAT ? to_f(((const __nv_bfloat16*)a.bias)[j]) : to_f(((const __half*)a.bias)[j]);
        a.bias_out[j] = v;
      }
    }
    return;
  }
  const int64_t r0 = (int64_t)b * CE_ROWS;
  int base = 0;
  if (a.before) {
    const int64_t whole = r0 / CE_COUNT_ROWS;
    int n = 0;
    for (int64_t i = threadIdx.x; i < whole; i += CE_THREADS) n += a.before[i];
    base = block_total(n, scratch) + rows_with_target(a, whole * CE_COUNT_ROWS, r0, scratch);
  } else base = rows_with_target(a, 0, r0, scratch);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 0) {
    const int64_t r = r0 + lane;
    const int64_t t = r < a.rows ? a.target[r] : a.ignore;
    const bool part = r < a.rows && t != a.ignore;
    const u32 mask = __ballot_sync(0xffffffffu, part);
    const int to = base + __popc(mask & ((1u << lane) - 1));
    place[lane] = part ? to : -1;
    if (part) {
      const int cls = t >= 0 && t < a.classes ? (int)t : -1;
      a.index[to] = (int)r;
      a.at[to] = cls;
      if constexpr (BACKWARD) {
        a.lse_g[to] = cls < 0 ? __int_as_float(0x7fc00000) : a.lse_in[r];
        a.rest_g[to] = a.rest_in ? a.rest_in[r] : 0.0f;
        float f = a.reduction == SAE_REDUCE_NONE ? a.dloss[r] / (a.g_top ? *a.g_top : 1.0f) : 1.0f;
        a.g[to] = f * a.p_scale;
      }
    } else if (r < a.rows) {
      if constexpr (!BACKWARD) {
        a.lse[r] = 0;
        if (a.rest) a.rest[r] = 0;
        if (a.loss) a.loss[r] = 0;
      }
    }
    if (b + 1 == a.row_blocks && lane == 0) {
      const int n = base + __popc(mask);
      *a.counted = n;
      a.counted[COUNT_TICKET] = 0;
      if constexpr (!BACKWARD) *a.count = n;
      else {
        float f = 1.0f;
        if (n == 0) f = 0.0f;                                  // sums of nothing
        else if (a.reduction == SAE_REDUCE_NONE) f = a.g_top ? *a.g_top : 1.0f;
        else f = a.reduction == SAE_REDUCE_MEAN ? *a.dloss / (float)*a.count_in : *a.dloss;
        *a.alpha = f / a.p_scale;
      }
    }
  }
  __syncthreads();
  const int es = a.type == SAE_TYPE_FLOAT ? 4 : 2;
  for (int i = warp; i < CE_ROWS; i += CE_THREADS / 32) {
    const int64_t r = r0 + i;
    if (r >= a.rows) break;
    const int to = place[i];
    if (to >= 0) {
      if (!a.xg) continue;
      const char* from = (const char*)a.x + r * a.x_pitch * es;
      for (int c = lane * UNIT; c < a.pitch; c += 32 * UNIT)
        put_unit(from + (int64_t)c * es, a.type, a.parts, min(UNIT, a.features - c), a.xg + (int64_t)to * a.pitch + c, a.xg_plane);
    } else if constexpr (BACKWARD) {
      if (a.dx) {
        char* row = (char*)a.dx + r * a.features * es;
        if (es == 4) for (int c = lane; c < a.features; c += 32) ((float*)row)[c] = 0.0f;
        else for (int c = lane; c < a.features; c += 32) ((unsigned short*)row)[c] = 0;
      }
    }
  }
  // (here, where other warps still copy: 0.5 us; in the kernels that need it, it took them 1 to 4 us each)
  if (BACKWARD && a.xg && b + 1 == a.row_blocks && threadIdx.x == 0) {
    const int n = a.counted[COUNT_ROWS], times = a.pieces.times(n), piece = a.pieces.piece * times;
    Product q = a.product;
    q.count = n;
    q.dx_blocks = (n + a.product_rows - 1) / a.product_rows;
    q.depth = piece;
    q.dw_tiles = a.both ? (min(piece, a.classes) + a.product_rows - 1) / a.product_rows * q.across : 0;
    a.counted[COUNT_TIMES] = times;
    a.counted[COUNT_SPLITS] = q.splits();
  }
  if (BACKWARD && a.xg && b + 1 == a.row_blocks) {  // the last block of k of dweight's product reads zeros behind the last row
    int last = -1;
    for (int i = 0; i < CE_ROWS; ++i) last = max(last, place[i]);
    const int n = last >= 0 ? last + 1 : base, wide = a.pitch / UNIT;
    const int end = (n + mma::BLOCK_K - 1) / mma::BLOCK_K * mma::BLOCK_K;
    for (int q = 0; q < a.parts; ++q)
      for (int64_t u = threadIdx.x; u < (int64_t)(end - n) * wide; u += CE_THREADS)
        *reinterpret_cast<uint4*>(a.xg + q * a.xg_plane + (int64_t)n * a.pitch + u * UNIT) = make_uint4(0, 0, 0, 0);
  }
}

// ---- the loss ------------------------------------------------------------------------------------------------------------
// Runs of tiles: row blocks one after another, each over all classes; a cluster takes an equal share of this list and leaves one run
// (maximum, sum) for each row block that it touches.
struct LossJob : mma::Plain {
  static constexpr int run = mma::JOIN_LONG;
  bool joins() const { return features > run * mma::BLOCK_K; }
  int cols;
  bool bfloat;
  mma::Segments seg;
  CUtensorMap x, w;
  const int* counted;
  int classes, features, rows;              // rows of a tile
  const float* bias;
  const int* at;
  float* at_z;
  float2* runs;

  struct Local { long long first, last; int wide, blocks, clusters, id; };
  __device__ __forceinline__ Local begin(const Shared&, int cluster, int clusters) const {
    Local l;
    l.id = cluster;
    l.wide = (classes + cols - 1) / cols;
    l.blocks = (*counted + rows - 1) / rows;
    const long long total = (long long)l.blocks * l.wide;
    l.clusters = (int)min((long long)clusters, total);
    l.first = cluster < l.clusters ? total * cluster / l.clusters : 0;
    l.last = cluster < l.clusters ? total * (cluster + 1) / l.clusters : 0;
    return l;
  }
  __device__ __forceinline__ bool tile(Local& l, int i, mma::Tile& t) const {
    const long long w = l.first + i;
    if (w >= l.last) return false;
    t.group = (int)(w / l.wide);
    t.a = &x;
    t.b = &this->w;
    t.row = t.a_row = t.group * rows;
    t.col = t.b_row = (int)(w - (long long)t.group * l.wide) * cols;
    t.a_plane = t.b_plane = t.a_k = t.b_k = t.a_turn = t.b_turn = 0;
    t.a_rows_first = t.b_rows_first = false;
    t.blocks = (features + mma::BLOCK_K - 1) / mma::BLOCK_K;
    return true;
  }
  // the cluster that has tile w
  __device__ __host__ static int cluster_of(long long w, long long total, int clusters) { return (int)(((w + 1) * clusters - 1) / total); }
  // most runs of a row block
  __device__ __host__ static int runs_of(int blocks, int clusters) { return (clusters + blocks - 1) / blocks + 1; }

  struct Epilogue {
    const LossJob& job;
    const Local l;
    const int row, half;
    int block, cls;
    float m, s;
    __device__ __forceinline__ Epilogue(const LossJob& j, const Local& l, int r, int h, u32) : job(j), l(l), row(r), half(h), block(-1), cls(-1) {}
    __device__ __forceinline__ void prepare(const mma::Tile&, int, mma::Control*) {}
    __device__ __forceinline__ void finish() {
      if (block < 0 || block * job.rows + row >= *job.counted) return;
      const long long total = (long long)l.blocks * l.wide;
      const int run = l.id - cluster_of((long long)block * l.wide, total, l.clusters);
      const long long at = ((long long)block * runs_of(l.blocks, l.clusters) + run) * 2 + half;
      job.runs[at * job.rows + row] = make_float2(m, s);
    }
    __device__ __forceinline__ void tile(const mma::Tile& t, const mma::Sums& sums) {
      if (t.group != block) {
        finish();
        block = t.group;
        const int r = t.row + row;
        cls = r < *job.counted ? job.at[r] : -1;
        m = __int_as_float(0xff800000);
        s = 0;
      }
      const int width = job.cols / 2;
      for (int c = half * width; c < (half + 1) * width; c += 32) {
        const int col = t.col + c;
        if (col >= job.classes) break;                      // the same for the whole warp
        float z[32];
        mma::sums_of(sums, c, z);
        if (job.bias) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 b = __ldg(reinterpret_cast<const float4*>(job.bias + col + i));
            z[i] += b.x; z[i + 1] += b.y; z[i + 2] += b.z; z[i + 3] += b.w;
          }
        } else if (col + 32 > job.classes) {
#pragma unroll
          for (int i = 0; i < 32; ++i) if (col + i >= job.classes) z[i] = __int_as_float(0xff800000);
        }
        const unsigned mine = (unsigned)(cls - col);
        if (mine < 32u) {
          float v = z[0];
#pragma unroll
          for (int i = 1; i < 32; ++i) v = mine == (unsigned)i ? z[i] : v;
          job.at_z[t.row + row] = v;
        }
        float top[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
        for (int i = 4; i < 32; ++i) top[i & 3] = fmaxf(top[i & 3], z[i]);
        const float cm = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        if (cm > m) { s *= exp2_approx((m - cm) * LOG2E); m = cm; }
        const float from = m == __int_as_float(0xff800000) ? 0.0f : m;      // subtracted first: large logits keep their differences
        float part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 32; ++i) part[i & 3] += exp2_approx((z[i] - from) * LOG2E);
        s += (part[0] + part[1]) + (part[2] + part[3]);
      }
    }
  };
};

struct JoinArgs {
  const float2* runs;
  const int *counted, *index, *at;            // index NULL: lse and rest of the gathered rows, for the gradients
  const float* at_z;
  float *loss, *lse, *rest;
  double* sums;
  unsigned* ticket;
  int rows, wide, clusters, reduction;
};

// A warp joins a row's runs; the last block adds the blocks' sums in their order.
__global__ void __launch_bounds__(CE_THREADS) k_ce_join(const __grid_constant__ JoinArgs a) {
  __shared__ double scratch[CE_THREADS / 32];
  __shared__ bool final_block;
  mma::let_next_start();
  mma::wait_for_previous();
  const int n = *a.counted, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int blocks = (n + a.rows - 1) / a.rows;
  const long long total = (long long)blocks * a.wide;
  const int clusters = (int)min((long long)a.clusters, total);
  double sum = 0;
  for (int i = blockIdx.x * CE_ROWS + warp; i < min(n, (int)(blockIdx.x + 1) * CE_ROWS); i += CE_THREADS / 32) {
    const int block = i / a.rows, row = i - block * a.rows;
    const int runs = LossJob::cluster_of((long long)(block + 1) * a.wide - 1, total, clusters) - LossJob::cluster_of((long long)block * a.wide, total, clusters) + 1;
    const long long first = (long long)block * LossJob::runs_of(blocks, clusters) * 2;
    float m = __int_as_float(0xff800000), s = 0;
    for (int k = lane; k < 2 * runs; k += 32) {
      const float2 v = a.runs[(first + k) * a.rows + row];
      const float top = fmaxf(m, v.x);
      if (top > __int_as_float(0xff800000)) s = s * exp2f((m - top) * LOG2E) + v.y * exp2f((v.x - top) * LOG2E);
      else s += v.y;
      m = top;
    }
    for (int o = 16; o; o >>= 1) {
      const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o), top = fmaxf(m, om);
      if (top > __int_as_float(0xff800000)) s = s * exp2f((m - top) * LOG2E) + os * exp2f((om - top) * LOG2E);
      else s += os;
      m = top;
    }
    if (lane == 0) {
      float rest;
      const float lse = lse_of(m, s, rest), z = a.at[i] >= 0 ? a.at_z[i] : __int_as_float(0x7fc00000);
      // log s + (m - z): the same value with one rounding less where lse is large
      const float loss = logf(s) + (m - z);
      const int to = a.index ? a.index[i] : i;
      a.lse[to] = a.index || a.at[i] >= 0 ? lse : z;
      if (a.rest) a.rest[to] = rest;
      if (a.loss && a.reduction == SAE_REDUCE_NONE) a.loss[to] = loss;
      sum += loss;
    }
  }
  if (a.reduction == SAE_REDUCE_NONE) return;
  if (lane == 0) scratch[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0;
    for (int i = 0; i < CE_THREADS / 32; ++i) sum += scratch[i];
    a.sums[blockIdx.x] = sum;
    __threadfence();
    final_block = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!final_block) return;
  __threadfence();
  sum = 0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += CE_THREADS) sum += __ldcg(a.sums + i);
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) scratch[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0;
    for (int i = 0; i < CE_THREADS / 32; ++i) sum += scratch[i];
    *a.loss = (float)(a.reduction == SAE_REDUCE_MEAN ? sum / (double)n : sum);
  }
}

// ---- the gradients --------------------------------------------------------------------------------------------------------
// p of one piece of the classes.
struct GradJob : mma::Plain {
  static constexpr int run = LossJob::run;       // (lse goes with the very z that it was made from)
  bool joins() const { return features > run * mma::BLOCK_K; }
  int cols;
  bool bfloat;
  mma::Segments seg;
  CUtensorMap x, w;
  const int* counted;
  Pieces pieces;
  int classes, features, rows, index;            // index: of the piece
  const float *bias, *lse, *rest, *g;
  const int* at;
  unsigned short* p;
  int64_t p_plane;
  int type;
  bool scaled;                                   // a row's factor may be another than 1
  float* bias_sums;                              // of every 32 rows, as p; NULL: not wanted

  struct Local { int first, step, blocks, start, tiles, pitch, count; };        // first class of the piece, tiles across it
  __device__ __forceinline__ Local begin(const Shared&, int cluster, int clusters) const {
    Local l = {cluster, clusters, 0, 0, 0, 0, *counted};
    l.blocks = (l.count + rows - 1) / rows;
    l.pitch = pieces.piece * counted[COUNT_TIMES];
    const int64_t start = (int64_t)index * l.pitch;
    l.start = (int)(start < classes ? start : classes);
    l.tiles = (min(l.pitch, classes - l.start) + cols - 1) / cols;
    return l;
  }
  __device__ __forceinline__ bool tile(Local& l, int i, mma::Tile& t) const {
    const long long n = l.first + (long long)i * l.step;
    if (n >= (long long)l.blocks * l.tiles) return false;
    const int v = (int)(n / l.blocks);
    t.row = t.a_row = (int)(n - (long long)v * l.blocks) * rows;
    t.col = v * cols;
    t.b_row = l.start + t.col;
    t.a = &x;
    t.b = &w;
    t.a_plane = t.b_plane = t.a_k = t.b_k = t.a_turn = t.b_turn = 0;
    t.a_rows_first = t.b_rows_first = false;
    t.blocks = (features + mma::BLOCK_K - 1) / mma::BLOCK_K;
    return true;
  }
  struct Epilogue {
    const GradJob& job;
    const Local& l;
    const int row, half;
    __device__ __forceinline__ Epilogue(const GradJob& j, const Local& l, int r, int h, u32) : job(j), l(l), row(r), half(h) {}
    __device__ __forceinline__ void prepare(const mma::Tile&, int, mma::Control*) {}
    __device__ __forceinline__ void finish() {}
    __device__ __forceinline__ void tile(const mma::Tile& t, const mma::Sums& sums) {
      const int r = t.row + row;
      const bool used = r < l.count;
      const float lse = used ? job.lse[r] : 0.0f, rest = used ? job.rest[r] * LOG2E : 0.0f, g = used ? job.g[r] : 0.0f;
      const int cls = used ? job.at[r] - l.start : -1;
      const int width = job.cols / 2;
      for (int c = half * width; c < (half + 1) * width; c += 32) {
        const int col = t.col + c, cc = l.start + col;
        float z[32];
        mma::sums_of(sums, c, z);
        if (job.bias) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 b = __ldg(reinterpret_cast<const float4*>(job.bias + cc + i));
            z[i] += b.x; z[i + 1] += b.y; z[i + 2] += b.z; z[i + 3] += b.w;
          }
        } else if (cc + 32 > job.classes) {
#pragma unroll
          for (int i = 0; i < 32; ++i) if (cc + i >= job.classes) z[i] = __int_as_float(0xff800000);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) z[i] = exp2_approx(log2_p(z[i], lse, rest));
        const unsigned mine = (unsigned)(cls - col);
        if (mine < 32u) {
#pragma unroll
          for (int i = 0; i < 32; ++i) z[i] = mine == (unsigned)i ? z[i] - 1.0f : z[i];
        }
        if (job.scaled) {
#pragma unroll
          for (int i = 0; i < 32; ++i) z[i] *= g;
        }
        if (!used) {                              // a row that is none stays exactly zero, whatever its sums are
#pragma unroll
          for (int i = 0; i < 32; ++i) z[i] = 0.0f;
        }
        unsigned short* const to = job.p + (int64_t)r * l.pitch + col;
        u32 w[16];
        if (job.type == SAE_TYPE_HALF) {
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = mma::pack_half(z[2 * i], z[2 * i + 1]);
          mma::store_words(to, w);
        } else if (job.type == SAE_TYPE_BFLOAT) {
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = mma::pack_bfloat(z[2 * i], z[2 * i + 1]);
          mma::store_words(to, w);
        } else {
          u32 w1[16], w2[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float a[3], b[3];
            three_parts(z[2 * i], a);
            three_parts(z[2 * i + 1], b);
            w[i] = mma::pack_bfloat(a[0], b[0]); w1[i] = mma::pack_bfloat(a[1], b[1]); w2[i] = mma::pack_bfloat(a[2], b[2]);
          }
          mma::store_words(to, w);
          mma::store_words(to + job.p_plane, w1);
          mma::store_words(to + 2 * job.p_plane, w2);
        }
        if (job.bias_sums) {                      // over the warp's 32 rows: halves are exchanged until each lane has one column
          const int lane = threadIdx.x & 31;
#pragma unroll
          for (int o = 16; o; o >>= 1)
#pragma unroll
            for (int i = 0; i < o; ++i) {
              const float keep = lane & o ? z[i + o] : z[i], give = lane & o ? z[i] : z[i + o];
              z[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
          job.bias_sums[(int64_t)((t.row + row) >> 5) * l.pitch + col + lane] = z[0];
        }
      }
    }
  };
};

// dx's sums (p w, float, added up over the pieces) and dweight of a piece (p' x): one list of tiles, the longer ones first, or either alone.
struct ProductJob : mma::Plain {
  static constexpr int STAGING = mma::SQUARE_BYTES;
  int run, longest;               // blocks of k: of a sum, most of a tile as far as the host knows
  bool joins() const { return longest > run; }
  int cols;
  bool bfloat;
  mma::Segments seg;
  CUtensorMap p[CE_WIDER], w, x;  // p: for pieces of 1, 2 .. times the classes
  const int* counted;
  Pieces pieces;
  int rows, across, features;     // rows of a tile, tiles across the features
  int classes, index;             // index: of the piece
  bool dx, dweight;
  // dx
  float* dx_sums;
  int sums_pitch;
  // dweight
  float* dw_sums;                 // of its splits, where it has more than one
  int dw_splits;
  void* out;
  int type;
  bool whole_rows;                // every row starts on 32 bytes
  const float* alpha;

  struct Local { int first, step, count, times, start, width, dx_blocks, splits, dx_tiles, dw_blocks, dw_tiles; bool dx_first; };
  __device__ __forceinline__ bool joined(const Local& l) const {
    return (dx && l.width > l.splits * (run * mma::BLOCK_K)) || (dweight && l.count > dw_splits * (run * mma::BLOCK_K));
  }
  __device__ __forceinline__ Local begin(const Shared&, int cluster, int clusters) const {
    Local l = {};
    l.first = cluster; l.step = clusters; l.count = *counted; l.splits = 1;
    l.times = counted[COUNT_TIMES];
    const int piece = pieces.piece * l.times;
    const int64_t start = (int64_t)index * piece;
    if (start >= classes) return l;
    l.start = (int)start;
    l.width = min(piece, classes - l.start);
    if (dx) l.dx_blocks = (l.count + rows - 1) / rows;
    if (dweight) l.dw_blocks = (l.width + rows - 1) / rows;
    l.dw_tiles = l.dw_blocks * across * dw_splits;
    if (dx) l.splits = counted[COUNT_SPLITS];
    l.dx_tiles = l.dx_blocks * across * l.splits;
    l.dx_first = l.width / l.splits + 500 > l.count;
    return l;
  }
  __device__ __forceinline__ bool tile(Local& l, int i, mma::Tile& t) const {
    const long long at = l.first + (long long)i * l.step;
    if (at >= (long long)l.dx_tiles + l.dw_tiles) return false;
    const bool is_dx = l.dx_first ? at < l.dx_tiles : at >= l.dw_tiles;
    const int n = (int)at - (is_dx == l.dx_first ? 0 : is_dx ? l.dw_tiles : l.dx_tiles), blocks = is_dx ? l.dx_blocks : l.dw_blocks, q = n / across;
    t.item = q / blocks;                          // the split
    t.row = t.a_row = (q - t.item * blocks) * rows;
    t.col = t.b_row = (n - q * across) * cols;
    t.a = &p[l.times - 1];
    t.b = is_dx ? &w : &x;
    t.a_plane = t.b_plane = t.a_turn = t.b_turn = 0;
    t.b_rows_first = true;
    t.a_rows_first = !is_dx;                      // (what the epilogue knows them by, too)
    const int all = ((is_dx ? l.width : l.count) + mma::BLOCK_K - 1) / mma::BLOCK_K, splits = is_dx ? l.splits : dw_splits;
    const int from = (int)((long long)all * t.item / splits), to = (int)((long long)all * (t.item + 1) / splits);
    t.a_k = from * mma::BLOCK_K;
    t.b_k = t.a_k + (is_dx ? l.start : 0);
    t.blocks = to - from;
    t.group = blocks * rows;                      // rows of a split's sums
    return true;
  }
  struct Epilogue {
    const ProductJob& job;
    const Local& l;
    const int row, half;
    const float alpha;
    const u32 staging;
    __device__ __forceinline__ Epilogue(const ProductJob& j, const Local& l, int r, int h, u32 at)
        : job(j), l(l), row(r), half(h), alpha(j.dweight && j.dw_splits == 1 ? *j.alpha : 1.0f), staging(at) {}
    __device__ __forceinline__ void prepare(const mma::Tile&, int, mma::Control*) {}
    __device__ __forceinline__ void finish() {}
    __device__ __forceinline__ void tile(const mma::Tile& t, const mma::Sums& sums) {
      const bool dx = !t.a_rows_first, apart = dx || job.dw_splits > 1, add = dx && job.index;
      const int r = t.row + row, w = job.cols / 2, limit = dx ? l.count : l.width;
      for (int c = half * w; c < (half + 1) * w; c += 32) {
        const int col = t.col + c;
        if (col >= job.features) break;
        __syncwarp();
        float v[32];
        mma::sums_of(sums, c, v);
        if (!apart && !job.whole_rows) {
          const int row0 = t.row + (row & ~31);
          if (row0 >= limit) continue;                    // the whole warp's
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] *= alpha;
          const int64_t to = (int64_t)(l.start + row0) * job.features + col;
          const int m = min(32, limit - row0), n = min(32, job.features - col);
          if (job.type == SAE_TYPE_FLOAT) mma::store_square((float*)job.out + to, job.features, v, m, n, staging);
          else if (job.type == SAE_TYPE_BFLOAT) mma::store_square((__nv_bfloat16*)job.out + to, job.features, v, m, n, staging);
          else mma::store_square((__half*)job.out + to, job.features, v, m, n, staging);
          continue;
        }
        if (r >= limit) continue;
        if (apart) {
          float* const to = (dx ? job.dx_sums : job.dw_sums) + ((int64_t)t.item * t.group + r) * job.sums_pitch + col;
          if (add) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              u32 old[16];
              mma::load_words(to + 16 * h, old);
#pragma unroll
              for (int i = 0; i < 16; ++i) v[16 * h + i] += __uint_as_float(old[i]);
            }
          }
          mma::store_row(to, v, 32);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] *= alpha;
          const int n = min(32, job.features - col);
          const int64_t to = (int64_t)(l.start + r) * job.features + col;
          if (job.type == SAE_TYPE_FLOAT) mma::store_row((float*)job.out + to, v, n);
          else if (job.type == SAE_TYPE_BFLOAT) mma::store_row((__nv_bfloat16*)job.out + to, v, n);
          else mma::store_row((__half*)job.out + to, v, n);
        }
      }
    }
  };
};

// dx = alpha * the sums over the splits, back to the rows that they belong to; dweight likewise.
struct DxArgs {
  const float* sums;
  const int *counted, *index;
  const float* alpha;
  void* dx;
  int sums_pitch, features, type, rows;
  int dw_rows, dw_splits;           // dweight: its rows and splits (0: this is dx)
};
template <typename T>
__device__ __forceinline__ void put_row(T* to, const float (&v)[UNIT], int n) {
  if (n == UNIT && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      Raw<T, 8> r;
      r.round(v);
      r.store(to);
    }
  } else {
#pragma unroll
    for (int i = 0; i < UNIT; ++i) if (i < n) to[i] = from_f<T>(v[i]);
  }
}
__global__ void __launch_bounds__(CE_THREADS) k_ce_dx(const __grid_constant__ DxArgs a) {
  mma::let_next_start();
  mma::wait_for_previous();
  const int count = a.dw_splits ? a.dw_rows : *a.counted, blocks = (count + a.rows - 1) / a.rows;
  if (!blocks) return;
  const int splits = a.dw_splits ? a.dw_splits : a.counted[COUNT_SPLITS];
  const int64_t plane = (int64_t)blocks * a.rows * a.sums_pitch;
  const float alpha = *a.alpha;
  const unsigned wide = (unsigned)(a.features + UNIT - 1) / UNIT;
  const int64_t u = (int64_t)blockIdx.x * CE_THREADS + threadIdx.x, r = u / wide;
  const int c = (int)(u - r * wide) * UNIT;
  if (r >= count) return;
  float v[UNIT] = {};
  const float* from = a.sums + r * a.sums_pitch + c;
  for (int s = 0; s < splits; ++s, from += plane) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(from)), y = __ldcg(reinterpret_cast<const float4*>(from) + 1);
    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
  }
#pragma unroll
  for (int k = 0; k < UNIT; ++k) v[k] *= alpha;
  const int n = min(UNIT, a.features - c);
  const int64_t to = (a.dw_splits ? r : (int64_t)a.index[r]) * a.features + c;
  if (a.type == SAE_TYPE_FLOAT) put_row((float*)a.dx + to, v, n);
  else if (a.type == SAE_TYPE_BFLOAT) put_row((__nv_bfloat16*)a.dx + to, v, n);
  else put_row((__half*)a.dx + to, v, n);
}

// dbias of a piece: the sums of every 32 rows, added in order (double).
__global__ void __launch_bounds__(CE_THREADS) k_ce_dbias(const float* sums, const Pieces pieces, int index, const int* counted, const float* alpha, int type, void* out) {
  __shared__ double scratch[CE_THREADS / 32][32];
  mma::let_next_start();
  mma::wait_for_previous();
  const int count = *counted, pitch = pieces.piece * counted[COUNT_TIMES], part = threadIdx.x >> 5, n = (count + 31) / 32;
  const int64_t start = (int64_t)index * pitch;
  for (int64_t block = blockIdx.x; block * 32 < pitch && start + block * 32 < pieces.classes; block += gridDim.x) {
    const int j = (int)block * 32 + (threadIdx.x & 31);
    const int64_t to = start + j;
    double s = 0;
    if (to < pieces.classes) for (int i = part; i < n; i += CE_THREADS / 32) s += __ldcg(sums + (int64_t)i * pitch + j);
    __syncthreads();
    scratch[part][threadIdx.x & 31] = s;
    __syncthreads();
    if (part || to >= pieces.classes) continue;
    for (int i = 1; i < CE_THREADS / 32; ++i) s += scratch[i][threadIdx.x & 31];
    const float v = (float)(s * *alpha);
    if (type == SAE_TYPE_FLOAT) ((float*)out)[to] = v;
    else if (type == SAE_TYPE_BFLOAT) ((__nv_bfloat16*)out)[to] = __float2bfloat16_rn(v);
    else ((__half*)out)[to] = __float2half_rn(v);
  }
}

}  // namespace

#include "sae_ce_float.cuh"

namespace {

// ---- host ---------------------------------------------------------------------------------------------------------------------
bool type_ok(int t) { return t == SAE_TYPE_FLOAT || t == SAE_TYPE_BFLOAT || t == SAE_TYPE_HALF; }

bool desc_ok(const sae_linear_ce_desc* d) {
  return d && type_ok(d->type) && (!d->has_bias || type_ok(d->bias_type)) && d->reduction >= SAE_REDUCE_NONE && d->reduction <= SAE_REDUCE_MEAN &&
         d->rows >= 0 && d->rows <= (1 << 24) && d->features >= 1 && d->features <= (1 << 17) && d->classes >= 1 && d->classes <= (1 << 24) &&
         (d->rows < 2 || d->x_pitch >= d->features) && (d->classes < 2 || d->weight_pitch >= d->features);
}

int device_sms() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return -1; }
  return sms;
}

// Float tensors of up to CE_FLOAT_ROWS rows take float arithmetic where that is faster than bfloat16 parts, by these fits (us).  Float: whole blocks of
// 32 rows, and a logit's way through memory.  Parts: w is read, laid out and read again; long sums of six products in few tiles.  Loss and gradients, there
// and in parts: 32 x 2048 x 1000 58 and 165, 128 x 2048 x 1000 121 and 166, 256 x 2048 x 1000 198 and 169; 8 x 768 x 30522 203 and 322, 32 rows 285 and 338,
// 64 rows 478 and 341; 17 x 1152 x 39231 460 and 572; 320 x 64 x 20000 259 and 147, 300 x 64 x 1000 43 and 53.
constexpr int64_t CE_FLOAT_ROWS = 320;
bool in_float(const sae_linear_ce_desc* d) {
  if (d->type != SAE_TYPE_FLOAT || d->rows > CE_FLOAT_ROWS || d->classes > (1 << 20)) return false;
  const double n = (double)d->rows, v = (double)d->classes, k = (double)d->features;
  return 35 + 2.6e-7 * (double)up(std::max<int64_t>(1, d->rows), 32) * v * k + 1.9e-5 * n * v < 40 + 7e-6 * v * k + 3e-3 * v + 4.5e-2 * k;
}
// Splits of k, from what does not depend on the rows, so that a row's result does not either: four blocks an SM for a single block of
// rows, and no split of less than 64 k (least k unknown: 0).
int float_splits(int64_t tiles, int64_t depth, int most, int sms) {
  int64_t s = std::min<int64_t>(4ll * sms / tiles, most);
  if (depth) s = std::min<int64_t>(s, depth / 64);
  return (int)std::max<int64_t>(1, s);
}

// Whether the loss of a float head takes one launch in place of three.  A block has all k of its rows there, at 1.06 us for 32: 128 x 64 x 10 6.4 us
// (11.6 with three), 256 x 512 x 64 21.7 (12.8); they meet at 7 blocks of k.
bool in_one_launch(const sae_linear_ce_desc* d) { return d->rows && d->rows <= 8 * CF_ROWS && d->classes <= CF_COLS && d->features <= 6 * CF_K; }

struct TileShape { int cg, cols; };

// The tile shape of a product of `depth` k: waves of tiles over the SMs (or pairs) times what a tile costs for each k.  A block of 64 k takes a pair
// 588 cycles for 256 x 256, one SM 630 for 128 x 128 (shared memory: the tensor cores read and TMA writes 64 KB in it) and about 500
// for 128 x 64.  splits: where sums may be added up in several parts of k, at 500 k for each, the best number of them counts.
struct CostedShape { TileShape s; double cost; };
CostedShape costed_shape(int i, int parts) {
  const CostedShape shapes[3] = {{{2, parts == 1 ? 256 : 128}, parts == 1 ? 2.0 : 1.6}, {{1, 128}, 2.1}, {{1, 64}, 1.7}};
  return shapes[i];
}
TileShape tile_shape(int64_t rows, int64_t cols, int64_t depth, int splits, int parts, int sms, double* time = nullptr) {
  TileShape best = {};
  double least = 0;
  for (int i = 0; i < 3; ++i) {
    const CostedShape c = costed_shape(i, parts);
    const int64_t tiles = (rows + 128 * c.s.cg - 1) / (128 * c.s.cg) * ((cols + c.s.cols - 1) / c.s.cols), units = sms / c.s.cg;
    for (int s = 1; s <= splits; ++s) {
      const double t = c.cost * (double)((tiles * s + units - 1) / units) * ((double)depth / s + (splits > 1 ? 500.0 : 0.0));
      if (least == 0 || t < least) { least = t; best = c.s; }
    }
  }
  if (time) *time = least;
  return best;
}
// Row blocks that dx's sums have place for: four splits where there are few of them.
int sums_room(int64_t blocks, int64_t across, int64_t clusters) { return (int)(blocks + 4 * clusters / across); }
// One shape for dx and dweight in one list, where that takes no longer than two launches with a shape for each.
bool shape_of_both(int64_t rows, int64_t features, int64_t classes, int64_t piece, int parts, int sms, double apart, TileShape* to) {
  double least = apart;
  bool found = false;
  for (int i = 0; i < 3; ++i) {
    const CostedShape c = costed_shape(i, parts);
    const int64_t across = (features + c.s.cols - 1) / c.s.cols, down = 128 * c.s.cg;
    const int64_t blocks = (rows + down - 1) / down;
    const Product q = {(int)blocks, (int)across, sms / c.s.cg, (int)piece, sums_room(blocks, across, sms / c.s.cg), (int)((std::min(piece, classes) + down - 1) / down * across), (int)rows};
    const double t = c.cost * q.time(q.splits());
    if (t <= least) { least = t; *to = c.s; found = true; }
  }
  return found;
}

struct CePlan {
  int parts, pitch;
  int64_t rows;                      // room for gathered rows
  bool copy_w;
  TileShape z, dx, dw;
  Pieces pieces;
  bool both;                         // dx and dweight in one list
  int sums_pitch, dx_room;
  size_t dw_sums;
  // offsets
  // in float arithmetic (dw_splits: in the other too)
  bool in_float;
  int z_splits, dx_splits, dw_splits, z_pitch, dx_pitch, dw_pitch;
  size_t fz, fdx, fdw;
  size_t xg, wg, bias, index, at, at_z, counted, before, runs, sums, lse_g, rest_g, g, alpha, top, p, bias_sums, dx_sums, bytes;
};

// Classes of a piece, in blocks of 256: as many as the bytes allow, or fewer where the tiles of its products then come out as
// whole waves.  Time in units of a tile's k: waves of p, the list of dx and dweight, and what two more launches cost.
// 8192 rows of 768, 30522 classes: 24 blocks at a time instead of 60, 72 tiles of dweight on 74 pairs instead of 180.
int piece_blocks(const sae_linear_ce_desc* d, int64_t rows, int parts, int sms) {
  const int64_t all = (d->classes + 255) / 256, most = std::max<int64_t>(1, std::min(all, CE_PIECE_BYTES / (rows * 2 * parts) / 256));
  const int64_t units = sms / 2, down = (d->rows + 255) / 256, across = (d->features + 255) / 256;
  const auto waves = [&](int64_t tiles) { return (double)((tiles + units - 1) / units); };
  int64_t best = most;
  double least = 0;
  for (int64_t b = most; b >= std::max<int64_t>(1, most / 4); --b) {
    const Product q = {(int)down, (int)across, (int)units, (int)(256 * b), sums_room(down, across, units), (int)(b * across), (int)d->rows};
    const double pieces = (double)((all + b - 1) / b);
    const double t = pieces * (parts * (waves(down * b) * (double)d->features + q.time(q.splits())) + 1700.0);
    if (least == 0 || t < 0.99 * least) { least = t; best = b; }
  }
  return (int)best;
}

CePlan make_plan(const sae_linear_ce_desc* d, const void* weight, bool backward, int sms) {
  CePlan p = {};
  p.parts = d->type == SAE_TYPE_FLOAT ? 3 : 1;
  p.pitch = (int)up(d->features, 8);
  p.rows = up(std::max<int64_t>(1, d->rows), 256);
  // (one row of weights has no pitch of its own: any that TMA takes will do)
  p.copy_w = p.parts > 1 || !aligned_to(weight, 16) || (d->classes > 1 && d->weight_pitch % 8);
  p.in_float = in_float(d);
  if (p.in_float) p.parts = 1;
  size_t at = 0;
  const auto take = [&](int64_t bytes) { const size_t o = at; at += (size_t)up(std::max<int64_t>(bytes, 1), 256); return o; };
  if (p.in_float) {
    const int64_t n = std::max<int64_t>(1, d->rows);
    p.index = take(n * 4);
    p.at = take(n * 4);
    p.counted = take(COUNT_WORDS * 4);
    p.before = take(d->rows > CE_SCAN_ROWS ? up(d->rows, CE_COUNT_ROWS) / CE_COUNT_ROWS * 4 : 0);
    p.z_pitch = (int)up(d->classes, 4);
    // (not split where the loss was made in one launch: the gradients take the very z that lse was made from)
    p.z_splits = in_one_launch(d) ? 1 : float_splits((d->classes + CF_COLS - 1) / CF_COLS, d->features, 8, sms);
    p.fz = take((int64_t)p.z_splits * n * p.z_pitch * 4);
    p.at_z = take(n * 4);
    p.sums = take(n * ((d->classes + CF_LOSS_CLASSES - 1) / CF_LOSS_CLASSES) * 8);
    if (backward) {
      p.lse_g = take(n * 4);
      p.rest_g = take(n * 4);
      p.g = take(n * 4);
      p.alpha = take(4);
      p.p = take(n * p.z_pitch * 4);
      p.dx_pitch = (int)up(d->features, 4);
      p.dx_splits = float_splits((d->features + CF_COLS - 1) / CF_COLS, d->classes, 32, sms);
      p.fdx = take((int64_t)p.dx_splits * n * p.dx_pitch * 4);
      p.dw_pitch = (int)up(d->features + 1, 4);
      p.dw_splits = float_splits((d->classes + CF_ROWS - 1) / CF_ROWS * ((d->features + CF_COLS) / CF_COLS), 0, 32, sms);
      p.fdw = take(p.dw_splits > 1 ? (int64_t)p.dw_splits * d->classes * p.dw_pitch * 4 : 0);
    }
    p.bytes = at;
    return p;
  }
  p.xg = take((int64_t)p.parts * p.rows * p.pitch * 2);
  p.wg = take(p.copy_w ? (int64_t)p.parts * d->classes * p.pitch * 2 : 0);
  p.bias = take(d->has_bias ? up(d->classes, 256) * 4 + 1024 : 0);
  p.index = take(p.rows * 4);
  p.at = take(p.rows * 4);
  p.counted = take(COUNT_WORDS * 4);
  p.before = take(d->rows > CE_SCAN_ROWS ? up(d->rows, CE_COUNT_ROWS) / CE_COUNT_ROWS * 4 : 0);
  p.z = tile_shape(d->rows, d->classes, d->features, 1, p.parts, sms);
  const int z_rows = 128 * p.z.cg, z_clusters = sms / p.z.cg;
  const int64_t z_blocks = up(p.rows, z_rows) / z_rows;
  p.at_z = take(p.rows * 4);
  p.runs = take((z_clusters + 2 * z_blocks + 2) * 2 * z_rows * (int64_t)sizeof(float2));
  p.sums = take(up(p.rows, CE_ROWS) / CE_ROWS * 8);
  if (backward) {
    p.lse_g = take(p.rows * 4);
    p.rest_g = take(p.rows * 4);
    p.g = take(p.rows * 4);
    p.alpha = take(4);
    p.top = take(4);
    const int piece = 256 * piece_blocks(d, p.rows, p.parts, sms);
    double dx_time = 0, dw_time = 0;
    p.dx = tile_shape(d->rows, d->features, piece, 8, p.parts, sms, &dx_time);
    p.dw = tile_shape(std::min<int64_t>(piece, d->classes), d->features, d->rows, 1, p.parts, sms, &dw_time);
    // A head of few classes has a tile or two of dweight, and all rows to add up in it (16384 x 64 x 10 float: 470 us on one SM).  In two
    // launches more where that leaves half of the SMs idle; no split of less than 512 rows.
    const int64_t dw_tiles = up(piece, 128 * p.dw.cg) / (128 * p.dw.cg) * (up(d->features, p.dw.cols) / p.dw.cols);
    p.dw_splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(sms / p.dw.cg / dw_tiles, d->rows / 512), 32));
    TileShape one;
    p.both = p.dw_splits == 1 && shape_of_both(d->rows, d->features, d->classes, piece, p.parts, sms, dx_time + dw_time + 800.0, &one);
    if (p.both) p.dx = p.dw = one;
    p.pieces = {piece, (int)((d->classes + piece - 1) / piece), (int)d->classes, 1, p.rows};
    if (p.dw_splits == 1) p.pieces.most = std::min(CE_WIDER, p.pieces.number);
    p.sums_pitch = (int)up(d->features, 32);
    const int rows = 128 * p.dx.cg, across = (int)up(d->features, p.dx.cols) / p.dx.cols, clusters = sms / p.dx.cg;
    p.dx_room = sums_room(up(p.rows, rows) / rows, across, clusters);
    p.p = take((int64_t)p.parts * p.rows * piece * 2);
    p.bias_sums = take(d->has_bias ? p.rows / 32 * piece * 4 : 0);
    p.dx_sums = take((int64_t)p.dx_room * rows * p.sums_pitch * 4);
    p.dw_sums = take(p.dw_splits > 1 ? (int64_t)p.dw_splits * up(piece, 128 * p.dw.cg) * p.sums_pitch * 4 : 0);
  }
  p.bytes = at;
  return p;
}

template <typename... P, typename... A>
int launch_shared(void (*kernel)(P...), dim3 grid, int threads, size_t shared, cudaStream_t st, bool first, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = first ? 0 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
  return SAE_OK;
}
template <typename... P, typename... A>
int launch(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t st, bool first, A... args) {
  return launch_shared(kernel, grid, threads, 0, st, first, args...);
}

template <class Job>
int products(const Job& job, const TileShape& s, int64_t tiles, int sms, cudaStream_t st) {
  const int units = (int)std::min<int64_t>(std::max<int64_t>(1, tiles), sms / s.cg);
  const cudaError_t e = mma::launch_products(job, s.cg, units, st);
  if (e != cudaSuccess) cudaGetLastError();
  return e == cudaSuccess ? SAE_OK : SAE_ERR_CUDA;
}

mma::Segments segments(int parts) {
  mma::Segments one = {1, {0}, {0}}, three = {6, {0, 2, 1, 0, 1, 0}, {2, 0, 1, 1, 0, 0}};
  return parts == 1 ? one : three;
}

RowsArgs rows_args(const sae_linear_ce_desc* d, const CePlan& p, const void* x, const void* w, const void* bias, const int64_t* target, char* ws, int sms) {
  RowsArgs a = {};
  a.x = x; a.target = target; a.x_pitch = d->x_pitch; a.rows = d->rows; a.ignore = d->ignore_index;
  a.type = d->type; a.parts = p.parts; a.features = (int)d->features; a.classes = (int)d->classes; a.pitch = p.pitch;
  a.xg = p.in_float ? nullptr : (unsigned short*)(ws + p.xg);      // (float arithmetic reads rows where they are)
  a.xg_plane = p.rows * p.pitch;
  a.index = (int*)(ws + p.index); a.at = (int*)(ws + p.at); a.counted = (int*)(ws + p.counted);
  a.w = w; a.w_pitch = d->weight_pitch; a.wg = (unsigned short*)(ws + p.wg); a.wg_plane = d->classes * p.pitch;
  a.bias = bias; a.bias_type = d->bias_type; a.bias_out = (float*)(ws + p.bias);
  a.bias_room = d->has_bias && !p.in_float ? (int)up(d->classes, 256) : 0;
  a.row_blocks = (int)std::max<int64_t>(1, up(d->rows, CE_ROWS) / CE_ROWS);
  a.w_blocks = p.copy_w && !p.in_float ? (int)(up(d->classes * (p.pitch / UNIT), CE_CHUNK) / CE_CHUNK) : 0;
  a.reduction = d->reduction;
  if (!p.in_float && p.pieces.number) {            // backwards
    a.pieces = p.pieces;
    a.product_rows = 128 * p.dx.cg;
    a.product.across = (int)(up(d->features, p.dx.cols) / p.dx.cols); a.product.clusters = sms / p.dx.cg; a.product.room = p.dx_room;
    a.both = p.both;
  }
  return a;
}

// Gathers rows and whatever else must be laid out; its first launch is the call's first.
template <bool BACKWARD>
int gather(const sae_linear_ce_desc* d, const CePlan& p, RowsArgs& a, char* ws, cudaStream_t st) {
  bool first = true;
  int rc = SAE_OK;
  if (d->rows > CE_SCAN_ROWS) {
    rc = launch(k_ce_count, up(d->rows, CE_COUNT_ROWS) / CE_COUNT_ROWS, CE_THREADS, st, true, a, (int*)(ws + p.before));
    a.before = (const int*)(ws + p.before);
    first = false;
  }
  if (rc == SAE_OK && BACKWARD && d->type == SAE_TYPE_HALF && d->reduction == SAE_REDUCE_NONE) {
    rc = launch(k_ce_top, 1, 1024, st, first, a, (float*)(ws + p.top));
    a.g_top = (const float*)(ws + p.top);
    first = false;
  }
  if (rc == SAE_OK) rc = launch(k_ce_rows<BACKWARD>, a.row_blocks + a.w_blocks + (a.bias_room + CE_THREADS - 1) / CE_THREADS, CE_THREADS, st, first, a);
  return rc;
}

bool maps(const sae_linear_ce_desc* d, const CePlan& p, const void* weight, char* ws, CUtensorMap* x, CUtensorMap* w) {
  const bool bfloat = d->type != SAE_TYPE_HALF;
  return mma::encode_map(x, ws + p.xg, bfloat, d->features, p.rows, p.parts, p.pitch, p.rows * p.pitch) &&
         (p.copy_w ? mma::encode_map(w, ws + p.wg, bfloat, d->features, d->classes, p.parts, p.pitch, d->classes * p.pitch)
                   : mma::encode_map(w, weight, bfloat, d->features, d->classes, 1, d->classes > 1 ? d->weight_pitch : p.pitch, p.pitch));
}

// More shared memory than a kernel has unasked, once for each device (`ready`: a bit for each that has been asked).
bool allow_shared(const void* kernel, int bytes, std::atomic<unsigned long long>& ready) {
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); return false; }
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  if (ready.load(std::memory_order_acquire) & bit) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) { cudaGetLastError(); return false; }
  ready.fetch_or(bit, std::memory_order_release);
  return true;
}

template <FloatProduct KIND>
int float_product(FloatArgs a, int64_t rows, int64_t cols, int splits, float* out, int64_t room, int pitch, cudaStream_t st) {
  a.splits = splits; a.out = out; a.room = room; a.out_pitch = pitch;
  const dim3 grid((unsigned)((cols + CF_COLS - 1) / CF_COLS), (unsigned)((rows + CF_ROWS - 1) / CF_ROWS), (unsigned)splits);
  static std::atomic<unsigned long long> ready{0};
  if (!allow_shared((const void*)k_cf_product<KIND>, FloatTile<KIND>::BYTES, ready)) return SAE_ERR_CUDA;
  return launch_shared(k_cf_product<KIND>, grid, CF_THREADS, FloatTile<KIND>::BYTES, st, false, a);
}

FloatArgs float_args(const sae_linear_ce_desc* d, const CePlan& p, const RowsArgs& a, char* ws) {
  FloatArgs f = {};
  f.x = (const float*)a.x; f.w = (const float*)a.w; f.p = (const float*)(ws + p.p);
  f.index = a.index; f.counted = a.counted;
  f.x_pitch = d->x_pitch; f.w_pitch = d->weight_pitch;
  f.p_pitch = p.z_pitch; f.features = a.features; f.classes = a.classes;
  f.x_vector = aligned_to(a.x, 16) && (d->rows < 2 || d->x_pitch % 4 == 0);
  f.w_vector = aligned_to(a.w, 16) && (d->classes < 2 || d->weight_pitch % 4 == 0);
  f.alpha = a.alpha;
  f.any = a.counted;
  return f;
}
FloatRowArgs float_rows(const sae_linear_ce_desc* d, const CePlan& p, const RowsArgs& a, char* ws) {
  FloatRowArgs r = {};
  r.z = (const float*)(ws + p.fz); r.bias = a.bias; r.index = a.index; r.at = a.at; r.counted = a.counted;
  r.room = std::max<int64_t>(1, d->rows); r.splits = p.z_splits; r.pitch = p.z_pitch; r.classes = a.classes; r.bias_type = a.bias_type; r.reduction = d->reduction;
  r.runs = (float2*)(ws + p.sums); r.at_z = (float*)(ws + p.at_z); r.ticket = (unsigned*)a.counted + COUNT_TICKET;
  return r;
}

int float_sums(const sae_linear_ce_desc* d, const FloatRowArgs& r, cudaStream_t st) {
  return launch(k_cf_loss, dim3((unsigned)std::max<int64_t>(1, d->rows), (unsigned)((d->classes + CF_LOSS_CLASSES - 1) / CF_LOSS_CLASSES)), CF_LOSS_THREADS, st, false, r);
}

int float_forward(const sae_linear_ce_desc* d, const CePlan& p, RowsArgs& a, float* loss, char* ws, cudaStream_t st) {
  if (in_one_launch(d)) {
    TinyArgs t = {};
    t.f = float_args(d, p, a, ws);
    t.target = a.target; t.ignore = a.ignore; t.count = a.count; t.bias = a.bias; t.bias_type = d->bias_type; t.loss = loss; t.lse = a.lse; t.rest = a.rest; t.rows = (int)d->rows;
    t.reduction = d->reduction;
    static std::atomic<unsigned long long> ready{0};
    if (!allow_shared((const void*)k_cf_tiny, FloatTile<CF_Z>::BYTES, ready)) return SAE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((d->rows + CF_ROWS - 1) / CF_ROWS));
    cfg.blockDim = dim3(CF_THREADS);
    cfg.dynamicSmemBytes = FloatTile<CF_Z>::BYTES;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cfg.gridDim.x; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, k_cf_tiny, t) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
    return SAE_OK;
  }
  int rc = gather<false>(d, p, a, ws, st);
  if (rc == SAE_OK && d->rows) rc = float_product<CF_Z>(float_args(d, p, a, ws), d->rows, d->classes, p.z_splits, (float*)(ws + p.fz), d->rows, p.z_pitch, st);
  FloatRowArgs r = float_rows(d, p, a, ws);
  r.loss = loss; r.lse = a.lse; r.rest = a.rest;
  return rc == SAE_OK ? float_sums(d, r, st) : rc;
}

int float_backward(const sae_linear_ce_desc* d, const CePlan& p, RowsArgs& a, void* dx, void* dweight, void* dbias, char* ws, cudaStream_t st) {
  int rc = gather<true>(d, p, a, ws, st);
  FloatArgs f = float_args(d, p, a, ws);
  if (rc == SAE_OK && d->rows) rc = float_product<CF_Z>(f, d->rows, d->classes, p.z_splits, (float*)(ws + p.fz), d->rows, p.z_pitch, st);
  FloatRowArgs r = float_rows(d, p, a, ws);
  r.lse_g = a.lse_g; r.rest_g = a.rest_g; r.g = a.g; r.p = (float*)(ws + p.p);
  if (rc == SAE_OK && d->rows && !a.rest_in) {     // z is there: its sums once more
    FloatRowArgs again = r;
    again.index = nullptr; again.lse = a.lse_g; again.rest = a.rest_g; again.reduction = SAE_REDUCE_NONE;
    rc = float_sums(d, again, st);
  }
  if (rc == SAE_OK && d->rows) rc = launch(k_cf_p, dim3((unsigned)((d->classes + CF_THREADS - 1) / CF_THREADS), (unsigned)d->rows), CF_THREADS, st, false, r);
  FloatSumArgs s = {};
  s.counted = a.counted; s.alpha = a.alpha; s.features = a.features; s.bias_type = d->bias_type;
  if (dx && d->rows) {
    if (rc == SAE_OK) rc = float_product<CF_DX>(f, d->rows, d->features, p.dx_splits, (float*)(ws + p.fdx), d->rows, p.dx_pitch, st);
    s.sums = (const float*)(ws + p.fdx); s.index = a.index; s.out = (float*)dx; s.room = d->rows; s.splits = p.dx_splits; s.pitch = p.dx_pitch; s.rows = -1;
    if (rc == SAE_OK) rc = launch(k_cf_sum, dim3((unsigned)(d->features / 32 + 1), (unsigned)d->rows), CF_THREADS, st, false, s);
  }
  if (dweight || dbias) {
    f.dweight = (float*)dweight; f.dw_vector = dweight && aligned_to(dweight, 16) && d->features % 4 == 0; f.dbias = dbias; f.bias_type = d->bias_type;
    if (rc == SAE_OK) rc = float_product<CF_DW>(f, d->classes, d->features + (dbias ? 1 : 0), p.dw_splits, (float*)(ws + p.fdw), d->classes, p.dw_pitch, st);
    if (p.dw_splits > 1) {
      // (only few classes are split: far fewer than a grid has rows)
      s.sums = (const float*)(ws + p.fdw); s.index = nullptr; s.out = (float*)dweight; s.dbias = dbias; s.room = d->classes; s.splits = p.dw_splits; s.pitch = p.dw_pitch;
      s.rows = (int)d->classes;
      if (rc == SAE_OK) rc = launch(k_cf_sum, dim3((unsigned)(d->features / 32 + 1), (unsigned)d->classes), CF_THREADS, st, false, s);
    }
  }
  return rc;
}

// The rows' sums of exponentials, from gathered rows: loss, lse and the rest of it; without a loss, lse and rest of the gathered rows.
int sums_of_rows(const sae_linear_ce_desc* d, const CePlan& p, const RowsArgs& a, const CUtensorMap& x, const CUtensorMap& w, float* loss, float* lse, float* rest, char* ws, int sms, cudaStream_t st) {
  LossJob job = {};
  job.x = x; job.w = w;
  job.cols = p.z.cols; job.bfloat = d->type != SAE_TYPE_HALF; job.seg = segments(p.parts);
  job.counted = a.counted; job.classes = a.classes; job.features = a.features; job.rows = 128 * p.z.cg;
  job.bias = d->has_bias ? a.bias_out : nullptr; job.at = a.at; job.at_z = (float*)(ws + p.at_z); job.runs = (float2*)(ws + p.runs);
  const int64_t wide = up(d->classes, p.z.cols) / p.z.cols, tiles = up(d->rows, job.rows) / job.rows * wide;
  const int rc = tiles ? products(job, p.z, tiles, sms, st) : SAE_OK;
  if (rc != SAE_OK) return rc;
  JoinArgs j = {};
  j.runs = job.runs; j.counted = a.counted; j.index = loss ? a.index : nullptr; j.at = a.at; j.at_z = job.at_z; j.loss = loss; j.lse = lse; j.rest = rest; j.sums = (double*)(ws + p.sums);
  j.ticket = (unsigned*)a.counted + COUNT_TICKET; j.rows = job.rows; j.wide = (int)wide; j.reduction = loss ? d->reduction : SAE_REDUCE_NONE;
  j.clusters = (int)std::min<int64_t>(std::max<int64_t>(1, tiles), sms / p.z.cg);
  return launch(k_ce_join, std::max<int64_t>(1, up(d->rows, CE_ROWS) / CE_ROWS), CE_THREADS, st, false, j);
}

}  // namespace

extern "C" {

int64_t sae_linear_ce_workspace(const sae_linear_ce_desc* d, const void* weight, int32_t backward) {
  if (!desc_ok(d)) return -1;
  const int sms = device_sms();
  return sms < 2 ? -1 : (int64_t)make_plan(d, weight, backward != 0, sms).bytes;
}

int sae_linear_ce_forward_with_rest(const sae_linear_ce_desc* d, const void* x, const void* weight, const void* bias, const int64_t* target, float* loss,
                                    float* lse, float* rest, int64_t* count, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc_ok(d) || !weight || !count || (d->rows && (!x || !target || !lse)) || (!loss && (d->rows || d->reduction != SAE_REDUCE_NONE)) || (d->has_bias && !bias) || !workspace) return SAE_ERR_INVALID_ARG;
  const int es = elem_bytes(d->type);
  if (!aligned_to(x, es) || !aligned_to(weight, es) || !aligned_to(bias, d->has_bias ? elem_bytes(d->bias_type) : 1) || !aligned_to(target, 8) || !aligned_to(loss, 4) ||
      !aligned_to(lse, 4) || !aligned_to(rest, 4) || !aligned_to(count, 8) || !aligned_to(workspace, 256)) return SAE_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms < 2) return SAE_ERR_CUDA;
  const CePlan p = make_plan(d, weight, false, sms);
  if (workspace_bytes < p.bytes) return SAE_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  char* ws = (char*)workspace;
  RowsArgs a = rows_args(d, p, x, weight, d->has_bias ? bias : nullptr, target, ws, sms);
  a.count = count; a.lse = lse; a.rest = rest; a.loss = d->reduction == SAE_REDUCE_NONE ? loss : nullptr;
  if (p.in_float) return float_forward(d, p, a, loss, ws, st);
  CUtensorMap xm, wm;
  if (!maps(d, p, weight, ws, &xm, &wm)) return SAE_ERR_CUDA;
  const int rc = gather<false>(d, p, a, ws, st);
  return rc == SAE_OK ? sums_of_rows(d, p, a, xm, wm, loss, lse, rest, ws, sms, st) : rc;
}

int sae_linear_ce_forward(const sae_linear_ce_desc* d, const void* x, const void* weight, const void* bias, const int64_t* target, float* loss,
                          float* lse, int64_t* count, void* workspace, size_t workspace_bytes, void* stream) {
  return sae_linear_ce_forward_with_rest(d, x, weight, bias, target, loss, lse, nullptr, count, workspace, workspace_bytes, stream);
}

int sae_linear_ce_backward(const sae_linear_ce_desc* d, const float* dloss, const void* x, const void* weight, const void* bias, const int64_t* target,
                           const float* lse, const int64_t* count, void* dx, void* dweight, void* dbias, void* workspace, size_t workspace_bytes,
                           void* stream) {
  return sae_linear_ce_backward_with_rest(d, dloss, x, weight, bias, target, lse, nullptr, count, dx, dweight, dbias, workspace, workspace_bytes, stream);
}

int sae_linear_ce_backward_with_rest(const sae_linear_ce_desc* d, const float* dloss, const void* x, const void* weight, const void* bias, const int64_t* target,
                                     const float* lse, const float* rest, const int64_t* count, void* dx, void* dweight, void* dbias, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  if (!desc_ok(d) || !weight || !count || (d->rows && (!x || !target || !lse)) || (!dloss && (d->rows || d->reduction != SAE_REDUCE_NONE)) || (d->has_bias && !bias) || (dbias && !d->has_bias) ||
      !workspace) return SAE_ERR_INVALID_ARG;
  const int es = elem_bytes(d->type), bs = d->has_bias ? elem_bytes(d->bias_type) : 1;
  if (!aligned_to(x, es) || !aligned_to(weight, es) || !aligned_to(bias, bs) || !aligned_to(target, 8) || !aligned_to(dloss, 4) || !aligned_to(lse, 4) ||
      !aligned_to(rest, 4) || !aligned_to(count, 8) || !aligned_to(dx, es) || !aligned_to(dweight, es) || !aligned_to(dbias, bs) || !aligned_to(workspace, 256)) return SAE_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms < 2) return SAE_ERR_CUDA;
  const CePlan p = make_plan(d, weight, true, sms);
  if (workspace_bytes < p.bytes) return SAE_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (!dx && !dweight && !dbias) return SAE_OK;
  char* ws = (char*)workspace;
  RowsArgs a = rows_args(d, p, x, weight, d->has_bias ? bias : nullptr, target, ws, sms);
  a.lse_in = lse; a.rest_in = rest; a.dloss = dloss; a.count_in = count; a.dx = dx;
  a.lse_g = (float*)(ws + p.lse_g); a.rest_g = (float*)(ws + p.rest_g); a.g = (float*)(ws + p.g); a.alpha = (float*)(ws + p.alpha);
  a.p_scale = d->type == SAE_TYPE_HALF ? 32768.0f : 1.0f;
  if (p.in_float) return float_backward(d, p, a, dx, dweight, dbias, ws, st);
  GradJob g = {};
  if (!maps(d, p, weight, ws, &g.x, &g.w)) return SAE_ERR_CUDA;
  const bool bfloat = d->type != SAE_TYPE_HALF;
  ProductJob job = {};
  for (int i = 0; i < p.pieces.most; ++i)
    if (!mma::encode_map(&job.p[i], ws + p.p, bfloat, (int64_t)p.pieces.piece * (i + 1), p.rows / (i + 1), p.parts, (int64_t)p.pieces.piece * (i + 1), p.rows * p.pieces.piece))
      return SAE_ERR_CUDA;
  int rc = gather<true>(d, p, a, ws, st);
  if (rc == SAE_OK && !rest && d->rows) rc = sums_of_rows(d, p, a, g.x, g.w, nullptr, a.lse_g, a.rest_g, ws, sms, st);
  g.cols = p.z.cols; g.bfloat = bfloat; g.seg = segments(p.parts);
  g.counted = a.counted; g.classes = a.classes; g.features = a.features; g.rows = 128 * p.z.cg;
  g.bias = d->has_bias ? a.bias_out : nullptr; g.lse = a.lse_g; g.rest = a.rest_g; g.g = a.g; g.at = a.at;
  g.p = (unsigned short*)(ws + p.p); g.p_plane = p.rows * p.pieces.piece; g.type = d->type; g.pieces = p.pieces;
  g.scaled = d->reduction == SAE_REDUCE_NONE || a.p_scale != 1.0f;
  g.bias_sums = dbias ? (float*)(ws + p.bias_sums) : nullptr;
  job.run = bfloat ? mma::JOIN_BFLOAT : mma::JOIN_HALF;
  job.bfloat = bfloat; job.seg = g.seg; job.w = g.w; job.x = g.x; job.counted = a.counted; job.pieces = p.pieces; job.features = a.features; job.classes = a.classes;
  job.dx_sums = (float*)(ws + p.dx_sums); job.dw_sums = (float*)(ws + p.dw_sums); job.sums_pitch = p.sums_pitch; job.dw_splits = p.dw_splits;
  job.out = dweight; job.type = d->type; job.alpha = a.alpha; job.whole_rows = aligned_to(dweight, 32) && d->features * es % 32 == 0;
  const auto across = [&](const TileShape& s) { return (int)(up(d->features, s.cols) / s.cols); };
  // (launches are sized for all rows and for pieces of any width)
  const auto product = [&](const TileShape& s, bool for_x, bool for_weight) {
    job.cols = s.cols; job.rows = 128 * s.cg; job.across = across(s); job.dx = for_x; job.dweight = for_weight;
    const int64_t classes = std::min<int64_t>((int64_t)p.pieces.piece * p.pieces.most, d->classes);
    job.longest = (int)(std::max(for_x ? classes : 0, for_weight ? d->rows / p.dw_splits : 0) / mma::BLOCK_K) + 1;
    return products(job, s, for_x ? sms : up(classes, job.rows) / job.rows * job.across * p.dw_splits, sms, st);
  };
  const bool want_x = dx && d->rows, both = p.both && want_x && dweight;
  for (int i = 0; i < p.pieces.number && rc == SAE_OK; ++i) {
    g.index = job.index = i;
    const int64_t z_tiles = up(d->rows, g.rows) / g.rows * (up(std::min<int64_t>((int64_t)p.pieces.piece * p.pieces.most, d->classes), g.cols) / g.cols);
    if (z_tiles) rc = products(g, p.z, z_tiles, sms, st);
    if (dbias && rc == SAE_OK)
      rc = launch(k_ce_dbias, (p.pieces.piece + 31) / 32, CE_THREADS, st, false, (const float*)g.bias_sums, p.pieces, i, (const int*)a.counted, (const float*)a.alpha, d->bias_type, dbias);
    if (both && rc == SAE_OK) rc = product(p.dx, true, true);
    if (!both && want_x && rc == SAE_OK) rc = product(p.dx, true, false);
    if (!both && dweight && rc == SAE_OK) {
      rc = product(p.dw, false, true);
      if (rc == SAE_OK && p.dw_splits > 1) {
        const int start = i * p.pieces.piece, classes = std::min(p.pieces.piece, a.classes - start);
        DxArgs x1 = {job.dw_sums, a.counted, nullptr, a.alpha, (char*)dweight + (int64_t)start * d->features * es, p.sums_pitch, a.features, d->type, job.rows, classes, p.dw_splits};
        rc = launch(k_ce_dx, (unsigned)(up((int64_t)classes * ((d->features + UNIT - 1) / UNIT), CE_THREADS) / CE_THREADS), CE_THREADS, st, false, x1);
      }
    }
  }
  if (want_x && rc == SAE_OK) {
    DxArgs x2 = {job.dx_sums, a.counted, a.index, a.alpha, dx, p.sums_pitch, a.features, d->type, 128 * p.dx.cg, 0, 0};
    rc = launch(k_ce_dx, (unsigned)(up(d->rows * ((d->features + UNIT - 1) / UNIT), CE_THREADS) / CE_THREADS), CE_THREADS, st, false, x2);
  }
  return rc;
}

}  // extern "C"
