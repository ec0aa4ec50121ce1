// The linear cross entropy of float tensors in small problems: ordinary float arithmetic.  Three bfloat16 parts cost a pass over the weights
// and six products each, which pays only when there is enough of them (in_float says where the two meet).  Products are tiles of 32 x 64 by
// 128 threads, split along k until the SMs are filled; whoever reads a product adds its splits in their order.
#pragma once
#include <cooperative_groups.h>

namespace {

constexpr int CF_ROWS = 32, CF_COLS = 64, CF_K = 32, CF_THREADS = 128, CF_LOSS_THREADS = 512, CF_LOSS_CLASSES = 2048;

enum FloatProduct { CF_Z, CF_DX, CF_DW };     // x w',  p w,  p' x

struct FloatArgs {
  const float *x, *w, *p;
  const int *index, *counted;
  int64_t x_pitch, w_pitch;
  int p_pitch, features, classes;
  int splits;
  float* out;                                 // [splits][room][out_pitch]
  int64_t room;
  int out_pitch;
  bool x_vector, w_vector;                    // rows start on 16 bytes
  bool dw_vector;                             // and dweight's
  // dweight in one split goes straight to the caller
  float* dweight;
  void* dbias;
  int bias_type;
  const float* alpha;
  const void* any;                            // an address that copies of nothing may name
};

__device__ __forceinline__ void store_bias(void* out, int type, int64_t j, float v) {
  if (type == SAE_TYPE_FLOAT) ((float*)out)[j] = v;
  else if (type == SAE_TYPE_BFLOAT) ((__nv_bfloat16*)out)[j] = __float2bfloat16_rn(v);
  else ((__half*)out)[j] = __float2half_rn(v);
}

// Four neighbours of a row to shared memory, those behind the first `n` as zeros.
__device__ __forceinline__ void four_in(float* to, const float* from, int n, bool vector, const void* any) {      // any: an address, where nothing is read
  const u32 at = smem_u32(to);
  n = max(0, min(n, 4));
  if (vector) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(n ? (const void*)from : any), "r"(4 * n) : "memory");
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at + 4 * i), "l"(i < n ? (const void*)(from + i) : any), "r"(i < n ? 4 : 0) : "memory");
  }
}

constexpr int CF_STAGES = 4;
// A and B as they lie in memory: rows of CF_K k, or rows of tile rows (columns) for each k; 4 more words a row, against bank conflicts.
template <FloatProduct KIND>
struct FloatTile {
  static constexpr bool A_ROWS = KIND == CF_DW, B_ROWS = KIND != CF_Z;         // k is the slow direction
  static constexpr int A_PITCH = (A_ROWS ? CF_ROWS : CF_K) + 4, B_PITCH = (B_ROWS ? CF_COLS : CF_K) + 4;
  static constexpr int A_SIZE = A_PITCH * (A_ROWS ? CF_K : CF_ROWS), B_SIZE = B_PITCH * (B_ROWS ? CF_K : CF_COLS);
  static constexpr int BYTES = CF_STAGES * (A_SIZE + B_SIZE) * 4;
  // a thread's rows and columns of the tile
  __device__ __forceinline__ static int row(int tr, int i) { return A_ROWS ? tr * 4 + i : tr + 8 * i; }
  __device__ __forceinline__ static int col(int tc, int j) { return B_ROWS ? tc * 4 + j : tc + 16 * j; }
};

// One tile: acc[i][j] for rows tr + 8 i (tr * 4 + i where A's rows are its fast direction) and columns tc + 16 j (tc * 4 + j).
// row_at(i): where in memory the i-th row of x is, -1: nowhere (a row of zeros).  I: rows of a thread, 1 where the tile has no more than 8.
template <FloatProduct KIND, int I, typename RowAt>
__device__ __forceinline__ void float_tile(const FloatArgs& a, float* smem, int row0, int col0, int rows, int cols, int depth, int c0, int c1, RowAt row_at, float (&acc)[4][4]) {
  typedef FloatTile<KIND> F;
  const int t = threadIdx.x;
  const auto fetch = [&](int chunk) {
    if (chunk < c1) {
      const int k0 = chunk * CF_K;
      float* const sa = smem + (chunk - c0) % CF_STAGES * (F::A_SIZE + F::B_SIZE);
      float* const sb = sa + F::A_SIZE;
#pragma unroll
      for (int u = t; u < CF_ROWS * CF_K / 4; u += CF_THREADS) {
        if constexpr (KIND == CF_DW) {
          const int k = u / (CF_ROWS / 4), r = u % (CF_ROWS / 4) * 4;
          four_in(sa + k * F::A_PITCH + r, a.p + (int64_t)(k0 + k) * a.p_pitch + row0 + r, k0 + k < depth ? rows - row0 - r : 0, true, a.any);
        } else {
          const int r = u / (CF_K / 4), k = u % (CF_K / 4) * 4;
          if constexpr (KIND == CF_Z) {
            const int at = row0 + r < rows ? row_at(row0 + r) : -1;
            four_in(sa + r * F::A_PITCH + k, a.x + (at >= 0 ? (int64_t)at * a.x_pitch : 0) + k0 + k, at >= 0 ? depth - k0 - k : 0, a.x_vector, a.any);
          } else four_in(sa + r * F::A_PITCH + k, a.p + (int64_t)(row0 + r) * a.p_pitch + k0 + k, row0 + r < rows ? depth - k0 - k : 0, true, a.any);
        }
      }
#pragma unroll
      for (int u = t; u < CF_COLS * CF_K / 4; u += CF_THREADS) {
        if constexpr (KIND == CF_Z) {
          const int c = u / (CF_K / 4), k = u % (CF_K / 4) * 4;
          four_in(sb + c * F::B_PITCH + k, a.w + (int64_t)(col0 + c) * a.w_pitch + k0 + k, col0 + c < cols ? depth - k0 - k : 0, a.w_vector, a.any);
        } else {
          const int k = u / (CF_COLS / 4), c = u % (CF_COLS / 4) * 4;
          const bool there = k0 + k < depth;
          const float* const row = KIND == CF_DX ? a.w + (int64_t)(k0 + k) * a.w_pitch : a.x + (there ? (int64_t)row_at(k0 + k) * a.x_pitch : 0);
          four_in(sb + k * F::B_PITCH + c, row + col0 + c, there ? cols - col0 - c : 0, KIND == CF_DX ? a.w_vector : a.x_vector, a.any);
        }
      }
    }
    copies_commit();
  };
  const int tr = t / 16, tc = t % 16;
#pragma unroll
  for (int i = 0; i < CF_STAGES - 1; ++i) fetch(c0 + i);
  for (int c = c0; c < c1; ++c) {
    copies_wait<CF_STAGES - 2>();
    __syncthreads();
    fetch(c + CF_STAGES - 1);
    const float* const sa = smem + (c - c0) % CF_STAGES * (F::A_SIZE + F::B_SIZE);
    const float* const sb = sa + F::A_SIZE;
#pragma unroll
    for (int k = 0; k < CF_K; k += 4) {
      if (KIND == CF_DW && c * CF_K + k >= depth) break;      // a few rows of x
      float x[4][4], y[4][4];             // [row or column][k]
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (F::A_ROWS || i < I) {
          const float4 v = *reinterpret_cast<const float4*>(F::A_ROWS ? sa + (k + i) * F::A_PITCH + tr * 4 : sa + F::row(tr, i) * F::A_PITCH + k);
          const float vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (F::A_ROWS) x[q][i] = vs[q]; else x[i][q] = vs[q];
          }
        }
        const float4 w = *reinterpret_cast<const float4*>(F::B_ROWS ? sb + (k + i) * F::B_PITCH + tc * 4 : sb + F::col(tc, i) * F::B_PITCH + k);
        const float ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (F::B_ROWS) y[q][i] = ws[q]; else y[i][q] = ws[q];
        }
      }
      if (KIND == CF_DW) {                // dbias: a feature that is always 1
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col0 + F::col(tc, j) == a.features) y[j][0] = y[j][1] = y[j][2] = y[j][3] = 1.0f;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(x[i][q], y[j][q], acc[i][j]);
    }
  }
  copies_wait<0>();
}

template <FloatProduct KIND>
__global__ void __launch_bounds__(CF_THREADS) k_cf_product(const __grid_constant__ FloatArgs a) {
  typedef FloatTile<KIND> F;
  extern __shared__ __align__(16) float smem[];
  mma::let_next_start();
  mma::wait_for_previous();
  const int count = *a.counted;
  const int rows = KIND == CF_DW ? a.classes : count, cols = KIND == CF_Z ? a.classes : a.features;
  const int depth = KIND == CF_Z ? a.features : KIND == CF_DX ? a.classes : count;
  const int row0 = blockIdx.y * CF_ROWS, col0 = blockIdx.x * CF_COLS;
  if (row0 >= rows) return;
  const int chunks = (depth + CF_K - 1) / CF_K, c0 = (int)((int64_t)chunks * blockIdx.z / a.splits), c1 = (int)((int64_t)chunks * (blockIdx.z + 1) / a.splits);
  float acc[4][4] = {};
  const auto row_at = [&](int i) { return a.index[i]; };
  if (KIND != CF_DW && rows - row0 <= 8) float_tile<KIND, 1>(a, smem, row0, col0, rows, cols, depth, c0, c1, row_at, acc);
  else float_tile<KIND, 4>(a, smem, row0, col0, rows, cols, depth, c0, c1, row_at, acc);
  const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
  const auto row_of = [&](int i) { return F::row(tr, i); };
  const auto col_of = [&](int j) { return F::col(tc, j); };
  if (KIND == CF_DW && a.splits == 1) {
    const float alpha = *a.alpha;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = row0 + row_of(i);
      if (r >= rows) continue;
      if (a.dw_vector && col0 + col_of(3) < a.features) {
        *reinterpret_cast<float4*>(a.dweight + r * a.features + col0 + col_of(0)) = make_float4(acc[i][0] * alpha, acc[i][1] * alpha, acc[i][2] * alpha, acc[i][3] * alpha);
        continue;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = col0 + col_of(j);
        if (c < a.features) { if (a.dweight) a.dweight[r * a.features + c] = acc[i][j] * alpha; }
        else if (c == a.features && a.dbias) store_bias(a.dbias, a.bias_type, r, acc[i][j] * alpha);
      }
    }
    return;
  }
  float* const out = a.out + (int64_t)blockIdx.z * a.room * a.out_pitch;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = row0 + row_of(i);
    if (r >= rows) continue;
    if constexpr (F::B_ROWS) {                    // four neighbours, of a pitch that is a multiple of 4
      if (col0 + col_of(0) < a.out_pitch) *reinterpret_cast<float4*>(out + (int64_t)r * a.out_pitch + col0 + col_of(0)) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = col0 + col_of(j);
        if (c < a.out_pitch) out[(int64_t)r * a.out_pitch + c] = acc[i][j];
      }
    }
  }
}

struct FloatRowArgs {
  const float* z;                             // [splits][room][pitch]
  const void* bias;
  const int *index, *at, *counted;
  int64_t room;
  int splits, pitch, classes, bias_type, reduction;
  // loss (index NULL: lse and rest of the gathered rows alone, for the gradients)
  float *loss, *lse, *rest;
  float2* runs;                               // [rows][blocks of a row]: maximum, sum
  float* at_z;                                // the target's logit
  unsigned* ticket;
  // p
  const float *lse_g, *rest_g, *g;
  float* p;
};
__device__ __forceinline__ float bias_of(const FloatRowArgs& a, int j) {
  if (!a.bias) return 0.0f;
  return a.bias_type == SAE_TYPE_FLOAT ? ((const float*)a.bias)[j]
         : a.bias_type == SAE_TYPE_BFLOAT ? to_f(((const __nv_bfloat16*)a.bias)[j]) : to_f(((const __half*)a.bias)[j]);
}
__device__ __forceinline__ float logit_of(const FloatRowArgs& a, int64_t row, int j) {
  float v = 0;
#pragma unroll 8
  for (int s = 0; s < a.splits; ++s) v += __ldcg(a.z + (s * a.room + row) * a.pitch + j);
  return v + bias_of(a, j);
}
__device__ __forceinline__ void join_runs(float& m, float& s, float om, float os) {
  const float top = fmaxf(m, om);
  if (top > __int_as_float(0xff800000)) s = s * exp2f((m - top) * LOG2E) + os * exp2f((om - top) * LOG2E);
  else s += os;
  m = top;
}

// Maximum and sum of up to CF_LOSS_CLASSES of a row by each block (30522 classes by one block: 64 us); the last block joins them and adds the rows'
// losses, all in their order.
__global__ void __launch_bounds__(CF_LOSS_THREADS) k_cf_loss(const __grid_constant__ FloatRowArgs a) {
  __shared__ float sm[CF_LOSS_THREADS / 32], ss[CF_LOSS_THREADS / 32];
  __shared__ double sd[CF_LOSS_THREADS / 32];
  __shared__ bool final_block;
  mma::let_next_start();
  mma::wait_for_previous();
  const int count = *a.counted, i = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = gridDim.y;
  constexpr float NONE = -INFINITY;
  if (i < count) {
    float m = NONE, s = 0;
    const int end = min(a.classes, ((int)blockIdx.y + 1) * CF_LOSS_CLASSES), target = a.at[i];
    for (int j0 = blockIdx.y * CF_LOSS_CLASSES + threadIdx.x; j0 < end; j0 += 4 * CF_LOSS_THREADS) {
      float z[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) z[q] = j0 + q * CF_LOSS_THREADS < end ? logit_of(a, i, j0 + q * CF_LOSS_THREADS) : NONE;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (j0 + q * CF_LOSS_THREADS == target) a.at_z[i] = z[q];
        if (z[q] > m) { s *= exp2f((m - z[q]) * LOG2E); m = z[q]; }
        s += m == NONE ? (z[q] != z[q] ? z[q] : 0.0f) : exp2f((z[q] - m) * LOG2E);
      }
    }
    for (int o = 16; o; o >>= 1) {
      const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
      join_runs(m, s, om, os);
    }
    if (lane == 0) { sm[warp] = m; ss[warp] = s; }
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int k = 1; k < CF_LOSS_THREADS / 32; ++k) join_runs(m, s, sm[k], ss[k]);
      a.runs[(int64_t)i * blocks + blockIdx.y] = make_float2(m, s);
    }
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    final_block = atomicAdd(a.ticket, 1u) == gridDim.x * gridDim.y - 1;
  }
  __syncthreads();
  if (!final_block) return;
  __threadfence();
  double sum = 0;
  for (int r = threadIdx.x; r < count; r += CF_LOSS_THREADS) {
    const float z = a.at[r] >= 0 ? __ldcg(a.at_z + r) : __int_as_float(0x7fc00000);
    float m = NONE, s = 0;
#pragma unroll 4
    for (int k = 0; k < blocks; ++k) {
      const float2 run = __ldcg(a.runs + (int64_t)r * blocks + k);
      join_runs(m, s, run.x, run.y);
    }
    float rest;
    const float loss = logf(s) + (m - z), lse = lse_of(m, s, rest);
    const int to = a.index ? a.index[r] : r;
    a.lse[to] = a.index || a.at[r] >= 0 ? lse : z;
    if (a.rest) a.rest[to] = rest;
    if (a.loss && a.reduction == SAE_REDUCE_NONE) a.loss[to] = loss;
    sum += loss;
  }
  if (a.reduction == SAE_REDUCE_NONE) return;
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sd[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < CF_LOSS_THREADS / 32; ++k) sum += sd[k];
    *a.loss = (float)(a.reduction == SAE_REDUCE_MEAN ? sum / (double)count : sum);
  }
}

__global__ void __launch_bounds__(CF_THREADS) k_cf_p(const __grid_constant__ FloatRowArgs a) {
  mma::let_next_start();
  mma::wait_for_previous();
  const int i = blockIdx.y, j = blockIdx.x * CF_THREADS + threadIdx.x;
  if (i >= *a.counted || j >= a.classes) return;
  const float p = exp2f(log2_p(logit_of(a, i, j), a.lse_g[i], a.rest_g[i] * LOG2E));
  a.p[(int64_t)i * a.pitch + j] = (j == a.at[i] ? p - 1.0f : p) * a.g[i];
}

// out = alpha * the sum of the splits; rows to where they belong, the column behind the features to dbias.
struct FloatSumArgs {
  const float* sums;
  const int *counted, *index;
  const float* alpha;
  float* out;
  void* dbias;
  int64_t room;
  int splits, pitch, features, bias_type, rows;      // rows < 0: those that are counted
};
// A block has 32 columns; each of its warps takes every fourth split.
__global__ void __launch_bounds__(CF_THREADS) k_cf_sum(const __grid_constant__ FloatSumArgs a) {
  __shared__ float parts[CF_THREADS / 32][32];
  mma::let_next_start();
  mma::wait_for_previous();
  const int64_t r = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  if (r >= (a.rows < 0 ? *a.counted : a.rows)) return;
  float v = 0;
  if (c < a.pitch) {
#pragma unroll 8
    for (int s = warp; s < a.splits; s += CF_THREADS / 32) v += __ldcg(a.sums + (s * a.room + r) * a.pitch + c);
  }
  parts[warp][lane] = v;
  __syncthreads();
  if (warp || c > a.features) return;
  v = (parts[0][lane] + parts[1][lane]) + (parts[2][lane] + parts[3][lane]);
  v *= *a.alpha;
  if (c == a.features) { if (a.dbias) store_bias(a.dbias, a.bias_type, r, v); }
  else if (a.out) a.out[(a.index ? (int64_t)a.index[r] : r) * a.features + c] = v;
}

// The whole forward pass of a head of up to 64 classes, few features and up to 256 rows: a block for 32 rows, the blocks one cluster, which
// adds up the loss.
struct TinyArgs {
  FloatArgs f;
  const int64_t* target;
  int64_t ignore, *count;
  const void* bias;
  float *loss, *lse, *rest;
  int rows, bias_type, reduction;
};
__global__ void __launch_bounds__(CF_THREADS) k_cf_tiny(const __grid_constant__ TinyArgs a) {
  extern __shared__ __align__(16) float smem[];
  __shared__ int at[CF_ROWS], cls[CF_ROWS];
  __shared__ double sums[CF_THREADS / 32], total;
  __shared__ int number;
  namespace cg = cooperative_groups;
  const cg::cluster_group cluster = cg::this_cluster();
  const int row0 = blockIdx.x * CF_ROWS, t = threadIdx.x, tr = t / 16, tc = t % 16;
  if (t < CF_ROWS) {
    const int64_t c = row0 + t < a.rows ? a.target[row0 + t] : a.ignore;
    at[t] = row0 + t < a.rows && c != a.ignore ? row0 + t : -1;
    cls[t] = c >= 0 && c < a.f.classes ? (int)c : -1;
    const u32 used = __ballot_sync(0xffffffffu, at[t] >= 0);
    if (t == 0) number = __popc(used);
  }
  __syncthreads();
  float acc[4][4] = {};
  float_tile<CF_Z, 4>(a.f, smem, row0, 0, a.rows, a.f.classes, a.f.features, 0, (a.f.features + CF_K - 1) / CF_K, [&](int i) { return at[i - row0]; }, acc);
  double sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = tr + 8 * i;
    float m = __int_as_float(0xff800000), s = 0, z_at = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = tc + 16 * j;
      if (c >= a.f.classes) { acc[i][j] = __int_as_float(0xff800000); continue; }
      if (a.bias)
        acc[i][j] += a.bias_type == SAE_TYPE_FLOAT ? ((const float*)a.bias)[c]
                     : a.bias_type == SAE_TYPE_BFLOAT ? to_f(((const __nv_bfloat16*)a.bias)[c]) : to_f(((const __half*)a.bias)[c]);
      m = fmaxf(m, acc[i][j]);
      if (c == cls[r]) z_at = acc[i][j];
    }
    // over the 16 lanes of a row
#pragma unroll
    for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
    for (int j = 0; j < 4; ++j) s += exp2f((acc[i][j] - (m == __int_as_float(0xff800000) ? 0.0f : m)) * LOG2E);
#pragma unroll
    for (int o = 8; o; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      z_at += __shfl_xor_sync(0xffffffffu, z_at, o);
    }
    if (tc == 0 && row0 + r < a.rows) {
      const bool used = at[r] >= 0;
      const float loss = used ? logf(s) + (m - (cls[r] >= 0 ? z_at : __int_as_float(0x7fc00000))) : 0.0f;
      float rest;
      const float lse = lse_of(m, s, rest);
      a.lse[row0 + r] = used ? lse : 0.0f;
      if (a.rest) a.rest[row0 + r] = used ? rest : 0.0f;
      if (a.reduction == SAE_REDUCE_NONE) a.loss[row0 + r] = loss;
      sum += loss;
    }
  }
  sum += __shfl_xor_sync(0xffffffffu, sum, 16);          // lanes 0 and 16 have the sums of their rows
  if (t % 32 == 0) sums[t / 32] = sum;
  __syncthreads();
  if (t == 0) {
    total = 0;
    for (int i = 0; i < CF_THREADS / 32; ++i) total += sums[i];
  }
  cluster.sync();
  if (cluster.block_rank() == 0 && t == 0) {
    double all = 0;
    int n = 0;
    for (unsigned i = 0; i < cluster.num_blocks(); ++i) {
      all += *cluster.map_shared_rank(&total, i);
      n += *cluster.map_shared_rank(&number, i);
    }
    *a.count = n;
    if (a.reduction != SAE_REDUCE_NONE) *a.loss = (float)(a.reduction == SAE_REDUCE_MEAN ? all / (double)n : all);
  }
  cluster.sync();                                        // no block leaves while its sums are read
}

}  // namespace
