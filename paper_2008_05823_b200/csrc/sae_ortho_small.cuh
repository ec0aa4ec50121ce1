// Orthogonalisation of a matrix that one SM holds: a thread block a matrix, all steps, nothing in memory but g and the result.
//
// With x as `small` rows of `big` columns (a matrix taller than wide is read and written transposed), x and S lie in shared memory as two
// float16 parts in blocks of 64 columns, R = 64 or 128 swizzled rows of 128 bytes each.  Such a block is an operand
// either way: its rows the matrix's rows and 64 k (S = x x'), or its rows k and 64 columns (x = B x), so nothing is laid out anew.
// S becomes B in its place, x is replaced block by block.  S and B are added up in as many sums as tensor memory has room for, joined in
// float: each product of 16 k cuts off what a sum has below its last bit.
// 64 rows go through products of 128 rows, whose second half is not looked at.
// What bounds it is the chain of 3 products and 3 epilogues a step (about 8 us); tiles of a matrix spread over SMs wait for one another through
// memory instead, 7 us a product: 64 x 576 took 130 us that way.
#pragma once

namespace {

constexpr int OS_THREADS = 256;
constexpr int OS_PART_BYTES = 64 * 128;                 // 64 rows of a block

template <int R> constexpr int small_blocks() { return R == 64 ? 12 : 5; }        // of 64 columns, that fit
template <int R> constexpr u32 small_bytes() { return (u32)(2 * small_blocks<R>() + 2 * (R / 64)) * (R * 128) + (R == 64 ? OS_PART_BYTES : 0) + 1024; }

// Rows of the kernel's form that holds a matrix; 0: none does.
int small_rows(int64_t small, int64_t big) {
  if (small <= 64 && big <= 64 * small_blocks<64>()) return 64;
  if (small <= 128 && big <= 64 * small_blocks<128>()) return 128;
  return 0;
}

struct SmallJob {
  const Matrix* mats;
  const Place* places;
  const int* order;
  int steps;
  double eps, scale;
  Factors factors[OT_STEPS];
};

// 32 values of a row as hi and lo to two blocks of 64 columns that start at `hi`, `lo`; the values begin at a column that 32 divides.
template <int R>
__device__ __forceinline__ void small_put(const float (&v)[32], u32 hi, u32 lo, int r, int col) {
  const u32 row = (u32)(col / 64) * (R * 128) + (u32)r * 128;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    u32 h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = v[8 * q + 2 * i], b = v[8 * q + 2 * i + 1];
      h[i] = mma::pack_half(a, b);
      const float2 x = mma::unpack_half(h[i]);
      l[i] = mma::pack_half(a - x.x, b - x.y);
    }
    const u32 at = row + (u32)((((col & 63) >> 3) + q) ^ (r & 7)) * 16;
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(hi + at), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(lo + at), "r"(l[0]), "r"(l[1]), "r"(l[2]), "r"(l[3]) : "memory");
  }
}

// The sum of `n` sums, R columns apart.
template <int R>
__device__ __forceinline__ void joined(float (&v)[32], u32 at, int n) {
  mma::tmem_load(at, v);
  for (int g = 1; g < n; ++g) {
    float w[32];
    mma::tmem_load(at + (u32)(g * R), w);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] += w[i];
  }
}

template <int R>
__global__ void __launch_bounds__(OS_THREADS, 1) k_ortho_small(const __grid_constant__ SmallJob job) {
  constexpr u32 BLOCK = R * 128;                         // bytes
  constexpr int SUMS = 512 / R;                          // S is added up in so many sums, which are joined in float
  extern __shared__ unsigned char raw[];
  __shared__ u64 bar;
  __shared__ u32 tmem_at, dead;
  __shared__ double scratch[OS_THREADS / 32];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) mma::tmem_alloc<1>(&tmem_at);
  mma::fence_before();
  __syncthreads();
  mma::fence_after();
  mma::let_next_start();
  mma::wait_for_previous();
  const u32 tmem = tmem_at;
  const int which = job.order[blockIdx.x];
  const Place p = job.places[which];
  const Matrix m = job.mats[which];
  const bool tall = p.rows > p.cols;
  const int small = min(p.rows, p.cols), big = max(p.rows, p.cols), blocks = (big + 63) / 64;
  const u32 base = (smem_u32(raw) + 1023u) & ~1023u;
  const u32 x[2] = {base, base + (u32)blocks * BLOCK}, s[2] = {base + 2u * (u32)blocks * BLOCK, base + (2u * (u32)blocks + R / 64) * BLOCK};

  // eight columns of a row: along the memory's rows, or one of eight of them
  const auto unit = [&](int u, int& i, int& j, float (&v)[UNIT]) {
    if (tall) { i = u % R; j = u / R * UNIT; }
    else { i = u / (blocks * 8); j = (u - i * (blocks * 8)) * UNIT; }
    const int n = i < small ? max(0, min(UNIT, big - j)) : 0;
    if (!tall && n) unit_of(m, p.in_type, i, j, n, v);
    else {
#pragma unroll
      for (int q = 0; q < UNIT; ++q) {
        float e[UNIT] = {};
        if (q < n) unit_of(m, p.in_type, j + q, i, 1, e);
        v[q] = e[0];
      }
    }
  };
  double sum = 0;
  for (int u = threadIdx.x; u < R * blocks * 8; u += OS_THREADS) {
    int i, j;
    float v[UNIT];
    unit(u, i, j, v);
#pragma unroll
    for (int q = 0; q < UNIT; ++q) sum += (double)v[q] * (double)v[q];
  }
  const double factor = job.scale / (sqrt(block_sum(sum, scratch)) + job.eps);
  for (int u = threadIdx.x; u < R * blocks * 8; u += OS_THREADS) {
    int i, j;
    float v[UNIT];
    unit(u, i, j, v);
    u32 h[4], l[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // (rows and columns that there are not stay zero, whatever the factor is)
      const float a = i < small && j + 2 * q < big ? (float)((double)v[2 * q] * factor) : 0.0f, b = i < small && j + 2 * q + 1 < big ? (float)((double)v[2 * q + 1] * factor) : 0.0f;
      h[q] = mma::pack_half(a, b);
      const float2 y = mma::unpack_half(h[q]);
      l[q] = mma::pack_half(a - y.x, b - y.y);
    }
    const u32 at = (u32)(j / 64) * BLOCK + (u32)i * 128 + (u32)(((j & 63) >> 3) ^ (i & 7)) * 16;
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(x[0] + at), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(x[1] + at), "r"(l[0]), "r"(l[1]), "r"(l[2]), "r"(l[3]) : "memory");
  }

  u32 phase = 0;
  bool ok = true;
  // what was written to shared memory and read from tensor memory is settled; then warp 0 issues, and all wait
  const auto products = [&](auto issue) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mma::fence_before();
    __syncthreads();
    mma::fence_after();
    if (warp == 0 && mma::one_lane()) {
      issue();
      mma::commit<1>(&bar);
    }
    __syncwarp();
    ok = mma::wait(&bar, phase & 1, &dead) && ok;
    ++phase;
    mma::fence_after();
  };
  const u32 square = mma::instruction(128, R, false, false, false);
  constexpr int seg[3][2] = {{0, 1}, {1, 0}, {0, 0}};
  const int quarter = warp & 3, half = warp >> 2, r = quarter * 32 + lane;
  const bool mine = quarter * 32 < R;                    // this warp's rows are looked at
  const u32 lanes = tmem + ((u32)quarter * 32 << 16);
  constexpr int CHUNKS = R / 64;                         // of 32 columns of S that a thread has

  for (int step = 0; step < job.steps; ++step) {
    const Factors f = job.factors[step];
    products([&] {
      for (int q = 0; q < 3; ++q)
        for (int b = 0; b < blocks; ++b) {
          const u64 a = mma::smem_desc(x[seg[q][0]] + (u32)b * BLOCK, false), c = mma::smem_desc(x[seg[q][1]] + (u32)b * BLOCK, false);
#pragma unroll
          for (u32 k = 0; k < 4; ++k) mma::product<1>(tmem + (u32)(b * 4 + k) % SUMS * R, a + 2 * k, c + 2 * k, square, q || b * 4 + (int)k >= SUMS);
        }
    });
    float own[CHUNKS][32];
    if (mine) {
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const int col = half * (R / 2) + k * 32;
        joined<R>(own[k], lanes + (u32)col, min(4 * blocks, SUMS));
#pragma unroll
        for (int i = 0; i < 32; ++i) own[k][i] *= f.s_sum;
        small_put<R>(own[k], s[0], s[1], r, col);
      }
    }
    products([&] {
      for (int q = 0; q < 3; ++q)
        for (int b = 0; b < R / 64; ++b) {
          const u64 a = mma::smem_desc(s[seg[q][0]] + (u32)b * BLOCK, false), c = mma::smem_desc(s[seg[q][1]] + (u32)b * BLOCK, false);
#pragma unroll
          for (u32 k = 0; k < 4; ++k) mma::product<1>(tmem + k * R, a + 2 * k, c + 2 * k, square, q || b);
        }
    });
    if (mine) {
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const int col = half * (R / 2) + k * 32;
        float v[32];
        joined<R>(v, lanes + (u32)col, 4);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          v[i] = __fmaf_rn(f.b_own, own[k][i], f.b_sum * v[i]);
          if (r == col + i) v[i] += f.b_diag;
        }
        small_put<R>(v, s[0], s[1], r, col);
      }
    }
    for (int b0 = 0; b0 < blocks; b0 += 8) {
      const int b1 = min(b0 + 8, blocks);
      products([&] {
        for (int b = b0; b < b1; b += 4) {               // four blocks, 256 columns, at a time
          const u32 wide = mma::instruction(128, 64 * min(4, b1 - b), false, false, true);
          u32 add = 0;
          for (int q = 0; q < 3; ++q) {
            const u64 c = mma::smem_desc(x[seg[q][1]] + (u32)b * BLOCK, true, BLOCK);
#pragma unroll
            for (u32 k = 0; k < R / 16; ++k) {
              const u64 a = mma::smem_desc(s[seg[q][0]] + k / 4 * BLOCK, false) + 2 * (k % 4);
              mma::product<1>(tmem + (u32)(b - b0) * 64, a, c + 128 * k, wide, add);
              add = 1;
            }
          }
        }
      });
      if (!mine) continue;
      for (int b = b0; b < b1; ++b) {
        const int col = b * 64 + half * 32;
        float v[32];
        mma::tmem_load(lanes + (u32)((b - b0) * 64 + half * 32), v);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= ok ? f.x_sum : __int_as_float(0x7fc00000);
        if (step + 1 < job.steps) small_put<R>(v, x[0], x[1], r, col);
        else if (r < small && col < big) {
          const int n = min(32, big - col);
          if (!tall) {
            const long long to = r * m.out_ld + col;
            if (p.out_type == SAE_TYPE_FLOAT) mma::store_row((float*)m.out + to, v, n);
            else if (p.out_type == SAE_TYPE_BFLOAT) mma::store_row((__nv_bfloat16*)m.out + to, v, n);
            else mma::store_row((__half*)m.out + to, v, n);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              if (i >= n) continue;
              const long long to = (col + i) * m.out_ld + r;
              if (p.out_type == SAE_TYPE_FLOAT) ((float*)m.out)[to] = v[i];
              else if (p.out_type == SAE_TYPE_BFLOAT) ((__nv_bfloat16*)m.out)[to] = __float2bfloat16_rn(v[i]);
              else ((__half*)m.out)[to] = __float2half_rn(v[i]);
            }
          }
        }
      }
    }
  }
  mma::fence_before();
  __syncthreads();
  mma::fence_after();
  if (!ok && warp == 0) {                                // products in flight end before the tensor memory is given back
    if (mma::one_lane()) mma::commit<1>(&bar);
    __syncwarp();
    mma::wait_slow(smem_u32(&bar), phase & 1, nullptr, mma::DRAIN_NS);
  }
  if (warp == 0) mma::tmem_free<1>(tmem);
}

template <int R>
cudaError_t launch_small(const SmallJob& job, int matrices, cudaStream_t st) {
  static std::atomic<unsigned long long> ready{0};
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(k_ortho_small<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)small_bytes<R>());
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)matrices);
  cfg.blockDim = dim3(OS_THREADS);
  cfg.dynamicSmemBytes = small_bytes<R>();
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_ortho_small<R>, job);
}

}  // namespace
