// Orthogonalisation of many matrices by Newton-Schulz products (sae_ortho_* of include/sae.h).
//
//   x <- g / (|g| + eps), then `steps` times  x <- a x + (b s + c s s) x  with s = x x' (x' x where a matrix is taller than wide)
//
// One call is a kernel for the norms, one that lays g out as two float16 parts, and ONE kernel for all products of all steps:
// S = s;  B = a + b S + c S S;  x = B x, tile by tile.  Its tiles are one list; a tile starts when the tiles of its
// matrix's product before are all written, which a counter of each matrix says.  Every cluster takes every n-th tile of the list in
// order, and all clusters run at once (cooperative launch), so the first tile that is not done can always be worked on.
// Against a launch for each product (15 of them): no gaps and no partly filled last wave between products.
// S and B are symmetric: only tiles on and above the diagonal are made and kept.  Blocks of k that lie below it are loaded from
// above it, with rows and k in exchanged order, which the matrix descriptors undo.
//
// Precision.  x is held as hi + lo, two float16 of a value scaled by a power of two (22 bits).  For results in bfloat16
// the products read hi alone (11 bits), and a lo is added in the last product's epilogue: a rounding of x itself to 11
// bits in every step would be multiplied by a^5 = 485 in the directions of small singular values (errors of 1.4e-2 for a gradient of a few
// strong directions over noise, 8e-4 this way).  Float32 and float16 results take hi and lo in all three products (hi lo + lo hi +
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
// Bytes of the matrices that go through all steps together, one such portion after another.  Portions that L2 holds (64 or 128 MB) have too few
// tiles to cover the wait from one product to the next: the 12-layer encoder takes 4070 and 2020 us with them, 1850 with 256 MB, 1800 with
// 512, 1880 with all at once.
constexpr int64_t OT_PORTION = 512ll << 20;
constexpr int OT_ARGS = 448;                  // matrices whose addresses travel as kernel arguments

constexpr int OT_SPLITS = 16;                 // of S's sums
constexpr int OT_SHAPES = 32, OT_BATCHES = 800;   // as many are looked up in shared memory
constexpr int OT_STEPS = 64;

// All matrices of one shape and precision: its maps, and what else a tile needs to know.
struct Maps { CUtensorMap x[2], s, b; };
struct Shape {
  __half *x[2], *s, *b;
  long long x_plane, s_plane;                 // elements of a part
  int rows, cols, small, tall;
  int x_pitch, s_pitch;
  int s_parts, plain;                         // plain: 16-bit matrices, whose x0 is hi alone, exactly
  int x_tiles, x_tile_cols, s_tiles;          // tiles of one matrix's products
  int first;                                  // its first matrix in the class's order
};
// Of a shape whose S has too few tiles, and is made in parts.
struct Parts {
  int n;                                      // of k
  float* sums;                                // [matrix][s_tile][n][rows of a tile][columns]
  u32* arrived;                               // [matrix][s_tile][16]: parts that the warp of this place has written
};
// One product of some neighbouring matrices of a shape: tiles begin .. end - 1 of the list.
struct Batch { int begin, end, first; u32 shape : 24, phase : 2, step : 6; };     // (up to 2^20 shapes, 64 steps)

struct Matrix { const void* in; void* out; long long in_ld, out_ld; };
struct Place { int rows, cols, x_pitch, in_type, out_type, first_chunk, chunks; __half* x; long long x_plane; u32 *done, *arrived; int num_arrived; float* ratio; int plain; };
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
  if (ch.unit == 0) {
    if (threadIdx.x == 0) *p.done = 0;
    for (int i = threadIdx.x; i < p.num_arrived; i += OT_THREADS) p.arrived[i] = 0;
  }
  double s = 0;
  for (int i = threadIdx.x; i < p.chunks; i += OT_THREADS) s += sums[p.first_chunk + i];
  // 16-bit elements times a power of two are float16 exactly (but for what is 2^-25 of the norm); the rest of the factor, from 1/2
  // to 1, goes into the first step's products
  double factor = scale / (sqrt(block_sum(s, scratch)) + eps), ratio = 1.0;
  if (p.plain && factor > 0 && factor < 1e300) {
    int e;
    ratio = frexp(factor, &e);
    factor = ldexp(1.0, e);
  }
  if (ch.unit == 0 && threadIdx.x == 0) *p.ratio = (float)ratio;
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
    if (!p.plain) *reinterpret_cast<uint4*>(to + p.x_plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// ---- products ---------------------------------------------------------------------------------------------------------
enum Phase { PHASE_S, PHASE_B, PHASE_X };
// S = s_sum acc;  B = b_diag 1 + b_own S + b_sum acc;  x = x_own lo + x_sum acc
struct Factors { float s_sum, b_diag, b_own, b_sum, x_own, x_sum; };

// A part of S's sums: left in memory, and the warp that finds itself the last of its place in the tile adds all parts up in their order, the same bits
// whoever that is, and writes S.
__device__ __forceinline__ void join_sums(const Shape& g, const Parts& parts_of, const mma::Tile& t, const mma::Sums sums, int tile_rows, int tile_cols, int row, int half, int chunks, float scale) {
  const int split = t.part / g.s_tiles, q = t.part - split * g.s_tiles, first = half * mma::epilogue_width(tile_cols), next = tile_rows * tile_cols, r = t.row + row;
  const long long tile = (long long)t.item * g.s_tiles + q;
  float* const parts = parts_of.sums + (tile * parts_of.n * tile_rows + row) * tile_cols + first;
  const bool there = r < g.small;
  for (int k = 0; k < chunks; ++k) {
    float v[32];
    __syncwarp();
    mma::sums_of(sums, first + k * 32, v);
    if (there) mma::store_row(parts + (long long)split * next + k * 32, v, 32);
  }
  __threadfence();
  __syncwarp();
  u32* const arrived = parts_of.arrived + tile * 16 + (row >> 5) * 2 + half;
  u32 before = 0;
  if ((threadIdx.x & 31) == 0) before = atomicAdd(arrived, 1u);
  if (__shfl_sync(0xffffffffu, before, 0) + 1 != (u32)parts_of.n) return;
  __threadfence();
  if ((threadIdx.x & 31) == 0) *arrived = 0;               // for the next step
  if (!there) return;
  __half* const to = g.s + (t.item * (long long)g.s_parts) * g.s_plane + (long long)r * g.s_pitch + t.col + first;
  for (int k = 0; k < chunks; ++k) {
    float v[32] = {};
#pragma unroll 2
    for (int s = 0; s < parts_of.n; ++s) {
      u32 w[2][16];
      mma::load_written(parts + (long long)s * next + k * 32, w[0]);
      mma::load_written(parts + (long long)s * next + k * 32 + 16, w[1]);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(w[i >> 4][i & 15]);
    }
    u32 hi[16], lo[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = v[2 * i] * scale, y = v[2 * i + 1] * scale;
      hi[i] = mma::pack_half(x, y);
      const float2 h = mma::unpack_half(hi[i]);
      lo[i] = mma::pack_half(x - h.x, y - h.y);
    }
    mma::store_words(to + k * 32, hi);
    if (g.s_parts > 1) mma::store_words(to + g.s_plane + k * 32, lo);
  }
}

// SPLIT: some shape's S is made in parts (a kernel of its own: asking took 15 products of 512 x 512 3 % longer).
template <bool SPLIT>
struct OrthoJob {
  static constexpr bool REPORTS = true, LONG = false;
  static constexpr int STAGING = 32 * 256;      // 32 rows of 128 elements
  int cols;
  bool bfloat;
  mma::Segments seg;
  const Maps* maps;
  const Shape* shapes;
  const Parts* parts;             // of S
  const Batch* batches;
  int num_shapes, num_batches, total, rows, steps, arrivals;   // rows of a tile; blocks that write one
  u32* done;                        // in the class's order
  const Matrix* mats;
  const Place* places;
  const int* order;
  const float* ratios;
  Factors factors[OT_STEPS];

  struct Shared {
    Shape shapes[OT_SHAPES];
    Batch batches[OT_BATCHES];
  };
  __device__ __forceinline__ void fill(Shared& s) const {
    if (num_shapes <= OT_SHAPES)
      for (int i = threadIdx.x; i < num_shapes * (int)(sizeof(Shape) / 4); i += (int)blockDim.x) reinterpret_cast<u32*>(s.shapes)[i] = reinterpret_cast<const u32*>(shapes)[i];
    if (num_batches <= OT_BATCHES)
      for (int i = threadIdx.x; i < num_batches * (int)(sizeof(Batch) / 4); i += (int)blockDim.x) reinterpret_cast<u32*>(s.batches)[i] = reinterpret_cast<const u32*>(batches)[i];
  }
  struct Local { const Shape* shapes; const Batch* batch; int first, step; };
  __device__ __forceinline__ Local begin(const Shared& s, int cluster, int clusters) const {
    return {num_shapes <= OT_SHAPES ? s.shapes : shapes, num_batches <= OT_BATCHES ? s.batches : batches, cluster, clusters};
  }
  // The tile (row, column) of a symmetric product that is number q of those not wholly below the diagonal.
  __device__ __host__ static void above(int q, int rows, int cols, int small, int& r, int& c) {
    const int wide = (small + cols - 1) / cols, per = rows / cols;
    for (r = 0; q >= wide - r * per; ++r) q -= wide - r * per;
    c = r * per + q;
  }
  // the first block of k that S and B have for a row (the rows of a tile have the same)
  __device__ __forceinline__ int kept_from(int row) const { return row / rows * rows / mma::BLOCK_K; }
  __device__ __forceinline__ bool tile(Local& l, int i, mma::Tile& t) const {
    const int w = l.first + i * l.step;
    if (w >= total) return false;
    while (w >= l.batch->end) ++l.batch;
    const Batch b = *l.batch;
    const Shape& g = l.shapes[b.shape];
    const Maps& m = maps[b.shape];
    const bool px = b.phase == PHASE_X;
    const int splits = SPLIT && b.phase == PHASE_S ? parts[b.shape].n : 1, per = px ? g.x_tiles : g.s_tiles * splits, n = (w - b.begin) / per;
    int q = (w - b.begin) - n * per, split = 0;
    if (SPLIT) t.part = q;
    if (SPLIT && splits > 1) { split = q / g.s_tiles; q -= split * g.s_tiles; }
    t.item = b.first + n;
    t.group = b.shape;
    int r, c;
    if (px) { r = q / g.x_tile_cols; c = q - r * g.x_tile_cols; }
    else above(q, rows, cols, g.small, r, c);
    t.a_row = t.row = r * rows;
    t.b_row = t.col = c * cols;
    t.a_k = t.b_k = t.a_turn = t.b_turn = 0;
    const int zx = t.item * 2, zs = t.item * g.s_parts, from = b.step & 1;
    int k = g.small;
    t.a_rows_first = t.b_rows_first = false;
    if (b.phase == PHASE_S) {
      t.a = t.b = &m.x[from];
      t.a_plane = t.b_plane = zx;
      t.a_rows_first = t.b_rows_first = g.tall;
      k = g.tall ? g.rows : g.cols;
    } else if (b.phase == PHASE_B) {
      t.a = t.b = &m.s;
      t.a_plane = t.b_plane = zs;
      t.a_turn = kept_from(t.row);
      t.b_turn = kept_from(t.col);
    } else {
      t.a = g.tall ? &m.x[from] : &m.b;
      t.b = g.tall ? &m.b : &m.x[from];
      t.a_plane = g.tall ? zx : zs;
      t.b_plane = g.tall ? zs : zx;
      t.b_rows_first = !g.tall;
      if (g.tall) t.b_turn = kept_from(t.col);
      else t.a_turn = kept_from(t.row);
    }
    t.blocks = (k + mma::BLOCK_K - 1) / mma::BLOCK_K;
    if (SPLIT && splits > 1) {
      const int from = t.blocks * split / splits;
      t.a_k = t.b_k = from * mma::BLOCK_K;
      t.blocks = t.blocks * (split + 1) / splits - from;
    }
    return true;
  }
  // Whether x has a lo when step s begins.  Where products read hi alone, the last step needs none: a rounding is multiplied by a at most there.
  __device__ __forceinline__ bool has_lo(const Shape& g, int s) const { return g.s_parts == 2 || (s ? s + 1 < steps : !g.plain); }
  // the matrix's counter, and what it shows when every product before this tile's is written
  __device__ __forceinline__ u32* counter(const Shape& g, const mma::Tile& t) const { return done + g.first + t.item; }
  __device__ __forceinline__ u32 before(const Shape& g, const Batch& b) const {
    const int s = SPLIT ? g.s_tiles * parts[b.shape].n : g.s_tiles;
    return (u32)((b.step * (s + g.s_tiles + g.x_tiles) + (b.phase > PHASE_S ? s : 0) + (b.phase > PHASE_B ? g.s_tiles : 0)) * arrivals);
  }
  __device__ __forceinline__ bool ready(const Local& l, const mma::Tile& t, u32* dead) const {
    const Shape& g = l.shapes[t.group];
    if (!mma::wait_counter(counter(g, t), before(g, *l.batch), dead)) return false;
    mma::fence_copies();
    return true;
  }

  __device__ __forceinline__ void report(const Local& l, const mma::Tile& t) const {
    mma::fence_copies();
    mma::add_counter(counter(l.shapes[t.group], t));
  }

  // A warp takes its rows 32 columns at a time.  Present values come in through shared memory, whole lines at a time, while the tile's products
  // run; a thread that reads 64 bytes of its own row keeps the load and store unit busy for 32 lines with every instruction.  Results go out
  // straight from the registers, 32 bytes a store: an SM's stores pass at 32 bytes a cycle, and lines put together in shared memory first
  // did not pass faster.  Copies by TMA, in or out, hold up those of the operands (16000 cycles a tile of 256 x 256, whose products take
  // 6144 at 768 rows).
  struct Epilogue {
    const OrthoJob& job;
    const Local& l;                   // the role's own: its batch is the tile's
    const int row, part;
    const u32 in;                     // shared memory, 16 pieces of 16 bytes a row
    int chunks;                       // of 32 columns that this warp has of the tile
    int own;                          // parts of present values that come in for a chunk
    bool here;                        // they do come in
    __device__ __forceinline__ Epilogue(const OrthoJob& j, const Local& l, int r, int p, u32 at)
        : job(j), l(l), row(r), part(p), in(at), chunks(0), own(0), here(false) {}

    __device__ __forceinline__ void finish() {}
    __device__ __forceinline__ void prepare(const mma::Tile& t, int number, mma::Control* ctl) {
      const Batch b = *l.batch;
      const Shape& g = l.shapes[t.group];
      const bool px = b.phase == PHASE_X, two = g.s_parts == 2;
      const int lane = threadIdx.x & 31, width = mma::epilogue_width(job.cols), row0 = t.row + (row & ~31), col0 = t.col + part * width;
      const int rows = px ? g.rows : g.small, cols = px ? g.cols : g.small;
      chunks = row0 >= rows ? 0 : (max(0, min(width, cols - col0)) + 31) / 32;
      own = b.phase == PHASE_S ? 0 : b.phase == PHASE_B ? g.s_parts : two ? 0 : job.has_lo(g, b.step);
      here = true;
      if (own && chunks) {
        here = __all_sync(0xffffffffu, mma::wait_shared(&ctl->ready, (u32)number + 1, &ctl->dead));      // (without them the tile is NaN)
        if (here) {
          const int pitch = px ? g.x_pitch : g.s_pitch, p = lane & 15;
          const long long plane = px ? g.x_plane : g.s_plane;
          const __half* from = (px ? g.x[b.step & 1] + (t.item * 2ll + 1) * plane : g.s + (long long)t.item * g.s_parts * plane) + (long long)row0 * pitch + col0;
          if (own == 2) from += (p >> 3) * plane + (p & 7) * 8;          // pieces 8 .. 15 are lo's
          else from += p * 8;
          if ((own == 2 ? p & 7 : p) < chunks * 4)
#pragma unroll
            for (int r = lane >> 4; r < 32; r += 2)
              if (row0 + r < rows) mma::piece_in(mma::staged_at(in, r, p), from + (long long)r * pitch);
        }
      }
    }
    __device__ __forceinline__ void tile(const mma::Tile& t, const mma::Sums& sums) {
      if (!chunks) return;
      const Batch b = *l.batch;
      const Shape& g = l.shapes[t.group];
      const Factors f = job.factors[b.step];
      const bool px = b.phase == PHASE_X, last = px && b.step + 1 == job.steps;
      const int r = t.row + row, cols = px ? g.cols : g.small, parts = px ? 1 + job.has_lo(g, b.step + 1) : g.s_parts;
      const float mine = px ? f.x_own : f.b_own;
      float sum = px ? f.x_sum : b.phase == PHASE_B ? f.b_sum : f.s_sum;
      if (b.step == 0 && b.phase != PHASE_B) {              // x0 is hi times this
        const float ratio = job.ratios[g.first + t.item];
        sum *= px ? ratio : ratio * ratio;
      }
      if (!here) sum = __int_as_float(0x7fc00000);
      if (SPLIT && b.phase == PHASE_S && job.parts[b.shape].n > 1) {
        join_sums(g, job.parts[b.shape], t, sums, job.rows, job.cols, row, part, chunks, sum);
        return;
      }
      const int lane_row = row & 31, rows = px ? g.rows : g.small, pitch = px ? g.x_pitch : g.s_pitch;
      const long long plane = px ? g.x_plane : g.s_plane;
      __half* const to = (px ? g.x[(b.step & 1) ^ 1] : b.phase == PHASE_B ? g.b : g.s) + t.item * (long long)(px ? 2 : g.s_parts) * plane + (long long)r * pitch;
      Matrix m = {};
      int type = 0;
      if (last) {
        const int i = job.order[g.first + t.item];
        m = job.mats[i];
        type = job.places[i].out_type;
      }
      if (own) {
        mma::pieces_arrived();
        __syncwarp();
      }
      for (int k = 0; k < chunks; ++k) {
        const int col = t.col + part * mma::epilogue_width(job.cols) + k * 32;
        float v[32];
        mma::sums_of(sums, col - t.col, v);
        if (sum != 1.0f) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] *= sum;
        }
        u32 hi[16], lo[16];
        if (own) {
          mma::staged_load(in, lane_row, 4 * k, hi);
          if (own == 2) mma::staged_load(in, lane_row, 8 + 4 * k, lo);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float2 x = mma::unpack_half(hi[i]);
            if (own == 2) { const float2 y = mma::unpack_half(lo[i]); x.x += y.x; x.y += y.y; }
            v[2 * i] = __fmaf_rn(mine, x.x, v[2 * i]);
            v[2 * i + 1] = __fmaf_rn(mine, x.y, v[2 * i + 1]);
          }
        }
        if (b.phase == PHASE_B && (unsigned)(r - col) < 32u) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] += r - col == i ? f.b_diag : 0.0f;
        }
        if (last) {
          if (r < g.rows) {
            const int w = min(32, cols - col);
            const long long out = r * m.out_ld + col;
            if (type == SAE_TYPE_FLOAT) mma::store_row((float*)m.out + out, v, w);
            else if (type == SAE_TYPE_BFLOAT) mma::store_row((__nv_bfloat16*)m.out + out, v, w);
            else mma::store_row((__half*)m.out + out, v, w);
          }
          continue;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) hi[i] = mma::pack_half(v[2 * i], v[2 * i + 1]);
        if (r < rows) mma::store_words(to + col, hi);
        if (parts == 1) continue;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float2 h = mma::unpack_half(hi[i]);
          lo[i] = mma::pack_half(v[2 * i] - h.x, v[2 * i + 1] - h.y);
        }
        if (r < rows) mma::store_words(to + plane + col, lo);
      }
    }
  };
};

}  // namespace

#include "sae_ortho_small.cuh"

namespace {

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

// Shapes whose products have the same number of parts: one launch.
struct Class {
  int parts, cg, cols;
  int first, n;                  // shapes
  int first_batch, batches, total;
  bool split;                    // some S is made in parts
};

// The largest |p(v)| and |a + b v^2 + c v^4| over 0 <= v <= top.
void bounds(const float* k, double top, double& p, double& q) {
  p = q = 0;
  for (int i = 0; i <= 4096; ++i) {
    const double v = top * i / 4096, s = v * v, e = k[0] + k[1] * s + k[2] * s * s;
    p = std::max(p, std::fabs(v * e));
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
  std::vector<double> s_scale, b_scale, ones;    // of every step
  double x_scale;
  std::vector<Class> classes;
  int small_n[2], small_first[2];                // matrices that one SM holds, of up to 64 and up to 128 rows, and where they begin in `order`
  char* arena;
  Maps* maps;
  Shape* shapes;
  Parts* parts;
  Batch* batches;
  u32* done;
  float* ratios;
  Matrix* mats;
  Place* places;
  Chunk* chunk_list;
  int* order;
  double* sums;
  float* split_sums;                             // of S, where it is made in parts
  u32* arrived;
};

namespace {

int cuda_status(sae_ortho* h, cudaError_t e) {
  h->last_cuda_error = (int)e;
  cudaGetLastError();
  return e == cudaErrorMemoryAllocation ? SAE_ERR_NOMEM : SAE_ERR_CUDA;
}

void release(sae_ortho* h) {
  cudaFree(h->arena); cudaFree(h->maps); cudaFree(h->shapes); cudaFree(h->parts); cudaFree(h->batches); cudaFree(h->done); cudaFree(h->ratios); cudaFree(h->mats); cudaFree(h->places); cudaFree(h->chunk_list); cudaFree(h->order); cudaFree(h->sums); cudaFree(h->split_sums); cudaFree(h->arrived);
  delete h;
}

template <typename T>
cudaError_t upload(T** to, const std::vector<T>& v, cudaStream_t st) {
  cudaError_t e = cudaMalloc((void**)to, std::max<size_t>(1, v.size()) * sizeof(T));
  if (e == cudaSuccess && !v.empty()) e = cudaMemcpyAsync(*to, v.data(), v.size() * sizeof(T), cudaMemcpyHostToDevice, st);
  return e;
}

// Tiles of a symmetric product that are not wholly below the diagonal.
int tiles_above(int small, int rows, int cols) {
  const int wide = (small + cols - 1) / cols, per = rows / cols;
  int n = 0;
  for (int r = 0; r * per < wide; ++r) n += wide - r * per;
  return n;
}

void count_tiles(Shape& g, int rows, int cols) {
  g.x_tile_cols = (g.cols + cols - 1) / cols;
  g.x_tiles = (g.rows + rows - 1) / rows * g.x_tile_cols;
  g.s_tiles = tiles_above(g.small, rows, cols);
}

// Parts of k that S's sums are made in, where a class has fewer tiles than SMs (or pairs): time in the units of choose_tiles.  A warp that joins
// sums waits about 3 us, and 0.5 us for 32 columns of each part.
int splits_of(const Class& c, const Shape& g, int64_t tiles, int units, int cols, double cost, double* time) {
  const int k = g.tall ? g.rows : g.cols, most = (int)std::min<int64_t>(units / std::max<int64_t>(1, tiles), OT_SPLITS);
  const double us = c.parts == 1 ? 400.0 : 130.0;
  int best = 1;
  *time = cost * k;
  for (int s = 2; s <= most; ++s) {
    const double t = cost * k / s + us * (3.0 + 0.5 * s * cols / 64);
    if (t < *time) { *time = t; best = s; }
  }
  return best;
}

// Tile shape of a class: time in units of a block's k loop, waves of tiles over the SMs (or pairs).
void choose_tiles(Class& c, std::vector<Shape>& shapes, std::vector<Parts>& parts, const std::vector<int>& count, int sms) {
  struct Form { int cg, cols; double cost; };
  const Form forms[3] = {{2, c.parts == 1 ? 256 : 128, c.parts == 1 ? 2.0 : 1.75}, {1, 128, 2.1}, {1, 64, 1.7}};
  double best = 0;
  const Form* form = forms;
  for (const Form& f : forms) {
    const int units = sms / f.cg;
    double work_s = 0, work_x = 0, longest_s = 0, longest_x = 0;
    int64_t tiles = 0;
    for (int i = c.first; i < c.first + c.n; ++i) {
      Shape g = shapes[i];
      count_tiles(g, 128 * f.cg, f.cols);
      tiles += (int64_t)g.s_tiles * count[i];
    }
    for (int i = c.first; i < c.first + c.n; ++i) {
      Shape g = shapes[i];
      count_tiles(g, 128 * f.cg, f.cols);
      const int big = g.tall ? g.rows : g.cols;
      work_s += (double)g.s_tiles * big * count[i];
      work_x += (double)(g.x_tiles + g.s_tiles) * g.small * count[i];
      double alone;
      splits_of(c, g, tiles, units, f.cols, f.cost, &alone);
      longest_s = std::max(longest_s, alone / f.cost);
      longest_x = std::max(longest_x, (double)g.small);
    }
    const double t = f.cost * (std::max(work_s / units, longest_s) + std::max(work_x / units, 2 * longest_x));
    if (best == 0 || t < best) { best = t; c.cg = f.cg; c.cols = f.cols; form = &f; }
  }
  int64_t tiles = 0;
  for (int i = c.first; i < c.first + c.n; ++i) {
    count_tiles(shapes[i], 128 * c.cg, c.cols);
    tiles += (int64_t)shapes[i].s_tiles * count[i];
  }
  for (int i = c.first; i < c.first + c.n; ++i) parts[i].n = splits_of(c, shapes[i], tiles, sms / c.cg, c.cols, form->cost, &best);
}

// The list of a class's products.  Portions of matrices that L2 holds go through all steps, one portion after another.
void list_products(Class& c, const std::vector<Shape>& shapes, const std::vector<Parts>& parts, const std::vector<int>& count, int steps, std::vector<Batch>& batches) {
  struct Piece { int shape, first, n; };
  std::vector<std::vector<Piece>> portions;
  int64_t room = 0;
  for (int i = c.first; i < c.first + c.n; ++i) {
    const Shape& g = shapes[i];
    const int64_t bytes = 8 * g.x_plane + 4 * g.s_parts * g.s_plane;
    for (int m = 0; m < count[i]; ++m) {
      if (portions.empty() || room < bytes) { portions.emplace_back(); room = OT_PORTION; }
      room -= bytes;
      auto& p = portions.back();
      if (!p.empty() && p.back().shape == i) ++p.back().n;
      else p.push_back({i, m, 1});
    }
  }
  c.first_batch = (int)batches.size();
  int64_t at = 0;
  for (const auto& p : portions)
    for (int s = 0; s < steps; ++s)
      for (int phase = 0; phase < 3; ++phase)
        for (const Piece& q : p) {
          const Shape& g = shapes[q.shape];
          Batch b = {};
          b.begin = (int)at;
          b.end = (int)(at += (int64_t)q.n * (phase == PHASE_X ? g.x_tiles : phase == PHASE_S ? g.s_tiles * parts[q.shape].n : g.s_tiles));
          b.first = q.first; b.shape = (u32)(q.shape - c.first); b.phase = (u32)phase; b.step = (u32)s;
          batches.push_back(b);
        }
  c.batches = (int)batches.size() - c.first_batch;
  if (at > (1 << 30)) throw std::bad_alloc();       // (more tiles than an int counts: no list of matrices that memory holds)
  c.total = (int)at;
}

void factors(const sae_ortho* h, const std::vector<double>& b_scale, Factors* f) {
  for (int i = 0; i < h->steps; ++i) {
    const float* k = h->coef.data() + 3 * i;
    const double sx = h->x_scale, ss = h->s_scale[i], sb = b_scale[i], to = i + 1 == h->steps ? 1.0 / sx : 1.0;
    f[i] = {(float)(ss / (sx * sx)), (float)(k[0] * sb), (float)(k[1] * sb / ss), (float)(k[2] * sb / (ss * ss)), (float)(k[0] * to), (float)(to / sb)};
  }
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

template <bool SPLIT>
cudaError_t launch_class(const sae_ortho* h, const Class& c) {
  static thread_local OrthoJob<SPLIT> job;
  job = {};
  job.cols = c.cols;
  job.rows = 128 * c.cg;
  if (c.parts == 2) job.seg = {3, {0, 1, 0}, {1, 0, 0}};
  else job.seg = {1, {0}, {0}};
  job.maps = h->maps + c.first;
  job.shapes = h->shapes + c.first;
  job.parts = h->parts + c.first;
  job.batches = h->batches + c.first_batch;
  job.num_shapes = c.n; job.num_batches = c.batches; job.total = c.total; job.steps = h->steps; job.arrivals = c.cg;
  job.done = h->done;
  job.ratios = h->ratios;
  job.mats = h->mats;
  job.places = h->places;
  job.order = h->order;
  // (one part: B hi is added to x hi times 1)
  factors(h, c.parts == 2 ? h->b_scale : h->ones, job.factors);
  return mma::launch_products(job, c.cg, std::min(c.total, h->num_sms / c.cg), h->stream, true);
}

}  // namespace

extern "C" {

int sae_ortho_init(const sae_ortho_config* cfg, sae_ortho** out) {
  if (!cfg || !out) return SAE_ERR_INVALID_ARG;
  *out = nullptr;
  if (cfg->abi_version != SAE_ABI_VERSION) return SAE_ERR_ABI;
  const int K = cfg->num_rows, T = cfg->num_matrices;
  if (K < 1 || K > 1024 || T < 1 || !cfg->rows || !cfg->cols || !cfg->coefficients || cfg->device < 0 || cfg->steps < 1 || cfg->steps > OT_STEPS ||
      !(cfg->eps >= 0.0f) || !std::isfinite(cfg->eps) || (long long)K * T > (1 << 20)) return SAE_ERR_INVALID_ARG;
  for (int j = 0; j < T; ++j) {
    const int it = cfg->types ? cfg->types[j] : SAE_TYPE_FLOAT, ot = cfg->result_types ? cfg->result_types[j] : it;
    if (cfg->rows[j] < 0 || cfg->cols[j] < 0 || cfg->rows[j] > (1 << 20) || cfg->cols[j] > (1 << 20) || cfg->rows[j] * cfg->cols[j] > (1ll << 30) ||
        !type_ok(it) || !type_ok(ot)) return SAE_ERR_INVALID_ARG;
  }
  // Where the singular values can get to decides how far x, S and B may be scaled up in float16.
  double s_scale[OT_STEPS], b_scale[OT_STEPS], top = 1.0, widest = 1.0;
  for (int i = 0; i < cfg->steps; ++i) {
    const float* k = cfg->coefficients + 3 * i;
    if (!std::isfinite(k[0]) || !std::isfinite(k[1]) || !std::isfinite(k[2])) return SAE_ERR_INVALID_ARG;
    double p, q;
    const double t = top * 1.01;                 // roundings
    bounds(k, t, p, q);
    if (!(p <= 16.0) || !(q <= 4096.0)) return SAE_ERR_INVALID_ARG;
    s_scale[i] = std::exp2(std::floor(std::log2(32768.0 / (t * t))));
    b_scale[i] = std::exp2(std::min(14.0, std::floor(std::log2(32768.0 / std::max(q, 1e-6)))));
    top = std::max(p, 1e-3);
    widest = std::max(widest, top * 1.01);
  }
  sae_ortho* h = new (std::nothrow) sae_ortho();
  if (!h) return SAE_ERR_NOMEM;
  h->K = K; h->T = T; h->device = cfg->device; h->stream = (cudaStream_t)cfg->stream; h->steps = cfg->steps; h->eps = cfg->eps;
  h->x_scale = std::exp2(std::floor(std::log2(32768.0 / widest)));
  std::vector<Maps> maps;
  std::vector<Shape> shapes;
  std::vector<Parts> parts;
  std::vector<int> count, order;
  std::vector<Place> places;
  std::vector<Chunk> chunks;
  std::vector<Batch> batches;
  DeviceGuard guard(cfg->device);
  cudaError_t e = guard.ok ? cudaSuccess : cudaGetLastError();
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, cfg->device);
  if (e == cudaSuccess) e = cudaMalloc((void**)&h->done, (size_t)K * T * sizeof(u32));
  if (e == cudaSuccess) e = cudaMalloc((void**)&h->ratios, (size_t)K * T * sizeof(float));
  bool mapped = true;
  if (e == cudaSuccess) {
    try {
      h->rows.assign(cfg->rows, cfg->rows + T);
      h->cols.assign(cfg->cols, cfg->cols + T);
      h->coef.assign(cfg->coefficients, cfg->coefficients + 3 * cfg->steps);
      h->s_scale.assign(s_scale, s_scale + cfg->steps); h->b_scale.assign(b_scale, b_scale + cfg->steps); h->ones.assign((size_t)cfg->steps, 1.0);
      for (int j = 0; j < T; ++j) {
        h->in_types.push_back(cfg->types ? cfg->types[j] : SAE_TYPE_FLOAT);
        h->out_types.push_back(cfg->result_types ? cfg->result_types[j] : h->in_types[j]);
      }
      // shapes: by parts (a class), then long sums before short ones
      std::map<std::tuple<int, int64_t, int64_t, int64_t, bool>, std::vector<int>> by;
      for (int k = 0; k < K; ++k)
        for (int j = 0; j < T; ++j)
          if (h->rows[j] && h->cols[j] && !small_rows(std::min(h->rows[j], h->cols[j]), std::max(h->rows[j], h->cols[j]))) {
            // bfloat16 results of a few rows or columns take both parts too: such products are short, and their roundings average out less
            const bool one = h->out_types[j] == SAE_TYPE_BFLOAT && std::min(h->rows[j], h->cols[j]) > 128;
            by[{one ? 1 : 2, -std::max(h->rows[j], h->cols[j]), h->rows[j], h->cols[j], one && h->in_types[j] != SAE_TYPE_FLOAT}].push_back(k * T + j);
          }
      places.resize((size_t)K * T);
      int64_t bytes = 0;
      for (auto& kv : by) {
        Shape g = {};
        g.s_parts = std::get<0>(kv.first);
        g.plain = std::get<4>(kv.first);
        g.rows = (int)std::get<2>(kv.first); g.cols = (int)std::get<3>(kv.first);
        g.tall = g.rows > g.cols;
        g.small = std::min(g.rows, g.cols);
        g.x_pitch = (int)up(g.cols, 64); g.s_pitch = (int)up(g.small, 64);
        g.x_plane = (long long)g.rows * g.x_pitch; g.s_plane = (long long)g.small * g.s_pitch;
        g.first = (int)order.size();
        for (int i : kv.second) order.push_back(i);
        count.push_back((int)kv.second.size());
        if (h->classes.empty() || h->classes.back().parts != g.s_parts) h->classes.push_back({g.s_parts, 1, 64, (int)shapes.size(), 0, 0, 0, 0, false});
        ++h->classes.back().n;
        shapes.push_back(g);
        bytes += 2 * up(2 * g.x_plane * count.back() * 2, 1024) + 2 * up(g.s_parts * g.s_plane * count.back() * 2, 1024);
      }
      for (int f = 0; f < 2; ++f) {
        h->small_first[f] = (int)order.size();
        // the longest first
        std::vector<std::pair<int64_t, int>> found;
        for (int k = 0; k < K; ++k)
          for (int j = 0; j < T; ++j)
            if (h->rows[j] && h->cols[j] && small_rows(std::min(h->rows[j], h->cols[j]), std::max(h->rows[j], h->cols[j])) == (f ? 128 : 64))
              found.push_back({-std::max(h->rows[j], h->cols[j]), k * T + j});
        std::sort(found.begin(), found.end());
        for (const auto& q : found) {
          const int j = q.second % T;
          Place& p = places[q.second];
          p.rows = (int)h->rows[j]; p.cols = (int)h->cols[j]; p.in_type = h->in_types[j]; p.out_type = h->out_types[j];
          order.push_back(q.second);
        }
        h->small_n[f] = (int)found.size();
      }
      if (bytes) e = cudaMalloc((void**)&h->arena, (size_t)bytes);
      if (e == cudaSuccess) {
        char* at = h->arena;
        maps.resize(shapes.size());
        for (size_t i = 0; i < shapes.size(); ++i) {
          Shape& g = shapes[i];
          const int n = count[i];
          const auto take = [&](int64_t elements) { __half* p = (__half*)at; at += up(elements * 2, 1024); return p; };
          for (int q = 0; q < 2; ++q) {
            g.x[q] = take(2 * g.x_plane * n);
            mapped = mapped && mma::encode_map(&maps[i].x[q], g.x[q], false, g.cols, g.rows, 2ll * n, g.x_pitch, g.x_plane);
          }
          g.s = take(g.s_parts * g.s_plane * n);
          g.b = take(g.s_parts * g.s_plane * n);
          mapped = mapped && mma::encode_map(&maps[i].s, g.s, false, g.small, g.small, (int64_t)g.s_parts * n, g.s_pitch, g.s_plane);
          mapped = mapped && mma::encode_map(&maps[i].b, g.b, false, g.small, g.small, (int64_t)g.s_parts * n, g.s_pitch, g.s_plane);
          for (int q = 0; q < n; ++q) {
            const int i2 = order[g.first + q], j = i2 % T;
            Place& p = places[i2];
            p.rows = g.rows; p.cols = g.cols; p.x_pitch = g.x_pitch; p.in_type = h->in_types[j]; p.out_type = h->out_types[j];
            p.x = g.x[0] + (long long)q * 2 * g.x_plane; p.x_plane = g.x_plane;
            p.done = h->done + g.first + q; p.ratio = h->ratios + g.first + q; p.plain = g.plain;
            p.first_chunk = (int)chunks.size();
            const int64_t units = (int64_t)g.rows * ((g.cols + UNIT - 1) / UNIT);
            for (int64_t u = 0; u < units; u += OT_CHUNK) chunks.push_back({i2, (int)u});
            p.chunks = (int)chunks.size() - p.first_chunk;
          }
        }
        parts.resize(shapes.size());
        int64_t split_sums = 0, arrived = 0;
        const auto sums_size = [&](const Class& c, int i) { return parts[i].n > 1 ? (int64_t)count[i] * shapes[i].s_tiles * parts[i].n * 128 * c.cg * c.cols : 0; };
        for (Class& c : h->classes) {
          choose_tiles(c, shapes, parts, count, h->num_sms);
          list_products(c, shapes, parts, count, cfg->steps, batches);
          for (int i = c.first; i < c.first + c.n; ++i) {
            split_sums += sums_size(c, i);
            c.split = c.split || parts[i].n > 1;
            if (parts[i].n > 1) arrived += (int64_t)count[i] * shapes[i].s_tiles * 16;
          }
        }
        if (split_sums) {
          e = cudaMalloc((void**)&h->split_sums, (size_t)split_sums * sizeof(float));
          if (e == cudaSuccess) e = cudaMalloc((void**)&h->arrived, (size_t)arrived * sizeof(u32));
          float* sums_at = h->split_sums;
          u32* arrived_at = h->arrived;
          for (const Class& c : h->classes)
            for (int i = c.first; i < c.first + c.n && e == cudaSuccess; ++i) {
              const Shape& g = shapes[i];
              if (parts[i].n == 1) continue;
              parts[i].sums = sums_at;
              parts[i].arrived = arrived_at;
              for (int q = 0; q < count[i]; ++q) {
                Place& p = places[order[g.first + q]];
                p.arrived = arrived_at + (int64_t)q * g.s_tiles * 16;
                p.num_arrived = g.s_tiles * 16;
              }
              sums_at += sums_size(c, i);
              arrived_at += (int64_t)count[i] * g.s_tiles * 16;
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
  if (e == cudaSuccess) e = upload(&h->maps, maps, h->stream);
  if (e == cudaSuccess) e = upload(&h->shapes, shapes, h->stream);
  if (e == cudaSuccess) e = upload(&h->parts, parts, h->stream);
  if (e == cudaSuccess) e = upload(&h->batches, batches, h->stream);
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
  if (!h->chunks && !h->small_n[0] && !h->small_n[1]) return SAE_OK;
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
  static thread_local SmallJob one;
  one.mats = h->mats; one.places = h->places; one.steps = h->steps; one.eps = h->eps; one.scale = h->x_scale;
  factors(h, h->b_scale, one.factors);
  for (int f = 0; f < 2 && e == cudaSuccess; ++f) {
    one.order = h->order + h->small_first[f];
    if (h->small_n[f]) e = f ? launch_small<128>(one, h->small_n[f], h->stream) : launch_small<64>(one, h->small_n[f], h->stream);
  }
  if (h->chunks && e == cudaSuccess)
    e = launch(k_ortho_norm, h->chunks, h->stream, first, (const Matrix*)h->mats, (const Place*)h->places, (const Chunk*)h->chunk_list, h->sums);
  if (h->chunks && e == cudaSuccess)
    e = launch(k_ortho_split, h->chunks, h->stream, false, (const Matrix*)h->mats, (const Place*)h->places, (const Chunk*)h->chunk_list, (const double*)h->sums, h->eps, h->x_scale);
  for (const Class& c : h->classes)
    if (e == cudaSuccess) e = c.split ? launch_class<true>(h, c) : launch_class<false>(h, c);
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
