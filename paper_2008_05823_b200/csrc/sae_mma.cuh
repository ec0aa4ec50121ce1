// Products of 16-bit matrices on the tensor cores (tcgen05), shared by the operators whose work is one: a persistent kernel
// that walks over output tiles, with the operator's own arithmetic at the end of each tile.
//
//   acc[i][j] = sum over segments (pa, pb), over k:  A_pa[i][k] * B_pb[j][k]          (float accumulators in tensor memory)
//
// A matrix of 16-bit elements is one part.  A matrix of more exact values is a sum of parts (planes of its tensor map), and
// the segments are the products of parts that matter: 22 bits as two float16 parts and 3 segments, a float as three
// bfloat16 parts and 6 segments.  Segments come smallest first, so that the sum is short of bits only in its last ones.
//
// Tile: 128 * CG rows by 64, 128 or 256 columns.  CG = 2: the two thread blocks of a cluster share one tile; each loads its 128 rows of
// A and its half of B, the tensor cores of both read both halves, so a byte that comes from L2 is used twice as often.
// Warps 0 and 3 load (TMA, boxes of 64 x 64 elements in 128-byte swizzled rows, a ring of 32 KB stages; warp 0 A, warp 3 B), warp 1 issues the
// products (one thread; in block 0 of a pair), warps 4 and up take the sums: warp w the lanes 32 (w % 4) .. + 31, which are
// the tile's rows, and one half of the columns.  Sums are held twice (2 x 256 columns of the 512), so the products
// of the next tile run while a tile is taken out.
//
// The tensor cores cut off what a sum has below its last bit, at each of the products that it is made of, and a sum of a few
// thousand terms of one sign ends up short by some 1e-5.  For operands of several parts the sums are therefore taken out every
// 64 of k, rounded to nearest where they are joined (in the 128 columns that tiles of up to 128 columns leave free); for operands of one part
// where sums are long.
//
// Operands lie in memory either way: k neighbouring ("K first", what x w' wants of x and w) or the rows neighbouring ("rows
// first", what p' x wants); the matrix descriptors say which, nothing is transposed.
//
// Every wait is bounded in time.  A role that gives up marks the block as dead, the other roles of it then give up too, and all that
// the block had yet to write becomes NaN, which reaches the results.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "sae_device.cuh"
#include "sae_vec.cuh"

namespace sae {
namespace mma {

constexpr int BLOCK_K = 64;
constexpr int BOX_ROWS = 64;
constexpr u32 BOX_BYTES = BLOCK_K * BOX_ROWS * 2;
constexpr u32 STAGE_BYTES = 4 * BOX_BYTES;      // 128 rows of A, up to 128 of B
constexpr int EPI_WARP = 4, EPI_WARPS = 8;
constexpr int MAX_STAGES = 6;
// 8 warps take the sums out (16 were no faster).  A job that brings values in by copies has STAGING bytes for each of them, at the cost of stages.
template <class Job>
struct Room {
  static constexpr int STAGES = (int)((227 * 1024 - 1024 - sizeof(typename Job::Shared) - 512 - EPI_WARPS * Job::STAGING) / STAGE_BYTES) < MAX_STAGES
                                    ? (int)((227 * 1024 - 1024 - sizeof(typename Job::Shared) - 512 - EPI_WARPS * Job::STAGING) / STAGE_BYTES) : MAX_STAGES;
  static constexpr int THREADS = 32 * (EPI_WARP + EPI_WARPS + Job::REPORTS);
  static constexpr u32 BYTES = STAGES * STAGE_BYTES + EPI_WARPS * Job::STAGING + 1024;
};
constexpr u32 TMEM_COLUMNS = 512;
constexpr u64 WAIT_NS = 2000000000ull, DRAIN_NS = 100000000ull;
constexpr int MAX_SEGMENTS = 6;
// Blocks of k after which sums are taken out and joined, rounded to nearest: sums of several parts, and long sums of one.  The tensor
// cores truncate a sum at every 16 k: by 4e-6 of a loss at 4096 features.  2048 x 4096 x 32000, joined every 512, 768 or 1024 k: the rows' losses off by
// 1.1e-7, 1.6e-7, 2.2e-7; loss 464, 450, 434 us (418 unjoined), gradients 1136, 1115, 1103 (1080); the
// plain form in float32 7e-7 at 2048 features.  Every 1024: a join waits 1000 cycles for a sum of 16 blocks, which takes 9400.
// A sum of terms of one sign is short by 6e-9 for each of its terms (65536 of them: 4e-4): sums that end in 16 bits are joined where they would lose more than a
// tenth of the type's smallest half step.
constexpr int JOIN_PARTS = 1, JOIN_LONG = 16, JOIN_HALF = 4096 / BLOCK_K, JOIN_BFLOAT = 32768 / BLOCK_K;

struct Segments {
  int n;
  unsigned char a[MAX_SEGMENTS], b[MAX_SEGMENTS];
};

// One output tile.
struct Tile {
  const CUtensorMap *a, *b;
  int a_row, b_row;        // first row of A (tile row) and of B (tile column)
  int a_plane, b_plane;    // planes of part 0
  int a_k, b_k, blocks;    // first k in A and in B, blocks of 64 of them (0: all sums are zero)
  bool a_rows_first, b_rows_first;
  int a_turn, b_turn;      // this many first blocks of k come from the transpose instead: (row, k) from (k, row), the other of K and rows first
  // for the epilogue
  int row, col;            // first output row and column
  int group, item, part;
};

// Where a tile's sums are: in tensor memory, there in two places to be added, all zero, or lost.
enum State { SUMS_HELD, SUMS_JOINED, SUMS_ZERO, SUMS_NAN };
struct Sums {
  State state;
  u32 at, held;            // this warp's lanes of the tile's first column
};

struct Control {
  u64 full[MAX_STAGES], empty[MAX_STAGES], acc_full[2], acc_empty[2], drain;
  u32 tmem, dead;
  u32 ready, stored[EPI_WARPS];       // tiles whose operands were found ready; tiles that each epilogue warp has written
};

// ---- PTX --------------------------------------------------------------------------------------------------------------
static __device__ __noinline__ bool wait_slow(u32 addr, u32 parity, volatile u32* dead, u64 limit_ns) {
  const u64 t0 = global_ns();
  for (;;) {
    if (mbar_try(addr, parity)) return true;
    if (dead && *dead) return false;
    if (global_ns() - t0 > limit_ns) { if (dead) *dead = 1; return false; }
  }
}
__device__ __forceinline__ bool wait(u64* bar, u32 parity, u32* dead) {
  const u32 addr = smem_u32(bar);
  if (mbar_try(addr, parity)) return true;
  return wait_slow(addr, parity, dead, WAIT_NS);
}
// Waits until a counter that other blocks of the grid add to has reached a value.  (Polled by relaxed loads, one fence at the end: an
// acquiring load throws L1 away each time and holds up the loads and stores of the whole SM.)
__device__ __forceinline__ bool counter_reached(const u32* counter, u32 least) {
  u32 v;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
  return (int)(v - least) >= 0;
}
static __device__ __noinline__ bool wait_counter(const u32* counter, u32 least, volatile u32* dead) {
  const u64 t0 = global_ns();
  while (!counter_reached(counter, least)) {
    __nanosleep(64);
    if (*dead) return false;
    if (global_ns() - t0 > WAIT_NS) { *dead = 1; return false; }
  }
  asm volatile("fence.acq_rel.gpu;" ::: "memory");
  return true;
}
__device__ __forceinline__ void add_counter(u32* counter) { asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory"); }
// The same within a block.
__device__ __forceinline__ void set_shared(u32* to, u32 v) { asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(smem_u32(to)), "r"(v) : "memory"); }
__device__ __forceinline__ bool shared_reached(u32* at, u32 least) {
  u32 v;
  asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(v) : "r"(smem_u32(at)) : "memory");
  return (int)(v - least) >= 0;
}
static __device__ __noinline__ bool wait_shared_slow(u32* at, u32 least, volatile u32* dead) {
  const u64 t0 = global_ns();
  for (;;) {
    for (int i = 0; i < 16; ++i) {
      if (shared_reached(at, least)) return true;
      __nanosleep(40);
    }
    if (*dead) return false;
    if (global_ns() - t0 > WAIT_NS) { *dead = 1; return false; }
  }
}
__device__ __forceinline__ bool wait_shared(u32* at, u32 least, u32* dead) { return shared_reached(at, least) || wait_shared_slow(at, least, dead); }
// Between plain accesses and TMA's: whoever wrote, and whoever is going to load.
__device__ __forceinline__ void fence_copies() { asm volatile("fence.proxy.async;" ::: "memory"); }

// One lane of a warp whose lanes run together.  The roles that issue copies and products are whole warps with this around what
// one thread does: a loop that only one lane runs has its operands moved one by one to the registers these instructions take
// (890 cycles for the four products of a stage, of which the tensor cores need 512).
__device__ __forceinline__ bool one_lane() {
  u32 r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ u32 of_block0(u32 addr) {      // the address of block 0's copy of a shared variable
  u32 r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
// (Relaxed: what it orders is tensor memory, read before; a release would first wait for the thread's stores to memory.)
__device__ __forceinline__ void arrive_cluster(u32 addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ u32 cluster_rank() {
  u32 r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
template <int CG>
__device__ __forceinline__ void load_box(u32 to, const CUtensorMap* map, int x, int y, int z, u32 bar) {
  if constexpr (CG == 1)
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc(u32* to) {
  if constexpr (CG == 1) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n\ttcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::"r"(smem_u32(to)), "n"(TMEM_COLUMNS) : "memory");
  else asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n\ttcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(smem_u32(to)), "n"(TMEM_COLUMNS) : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_free(u32 addr) {
  if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(TMEM_COLUMNS) : "memory");
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(TMEM_COLUMNS) : "memory");
}
template <int CG>
__device__ __forceinline__ void product(u32 tmem, u64 a, u64 b, u32 idesc, u32 add) {
  if constexpr (CG == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// The barrier (of both blocks of a pair) gets an arrival when all products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(u64* bar) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of this warp's 32 lanes: thread = lane (a row), register = column.
__device__ __forceinline__ void tmem_load(u32 addr, float (&v)[32]) {
  u32* r = reinterpret_cast<u32*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_store(u32 addr, const float (&v)[32]) {
  const u32* r = reinterpret_cast<const u32*>(v);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
      "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
      : "memory");
}
// What a kernel started early (programmatic launch) does before it touches what the one before it writes.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- descriptors --------------------------------------------------------------------------------------------------------
// 128-byte swizzled rows.  K first: 8 rows of 128 bytes (64 k) are one kilobyte, groups of 8 rows follow one another.  Rows
// first: 64 rows of the matrix are the 128 bytes, 8 k are one kilobyte, and the next 64 rows are `next` bytes on.
__device__ __forceinline__ u64 smem_desc(u32 addr, bool rows_first, u32 next = BOX_BYTES) {
  const u64 lead = rows_first ? next >> 4 : 1, stride = 1024 >> 4;
  return (u64)((addr >> 4) & 0x3fff) | lead << 16 | stride << 32 | 1ull << 46 | 2ull << 61;
}
constexpr u32 FLOAT_SUMS = 1u << 4, BFLOAT_OPERANDS = 1u << 7 | 1u << 10;
__device__ __forceinline__ u32 instruction(int rows, int cols, bool bfloat, bool a_rows_first, bool b_rows_first) {
  return FLOAT_SUMS | (bfloat ? BFLOAT_OPERANDS : 0u) | (u32)a_rows_first << 15 | (u32)b_rows_first << 16 | (u32)(cols >> 3) << 17 | (u32)(rows >> 4) << 24;
}

// 32 sums of a row, from column c of the tile on, whatever state they are in.
__device__ __forceinline__ void sums_of(const Sums& s, int c, float (&v)[32]) {
  if (s.state <= SUMS_JOINED) {
    tmem_load(s.at + (u32)c, v);
    if (s.state == SUMS_JOINED) {
      float w[32];
      tmem_load(s.held + (u32)c, w);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] += w[i];
    }
  } else {
    const float fill = s.state == SUMS_ZERO ? 0.0f : __int_as_float(0x7fc00000);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = fill;
  }
}

// The columns of a tile that an epilogue warp takes.
__device__ __forceinline__ int epilogue_width(int cols) { return cols / 2; }

// ---- the kernel -----------------------------------------------------------------------------------------------------------
// Job: int cols; bool bfloat; Segments seg;
//      Shared, fill(shared): what the roles look up, in shared memory
//      Local begin(shared, cluster, clusters): a role's place in the list of tiles;  bool tile(local, i, Tile&): this cluster's i-th
//      tile, asked for in order
//      Epilogue(job, local, row of the tile, which part of the columns, the warp's staging): prepare(t, number, control), while the sums are
//      made;  tile(t, sums);  finish(), behind the last tile
//      REPORTS: tiles depend on one another.  A warp of its own, the last, runs ahead with ready(local, t, dead), which waits until a tile's
//      operands are there (false: gave up); report(local, t) is called by warp 2 when the block has written its part of a
//      tile.  Both wait a microsecond or two for the memory; with the loading warps waiting themselves, 12 encoder layers took 1702 us, not 1601.
//      LONG: sums of one part may be joined: after `run` blocks of k, in this call (joins(), on the host) and this kernel (joined(local): false only where
//      none is longer)
// JOIN: how sums are taken out and held on the way: not (0), after each block (1, sums of parts), after `run` blocks (2).  Up to 128 columns there is room for two sums beside the held ones;
// of 256 columns there is one, taken out for good before the next tile's first block of k, and the epilogue reads the held ones.
template <class Job, int CG, int JOIN>
__global__ void __launch_bounds__(Room<Job>::THREADS, 1) k_products(const __grid_constant__ Job job) {
  constexpr int STAGES = Room<Job>::STAGES;
  extern __shared__ unsigned char smem_raw[];
  __shared__ Control ctl;
  __shared__ typename Job::Shared shared;
  const u32 tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const u32 rank = CG == 2 ? cluster_rank() : 0;
  const int cluster = blockIdx.x / CG, clusters = gridDim.x / CG;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&ctl.full[i], 1); mbar_init(&ctl.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&ctl.acc_full[i], 1); mbar_init(&ctl.acc_empty[i], EPI_WARPS * CG); }
    mbar_init(&ctl.drain, 1);
    ctl.dead = ctl.ready = 0;
    for (int i = 0; i < EPI_WARPS; ++i) ctl.stored[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  job.fill(shared);
  if (warp == 2) tmem_alloc<CG>(&ctl.tmem);
  fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync();
  fence_after();
  let_next_start();
  wait_for_previous();
  const u32 tmem = ctl.tmem;
  typename Job::Local local = job.begin(shared, cluster, clusters);
  const int b_rows = job.cols / CG;               // rows of B that a block loads
  bool single = false;
  if constexpr (JOIN > 1) single = job.cols > 128 && job.joined(local);
  const u32 buffers = single ? 0 : 1;             // (a mask)
  int length = JOIN;                              // blocks of k of a sum
  if constexpr (JOIN > 1) length = job.run;

  if (warp == 0 || warp == 3) {
    const u32 bytes = CG * (2 * BOX_BYTES + (u32)b_rows * BLOCK_K * 2);
    u32 n = 0;
    Tile t;
    bool ok = true;
    for (int i = 0; ok && job.tile(local, i, t); ++i) {
      if constexpr (Job::REPORTS) {
        if (!__all_sync(0xffffffffu, wait_shared(&ctl.ready, (u32)i + 1, &ctl.dead))) { ok = false; break; }
      }
      const int a_row = t.a_row + (int)rank * 128, b_row = t.b_row + (int)rank * b_rows, run = JOIN ? length : t.blocks;
      for (int k0 = 0; k0 < t.blocks && ok; k0 += run) {
        const int k1 = JOIN ? min(k0 + run, t.blocks) : t.blocks;
        for (int s = 0; s < job.seg.n && ok; ++s) {
          const int za = t.a_plane + job.seg.a[s], zb = t.b_plane + job.seg.b[s];
          for (int kb = k0; kb < k1; ++kb, ++n) {
            const u32 stage = n % STAGES;
            if (!__all_sync(0xffffffffu, wait(&ctl.empty[stage], ((n / STAGES) & 1) ^ 1, &ctl.dead))) { ok = false; break; }
            const u32 at = tiles + stage * STAGE_BYTES;
            u32 bar = smem_u32(&ctl.full[stage]);
            if constexpr (CG == 2) bar = of_block0(bar);
            const int ka = t.a_k + kb * BLOCK_K, kw = t.b_k + kb * BLOCK_K;
            const bool a_rows_first = t.a_rows_first != (kb < t.a_turn), b_rows_first = t.b_rows_first != (kb < t.b_turn);
            if (one_lane()) {
              if (warp == 0) {
                if (rank == 0) mbar_arrive_expect_tx(&ctl.full[stage], bytes);
#pragma unroll
                for (int r = 0; r < 128; r += BOX_ROWS)
                  load_box<CG>(at + r * BLOCK_K * 2, t.a, a_rows_first ? a_row + r : ka, a_rows_first ? ka : a_row + r, za, bar);
              } else {
#pragma unroll
                for (int r = 0; r < 128; r += BOX_ROWS)
                  if (r < b_rows)
                    load_box<CG>(at + 2 * BOX_BYTES + r * BLOCK_K * 2, t.b, b_rows_first ? b_row + r : kw, b_rows_first ? kw : b_row + r, zb, bar);
              }
            }
            __syncwarp();
          }
        }
      }
    }
    if (!ok && rank == 0 && warp == 0)             // copies in flight land before the block ends
      for (u32 m = n > STAGES ? n - STAGES : 0; m < n; ++m) wait_slow(smem_u32(&ctl.full[m % STAGES]), (m / STAGES) & 1, nullptr, DRAIN_NS);
  } else if (warp == 1 && rank == 0) {
    u32 n = 0, taken = 0;
    Tile t;
    bool ok = true;
    for (int i = 0; ok && job.tile(local, i, t); ++i) {
      int left = t.blocks;
      do {
        const int blocks = JOIN ? min(left, length) : left;
        const u32 buf = taken & buffers;
        if (!__all_sync(0xffffffffu, wait(&ctl.acc_empty[buf], ((taken >> buffers) & 1) ^ 1, &ctl.dead))) { ok = false; break; }
        fence_after();
        const u32 acc = tmem + buf * 256;
        u32 add = 0;
        const int k0 = t.blocks - left;
        for (int j = 0; j < job.seg.n * blocks; ++j, ++n) {
          const u32 stage = n % STAGES;
          if (!__all_sync(0xffffffffu, wait(&ctl.full[stage], (n / STAGES) & 1, &ctl.dead))) { ok = false; break; }
          fence_after();
          const u32 at = tiles + stage * STAGE_BYTES;
          const int kb = k0 + (JOIN == 1 ? 0 : j);        // (JOIN 1: the segments of one block; otherwise there is one segment)
          const bool a_rows_first = t.a_rows_first != (kb < t.a_turn), b_rows_first = t.b_rows_first != (kb < t.b_turn);
          const u32 idesc = instruction(128 * CG, job.cols, job.bfloat, a_rows_first, b_rows_first);
          const u32 a_step = (a_rows_first ? 2048 : 32) >> 4, b_step = (b_rows_first ? 2048 : 32) >> 4;
          const u64 a = smem_desc(at, a_rows_first), b = smem_desc(at + 2 * BOX_BYTES, b_rows_first);
          if (one_lane()) {
#pragma unroll
            for (u32 k = 0; k < BLOCK_K / 16; ++k) product<CG>(acc, a + k * a_step, b + k * b_step, idesc, k ? 1 : add);
            commit<CG>(&ctl.empty[stage]);
          }
          __syncwarp();
          add = 1;
        }
        if (!ok) break;
        if (one_lane()) commit<CG>(&ctl.acc_full[buf]);
        __syncwarp();
        ++taken;
        left -= blocks;
      } while (left > 0);
    }
    if (*(volatile u32*)&ctl.dead) {               // products in flight end before the tensor memory is given back
      if (one_lane()) asm volatile("tcgen05.commit.cta_group::%1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&ctl.drain)), "n"(CG) : "memory");
      wait_slow(smem_u32(&ctl.drain), 0, nullptr, DRAIN_NS);
    }
  } else if (Job::REPORTS && warp == 2) {
    Tile t;
    for (int i = 0; job.tile(local, i, t); ++i) {
      if (!__all_sync(0xffffffffu, wait_shared(&ctl.stored[lane % EPI_WARPS], (u32)i + 1, &ctl.dead))) break;
      if constexpr (Job::REPORTS) if (one_lane()) job.report(local, t);
      __syncwarp();
    }
  } else if (Job::REPORTS && warp == EPI_WARP + EPI_WARPS) {
    Tile t;
    for (int i = 0; job.tile(local, i, t); ++i) {
      bool there = true;
      if constexpr (Job::REPORTS) if (lane == 0) there = job.ready(local, t, &ctl.dead);
      if (!__shfl_sync(0xffffffffu, there, 0)) break;
      if (lane == 0) set_shared(&ctl.ready, (u32)i + 1);
      __syncwarp();
    }
  } else if (warp >= EPI_WARP) {
    const int quarter = warp & 3, part = (warp - EPI_WARP) >> 2;
    typename Job::Epilogue epi(job, local, (int)rank * 128 + quarter * 32 + lane, part, tiles + STAGES * STAGE_BYTES + (warp - EPI_WARP) * Job::STAGING);
    Tile t;
    bool ok = true;
    u32 taken = 0;
    const u32 lanes = tmem + ((u32)quarter * 32 << 16);
    for (int i = 0; job.tile(local, i, t); ++i) {
      epi.prepare(t, i, &ctl);
      int left = t.blocks;
      bool first = true;
      for (;;) {
        const u32 buf = taken & buffers;
        if (ok && !wait(&ctl.acc_full[buf], (taken >> buffers) & 1, &ctl.dead)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        fence_after();
        const bool last = !JOIN || left <= length || !ok;
        const u32 held = lanes + (single ? 256 : 384);
        Sums s = {!ok ? SUMS_NAN : job.seg.n * t.blocks == 0 ? SUMS_ZERO : first ? SUMS_HELD : SUMS_JOINED, lanes + buf * 256, held};
        const bool join = JOIN && s.state <= SUMS_JOINED && (single || !last);
        if constexpr (JOIN > 0) {
          if (join) {
            const int width = epilogue_width(job.cols);
            for (int c = part * width; c < (part + 1) * width; c += 32) {
              float v[32];
              sums_of(s, c, v);
              tmem_store(s.held + (u32)c, v);
            }
          }
        }
        if (last && !join) epi.tile(t, s);
        fence_before();
        __syncwarp();
        if (lane == 0 && ok) {
          const u32 bar = smem_u32(&ctl.acc_empty[buf]);
          if constexpr (CG == 2) arrive_cluster(of_block0(bar));
          else mbar_arrive(&ctl.acc_empty[buf]);
        }
        if (JOIN > 1 && last && join) epi.tile(t, {SUMS_HELD, held, held});
        if constexpr (Job::REPORTS) {
          if (last) {
            __syncwarp();
            if (lane == 0) set_shared(&ctl.stored[warp - EPI_WARP], (u32)i + 1);
          }
        }
        ++taken;
        if (last) break;
        first = false;
        left -= length;
      }
    }
    epi.finish();
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync();
  fence_after();
  if (warp == 2) tmem_free<CG>(tmem);
}

__device__ __forceinline__ u32 pack_half(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const u32*>(&v);
}
__device__ __forceinline__ u32 pack_bfloat(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const u32*>(&v);
}
// 16 words (32 elements of 16 bits), 32-byte aligned: whole sectors.
__device__ __forceinline__ void store_words(void* to, const u32 (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"((char*)to + i * 4), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                 : "memory");
}
__device__ __forceinline__ void load_words(const void* from, u32 (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7]) : "l"((const char*)from + i * 4)
                 : "memory");
}
// The same past L1, which does not see what other SMs have written during the kernel.
__device__ __forceinline__ void load_written(const void* from, u32 (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("ld.relaxed.gpu.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7]) : "l"((const char*)from + i * 4)
                 : "memory");
}
// Rows of 16 pieces of 16 bytes in shared memory.  Pieces change places with the row, so that a lane that takes pieces of its own row and
// lanes that take the pieces of one row both meet different banks.
__device__ __forceinline__ u32 staged_at(u32 base, int r, int piece) { return base + (u32)(r * 16 + (piece ^ (r & 7))) * 16; }
__device__ __forceinline__ uint4 staged_piece(u32 at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void staged_load(u32 base, int r, int piece, u32 (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = staged_piece(staged_at(base, r, piece + i));
    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
  }
}
// 16 bytes to shared memory, past L1 (which does not see what other SMs write).
__device__ __forceinline__ void piece_in(u32 to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void pieces_arrived() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ float2 unpack_half(u32 w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// `n` <= 32 values of a row, rounded to a type, to any aligned address.
template <typename T>
__device__ __forceinline__ void store_row(T* to, const float (&v)[32], int n) {
  if (n == 32 && (reinterpret_cast<uintptr_t>(to) & 31) == 0) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32 w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[h * 16 + i]);
        store_words(to + h * 16, w);
      }
    } else {
      u32 w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = sizeof(T) == 2 && std::is_same<T, __half>::value ? pack_half(v[2 * i], v[2 * i + 1]) : pack_bfloat(v[2 * i], v[2 * i + 1]);
      store_words(to, w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 4) to[i] = v[i];
        else if constexpr (std::is_same<T, __half>::value) to[i] = __float2half_rn(v[i]);
        else to[i] = __float2bfloat16_rn(v[i]);
      }
  }
}

// A warp's 32 x 32 values to a matrix whose rows start anywhere: through shared memory (`at`, 32 rows of 33 words), so that a store
// covers a row's neighbouring columns.  rows, cols: how many of each there are.
template <typename T>
__device__ __forceinline__ void store_square(T* to, int64_t pitch, const float (&v)[32], int rows, int cols, u32 at) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + (u32)(lane * 33 + i) * 4), "f"(v[i]) : "memory");
  __syncwarp();
#pragma unroll 8
  for (int r = 0; r < rows; ++r) {
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at + (u32)(r * 33 + lane) * 4) : "memory");
    if (lane < cols) to[r * pitch + lane] = from_f<T>(x);
  }
  __syncwarp();
}
constexpr int SQUARE_BYTES = 32 * 33 * 4;

// ---- host -------------------------------------------------------------------------------------------------------------------
// A map of `planes` matrices of `rows` rows of `inner` 16-bit elements; pitches in elements, multiples of 8.
inline bool encode_map(CUtensorMap* map, const void* base, bool bfloat, int64_t inner, int64_t rows, int64_t planes, int64_t row_pitch, int64_t plane_pitch) {
  static const PFN_cuTensorMapEncodeTiled encode = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
    return (PFN_cuTensorMapEncodeTiled)p;
  }();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)row_pitch * 2, (cuuint64_t)plane_pitch * 2};
  const cuuint32_t box[3] = {BLOCK_K, BOX_ROWS, 1}, step[3] = {1, 1, 1};
  return encode(map, bfloat ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Job, int CG, int JOIN>
cudaError_t launch_products(const Job& job, int blocks, cudaStream_t st, bool together) {
  // the attribute belongs to a device's context: set once for each
  static std::atomic<unsigned long long> ready{0};
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(k_products<Job, CG, JOIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Room<Job>::BYTES);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(Room<Job>::THREADS);
  cfg.dynamicSmemBytes = Room<Job>::BYTES;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (CG == 2) { at[n].id = cudaLaunchAttributeClusterDimension; at[n].val.clusterDim.x = 2; at[n].val.clusterDim.y = 1; at[n].val.clusterDim.z = 1; ++n; }
  if (together) { at[n].id = cudaLaunchAttributeCooperative; at[n].val.cooperative = 1; ++n; }
  else { at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[n].val.programmaticStreamSerializationAllowed = 1; ++n; }
  cfg.attrs = at;
  cfg.numAttrs = (unsigned)n;
  return cudaLaunchKernelEx(&cfg, k_products<Job, CG, JOIN>, job);
}

// together: blocks wait for one another, so all of them have to run at once.  Otherwise the kernel may start while the one before it
// still runs.  Sums of several parts are joined on the way.
template <class Job>
cudaError_t launch_products(const Job& job, int cg, int tiles_at_once, cudaStream_t st, bool together = false) {
  const auto with = [&](auto join) {
    return cg == 2 ? launch_products<Job, 2, decltype(join)::value>(job, 2 * tiles_at_once, st, together) : launch_products<Job, 1, decltype(join)::value>(job, tiles_at_once, st, together);
  };
  if (job.seg.n > 1) return with(std::integral_constant<int, JOIN_PARTS>());
  if constexpr (Job::LONG)
    if (job.joins()) return with(std::integral_constant<int, 2>());
  return with(std::integral_constant<int, 0>());
}

// For jobs whose operands are there before the kernel runs, and that look up nothing.
struct Plain {
  static constexpr int STAGING = 0;
  static constexpr bool REPORTS = false, LONG = true;
  struct Shared {};
  __device__ __forceinline__ void fill(Shared&) const {}
  template <class Local> __device__ __forceinline__ bool joined(const Local&) const { return true; }
};

}  // namespace mma
}  // namespace sae
