// Group norm with an activation, channels last, forward and backward.  Declarations and contract: include/sae.h.
//
// x is [N][P][C] (P pixels, the channels of a pixel neighbours in memory); group j is the Cg channels from j * Cg on, over
// all P pixels of a sample, M = P * Cg values:
//   mean = sum x / M,  var = sum (x - mean)^2 / M,  rstd = 1 / sqrt(var + eps)
//   xhat = (x - mean) * rstd,  z = xhat * w_c + b_c (+ residual),  y = act(z)
//   dz = dy * act'(z),  db_c = sum dz,  dw_c = sum dz * xhat,  g = dz * w_c,
//   dx = rstd * (g - mean_group(g) - xhat * mean_group(g * xhat))
// z is computed by the same separately rounded operations in both directions, so that relu's mask in the backward pass is
// the forward pass's own.
//
// Everything is bound by HBM.  A group of neighbouring channels is a column of short runs, so a thread takes 16 bytes of a
// pixel, always the same channels, and walks down the pixels; the threads of a block stand side by side over the channels
// first, which makes a block's loads whole lines whatever the group size is.
#include "../../include/sae.h"
#include "sae_gn_stream.cuh"
#include "sae_gn_unit.cuh"

#include <algorithm>
#include <atomic>

using namespace sae;

namespace {

// ---- host -----------------------------------------------------------------------------------------------------------
struct Plan {
  int vec;
  bool unit;                             // one pass: `u`, `threads` and `smem`; else two: `s` and `portion`
  Unit u;
  int threads;
  size_t smem;
  Stream s;
  int portion;                           // samples a launch takes
  size_t bytes;                          // workspace
};

int elem(int type) { return type == SAE_TYPE_FLOAT ? 4 : 2; }
bool type_ok(int t) { return t == SAE_TYPE_FLOAT || t == SAE_TYPE_BFLOAT || t == SAE_TYPE_HALF; }

bool desc_ok(const sae_group_norm_desc* d) {
  if (!d || !type_ok(d->type) || !type_ok(d->param_type) || d->activation < SAE_ACT_NONE || d->activation > SAE_ACT_GELU) return false;
  if (d->samples < 0 || d->samples > (1 << 24) || d->pixels < 0 || d->pixels > (1ll << 30) || d->channels < 1 || d->channels > (1 << 20)) return false;
  if (d->groups < 1 || d->channels % d->groups || !(d->eps >= 0.0f) || d->samples * d->groups > 0x7fffffffll) return false;
  const long long s[6] = {d->x_sample, d->x_pixel, d->residual_sample, d->residual_pixel, d->dy_sample, d->dy_pixel};
  for (long long v : s) if (v < 0) return false;
  return true;
}

// Elements a thread takes at a time, and, where that is less than 16 bytes, the wider vector that rows of several pixels allow.
struct Width { int vec, row_vec; };

int common(long long a, long long b) { while (b) { const long long t = a % b; a = b; b = t; } return (int)a; }
int row_pixels(const sae_group_norm_desc* d, int vec) { return vec / common(d->channels, vec); }

// Sixteen bytes where every tensor of the call lets it (base, strides and the channel count), else four, else one element.
Width vector_width(const sae_group_norm_desc* d, const void* const* ptrs, int n, bool residual, bool dy) {
  const int es = elem(d->type), most = 16 / es;
  uintptr_t base = 0;
  for (int i = 0; i < n; ++i) base |= reinterpret_cast<uintptr_t>(ptrs[i]);
  const long long samples = d->x_sample | d->residual_sample | d->dy_sample;
  const uintptr_t m = base | (uintptr_t)((samples | d->x_pixel | d->residual_pixel | d->dy_pixel | d->channels) * es);
  Width w = {(m & 15) == 0 ? most : es == 2 && (m & 3) == 0 ? 2 : 1, 0};
  const bool gapless = d->x_pixel == d->channels && (!residual || d->residual_pixel == d->channels) && (!dy || d->dy_pixel == d->channels);
  if (w.vec < most && gapless && (base & 15) == 0 && samples % most == 0) w.row_vec = most;
  return w;
}

constexpr int SMEM_MOST = 113 * 1024;     // no kernel here takes more: two blocks an SM at least
constexpr int SMEM_THIRD = 72 * 1024;    // three blocks an SM
// One pass or two: the unit kernels read everything once but load, reduce and store in turns (2.4 to 3.3 TB/s); the streaming
// kernels are two launches, and read once from HBM and once from L2 (4.2 to 5 TB/s).  Both were measured over 92 calls forwards and
// 88 backwards of 2 to 160 MB of traffic, 7x7 to 128x128 pixels, 16 to 2048 channels, bfloat16 and float.  Below 32 MB one pass wins
// almost everywhere: 128x32x32x16 float (16 and 24 MB) 8.3 / 14.3 us against 10.3 / 18.4 forwards / backwards, 16x14x14x1024 bf16
// with a residual (18 and 31 MB) 8.3 / 14.4 against 12.4 / 18.9.  Above it two passes win where a unit takes a whole
// cluster: 16x56x56x256 bf16 with a residual (74 and 123 MB) 28.8 / 57.3 against 20.6 / 34.0; one pass still wins where a unit is small
// (512x32x32x16 bf16 with a residual, 48 and 80 MB: 18.5 / 31.5 against 26.7 / 47.2).  Against the better form of each call the rule loses 2.6 % of
// the time forwards and 3.7 % backwards, the best single number of each direction 2.4 % (64 and 48 MB).
constexpr long long UNIT_TRAFFIC = 32ll << 20;
// With vectors of less than 16 bytes a unit's threads hold little each; two passes have whole vectors over rows of pixels where those
// have no gaps.  Over 57 such calls: 8x33x47x90 bf16 (4.3 and 6.4 MB) 8.3 / 12.1 us in one pass, 12.4 / 14.4 in two; 10x60x60x111
// bf16 (15 and 23 MB) 27.4 / 38.6 against 16.4 / 18.5.  The number is a compromise: 35 channels are better off in two passes
// from 1 MB on (22.6 / 28.8 against 14 / 12.4), 512 samples of 8x8x30 in one (10.3 / 18.5 against 26.7 / 24.6).
constexpr long long NARROW_TRAFFIC = 4ll << 20;

// One pass over a unit of `seg` bytes a pixel or a little less (whole groups, whole vectors), in clusters of up to `most` blocks
// of up to `room` bytes; false if the unit does not fit.
bool unit_plan(const sae_group_norm_desc* d, int vec, int tensors, bool backward, int seg, int most, size_t room, int sms, Plan& p) {
  const int es = elem(d->type), VB = vec * es, cg_ = (int)(d->channels / d->groups);
  int step = cg_;
  while (step % vec) step += cg_;                                  // whole groups and whole vectors
  if (step > d->channels) return false;
  long long cc = std::max(1, seg / (step * es)) * (long long)step;
  cc = std::min<long long>(cc, d->channels);
  int log = 0;
  while ((1ll << log) * vec < cc) ++log;
  const int cvt = 1 << log;
  if (cvt > GN_THREADS) return false;
  cc = std::min<long long>(d->channels, (long long)cvt * vec / step * step);      // fill the lanes
  const long long vectors = d->pixels * cvt;
  int th = GN_THREADS;
  while (th > 64 && vectors < th * 2ll) th /= 2;
  th = std::max(th, cvt);
  if (th < 32) th = 32;
  const int rows = th >> log, SL = vec;
  const size_t fixed = (size_t)(log < 5 ? th / 32 : rows) * cvt * SL * 4 * (backward ? 2 : 1) + (size_t)cc * 8 * 3 + 64;
  if (fixed >= room) return false;
  const long long slots_most = (long long)((room - fixed) / ((size_t)th * VB * tensors));
  if (slots_most < 1) return false;
  long long S = (d->pixels + slots_most * rows - 1) / (slots_most * rows);
  if (S > most) return false;
  // few units: shorter runs over more blocks, as long as a thread keeps two vectors
  const int chunks = (int)((d->channels + cc - 1) / cc);
  const long long units = (long long)d->samples * chunks;
  while (S * 2 <= std::min(most, 8) && units * S * 2 <= sms * 2 && d->pixels >= S * 2 * rows * 2) S *= 2;
  Unit& u = p.u;
  u.log_cvt = log; u.cc = (int)cc; u.chunks = chunks; u.S = (int)S;
  u.px = (int)((d->pixels + S - 1) / S);
  u.slots = (u.px + rows - 1) / rows;
  p.unit = true;
  p.threads = th;
  p.smem = fixed + (size_t)u.slots * th * VB * tensors;
  return true;
}

// Two passes, each of about one wave of blocks; a portion is what a grid's third dimension holds.
void stream_plan(const sae_group_norm_desc* d, int vec, int rep, bool backward, bool residual, int sms, Plan& p) {
  Stream& s = p.s;
  s.rep = rep;
  s.vc = rep * (int)d->channels;
  const long long pixels = d->pixels / rep;                        // rows of them
  const int cv = (s.vc + vec - 1) / vec;
  s.tiles = (cv + GN_THREADS - 1) / GN_THREADS;
  s.cvt = (cv + s.tiles - 1) / s.tiles;
  s.tiles = (cv + s.cvt - 1) / s.cvt;
  const int rows = GN_THREADS / s.cvt, tile_c = s.cvt * vec, cg_ = (int)(d->channels / d->groups);
  s.tile_groups = std::min(d->groups, tile_c / cg_ + 2);
  p.portion = (int)std::min<long long>(d->samples, 32768);
  const bool whole = cg_ % vec == 0;
  const long long wave = (long long)sms * (backward && !whole ? 2 : 3), blocks = (long long)p.portion * s.tiles;
  // one wave of blocks, but at least eight vectors for a thread
  const long long most = std::max<long long>(1, pixels / ((long long)rows * 8));
  s.slices = (int)std::min<long long>(1024, std::min(std::max<long long>(1, wave / blocks), most));
  s.px = (int)((pixels + s.slices - 1) / s.slices);
  s.slices = (int)((pixels + s.px - 1) / s.px);
  const size_t runs = (size_t)d->samples * s.slices;
  p.bytes = runs * s.tiles * s.tile_groups * sizeof(float2) + (backward ? 2 * runs * d->channels * sizeof(float) : 0);
}

Plan make_plan(const sae_group_norm_desc* d, Width w, bool backward, bool residual, int sms) {
  Plan p = {};
  const int vec = w.vec;
  p.vec = vec;
  // rows of several pixels: no pixels left over, one tile
  int rep = w.row_vec ? row_pixels(d, w.row_vec) : 1;
  if (rep > 1 && (d->pixels % rep || rep * d->channels / w.row_vec > GN_THREADS)) rep = 1;
  // backward: a second slot for dz in float where its type cannot hold it
  const bool second = residual || (backward && elem(d->type) == 2 && d->activation >= SAE_ACT_SILU);
  const int tensors = (backward ? 2 : 1) + (second ? 1 : 0);
  const int segs[3] = {128, 64, 32};                               // shorter runs of a pixel where longer ones do not fit
  const long long traffic = d->samples * d->pixels * d->channels * elem(d->type) * (backward ? 3 + 2 * residual : 2 + residual);
  if (traffic <= (vec * elem(d->type) < 16 ? NARROW_TRAFFIC : UNIT_TRAFFIC)) {
    // a unit a block, if that fills the SMs; else clusters, of narrower units where wide ones are too few to fill them and leave
    // a thread more than four vectors (3x33x47x90 float: 12.5 us with 72 blocks, 9.4 with 360)
    unit_plan(d, vec, tensors, backward, segs[0], 1, SMEM_MOST, sms, p);
    if (p.unit && d->samples * p.u.chunks < sms) p.unit = false;
    for (int i = 0; i < 3 && !p.unit; ++i) {
      if (!unit_plan(d, vec, tensors, backward, segs[i], 8, SMEM_THIRD, sms, p) || i == 2) continue;
      Plan q = p;
      q.unit = false;
      if (d->samples * p.u.chunks * p.u.S < sms && p.u.slots > 4 && unit_plan(d, vec, tensors, backward, segs[i + 1], 8, SMEM_THIRD, sms, q)) p.unit = false;
    }
    for (int i = 0; i < 3 && !p.unit; ++i) unit_plan(d, vec, tensors, backward, segs[i], 8, SMEM_MOST, sms, p);
  }
  if (p.unit) p.bytes = backward ? (size_t)2 * 4 * d->samples * d->channels : 0;
  else {
    if (rep > 1) p.vec = w.row_vec;
    stream_plan(d, p.vec, rep, backward, residual, sms, p);
  }
  return p;
}

int device_sms() {
  static std::atomic<int> known[64];
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 0; }
  if (dev >= 0 && dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
  if (dev >= 0 && dev < 64) known[dev].store(sms, std::memory_order_relaxed);
  return sms;
}

Args make_args(const sae_group_norm_desc* d, const Plan& p, void* ws) {
  Args a = {};
  a.x_n = d->x_sample; a.x_p = d->x_pixel; a.r_n = d->residual_sample; a.r_p = d->residual_pixel; a.d_n = d->dy_sample; a.d_p = d->dy_pixel;
  a.N = (int)d->samples; a.P = (int)d->pixels; a.C = (int)d->channels; a.G = d->groups; a.Cg = a.C / a.G;
  a.act = d->activation; a.ptype = d->param_type; a.eps = d->eps;
  if (!p.unit && p.s.rep > 1) { a.P /= p.s.rep; a.x_p *= p.s.rep; a.r_p *= p.s.rep; a.d_p *= p.s.rep; }
  const size_t runs = (size_t)a.N * (p.unit ? 1 : p.s.slices);
  a.part_s = (float2*)ws;
  a.part_a = (float*)(a.part_s + (p.unit ? 0 : runs * p.s.tiles * p.s.tile_groups));
  a.part_b = a.part_a + runs * a.C;
  return a;
}

// Dynamic shared memory above 48 KB needs an opt-in, once a device and kernel.
template <auto KERNEL>
int opt_in() {
  static thread_local int opted = -1;               // one variable for each kernel
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
  if (opted != dev) {
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
    opted = dev;
  }
  return SAE_OK;
}

// A unit kernel in clusters of S blocks.
template <void (*KERNEL)(const Args, const Unit)>
int launch_units(const Args& a, const Plan& p, cudaStream_t st) {
  const int rc = opt_in<KERNEL>();
  if (rc != SAE_OK) return rc;
  cudaLaunchConfig_t cfg = {};
  const int ny = std::min(a.N, 32768);
  cfg.gridDim = dim3((unsigned)(p.u.chunks * p.u.S), (unsigned)ny, (unsigned)((a.N + ny - 1) / ny));
  cfg.blockDim = dim3((unsigned)p.threads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)p.u.S, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = p.u.S > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, KERNEL, a, p.u) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
  return SAE_OK;
}

// One of a call's streaming kernels: all but the first may start before their predecessor's end (they wait for it themselves).
template <auto KERNEL, typename... A>
int launch(dim3 grid, size_t smem, cudaStream_t st, bool first, A... args) {
  if (smem > 48 * 1024) {
    const int rc = opt_in<KERNEL>();
    if (rc != SAE_OK) return rc;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(GN_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = first ? 0 : 1;
  if (cudaLaunchKernelEx(&cfg, KERNEL, args...) != cudaSuccess) { cudaGetLastError(); return SAE_ERR_CUDA; }
  return SAE_OK;
}

template <typename T, int V, bool WHOLE>
int forward_as(const Args& a, const Plan& p, cudaStream_t st) {
  if (p.unit) return launch_units<k_gn_unit<T, V, WHOLE>>(a, p, st);
  Stream s = p.s;
  const int rows = GN_THREADS / s.cvt;
  const size_t stat = (s.tile_groups + GN_THREADS) * sizeof(float2);
  constexpr int VB = V * (int)sizeof(T);
  int rc = SAE_OK;
  for (s.n0 = 0; s.n0 < a.N && rc == SAE_OK; s.n0 += p.portion) {
    const unsigned n = (unsigned)std::min(p.portion, a.N - s.n0);
    const dim3 grid((unsigned)s.slices, (unsigned)s.tiles, n);
    rc = launch<k_gn_statistics<T, V, WHOLE>>(grid, std::max(ring_bytes(VB, 1), (size_t)(rows * s.cvt * (WHOLE ? 1 : V) + s.tile_groups) * 4), st, s.n0 == 0, a, s);
    if (rc != SAE_OK) break;
    if (a.res) rc = launch<k_gn_apply<T, V, WHOLE, true>>(grid, ring_bytes(VB, 2) + stat, st, false, a, s);
    else rc = launch<k_gn_apply<T, V, WHOLE, false>>(grid, ring_bytes(VB, 1) + stat, st, false, a, s);
  }
  return rc;
}

template <typename T, int V, bool WHOLE, int ACT, bool RES>
int grad_sums(const Args& a, const Stream& s, dim3 grid, cudaStream_t st, bool first) {
  constexpr int kept = sums_kept(V);
  return launch<k_gn_grad_sums<T, V, WHOLE, ACT, RES>>(
      grid, std::max(ring_bytes(V * sizeof(T), RES ? 3 : 2, kept) + kept * GN_THREADS, (size_t)(2 * (GN_THREADS / s.cvt) * s.cvt * V) * 4), st, first, a, s);
}
template <typename T, int V, bool WHOLE, int ACT, bool RES>
int grad_apply(const Args& a, const Stream& s, dim3 grid, cudaStream_t st, bool) {
  return launch<k_gn_grad_apply<T, V, WHOLE, ACT, RES>>(grid, ring_bytes(V * sizeof(T), RES ? 3 : 2) + (s.tile_groups + GN_THREADS) * sizeof(float2), st, false, a, s);
}
#define GN_ACT(fn, ...)                                                                                              \
  (a.act == SAE_ACT_NONE ? fn<T, V, WHOLE, 0, false>(__VA_ARGS__)                                                     \
   : a.act == SAE_ACT_RELU ? (a.res ? fn<T, V, WHOLE, 1, true>(__VA_ARGS__) : fn<T, V, WHOLE, 1, false>(__VA_ARGS__)) \
                           : (a.res ? fn<T, V, WHOLE, 2, true>(__VA_ARGS__) : fn<T, V, WHOLE, 2, false>(__VA_ARGS__)))

template <typename T, int V, bool WHOLE>
int backward_as(const Args& all, const Plan& p, cudaStream_t st) {
  const unsigned param_blocks = all.dw || all.db ? (unsigned)((all.C + 31) / 32) : 0;
  int rc = SAE_OK;
  if (p.unit) {
    rc = launch_units<k_gn_grad_unit<T, V, WHOLE>>(all, p, st);
    if (rc == SAE_OK && param_blocks) rc = launch<k_gn_param_grads>(dim3(param_blocks), 0, st, false, all, (long long)all.N);
    return rc;
  }
  Stream s = p.s;
  // where dresidual holds dz unrounded, the second pass reads it in place of dy and the residual
  s.held = all.dres && (sizeof(T) == 4 || all.act <= SAE_ACT_RELU);
  for (s.n0 = 0; s.n0 < all.N && rc == SAE_OK; s.n0 += p.portion) {
    const unsigned n = (unsigned)std::min(p.portion, all.N - s.n0);
    dim3 grid((unsigned)s.slices, (unsigned)s.tiles, n);
    Args a = all;
    s.param_z = 0;
    rc = GN_ACT(grad_sums, a, s, grid, st, s.n0 == 0);
    if (s.held) {
      a.dy = a.dres; a.d_n = (long long)a.P * s.vc; a.d_p = s.vc;
      a.act = SAE_ACT_NONE; a.res = nullptr;
    }
    if (s.n0 + p.portion >= all.N) s.param_z = (int)((param_blocks + grid.x * grid.y - 1) / (grid.x * grid.y));
    grid.z += (unsigned)s.param_z;
    if (rc == SAE_OK) rc = GN_ACT(grad_apply, a, s, grid, st, false);
  }
  return rc;
}

template <typename T, int V>
int forward(const Args& a, const Plan& p, cudaStream_t st) {
  if constexpr (V > 2) { if (a.Cg % V == 0) return forward_as<T, V, true>(a, p, st); }
  return forward_as<T, V, V == 1>(a, p, st);
}
template <typename T, int V>
int backward(const Args& a, const Plan& p, cudaStream_t st) {
  if constexpr (V > 2) { if (a.Cg % V == 0) return backward_as<T, V, true>(a, p, st); }
  return backward_as<T, V, V == 1>(a, p, st);
}

// An element type and a vector width as template arguments.
#define GN_DISPATCH16(fn, T, vec, ...) ((vec) == 8 ? fn<T, 8>(__VA_ARGS__) : (vec) == 2 ? fn<T, 2>(__VA_ARGS__) : fn<T, 1>(__VA_ARGS__))
#define GN_DISPATCH(fn, type, vec, ...)                                                                  \
  ((type) == SAE_TYPE_FLOAT ? ((vec) == 4 ? fn<float, 4>(__VA_ARGS__) : fn<float, 1>(__VA_ARGS__))        \
   : (type) == SAE_TYPE_BFLOAT ? GN_DISPATCH16(fn, __nv_bfloat16, vec, __VA_ARGS__) : GN_DISPATCH16(fn, __half, vec, __VA_ARGS__))

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

extern "C" {

int64_t sae_group_norm_workspace(const sae_group_norm_desc* d, int32_t backward) {
  if (!desc_ok(d)) return -1;
  const int sms = device_sms();
  if (sms < 1) return -1;
  if (d->samples == 0 || d->pixels == 0) return 0;
  // the tensors' alignment and whether there is a residual are not known yet: the most that any form needs
  size_t most = 0;
  const int widths[3] = {16 / elem(d->type), 2, 1};
  for (int i = 0; i < 3; ++i) {
    if ((i == 1 && elem(d->type) == 4) || d->channels % widths[i]) continue;
    for (int r = 0; r < 4; ++r)
      most = std::max(most, make_plan(d, {widths[i], i && r >= 2 ? widths[0] : 0}, backward != 0, r & 1, sms).bytes);
  }
  return (int64_t)most;
}

int sae_group_norm_forward(const sae_group_norm_desc* d, const void* x, const void* residual, const void* weight, const void* bias,
                           void* y, float* mean, float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc_ok(d)) return SAE_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->samples == 0) return SAE_OK;
  if (!mean || !rstd) return SAE_ERR_INVALID_ARG;
  if (d->pixels == 0) {                     // the mean of nothing
    const size_t g = (size_t)d->samples * d->groups * sizeof(float);
    return cudaMemsetAsync(mean, 0xff, g, st) == cudaSuccess && cudaMemsetAsync(rstd, 0xff, g, st) == cudaSuccess ? SAE_OK : SAE_ERR_CUDA;
  }
  const int es = elem(d->type);
  if (!x || !y || !aligned_to(x, es) || !aligned_to(y, es) || !aligned_to(residual, es) || !aligned_to(weight, elem(d->param_type)) ||
      !aligned_to(bias, elem(d->param_type))) return SAE_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms < 1) return SAE_ERR_CUDA;
  const void* ptrs[3] = {x, y, residual};
  const Plan p = make_plan(d, vector_width(d, ptrs, 3, residual != nullptr, false), false, residual != nullptr, sms);
  if ((p.bytes && !workspace) || !aligned_to(workspace, 16) || workspace_bytes < p.bytes) return SAE_ERR_INVALID_ARG;
  Args a = make_args(d, p, workspace);
  a.x = x; a.res = residual; a.w = weight; a.b = bias; a.out = y; a.mean = mean; a.rstd = rstd;
  return GN_DISPATCH(forward, d->type, p.vec, a, p, st);
}

int sae_group_norm_backward(const sae_group_norm_desc* d, const void* dy, const void* x, const void* residual, const float* mean,
                            const float* rstd, const void* weight, const void* bias, void* dx, void* dresidual, void* dweight,
                            void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!desc_ok(d)) return SAE_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->samples == 0 || d->pixels == 0) {  // sums of nothing
    const size_t c = (size_t)d->channels * elem(d->param_type);
    if (dweight && cudaMemsetAsync(dweight, 0, c, st) != cudaSuccess) return SAE_ERR_CUDA;
    if (dbias && cudaMemsetAsync(dbias, 0, c, st) != cudaSuccess) return SAE_ERR_CUDA;
    return SAE_OK;
  }
  const int es = elem(d->type), ps = elem(d->param_type);
  if (!dy || !x || !mean || !rstd || !dx || !aligned_to(dy, es) || !aligned_to(x, es) || !aligned_to(residual, es) || !aligned_to(dx, es) ||
      !aligned_to(dresidual, es) || !aligned_to(weight, ps) || !aligned_to(bias, ps) || !aligned_to(dweight, ps) || !aligned_to(dbias, ps))
    return SAE_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms < 1) return SAE_ERR_CUDA;
  const void* ptrs[5] = {dy, x, residual, dx, dresidual};
  const Plan p = make_plan(d, vector_width(d, ptrs, 5, residual != nullptr, true), true, residual != nullptr, sms);
  if ((p.bytes && !workspace) || !aligned_to(workspace, 16) || workspace_bytes < p.bytes) return SAE_ERR_INVALID_ARG;
  Args a = make_args(d, p, workspace);
  a.x = x; a.dy = dy; a.res = residual; a.w = weight; a.b = bias; a.out = dx; a.dres = dresidual; a.dw = dweight; a.db = dbias;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  return GN_DISPATCH(backward, d->type, p.vec, a, p, st);
}

}  // extern "C"
