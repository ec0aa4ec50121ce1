// What the group-norm kernels share: arguments, parameters, activations and the sums over a block.
#pragma once
#include "../../include/sae.h"
#include "sae_vec.cuh"

namespace sae {

constexpr int GN_THREADS = 256;

struct Args {
  const void *x, *res, *dy, *w, *b;
  void *out, *dres;                      // y or dx; dense
  float *mean, *rstd;                    // [N][G]: written forwards, read backwards
  void *dw, *db;
  long long x_n, x_p, r_n, r_p, d_n, d_p;   // strides of a sample and of a pixel, in elements
  int N, P, C, G, Cg;
  int act, ptype;
  float eps;
  float *part_a, *part_b;                // backwards, [N][slices][C]: each channel's sum dz and sum dz * xhat over a run of pixels
  float2* part_s;                        // two passes, [N][slices][tiles][tile_groups], of a run's part of a group: forwards its mean and
                                         // the squares about it, backwards sum g and sum g * xhat
};

__device__ __forceinline__ float param(const void* p, int type, int c, float none) {
  if (!p) return none;
  if (type == SAE_TYPE_FLOAT) return __ldg((const float*)p + c);
  if (type == SAE_TYPE_BFLOAT) return to_f(((const __nv_bfloat16*)p)[c]);
  return to_f(((const __half*)p)[c]);
}
__device__ __forceinline__ void put_param(void* p, int type, int c, float v) {
  if (type == SAE_TYPE_FLOAT) ((float*)p)[c] = v;
  else if (type == SAE_TYPE_BFLOAT) ((__nv_bfloat16*)p)[c] = from_f<__nv_bfloat16>(v);
  else ((__half*)p)[c] = from_f<__half>(v);
}

// ---- activations ------------------------------------------------------------------------------------------------
// Results of 16 bits are computed with the special-function unit's 2^x and 1/x, two elements at a time where there is arithmetic:
// relative errors of a few units of a float, |z| (silu) or z^2 (gelu) more from the exponent's rounding, and zero for what lies below
// 2^-126.  Float results are computed with expf, erff and true divisions.
__device__ __forceinline__ float fast_exp2(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float fast_rcp(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

template <int V>
__device__ __forceinline__ void vset(float (&o)[V], float v) {
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = v;
}

// s = 1 / (1 + exp(-z))
template <typename T, int V>
__device__ __forceinline__ void sigmoid(float (&s)[V], const float (&z)[V]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = __fdiv_rn(1.0f, 1.0f + expf(-z[i]));
  } else {
    float c[V], one[V];
    vset<V>(c, -1.44269504f);
    vset<V>(one, 1.0f);
    vmul<V>(s, z, c);
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = fast_exp2(s[i]);
    vadd<V>(s, s, one);
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = fast_rcp(s[i]);
  }
}

// The normal distribution's cdf and exp(-z^2 / 2).  16 bits: the tail beyond |z| is exp(-z^2 / 2) times a smooth function of |z|, which
// as t times a polynomial in t = 1 / (1 + 0.305 |z|) has a relative error of 9.4e-8 up to |z| = 13.3, where the exponential ends (the
// coefficients are fitted for the least relative error there; in float, 6.7 units).  An approximation of erf with a small absolute
// error would not do: its share in the tail grows, 4.7e-4 at z = -4 and 2 % at -10 for formula 7.1.26 of Abramowitz and Stegun.
template <typename T, int V>
__device__ __forceinline__ void normal(float (&cdf)[V], float (&e)[V], const float (&z)[V]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) { cdf[i] = 0.5f * (1.0f + erff(z[i] * 0.70710678f)); e[i] = expf(-0.5f * z[i] * z[i]); }
  } else {
    float t[V], p[V], c[V];
    vset<V>(c, -0.72134752f);                                                   // -log2(e) / 2
    vmul<V>(e, z, z);
    vmul<V>(e, e, c);
    vset<V>(c, 1.0f);
    vset<V>(p, 0.305f);
#pragma unroll
    for (int i = 0; i < V; ++i) { e[i] = fast_exp2(e[i]); t[i] = fabsf(z[i]); }
    vfma<V>(t, t, p, c);
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = fast_rcp(t[i]);
    vset<V>(p, 0.0366991796f);
    vset<V>(c, -0.15298827f); vfma<V>(p, p, t, c);
    vset<V>(c, 0.185716823f); vfma<V>(p, p, t, c);
    vset<V>(c, -0.037976753f); vfma<V>(p, p, t, c);
    vset<V>(c, 0.121021636f); vfma<V>(p, p, t, c);
    vset<V>(c, 0.103420876f); vfma<V>(p, p, t, c);
    vset<V>(c, 0.122466817f); vfma<V>(p, p, t, c);
    vset<V>(c, 0.121639736f); vfma<V>(p, p, t, c);
    vmul<V>(t, t, e);
    vmul<V>(p, p, t);                                                           // the tail beyond |z|
#pragma unroll
    for (int i = 0; i < V; ++i) cdf[i] = z[i] >= 0.0f ? 1.0f - p[i] : p[i];
  }
}

template <typename T, int V>
__device__ __forceinline__ void activate(float (&z)[V], int act) {
  if (act == SAE_ACT_RELU) {                                                    // a NaN stays
#pragma unroll
    for (int i = 0; i < V; ++i) asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(z[i]) : "f"(z[i]));
  } else if (act == SAE_ACT_SILU) {
    float s[V];
    sigmoid<T, V>(s, z);
    vmul<V>(z, z, s);
  } else if (act == SAE_ACT_GELU) {
    float cdf[V], e[V];
    normal<T, V>(cdf, e, z);
    vmul<V>(z, z, cdf);
  }
}

// dz[i] = dy[i] * act'(z[i])
template <typename T, int V>
__device__ __forceinline__ void slope(float (&dz)[V], const float (&z)[V], int act) {
  if (act == SAE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) dz[i] = z[i] > 0.0f ? dz[i] : 0.0f;
  } else if (act == SAE_ACT_SILU) {                                             // s (1 + z (1 - s))
    float s[V], t[V], one[V];
    sigmoid<T, V>(s, z);
    vset<V>(one, 1.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = -s[i];
    vadd<V>(t, t, one);
    vfma<V>(t, t, z, one);
    vmul<V>(t, t, s);
    vmul<V>(dz, dz, t);
  } else if (act == SAE_ACT_GELU) {                                             // cdf + z exp(-z^2 / 2) / sqrt(2 pi)
    float cdf[V], e[V], c[V];
    normal<T, V>(cdf, e, z);
    vset<V>(c, 0.39894228f);
    vmul<V>(e, e, c);
    vfma<V>(e, e, z, cdf);
    vmul<V>(dz, dz, e);
  }
}

// V neighbouring parameters at once: c is a multiple of V, and the parameters' own alignment is checked here.
template <int V>
__device__ __forceinline__ void params(const void* p, int type, int c, float none, float (&o)[V]) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = none;
  } else if (V >= 4 && type == SAE_TYPE_FLOAT && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i + 3 < V; i += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>((const float*)p + c + i));
      o[i] = f.x; o[i + 1] = f.y; o[i + 2] = f.z; o[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = param(p, type, c + i, none);
  }
}

// Small non-negative integers (below 2^20) over a divisor, by its reciprocal.
__device__ __forceinline__ int quotient(int a, float inv) { return (int)(((float)a + 0.5f) * inv); }

// xhat and dz of a vector.
template <typename T, int V>
__device__ __forceinline__ void vector_grad(const Raw<T, V>& x, const Raw<T, V>& d, const Raw<T, V>* res, const float (&less)[V], const float (&scale)[V],
                                          const float (&w)[V], const float (&b)[V], int act, float (&xh)[V], float (&dz)[V]) {
  float z[V];
  x.widen(xh);
  d.widen(dz);
  vadd<V>(xh, xh, less);
  vmul<V>(xh, xh, scale);
  if (act == SAE_ACT_NONE) return;
  vmul_add<V>(z, xh, w, b);
  if (res) {
    float v[V];
    res->widen(v);
    vadd<V>(z, z, v);
  }
  slope<T, V>(dz, z, act);
}

// A thread's V channel sums as one, or as they are.
template <int V, int SL>
__device__ __forceinline__ void narrow(const float (&v)[V], float (&o)[SL]) {
  if constexpr (SL == V) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = v[i];
  } else {
    float t = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) t += v[i];
    o[0] = t;
  }
}

// Adds up v over the rows of a block, column by column: afterwards sh[r * pitch + column * SL + i] holds the sums of row r's
// warp (columns fewer than a warp's lanes: those are joined here) and `rows` such rows are left to add.  Ends with a barrier.
template <int SL>
__device__ __forceinline__ int fold_rows(float (&v)[SL], float* sh, int log_cvt) {
  const int cvt = 1 << log_cvt, tid = threadIdx.x;
  int rows = (int)blockDim.x >> log_cvt, row = tid >> log_cvt;
  bool write = true;
  if (log_cvt < 5) {
    for (int o = 16; o >= cvt; o >>= 1) {
#pragma unroll
      for (int i = 0; i < SL; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    rows = (int)blockDim.x >> 5;
    row = tid >> 5;
    write = (tid & 31) < cvt;
  }
  if (write) {
    float* to = sh + (row * cvt + (tid & (cvt - 1))) * SL;
#pragma unroll
    for (int i = 0; i < SL; ++i) to[i] = v[i];
  }
  __syncthreads();
  return rows;
}

// The folded values of each group: one warp a group, `per` neighbouring values of it in a row.  out[j] is written by lane 0.
template <typename F>
__device__ __forceinline__ void fold_groups(const float* sh, int rows, int pitch, int per, int groups, F out) {
  const int lane = threadIdx.x & 31;
  const float inv_per = 1.0f / (float)per;
  for (int j = threadIdx.x >> 5; j < groups; j += (int)blockDim.x >> 5) {
    float s = 0.0f;
    for (int e = lane; e < rows * per; e += 32) {
      const int r = (int)(((float)e + 0.5f) * inv_per);
      s += sh[r * pitch + j * per + (e - r * per)];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) out(j, s);
  }
}

// Adds up 2 V values a lane over the lanes whose numbers differ in the bits above log_cvt: in each round a lane hands half of
// its values to the partner and takes the partner's other half, so the work halves from round to round.  Afterwards values
// v[0 .. left) of a lane are the sums of the values from `from` on; `left` is returned.  The order is fixed.
template <int W>
__device__ __forceinline__ int scatter_sum(float (&v)[W], int log_cvt, int& from) {
  const int lane = threadIdx.x & 31;
  int left = W;
  from = 0;
#pragma unroll
  for (int r = 0; r < 5; ++r) {
    const int o = 16 >> r;
    if (o < (1 << log_cvt)) break;
    const bool upper = (lane & o) != 0;
    if ((W >> r) >= 2) {
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        if (i < (W >> r) / 2) {
          const float keep = upper ? v[i + (W >> r) / 2] : v[i], give = upper ? v[i] : v[i + (W >> r) / 2];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
      left = (W >> r) / 2;
      if (upper) from += left;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
  return left;
}

}  // namespace sae
