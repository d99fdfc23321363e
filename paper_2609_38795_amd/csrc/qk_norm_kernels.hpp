// RMSNorm of every query and key head with the position rotation in the same pass, and its gradient.
//
// For a head x of hd values (half = hd / 2), gain g, and the angles of the row's position:
//   r = 1 / sqrt(mean(x^2) + eps),  y = x r g,
//   out_i        = y_i cos_i - y_(i+half) sin_i,   out_(i+half) = y_(i+half) cos_i + y_i sin_i.
// With d the gradient of out, turned back by the same angles, and xh = x r:
//   dg = sum over rows and heads of d xh,   dx = r (g d - xh mean(g d xh)).
// Statistics, rotation and sums are fp32; each result is rounded to its type once.
#pragma once

#include "device_common.hpp"
#include "gemm_kernels.hpp"

namespace alr {

struct QkArgs {
  const void *q, *k;     // rows of H * hd and of G * hd values
  long q_rs, k_rs;
  const void *gq, *gk;   // [hd]
  const void *dq_in, *dk_in;  // gradients of the outputs (backward)
  long dq_in_rs, dk_in_rs;
  void *q_out, *k_out;   // outputs, or gradients of q and k (may be the inputs' own rows)
  long q_out_rs, k_out_rs;
  const int* pos;        // [n, 3] positions, or null: the row's index on every axis
  int pos_add;
  const f32x2* tab;      // (cos, sin) [max_pos, half]
  int max_pos, hd, sec0, sec01;  // frequencies < sec0 follow axis 0, < sec01 axis 1, the rest axis 2
  int H, G;
  long n;
  float eps;
  float* part;           // backward: gain gradients of each workgroup [wg, 2, hd]
};

// (cos, sin) of row r at frequency i; nan for a position outside the table
__device__ __forceinline__ f32x2 qk_factor(const QkArgs& a, long r, int i) {
  const int axis = i < a.sec0 ? 0 : i < a.sec01 ? 1 : 2;
  const long p = (a.pos ? (long)a.pos[3 * r + axis] : r) + a.pos_add;
  const float bad = __builtin_nanf("");
  return p >= 0 && p < a.max_pos ? a.tab[p * (a.hd >> 1) + i] : f32x2{bad, bad};
}

// Any head size up to 256, any alignment: one wave per head, a pair (i, i + half) per lane and step.
template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_any_kernel(QkArgs a) {
  const int lane = threadIdx.x & 63, half = a.hd >> 1, heads = a.H + a.G;
  const long units = a.n * heads;
  for (long u = (long)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (long)gridDim.x * 4) {
    const long r = u / heads;
    const int h = (int)(u - r * heads);
    const bool isq = h < a.H;
    const T* x = isq ? static_cast<const T*>(a.q) + r * a.q_rs + (long)h * a.hd
                     : static_cast<const T*>(a.k) + r * a.k_rs + (long)(h - a.H) * a.hd;
    T* y = isq ? static_cast<T*>(a.q_out) + r * a.q_out_rs + (long)h * a.hd
               : static_cast<T*>(a.k_out) + r * a.k_out_rs + (long)(h - a.H) * a.hd;
    const T* g = static_cast<const T*>(isq ? a.gq : a.gk);
    float lo[2], hi[2], ss = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = lane + 64 * t;
      lo[t] = i < half ? Elt<T>::ld(x + i) : 0.f;
      hi[t] = i < half ? Elt<T>::ld(x + i + half) : 0.f;
      ss += lo[t] * lo[t] + hi[t] * hi[t];
    }
    const float inv = 1.0f / sqrtf(wave_sum(ss) / (float)a.hd + a.eps);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = lane + 64 * t;
      if (i >= half) continue;
      const f32x2 w = qk_factor(a, r, i);
      const float l = lo[t] * inv * Elt<T>::ld(g + i), m = hi[t] * inv * Elt<T>::ld(g + i + half);
      Elt<T>::st(y + i, rope_a(l, m, w[0], w[1]));
      Elt<T>::st(y + i + half, rope_b(l, m, w[0], w[1]));
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_back_any_kernel(QkArgs a) {
  __shared__ float sum[2][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = a.hd >> 1, heads = a.H + a.G;
  const long units = a.n * heads;
  float dg[2][2][2] = {};  // [q, k][step][low, high]
  for (long u = (long)blockIdx.x * 4 + wave; u < units; u += (long)gridDim.x * 4) {
    const long r = u / heads;
    const int h = (int)(u - r * heads);
    const bool isq = h < a.H;
    const long hq = (long)h * a.hd, hk = (long)(h - a.H) * a.hd;
    const T* x = isq ? static_cast<const T*>(a.q) + r * a.q_rs + hq
                     : static_cast<const T*>(a.k) + r * a.k_rs + hk;
    const T* dy = isq ? static_cast<const T*>(a.dq_in) + r * a.dq_in_rs + hq
                      : static_cast<const T*>(a.dk_in) + r * a.dk_in_rs + hk;
    T* dx = isq ? static_cast<T*>(a.q_out) + r * a.q_out_rs + hq
                : static_cast<T*>(a.k_out) + r * a.k_out_rs + hk;
    const T* g = static_cast<const T*>(isq ? a.gq : a.gk);
    float x2[2][2], d[2][2], ss = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = lane + 64 * t;
      const bool in = i < half;
      x2[t][0] = in ? Elt<T>::ld(x + i) : 0.f;
      x2[t][1] = in ? Elt<T>::ld(x + i + half) : 0.f;
      const float lo = in ? Elt<T>::ld(dy + i) : 0.f, hi = in ? Elt<T>::ld(dy + i + half) : 0.f;
      const f32x2 w = in ? qk_factor(a, r, i) : f32x2{1.f, 0.f};
      d[t][0] = rope_a(lo, hi, w[0], -w[1]);
      d[t][1] = rope_b(lo, hi, w[0], -w[1]);
      ss += x2[t][0] * x2[t][0] + x2[t][1] * x2[t][1];
    }
    const float inv = 1.0f / sqrtf(wave_sum(ss) / (float)a.hd + a.eps);
    float dot = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = lane + 64 * t;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        x2[t][e] *= inv;
        const float p = d[t][e] * x2[t][e];
        if (isq)
          dg[0][t][e] += p;
        else
          dg[1][t][e] += p;
        d[t][e] *= i < half ? Elt<T>::ld(g + i + e * half) : 0.f;
        dot += d[t][e] * x2[t][e];
      }
    }
    dot = wave_sum(dot) / (float)a.hd;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = lane + 64 * t;
      if (i >= half) continue;
#pragma unroll
      for (int e = 0; e < 2; ++e) Elt<T>::st(dx + i + e * half, inv * (d[t][e] - x2[t][e] * dot));
    }
  }
  // the waves' sums one after the other: the order is fixed
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int i = lane + 64 * t;
        if (i >= half) continue;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            float& s = sum[b][i + e * half];
            s = (w == 0 ? 0.f : s) + dg[b][t][e];
          }
      }
    }
    __syncthreads();
  }
  float* out = a.part + (long)blockIdx.x * 2 * a.hd;
  for (int i = threadIdx.x; i < 2 * a.hd; i += 256) out[i] = sum[i / a.hd][i % a.hd];
}

// Gain gradients: the workgroups' partial sums added in order of the workgroups, 32 columns a
// workgroup, its 8 thread rows taking every 8th partial and meeting at the end.
__global__ __launch_bounds__(256) void qk_gain_grad_kernel(const float* __restrict__ part, int n_wg,
                                                           int hd, float* __restrict__ dgq,
                                                           float* __restrict__ dgk) {
  __shared__ float s[8][32];
  const int col = threadIdx.x & 31, sub = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
  float t = 0.f;
  if (c < 2 * hd)
    for (int w = sub; w < n_wg; w += 8) t += part[(long)w * 2 * hd + c];
  s[sub][col] = t;
  __syncthreads();
  if (sub != 0 || c >= 2 * hd) return;
  for (int i = 1; i < 8; ++i) t += s[i][col];
  if (c < hd) {
    if (dgq) dgq[c] = t;
  } else if (dgk) {
    dgk[c - hd] = t;
  }
}

// Factor rows that turn nothing: what the QKV epilogue is given where the norm and the rotation
// follow it in a pass of their own.
__global__ __launch_bounds__(256) void unit_factor_kernel(f32x2* __restrict__ rope, long n) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i < n) rope[i] = f32x2{1.f, 0.f};
}

}  // namespace alr
