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

// Sum over each aligned group of LPH lanes, the same in all of them (DPP permutations as group_sum).
template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
  if constexpr (LPH == 32) v = sum_xor16(v);
  if constexpr (LPH >= 16) v += dpp_perm<0x140>(v);
  if constexpr (LPH >= 8) v += dpp_perm<0x141>(v);
  if constexpr (LPH >= 2) v += dpp_perm<0xB1>(v);
  if constexpr (LPH >= 4) v += dpp_perm<0x4E>(v);
  return v;
}

// Heads whose half is whole 16-byte runs, in rows on 16-byte boundaries: LPH lanes per head, each with
// one run of VEC values of the low half and the one that is turned with it, 64 / LPH heads of a row at a
// time.  The factors of the row's position are read once per wave, and the loads of U such steps go out before
// the first use.  What bounds it is HBM: 32768 rows of 40 bf16 heads of 128 take 125 us (5.4 TB/s, a large
// copy's 5.2); a wave per head, with a pair per lane, took 516.  Seven rows take the kernel 4 us.  Registers leave
// three waves a SIMD in bf16 (129, four waves from 128 on), four in fp32.
template <typename T, int LPH>
struct QkLane {
  static constexpr int VEC = 16 / (int)sizeof(T), HPW = 64 / LPH;
  int j0, head;  // the lane's first index within the half; its head within a step
  bool on;       // lanes past the half idle (halves of 5 or 6 runs)
  __device__ __forceinline__ explicit QkLane(int half) {
    const int lane = threadIdx.x & 63;
    j0 = (lane & (LPH - 1)) * VEC;
    head = lane / LPH;
    on = j0 < half;
  }
  __device__ __forceinline__ static void widen(u32x4 w, float (&v)[VEC]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        v[k] = __uint_as_float(w[k]);
      } else {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
    }
  }
  __device__ __forceinline__ static u32x4 narrow(const float (&v)[VEC]) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4)
        w[k] = __float_as_uint(v[k]);
      else
        w[k] = pack2bf(v[2 * k], v[2 * k + 1]);
    }
    return w;
  }
  __device__ __forceinline__ u32x4 run(const T* p) const {
    return on ? *reinterpret_cast<const u32x4*>(p) : u32x4{0, 0, 0, 0};
  }
  // (cos, sin) of row r at the lane's run
  __device__ __forceinline__ void factors(const QkArgs& a, long r, float (&cs)[VEC],
                                          float (&sn)[VEC]) const {
    const int i1 = j0 + VEC - 1;
    const bool one_axis = (j0 < a.sec0) == (i1 < a.sec0) && (j0 < a.sec01) == (i1 < a.sec01);
    if (!on) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) cs[e] = 1.f, sn[e] = 0.f;
    } else if (one_axis) {
      const int axis = j0 < a.sec0 ? 0 : j0 < a.sec01 ? 1 : 2;
      const long p = (a.pos ? (long)a.pos[3 * r + axis] : r) + a.pos_add;
      const bool ok = p >= 0 && p < a.max_pos;
      const float bad = __builtin_nanf("");
      const f32x4* t = reinterpret_cast<const f32x4*>(a.tab + (ok ? p : 0) * (a.hd >> 1) + j0);
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        const f32x4 w = t[e];
        cs[2 * e] = ok ? w[0] : bad;
        sn[2 * e] = w[1];
        cs[2 * e + 1] = ok ? w[2] : bad;
        sn[2 * e + 1] = w[3];
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const f32x2 w = qk_factor(a, r, j0 + e);
        cs[e] = w[0];
        sn[e] = w[1];
      }
    }
  }
};

// A row's heads come as steps of HPW heads, those of q and then those of k; a wave takes the steps
// [part * per, (part + 1) * per) of one row.
struct QkSteps {
  int q, k, per, splits;  // steps of q and of k; steps and parts of a row
};

template <typename T, int LPH>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a, QkSteps st) {
  using L = QkLane<T, LPH>;
  constexpr int VEC = L::VEC, U = 4;
  const int half = a.hd >> 1;
  const L ln(half);
  const long units = a.n * st.splits;
  for (long unit = (long)blockIdx.x * 4 + (threadIdx.x >> 6); unit < units;
       unit += (long)gridDim.x * 4) {
    const long r = unit / st.splits;
    const int s0 = (int)(unit - r * st.splits) * st.per, s1 = min(s0 + st.per, st.q + st.k);
    float cs[VEC], sn[VEC];
    ln.factors(a, r, cs, sn);
    auto steps = [&](int b, int e, int heads, const T* x, T* y, const T* g) {
      if (b >= e) return;
      float glo[VEC], ghi[VEC];
      L::widen(ln.run(g + ln.j0), glo);
      L::widen(ln.run(g + ln.j0 + half), ghi);
      for (int s = b; s < e; s += U) {
        u32x4 lo[U], hi[U];
  #pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = (s + u) * L::HPW + ln.head;
          const bool in = s + u < e && h < heads;
          const T* p = x + (long)(in ? h : 0) * a.hd + ln.j0;
          lo[u] = in ? ln.run(p) : u32x4{0, 0, 0, 0};
          hi[u] = in ? ln.run(p + half) : u32x4{0, 0, 0, 0};
        }
  #pragma unroll
        for (int u = 0; u < U; ++u) {
          if (s + u >= e) break;
          const int h = (s + u) * L::HPW + ln.head;
          float l[VEC], m[VEC], ss = 0.f;
          L::widen(lo[u], l);
          L::widen(hi[u], m);
  #pragma unroll
          for (int k = 0; k < VEC; ++k) ss = fmaf(l[k], l[k], fmaf(m[k], m[k], ss));
          const float inv = 1.0f / sqrtf(head_sum<LPH>(ss) / (float)a.hd + a.eps);
          float yl[VEC], yh[VEC];
  #pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float nl = l[k] * inv * glo[k], nh = m[k] * inv * ghi[k];
            yl[k] = rope_a(nl, nh, cs[k], sn[k]);
            yh[k] = rope_b(nl, nh, cs[k], sn[k]);
          }
          if (h < heads && ln.on) {
            T* o = y + (long)h * a.hd + ln.j0;
            *reinterpret_cast<u32x4*>(o) = L::narrow(yl);
            *reinterpret_cast<u32x4*>(o + half) = L::narrow(yh);
          }
        }
      }
    };
    steps(s0, min(s1, st.q), a.H, static_cast<const T*>(a.q) + r * a.q_rs,
          static_cast<T*>(a.q_out) + r * a.q_out_rs, static_cast<const T*>(a.gq));
    steps(max(s0 - st.q, 0), s1 - st.q, a.G, static_cast<const T*>(a.k) + r * a.k_rs,
          static_cast<T*>(a.k_out) + r * a.k_out_rs, static_cast<const T*>(a.gk));
  }
}

// Backward: the grid's waves walk the (row, part) units; a lane keeps the gain gradients of its runs in
// registers until the end, then the heads of a wave meet by shuffles and the waves in LDS.  8192 rows of 32
// bf16 heads of 128: 46 us (4.4 TB/s of two reads and a write), and 5 for the gains' sums; 2047 rows of 20 fp32
// heads of 64: 10 and 3.  186 registers in bf16 leave two waves a SIMD, half of those the grid brings; 129 in fp32, three.
template <typename T, int LPH>
__global__ __launch_bounds__(256) void qk_norm_rope_back_kernel(QkArgs a, QkSteps st) {
  using L = QkLane<T, LPH>;
  constexpr int VEC = L::VEC;
  __shared__ float sum[4][2][256];
  const int half = a.hd >> 1, wave = threadIdx.x >> 6;
  const L ln(half);
  float dg[2][2][VEC] = {};  // [q, k][low, high]
  const long units = a.n * st.splits;
  for (long unit = (long)blockIdx.x * 4 + wave; unit < units; unit += (long)gridDim.x * 4) {
    const long r = unit / st.splits;
    const int s0 = (int)(unit - r * st.splits) * st.per, s1 = min(s0 + st.per, st.q + st.k);
    float cs[VEC], sn[VEC];
    ln.factors(a, r, cs, sn);
    auto steps = [&](int b, int e, int heads, const T* x, const T* dy, T* dx, const T* g,
                     float (&acc)[2][VEC]) {
      constexpr int U = 2;
      if (b >= e) return;
      float gain[2][VEC];
      L::widen(ln.run(g + ln.j0), gain[0]);
      L::widen(ln.run(g + ln.j0 + half), gain[1]);
      for (int s = b; s < e; s += U) {
        u32x4 wx[U][2], wd[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = (s + u) * L::HPW + ln.head;
          const bool in = s + u < e && h < heads;
          const long at = (long)(in ? h : 0) * a.hd + ln.j0;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            wx[u][t] = in ? ln.run(x + at + t * half) : u32x4{0, 0, 0, 0};
            wd[u][t] = in ? ln.run(dy + at + t * half) : u32x4{0, 0, 0, 0};
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (s + u >= e) break;
          const int h = (s + u) * L::HPW + ln.head;
          float xv[2][VEC], d[2][VEC], lo[VEC], hi[VEC], ss = 0.f;
          L::widen(wx[u][0], xv[0]);
          L::widen(wx[u][1], xv[1]);
          L::widen(wd[u][0], lo);
          L::widen(wd[u][1], hi);
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            d[0][k] = rope_a(lo[k], hi[k], cs[k], -sn[k]);
            d[1][k] = rope_b(lo[k], hi[k], cs[k], -sn[k]);
            ss = fmaf(xv[0][k], xv[0][k], fmaf(xv[1][k], xv[1][k], ss));
          }
          // lanes past the last head hold zeros, whose factor would be infinite without eps, and 0 * inf nan
          const float root = sqrtf(head_sum<LPH>(ss) / (float)a.hd + a.eps);
          const float inv = h < heads ? 1.0f / root : 0.f;
          float dot = 0.f;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
              xv[t][k] *= inv;
              acc[t][k] = fmaf(d[t][k], xv[t][k], acc[t][k]);
              d[t][k] *= gain[t][k];
              dot = fmaf(d[t][k], xv[t][k], dot);
            }
          dot = head_sum<LPH>(dot) / (float)a.hd;
          if (h < heads && ln.on) {
            T* o = dx + (long)h * a.hd + ln.j0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
              for (int k = 0; k < VEC; ++k) d[t][k] = inv * (d[t][k] - xv[t][k] * dot);
              *reinterpret_cast<u32x4*>(o + t * half) = L::narrow(d[t]);
            }
          }
        }
      }
    };
    steps(s0, min(s1, st.q), a.H, static_cast<const T*>(a.q) + r * a.q_rs,
          static_cast<const T*>(a.dq_in) + r * a.dq_in_rs, static_cast<T*>(a.q_out) + r * a.q_out_rs,
          static_cast<const T*>(a.gq), dg[0]);
    steps(max(s0 - st.q, 0), s1 - st.q, a.G, static_cast<const T*>(a.k) + r * a.k_rs,
          static_cast<const T*>(a.dk_in) + r * a.dk_in_rs, static_cast<T*>(a.k_out) + r * a.k_out_rs,
          static_cast<const T*>(a.gk), dg[1]);
  }
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        float v = dg[b][t][k];
#pragma unroll
        for (int o = LPH; o < 64; o <<= 1) v += __shfl_xor(v, o);
        if (ln.head == 0 && ln.on) sum[wave][b][t * half + ln.j0 + k] = v;
      }
  __syncthreads();
  float* out = a.part + (long)blockIdx.x * 2 * a.hd;
  for (int i = threadIdx.x; i < 2 * a.hd; i += 256) {
    const int b = i / a.hd, c = i - b * a.hd;
    out[i] = ((sum[0][b][c] + sum[1][b][c]) + sum[2][b][c]) + sum[3][b][c];
  }
}

// Gain gradients: the workgroups' partial sums, 16 columns a workgroup; each of its 64 thread rows takes
// every 64th partial, four loads in flight, and they meet in LDS in order.
__global__ __launch_bounds__(1024) void qk_gain_grad_kernel(const float* __restrict__ part, int n_wg,
                                                            int hd, float* __restrict__ dgq,
                                                            float* __restrict__ dgk) {
  __shared__ float s[64][17];
  const int col = threadIdx.x & 15, sub = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  float t = 0.f;
  if (c < 2 * hd)
    for (int w = sub; w < n_wg; w += 256) {
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        v[u] = w + 64 * u < n_wg ? part[(long)(w + 64 * u) * 2 * hd + c] : 0.f;
      t += ((v[0] + v[1]) + v[2]) + v[3];
    }
  s[sub][col] = t;
  __syncthreads();
  for (int half = 32; half > 0; half >>= 1) {
    if (sub < half) s[sub][col] += s[sub + half][col];
    __syncthreads();
  }
  if (sub != 0 || c >= 2 * hd) return;
  if (c < hd) {
    if (dgq) dgq[c] = s[0][col];
  } else if (dgk) {
    dgk[c - hd] = s[0][col];
  }
}

// Factor rows that turn nothing: what the QKV epilogue is given where the norm and the rotation
// follow it in a pass of their own.
__global__ __launch_bounds__(256) void unit_factor_kernel(f32x2* __restrict__ rope, long n) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i < n) rope[i] = f32x2{1.f, 0.f};
}

}  // namespace alr
