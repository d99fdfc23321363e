// The distillation loss on top-8 + tail labels and its gradient (Sec. 3.1, Eq. 1).
//
// Row r holds a drafter's logits z; its label lists up to 8 tokens with log-probs (ids, logp) and
// the mass of all others (tail).  With q = softmax(z), pi_j = exp(logp_j), tau = tail, S the set of
// listed tokens, q_tail = sum of q over the tokens outside S, and P = sum_j pi_j + tau:
//   row_loss   = - sum_j pi_j log q_(id_j) - tau log q_tail          (0 log 0 = 0)
//   loss       = scale * sum_r w_r row_loss_r / W,  W = sum_r w_r    (0 where W is 0)
//   d loss/dz_v = scale w / W * (P q_v - sum_{j: id_j = v} pi_j)     for v in S
//               = scale w / W * (P q_tail - tau) * q_v / q_tail      otherwise
// The tail is summed over the tokens outside S directly, with a maximum of its own, so nothing
// cancels where the listed tokens hold nearly all mass and q_v / q_tail never overflows.
#pragma once

#include "row_chunks.hpp"

namespace alr {

constexpr int DISTILL_K = 8;

struct DistillArgs {
  const void* z;
  long z_rs;
  const int* ids;        // [n, 8]
  const float* logp;     // [n, 8]
  const float* tail;     // [n]
  const float* weight;   // [n] or null: 1
  const float* up;       // gradient of the loss, one value, or null: 1
  float scale;
  long n;
  int V;
  float* row_loss;       // [n]
  void* dz;              // rows of V, or unused
  long dz_rs;
};

// Sum of v over the workgroup in a fixed order, in every thread; red: one entry a wave.
__device__ __forceinline__ double block_sum_f64(double v, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) t += red[i];
  __syncthreads();
  return t;
}

__device__ __forceinline__ double weight_sum(const float* w, long n, double* red) {
  double s = 0.0;
  if (w) {
    for (long i = threadIdx.x; i < n; i += blockDim.x) s += (double)w[i];
    return block_sum_f64(s, red);
  }
  return (double)n;
}

// loss_out = (scale * sum w row_loss / W, W), summed in 64 bits in an order that only n fixes.
__global__ __launch_bounds__(1024) void distill_reduce_kernel(const float* __restrict__ row_loss,
                                                              const float* __restrict__ weight,
                                                              long n, float scale,
                                                              float* __restrict__ loss_out) {
  __shared__ double red[16];
  double s = 0.0;
  for (long i = threadIdx.x; i < n; i += blockDim.x) {
    const float w = weight ? weight[i] : 1.f;
    if (w != 0.f) s += (double)w * (double)row_loss[i];
  }
  s = block_sum_f64(s, red);
  const double W = weight_sum(weight, n, red);
  if (threadIdx.x == 0) {
    loss_out[0] = W != 0.0 ? (float)((double)scale * s / W) : 0.f;
    loss_out[1] = (float)W;
  }
}

// max and sum of exp(z - max): the running pair of a softmax
struct TailSum {
  float m, s;
};
__device__ __forceinline__ TailSum merge_tail(TailSum a, TailSum b) {
  const float m = fmaxf(a.m, b.m), ref = m == -INFINITY ? 0.f : m;
  return {m, a.s * fast_exp2((a.m - ref) * LOG2E) + b.s * fast_exp2((b.m - ref) * LOG2E)};
}

// One workgroup per row.  Each wave owns a run of `cpw` x 64 chunks of the row.
template <typename T, int THREADS, bool GRAD>
__global__ __launch_bounds__(THREADS) void distill_rows_kernel(DistillArgs a) {
  constexpr int NW = THREADS / 64, EPC = RowChunks<T>::EPC;
  __shared__ TailSum red[NW];
  __shared__ double red64[NW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float inv_w = 0.f;
  if constexpr (GRAD) {
    const double W = weight_sum(a.weight, a.n, red64);
    inv_w = W != 0.0 ? (float)((double)a.scale / W) : 0.f;
    if (a.up) inv_w *= a.up[0];
  }
  for (long r = blockIdx.x; r < a.n; r += gridDim.x) {
    RowChunks<T> row(static_cast<const T*>(a.z) + r * a.z_rs, a.V);
    const int cpw = (row.nch + THREADS - 1) / THREADS;
    T* dz = GRAD ? static_cast<T*>(a.dz) + r * a.dz_rs : nullptr;
    const bool vec =
        ((reinterpret_cast<uintptr_t>(dz) - (uintptr_t)row.mis * sizeof(T)) & 15) == 0;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {  // the row is not read
      if (threadIdx.x == 0) a.row_loss[r] = 0.f;
      if constexpr (GRAD) {
        const float zero[EPC] = {};
        for (int i = 0; i < cpw; ++i) {
          const int c = (wave * cpw + i) * 64 + lane;
          if (c < row.nch) store_chunk(row, dz, vec, c, zero);
        }
      }
      continue;
    }
    row.edges();
    // the label; an id outside the vocabulary is passed over with its probability
    int id[DISTILL_K];
    float pi[DISTILL_K], zj[DISTILL_K];
    bool first[DISTILL_K];
    uint32_t hit = 0;  // bit i % 32: chunk i of this thread may hold a listed token
#pragma unroll
    for (int j = 0; j < DISTILL_K; ++j) {
      id[j] = a.ids[r * DISTILL_K + j];
      const bool ok = id[j] >= 0 && id[j] < a.V;
      if (!ok) id[j] = -1;
      pi[j] = ok ? expf(a.logp[r * DISTILL_K + j]) : 0.f;
      zj[j] = ok ? row.at(id[j]) : -INFINITY;
      first[j] = ok;
#pragma unroll
      for (int k = 0; k < j; ++k)
        if (id[k] == id[j]) first[j] = false;
      const int c = (id[j] + row.mis) / EPC, g = c >> 6;
      if (ok && (c & 63) == lane && g / cpw == wave) hit |= 1u << ((g - wave * cpw) & 31);
    }
    const float tau = a.tail[r];
    auto listed = [&](int e) {
      bool in = false;
#pragma unroll
      for (int j = 0; j < DISTILL_K; ++j) in |= id[j] == e && e >= 0;
      return in;
    };

    TailSum t = {-INFINITY, 0.f};
    for (int i = 0; i < cpw; ++i) {
      const int c = (wave * cpw + i) * 64 + lane;
      if (c >= row.nch) break;
      float v[EPC];
      unpack<T>(row.whole(c, row.load(c)), v);
      if (hit >> (i & 31) & 1)
#pragma unroll
        for (int k = 0; k < EPC; ++k)
          if (listed(row.first(c) + k)) v[k] = -INFINITY;
      float m = t.m;
#pragma unroll
      for (int k = 0; k < EPC; ++k) m = fmaxf(m, v[k]);
      const float ref = m == -INFINITY ? 0.f : m;
      float s = t.s * fast_exp2((t.m - ref) * LOG2E);
#pragma unroll
      for (int k = 0; k < EPC; ++k) s += fast_exp2((v[k] - ref) * LOG2E);
      t = {m, s};
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t = merge_tail(t, TailSum{__shfl_xor(t.m, o), __shfl_xor(t.s, o)});
    if (lane == 0) red[wave] = t;
    __syncthreads();
    t = red[0];
#pragma unroll
    for (int k = 1; k < NW; ++k) t = merge_tail(t, red[k]);
    __syncthreads();  // red is written again for the next row

    float mx = t.m;
#pragma unroll
    for (int j = 0; j < DISTILL_K; ++j) mx = fmaxf(mx, first[j] ? zj[j] : -INFINITY);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float s = t.s * expf(t.m - ref);
#pragma unroll
    for (int j = 0; j < DISTILL_K; ++j)
      if (first[j]) s += expf(zj[j] - ref);
    const float ls = logf(s);
    const float lq_tail = (t.m - ref) + (logf(t.s) - ls);
    float loss = tau > 0.f ? -tau * lq_tail : 0.f, mass = tau;
#pragma unroll
    for (int j = 0; j < DISTILL_K; ++j) {
      if (pi[j] > 0.f) loss -= pi[j] * ((zj[j] - ref) - ls);
      mass += pi[j];
    }
    if (threadIdx.x == 0) a.row_loss[r] = loss;
    if constexpr (GRAD) {
      const float cw = inv_w * w;
      const float ref_t = t.m == -INFINITY ? 0.f : t.m;
      // no tail at all: every value outside the list is -inf and gets 0
      const float bt = t.s == 0.f ? 0.f : cw * (mass * expf(lq_tail) - tau) / t.s;
      for (int i = 0; i < cpw; ++i) {
        const int c = (wave * cpw + i) * 64 + lane;
        if (c >= row.nch) break;
        float v[EPC];
        unpack<T>(row.whole(c, row.load(c)), v);
        float g[EPC];
#pragma unroll
        for (int k = 0; k < EPC; ++k) g[k] = bt * fast_exp2((v[k] - ref_t) * LOG2E);
        if (hit >> (i & 31) & 1)
#pragma unroll
          for (int k = 0; k < EPC; ++k) {
            const int e = row.first(c) + k;
            if (!listed(e)) continue;
            float d = mass * expf((v[k] - ref) - ls);
#pragma unroll
            for (int j = 0; j < DISTILL_K; ++j)
              if (id[j] == e) d -= pi[j];
            g[k] = cw * d;
          }
        store_chunk(row, dz, vec, c, g);
      }
    }
  }
}

}  // namespace alr
