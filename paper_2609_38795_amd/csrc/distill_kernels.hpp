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
  const float* w_sum;    // sum of the weights as the two halves of a double, or null: each workgroup forms it
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

__device__ __forceinline__ float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// One workgroup per row, which reads it for the sums and, with a gradient, again, mostly from the last-level
// cache (keeping part of a row of 128256 in LDS or registers in between measured no faster).  The running maximum of the sums
// costs one exponential a chunk; they are formed while later loads are under way.  What bounds it is HBM.  Call
// times: the loss of 768 fp32 rows of 152064, 77 us (6.1 TB/s); with the gradient in bf16, 4096 rows of 32000, 141
// us and 2048 rows of 128256, 256 us (3.7 and 4.1 TB/s of one read and one write; the second read is the rest).
//
// Chunks that hold listed tokens (eight at most) are left out of both passes: lane j of every wave loads entry
// j's chunk at the start, and the first wave's lanes take them at the end of each pass, all at once.
template <typename T, int THREADS, bool GRAD>
__global__ __launch_bounds__(THREADS) void distill_rows_kernel(DistillArgs a) {
  constexpr int NW = THREADS / 64, EPC = RowChunks<T>::EPC;
  __shared__ TailSum red[NW];
  __shared__ double red64[NW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double inv_w = 0.0;  // 64 bits: 1 / W may lie outside fp32 where a weight's share of W does not
  if constexpr (GRAD) {
    const double W = a.w_sum ? __hiloint2double(__float_as_int(a.w_sum[1]), __float_as_int(a.w_sum[0]))
                             : weight_sum(a.weight, a.n, red64);
    inv_w = W != 0.0 ? (double)a.scale / W : 0.0;
    if (a.up) inv_w *= (double)a.up[0];
  }
  for (long r = blockIdx.x; r < a.n; r += gridDim.x) {
    RowChunks<T> row(static_cast<const T*>(a.z) + r * a.z_rs, a.V);
    const int cpt = (row.nch + THREADS - 1) / THREADS;  // chunk i of a thread: i * THREADS + its index
    T* dz = GRAD ? static_cast<T*>(a.dz) + r * a.dz_rs : nullptr;
    const bool vec =
        ((reinterpret_cast<uintptr_t>(dz) - (uintptr_t)row.mis * sizeof(T)) & 15) == 0;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {  // the row is not read
      if (threadIdx.x == 0) a.row_loss[r] = 0.f;
      if constexpr (GRAD) {
        const float zero[EPC] = {};
        for (int i = 0; i < cpt; ++i) {
          const int c = i * THREADS + (int)threadIdx.x;
          if (c < row.nch) store_chunk(row, dz, vec, c, zero);
        }
      }
      continue;
    }
    row.edges();
    // The label: an id outside the vocabulary is passed over with its probability.  hit: bit i % 32 tells that
    // chunk i of this thread may hold a listed token (is_hit, that it does).
    int id[DISTILL_K], lane_id = -1;
    uint32_t hit = 0;
#pragma unroll
    for (int j = 0; j < DISTILL_K; ++j) {
      id[j] = a.ids[r * DISTILL_K + j];
      if (id[j] < 0 || id[j] >= a.V) id[j] = -1;
      const int c = (id[j] + row.mis) / EPC;
      if (id[j] >= 0 && c % THREADS == (int)threadIdx.x) hit |= 1u << (c / THREADS & 31);
      if (lane == j) lane_id = id[j];
    }
    const int lane_c = lane_id >= 0 ? (lane_id + row.mis) / EPC : 0;
    const u32x4 lane_x = row.whole(lane_c, row.load(lane_c));
    const float lane_lp = lane_id >= 0 ? a.logp[r * DISTILL_K + lane] : -INFINITY;
    const float tau = a.tail[r];
    auto is_hit = [&](int i, int c) {
      if (!(hit >> (i & 31) & 1)) return false;
      bool in = false;
#pragma unroll
      for (int j = 0; j < DISTILL_K; ++j) in |= id[j] >= 0 && (id[j] + row.mis) / EPC == c;
      return in;
    };

    TailSum t = {-INFINITY, 0.f};
    auto add_up = [&](const float(&v)[EPC]) {
      float m = t.m;
#pragma unroll
      for (int k = 0; k < EPC; ++k) m = fmaxf(m, v[k]);
      const float ref = m == -INFINITY ? 0.f : m;
      float s = t.s * fast_exp2((t.m - ref) * LOG2E);
#pragma unroll
      for (int k = 0; k < EPC; ++k) s += fast_exp2((v[k] - ref) * LOG2E);
      t = {m, s};
    };
    walk<4, THREADS>(row, (int)threadIdx.x, 0, cpt, [&](int i, int c, u32x4 x) {
      float v[EPC];
      unpack<T>(x, v);
      if (!is_hit(i, c)) add_up(v);
    });
    // the entries, in the first eight lanes of each wave: their logits, which of a chunk's values are listed
    // (in the first lane of each chunk), which is the first entry of its token
    float lane_v[EPC], lane_z = -INFINITY;
    unpack<T>(lane_x, lane_v);
#pragma unroll
    for (int k = 0; k < EPC; ++k)
      if (lane_id >= 0 && row.first(lane_c) + k == lane_id) lane_z = lane_v[k];
    uint32_t in = 0;
    bool first_c = lane_id >= 0, first = first_c;
#pragma unroll
    for (int j = 0; j < DISTILL_K; ++j) {
      if (id[j] < 0 || (id[j] + row.mis) / EPC != lane_c) continue;
      in |= 1u << (id[j] + row.mis) % EPC;
      if (j < lane) first_c = false;
      if (j < lane && id[j] == lane_id) first = false;
    }
    if (wave == 0 && first_c) {
      float v[EPC];
#pragma unroll
      for (int k = 0; k < EPC; ++k) v[k] = in >> k & 1 ? -INFINITY : lane_v[k];
      add_up(v);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t = merge_tail(t, TailSum{__shfl_xor(t.m, o), __shfl_xor(t.s, o)});
    if constexpr (NW > 1) {
      if (lane == 0) red[wave] = t;
      __syncthreads();
      t = red[0];
#pragma unroll
      for (int k = 1; k < NW; ++k) t = merge_tail(t, red[k]);
      __syncthreads();  // red is written again for the next row
    }

    const float lane_pi = expf(lane_lp);  // 0 where there is no entry
    const float mx = fmaxf(t.m, wave_max(lane_z));
    const float ref = mx == -INFINITY ? 0.f : mx;
    const float s = t.s * expf(t.m - ref) + lane_value(group_sum<8>(first ? expf(lane_z - ref) : 0.f), 0);
    const float ls = logf(s);
    const float lq_tail = (t.m - ref) + (logf(t.s) - ls);
    const float terms = lane_pi > 0.f ? lane_pi * ((lane_z - ref) - ls) : 0.f;
    const float loss = (tau > 0.f ? -tau * lq_tail : 0.f) - lane_value(group_sum<8>(terms), 0);
    const float mass = tau + lane_value(group_sum<8>(lane_pi), 0);
    if (threadIdx.x == 0) a.row_loss[r] = loss;
    if constexpr (GRAD) {
      const float cw = (float)(inv_w * (double)w);
      const float ref_t = t.m == -INFINITY ? 0.f : t.m;
      // no tail at all: every value outside the list is -inf and gets 0
      const float bt = t.s == 0.f ? 0.f : cw * (mass * expf(lq_tail) - tau) / t.s;
      walk<4, THREADS>(row, (int)threadIdx.x, 0, cpt, [&](int i, int c, u32x4 x) {
        if (c >= row.nch || is_hit(i, c)) return;
        float v[EPC];
        unpack<T>(x, v);
#pragma unroll
        for (int k = 0; k < EPC; ++k) v[k] = bt * fast_exp2((v[k] - ref_t) * LOG2E);
        store_chunk(row, dz, vec, c, v);
      });
      if (wave == 0) {
#pragma unroll
        for (int k = 0; k < EPC; ++k) {
          const int e = row.first(lane_c) + k;
          float d = mass * expf((lane_v[k] - ref) - ls);
#pragma unroll
          for (int j = 0; j < DISTILL_K; ++j)
            if (id[j] == e) d -= lane_value(lane_pi, j);
          lane_v[k] = in >> k & 1 ? cw * d : bt * fast_exp2((lane_v[k] - ref_t) * LOG2E);
        }
        if (first_c) store_chunk(row, dz, vec, lane_c, lane_v);
      }
    }
  }
}

// out[0], out[1] = low and high half of the weights' sum, ahead of the gradients of many rows: the two floats
// that the loss and W are written to afterwards (aligned to 4 bytes only).
__global__ __launch_bounds__(1024) void weight_sum_kernel(const float* __restrict__ w, long n,
                                                          float* __restrict__ out) {
  __shared__ double red[16];
  const double W = weight_sum(w, n, red);
  if (threadIdx.x == 0) {
    out[0] = __int_as_float(__double2loint(W));
    out[1] = __int_as_float(__double2hiint(W));
  }
}

}  // namespace alr
