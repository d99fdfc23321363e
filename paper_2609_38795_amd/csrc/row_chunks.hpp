// Rows of logits as 16-byte chunks, for the kernels that walk a whole vocabulary row per
// workgroup (distillation loss, sampling): any row length, stride and alignment.
#pragma once

#include "device_common.hpp"

namespace alr {

constexpr float LOG2E = 1.44269504088896340736f;

// One row of V values of T, whose first value may sit anywhere within a 16-byte line: chunk c
// holds the values [c * EPC - mis, c * EPC - mis + EPC) that exist, and -inf in the places of the others.
// Chunks [cf, cl) lie inside the row and are moved by one 16-byte access; the one or two at its ends are read value
// by value, once per row (edges()), so nothing outside the row is touched.
template <typename T>
struct RowChunks {
  static constexpr int EPC = 16 / (int)sizeof(T);
  static constexpr uint32_t NEG = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;  // -inf
  const T* p;
  int V, mis, nch, cf, cl;
  u32x4 e0, e1;  // the chunks at the ends

  __device__ __forceinline__ RowChunks(const T* row, int V_) : p(row), V(V_) {
    mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    nch = (V + mis + EPC - 1) / EPC;
    cf = mis ? 1 : 0;
    cl = (V + mis) / EPC;
  }
  __device__ __forceinline__ void edges() {
    e0 = e1 = u32x4{NEG, NEG, NEG, NEG};
    if (cf) e0 = edge(0);
    if (cl < nch) e1 = edge(nch - 1);
  }
  __device__ __forceinline__ int first(int c) const { return c * EPC - mis; }
  __device__ __forceinline__ bool inside(int c) const { return c >= cf && c < cl; }
  // What load() gives is chunk c where that lies inside the row; whole() makes it chunk c in any
  // case.  In two steps, so that several loads can be under way before the first is looked at.
  __device__ __forceinline__ u32x4 load(int c) const {
    if (cf >= cl) return u32x4{NEG, NEG, NEG, NEG};
    return *reinterpret_cast<const u32x4*>(p + first(min(max(c, cf), cl - 1)));
  }
  __device__ __forceinline__ u32x4 whole(int c, u32x4 w) const {
    if (!inside(c)) {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = c == 0 && cf ? e0[k] : c == nch - 1 ? e1[k] : NEG;
    }
    return w;
  }
  __device__ __forceinline__ u32x4 edge(int c) const {
    u32x4 w;
    const int e = first(c);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        const int a = e + k;
        w[k] = a >= 0 && a < V ? __float_as_uint(p[a]) : NEG;
      } else {
        const int a = e + 2 * k, b = a + 1;
        const uint32_t lo = a >= 0 && a < V ? (uint32_t)p[a] : 0xFF80u;
        const uint32_t hi = b >= 0 && b < V ? (uint32_t)p[b] : 0xFF80u;
        w[k] = lo | hi << 16;
      }
    }
    return w;
  }
};

template <typename T>
__device__ __forceinline__ void unpack(u32x4 w, float (&v)[RowChunks<T>::EPC]) {
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

// f(i, c, chunk c) for the chunks c = c0 + i * STRIDE, i0 <= i < i1.  U loads go out ahead of the U chunks in
// hand, so that a wave always has some under way.
template <int U, int STRIDE, typename T, typename F>
__device__ __forceinline__ void walk(const RowChunks<T>& row, int c0, int i0, int i1, F f) {
  u32x4 w[U], next[U];
  if (i0 >= i1) return;
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = row.load(c0 + (i0 + u) * STRIDE);
#pragma unroll 1
  for (int i = i0; i < i1; i += U) {
    if (i + U < i1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = row.load(c0 + (i + U + u) * STRIDE);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= i1) break;
      const int c = c0 + (i + u) * STRIDE;
      f(i + u, c, row.whole(c, w[u]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
  }
}

// Writes chunk c of a row that `g` describes to the row `out`, rounded once to T; vec: out's chunks
// are 16-byte aligned where g's are.
template <typename T>
__device__ __forceinline__ void store_chunk(const RowChunks<T>& g, T* out, bool vec, int c,
                                            const float (&v)[RowChunks<T>::EPC]) {
  constexpr int EPC = RowChunks<T>::EPC;
  const int e0 = g.first(c);
  if (vec && g.inside(c)) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4)
        w[k] = __float_as_uint(v[k]);
      else
        w[k] = pack2bf(v[2 * k], v[2 * k + 1]);
    }
    *reinterpret_cast<u32x4*>(out + e0) = w;
    return;
  }
#pragma unroll
  for (int k = 0; k < EPC; ++k)
    if (e0 + k >= 0 && e0 + k < g.V) Elt<T>::st(out + e0 + k, v[k]);
}

}  // namespace alr
