// One token per row of logits from a given uniform number: temperature, top-k, top-p, min-p.
//
// Weights w_v = exp((z_v - max z) / T).  Tokens are ranked by decreasing logit, equal logits by
// increasing id, and a prefix of the ranking is kept: the shortest of the first k, the smallest
// prefix that holds at least p of the first k's weight, and the tokens with w >= min_p.  The token is
// the first, in the order of the ids, whose cumulative kept weight exceeds u times the total.
//
// Each of those prefixes is "logits above a cut, and the first few ids at the cut", so no row is
// sorted: a histogram over (max - z) finds the interval of logits that the k-th token, or the p-th of
// the weight, falls into, histograms over the bits of the logits narrow it to one value, and a scan
// over the ids settles the ties.
//
// Weights are whole numbers of 2^-shift (shift >= 43, from 64-bit exponentials), so every sum is exact
// and does not depend on the order in which it is formed: what a row gives depends on its own values
// alone, and is what 64-bit arithmetic gives up to 2^-shift of the largest weight.
#pragma once

#include "row_chunks.hpp"

namespace alr {

struct SampleArgs {
  const void* z;
  long z_rs;
  int z_perm;             // row r at z + perm[r] * z_rs instead of r * z_rs
  const int* perm;        // caller's index of row r, or null: r
  int block, s;           // uniform, forced, tokens and logp at [index * block + s]
  long n;
  int V, shift;
  const float* temperature;  // [index], or null: 1
  const int* top_k;          // [index], or null; <= 0: off
  const float* top_p;        // [index], or null; >= 1 or NaN: off
  const float* min_p;        // [index], or null; <= 0 or NaN: off
  const float* uniform;
  const int* forced;      // or null; fed instead of the token where >= 0
  int* next_tok;          // [r] or null: the token to feed
  int* tokens;
  float* logp;            // or null
};

typedef unsigned long long u64;

constexpr int SAMPLE_BINS = 2048;
constexpr int SAMPLE_GROUPS = 4;  // parts of a wave's run whose weights are summed apart

__device__ __forceinline__ u64 shfl_xor_u64(u64 v, int o) {
  const uint32_t lo = __shfl_xor((uint32_t)v, o), hi = __shfl_xor((uint32_t)(v >> 32), o);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 shfl_up_u64(u64 v, int o) {
  const uint32_t lo = __shfl_up((uint32_t)v, o), hi = __shfl_up((uint32_t)(v >> 32), o);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += shfl_xor_u64(v, o);
  return v;
}
// sum over the lanes before this one
__device__ __forceinline__ u64 wave_before_u64(u64 v) {
  u64 t = v;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 x = shfl_up_u64(t, o);
    if (lane >= o) t += x;
  }
  return t - v;
}

// Unsigned order of the floats' order; -0 as +0.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k);
}

// 2^y for y <= 0 in 64 bits, times 2^shift: y = n + f with |f| <= 1/2, 2^f by the series of
// exp(f ln 2) up to the 11th power (the next term is below 2^-47).
__device__ __forceinline__ double exp2_scaled(double y, int shift) {
  constexpr double MAGIC = 6755399441055744.0;  // 1.5 x 2^52: adding it rounds to a whole number
  y = fmax(y, -1000.0);
  const double t = y + MAGIC;
  const int n = (int)(uint32_t)__double_as_longlong(t);
  const double f = y - (t - MAGIC);
  constexpr double L = 0.693147180559945309417232;
  constexpr double c2 = L * L / 2, c3 = c2 * L / 3, c4 = c3 * L / 4, c5 = c4 * L / 5, c6 = c5 * L / 6,
                   c7 = c6 * L / 7, c8 = c7 * L / 8, c9 = c8 * L / 9, c10 = c9 * L / 10,
                   c11 = c10 * L / 11;
  double p = fma(f, c11, c10);
  p = fma(f, p, c9);
  p = fma(f, p, c8);
  p = fma(f, p, c7);
  p = fma(f, p, c6);
  p = fma(f, p, c5);
  p = fma(f, p, c4);
  p = fma(f, p, c3);
  p = fma(f, p, c2);
  p = fma(f, p, L);
  p = fma(f, p, 1.0);
  return __builtin_ldexp(p, n + shift);
}

// The weight of a logit, in units of 2^-shift of the largest one's.
struct Weigher {
  double m, c;  // the row's largest logit; log2(e) / T
  int shift;
  __device__ __forceinline__ double of(float z) const {
    return exp2_scaled(((double)z - m) * c, shift);
  }
  __device__ __forceinline__ u64 units(float z) const {  // of() <= 2^51: rounded by adding 2^52
    constexpr double ONE52 = 4503599627370496.0;
    return (u64)__double_as_longlong(of(z) + ONE52) & ((1ull << 52) - 1);
  }
};

struct SampleShared {
  uint32_t cnt[2][SAMPLE_BINS];  // of the first level, of the narrowing ones
  u64 mass[2][SAMPLE_BINS];
  u64 scan_c[16], scan_m[16];
  u64 group[16][SAMPLE_GROUPS];
  float fred[16];
  uint32_t ured[2][16];
  int bin;
  u64 above_c, above_m;
};

template <int NW>
__device__ __forceinline__ float block_max_f(float v, SampleShared& sh) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) sh.fred[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = sh.fred[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) t = fmaxf(t, sh.fred[i]);
  __syncthreads();
  return t;
}

// min and max of unsigned values over the workgroup
template <int NW>
__device__ __forceinline__ void block_range(uint32_t& lo, uint32_t& hi, SampleShared& sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor(lo, o));
    hi = max(hi, (uint32_t)__shfl_xor(hi, o));
  }
  if ((threadIdx.x & 63) == 0) {
    sh.ured[0][threadIdx.x >> 6] = lo;
    sh.ured[1][threadIdx.x >> 6] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    lo = min(lo, sh.ured[0][i]);
    hi = max(hi, sh.ured[1][i]);
  }
  __syncthreads();
}

template <int THREADS>
__device__ __forceinline__ void clear_bins(SampleShared& sh, int level) {
  for (int b = threadIdx.x; b < SAMPLE_BINS; b += THREADS) {
    sh.cnt[level][b] = 0;
    sh.mass[level][b] = 0;
  }
  __syncthreads();
}

// What is looked for in the bins of a level: the bin with the token of rank `count`
// (counting from 1), or the one in which the weight of the ranking's prefix reaches `mass`, or, before the
// whole weight is known, `share` of the weight that the bins hold.
struct Aim {
  bool by_mass;
  u64 count, mass;
  double share;  // > 0: mass = share of the total, rounded up
};

// Finds the bin; above_c and above_m come in as what ranks before the level's bins and go out as
// what ranks before the bin.  Returns -1 where the level's tokens are fewer than `count`.
// Everything else that needs the level's total weight gets it in `total`.
template <int THREADS>
__device__ __forceinline__ int find_bin(SampleShared& sh, int level, Aim& aim, u64& above_c,
                                        u64& above_m, u64& total) {
  constexpr int NW = THREADS / 64, PER = SAMPLE_BINS / THREADS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = threadIdx.x * PER;
  u64 c = 0, m = 0;
#pragma unroll 4
  for (int i = 0; i < PER; ++i) {
    c += sh.cnt[level][b0 + i];
    m += sh.mass[level][b0 + i];
  }
  u64 c_before = wave_before_u64(c), m_before = wave_before_u64(m);
  if (lane == 63) {
    sh.scan_c[wave] = c_before + c;
    sh.scan_m[wave] = m_before + m;
  }
  if (threadIdx.x == 0) sh.bin = -1;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < wave) {
      c_before += sh.scan_c[i];
      m_before += sh.scan_m[i];
    }
    all += sh.scan_m[i];
  }
  total = all;
  if (aim.by_mass && aim.share > 0.0) {
    aim.mass = (u64)ceil(aim.share * (double)all);
    aim.share = 0.0;
  }
  if (aim.by_mass && aim.mass < 1) aim.mass = 1;
  c_before += above_c;
  m_before += above_m;
  const u64 want = aim.by_mass ? aim.mass : aim.count;
  u64 at = aim.by_mass ? m_before : c_before;
  if (at < want && at + (aim.by_mass ? m : c) >= want) {
    for (int i = 0; i < PER; ++i) {
      const u64 x = aim.by_mass ? sh.mass[level][b0 + i] : sh.cnt[level][b0 + i];
      if (at + x >= want) {
        sh.bin = b0 + i;
        sh.above_c = c_before;
        sh.above_m = m_before;
        break;
      }
      at += x;
      c_before += sh.cnt[level][b0 + i];
      m_before += sh.mass[level][b0 + i];
    }
  }
  __syncthreads();
  const int bin = sh.bin;
  if (bin >= 0) {
    above_c = sh.above_c;
    above_m = sh.above_m;
  }
  __syncthreads();  // the level's bins and sh.bin may be written again
  return bin;
}

// Where the kept prefix ends: logits above `z`, and of those equal to z the first `ties` ids.
struct Cut {
  float z;
  u64 ties;
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a) {
  constexpr int NW = THREADS / 64, EPC = RowChunks<T>::EPC;
  static_assert(SAMPLE_BINS % THREADS == 0 && NW <= 16, "bins per thread");
  __shared__ SampleShared sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long r = blockIdx.x; r < a.n; r += gridDim.x) {
    const long idx = a.perm ? (long)a.perm[r] : r, o = idx * a.block + a.s;
    const RowChunks<T> row(static_cast<const T*>(a.z) + (a.z_perm ? idx : r) * a.z_rs, a.V);
    const int cpw = (row.nch + THREADS - 1) / THREADS;
    // f(value, id) over this wave's run of the row, chunks [i0, i1) of it
    auto each = [&](int i0, int i1, auto f) {
      for (int i = i0; i < i1; ++i) {
        const int c = (wave * cpw + i) * 64 + lane;
        if (c >= row.nch) break;
        float v[EPC];
        unpack<T>(row.load(c), v);
#pragma unroll
        for (int k = 0; k < EPC; ++k) f(v[k], row.first(c) + k);
      }
    };
    auto emit = [&](int tok, float lp) {
      a.tokens[o] = tok;
      if (a.logp) a.logp[o] = lp;
      if (a.next_tok) {
        const int f = a.forced ? a.forced[o] : -1;
        a.next_tok[r] = f >= 0 ? f : max(tok, 0);
      }
    };

    float m = -INFINITY;
    each(0, cpw, [&](float z, int) { m = fmaxf(m, z); });
    m = block_max_f<NW>(m, sh);
    if (m == -INFINITY) {  // nothing to draw
      if (threadIdx.x == 0) emit(-1, -INFINITY);
      continue;
    }
    const float temp = a.temperature ? a.temperature[idx] : 1.f;
    if (!(temp > 0.f) || m == INFINITY) {  // greedy: the lowest id at the maximum
      uint32_t lo = 0xFFFFFFFFu, hi = 0;
      each(0, cpw, [&](float z, int e) {
        if (z == m) lo = min(lo, (uint32_t)e);
      });
      block_range<NW>(lo, hi, sh);
      if (threadIdx.x == 0) emit((int)lo, 0.f);
      continue;
    }
    const Weigher wt{(double)m, 1.4426950408889634074 / (double)temp, a.shift};
    const int k = a.top_k ? a.top_k[idx] : 0;
    const float p = a.top_p ? a.top_p[idx] : 1.f;
    const bool by_k = k > 0 && k < a.V, by_p = p < 1.f;
    Cut cut = {-INFINITY, 0};
    if (by_k || by_p) {
      // level 0: bins of 1/64 in (max - z) / T, the last one for all that lies below
      const float cs = fminf(64.f / temp, 1e30f);
      auto bin0 = [&](float z) { return (int)fminf((m - z) * cs, (float)(SAMPLE_BINS - 1)); };
      clear_bins<THREADS>(sh, 0);
      each(0, cpw, [&](float z, int) {
        if (z == z && z != -INFINITY) {
          const int b = bin0(z);
          if (by_k) atomicAdd(&sh.cnt[0][b], 1u);
          if (by_p) atomicAdd(&sh.mass[0][b], wt.units(z));
        }
      });
      __syncthreads();
      // narrows a bin of level 0 to one logit
      auto narrow = [&](int bin, Aim aim, u64& above_c, u64& above_m) {
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        each(0, cpw, [&](float z, int) {
          if (z == z && z != -INFINITY && bin0(z) == bin) {
            const uint32_t key = order_key(z);
            lo = min(lo, key);
            hi = max(hi, key);
          }
        });
        block_range<NW>(lo, hi, sh);
        while (lo < hi) {
          const int shift = max(0, 21 - (int)__clz(hi - lo));  // (hi - lo) >> shift < 2048
          clear_bins<THREADS>(sh, 1);
          each(0, cpw, [&](float z, int) {
            const uint32_t key = order_key(z);
            if (z == z && key >= lo && key <= hi) {
              const uint32_t b = (hi - key) >> shift;
              if (by_k) atomicAdd(&sh.cnt[1][b], 1u);
              if (by_p) atomicAdd(&sh.mass[1][b], wt.units(z));
            }
          });
          __syncthreads();
          u64 all;
          const int b = find_bin<THREADS>(sh, 1, aim, above_c, above_m, all);
          if (b < 0) break;  // not reached: the level holds what the one above it counted
          hi -= (uint32_t)b << shift;
          lo = max(lo, hi - min(hi, (1u << shift) - 1));
        }
        return key_value(hi);
      };
      u64 total, mass_k = 0;
      if (by_k) {
        u64 above_c = 0, above_m = 0;
        Aim aim{false, (u64)k, 0, 0.0};
        const int bin = find_bin<THREADS>(sh, 0, aim, above_c, above_m, total);
        if (bin >= 0) {
          cut.z = narrow(bin, aim, above_c, above_m);
          cut.ties = (u64)k - above_c;
          mass_k = above_m + cut.ties * wt.units(cut.z);
        } else {
          mass_k = total;  // fewer than k tokens can be drawn
        }
      }
      if (by_p) {
        u64 above_c = 0, above_m = 0;
        Aim aim{true, 0, 0, 0.0};
        if (by_k)
          aim.mass = p > 0.f ? (u64)ceil((double)p * (double)mass_k) : 0;
        else
          aim.share = p > 0.f ? (double)p : 0.0;
        const int bin = find_bin<THREADS>(sh, 0, aim, above_c, above_m, total);
        if (bin >= 0) {
          const float z = narrow(bin, aim, above_c, above_m);
          const u64 need = aim.mass - above_m, one = max(wt.units(z), 1ull);
          const u64 ties = (need + one - 1) / one;
          if (z > cut.z) {
            cut = {z, ties};
          } else if (z == cut.z) {
            cut.ties = min(cut.ties, ties);
          }
        }
      }
    }
    const float mp = a.min_p ? a.min_p[idx] : 0.f;
    if (mp > 0.f) {
      // the lowest float whose weight is at least min_p: near m + T ln p, then step by step
      const double want = fmin((double)mp, 1.0);
      auto keeps = [&](float z) { return exp2_scaled(((double)z - wt.m) * wt.c, 0) >= want; };
      uint32_t key = order_key((float)fmax(wt.m + log2(want) / wt.c, -3.4e38));
      const uint32_t top = order_key(m);
      key = min(key, top);
      for (int i = 0; i < 64 && key < top && !keeps(key_value(key)); ++i) ++key;
      for (int i = 0; i < 64 && key > 0x00800000u && keeps(key_value(key - 1)); ++i) --key;
      const float z = key_value(key);
      if (z > cut.z) cut = {z, ~0ull};
    }
    // ids up to id_lim are kept at the cut itself
    uint32_t id_lim = 0xFFFFFFFFu;
    if (cut.z != -INFINITY && cut.ties != ~0ull) {
      u64 here = 0;
      each(0, cpw, [&](float z, int) { here += z == cut.z ? 1 : 0; });
      const u64 mine = wave_sum_u64(here);
      if (lane == 0) sh.scan_c[wave] = mine;
      if (threadIdx.x == 0) sh.bin = -1;
      __syncthreads();
      u64 before = 0, all = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        if (i < wave) before += sh.scan_c[i];
        all += sh.scan_c[i];
      }
      if (cut.ties < all && before < cut.ties && before + mine >= cut.ties) {
        // the wave that holds the last tie kept
        for (int i = 0; i < cpw; ++i) {
          u64 x = 0;
          each(i, i + 1, [&](float z, int) { x += z == cut.z ? 1 : 0; });
          const u64 sum = wave_sum_u64(x);
          if (before + sum >= cut.ties) {
            u64 at = before + wave_before_u64(x);
            each(i, i + 1, [&](float z, int e) {
              if (z == cut.z && ++at == cut.ties) sh.bin = e;
            });
            break;
          }
          before += sum;
        }
      }
      __syncthreads();
      if (sh.bin >= 0) id_lim = (uint32_t)sh.bin;
      __syncthreads();
    }
    auto kept = [&](float z, int e) { return z > cut.z || (z == cut.z && (uint32_t)e <= id_lim); };

    // the draw: weights of each wave's run, in parts, then the part, the chunk and the token
    const int per = (cpw + SAMPLE_GROUPS - 1) / SAMPLE_GROUPS;
    u64 run = 0;
#pragma unroll
    for (int g = 0; g < SAMPLE_GROUPS; ++g) {
      u64 x = 0;
      each(g * per, min(cpw, (g + 1) * per), [&](float z, int e) {
        if (kept(z, e)) x += wt.units(z);
      });
      x = wave_sum_u64(x);
      if (lane == 0) sh.group[wave][g] = x;
      run += x;
    }
    if (lane == 0) sh.scan_m[wave] = run;
    __syncthreads();
    u64 before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      if (i < wave) before += sh.scan_m[i];
      total += sh.scan_m[i];
    }
    const double u = fmin(fmax((double)a.uniform[o], 0.0), 1.0 - 0x1p-24);
    const u64 want = (u64)(u * (double)total);  // the first cumulative weight above it
    if (before <= want && before + run > want) {
      int g = 0;
      while (g + 1 < SAMPLE_GROUPS && before + sh.group[wave][g] <= want) before += sh.group[wave][g++];
      for (int i = g * per; i < min(cpw, (g + 1) * per); ++i) {
        u64 x = 0;
        each(i, i + 1, [&](float z, int e) {
          if (kept(z, e)) x += wt.units(z);
        });
        const u64 sum = wave_sum_u64(x);
        if (before + sum > want) {
          u64 at = before + wave_before_u64(x);
          each(i, i + 1, [&](float z, int e) {
            if (!kept(z, e)) return;
            const u64 w = wt.units(z);
            if (at <= want && at + w > want) {
              const double lw = ((double)z - wt.m) * wt.c - log2((double)total) + wt.shift;
              emit(e, (float)(lw * 0.69314718055994530942));
            }
            at += w;
          });
          break;
        }
        before += sum;
      }
    }
    __syncthreads();  // the shared arrays are written again for the next row
  }
}

}  // namespace alr
