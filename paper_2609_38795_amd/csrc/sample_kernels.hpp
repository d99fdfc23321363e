// One token per row of logits from a given uniform number: temperature, top-k, top-p, min-p.
//
// Weights w_v = exp((z_v - max z) / T).  Tokens are ranked by decreasing logit, equal logits by
// increasing id, and a prefix of the ranking is kept: the shortest of the first k, the smallest
// prefix that holds at least p of the first k's weight, and the tokens with w >= min_p.  The token is
// the first, in the order of the ids, whose cumulative kept weight exceeds u times the total.
//
// Each of those prefixes is "logits above a cut, and the first few ids at the cut", so no row is
// sorted: the cut, the ties at it and the token are each the pick of one value among ranked ones.
//
// Four launches.  Two scans, by up to 16 workgroups a row so that few rows fill the card too: the
// first takes the maximum and, from the maxima of a thousand parts, a line above which a few thousand
// logits lie; the second sets those aside, and adds up the row's weight where top_p is of the whole
// row.  A third settles every row whose limits fall within its list, a fourth the others, from
// histograms of the row.  1024 rows of 128256 fp32 with all limits, in microseconds: 82 (6.4 TB/s, part of it from
// the last-level cache), 135 (80 to read the rows, 20 to set the lists aside, 35 for the weights of the 192 rows
// that need them, 13 if their work were spread evenly), 63, 116: 396 for the
// call, where a first kernel that did it all in one launch, a row per workgroup and a pass of the row per
// narrowing, took 989, and one with the list and all else in one launch 505.  128 rows without limits:
// 12 + 18 + 8, 37 for the call.
//
// Weights are whole numbers of 2^-shift (shift >= 43), from 64-bit exponentials, so every sum is exact
// and does not depend on the order in which it is formed: what a row gives depends on its own values
// alone, and is what 64-bit arithmetic gives up to 2^-43 of a weight and of the largest one.
#pragma once

#include "row_chunks.hpp"

namespace alr {

typedef unsigned long long u64;

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
  // scratch of `cap` rows; a call of more rows comes in several, `row0` being the first of each
  struct SampleRow* rows;
  f32x2* lists;           // [cap, SAMPLE_LIST]
  struct SampleSeg* segs; // [cap, SAMPLE_SEGS]
  unsigned long long* parts;  // [cap, SAMPLE_GROUPS]
  uint32_t* slow;         // [1 + cap]: how many rows their list does not settle, and which
  long row0;
  int n_seg;              // segments of a row, each a workgroup's, in the scans
};

constexpr int SAMPLE_BINS = 1024, SAMPLE_BITS = 10;
constexpr int SAMPLE_GROUPS = 64;   // parts of a row whose weights are summed apart for the draw
constexpr int SAMPLE_LIST = 4096;   // logits of a row that may be set aside
constexpr int SAMPLE_SEGS = 16;     // segments of a row at most

// What the scans of a row leave for the kernel that settles it.
struct SampleRow {
  u64 whole;        // weight of the row (a top_p of the whole row)
  uint32_t n_list;  // logits set aside; more than SAMPLE_LIST: they did not fit
  uint32_t greedy;  // lowest id at the maximum (greedy rows)
  float m, line;
};
// Of a segment of a row: its maximum, and number, sum and sum of squares of the maxima of its parts.
struct SampleSeg {
  float m, c, s1, s2;
};

// A row's limits.
struct Limits {
  uint32_t k;
  float temp, p, mp;
  bool by_k, by_p, greedy, any;
  __device__ __forceinline__ Limits(const SampleArgs& a, long idx, float m) {
    temp = a.temperature ? a.temperature[idx] : 1.f;
    k = a.top_k ? (uint32_t)max(a.top_k[idx], 0) : 0;
    p = a.top_p ? a.top_p[idx] : 1.f;
    mp = a.min_p ? a.min_p[idx] : 0.f;
    by_k = k > 0 && k < (uint32_t)a.V;
    by_p = p < 1.f;
    greedy = !(temp > 0.f) || m == INFINITY;
    any = by_k || by_p || mp > 0.f;
  }
  // top_p's share is of the first k, whether or not min_p ends before it
  __device__ __forceinline__ bool below_counts() const { return by_k && by_p; }
};

// v of the lane that a DPP control names, 0 where there is none or the row is masked off
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_or_0(u64 v) {
  return (u64)dpp_or_0<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | dpp_or_0<CTRL, ROWS>((uint32_t)v);
}
// Sum over this lane and those before it: within rows of 16 lanes, then rows 1 and 3 take the last lane
// of the row before them, then rows 2 and 3 lane 31.  All lanes must be active.
template <typename N>
__device__ __forceinline__ N wave_upto(N v) {
  v += dpp_or_0<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += dpp_or_0<0x112, 0xF>(v);
  v += dpp_or_0<0x114, 0xF>(v);
  v += dpp_or_0<0x118, 0xF>(v);
  v += dpp_or_0<0x142, 0xA>(v);  // row_bcast 15
  v += dpp_or_0<0x143, 0xC>(v);  // row_bcast 31
  return v;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ u64 last_lane(u64 v) {
  return (u64)last_lane((uint32_t)(v >> 32)) << 32 | last_lane((uint32_t)v);
}
template <typename N>
__device__ __forceinline__ N wave_total(N v) {
  return last_lane(wave_upto(v));
}

// Unsigned order of the floats' order; -0 as +0.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k);
}

// The weight of a logit, in units of 2^-shift of the largest one's: with y = (z - m) 32 log2(e) / T =
// k + f, |f| <= 1/2, the weight is 2^(k / 32) times a polynomial of 2^(f / 32).  2^((k mod 32) / 32) comes from a
// table, the rest of k is added to its exponent, and adding 2^52 rounds to whole units.  The polynomial is
// the series of exp up to the 5th power with that power replaced by the lower ones that differ least
// from it on [-1/2, 1/2] (Chebyshev): 2^-43 of the weight.  Some 25 instructions, which bound every pass that weighs
// whole rows: in a scan of 1024 rows of 128256 that sets lists aside, weighing all rows takes 175 us and none 104,
// 85 cycles of a SIMD for the 64 weights of a wave.
struct Weigher {
  double m, c, floor;  // the row's largest logit; 32 log2(e) / T; the lowest z - m: weights below are 0
  int shift;
  const double* tab;   // 2^(shift + j / 32), j < 32
  __device__ __forceinline__ void set(float m_, float temp, int shift_, const double* tab_) {
    m = (double)m_;
    c = fmax(32.0 * 1.4426950408889634074 / (double)temp, 1e-300);
    floor = -28800.0 / c;
    shift = shift_;
    tab = tab_;
  }
  static constexpr u64 BIAS = 0x4330000000000000ull;  // the bits of 2^52
  __device__ __forceinline__ u64 units(float z) const { return biased(z) - BIAS; }
  // units() + BIAS: what a long sum adds up, to take the biases off once at its end
  __device__ __forceinline__ u64 biased(float z) const {
    constexpr double MAGIC = 6755399441055744.0, ONE52 = 4503599627370496.0;
    constexpr double L = 0.693147180559945309417232 / 32, A2 = 0.25;  // A2: (half width)^2
    constexpr double c5 = L * L * L * L * L / 120;
    constexpr double c1 = L - c5 * A2 * A2 * 5 / 16, c2 = L * L / 2, c3 = L * L * L / 6 + c5 * A2 * 5 / 4,
                     c4 = L * L * L * L / 24;
    const double d = fmax((double)z - m, floor);
    const double t = fma(d, c, MAGIC);
    const double f = fma(d, c, -(t - MAGIC));
    const uint32_t k = (uint32_t)__double_as_longlong(t);
    const u64 w = (u64)__double_as_longlong(tab[k & 31]) + ((u64)((k & ~31u) << 15) << 32);
    double p = fma(f, c4, c3);
    p = fma(f, p, c2);
    p = fma(f, p, c1);
    p = fma(f, p, 1.0);
    return (u64)__double_as_longlong(fma(p, __longlong_as_double((long long)w), ONE52));
  }
  __device__ __forceinline__ double log2_of(float z) const { return ((double)z - m) * c * (1.0 / 32); }
};

template <int LEVELS>
struct SampleSharedOf {
  double tab[32];
  uint32_t cnt[LEVELS][SAMPLE_BINS];  // of the narrowing levels; of the first one, over a row
  u64 mass[LEVELS][SAMPLE_BINS];
  f32x2 list[SAMPLE_LIST];       // (logit, id) of the logits set aside, a run of it per wave
  uint32_t scan_c[16], few_n;
  u64 scan_m[16];
  u64 part[SAMPLE_GROUPS];
  uint32_t few_key[64];
  u64 few_w[64];
  uint32_t ured[2][16];
  int bin;
  uint32_t above_c;
  u64 above_m;
};

// min and max of unsigned values over the workgroup
template <int NW, typename S>
__device__ __forceinline__ void block_range(uint32_t& lo, uint32_t& hi, S& sh) {
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

// a count and a sum of weights over the workgroup
template <int NW, typename S>
__device__ __forceinline__ void block_sums(uint32_t& c, u64& m, S& sh) {
  c = wave_total(c);
  m = wave_total(m);
  if ((threadIdx.x & 63) == 0) {
    sh.scan_c[threadIdx.x >> 6] = c;
    sh.scan_m[threadIdx.x >> 6] = m;
  }
  __syncthreads();
  c = 0;
  m = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    c += sh.scan_c[i];
    m += sh.scan_m[i];
  }
  __syncthreads();
}

template <int THREADS, typename S>
__device__ __forceinline__ void clear_bins(S& sh, int level) {
#pragma unroll
  for (int b = threadIdx.x; b < SAMPLE_BINS; b += THREADS) {
    sh.cnt[level][b] = 0;
    sh.mass[level][b] = 0;
  }
  __syncthreads();
}

// What is looked for among ranked values: the `want`-th (counting from 1), or, by_mass, the one with which
// the weights added up reach `want` >= 1.
struct Aim {
  bool by_mass;
  u64 want;
};

// Finds the aim's bin; above_c and above_m come in as what lies before the level's bins and go out as
// what lies before the bin.  Returns -1 where the bins do not reach it.  total_of is told the
// total weight of the bins.
template <int THREADS, typename S, typename F>
__device__ __forceinline__ int find_bin(S& sh, int level, Aim aim, uint32_t& above_c,
                                        u64& above_m, F total_of) {
  constexpr int NW = THREADS / 64, PER = SAMPLE_BINS / THREADS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b0 = threadIdx.x * PER;
  uint32_t c = 0;
  u64 m = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    c += sh.cnt[level][b0 + i];
    m += sh.mass[level][b0 + i];
  }
  uint32_t c_upto = wave_upto(c);
  u64 m_upto = wave_upto(m);
  if (lane == 63) {
    sh.scan_c[wave] = c_upto;
    sh.scan_m[wave] = m_upto;
  }
  if (threadIdx.x == 0) sh.bin = -1;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < wave) {
      c_upto += sh.scan_c[i];
      m_upto += sh.scan_m[i];
    }
    all += sh.scan_m[i];
  }
  total_of(all);
  uint32_t c_before = above_c + c_upto - c;
  u64 m_before = above_m + m_upto - m;
  u64 at = aim.by_mass ? m_before : c_before;
  if (at < aim.want && at + (aim.by_mass ? m : c) >= aim.want) {
    for (int i = 0; i < PER; ++i) {
      const u64 x = aim.by_mass ? sh.mass[level][b0 + i] : sh.cnt[level][b0 + i];
      if (at + x >= aim.want) {
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
  __syncthreads();  // sh.bin may be written again
  return bin;
}

// Among the values that `each` visits (f(key, logit) per value of interest), those with keys within [lo, hi]:
// the key that the aim falls on, keys counted from the largest down, or, `up`, from the smallest up;
// above_c and above_m come in as what lies before hi (lo) and end as what lies before that key.  A level
// of bins over the keys' range leaves few values as a rule, which are ranked against each other; else another
// level splits the bin.  False where the values do not reach the aim.
template <int THREADS, typename S, typename E>
__device__ __forceinline__ bool pick(S& sh, const Weigher& wt, bool up, Aim aim, uint32_t lo,
                                     uint32_t hi, uint32_t& above_c, u64& above_m, uint32_t& found,
                                     E each) {
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range ? max(0, 32 - SAMPLE_BITS - (int)__clz(range)) : 0;  // range >> shift: a bin
    if (threadIdx.x == 0) sh.few_n = 0;
    clear_bins<THREADS>(sh, 0);
    each([&](uint32_t key, float z) {
      if (key >= lo && key <= hi) {
        const uint32_t b = (up ? key - lo : hi - key) >> shift;
        atomicAdd(&sh.cnt[0][b], 1u);
        atomicAdd(&sh.mass[0][b], wt.units(z));
      }
    });
    __syncthreads();
    const int b = find_bin<THREADS>(sh, 0, aim, above_c, above_m, [](u64) {});
    if (b < 0) return false;
    const uint32_t width = (1u << shift) - 1, n = sh.cnt[0][b];
    if (up) {
      lo += (uint32_t)b << shift;
      hi = min(hi, lo + min(0xFFFFFFFFu - lo, width));
    } else {
      hi -= (uint32_t)b << shift;
      lo = max(lo, hi - min(hi, width));
    }
    __syncthreads();  // cnt may be cleared again
    if (lo == hi) {
      found = lo;
      return true;
    }
    if (n > 64) continue;
    each([&](uint32_t key, float z) {
      if (key >= lo && key <= hi) {
        const uint32_t at = atomicAdd(&sh.few_n, 1u);
        sh.few_key[at] = key;
        sh.few_w[at] = wt.units(z);
      }
    });
    __syncthreads();
    // every wave ranks them: lane l's value against all
    const int lane = threadIdx.x & 63;
    const uint32_t mine = sh.few_key[min((uint32_t)lane, n - 1)];
    uint32_t c = 0, c_own = 0;
    u64 m = 0, m_own = 0;
    for (uint32_t i = 0; i < n; ++i) {
      const uint32_t key = sh.few_key[i];
      const u64 w = sh.few_w[i];
      if (key == mine) {
        ++c_own;
        m_own += w;
      } else if (up ? key < mine : key > mine) {
        ++c;
        m += w;
      }
    }
    const u64 at = aim.by_mass ? above_m + m : above_c + c;
    const bool hit = (uint32_t)lane < n && at < aim.want && at + (aim.by_mass ? m_own : c_own) >= aim.want;
    const int src = __ffsll((unsigned long long)__ballot(hit)) - 1;
    found = (uint32_t)__builtin_amdgcn_readlane((int)mine, src);
    above_c += (uint32_t)__builtin_amdgcn_readlane((int)c, src);
    above_m += (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(m >> 32), src) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)m, src);
    __syncthreads();
    return true;
  }
}

// Where the kept prefix ends: logits above `z`, and of those equal to z the first `ties` ids.
struct Cut {
  float z;
  u64 ties;
};
constexpr u64 ALL_TIES = ~0ull;

// The lowest float whose weight is at least min_p: near m + T ln p (or the lowest of all), then step by step.
__device__ __forceinline__ float min_p_cut(const Weigher& wt, float m, float mp) {
  const double want = fmin((double)mp, 1.0);
  auto keeps = [&](float z) { return exp2(wt.log2_of(z)) >= want; };
  if (want == 1.0) return m;  // the others' weights are below 1, though they may round to it
  const uint32_t top = order_key(m);
  uint32_t key = min(order_key((float)fmax(wt.m + 32 * log2(want) / wt.c, -(double)3.402823466e38f)), top);
  for (int i = 0; i < 64 && key < top && !keeps(key_value(key)); ++i) ++key;
  for (int i = 0; i < 64 && key > 0x00800000u && keeps(key_value(key - 1)); ++i) --key;
  return key_value(key);
}

__device__ __forceinline__ bool real(float z) { return z > -INFINITY; }  // neither nan nor -inf

// Rows of different limits cost differently and limits tend to repeat, so a group of eight rows is dealt
// to the eight XCDs in a rotating order.
__device__ __forceinline__ long dealt_row(long b, long n) {
  return (b | 7) < n ? (b & ~7L) | ((b + (b >> 3)) & 7) : b;
}

// A wave's run of logits set aside, in LDS.
template <int RUN>
struct Aside {
  f32x2* run;
  uint32_t mine = 0;
  __device__ __forceinline__ explicit Aside(f32x2* r) : run(r) {}
  // The logits of a chunk whose bit is set in `in`, one of every lane that has any left at a time: they
  // are few, so one or two rounds do.
  template <int EPC>
  __device__ __forceinline__ void add(const float (&v)[EPC], int e0, uint32_t in) {
    while (true) {
      const u64 bits = __ballot(in != 0);
      if (bits == 0) return;
      const int q = __ffs((int)in) - 1;
      float z = v[0];
#pragma unroll
      for (int i = 1; i < EPC; ++i) z = q == i ? v[i] : z;
      const uint32_t at = mine + __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32),
                                                          __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
      if (in != 0 && at < RUN) run[at] = f32x2{z, __int_as_float(e0 + q)};
      mine += (uint32_t)__popcll(bits);
      in &= in - 1;
    }
  }
};

// First scan: every segment's maximum, and the statistics of the maxima of its parts, of which a row has
// about a thousand (a segment of few chunks merges lanes).
template <typename T>
__device__ __forceinline__ SampleSeg scan_max(const RowChunks<T>& row, int n_seg, int seg, float (*red)[4]) {
  constexpr int EPC = RowChunks<T>::EPC;
  const int per = (row.nch + n_seg * 256 - 1) / (n_seg * 256);  // chunks of a thread
  float part[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  walk<4, 256>(row, seg * per * 256 + (int)threadIdx.x, 0, per, [&](int i, int, u32x4 w) {
    float v[EPC];
    unpack<T>(w, v);
    float x = v[0];
#pragma unroll
    for (int k = 1; k < EPC; ++k) x = fmaxf(x, v[k]);
    const int h = i & 3;
#pragma unroll
    for (int k = 0; k < 4; ++k) part[k] = fmaxf(part[k], h == k ? x : -INFINITY);
  });
  if (n_seg >= 2) {
    part[0] = fmaxf(part[0], part[1]);
    part[2] = fmaxf(part[2], part[3]);
  }
  if (n_seg >= 4) part[0] = fmaxf(part[0], part[2]);
  if (n_seg >= 8) part[0] = fmaxf(part[0], dpp_perm<0xB1>(part[0]));
  if (n_seg >= 16) part[0] = fmaxf(part[0], dpp_perm<0x4E>(part[0]));
  SampleSeg s = {-INFINITY, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k == 0 || (k == 2 && n_seg == 2) || n_seg == 1) {
      s.m = fmaxf(s.m, part[k]);
      if (part[k] != -INFINITY) {
        s.c += 1.f;
        s.s1 += part[k];
        s.s2 += part[k] * part[k];
      }
    }
  s.m = wave_max(s.m);
  s.c = wave_sum(s.c);
  s.s1 = wave_sum(s.s1);
  s.s2 = wave_sum(s.s2);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[wave][0] = s.m;
    red[wave][1] = s.c;
    red[wave][2] = s.s1;
    red[wave][3] = s.s2;
  }
  __syncthreads();
  s = {-INFINITY, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s.m = fmaxf(s.m, red[i][0]);
    s.c += red[i][1];
    s.s1 += red[i][2];
    s.s2 += red[i][3];
  }
  __syncthreads();
  return s;
}

// The line: 1.5 standard deviations below the mean of the parts' maxima (an estimate: any line is right).
__device__ __forceinline__ float line_of(const SampleSeg& s, int V) {
  if (V <= SAMPLE_LIST / 2) return -INFINITY;
  const float mean = s.s1 / s.c;
  const float line = mean - 1.5f * sqrtf(fmaxf(s.s2 / s.c - mean * mean, 0.f));
  return line == line ? line : -INFINITY;
}

struct ScanShared {
  double tab[32];
  f32x2 list[SAMPLE_LIST];
  float red[4][4];
  uint32_t n[4], base;
};

// Second scan: the logits above the line set aside; for a top_p of the whole row its weight; without limits,
// the weights of the row's parts; for a greedy row the lowest id at the maximum.
template <typename T>
__device__ __forceinline__ void scan_list(const SampleArgs& a, const RowChunks<T>& row, int seg, long idx,
                                          long slot, const SampleSeg& st, ScanShared& sh) {
  constexpr int EPC = RowChunks<T>::EPC, RUN = SAMPLE_LIST / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_seg = a.n_seg;
  const float m = st.m;
  SampleRow& hdr = a.rows[slot];
  float line = line_of(st, a.V);
  const Limits lim(a, idx, m);
  Weigher wt;
  wt.set(m, lim.temp, a.shift, sh.tab);
  if (m != -INFINITY && !lim.greedy && lim.mp > 0.f && !lim.below_counts())
    line = fmaxf(line, min_p_cut(wt, m, lim.mp));  // nothing below min_p counts
  if (seg == 0 && threadIdx.x == 0) {
    hdr.m = m;
    hdr.line = line;
  }
  if (m == -INFINITY) return;
  const int per = (row.nch + n_seg * 256 - 1) / (n_seg * 256), c0 = seg * per * 256 + (int)threadIdx.x;
  if (lim.greedy) {
    uint32_t lo = 0xFFFFFFFFu;
    walk<4, 256>(row, c0, 0, per, [&](int, int c, u32x4 w) {
      float v[EPC];
      unpack<T>(w, v);
#pragma unroll
      for (int q = 0; q < EPC; ++q)
        if (v[q] == m) lo = min(lo, (uint32_t)(row.first(c) + q));
    });
    if (lo != 0xFFFFFFFFu) atomicMin(&hdr.greedy, lo);
    return;
  }
  if (!lim.any) {
    const int gc = (row.nch + SAMPLE_GROUPS - 1) / SAMPLE_GROUPS, steps = (gc + 63) / 64;
    for (int g = seg * (SAMPLE_GROUPS / n_seg) + wave; g < (seg + 1) * (SAMPLE_GROUPS / n_seg); g += 4) {
      u64 x = 0;
      walk<4, 64>(row, g * gc + lane, 0, steps, [&](int, int c, u32x4 w) {
        float v[EPC];
        unpack<T>(w, v);
        u64 y = 0;
#pragma unroll
        for (int q = 0; q < EPC; ++q) y += wt.biased(v[q]);
        x += c < (g + 1) * gc ? y - EPC * Weigher::BIAS : 0;
      });
      x = wave_total(x);
      if (lane == 0) a.parts[slot * SAMPLE_GROUPS + g] = x;
    }
    return;
  }
  Aside<RUN> aside(sh.list + wave * RUN);
  const float bound = fmaxf(line, -3.402823466e38f);  // -inf is never kept
  if (lim.by_p && !lim.by_k) {
    u64 x = 0;
    walk<4, 256>(row, c0, 0, per, [&](int, int c, u32x4 w) {
      float v[EPC];
      uint32_t in = 0;
      unpack<T>(w, v);
#pragma unroll
      for (int q = 0; q < EPC; ++q) {
        x += wt.biased(v[q]);
        in |= v[q] >= bound ? 1u << q : 0;
      }
      aside.add(v, row.first(c), in);
    });
    x = wave_total(x - (u64)(per * EPC) * Weigher::BIAS);
    if (lane == 0) atomicAdd(&hdr.whole, x);
  } else {
    walk<4, 256>(row, c0, 0, per, [&](int, int c, u32x4 w) {
      float v[EPC];
      uint32_t in = 0;
      unpack<T>(w, v);
#pragma unroll
      for (int q = 0; q < EPC; ++q) in |= v[q] >= bound ? 1u << q : 0;
      aside.add(v, row.first(c), in);
    });
  }
  if (lane == 0) sh.n[wave] = aside.mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t n = 0;
    bool fits = true;
    for (int i = 0; i < 4; ++i) {
      n += sh.n[i];
      fits &= sh.n[i] <= RUN;
    }
    // what does not fit puts the count out of reach (it stays below 2^32: segments are few)
    sh.base = n ? atomicAdd(&hdr.n_list, fits ? n : SAMPLE_LIST + 1u) : 0;
  }
  __syncthreads();
  uint32_t at = sh.base;
  for (int i = 0; i < wave; ++i) at += sh.n[i];
  for (uint32_t i = lane; i < min(aside.mine, (uint32_t)RUN); i += 64)
    if (at + i < SAMPLE_LIST) a.lists[slot * SAMPLE_LIST + at + i] = aside.run[i];
  __syncthreads();
}

// The first (FIRST) and the second scan, a.n_seg workgroups a row.  Both walk the segments in opposite
// orders: the second begins with what the last-level cache still holds of the first.
template <typename T, bool FIRST>
__global__ __launch_bounds__(256, 4) void sample_scan_kernel(SampleArgs a) {
  __shared__ ScanShared sh;
  if (!FIRST && threadIdx.x < 32) sh.tab[threadIdx.x] = exp2((double)threadIdx.x / 32 + a.shift);
  const long wg = FIRST ? blockIdx.x : gridDim.x - 1 - blockIdx.x, b = wg / a.n_seg;
  const int seg = (int)(wg - b * a.n_seg);
  const long slot = dealt_row(b, a.n), r = a.row0 + slot, idx = a.perm ? (long)a.perm[r] : r;
  RowChunks<T> row(static_cast<const T*>(a.z) + (a.z_perm ? idx : r) * a.z_rs, a.V);
  row.edges();
  SampleSeg s;
  if constexpr (FIRST) {
    s = scan_max(row, a.n_seg, seg, sh.red);
    if (threadIdx.x != 0) return;
    if (blockIdx.x == 0) a.slow[0] = 0;
    if (seg == 0) {
      a.rows[slot].whole = 0;
      a.rows[slot].n_list = 0;
      a.rows[slot].greedy = 0xFFFFFFFFu;
    }
    a.segs[slot * SAMPLE_SEGS + seg] = s;
  } else {
    s = {-INFINITY, 0.f, 0.f, 0.f};
    for (int i = 0; i < a.n_seg; ++i) {
      const SampleSeg x = a.segs[slot * SAMPLE_SEGS + i];
      s.m = fmaxf(s.m, x.m);
      s.c += x.c;
      s.s1 += x.s1;
      s.s2 += x.s2;
    }
    __syncthreads();  // the table
    scan_list(a, row, seg, idx, slot, s, sh);
  }
}

// Settles a row from what the scans left.  Limits that fall within the list are settled there, and so is the
// draw; without limits the part of the row that the number falls into is read again.  What bounds it is the
// chain of picks, each some eight barriers long: 17 us for one row, 63 for 1024.  Rows whose list falls short (a
// nucleus of a flat distribution, a k of thousands) are left to the SLOW form, a launch of its own, whose
// workgroups have a CU to themselves: a histogram of the row, the list becomes that of the bin the limit falls
// into, and the draw reads the row again.  A row of 128256 takes it 100 us (histogram 36, list 25, draw 29), bound
// by LDS atomics and one CU's loads in flight.  1024 threads, though the bf16 form keeps 16 registers in scratch:
// 512 threads with twice the loads ahead and none in scratch took 133 us for the rows of the case above, not 115.
template <typename T, int THREADS, bool SLOW>
__global__ __launch_bounds__(THREADS, 4) void sample_settle_kernel(SampleArgs a) {
  constexpr int NW = THREADS / 64, EPC = RowChunks<T>::EPC, RUN = SAMPLE_LIST / NW;
  static_assert(SAMPLE_BINS % THREADS == 0 && NW <= 16, "bins per thread");
  __shared__ SampleSharedOf<SLOW ? 2 : 1> sh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (in the order of the list, so that no workgroup with work waits behind one in a row of empty ones)
  if (SLOW && blockIdx.x >= a.slow[0]) return;
  const long slot = SLOW ? (long)a.slow[1 + blockIdx.x] : dealt_row(blockIdx.x, a.n), r = a.row0 + slot;
  const long idx = a.perm ? (long)a.perm[r] : r, o = idx * a.block + a.s;
  auto emit = [&](int tok, float lp) {
    a.tokens[o] = tok;
    if (a.logp) a.logp[o] = lp;
    if (a.next_tok) {
      const int f = a.forced ? a.forced[o] : -1;
      a.next_tok[r] = f >= 0 ? f : max(tok, 0);
    }
  };
  const SampleRow hdr = a.rows[slot];
  const float m = hdr.m, line = hdr.line;
  auto leave_to_slow = [&]() {
    if (threadIdx.x == 0) a.slow[1 + atomicAdd(a.slow, 1u)] = (uint32_t)slot;
  };
  if (m == -INFINITY) {  // nothing to draw
    if (threadIdx.x == 0) emit(-1, -INFINITY);
    return;
  }
  const Limits lim(a, idx, m);
  if (lim.greedy) {
    if (threadIdx.x == 0) emit((int)hdr.greedy, 0.f);
    return;
  }
  if (threadIdx.x < 32) sh.tab[threadIdx.x] = exp2((double)threadIdx.x / 32 + a.shift);
  __syncthreads();
  Weigher wt;
  wt.set(m, lim.temp, a.shift, sh.tab);
  RowChunks<T> row(static_cast<const T*>(a.z) + (a.z_perm ? idx : r) * a.z_rs, a.V);
  const int cpt = (row.nch + THREADS - 1) / THREADS;
  // f(logits, first id) for the thread's chunks
  auto chunks = [&](auto u_, auto f) {
    walk<decltype(u_)::value, THREADS>(row, (int)threadIdx.x, 0, cpt, [&](int, int c, u32x4 w) {
      float v[EPC];
      unpack<T>(w, v);
      f(v, row.first(c));
    });
  };
  using four = std::integral_constant<int, 4>;  // loads of a thread under way; `one` needs fewer registers
  using one = std::integral_constant<int, 1>;
  auto each = [&](auto u_, auto f) {
    chunks(u_, [&](const float(&v)[EPC], int e0) {
#pragma unroll
      for (int k = 0; k < EPC; ++k) f(v[k], e0 + k);
    });
  };
  const uint32_t k = lim.k;
  const bool by_k = lim.by_k, by_p = lim.by_p;
  auto share_of = [&](u64 w) { return max((u64)ceil(fmax((double)lim.p, 0.0) * (double)w), 1ull); };
  const double u = fmin(fmax((double)a.uniform[o], 0.0), 1.0 - 0x1p-24);
  auto emit_drawn = [&](float z, int e, u64 total) {
    emit(e, (float)((wt.log2_of(z) + wt.shift - log2((double)total)) * 0.69314718055994530942));
  };

  Cut cut = {-INFINITY, ALL_TIES};
  if (lim.mp > 0.f) cut.z = min_p_cut(wt, m, lim.mp);
  uint32_t id_lim = 0xFFFFFFFFu;  // ids up to it are kept at the cut itself
  auto kept = [&](float z, int e) { return z > cut.z || (z == cut.z && (uint32_t)e <= id_lim); };

  Aside<RUN> aside(sh.list + wave * RUN);
  uint32_t n_list = 0;
  auto each_listed = [&](auto f) {
    for (uint32_t i = lane; i < aside.mine; i += 64) {
      const f32x2 x = aside.run[i];
      f(x[0], __float_as_int(x[1]));
    }
  };
  auto list_closed = [&]() {  // whether every wave's share fitted its run
    if (lane == 0) sh.scan_c[wave] = aside.mine;
    __syncthreads();
    bool fits = true;
    n_list = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      fits &= sh.scan_c[i] <= RUN;
      n_list += sh.scan_c[i];
    }
    __syncthreads();
    return fits;
  };
  // bins of the whole row, of 1/32 in (max - z) / T, the last one for all that lies below
  const float cs = fminf(32.f / lim.temp, 1e30f);
  auto bin0 = [&](float z) { return (int)fminf((m - z) * cs, (float)(SAMPLE_BINS - 1)); };
  bool binned = false;
  auto bin_row = [&]() {
    clear_bins<THREADS>(sh, 1);
    if (by_p)
      each(four{}, [&](float z, int) {
        if (real(z)) {
          const int q = bin0(z);
          if (by_k) atomicAdd(&sh.cnt[1][q], 1u);
          atomicAdd(&sh.mass[1][q], wt.units(z));
        }
      });
    else
      each(four{}, [&](float z, int) {
        if (real(z)) atomicAdd(&sh.cnt[1][bin0(z)], 1u);
      });
    __syncthreads();
    binned = true;
  };

  const bool fits = hdr.n_list <= SAMPLE_LIST;
  // what is not listed is not kept: the list is the row, or ends where min_p does
  const bool all = line == -INFINITY || (!lim.below_counts() && cut.z >= line);
  // listed: every logit that may be kept is in the list (and the limits are settled there)
  bool listed = !SLOW && lim.any && fits && (by_k ? hdr.n_list >= k || all : by_p || all);
  if (!SLOW && lim.any && !listed) {
    leave_to_slow();
    return;
  }
  if (!SLOW && listed) {
    n_list = hdr.n_list;
    for (uint32_t i = threadIdx.x; i < n_list; i += THREADS)
      aside.run[i / THREADS * 64 + lane] = a.lists[slot * SAMPLE_LIST + i];
    const uint32_t rest = n_list % THREADS, skip = (uint32_t)wave * 64;
    aside.mine = n_list / THREADS * 64 + (rest > skip ? min(rest - skip, 64u) : 0);
  }
  u64 w_k = hdr.whole, total = 0;  // weight of the first k, or of all; of the kept
  if (SLOW) row.edges();

  // The limits, ties and the draw, one after the other, each the pick of a value among ranked ones: of a
  // logit by count (k) or by weight (p), of an id by count (ties at the cut) or by weight (the draw).
  bool from_list = listed;  // else: from the list of a bin, or from the row itself
  int bin_listed = -1;
#pragma unroll 1
  for (int stage = lim.any ? 0 : 4; stage < 4; ++stage) {  // k, p, ties, draw
    const bool up = stage >= 2;
    // values of interest: above `from`, or at it with ids up to `to_id`; none above `upto`
    float from = -INFINITY, upto = INFINITY;
    uint32_t to_id = 0xFFFFFFFFu, lo = order_key(line), hi = order_key(m), c = 0, found = 0;
    u64 w = 0;
    Aim aim{stage == 1 || stage == 3, k};
    if (stage == 0 && !by_k) continue;
    if (stage == 1 && !by_p) continue;
    if (stage == 2) {
      if (cut.ties == ALL_TIES) continue;
      if (SLOW) from_list = bin_listed >= 0 && bin_listed == bin0(cut.z);
      from = upto = cut.z;
      aim.want = cut.ties;
    }
    if (stage == 3) {
      if (SLOW) break;
      from = cut.z;
      to_id = id_lim;
    }
    if (up) {
      lo = 0;
      hi = (uint32_t)a.V - 1;
    }
    auto visit = [&](auto f) {
      each_listed([&](float z, int e) {
        if ((z > from || (z == from && (uint32_t)e <= to_id)) && z <= upto) f(up ? (uint32_t)e : order_key(z), z);
      });
    };
    auto visit_row = [&](auto f) {
      each(one{}, [&](float z, int e) {
        if (real(z) && z >= from && z <= upto) f(up ? (uint32_t)e : order_key(z), z);
      });
    };
    if (SLOW && !up) {
      // narrowed to a bin of the row, whose logits become the list
      if (!binned) bin_row();
      if (stage == 1) aim.want = share_of(w_k);
      const int bin = find_bin<THREADS>(sh, 1, aim, c, w, [&](u64 sum) {
        if (stage == 0) w_k = sum;
      });
      if (bin < 0) continue;  // fewer than k can be drawn
      aside.mine = 0;
      lo = 0xFFFFFFFFu;
      hi = 0;
      chunks(four{}, [&](const float(&v)[EPC], int e0) {
        uint32_t in = 0;
#pragma unroll
        for (int q = 0; q < EPC; ++q) {
          const bool is = real(v[q]) && bin0(v[q]) == bin;
          lo = min(lo, is ? order_key(v[q]) : 0xFFFFFFFFu);
          hi = max(hi, is ? order_key(v[q]) : 0u);
          in |= is ? 1u << q : 0;
        }
        aside.add(v, e0, in);
      });
      block_range<NW>(lo, hi, sh);
      from_list = list_closed();  // too long where many logits are equal: then from the row
      bin_listed = from_list ? bin : -1;
    } else {
      uint32_t here = 0;
      if (stage == 1) {
        if (by_k && n_list < k) {  // fewer than k: the share is of them all
          w_k = 0;
          visit([&](uint32_t, float z) { w_k += wt.units(z); });
          block_sums<NW>(here, w_k, sh);
        }
        aim.want = share_of(w_k);
      } else if (stage == 2) {
        if (!SLOW || from_list)
          visit([&](uint32_t, float) { ++here; });
        else
          visit_row([&](uint32_t, float) { ++here; });
        block_sums<NW>(here, total, sh);
        total = 0;
        if (cut.ties >= here) continue;
      } else if (stage == 3) {
        visit([&](uint32_t, float z) { total += wt.units(z); });
        block_sums<NW>(here, total, sh);
        aim.want = (u64)(u * (double)total) + 1;
      }
      if (!up && line == -INFINITY) {  // a short row: its range
        lo = 0xFFFFFFFFu;
        hi = 0;
        visit([&](uint32_t q, float) {
          lo = min(lo, q);
          hi = max(hi, q);
        });
        block_range<NW>(lo, hi, sh);
      }
    }
    bool reached;
    if (!SLOW || from_list)
      reached = pick<THREADS>(sh, wt, up, aim, lo, hi, c, w, found, visit);
    else
      reached = pick<THREADS>(sh, wt, up, aim, lo, hi, c, w, found, visit_row);
    if (!SLOW && !reached && stage == 1 && !all) {  // the list ends before top_p does
      leave_to_slow();
      return;
    }
    if (stage == 2) {
      id_lim = found;
    } else if (stage == 3) {
      each_listed([&](float z, int e) {
        if ((uint32_t)e == found) emit_drawn(z, e, total);
      });
    } else if (reached) {
      const float z = key_value(found);
      const u64 one = max(wt.units(z), 1ull);
      const u64 ties = stage == 0 ? k - c : (aim.want - w + one - 1) / one;
      if (stage == 0) w_k = w + ties * wt.units(z);
      if (z > cut.z)
        cut = {z, ties};
      else if (z == cut.z)  // the shorter of two prefixes
        cut.ties = min(cut.ties, ties);
    }
  }
  if (!SLOW && lim.any) return;

  // the draw from the row: the part that the number falls into, then its run of chunks, the lane and the token
  if (!SLOW) row.edges();
  // weight of a chunk's kept logits (the one chunk in which the ties end is looked at closely)
  const int last = (int)min(id_lim, 0x7FFFFFFFu);
  const float least = cut.z, above = cut.z == -INFINITY ? cut.z : key_value(order_key(cut.z) + 1);
  auto weight_of = [&](const float(&v)[EPC], int e0) {
    const bool ends = e0 <= last && e0 + EPC - 1 > last;
    const float bound = e0 > last ? above : least;
    u64 x = 0;
#pragma unroll
    for (int q = 0; q < EPC; ++q) {
      float z = v[q] >= bound ? v[q] : -INFINITY;
      if (ends && !kept(v[q], e0 + q)) z = -INFINITY;
      x += wt.biased(z);
    }
    return x - EPC * Weigher::BIAS;
  };
  const int gc = (row.nch + SAMPLE_GROUPS - 1) / SAMPLE_GROUPS, steps = (gc + 63) / 64;
  auto group_chunks = [&](int g, int i0, int i1, auto f) {  // f(weight of the lane's chunk i, its logits, first id)
    walk<2, 64>(row, g * gc + lane, i0, i1, [&](int i, int c, u32x4 w) {
      float v[EPC];
      unpack<T>(w, v);
      const u64 x = weight_of(v, row.first(c));
      f(i, c < (g + 1) * gc ? x : 0, v, row.first(c));
    });
  };
  if (SLOW) {
#pragma unroll 1
    for (int g = wave; g < SAMPLE_GROUPS; g += NW) {
      u64 x = 0;
      group_chunks(g, 0, steps, [&](int, u64 y, const float(&)[EPC], int) { x += y; });
      x = wave_total(x);
      if (lane == 0) sh.part[g] = x;
    }
    __syncthreads();
  } else if (threadIdx.x < SAMPLE_GROUPS) {
    sh.part[threadIdx.x] = a.parts[slot * SAMPLE_GROUPS + threadIdx.x];
  }
  if (wave != 0) return;
  // one wave from here: lane g has part g
  const u64 mine = sh.part[lane], upto = wave_upto(mine);
  total = last_lane(upto);
  const u64 want = (u64)(u * (double)total);  // the first cumulative weight above it
  const int g = __ffsll((unsigned long long)__ballot(upto > want)) - 1;
  u64 before = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((upto - mine) >> 32), g) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(upto - mine), g);
  group_chunks(g, 0, steps, [&](int, u64 own, const float(&v)[EPC], int e0) {
    const u64 sum = wave_upto(own);
    if (before <= want && before + last_lane(sum) > want) {
      u64 at = before + sum - own;
#pragma unroll
      for (int q = 0; q < EPC; ++q)
        if (kept(v[q], e0 + q)) {
          const u64 w = wt.units(v[q]);
          if (own != 0 && at <= want && at + w > want) emit_drawn(v[q], e0 + q, total);
          at += w;
        }
    }
    before += last_lane(sum);
  });
}

}  // namespace alr
