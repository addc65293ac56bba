// Sampling with temperature, top-k, top-p and min-p from given uniforms.
//
// Everything that decides -- which tokens are kept, and which is drawn -- is made
// of comparisons of logits, counts, and sums of weights w = exp((l - max) / T).
// The weights are computed in 64 bits (fp32 ones would move a border between two
// tokens every few ten thousand rows of a 150k vocabulary) and summed as 64-bit
// integers in units of 2^-44 (V <= 2^19 weights of at most 1 fit), so sums are
// exact, associative, and the same in whatever order atomics or waves add them.
//
// top-k, top-p and min-p each keep a prefix of the tokens ordered by (logit
// descending, index ascending); so does their combination, up to min-p, which is
// a test of the weight alone.  The prefix is found by its last token:
//   1. the row's max;
//   2. a histogram of count and mass over d = max - l, in bins that are the
//      upper bits of d as a float (relative width 2^-7, so that a bin holds a few
//      per cent of a broad row at most, whatever the scale of the logits); the bin
//      in which the count reaches top_k, or the mass top_p;
//   3. if no more than kCap tokens lie up to that bin, they are collected, sorted,
//      and everything else happens on the sorted list in LDS;
//      otherwise the last token is found by a radix search over the logits' bits
//      (three more passes), and its index among equal logits by one more.
#include "../../include/nightjar_serve.h"
#include "common.h"
#include "kernels.h"

namespace nj {
namespace {

constexpr int kErrSampling = 32;  // NJ_DEV_BAD_SAMPLING
constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr int kCap = 4096;        // tokens of the sorted list
constexpr int kTile = 256;        // tokens per running-sum tile (four per lane of a wave)
constexpr int kMaxTiles = 2048;   // V <= 524288
typedef unsigned long long u64;

// exp2(x) for x <= 0 in 64 bits: 2^n times the Taylor series of 2^f, |f| <= 1/2
// (the terms behind f^11 are below 1e-14).  exp2(0) = 1 exactly; below 2^-200: 0.
__device__ __forceinline__ double exp2_64(double x) {
  if (!(x > -200.0)) return 0.0;
  const double n = rint(x), f = (x - n) * 0.69314718055994530942;
  double p = 1.0 / 39916800.0;
  p = fma(p, f, 1.0 / 3628800.0);
  p = fma(p, f, 1.0 / 362880.0);
  p = fma(p, f, 1.0 / 40320.0);
  p = fma(p, f, 1.0 / 5040.0);
  p = fma(p, f, 1.0 / 720.0);
  p = fma(p, f, 1.0 / 120.0);
  p = fma(p, f, 1.0 / 24.0);
  p = fma(p, f, 1.0 / 6.0);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return p * __longlong_as_double((long long)(1023 + (int)n) << 52);
}
__device__ __forceinline__ u64 fixed44(double w) { return (u64)(w * 0x1p44 + 0.5); }

// Logits as unsigned integers that order as the logits do (-0 below +0 is made equal first).
__device__ __forceinline__ uint32_t order_key(float l) {
  const uint32_t u = __float_as_uint(l == 0.f ? 0.f : l);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// Bin of d = max - l >= 0: the upper 16 bits of d (8 of exponent, 7 of
// mantissa) from 2^-8 on; smaller ones share bin 0, from 2^8 on the last.
__device__ __forceinline__ int d_bin(float d) {
  const int k = (int)(__float_as_uint(d) >> 16) - ((127 - 8) << 7);
  return min(max(k, 0), kBins - 1);
}

struct SampleK {
  const float* logits;
  long long lstride;
  int V;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniforms;
  int32_t* tokens;
  float* probs;
  long long pstride;
  int* err;
  int vec;  // rows of logits may be read in 16-byte pieces
  int pvec; // rows of probs may be written in them
};

struct Shared {
  union {
    struct {
      u64 mass[kBins];
      uint32_t count[kBins];
    } h;
    u64 list[kCap];
  };
  u64 tsum[kMaxTiles];
  u64 red[kWaves];
  u64 out64[4];
  int out32[4];
};

// All threads: sum / exclusive prefix over the workgroup in thread order.
__device__ __forceinline__ u64 wg_scan(u64 v, u64* sh, u64& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 inc = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const u64 up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  __syncthreads();
  if (lane == 63) sh[wave] = inc;
  __syncthreads();
  u64 base = 0, t = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) base = t;
    t += sh[w];
  }
  total = t;
  return base + inc - v;
}

// f(j, l[4]) for every four tokens j .. j+3 of the row, thread t of each
// round the four at round * 4096 + 4 t; tokens past the end are -inf.
template <typename F>
__device__ __forceinline__ void each4(const SampleK& a, const float* __restrict__ row, F f) {
  const int rounds = (a.V + 4 * kThreads - 1) / (4 * kThreads);
  for (int r = 0; r < rounds; ++r) {
    const int j = r * 4 * kThreads + 4 * (int)threadIdx.x;
    float l[4];
    if (a.vec && j + 3 < a.V) {
      const f32x4 q = *reinterpret_cast<const f32x4*>(row + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) l[e] = q[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) l[e] = j + e < a.V ? row[j + e] : -INFINITY;
    }
    f(r, j, l);
  }
}

// Sorts list[0..n) ascending, n a power of two.
__device__ void bitonic_sort(u64* list, int n) {
  for (int k = 2; k <= n; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      for (int t = threadIdx.x; t < n / 2; t += kThreads) {
        const int i = 2 * t - (t & (j - 1)), p = i + j;
        const u64 x = list[i], y = list[p];
        if ((x > y) == ((i & k) == 0)) {
          list[i] = y;
          list[p] = x;
        }
      }
    }
  __syncthreads();
}

// What is kept of a row: tokens above logit tau, those equal to it up to index
// tau_idx, each with weight >= min_p.
struct Keep {
  float tau;
  int tau_idx;
};

struct RadixOut {
  uint32_t key;    // of the last token
  uint32_t need;   // how many of the tokens with this key are kept (>= 1)
  u64 mass;        // of the tokens kept
};

// Radix search: the last token, in order, at which the count reaches k (by_mass
// false) or the mass reaches `target`; finite logits only.
template <typename W>
__device__ RadixOut radix_search(const SampleK& a, const float* row, Shared& sh, bool by_mass, u64 target, W weight) {
  uint32_t prefix = 0, mask = 0;
  u64 before = 0, mass_before = 0;  // of the tokens above the current prefix: count (or mass), mass
  uint32_t ties = 0;
  u64 tie_w = 0;
  const int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
  for (int p = 0; p < 3; ++p) {
    const int sft = shifts[p], nb = 1 << widths[p];
    __syncthreads();
    for (int i = threadIdx.x; i < nb; i += kThreads) {
      sh.h.mass[i] = 0;
      sh.h.count[i] = 0;
    }
    __syncthreads();
    each4(a, row, [&](int, int, const float(&l)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t k = order_key(l[e]);
        if (l[e] != -INFINITY && (k & mask) == prefix) {
          const int bin = (k >> sft) & (nb - 1);
          atomicAdd(&sh.h.count[bin], 1u);
          const u64 w = weight(l[e]);
          if (w) atomicAdd(&sh.h.mass[bin], w);
        }
      }
    });
    __syncthreads();
    // from the largest bin down: thread t holds bins nb-1-2t, nb-2-2t
    const int b0 = nb - 1 - 2 * (int)threadIdx.x;
    const u64 c0 = b0 >= 0 ? sh.h.count[b0] : 0, c1 = b0 >= 1 ? sh.h.count[b0 - 1] : 0;
    const u64 m0 = b0 >= 0 ? sh.h.mass[b0] : 0, m1 = b0 >= 1 ? sh.h.mass[b0 - 1] : 0;
    u64 tot;
    const u64 cb = wg_scan(by_mass ? m0 + m1 : c0 + c1, sh.red, tot);
    const u64 mb = wg_scan(m0 + m1, sh.red, tot);
    const u64 s0 = by_mass ? m0 : c0, s1 = by_mass ? m1 : c1;
    const u64 x0 = before + cb, x1 = x0 + s0, x2 = x1 + s1;
    // (a target of 0 mass is met by the very first token: it counts as 1)
    const u64 want = target ? target : 1;
    if (x0 < want && want <= x1) {
      sh.out32[0] = b0;
      sh.out64[0] = x0;
      sh.out64[1] = mass_before + mb;
      sh.out32[1] = (int)c0;
      sh.out64[2] = m0;
    } else if (x1 < want && want <= x2) {
      sh.out32[0] = b0 - 1;
      sh.out64[0] = x1;
      sh.out64[1] = mass_before + mb + m0;
      sh.out32[1] = (int)c1;
      sh.out64[2] = m1;
    }
    __syncthreads();
    prefix |= (uint32_t)sh.out32[0] << sft;
    mask |= (uint32_t)(nb - 1) << sft;
    before = sh.out64[0];
    mass_before = sh.out64[1];
    ties = (uint32_t)sh.out32[1];
    tie_w = sh.out64[2];
  }
  // `ties` equal logits of one weight each
  const u64 each = tie_w / (ties ? ties : 1), want = target ? target : 1;
  u64 need = by_mass ? (each ? (want - before + each - 1) / each : 1) : want - before;
  need = need < 1 ? 1 : need > ties ? ties : need;
  return {prefix, (uint32_t)need, mass_before + need * each};
}

// Index of the need-th (from 1) token with logit tau, in index order.
__device__ int nth_equal(const SampleK& a, const float* row, Shared& sh, float tau, uint32_t need) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  for (int i = threadIdx.x; i < kMaxTiles; i += kThreads) sh.tsum[i] = 0;
  __syncthreads();
  each4(a, row, [&](int r, int, const float(&l)[4]) {
    int c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) c += l[e] == tau;
    for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o);
    if (lane == 0) sh.tsum[r * kWaves + wave] = c;
  });
  __syncthreads();
  u64 tot;
  const u64 c0 = sh.tsum[2 * threadIdx.x], c1 = sh.tsum[2 * threadIdx.x + 1];
  const u64 base = wg_scan(c0 + c1, sh.red, tot);
  if (base < need && need <= base + c0 + c1) {
    const bool second = need > base + c0;
    sh.out32[0] = 2 * threadIdx.x + second;
    sh.out32[1] = (int)(need - base - (second ? c0 : 0));
  }
  __syncthreads();
  const int tile = sh.out32[0], rest = sh.out32[1];
  if (wave == 0) {
    int c = 0, j = tile * kTile + 4 * lane;
    for (int e = 0; e < 4; ++e) c += j + e < a.V && row[j + e] == tau;
    int inc = c;
    for (int o = 1; o < kWave; o <<= 1) {
      const int up = __shfl_up(inc, o);
      if (lane >= o) inc += up;
    }
    if (inc - c < rest && rest <= inc) {
      int left = rest - (inc - c);
      for (int e = 0; e < 4; ++e)
        if (j + e < a.V && row[j + e] == tau && --left == 0) sh.out32[2] = j + e;
    }
  }
  __syncthreads();
  return sh.out32[2];
}

// One workgroup per row.
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleK a) {
  __shared__ Shared sh;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
  const float* row = a.logits + (size_t)r * a.lstride;
  const float T = a.temperature ? a.temperature[r] : 1.f, P = a.top_p ? a.top_p[r] : 1.f, Q = a.min_p ? a.min_p[r] : 0.f;
  const float u = a.uniforms[r];
  int K = a.top_k ? a.top_k[r] : 0;
  if (K <= 0 || K > V) K = V;
  const bool greedy = T == 0.f;
  if (greedy) K = 1;

  // 1. the max; a NaN shows as a count
  float m = -INFINITY;
  int nan = 0;
  each4(a, row, [&](int, int, const float(&l)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m = fmaxf(m, l[e]);
      nan |= l[e] != l[e];
    }
  });
  for (int o = 32; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor(m, o));
    nan |= __shfl_xor(nan, o);
  }
  if (lane == 0) sh.red[wave] = ((u64)(nan != 0) << 32) | __float_as_uint(m);
  __syncthreads();
  m = -INFINITY;
  for (int w = 0; w < kWaves; ++w) {
    m = fmaxf(m, __uint_as_float((uint32_t)sh.red[w]));
    nan |= (int)(sh.red[w] >> 32);
  }
  const bool ok = T >= 0.f && T < INFINITY && P >= 0.f && Q >= 0.f && Q <= 1.f && u >= 0.f && u < 1.f && !nan &&
                  m > -INFINITY && m < INFINITY;
  if (!ok) {
    if (tid == 0) {
      a.tokens[r] = -1;
      flag_error(a.err, kErrSampling);
    }
    if (a.probs)
      for (int j = tid; j < V; j += kThreads) a.probs[(size_t)r * a.pstride + j] = 0.f;
    return;
  }
  const double md = m, scale = 1.4426950408889634074 / (greedy ? 1.0 : (double)T), mind = Q;
  auto weight64 = [&](float l) { return exp2_64(((double)l - md) * scale); };
  auto weight = [&](float l) { return fixed44(weight64(l)); };
  const bool by_count = K < V, by_mass = P < 1.f;

  Keep keep{-INFINITY, V};
  u64 total = 0;
  int token = -1;
  bool listed = false;
  if (by_count || by_mass) {
    // 2. the histogram
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) {
      sh.h.mass[i] = 0;
      sh.h.count[i] = 0;
    }
    __syncthreads();
    each4(a, row, [&](int, int, const float(&l)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (l[e] != -INFINITY) {
          const int bin = d_bin(m - l[e]);
          atomicAdd(&sh.h.count[bin], 1u);
          if (!by_count) {
            const u64 w = weight(l[e]);
            if (w) atomicAdd(&sh.h.mass[bin], w);
          }
        }
    });
    __syncthreads();
    u64 ctot, mtot;
    const u64 c0 = sh.h.count[2 * tid], c1 = sh.h.count[2 * tid + 1];
    const u64 m0 = by_count ? 0 : sh.h.mass[2 * tid], m1 = by_count ? 0 : sh.h.mass[2 * tid + 1];
    const u64 cb = wg_scan(c0 + c1, sh.red, ctot), mb = wg_scan(m0 + m1, sh.red, mtot);
    // the bin where the count reaches min(K, finite tokens), or the mass the target
    const u64 kk = min((u64)K, ctot);
    u64 target = by_count ? 0 : (u64)ceil((double)P * (double)mtot);
    {
      const u64 want = by_count ? kk : (target ? target : 1);
      const u64 x0 = by_count ? cb : mb, s0 = by_count ? c0 : m0, s1 = by_count ? c1 : m1;
      if (x0 < want && want <= x0 + s0) {
        sh.out32[0] = 2 * tid;
        sh.out64[0] = cb + c0;
      } else if (x0 + s0 < want && want <= x0 + s0 + s1) {
        sh.out32[0] = 2 * tid + 1;
        sh.out64[0] = cb + c0 + c1;
      }
    }
    __syncthreads();
    const int bin = sh.out32[0];
    const int n = (int)min(sh.out64[0], (u64)kCap + 1);
    if (n <= kCap) {
      // 3. the tokens up to that bin, sorted by (logit descending, index)
      listed = true;
      if (tid == 0) sh.out32[1] = 0;
      __syncthreads();
      each4(a, row, [&](int, int j, const float(&l)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (l[e] != -INFINITY && d_bin(m - l[e]) <= bin) {
            const int at = atomicAdd(&sh.out32[1], 1);
            if (at < kCap) sh.list[at] = ((u64)~order_key(l[e]) << 32) | (uint32_t)(j + e);
          }
      });
      __syncthreads();
      int n2 = 2;
      while (n2 < n) n2 <<= 1;
      for (int i = n + tid; i < n2; i += kThreads) sh.list[i] = ~0ull;
      bitonic_sort(sh.list, n2);
      // prefix sums of the weights, four tokens a thread
      u64 w[4], ls = 0, tot;
      double wd[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * tid + e;
        wd[e] = i < n && i < (int)kk ? weight64(key_logit(~(uint32_t)(sh.list[i] >> 32))) : 0.0;
        w[e] = fixed44(wd[e]);
        ls += w[e];
      }
      u64 run = wg_scan(ls, sh.red, tot);
      if (by_count) target = by_mass ? (u64)ceil((double)P * (double)tot) : ~0ull;
      // kept: i < kk, the sum before it below the target (or i = 0), w >= min_p
      int cnt = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * tid + e;
        cnt += i < n && i < (int)kk && (i == 0 || run < target) && wd[e] >= mind;
        run += w[e];
      }
      u64 all;
      wg_scan((u64)cnt, sh.red, all);
      const int L = (int)all;
      const u64 last = sh.list[L - 1];
      keep = {key_logit(~(uint32_t)(last >> 32)), (int)(uint32_t)last};
      // the kept tokens in index order
      int l2 = 2;
      while (l2 < L) l2 <<= 1;
      __syncthreads();
      for (int i = tid; i < l2; i += kThreads) {
        const u64 v = i < L ? sh.list[i] : ~0ull;
        sh.list[i] = (v << 32) | (v >> 32);
      }
      bitonic_sort(sh.list, l2);
      ls = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * tid + e;
        w[e] = i < L ? weight(key_logit(~(uint32_t)sh.list[i])) : 0;
        ls += w[e];
      }
      run = wg_scan(ls, sh.red, total);
      const u64 t = (u64)((double)u * (double)total);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (run <= t && t < run + w[e]) sh.out32[2] = (int)(uint32_t)(sh.list[4 * tid + e] >> 32);
        run += w[e];
      }
      __syncthreads();
      token = sh.out32[2];
    } else {
      RadixOut x{};
      if (by_count) {
        x = radix_search(a, row, sh, false, kk, weight);
        target = (u64)ceil((double)P * (double)x.mass);
      }
      if (by_mass) x = radix_search(a, row, sh, true, target, weight);
      const float tau = key_logit(x.key);
      keep = {tau, nth_equal(a, row, sh, tau, x.need)};
    }
  }
  auto kept = [&](float l, int j) { return l != -INFINITY && (l > keep.tau || (l == keep.tau && j <= keep.tau_idx)); };
  if (!listed) {
    // the draw over the whole row: weights of 256-token tiles, the tile, the token
    __syncthreads();
    for (int i = tid; i < kMaxTiles; i += kThreads) sh.tsum[i] = 0;
    __syncthreads();
    each4(a, row, [&](int rd, int j, const float(&l)[4]) {
      u64 s = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (kept(l[e], j + e)) {
          const double w = weight64(l[e]);
          if (w >= mind) s += fixed44(w);
        }
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
      if (lane == 0) sh.tsum[rd * kWaves + wave] = s;
    });
    __syncthreads();
    const u64 s0 = sh.tsum[2 * tid], s1 = sh.tsum[2 * tid + 1];
    const u64 base = wg_scan(s0 + s1, sh.red, total);
    const u64 t = (u64)((double)u * (double)total);
    if (base <= t && t < base + s0 + s1) {
      const bool second = t >= base + s0;
      sh.out32[0] = 2 * tid + second;
      sh.out64[0] = base + (second ? s0 : 0);
    }
    __syncthreads();
    if (wave == 0) {
      const int j = sh.out32[0] * kTile + 4 * lane;
      u64 w[4], ls = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = 0;
        if (j + e < V && kept(row[j + e], j + e)) {
          const double x = weight64(row[j + e]);
          if (x >= mind) w[e] = fixed44(x);
        }
        ls += w[e];
      }
      u64 inc = ls;
      for (int o = 1; o < kWave; o <<= 1) {
        const u64 up = __shfl_up(inc, o);
        if (lane >= o) inc += up;
      }
      u64 run = sh.out64[0] + inc - ls;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (run <= t && t < run + w[e]) sh.out32[2] = j + e;
        run += w[e];
      }
    }
    __syncthreads();
    token = sh.out32[2];
  }
  if (tid == 0) a.tokens[r] = token;
  if (a.probs) {
    const double inv = 0x1p44 / (double)total;
    float* out = a.probs + (size_t)r * a.pstride;
    each4(a, row, [&](int, int j, const float(&l)[4]) {
      f32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double w = kept(l[e], j + e) ? weight64(l[e]) : 0.0;
        p[e] = w >= mind ? (float)(w * inv) : 0.f;
      }
      if (a.pvec && j + 3 < V)
        *reinterpret_cast<f32x4*>(out + j) = p;
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < V) out[j + e] = p[e];
    });
  }
}

}  // namespace
}  // namespace nj

using namespace nj;

namespace {
constexpr int kSampleMaxVocab = 524288;
bool sample_sizes(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1 || vocab > kSampleMaxVocab)
    return !set_last_error(NJ_EINVAL, "sample: rows must be >= 1 and vocab in 1 .. %d", kSampleMaxVocab);
  return true;
}
}  // namespace

extern "C" {

size_t nightjar_sample_workspace_bytes(int32_t rows, int32_t vocab) { return sample_sizes(rows, vocab) ? 256 : 0; }

int nightjar_sample(const float* logits, int64_t logits_stride, int32_t rows, int32_t vocab, const float* temperature,
                    const int32_t* top_k, const float* top_p, const float* min_p, const float* uniforms,
                    int32_t* tokens, float* probs, int64_t probs_stride, void* workspace, size_t workspace_bytes,
                    void* stream) {
  if (!sample_sizes(rows, vocab)) return NJ_EINVAL;
  if (!logits || !uniforms || !tokens || !workspace) return set_last_error(NJ_EINVAL, "sample: a required pointer is NULL");
  if (logits_stride < vocab || (probs && probs_stride < vocab))
    return set_last_error(NJ_EINVAL, "sample: a row stride is smaller than vocab");
  if (probs) {
    const uintptr_t l0 = (uintptr_t)logits, l1 = l0 + ((size_t)(rows - 1) * logits_stride + vocab) * 4;
    const uintptr_t p0 = (uintptr_t)probs, p1 = p0 + ((size_t)(rows - 1) * probs_stride + vocab) * 4;
    if (l0 < p1 && p0 < l1) return set_last_error(NJ_EINVAL, "sample: probs and logits overlap");
  }
  const size_t need = nightjar_sample_workspace_bytes(rows, vocab);
  if (workspace_bytes < need) return set_last_error(NJ_EINVAL, "sample: workspace too small: %zu < %zu bytes", workspace_bytes, need);
  if (((uintptr_t)workspace & 255) != 0) return set_last_error(NJ_EINVAL, "sample: workspace must be 256-byte aligned");
  const bool lv = ((uintptr_t)logits & 15) == 0 && logits_stride % 4 == 0;
  const bool pv = ((uintptr_t)probs & 15) == 0 && probs_stride % 4 == 0;
  SampleK a{logits, logits_stride, vocab, temperature, top_k, top_p, min_p, uniforms, tokens, probs, probs_stride,
            static_cast<int*>(workspace), lv, pv};
  hipLaunchKernelGGL(sample_kernel, dim3(rows), dim3(kThreads), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "sample: %s", hipGetErrorString(e));
}

}  // extern "C"
