// Sampling with temperature, top-k, top-p and min-p from given uniforms.
//
// What decides -- which tokens are kept, and which is drawn -- is made of
// comparisons of logits, counts, and sums of weights w = exp((l - max) / T).  The
// weights are computed and summed in 64 bits (fp32 ones would move a border between
// two tokens every few ten thousand rows of a 150k vocabulary), in an order that does
// not depend on how the work is split.
//
// top-k, top-p and min-p each keep a prefix of the tokens ordered by (logit
// descending, index ascending), and so do they together.  The vocabulary is cut into
// tiles of 256 tokens:
//   sample_tiles  (rows x tile groups) reads every logit once: each tile's max,
//                 and, where the row needs it, its weights' sum relative to that max.
//   sample_rows   (one workgroup per row) knows from the tiles' maxima which tiles
//                 can hold kept tokens -- the k-th largest tile max bounds the k-th
//                 largest logit from below -- reads only those, sorts what they hold
//                 above the bound in LDS, and keeps and draws there.  A row that is
//                 not truncated is drawn from the tiles' sums and one tile.
//                 A row that keeps more tokens than the list holds goes the long way:
//                 a histogram of the row brackets the last token kept, and a pass over
//                 it sums what lies above and lists the bracket.
//   sample_probs  (rows x tile groups, if wanted) writes the distribution; tiles
//                 without a kept token are written without being read.
// A vocabulary of up to 64 tiles takes the three in one launch.
// Bound by the one read of the logits (and the write of the distribution) in large
// batches: 256 untruncated rows of 152064 57 us, 2.7 TB/s, 61 rows of 128256 by top-p with
// the distribution 32 us; by the chain of a row's dependent steps in small ones: one row by
// top-k and top-p 14 us; by a long row's two passes where there is one: 100 flat rows of
// 152064 by top-p 123 us.
#include <limits.h>

#include "../../include/nightjar_serve.h"
#include "common.h"
#include "kernels.h"

namespace nj {
namespace {

constexpr int kErrSampling = 32;  // NJ_DEV_BAD_SAMPLING
constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 4096, kBitBins = 2048;
constexpr int kCap = 4096;        // tokens of a list
constexpr int kTile = 256;        // tokens per running-sum tile (four per lane of a wave)
constexpr int kMaxTiles = 2048;   // V <= 524288
constexpr int kSmallTiles = 4 * kWaves;  // a small vocabulary: four tiles a wave of one workgroup
typedef unsigned long long u64;

// exp2(x) for x <= 0 in 64 bits: 2^n (1 + f q(f)), |f| <= 1/2, where q is the polynomial
// that meets (2^f - 1) / f at the nine Chebyshev points of that interval: relative error
// below 4e-14.  exp2(0) = 1 exactly; below 2^-1020 (and at -inf) 2^-1020.  n is rounded by
// adding 1.5 * 2^52, whose low word it leaves it in, and goes to the exponent's bits:
// additions only, 64-bit roundings and conversions being slow.
__device__ __forceinline__ double exp2_64(double x) {
  x = fmax(x, -1020.0);
  const double big = x + 0x1.8p52, f = x - (big - 0x1.8p52);
  double p = 0x1.b63871ee00eb4p-24;
  p = fma(p, f, 0x1.63d13637e6140p-20);
  p = fma(p, f, 0x1.ffcb952643063p-17);
  p = fma(p, f, 0x1.4308ac85a8ca4p-13);
  p = fma(p, f, 0x1.5d87fe86f8453p-10);
  p = fma(p, f, 0x1.3b2ab7181b769p-7);
  p = fma(p, f, 0x1.c6b08d7047e8ap-5);
  p = fma(p, f, 0x1.ebfbdff823cedp-3);
  p = fma(p, f, 0x1.62e42fefa39efp-1);
  p = fma(p, f, 1.0);
  return __hiloint2double(__double2hiint(p) + (int)((uint32_t)__double2loint(big) << 20), __double2loint(p));
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
struct RowHead {   // what sample_probs needs of a row
  double inv;      // 1 / total weight; 0: the row could not be sampled
  float max, tau;  // kept: logits above tau, and those equal to it up to index tau_idx
  int tau_idx;
};

struct SampleK {
  const float* logits;
  long long lstride;
  int V, ntile;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniforms;
  int32_t* tokens;
  float* probs;
  long long pstride;
  int* err;
  double* tmass;  // [rows][ntile]: sum of exp((l - tile max) / T) over the tile
  float* tmax;    // [rows][ntile]: tile max; +inf if the tile holds a NaN
  RowHead* head;  // [rows]
  int vec;        // rows of logits may be read in 16-byte pieces
  int pvec;       // rows of probs may be written in them
};

// A row's settings.  mass: the tiles' sums are needed (top-p without top-k, or no
// truncation at all).
struct RowSet {
  float T, P, Q, u;
  int K;
  bool ok, greedy, by_count, by_mass, mass;
  double scale;  // log2 e / T
};
__device__ __forceinline__ RowSet row_set(const SampleK& a, int r) {
  RowSet s;
  s.T = a.temperature ? a.temperature[r] : 1.f;
  s.P = a.top_p ? a.top_p[r] : 1.f;
  s.Q = a.min_p ? a.min_p[r] : 0.f;
  s.u = a.uniforms[r];
  s.K = a.top_k ? a.top_k[r] : 0;
  if (s.K <= 0 || s.K > a.V) s.K = a.V;
  s.ok = s.T >= 0.f && s.T < INFINITY && s.P >= 0.f && s.Q >= 0.f && s.Q <= 1.f && s.u >= 0.f && s.u < 1.f;
  s.greedy = s.T == 0.f;
  s.by_count = s.K < a.V;
  s.by_mass = s.P < 1.f;
  s.mass = s.ok && !s.greedy && !s.by_count && (s.by_mass || s.Q == 0.f);
  s.scale = 1.4426950408889634074 / (s.greedy ? 1.0 : (double)s.T);
  return s;
}

// Four tokens of a lane in each of the wave's N tiles (the same in all lanes): tile
// t[i]'s tokens 4 lane ..; past the end -inf.  Whole tiles are loaded without conditions,
// so that all loads are in flight together.
template <int N>
__device__ __forceinline__ void tile_quads(const SampleK& a, const float* __restrict__ row, const int (&t)[N], f32x4 (&l)[N]) {
  const int j = 4 * (int)(threadIdx.x & 63);
  bool whole = a.vec;
#pragma unroll
  for (int i = 0; i < N; ++i) whole &= (t[i] + 1) * kTile <= a.V;
  if (whole) {
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = *reinterpret_cast<const f32x4*>(row + t[i] * kTile + j);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) l[i][e] = t[i] * kTile + j + e < a.V ? row[t[i] * kTile + j + e] : -INFINITY;
  }
}
__device__ __forceinline__ f32x4 tile_quad(const SampleK& a, const float* __restrict__ row, int t) {
  f32x4 l[1];
  tile_quads<1>(a, row, {__builtin_amdgcn_readfirstlane(t)}, l);
  return l[0];
}
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Running sums over a wave (inclusive) in a fixed order, each step one move between
// lanes in registers; lane 63 ends with the wave's.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T dpp_add(T v) {
  union {
    T v;
    int h[sizeof(T) / 4];
  } x{v}, y;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) y.h[i] = __builtin_amdgcn_update_dpp(0, x.h[i], CTRL, ROWS, 0xf, false);
  return v + y.v;
}
template <typename T>
__device__ __forceinline__ T row_scan(T v) {  // over each 16 lanes
  v = dpp_add<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  return dpp_add<0x118, 0xf>(v);
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
  v = row_scan(v);
  v = dpp_add<0x142, 0xa>(v);     // row_bcast 15, 31
  return dpp_add<0x143, 0xc>(v);
}
template <typename T>
__device__ __forceinline__ T lane_value(T v, int lane) {
  union {
    T v;
    int h[sizeof(T) / 4];
  } x{v};
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) x.h[i] = __builtin_amdgcn_readlane(x.h[i], lane);
  return x.v;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_max(float v) {
  const int i = __float_as_int(v);
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(i, i, CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float v) {
  v = dpp_max<0x111, 0xf>(v);
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  return lane_value(v, 63);
}

// A wave's tiles t0 .., read at once: their maxima and, if asked for, sums.
constexpr int kWaveTiles = 4;
__device__ __forceinline__ void tile_stats(const SampleK& a, int r, int t0) {
  const int lane = threadIdx.x & 63;
  const float* row = a.logits + (size_t)r * a.lstride;
  f32x4 l[kWaveTiles];
  tile_quads<kWaveTiles>(a, row, {t0, t0 + 1, t0 + 2, t0 + 3}, l);
  const RowSet s = row_set(a, r);
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i) {
    if (t0 + i >= a.ntile) break;  // uniform
    float m = fmaxf(fmaxf(l[i][0], l[i][1]), fmaxf(l[i][2], l[i][3]));
    const bool nan = l[i][0] != l[i][0] || l[i][1] != l[i][1] || l[i][2] != l[i][2] || l[i][3] != l[i][3];
    m = wave_max(nan ? INFINITY : m);
    if (lane == 0) a.tmax[(size_t)r * a.ntile + t0 + i] = m;
    if (s.mass) {
      double w = 0.0;
      if (m > -INFINITY && m < INFINITY) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w += exp2_64(((double)l[i][e] - (double)m) * s.scale);
        w = wave_scan(w);
      }
      if (lane == 63) a.tmass[(size_t)r * a.ntile + t0 + i] = w;
    }
  }
}
// grid (rows, ceil(ntile / kTilesPerWg))
constexpr int kTilesPerWg = 4 * kWaveTiles;
__global__ __launch_bounds__(256) void sample_tiles_kernel(SampleK a) {
  tile_stats(a, blockIdx.x, blockIdx.y * kTilesPerWg + wave_id() * kWaveTiles);
}

struct Shared {
  union {
    __attribute__((aligned(16))) uint32_t bins[2 * kBins];
    struct {
      u64 mass[kBitBins];
      uint32_t count[kBitBins];
    } h;
    __attribute__((aligned(16))) u64 list[kCap];
  };
  union {
    u64 tsum[kMaxTiles];   // long way: tile sums
    double tmass[kMaxTiles];
  };
  __attribute__((aligned(16))) float tmax[kMaxTiles];
  uint16_t tiles[kMaxTiles];  // tiles to read
  u64 red[kWaves];
  u64 out64[4];
  int out32[4];
};

// Sum over the threads before this one (and of all, in total), in a fixed order.
template <typename T>
__device__ __forceinline__ T wg_scan(T v, void* scratch, T& total) {
  T* sh = static_cast<T*>(scratch);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T inc = wave_scan(v);
  __syncthreads();
  if (lane == 63) sh[wave] = inc;
  __syncthreads();
  const T x = row_scan(sh[lane & (kWaves - 1)]);
  total = lane_value(x, kWaves - 1);
  return (wave ? lane_value(x, wave - 1) : T(0)) + (inc - v);
}
template <typename T>
__device__ __forceinline__ T wg_sum(T v, void* scratch) {
  T total;
  wg_scan(v, scratch, total);
  return total;
}
__device__ __forceinline__ float wg_max(float v, void* scratch) {
  float* sh = static_cast<float*>(scratch);
  v = wave_max(v);
  __syncthreads();
  sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return wave_max(sh[threadIdx.x & (kWaves - 1)]);
}
// (ints below 2^24 and INT_MAX, as floats are exact up to there)
__device__ __forceinline__ int wg_min(int v, void* scratch) {
  const float m = wg_max(v == INT_MAX ? -INFINITY : -(float)v, scratch);
  return m == -INFINITY ? INT_MAX : (int)-m;
}

// f(round, j, l[4]) for every four tokens j .. j+3 of the row, thread t of each round
// the four at round * 4096 + 4 t; tokens past the end are -inf.  While four whole rounds
// are worked on, the next four are loaded, without conditions: a load under one is
// waited for before its register's other value can be written.
template <typename F>
__device__ __forceinline__ void each4(const SampleK& a, const float* __restrict__ row, F f) {
  constexpr int NR = 4;
  const int whole = a.vec ? a.V / (4 * kThreads) / NR * NR : 0, t4 = 4 * (int)threadIdx.x;
  if (whole) {
    const f32x4* src = reinterpret_cast<const f32x4*>(row) + threadIdx.x;
    f32x4 next[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) next[i] = src[i * kThreads];
#pragma unroll 1
    for (int r = 0; r < whole; r += NR) {
      f32x4 l[NR];
      const int ahead = min(r + NR, whole - NR);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        l[i] = next[i];
        next[i] = src[(ahead + i) * kThreads];
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) f(r + i, (r + i) * 4 * kThreads + t4, l[i]);
    }
  }
#pragma unroll 1
  for (int r = whole; r * 4 * kThreads < a.V; ++r) {
    const int j = r * 4 * kThreads + t4;
    f32x4 l;
    if (a.vec && j + 3 < a.V)
      l = *reinterpret_cast<const f32x4*>(row + j);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) l[e] = j + e < a.V ? row[j + e] : -INFINITY;
    f(r, j, l);
  }
}

// Sorts list[0..n) ascending, 1 <= n <= kCap, keys distinct.  Up to 256 keys each finds
// its place by counting the smaller ones; up to 1024 go through a bitonic network with a
// key a thread, whose partners in the wave meet in registers (45 of its 55 steps); more
// through one in LDS, two barriers a step.
__device__ __forceinline__ void sort_list(u64* list, int n) {
  const int t = threadIdx.x;
  int n2 = kWave;
  while (n2 < n) n2 <<= 1;
  for (int i = n + t; i < n2; i += kThreads) list[i] = ~0ull;
  if (n <= 256) {
    int* rank = reinterpret_cast<int*>(list + kThreads);
    if (t < n2) rank[t] = 0;
    __syncthreads();
    const int parts = kThreads / n2, i = t & (n2 - 1), per = n2 / parts;
    const u64 x = list[i];
    int cnt = 0;
#pragma unroll 4
    for (int j = t / n2 * per; j < (t / n2 + 1) * per; ++j) cnt += list[j] < x;
    atomicAdd(&rank[i], cnt);
    __syncthreads();
    if (t < n) list[rank[t]] = x;
  } else if (n <= kThreads) {
    __syncthreads();
    const bool in = t < n2;  // (whole waves)
    u64 x = in ? list[t] : 0;
    for (int k = 2; k <= n2; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        u64 y = 0;
        if (j < kWave) {
          y = __shfl_xor(x, j);
        } else {
          __syncthreads();
          if (in) list[t] = x;
          __syncthreads();
          if (in) y = list[t ^ j];
        }
        const bool low = (t & j) == 0, up = (t & k) == 0;
        x = (x < y) == (low == up) ? x : y;
      }
    __syncthreads();
    if (in) list[t] = x;
  } else {
    for (int k = 2; k <= n2; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        __syncthreads();
        for (int p = t; p < n2 / 2; p += kThreads) {
          const int i = 2 * p - (p & (j - 1));
          const u64 x = list[i], y = list[i + j];
          if ((x > y) == ((i & k) == 0)) {
            list[i] = y;
            list[i + j] = x;
          }
        }
      }
  }
  __syncthreads();
}

struct RadixOut {
  uint32_t key;    // of the last token
  uint32_t need;   // how many of the tokens with this key are kept (>= 1)
  u64 mass;        // of the tokens kept
};

// Bin of d = max - l >= 0: the upper 17 bits of d (8 of exponent, 8 of mantissa)
// from 2^-8 on; smaller ones share bin 0, from 2^8 on the last.  A bin's relative
// width is 2^-8, so that it holds a per cent or two of a broad row at most, whatever the
// scale of the logits.
__device__ __forceinline__ int d_bin(float d) {
  const int k = (int)(__float_as_uint(d) >> 15) - ((127 - 8) << 8);
  return min(max(k, 0), kBins - 1);
}

// Radix search: the last token, in order, at which the count reaches k (by_mass
// false) or the mass reaches `target`; finite logits only.
template <typename W>
__device__ __forceinline__ RadixOut radix_search(const SampleK& a, const float* row, Shared& sh, bool by_mass, u64 target, W weight) {
  uint32_t prefix = 0, mask = 0;
  u64 before = 0, mass_before = 0;  // of the tokens above the current prefix: count (or mass), mass
  uint32_t ties = 0;
  u64 tie_w = 0, want = target ? target : 1;  // (a target of 0 is met by the very first token: it counts as 1)
  const int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
  for (int p = 0; p < 3; ++p) {
    const int sft = shifts[p], nb = 1 << widths[p];
    __syncthreads();
    for (int i = threadIdx.x; i < nb; i += kThreads) {
      sh.h.mass[i] = 0;
      sh.h.count[i] = 0;
    }
    __syncthreads();
    each4(a, row, [&](int, int, const f32x4& l) {
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
    u64 tot, mtot;
    const u64 cb = wg_scan(by_mass ? m0 + m1 : c0 + c1, sh.red, tot);
    const u64 mb = wg_scan(m0 + m1, sh.red, mtot);
    if (p == 0) want = min(want, tot);  // fewer finite logits than top_k
    const u64 s0 = by_mass ? m0 : c0, s1 = by_mass ? m1 : c1;
    const u64 x0 = before + cb, x1 = x0 + s0, x2 = x1 + s1;
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
  const u64 each = tie_w / (ties ? ties : 1);
  u64 need = by_mass ? (each ? (want - before + each - 1) / each : 1) : want - before;
  need = need < 1 ? 1 : need > ties ? ties : need;
  return {prefix, (uint32_t)need, mass_before + need * each};
}

// Index of the need-th (from 1) token with logit tau, in index order.
__device__ __forceinline__ int nth_equal(const SampleK& a, const float* row, Shared& sh, float tau, uint32_t need) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  for (int i = threadIdx.x; i < kMaxTiles; i += kThreads) sh.tsum[i] = 0;
  __syncthreads();
  each4(a, row, [&](int r, int, const f32x4& l) {
    int c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) c += l[e] == tau;
    c = wave_scan(c);
    if (lane == 63) sh.tsum[r * kWaves + wave] = c;
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
    const int inc = wave_scan(c);
    if (inc - c < rest && rest <= inc) {
      int left = rest - (inc - c);
      for (int e = 0; e < 4; ++e)
        if (j + e < a.V && row[j + e] == tau && --left == 0) sh.out32[2] = j + e;
    }
  }
  __syncthreads();
  return sh.out32[2];
}

// The tokens that `in` takes from the tiles whose max is at least `cut`, to sh.list in
// no order, as sort keys (logit descending, index); returns their number (more than
// kCap: the list is cut off).  Where tokens fall on tiles at random and kCap reach the
// cut, 1 - exp(-kCap / tiles) of the tiles hold one: with `guess` and more of them, none
// is read, and kCap + 1 returned.
template <typename F>
__device__ __forceinline__ int collect(const SampleK& a, const float* row, Shared& sh, float cut, bool guess, F in) {
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  __syncthreads();
  if (tid < 2) sh.out32[tid] = 0;
  __syncthreads();
  for (int t = tid; t < a.ntile; t += kThreads)
    if (sh.tmax[t] >= cut && sh.tmax[t] > -INFINITY) sh.tiles[atomicAdd(&sh.out32[0], 1)] = (uint16_t)t;
  __syncthreads();
  const int nq = __builtin_amdgcn_readfirstlane(sh.out32[0]);
  if (guess && nq > (1.f - __expf(-(float)kCap / a.ntile)) * a.ntile + 0.5f) return kCap + 1;
  constexpr int NI = 4;  // tiles in flight per wave
  for (int i = wave; i < nq; i += NI * kWaves) {
    f32x4 l[NI];
    int t[NI];
#pragma unroll
    for (int q = 0; q < NI; ++q) t[q] = __builtin_amdgcn_readfirstlane(sh.tiles[min(i + q * kWaves, nq - 1)]);
    tile_quads<NI>(a, row, t, l);
#pragma unroll
    for (int q = 0; q < NI; ++q) {
      if (i + q * kWaves >= nq) break;  // uniform
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool take = l[q][e] != -INFINITY && in(l[q][e]);
        const u64 who = __ballot(take);
        if (!who) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.out32[1], __popcll(who));
        at = __builtin_amdgcn_readfirstlane(at);
        if (guess && at > kCap) i = nq;  // (too many already)
        at += __popcll(who & ((1ull << lane) - 1));
        if (take && at < kCap) sh.list[at] = ((u64)~order_key(l[q][e]) << 32) | (uint32_t)(t[q] * kTile + 4 * lane + e);
      }
    }
  }
  __syncthreads();
  return sh.out32[1];
}

// The smallest d of bin b >= 1.
__device__ __forceinline__ float bin_edge(int b) { return __uint_as_float((uint32_t)(b + ((127 - 8) << 8)) << 15); }
// A bound from below of the logits whose bin is at most b (see d_bin).
__device__ __forceinline__ float bin_floor(float m, int b) {
  if (b >= kBins - 1) return -INFINITY;
  const float x = m - bin_edge(b + 1);
  return x - fabsf(x) * 0x1p-22f;
}

// This thread's four bins, copies joined, as running sums behind what comes before (x[0]).
template <typename T>
__device__ __forceinline__ void scan_bins(Shared& sh, T (&x)[5], T& all) {
  const uint4 a = reinterpret_cast<const uint4*>(sh.bins)[threadIdx.x], b = reinterpret_cast<const uint4*>(sh.bins + kBins)[threadIdx.x];
  const T n[4] = {(T)a.x + b.x, (T)a.y + b.y, (T)a.z + b.z, (T)a.w + b.w};
  x[0] = wg_scan(n[0] + n[1] + n[2] + n[3], sh.red, all);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i + 1] = x[i] + n[i];
}
// The first bin for whose running sum `reached` holds (it holds for all behind it too);
// INT_MAX if there is none.
template <typename F>
__device__ __forceinline__ int first_bin(Shared& sh, const u64 (&x)[5], F reached) {
  int b = INT_MAX;
#pragma unroll
  for (int i = 3; i >= 0; --i)
    if (reached(x[i + 1])) b = 4 * threadIdx.x + i;
  return wg_min(b, sh.red);
}
// The bin in which the running sum comes to k (0 < k <= the sum of all).
__device__ __forceinline__ int bin_of(Shared& sh, const uint32_t (&x)[5], uint32_t k) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (x[i] < k && k <= x[i + 1]) sh.out32[3] = 4 * threadIdx.x + i;
  __syncthreads();
  return sh.out32[3];
}
__device__ __forceinline__ void clear_bins(Shared& sh) {
  __syncthreads();
  for (int i = threadIdx.x; i < kBins / 2; i += kThreads) reinterpret_cast<uint4*>(sh.bins)[i] = uint4{0, 0, 0, 0};
  __syncthreads();
}
__device__ __forceinline__ void add_bin(Shared& sh, int bin, uint32_t v) { atomicAdd(&sh.bins[bin + (threadIdx.x & 1) * kBins], v); }

// The histogram of a row's mass, in units of which it has at most 2^31: a token's weight
// is computed in fp32 and cut to whole ones, and good for 2^-17.
__device__ __forceinline__ double mass_unit(double mass) { return 0x1p31 / mass; }
__device__ __forceinline__ uint32_t mass_units(float d, float scale, float shift) {
  return (uint32_t)__builtin_amdgcn_exp2f(fmaf(-d, scale, shift));
}
// Its bins are even in max - l, `per` to the unit: over 32 bits of weight, or as far as four
// times the lowest tile's max where that is nearer (a hot or narrow row).
__device__ __forceinline__ float mass_bins(float lowest, double scale) {
  return kBins / fmaxf(fminf((float)(32.0 / scale), 4.f * lowest), 0x1p-80f);
}
__device__ __forceinline__ int mass_bin(float x) { return (int)fminf(x, kBins - 1.f); }
// The bracket that it gives of the last token of a prefix of mass `want`: near <= (max - l) * per < far.
__device__ __forceinline__ void bracket(Shared& sh, const u64 (&x)[5], int V, double want, double unit, float& near, float& far) {
  const u64 lo = (u64)floor(want * unit), hi = (u64)ceil(want * unit);
  const int first = first_bin(sh, x, [&](u64 x) { return x + (x >> 16) + V >= lo; });
  const int last = first_bin(sh, x, [&](u64 x) { return x - (x >> 16) > hi; });
  near = (float)min(first, kBins - 1);
  far = last < kBins - 1 ? (float)(last + 1) : INFINITY;
}
// The sum of a wave's four tokens a lane that are kept and lie above the bracket, w >= least;
// `put` takes the kept tokens inside it (open: there is one).
template <typename K, typename W, typename P>
__device__ __forceinline__ double sum_above(const f32x4& l, int j, float m, float per, bool open, float near, float far, double least, K kept,
                                            W weight, P put) {
  double sum = 0.0;
  bool any = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = (m - l[e]) * per;
    const bool k = kept(l[e], j + e);
    any |= k && !(x < near) && x < far;
    const double w = weight(l[e]);
    // (where w < min_p above the bracket, nothing in it is kept either, so that the sum may lack these)
    if (k && (!open || x < near) && w >= least) sum += w;
  }
  if (open && __any(any)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = (m - l[e]) * per;
      if (kept(l[e], j + e) && !(x < near) && x < far) put(((u64)~order_key(l[e]) << 32) | (uint32_t)(j + e));
    }
  }
  return wave_scan(sum);
}

__device__ __forceinline__ float list_logit(u64 v) { return key_logit(~(uint32_t)(v >> 32)); }

// Sorts the n listed tokens; of them, the last in order at which their number, or the
// mass from `before` on, reaches `want` (the very last if none does), and the mass up to it.
template <typename W>
__device__ __forceinline__ u64 last_listed(Shared& sh, int n, u64 want, bool by_mass, u64 before, float& tau, int& tau_idx,
                                           W weight) {
  const int tid = threadIdx.x;
  sort_list(sh.list, n);
  u64 w[4], ls = 0, all;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = 4 * tid + e;
    w[e] = i < n ? weight(list_logit(sh.list[i])) : 0;
    ls += w[e];
  }
  u64 run = before + wg_scan(ls, sh.red, all), upto = 0;
  int at = INT_MAX;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = 4 * tid + e;
    run += w[e];
    if (i < n && at == INT_MAX && ((by_mass ? run >= want : (u64)i + 1 >= want) || i == n - 1)) {
      at = i;
      upto = run;
    }
  }
  const int last = wg_min(at, sh.red);
  if (at == last) sh.out64[1] = upto;
  __syncthreads();
  tau = list_logit(sh.list[last]);
  tau_idx = (int)(uint32_t)sh.list[last];
  return sh.out64[1];
}

// A row by one workgroup, its tiles' maxima and sums being known.
__device__ __forceinline__ void sample_row(const SampleK& a, int r, Shared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
  const float* row = a.logits + (size_t)r * a.lstride;
  const RowSet s = row_set(a, r);
  float m = -INFINITY;
  for (int t = tid; t < a.ntile; t += kThreads) {
    sh.tmax[t] = a.tmax[(size_t)r * a.ntile + t];
    m = fmaxf(m, sh.tmax[t]);
    if (s.mass) sh.tmass[t] = a.tmass[(size_t)r * a.ntile + t];
  }
  m = wg_max(m, sh.red);
  if (!s.ok || !(m > -INFINITY && m < INFINITY)) {  // (a NaN shows as +inf)
    if (tid == 0) {
      a.tokens[r] = -1;
      a.head[r] = {0.0, m, INFINITY, -1};
      flag_error(a.err, kErrSampling);
    }
    return;
  }
  const double md = m, mind = s.Q;
  auto weight = [&](float l) { return exp2_64(((double)l - md) * s.scale); };

  if (s.greedy) {  // the first tile that holds the max, and its first place there
    int first = INT_MAX;
    for (int t = tid; t < a.ntile; t += kThreads)
      if (sh.tmax[t] == m) {
        first = t;
        break;
      }
    first = wg_min(first, sh.red);
    int at = INT_MAX;
    if (wave == 0) {
      const f32x4 l = tile_quad(a, row, first);
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (l[e] == m) at = first * kTile + 4 * lane + e;
    }
    at = wg_min(at, sh.red);
    if (tid == 0) {
      a.tokens[r] = at;
      a.head[r] = {1.0, m, m, at};
    }
    return;
  }

  double mass = 0.0;  // of the whole row
  if (s.mass) {
    for (int t = tid; t < a.ntile; t += kThreads) {
      sh.tmass[t] = sh.tmax[t] > -INFINITY ? sh.tmass[t] * weight(sh.tmax[t]) : 0.0;
      mass += sh.tmass[t];
    }
    mass = wg_sum(mass, sh.red);
  }

  const bool whole = !s.by_count && !s.by_mass && s.Q == 0.f;  // no truncation: drawn from the tiles' sums

  // The short way: a logit that every kept token reaches, and the tokens above it.
  // top-k: some tile's max.  K tokens at least reach the K-th; where tokens fall on tiles
  // at random, n of them reach the max of rank (1 - exp(-n / tiles)) tiles: a little more
  // than K is aimed at.  Where that comes to all tiles, or falls short of K, a histogram of
  // the row (which costs a pass over it) gives the K-th token's bin.
  // top-p alone: guesses, lowered while the tokens above fall short of the target.
  // min-p alone: its own border (a little below: the test itself decides).
  float cut = -INFINITY;
  bool exact = false;
  constexpr int kManyTiles = 128;
  const double bit = s.T * 0.69314718055994530942;  // of weight, in logits
  int n = 0;
  bool listed = false;
  for (int round = 0; !listed && !whole && !(s.by_count && s.K > kCap); ++round) {
    if (s.by_count) {
      const int rank = (int)ceilf((1.f - __expf(-(1.1f * s.K + 4.f * sqrtf((float)s.K)) / a.ntile)) * a.ntile);
      exact = round > 0 || rank >= a.ntile;
      clear_bins(sh);
      if (exact)
        each4(a, row, [&](int, int, const f32x4& l) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (l[e] > -INFINITY) add_bin(sh, d_bin(m - l[e]), 1);
        });
      else
        for (int t = tid; t < a.ntile; t += kThreads) add_bin(sh, d_bin(m - sh.tmax[t]), 1);
      __syncthreads();
      uint32_t x[5], all;
      scan_bins(sh, x, all);
      cut = bin_floor(m, bin_of(sh, x, exact ? min((uint32_t)s.K, all) : max(min(rank, s.K), 1)));
    } else {
      // (top-p: 2^-5, -8, -12, -16, -24; selected, as a table would be read from memory)
      const float guess = round == 0 ? -5.f : round == 1 ? -8.f : round == 2 ? -12.f : round == 3 ? -16.f : -24.f;
      cut = !s.by_mass ? (float)(md + (log2(mind) - 1e-6) * bit) : round < 5 ? (float)(md + guess * bit) : -INFINITY;
      cut = fminf(cut, m) - fabsf(cut) * 0x1p-22f;
      if (s.by_mass && cut > -INFINITY && a.ntile > kManyTiles) {
        // The tokens above it hold no less than their tiles' maxima and no more than these tiles: is that, or (where many
        // tiles would be read) half way between, enough?
        double tops = 0.0, most = 0.0;
        for (int t = tid; t < a.ntile; t += kThreads)
          if (sh.tmax[t] >= cut) {
            tops += weight(sh.tmax[t]);
            most += sh.tmass[t];
          }
        if (__syncthreads_count(most > 0.0) > kManyTiles) most = 0.5 * (most + tops);
        if (wg_sum(most, sh.red) < (double)s.P * mass) continue;
      }
    }
    n = collect(a, row, sh, cut, !s.by_count, [&](float l) { return l >= cut; });
    if (n > kCap) break;
    if (s.by_count) {
      if (n < s.K && !exact) continue;
    } else if (s.by_mass) {
      double w = 0.0;
      for (int i = tid; i < n; i += kThreads) w += weight(list_logit(sh.list[i]));
      w = wg_sum(w, sh.red);
      if (w < (double)s.P * mass && cut > -INFINITY) continue;
    }
    listed = true;
  }
  float tau = -INFINITY;  // kept: above tau, and equal to it up to tau_idx
  int tau_idx = -1;
  if (listed) {
    const int kk = min(s.K, n);
    for (int i = tid; i < kMaxTiles; i += kThreads) sh.tsum[i] = 0;
    sort_list(sh.list, n);
    const bool four = n > kThreads;  // tokens a thread
    double w[4], ls = 0.0, tot;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = four ? 4 * tid + e : tid;
      w[e] = i < kk && (four || e == 0) ? weight(list_logit(sh.list[i])) : 0.0;
      ls += w[e];
    }
    double run = wg_scan(ls, sh.red, tot);
    // kept: the first K, the sum before below the target (or the first of all), w >= min_p
    const double target = !s.by_mass ? INFINITY : (double)s.P * (s.by_count ? tot : mass);
    int cnt = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = four ? 4 * tid + e : tid;
      if (i < kk && (four || e == 0) && (i == 0 || run < target) && w[e] >= mind) {
        ++cnt;
        atomicAdd(&sh.tsum[(uint32_t)sh.list[i] / kTile], fixed44(w[e]));
      }
      run += w[e];
    }
    const u64 last = sh.list[(four ? wg_sum(cnt, sh.red) : __syncthreads_count(cnt)) - 1];
    tau = list_logit(last);
    tau_idx = (int)(uint32_t)last;
  }

  // The long way, in passes over the row.  By count: a histogram over d_bin finds the
  // bin of the K-th token, a list of that bin the token.  By mass, the mass of what is
  // left so far being known: a histogram of fp32 weights in 32 bits (64-bit ones, added in
  // 64 bits, took twice as long) brackets the bin of the last token; the pass that
  // sums what lies above exactly lists the bracket, and the token is found there.  A list
  // too small (equal logits by the thousand) is replaced by a search over the logits' bits.
  auto kept = [&](float l, int j) { return l > tau || (l == tau && j <= tau_idx); };
  auto weight44 = [&](float l) { return fixed44(weight(l)); };
  enum { kCount, kMass, kBits, kSum, kDraw };
  bool mass_left = s.by_mass;  // top-p is still to do
  u64 goal = 0;                // of the search over the bits
  float per = 0.f;  // bins per unit of max - l
#pragma unroll 1
  for (int step = whole || listed ? kDraw : s.by_count ? kCount : s.by_mass ? kMass : kSum; step != kDraw;) {
    const double unit = mass_unit(mass), want = (double)s.P * mass;
    float near = 0.f, far = INFINITY;
    if (step == kBits) {
      const RadixOut x = radix_search(a, row, sh, s.by_mass && !mass_left, goal, weight44);
      tau = key_logit(x.key);
      tau_idx = nth_equal(a, row, sh, tau, x.need);
      step = kSum;
    }
    if (step == kMass) {
      float lowest = INFINITY;  // tile's max, of those with any token
      for (int t = tid; t < a.ntile; t += kThreads)
        if (sh.tmax[t] > -INFINITY) lowest = fminf(lowest, sh.tmax[t]);
      per = mass_bins(m + wg_max(-lowest, sh.red), s.scale);
    }
    if (step != kSum) {
      clear_bins(sh);
      const float scale = (float)s.scale, shift = (float)log2(unit);
      each4(a, row, [&](int, int j, const f32x4& l) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t u = l[e] > -INFINITY;
          const float d = m - l[e];
          if (step == kMass) u = kept(l[e], j + e) ? mass_units(d, scale, shift) : 0;
          if (u) add_bin(sh, step == kMass ? mass_bin(d * per) : d_bin(d), u);
        }
      });
      __syncthreads();
      if (step == kMass) {
        u64 x[5], all;
        scan_bins(sh, x, all);
        bracket(sh, x, V, want, unit, near, far);
      } else {
        uint32_t x[5], all;
        scan_bins(sh, x, all);
        const uint32_t k = min((uint32_t)s.K, all);  // (fewer finite logits than K)
        const int bin = bin_of(sh, x, k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * tid + i == bin) sh.out64[0] = x[i];
        const int nb = collect(a, row, sh, bin_floor(m, bin), false, [&](float l) { return d_bin(m - l) == bin; });
        if (nb > kCap) {
          step = kBits;
          goal = k;
          continue;
        }
        last_listed(sh, nb, k - sh.out64[0], false, 0, tau, tau_idx, [](float) { return (u64)0; });
        step = kSum;
      }
    }
    // the sums of the tiles: of what is kept, or of what lies above the bracket
    const bool open = step == kMass;
    const double least = !open && mass_left ? 0.0 : mind;  // (top-p is of what top-k keeps, before min-p)
    __syncthreads();
    for (int i = tid; i < kMaxTiles; i += kThreads) sh.tsum[i] = 0;
    if (tid == 0) sh.out32[1] = 0;
    __syncthreads();
    each4(a, row, [&](int rd, int j, const f32x4& l) {
      const double sum = sum_above(l, j, m, per, open, near, far, least, kept, weight, [&](u64 x) {
        const int at = atomicAdd(&sh.out32[1], 1);
        if (at < kCap) sh.list[at] = x;
      });
      if (lane == 63) sh.tsum[rd * kWaves + wave] = fixed44(sum);
    });
    __syncthreads();
    const u64 all = wg_sum(sh.tsum[2 * tid] + sh.tsum[2 * tid + 1], sh.red);
    if (!open) {
      mass = (double)all * 0x1p-44;
      step = mass_left ? kMass : kDraw;
      continue;
    }
    mass_left = false;
    const int nb = sh.out32[1];
    goal = (u64)ceil(want * 0x1p44);
    if (nb < 1 || nb > kCap) {
      step = kBits;
      continue;
    }
    last_listed(sh, nb, goal, true, all, tau, tau_idx, weight44);
    for (int i = tid; i < nb; i += kThreads) {
      const u64 x = sh.list[i];
      const int j = (int)(uint32_t)x;
      const double w = weight(list_logit(x));
      if (kept(list_logit(x), j) && w >= mind) atomicAdd(&sh.tsum[j / kTile], fixed44(w));
    }
    step = kDraw;
  }

  // the tile in which the running sum passes u * total, and the token
  __syncthreads();
  u64 m0 = 0, m1 = 0, all;  // (integers: exactly one thread's two tiles hold the place)
  if (whole) {
    if (2 * tid < a.ntile) m0 = fixed44(sh.tmass[2 * tid]);
    if (2 * tid + 1 < a.ntile) m1 = fixed44(sh.tmass[2 * tid + 1]);
  } else {
    m0 = sh.tsum[2 * tid];
    m1 = sh.tsum[2 * tid + 1];
  }
  const u64 base = wg_scan(m0 + m1, sh.red, all);
  const double total = (double)all * 0x1p-44, t = (double)s.u * total;
  const u64 place = (u64)((double)s.u * (double)all);
  if (base <= place && place < base + m0 + m1) {
    const bool second = place >= base + m0;
    sh.out32[0] = 2 * tid + second;
    sh.out64[0] = base + (second ? m0 : 0);
  }
  __syncthreads();
  const int tile = sh.out32[0];
  if (wave == 0) {
    const f32x4 l = tile_quad(a, row, tile);
    const int j = tile * kTile + 4 * lane;
    double w[4], ls = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = kept(l[e], j + e) ? weight(l[e]) : 0.0;
      if (!(w[e] >= mind)) w[e] = 0.0;
      ls += w[e];
    }
    double run = (double)sh.out64[0] * 0x1p-44 + (wave_scan(ls) - ls);
    int at = INT_MAX, last = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      run += w[e];
      if (w[e] > 0.0) {
        if (run > t && at == INT_MAX) at = j + e;
        last = j + e;
      }
    }
    for (int o = 32; o > 0; o >>= 1) {
      at = min(at, __shfl_xor(at, o));
      last = max(last, __shfl_xor(last, o));
    }
    if (lane == 0) {
      a.tokens[r] = at == INT_MAX ? last : at;
      a.head[r] = {1.0 / total, m, tau, tau_idx};
    }
  }
}

__global__ __launch_bounds__(kThreads) void sample_rows_kernel(SampleK a) {
  __shared__ Shared sh;
  sample_row(a, blockIdx.x, sh);
}

// The distribution over a wave's tiles t0 ...
__device__ __forceinline__ void tile_probs(const SampleK& a, int r, int t0) {
  const int lane = threadIdx.x & 63;
  const float* row = a.logits + (size_t)r * a.lstride;
  float* out = a.probs + (size_t)r * a.pstride;
  const RowHead h = a.head[r];
  const RowSet s = row_set(a, r);
  f32x4 l[kWaveTiles];
  bool any[kWaveTiles];
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i) {
    const float m = a.tmax[(size_t)r * a.ntile + min(t0 + i, a.ntile - 1)];
    any[i] = h.inv > 0.0 && m >= h.tau && m > -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i)
    if (t0 + i < a.ntile && any[i]) l[i] = tile_quad(a, row, t0 + i);
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i) {
    if (t0 + i >= a.ntile) break;
    const int j = (t0 + i) * kTile + 4 * lane;
    f32x4 p = f32x4{0.f, 0.f, 0.f, 0.f};
    if (any[i]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool kept = l[i][e] != -INFINITY && (l[i][e] > h.tau || (l[i][e] == h.tau && j + e <= h.tau_idx));
        const double w = kept ? exp2_64(((double)l[i][e] - (double)h.max) * s.scale) : 0.0;
        p[e] = w >= (double)s.Q ? (float)(w * h.inv) : 0.f;
      }
    }
    if (a.pvec && j + 3 < a.V)
      *reinterpret_cast<f32x4*>(out + j) = p;
    else
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < a.V) out[j + e] = p[e];
  }
}
// grid (rows, ceil(ntile / kTilesPerWg))
__global__ __launch_bounds__(256) void sample_probs_kernel(SampleK a) {
  tile_probs(a, blockIdx.x, blockIdx.y * kTilesPerWg + wave_id() * kWaveTiles);
}

// A vocabulary of up to kSmallTiles tiles: the three in one launch, a workgroup a row
// (5 rows of 2048 with the distribution: 17.7 us, in three launches 19.5).
__global__ __launch_bounds__(kThreads) void sample_small_kernel(SampleK a) {
  __shared__ Shared sh;
  const int t0 = wave_id() * kWaveTiles;
  if (t0 < a.ntile) tile_stats(a, blockIdx.x, t0);
  __syncthreads();
  sample_row(a, blockIdx.x, sh);
  if (!a.probs) return;
  __syncthreads();
  if (t0 < a.ntile) tile_probs(a, blockIdx.x, t0);
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

// [error word][row heads][tile sums][tile maxima]
struct SampleLayout {
  size_t head, mass, max, total;
};
SampleLayout sample_layout(int32_t rows, int32_t vocab) {
  auto al = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t tiles = (size_t)rows * ((vocab + kTile - 1) / kTile);
  SampleLayout L{};
  L.head = 256;
  L.mass = L.head + al((size_t)rows * sizeof(RowHead));
  L.max = L.mass + al(tiles * 8);
  L.total = L.max + al(tiles * 4);
  return L;
}
}  // namespace

extern "C" {

size_t nightjar_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  return sample_sizes(rows, vocab) ? sample_layout(rows, vocab).total : 0;
}

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
  const SampleLayout L = sample_layout(rows, vocab);
  char* ws = static_cast<char*>(workspace);
  const int ntile = (vocab + kTile - 1) / kTile;
  SampleK a{logits, logits_stride, vocab, ntile, temperature, top_k, top_p, min_p, uniforms, tokens, probs, probs_stride,
            reinterpret_cast<int*>(ws), reinterpret_cast<double*>(ws + L.mass), reinterpret_cast<float*>(ws + L.max),
            reinterpret_cast<RowHead*>(ws + L.head), lv, pv};
  hipStream_t s = (hipStream_t)stream;
  if (ntile <= kSmallTiles) {
    hipLaunchKernelGGL(sample_small_kernel, dim3(rows), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "sample: %s", hipGetErrorString(e));
  }
  const dim3 grid(rows, (ntile + kTilesPerWg - 1) / kTilesPerWg);
  hipLaunchKernelGGL(sample_tiles_kernel, grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(sample_rows_kernel, dim3(rows), dim3(kThreads), 0, s, a);
    e = hipGetLastError();
  }
  if (e == hipSuccess && probs) {
    hipLaunchKernelGGL(sample_probs_kernel, grid, dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "sample: %s", hipGetErrorString(e));
}

}  // extern "C"
