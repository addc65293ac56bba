// Attention of a chunk of new tokens over a paged cache: row i of a sequence
// sees positions 0 .. c + i, all of them in the pages.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "../../include/nightjar_serve.h"
#include "chunk.h"
#include "kernels.h"

namespace nj {
namespace {

constexpr int kHD = 128;  // head dim of the bf16 path
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct ChunkAttnK {
  ChunkK c;
  const void* q;
  const void* kp;
  const void* vp;
  const uint8_t* ks;
  const uint8_t* vs;
  void* out;
  int H, Hkv, D;
  float scale_log2;
  int G, tokens;      // query heads per KV head, tokens of a tile (kTileRows / G)
  float inv_tokens;   // 1 / tokens
  int pieces[2];      // kPieces per KV head, by class (>= 1)
  int min_cut[2];     // shortest run of keys
  int join_max;       // tiles in more parts are joined by chunk_merge_kernel
  int threshold;      // sequences of more than this many query rows per KV head are cut into tiles, others streamed
  float* part_o[2];   // per class: [slot][rows of the class][kHD], unnormalised
  float* part_ml[2];  // [slot][rows][2]: max (log2 domain), sum
  int* counters[2];   // [slot][kCounterStride]: parts done, at a tile's first slot; zero between calls
};

// ---------------------------------------------------------------------------
// Work.  A sequence's query rows for one KV head are its n tokens times the G
// heads that share it, tokens first.  Class kTiles cuts them into tiles of up to
// 128 rows (whole tokens), class kStream takes sequences of up to 32 rows whole.
// Tiles that see many keys are cut along them, into runs of about L tokens, L the
// same for the whole class: its T tiles see W keys in all, and runs of W / kPieces fill
// the chip (and even out lengths where T is large), but none is shorter than min_cut,
// below which joining the parts costs more than it saves.  That makes at most
// T + kPieces pieces, of which at most 2 kPieces belong to cut tiles.  Every workgroup
// works this out by itself from starts and context lengths (one round of loads per 64
// sequences, sums by DPP) instead of reading a list that another kernel would have to
// write first.  The parts are joined by the last of them to be done (streamed pieces,
// a few KB each) or by a launch of their own (tiles, 64 KB a part, where the batch may
// hold few of them).
// ---------------------------------------------------------------------------
enum { kTiles = 0, kStream = 1 };
constexpr int kTileRows = 128, kStreamRows = 32;
constexpr int kPieces[2] = {512, 512};  // over all KV heads: two workgroups a CU
constexpr int kSlots[2] = {2 * kPieces[0], 2 * kPieces[1]};
// Shortest runs, in tokens: of tiles, of streamed pieces of one row tile, and of two
// (whose parts take longer to join).  One sequence of 1000 tokens, 4 rows: 10.6 us with
// runs of 256, 12.5 of 512, 14.2 whole; 16 of 1024 tokens, 24 rows: 25.5, 26.0 and
// 23.1 us.
constexpr int kMinCutTiles = 256, kMinCutStream[2] = {256, 1024};

struct Piece {
  ChunkSeq s;
  int tile;  // first token tile * tokens
  int split, nsplit;
  int slot;  // of split 0 (nsplit > 1)
  int b;
};

// Sum over the lanes up to this one: within rows of 16 lanes, then across them.
__device__ __forceinline__ int wave_scan_i(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return v;
}
__device__ __forceinline__ int wave_sum_i(int v) { return __builtin_amdgcn_readlane(wave_scan_i(v), 63); }
// ceil(x / L) for 0 <= x < 2^26 and L >= 1 with inv = 1 / L in fp32: the quotient is
// off by one at most, which the products tell.
__device__ __forceinline__ int ceil_div(int x, int L, float inv) {
  const int q = (int)((float)x * inv), d = x - q * L;
  return q + (d > 0 ? 1 : 0) + (d > L ? 1 : 0) - (d <= -L ? 1 : 0);
}

// Tiles of a sequence in class C (0: not of this class).
template <int C>
__device__ __forceinline__ int class_tiles(const ChunkAttnK& a, const ChunkSeq& s) {
  if (s.n == 0 || (s.n * a.G > a.threshold) != (C == kTiles)) return 0;
  return C == kTiles ? ceil_div(s.n, a.tokens, a.inv_tokens) : 1;
}

// Piece `item` of class C (per KV head); with TILES the tile of that number among
// those in more than join_max parts.  False if there is none.  Run by one wave.
template <int C, bool TILES>
__device__ bool find_piece(const ChunkAttnK& a, int item, Piece& out) {
  const int lane = threadIdx.x & 63, B = a.c.B;
  // the class's tiles and the keys that they see (in blocks of 16)
  int tiles = 0, t0 = 0;
  uint64_t keys = 0;
  ChunkSeq s0{0, 0, 0, false};
  for (int b0 = 0; b0 < B; b0 += kWave) {
    const int b = b0 + lane;
    const ChunkSeq s = b < B ? chunk_seq(a.c, b) : ChunkSeq{0, 0, 0, false};
    const int t = class_tiles<C>(a, s);
    if (b0 == 0) {
      s0 = s;
      t0 = t;
    }
    tiles += t;
    keys += (uint64_t)t * ((s.c + s.n + 15) >> 4);
  }
  if (wave_sum_i(tiles) == 0) return false;
  // (at most 2^24 tiles of 2^21 blocks in all: 64 bits)
  const uint64_t all = ((uint64_t)(uint32_t)wave_sum_i((int)(keys >> 16)) << 16) + (uint32_t)wave_sum_i((int)(keys & 0xffff));
  // (rounded up: L > W / pieces is what bounds the pieces)
  const int L = max((int)fminf((float)all * (16.00002f / (float)a.pieces[C]) + 1.f, 0x1p30f), a.min_cut[C]);
  auto seq = [&](int b0, int& t) {
    const int b = b0 + lane;
    const ChunkSeq s = b0 == 0 ? s0 : b < B ? chunk_seq(a.c, b) : ChunkSeq{0, 0, 0, false};
    t = b0 == 0 ? t0 : class_tiles<C>(a, s);
    return s;
  };
  // the piece
  int before = 0, slots = 0;
  const float inv = 1.0f / (float)L;
  for (int b0 = 0; b0 < B; b0 += kWave) {
    int t;
    const ChunkSeq s = seq(b0, t);
    // (tiles: rounded to nearest, as a part of a tile pays off from about 1.5 runs on)
    const int len = s.c + s.n, ns = t ? ceil_div(C == kTiles ? max(len - (L - L / 2 - 1), 1) : len, L, inv) : 0;
    const int sl = ns > 1 ? t * ns : 0, mine = TILES ? (ns > a.join_max ? t : 0) : t * ns;
    const int inc = wave_scan_i(mine), sinc = wave_scan_i(sl);
    const uint64_t hit = __ballot(before + inc > item);
    if (hit) {
      // (the same in every lane: kept in scalar registers)
      const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      const int at = item - (before + of(inc - mine));
      out.b = b0 + l;
      out.s = {of(s.s0), of(s.n), of(s.c), false};
      out.nsplit = of(ns);
      // the last tiles see the most keys: they go first
      const int rank = TILES ? at : at / out.nsplit;
      out.tile = __builtin_amdgcn_readfirstlane(of(t) - 1 - rank);
      out.split = TILES ? 0 : __builtin_amdgcn_readfirstlane(at % out.nsplit);
      out.slot = __builtin_amdgcn_readfirstlane(slots + of(sinc - sl) + rank * out.nsplit);
      return true;
    }
    before += __builtin_amdgcn_readlane(inc, 63);
    slots += __builtin_amdgcn_readlane(sinc, 63);
  }
  return false;
}

// The workgroup's piece: found by its first wave.
template <int C, bool TILES = false>
__device__ __forceinline__ bool wg_piece(const ChunkAttnK& a, int item, Piece& pc) {
  __shared__ int s_pc[9];
  if (threadIdx.x < kWave) {
    Piece p{};
    const bool ok = find_piece<C, TILES>(a, item, p);
    if (threadIdx.x == 0) {
      const int v[9] = {p.s.s0, p.s.n, p.s.c, p.tile, p.split, p.nsplit, p.slot, p.b, ok};
#pragma unroll
      for (int i = 0; i < 9; ++i) s_pc[i] = v[i];
    }
  }
  __syncthreads();
  auto of = [&](int i) { return __builtin_amdgcn_readfirstlane(s_pc[i]); };
  pc = {{of(0), of(1), of(2), false}, of(3), of(4), of(5), of(6), of(7)};
  return of(8) != 0;
}

// Keys of split `split` of a piece that sees `len` keys: whole steps of 64.
__device__ __forceinline__ void split_range(int len, int split, int nsplit, int& k0, int& k1) {
  const int per = ((len + nsplit - 1) / nsplit + 63) & ~63;
  k0 = __builtin_amdgcn_readfirstlane(min(split * per, len));
  k1 = __builtin_amdgcn_readfirstlane(min(k0 + per, len));
}

// ---------------------------------------------------------------------------
// Fragments.  Scores are computed transposed, S^T (32 tokens x 32 rows) = K . Q^T
// with mfma 32x32x16, and fed to O^T (32 dims x 32 rows) += V^T . P^T straight
// from their registers: the tokens are dealt to the first product's rows so that
// the 16 scores that a lane gets of its query row (lane % 32) are the tokens its
// half of the wave supplies to the second product.  V blocks are dim-major, so the
// second product's A operand is a run of tokens of one dim, in one load.
//   MFMA row m = 8 j + 4 h + e  <->  bf16 pages: token 16 (j / 2) + 8 h + 4 (j % 2) + e
//   (a lane's registers 8 s .. 8 s + 7: tokens 8 h .. 8 h + 7 of block s)
// ---------------------------------------------------------------------------
__device__ __forceinline__ int mfma_token(int m) { return 16 * (m >> 4) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3); }

__device__ __forceinline__ bf16x8 ld8(const void* p) { return __builtin_bit_cast(bf16x8, *static_cast<const u32x4*>(p)); }

// Max over the two lanes that share a query row.
__device__ __forceinline__ float half_max(float v) {
  const uint32_t x = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Max of 8, 16 or 32 values, three operands at a time (NaN is dropped, as by fmaxf).
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float max_of(const float (&v)[8]) {
  return max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), fmaxf(v[6], v[7]));
}
__device__ __forceinline__ float max_of(const float (&v)[16]) {
  return max3(max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[8])),
              max3(max3(v[9], v[10], v[11]), max3(v[12], v[13], v[14]), v[15]), v[15]);
}

__device__ __forceinline__ float max_of(const float (&v)[32]) {
  float m[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) m[i] = fmaxf(v[2 * i], v[2 * i + 1]);
  return max_of(m);
}

// One online-softmax step over N scores of a lane's query row (-inf where
// masked): reference = the row's max, so that a leading token's probability is
// exactly 1 in bf16; the accumulators are rescaled only when some row's max rose.
// Scores become probabilities relative to 2^m_run.
template <int N>
__device__ __forceinline__ void softmax_step(float (&st)[N], float scale, float& m_run, float& l_run, f32x16 (&o)[4]) {
  const float bm = half_max(max_of(st)) * scale;
  const bool rises = bm > m_run;
  if (__builtin_amdgcn_ballot_w64(rises)) {
    const float mn = rises ? bm : m_run;
    const float alpha = rises ? __builtin_amdgcn_exp2f(m_run - mn) : 1.f;
    l_run *= alpha;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
    m_run = mn;
  }
  const float ms = m_run == -INFINITY ? 0.f : m_run;  // nothing valid yet: exp2(-inf) = 0 all the same
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    st[i] = __builtin_amdgcn_exp2f(fmaf(st[i], scale, -ms));
    sum[i & 3] += st[i];
  }
  l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

__device__ __forceinline__ bf16x8 pack8(const float* p) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(p[2 * e], p[2 * e + 1]);
  return __builtin_bit_cast(bf16x8, w);
}

// Zeroes the tokens from nv on of a V fragment's eight.
__device__ __forceinline__ bf16x8 keep_tokens(bf16x8 v, int nv) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] &= nv >= 2 * e + 2 ? 0xffffffffu : nv == 2 * e + 1 ? 0xffffu : 0u;
  return __builtin_bit_cast(bf16x8, w);
}
// Nonzero in bits 15 or 31 where a fragment holds a NaN or an infinity: an exponent
// of all ones carries into the sign's place.
constexpr uint32_t kNonfiniteBits = 0x80008000u;
__device__ __forceinline__ uint32_t nonfinite_bits(bf16x8 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  uint32_t any = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) any |= (w[e] & 0x7f807f80u) + 0x00800080u;
  return any;
}

// Element i of an array of page type PT (e4m3: the code's value, without its scale).
template <int PT>
__device__ __forceinline__ float page_at(const void* p, size_t i) {
  if constexpr (PT == kPageF32) return static_cast<const float*>(p)[i];
  if constexpr (PT == kPageBF16) return bf2f(static_cast<const bf16_t*>(p)[i]);
  if constexpr (PT == kPageE4M3) return __builtin_amdgcn_cvt_f32_fp8((int)static_cast<const uint8_t*>(p)[i], 0);
}

// One query row over keys k0 .. k1-1 by a workgroup of 256, 256 keys at a time (any head
// dim up to 512, D % 8 == 0): a thread scores one key, then sums dims t % D and t + 256
// of the 16-key blocks t / D, t / D + 256 / D, ..: a dim's 16 keys of a block lie side
// by side.  Keys outside the range count for nothing, whatever they hold.  m in the log2
// domain; o unnormalised.
constexpr int kMaxD = 512;
struct RowLds {
  float q[kMaxD], p[256], o[256], red[4];
  int id[16];
};
template <int PT, typename T>
__device__ void attend_row(const ChunkAttnK& a, int b, int g, const T* q, int k0, int k1, RowLds& sh, float& m, float& l,
                           float (&o)[2]) {
  const int t = threadIdx.x, D = a.D, groups = max(1, 256 / D);
  __syncthreads();
  for (int d = t; d < D; d += 256) sh.q[d] = to_f(q[d]);
  m = -INFINITY;
  l = o[0] = o[1] = 0.f;
  bool bad = false;
  for (int b0 = k0; b0 < k1; b0 += 256) {  // k0: a block's first token
    __syncthreads();
    if (t < 16) {
      const int blk = b0 / kBlock + t;
      int id = blk * kBlock < k1 ? a.c.table[(size_t)b * a.c.max_blocks + blk] : 0;
      if (id < 0 || id >= a.c.num_blocks) {
        bad = true;
        id = -1;
      }
      sh.id[t] = id;
    }
    __syncthreads();
    const int k = b0 + t, id = sh.id[t / kBlock];
    float sc = -INFINITY;
    if (k < k1 && id >= 0) {
      const size_t slot = ((size_t)id * a.Hkv + g) * kBlock + t % kBlock;
      float dots[8] = {};
#pragma unroll 4
      for (int d = 0; d < D; d += 8)
#pragma unroll
        for (int e = 0; e < 8; ++e) dots[e] = fmaf(sh.q[d + e], page_at<PT>(a.kp, slot * D + d + e), dots[e]);
      float dot = ((dots[0] + dots[1]) + (dots[2] + dots[3])) + ((dots[4] + dots[5]) + (dots[6] + dots[7]));
      if constexpr (PT == kPageE4M3) dot *= __uint_as_float((uint32_t)a.ks[slot] << 23);
      sc = dot * a.scale_log2;
    }
    const float mn = fmaxf(m, block_max<256>(sc, sh.red));
    const float ms = mn == -INFINITY ? 0.f : mn;
    const float p = exp2f(sc - ms), al = m == -INFINITY ? 0.f : exp2f(m - mn);
    m = mn;
    l = l * al + block_sum<256>(p, sh.red);
    sh.p[t] = p;
    __syncthreads();
    const int nblk = (min(k1 - b0, 256) + kBlock - 1) / kBlock;
    for (int e = 0; e < 2; ++e) {
      const int d = D < 256 ? t % D : t + 256 * e;
      if (d >= D || (e && D < 256)) break;
      float acc = o[e] * al;
      for (int jb = D < 256 ? t / D : 0; jb < nblk && t < groups * D; jb += groups) {
        const int jd = sh.id[jb], nj = k1 - (b0 + jb * kBlock);
        if (jd < 0) continue;
        const size_t head = ((size_t)jd * a.Hkv + g) * kBlock;
        float v[kBlock];
#pragma unroll
        for (int j = 0; j < kBlock; ++j) v[j] = page_at<PT>(a.vp, head * D + (size_t)d * kBlock + j);
#pragma unroll
        for (int j = 0; j < kBlock; ++j) {
          if constexpr (PT == kPageE4M3) v[j] *= __uint_as_float((uint32_t)a.vs[head + j] << 23);
          if (j < nj) acc = fmaf(sh.p[jb * kBlock + j], v[j], acc);
        }
      }
      o[e] = acc;
    }
  }
  if (groups > 1) {  // the groups' sums, in order
    sh.o[t] = o[0];
    __syncthreads();
    o[0] = 0.f;
    for (int q = 0; q < groups && t < D; ++q) o[0] += sh.o[q * D + t];
  }
  if (bad) flag_error(a.c.err, kErrBlock);
}

// One workgroup per (row, head).
template <int PT, typename T>
__global__ __launch_bounds__(256) void chunk_attn_row_kernel(ChunkAttnK a) {
  __shared__ RowLds sh;
  if (blockIdx.x == 0 && blockIdx.y == 0) chunk_check(a.c);
  const int row = blockIdx.x, h = blockIdx.y, t = threadIdx.x, D = a.D;
  const int b = chunk_find(a.c.B, row, [&](int i) { return a.c.starts[i]; });
  if (b < 0) return;
  const ChunkSeq s = chunk_seq(a.c, b);
  const int i = row - s.s0;
  if (i < 0 || i >= s.n) return;  // (before it: where starts decrease)
  float m, l, o[2];
  const size_t at = ((size_t)row * a.H + h) * D;
  attend_row<PT, T>(a, b, h / (a.H / a.Hkv), static_cast<const T*>(a.q) + at, 0, s.c + i + 1, sh, m, l, o);
  for (int e = 0; e < 2; ++e) {
    const int d = t + 256 * e;
    if (d < D) static_cast<T*>(a.out)[at + d] = from_f<T>(o[e] / l);
  }
}

// Parts of a tile whose keys were cut: written and read past the caches of the XCDs
// (device-coherent accesses, as between the parts of a split GEMM tile), counted in
// at the tile's first slot, and joined by the last to arrive:
//   out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s.
template <int C>
struct Parts {
  static constexpr int ROWS = C == kTiles ? kTileRows : kStreamRows;
  __amdgpu_buffer_rsrc_t o, ml;
  __device__ __forceinline__ Parts(const ChunkAttnK& a)
      : o(coherent_rsrc(a.part_o[C], kSlots[C] * ROWS * kHD * 4)), ml(coherent_rsrc(a.part_ml[C], kSlots[C] * ROWS * 8)) {}
  __device__ __forceinline__ uint32_t row(const ChunkAttnK& a, const Piece& pc, int split, int kvh, int r) const {
    return (uint32_t)(((pc.slot + split) * a.Hkv + kvh) * ROWS + r);
  }
  __device__ __forceinline__ void put(uint32_t row, int d, f32x4 v) const { coherent_store(o, (row * kHD + d) * 4, v); }
  __device__ __forceinline__ void put_ml(uint32_t row, float m, float l) const {
    coherent_store_f32(ml, row * 8, m);
    coherent_store_f32(ml, row * 8 + 4, l);
  }
};

// A thread joins units of 4 dims of a row.  Tiles have many units and few parts:
// four units at once, four parts of each in flight.  Streamed pieces have few units
// and up to a hundred parts: one unit, 16 parts in flight, and where the rows leave
// threads over, these take parts of their own (part p to group p % groups) and meet
// in LDS (8 KB).
template <int C>
__device__ void join_parts(const ChunkAttnK& a, const Piece& pc, int kvh, int tokens, const Parts<C>& parts, char* lds) {
  constexpr int NU = C == kTiles ? 4 : 1, NJ = C == kTiles ? 4 : 16;
  __shared__ int s_last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's part is written
  __syncthreads();
  int* cnt = a.counters[C] + (size_t)(pc.slot * a.Hkv + kvh) * kCounterStride;
  if (threadIdx.x == 0)
    s_last = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pc.nsplit - 1;
  __syncthreads();
  if (!s_last) return;
  if (threadIdx.x == 0) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int i0 = pc.tile * tokens, R = min(tokens, pc.s.n - i0) * a.G, units = R * (kHD / 4);
  const int groups = C == kTiles ? 1 : max(1, 256 / units);
  const int grp = groups > 1 ? (int)threadIdx.x / units : 0, t0 = groups > 1 ? (int)threadIdx.x % units : (int)threadIdx.x;
  auto write = [&](int u, f32x4 acc, float sum) {
    const int r = u / (kHD / 4), d = (u % (kHD / 4)) * 4;
    const float inv = 1.0f / sum;
    bf16_t* dst = static_cast<bf16_t*>(a.out) + ((size_t)(pc.s.s0 + i0 + r / a.G) * a.H + kvh * a.G + r % a.G) * kHD + d;
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
  };
  for (int u0 = 0; u0 < units; u0 += 256 * NU) {
    f32x4 acc[NU];
    float mx[NU], sum[NU];
#pragma unroll
    for (int q = 0; q < NU; ++q) {
      acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
      mx[q] = -INFINITY;
      sum[q] = 0.f;
    }
    for (int s0 = grp; s0 < pc.nsplit; s0 += groups * NJ) {
      f32x4 ov[NU][NJ];
      float2 ml[NU][NJ];
#pragma unroll
      for (int q = 0; q < NU; ++q) {
        if (u0 + q * 256 >= units) break;  // uniform
        const int u = min(u0 + q * 256 + t0, units - 1);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint32_t row = parts.row(a, pc, min(s0 + j * groups, pc.nsplit - 1), kvh, u / (kHD / 4));
          ml[q][j] = coherent_load_f32x2(parts.ml, row * 8);
          ov[q][j] = coherent_load(parts.o, (row * kHD + (u % (kHD / 4)) * 4) * 4);
        }
      }
#pragma unroll
      for (int q = 0; q < NU; ++q) {
        if (u0 + q * 256 >= units) break;
        float mn = mx[q];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          if (s0 + j * groups < pc.nsplit) mn = fmaxf(mn, ml[q][j].x);
        // (a part without keys, or with nothing but NaN scores, has m = -inf: weight 0, and its NaN stays)
        const float f = mx[q] == -INFINITY ? 0.f : exp2f(mx[q] - mn);
        acc[q] *= f;
        sum[q] *= f;
        mx[q] = mn;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          if (s0 + j * groups < pc.nsplit) {
            const float w = ml[q][j].x == -INFINITY ? 0.f : exp2f(ml[q][j].x - mn);
            sum[q] += w * ml[q][j].y;
            acc[q] += w * ov[q][j];
          }
      }
    }
    if (groups == 1) {
#pragma unroll
      for (int q = 0; q < NU; ++q)
        if (u0 + q * 256 + t0 < units) write(u0 + q * 256 + t0, acc[q], sum[q]);
    } else {
      f32x4* s_acc = reinterpret_cast<f32x4*>(lds);
      float2* s_ml = reinterpret_cast<float2*>(lds + 256 * 16);
      s_acc[threadIdx.x] = acc[0];
      s_ml[threadIdx.x] = float2{mx[0], sum[0]};
      __syncthreads();
      if (grp == 0) {
        float mn = mx[0];
        for (int g = 1; g < groups; ++g) mn = fmaxf(mn, s_ml[g * units + t0].x);
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
        for (int g = 0; g < groups; ++g) {
          const float2 ml = s_ml[g * units + t0];
          const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mn);
          l += w * ml.y;
          o += w * s_acc[g * units + t0];
        }
        write(t0, o, l);
      }
    }
  }
}

// A piece whose masked tokens hold NaN or infinities in V (a later token of the
// chunk, seen by some of its rows): in the matrix products 0 times those would
// reach the rows that do not see them.  The piece's rows again, one at a time, each
// over the keys that it sees.
template <int PT, int C>
__device__ void redo_piece(const ChunkAttnK& a, const Piece& pc, int kvh, int G, int tokens, int k0, int k1, char* lds,
                           const Parts<C>& parts) {
  RowLds& sh = *reinterpret_cast<RowLds*>(lds);
  const int i0 = pc.tile * tokens, R = min(tokens, pc.s.n - i0) * G;
  for (int r = 0; r < R; ++r) {
    const int i = i0 + r / G, row = pc.s.s0 + i;
    float m, l, o[2];
    const size_t at = ((size_t)row * a.H + kvh * G + r % G) * kHD;
    attend_row<PT, bf16_t>(a, pc.b, kvh, static_cast<const bf16_t*>(a.q) + at, k0, min(k1, pc.s.c + i + 1), sh, m, l, o);
    if (threadIdx.x >= kHD) continue;
    if (pc.nsplit == 1) {
      static_cast<bf16_t*>(a.out)[at + threadIdx.x] = f2bf(o[0] / l);
    } else {
      const uint32_t prow = parts.row(a, pc, pc.split, kvh, r);
      coherent_store_f32(parts.o, (prow * kHD + threadIdx.x) * 4, o[0]);
      if (threadIdx.x == 0) parts.put_ml(prow, m, l);
    }
  }
}

// A lane's row of a piece: 4 consecutive dims per register quad.
__device__ __forceinline__ void store_row(const ChunkAttnK& a, int row, int head, const f32x16 (&o)[4], float inv) {
  bf16_t* dst = static_cast<bf16_t*>(a.out) + ((size_t)row * a.H + head) * kHD + 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * j) =
          u32x2{pack_bf16x2(o[dt][4 * j] * inv, o[dt][4 * j + 1] * inv),
                pack_bf16x2(o[dt][4 * j + 2] * inv, o[dt][4 * j + 3] * inv)};
}

// ---------------------------------------------------------------------------
// Tiles: 128 query rows per workgroup, 32 per wave; keys and values pass through
// LDS 64 tokens (four blocks) at a time, two buffers.  LDS holds bf16 whatever the
// pages hold: bf16 pages are copied by the load itself (global_load_lds_dwordx4),
// e4m3 ones are converted once per workgroup on the way (exact: a code times a
// power of two).
//
// Bound by the matrix cores and the softmax's vector work about alike: 64 tokens
// take a wave 32 MFMAs of 32 clocks and ~200 vector instructions.  A prompt of 4096 (8B
// layout, bf16): 165 us, 0.83 PFLOP/s; 512 tokens after 8000: bf16 97, 0.71, e4m3 104.
//
// Swizzle, in 16-byte units: K token t of a block keeps unit u at u ^ t; V dim d
// keeps its two halves swapped when bit 4 of d is set.  The 16 lanes that a
// fragment read serves together (0-3, 12-15, 20-27; 4-11, 16-19, 28-31; the same
// from 32 on) then hit 16 different units of the 256 bytes of banks.
// ---------------------------------------------------------------------------
constexpr int kStep = 64;                        // tokens per stage
constexpr int kStageBytes = kStep * kHD * 2 * 2; // K of four blocks, then V of them
constexpr int kBlkBytes = kBlock * kHD * 2;
template <int PT>
__global__ __launch_bounds__(256, 2) void chunk_tile_kernel(ChunkAttnK a) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStageBytes];
  const int kvh = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
  if (blockIdx.x == 0) chunk_check(a.c);
  Piece pc;
  if (!wg_piece<kTiles>(a, blockIdx.x / a.Hkv, pc)) return;
  const int G = a.G, tokens = a.tokens;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int i0 = pc.tile * tokens, len = pc.s.c + min(i0 + tokens, pc.s.n);
  int k0, k1;
  split_range(len, pc.split, pc.nsplit, k0, k1);

  // this lane's query row, its last visible key, and the wave's last
  const int r = wave * 32 + r32, i = i0 + r / G, head = kvh * G + r % G;
  const bool row_ok = r < tokens * G && i < pc.s.n;
  const int ic = min(i, pc.s.n - 1), vis = pc.s.c + ic;
  const int row = pc.s.s0 + ic;
  const int vis_hi = pc.s.c + __builtin_amdgcn_readfirstlane(min(i0 + (wave * 32 + 31) / G, pc.s.n - 1));
  const bool wave_on = wave * 32 < tokens * G && i0 + wave * 32 / G < pc.s.n;
  bf16x8 qf[8];
  {
    const bf16_t* src = static_cast<const bf16_t*>(a.q) + ((size_t)row * a.H + min(head, a.H - 1)) * kHD + 8 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = ld8(src + 16 * s);
  }
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;

  uint32_t odd = 0;  // kNonfiniteBits: see redo_piece
  const int nit = (k1 - k0 + kStep - 1) / kStep;
  // page ids of this wave's block of 64 stages (lane l: stage idbase + l); bad
  // ones and blocks behind the last key read page 0, whose tokens are masked (or,
  // for a bad id, make the output undefined)
  int idv = 0, idbase = 0;
  bool bad = false;
  auto read_ids = [&](int it0) {
    idbase = it0;
    const int blk = (k0 + (it0 + lane) * kStep) / kBlock + wave;
    int id = 0;
    if (blk * kBlock < k1) {
      id = a.c.table[(size_t)pc.b * a.c.max_blocks + blk];
      if (id < 0 || id >= a.c.num_blocks) {
        bad = true;
        id = 0;
      }
    }
    idv = id;
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // bf16: source offsets of the four 1 KB pieces of a K block (its rows 4 q ..) and of a V block
  uint32_t kofs[4], vofs[4];
  if constexpr (PT == kPageBF16) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int p = q * 64 + lane, t = p >> 4, d = p >> 1;
      kofs[q] = (uint32_t)(t * kHD * 2 + (((p & 15) ^ t) * 16));
      vofs[q] = (uint32_t)(d * kBlock * 2 + (((p & 1) ^ ((d >> 4) & 1)) * 16));
    }
  }
  // e4m3: a block's K and V codes, two 16-byte pieces a lane, and their scales
  u32x4 kc[2], vc[2], vsc;
  uint32_t ksc[2];
  auto load = [&](int it) {
    if (it - idbase >= 64) read_ids(it);
    const int id = __builtin_amdgcn_readlane(idv, it - idbase);
    const size_t hd = (size_t)id * a.Hkv + kvh;
    if constexpr (PT == kPageBF16) {
      const char* ksrc = static_cast<const char*>(a.kp) + hd * kBlkBytes;
      const char* vsrc = static_cast<const char*>(a.vp) + hd * kBlkBytes;
      const uint32_t dst = lds0 + (it & 1) * kStageBytes + wave * kBlkBytes;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(kofs[q]), "s"(ksrc), "s"(dst + q * 1024) : "memory", "m0");
#pragma unroll
      for (int q = 0; q < 4; ++q)
        asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(vofs[q]), "s"(vsrc), "s"(dst + kStageBytes / 2 + q * 1024) : "memory", "m0");
    } else {
      const char* ksrc = static_cast<const char*>(a.kp) + hd * (kBlkBytes / 2);
      const char* vsrc = static_cast<const char*>(a.vp) + hd * (kBlkBytes / 2);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        kc[q] = *reinterpret_cast<const u32x4*>(ksrc + (q * 64 + lane) * 16);
        vc[q] = *reinterpret_cast<const u32x4*>(vsrc + (q * 64 + lane) * 16);
        ksc[q] = a.ks[hd * kBlock + q * 8 + (lane >> 3)];
      }
      vsc = *reinterpret_cast<const u32x4*>(a.vs + hd * kBlock);
    }
  };
  auto convert = [&](int it) {
    if constexpr (PT == kPageE4M3) {
      char* kd = smem + (it & 1) * kStageBytes + wave * kBlkBytes;
      char* vd = kd + kStageBytes / 2;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int p = q * 64 + lane, t = p >> 3, u = 2 * (p & 7);
        u32x4 w[2];
        const float sc = __uint_as_float(ksc[q] << 23);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)kc[q][c], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)kc[q][c], true);
          w[c >> 1][2 * (c & 1)] = pack_bf16x2(lo[0] * sc, lo[1] * sc);
          w[c >> 1][2 * (c & 1) + 1] = pack_bf16x2(hi[0] * sc, hi[1] * sc);
        }
        *reinterpret_cast<u32x4*>(kd + t * 256 + ((u ^ t) * 16)) = w[0];
        *reinterpret_cast<u32x4*>(kd + t * 256 + (((u + 1) ^ t) * 16)) = w[1];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[q][c], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[q][c], true);
          auto vscale = [&](int e) { return __uint_as_float(((vsc[c] >> (8 * e)) & 0xffu) << 23); };
          w[c >> 1][2 * (c & 1)] = pack_bf16x2(lo[0] * vscale(0), lo[1] * vscale(1));
          w[c >> 1][2 * (c & 1) + 1] = pack_bf16x2(hi[0] * vscale(2), hi[1] * vscale(3));
        }
        const int swap = (p >> 4) & 1;
        *reinterpret_cast<u32x4*>(vd + p * 32 + (0 ^ swap) * 16) = w[0];
        *reinterpret_cast<u32x4*>(vd + p * 32 + (1 ^ swap) * 16) = w[1];
      }
    }
  };
  // fragment addresses: K row of MFMA row r32, V dim r32
  const int mt = mfma_token(r32);
  const int kaddr = (mt >> 4) * kBlkBytes + (mt & 15) * 256 + ((h ^ (mt & 15)) * 16);
  const int vaddr = kStageBytes / 2 + r32 * 32 + ((h ^ (r32 >> 4)) * 16);

  // One stage's products: both score products, one softmax step over the 64 tokens
  // (one rescale test), and behind it the second products, among which the compiler
  // spreads the exponentials.  V's first fragments are read under the softmax.
  auto stage = [&](auto maskedc, int it) {
    constexpr bool masked = decltype(maskedc)::value;
    const char* buf = smem + (it & 1) * kStageBytes;
    const int t0 = k0 + it * kStep;
    f32x16 acc[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][e] = 0.f;
#pragma unroll
      for (int s = 0; s < 8; ++s)
        acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ld8(buf + ((kaddr ^ (32 * s)) + x * 2 * kBlkBytes)), qf[s], acc[x], 0, 0, 0);
    }
    bf16x8 vf[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) vf[dt] = ld8(buf + vaddr + dt * 1024);
    float st[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) st[e] = acc[e >> 4][e & 15];
    if constexpr (masked) {
      const int lim = min(vis, k1 - 1) - t0;
#pragma unroll
      for (int e = 0; e < 32; ++e) st[e] = 16 * (e >> 3) + 8 * h + (e & 7) <= lim ? st[e] : -INFINITY;
    }
    softmax_step(st, a.scale_log2, m_run, l_run, o);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const bf16x8 pf = pack8(st + 8 * x);
      bf16x8 vn[4];
      if (x < 3) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) vn[dt] = ld8(buf + vaddr + (x + 1) * kBlkBytes + dt * 1024);
      }
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        if constexpr (masked) {  // a masked token's V must not be NaN or infinite: 0 times it would not be 0
          vf[dt] = keep_tokens(vf[dt], k1 - t0 - 16 * x - 8 * h);
          odd |= nonfinite_bits(vf[dt]);
        }
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt], pf, o[dt], 0, 0, 0);
      }
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) vf[dt] = vn[dt];
    }
  };
  auto next = [&](int it) {
    // this stage is in LDS, and every wave is done with the buffer that the next one goes to
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (it + 1 < nit) load(it + 1);
  };
  if (nit > 0) {
    read_ids(0);
    load(0);
    convert(0);
  }
  // no load of the compiler's own is left for the loop to wait for: it would wait for the stage loads with it
  __builtin_amdgcn_s_waitcnt(0x0f70);
  // Stages that every row of the tile sees whole come first, in a loop without masks (as selects they took a third
  // of the vector work).
  const int vis0 = pc.s.c + i0;  // the first row's last key
  const int full = min(max((min(vis0 + 1, k1) - k0) / kStep, 0), nit);
  for (int it = 0; it < full; ++it) {
    next(it);
    if (wave_on) stage(std::false_type{}, it);
    if (it + 1 < nit) convert(it + 1);
  }
  for (int it = full; it < nit; ++it) {
    next(it);
    if (wave_on && k0 + it * kStep <= vis_hi) stage(std::true_type{}, it);
    if (it + 1 < nit) convert(it + 1);
  }
  if (__builtin_amdgcn_ballot_w64(bad) && lane == 0) flag_error(a.c.err, kErrBlock);
  const Parts<kTiles> parts(a);
  const float l = l_run + __shfl_xor(l_run, 32);
  if (__syncthreads_or((odd & kNonfiniteBits) != 0)) {
    redo_piece<PT, kTiles>(a, pc, kvh, G, tokens, k0, k1, smem, parts);
  } else if (pc.nsplit == 1) {
    if (row_ok) store_row(a, row, head, o, 1.0f / l);
  } else if (row_ok) {
    const uint32_t prow = parts.row(a, pc, pc.split, kvh, r);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        parts.put(prow, 32 * dt + 8 * j + 4 * h, f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]});
    if (h == 0) parts.put_ml(prow, m_run, l);
  }
  if (pc.nsplit > 1 && pc.nsplit <= a.join_max) join_parts<kTiles>(a, pc, kvh, tokens, parts, smem);
}

// ---------------------------------------------------------------------------
// Streamed: up to 16 RT query rows (decoding steps and short chunks), RT = 1 or 2
// row tiles.  Each wave takes steps of its own (step w, w + 4, .. of the piece)
// straight from memory into MFMA fragments, and the four waves' results are joined
// in LDS.  Bound by the read of the cache; what is in flight (16 KB a wave) sets
// the rate: single tokens of 200 sequences (7B layout, e4m3) 94 us, 4.5 TB/s, of 64
// (8B) bf16 55, 4.2, e4m3 32, 3.7, of one with 8000 tokens 12.
//
// A step is 32 tokens in bf16 and 64 in e4m3: every load is then 16 bytes a lane,
// 16 KB a step.  W = 8 or 16 tokens per lane group g = lane / 16: row m of score
// tile j (mfma 16x16x32) is token W (m / 4) + 4 j + m % 4, so that group g ends up
// with the scores of tokens W g .. in order, the very run of a dim of a V block that
// the group's loads bring for the second product.  e4m3: 16 codes of K are two
// k-steps of the first product (q's fragments are dealt the same way) and take the
// token's scale as they are converted; V's scales multiply the probabilities.
// ---------------------------------------------------------------------------
// Eight e4m3 codes as bf16, times a power of two (exact).
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t c0, uint32_t c1, float sc) {
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c0, sc, false));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c0, sc, true));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c1, sc, false));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c1, sc, true));
  return __builtin_bit_cast(bf16x8, w);
}

// Max over the four lanes that share a query row (lane % 16).
__device__ __forceinline__ float quarter_max(float v) {
  const uint32_t x = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

constexpr int kMergeRow = kHD + 4;  // LDS row stride of the wave merge, in floats
template <int PT, int RT>
__global__ __launch_bounds__(256, RT == 1 ? 3 : 2) void chunk_stream_kernel(ChunkAttnK a) {
  constexpr bool E4 = PT == kPageE4M3;
  constexpr int NP = 4, ROWS = 16 * RT;
  constexpr int W = E4 ? 16 : 8, ST = 4 * W, NT = W / 4;  // tokens of a lane group and of a step, score tiles
  __shared__ __attribute__((aligned(16))) float s_o[NP][ROWS * kMergeRow];
  __shared__ float s_m[NP][ROWS], s_l[NP][ROWS];
  const int kvh = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
  if (blockIdx.x == 0) chunk_check(a.c);
  Piece pc;
  if (!wg_piece<kStream>(a, blockIdx.x / a.Hkv, pc)) return;
  const int G = a.G, R = pc.s.n * G, len = pc.s.c + pc.s.n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  int k0, k1;
  split_range(len, pc.split, pc.nsplit, k0, k1);
  const int np = (k1 - k0 + ST - 1) / ST;                   // steps of the piece
  const int n = np > wave ? (np - wave + NP - 1) / NP : 0;  // this wave's

  bf16x8 qf[RT][4];
  int vis[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int qr = min(16 * t + r16, R - 1), qi = qr / G;  // padding rows repeat the last one
    const bf16_t* src = static_cast<const bf16_t*>(a.q) + ((size_t)(pc.s.s0 + qi) * a.H + kvh * G + qr % G) * kHD;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[t][s] = ld8(src + (E4 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g));
    vis[t] = pc.s.c + qi;
  }
  // page ids of 64 / NT of the wave's steps: lane l holds block l % NT of step
  // idbase + l / NT; -1 behind the last key (its tokens are masked) and for a bad
  // id (the output is then undefined): both read page 0
  constexpr int kIds = kWave / NT;
  int idv = -1, idbase = 0;
  bool bad = false;
  auto read_ids = [&](int j0) {
    idbase = j0;
    const int blk = k0 / kBlock + NT * (wave + NP * (j0 + lane / NT)) + lane % NT;
    int id = -1;
    if (blk * kBlock < k1) {
      id = a.c.table[(size_t)pc.b * a.c.max_blocks + blk];
      if (id < 0 || id >= a.c.num_blocks) {
        bad = true;
        id = -1;
      }
    }
    idv = id;
  };
  read_ids(0);
  uint32_t odd = 0;  // kNonfiniteBits: see redo_piece
  // One step's fragments.  The next step's loads go out as soon as these are used,
  // K under the softmax and the second product, V behind it (the order is pinned:
  // hoisted loads would need registers of their own).  The wave's last step is
  // code of its own: loads that may or may not have been issued would make the
  // compiler wait for every load in flight, and loads past
  // the end would all be of one page.
  u32x4 kr[8], vr[8], vsc;
  uint32_t ksc[NT];
  size_t vhd = 0;  // (page, head) of the V to load
  const int ktok = W * (r16 >> 2) + (r16 & 3);  // token of score tile 0 (tile j: + 4 j, in the same block)
  auto load_k = [&](int j) {
    if (j - idbase >= kIds) read_ids(j);
    // this lane's blocks of the step: of its token for K, of its run for V
    const size_t hd = (size_t)max(__shfl(idv, NT * (j - idbase) + (ktok >> 4)), 0) * a.Hkv + kvh;
    vhd = (size_t)max(__shfl(idv, NT * (j - idbase) + (W * g >> 4)), 0) * a.Hkv + kvh;
    if constexpr (E4) {
      const char* src = static_cast<const char*>(a.kp) + (hd * kBlock + (ktok & 15)) * kHD + 16 * g;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int s = 0; s < 2; ++s) kr[2 * t + s] = *reinterpret_cast<const u32x4*>(src + 4 * t * kHD + 64 * s);
        ksc[t] = a.ks[hd * kBlock + (ktok & 15) + 4 * t];
      }
    } else {
      const char* src = static_cast<const char*>(a.kp) + ((hd * kBlock + (ktok & 15)) * kHD + 8 * g) * 2;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int s = 0; s < 4; ++s) kr[4 * t + s] = *reinterpret_cast<const u32x4*>(src + 4 * t * kHD * 2 + 64 * s);
    }
  };
  auto load_v = [&]() {
    const size_t hd = vhd;
    const char* src = static_cast<const char*>(a.vp) +
                      (E4 ? (hd * kHD + r16) * kBlock : ((hd * kHD + r16) * kBlock + 8 * (g & 1)) * 2);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) vr[dt] = *reinterpret_cast<const u32x4*>(src + dt * 16 * kBlock * (E4 ? 1 : 2));
    if constexpr (E4) vsc = *reinterpret_cast<const u32x4*>(a.vs + hd * kBlock);
  };
  float m_run[RT], l_run[RT];
  f32x4 o[RT][8];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[t][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto step = [&](auto lastc, int j) {
    constexpr bool last = decltype(lastc)::value;
    f32x4 acc[RT][NT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float sc = E4 ? __uint_as_float(ksc[i] << 23) : 1.f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        bf16x8 kf;
        if constexpr (E4) {
          const u32x4 c = kr[2 * i + (s >> 1)];
          kf = codes_to_bf16(c[2 * (s & 1)], c[2 * (s & 1) + 1], sc);
        } else {
          kf = __builtin_bit_cast(bf16x8, kr[4 * i + s]);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][s], acc[t][i], 0, 0, 0);
      }
      if constexpr (E4) __builtin_amdgcn_sched_barrier(0);  // conversions hoisted further would need registers of their own
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!last) load_k(j + 1);
    __builtin_amdgcn_sched_barrier(0);
    const int t0 = k0 + ST * (wave + NP * j);
    // (a wave's steps are NP * ST >= 128 tokens apart and the rows see up to 32 tokens more or less: only its last
    // step has anything to mask)
    const bool masked = last && (t0 + ST - 1 > pc.s.c || t0 + ST > k1);
    float st[RT][W];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int e = 0; e < W; ++e) st[t][e] = acc[t][e >> 2][e & 3];
      if (masked) {
        const int lim = min(vis[t], k1 - 1) - t0 - W * g;
#pragma unroll
        for (int e = 0; e < W; ++e) st[t][e] = e <= lim ? st[t][e] : -INFINITY;
      }
      // online softmax, reference = the row's max (see softmax_step)
      const float bm = quarter_max(max_of(st[t])) * a.scale_log2;
      const bool rises = bm > m_run[t];
      if (__builtin_amdgcn_ballot_w64(rises)) {
        const float mn = rises ? bm : m_run[t];
        const float alpha = rises ? __builtin_amdgcn_exp2f(m_run[t] - mn) : 1.f;
        l_run[t] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[t][dt] *= alpha;
        m_run[t] = mn;
      }
      const float ms = m_run[t] == -INFINITY ? 0.f : m_run[t];
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < W; ++e) {
        st[t][e] = __builtin_amdgcn_exp2f(fmaf(st[t][e], a.scale_log2, -ms));
        sum[e & 3] += st[t][e];
      }
      l_run[t] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    if (masked) {  // a masked token's V must not be NaN or infinite: 0 times it would not be 0
      const int nv = k1 - t0 - W * g;  // tokens of the lane's run before the end: the others may be anything, and are zeroed
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        if constexpr (E4) {
          uint32_t any = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int k = min(max(nv - 4 * c, 0), 4);
            if (dt == 0) vsc[c] &= k == 4 ? 0xffffffffu : (1u << (8 * k)) - 1u;  // (any scale byte, 255 = infinity too)
            vr[dt][c] &= k == 4 ? 0xffffffffu : (1u << (8 * k)) - 1u;
            any |= (vr[dt][c] & 0x7f7f7f7fu) + 0x01010101u;  // a NaN code (magnitude 0x7f) carries into its top bit
          }
          odd |= any & 0x80808080u ? kNonfiniteBits : 0;
        } else {
          const bf16x8 v = keep_tokens(__builtin_bit_cast(bf16x8, vr[dt]), nv);
          vr[dt] = __builtin_bit_cast(u32x4, v);
          odd |= nonfinite_bits(v);
        }
      }
    }
    {
#pragma unroll
      for (int t = 0; t < RT; ++t)
        if constexpr (E4) {
#pragma unroll
          for (int e = 0; e < W; ++e) {
            st[t][e] *= __uint_as_float(((vsc[e >> 2] >> (8 * (e & 3))) & 0xffu) << 23);
          }
        }
#pragma unroll
      for (int x = 0; x < W / 8; ++x) {
        bf16x8 pf[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) pf[t] = pack8(&st[t][8 * x]);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          bf16x8 vf;  // k-step x (tokens W g + 8 x ..) of dims 16 dt ..
          if constexpr (E4)
            vf = codes_to_bf16(vr[dt][2 * x], vr[dt][2 * x + 1], 1.f);
          else
            vf = __builtin_bit_cast(bf16x8, vr[dt]);
#pragma unroll
          for (int t = 0; t < RT; ++t) o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t], o[t][dt], 0, 0, 0);
          if constexpr (E4)
            if (dt % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!last) load_v();
    __builtin_amdgcn_sched_barrier(0);
  };
  if (n > 0) {
    load_k(0);
    load_v();
    for (int j = 0; j < n - 1; ++j) step(std::false_type{}, j);
    step(std::true_type{}, n - 1);
  }
  if (__builtin_amdgcn_ballot_w64(bad) && lane == 0) flag_error(a.c.err, kErrBlock);

  const Parts<kStream> parts(a);
  if (__syncthreads_or((odd & kNonfiniteBits) != 0)) {
    redo_piece<PT, kStream>(a, pc, kvh, G, pc.s.n, k0, k1, reinterpret_cast<char*>(s_o), parts);
    if (pc.nsplit > 1) join_parts<kStream>(a, pc, kvh, pc.s.n, parts, reinterpret_cast<char*>(s_o));
    return;
  }
  // join the waves, then store the rows or this split's part
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float l = l_run[t];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      s_m[wave][16 * t + r16] = m_run[t];
      s_l[wave][16 * t + r16] = l;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *reinterpret_cast<f32x4*>(&s_o[wave][(16 * t + r16) * kMergeRow + 16 * dt + 4 * g]) = o[t][dt];
  }
  __syncthreads();
  for (int u = threadIdx.x; u < R * (kHD / 4); u += 256) {
    const int rr = u / (kHD / 4), d = (u % (kHD / 4)) * 4;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < NP; ++w) mx = fmaxf(mx, s_m[w][rr]);
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NP; ++w) {
      const float m = s_m[w][rr], f = m == -INFINITY ? 0.f : exp2f(m - mx);
      sum += f * s_l[w][rr];
      acc += f * *reinterpret_cast<const f32x4*>(&s_o[w][rr * kMergeRow + d]);
    }
    if (pc.nsplit == 1) {
      const float inv = 1.0f / sum;
      bf16_t* dst = static_cast<bf16_t*>(a.out) + ((size_t)(pc.s.s0 + rr / G) * a.H + kvh * G + rr % G) * kHD + d;
      *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    } else {
      const uint32_t prow = parts.row(a, pc, pc.split, kvh, rr);
      parts.put(prow, d, acc);
      if (d == 0) parts.put_ml(prow, mx, sum);
    }
  }
  if (pc.nsplit > 1) join_parts<kStream>(a, pc, kvh, pc.s.n, parts, reinterpret_cast<char*>(s_o));
}

// Joins the parts of tiles: 64 KB each, which one workgroup (the last part's) would
// read at what a single CU draws, ~45 GB/s (40 tokens over 8000 in 32 parts: 79 us,
// with this launch 32; 20 tokens over 2000: 27, 19).  grid (tiles * Hkv, groups of 8
// rows).
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkAttnK a) {
  const int kvh = __builtin_amdgcn_readfirstlane(blockIdx.x % a.Hkv);
  Piece pc;
  if (!wg_piece<kTiles, true>(a, blockIdx.x / a.Hkv, pc)) return;
  const int r = blockIdx.y * 8 + threadIdx.x / (kHD / 4), d = (threadIdx.x % (kHD / 4)) * 4;
  const int i0 = pc.tile * a.tokens, R = min(a.tokens, pc.s.n - i0) * a.G;
  if (r >= R) return;
  const float* ml = a.part_ml[kTiles] + (((size_t)pc.slot * a.Hkv + kvh) * kTileRows + r) * 2;
  const float* po = a.part_o[kTiles] + (((size_t)pc.slot * a.Hkv + kvh) * kTileRows + r) * kHD + d;
  const size_t step = (size_t)a.Hkv * kTileRows;
  constexpr int NJ = 8;  // parts in flight
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  float mx = -INFINITY, sum = 0.f;
  for (int s0 = 0; s0 < pc.nsplit; s0 += NJ) {
    f32x4 ov[NJ];
    float2 v[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const size_t at = min(s0 + j, pc.nsplit - 1) * step;
      v[j] = *reinterpret_cast<const float2*>(ml + at * 2);
      ov[j] = *reinterpret_cast<const f32x4*>(po + at * kHD);
    }
    float mn = mx;
#pragma unroll
    for (int j = 0; j < NJ; ++j) mn = fmaxf(mn, v[j].x);
    const float f = mx == -INFINITY ? 0.f : exp2f(mx - mn);
    acc *= f;
    sum *= f;
    mx = mn;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (s0 + j < pc.nsplit) {
        const float w = v[j].x == -INFINITY ? 0.f : exp2f(v[j].x - mn);
        sum += w * v[j].y;
        acc += w * ov[j];
      }
  }
  const float inv = 1.0f / sum;
  bf16_t* dst = static_cast<bf16_t*>(a.out) + ((size_t)(pc.s.s0 + i0 + r / a.G) * a.H + kvh * a.G + r % a.G) * kHD + d;
  *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
}

}  // namespace
}  // namespace nj

using namespace nj;

namespace {

bool chunk_sizes(const nj_model_desc* d, const char* what) {
  if (!d) return !set_last_error(NJ_EINVAL, "%s: desc is NULL", what);
  if (d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads % d->n_kv_heads)
    return !set_last_error(NJ_EINVAL, "%s: n_heads must be a positive multiple of n_kv_heads", what);
  if (d->block_size != kBlock) return !set_last_error(NJ_EINVAL, "%s: block_size must be 16", what);
  if (d->dtype != NJ_F32 && d->dtype != NJ_BF16) return !set_last_error(NJ_EINVAL, "%s: dtype must be NJ_F32 or NJ_BF16", what);
  if (d->head_dim < 8 || d->head_dim % 8 || d->head_dim > 512)
    return !set_last_error(NJ_EINVAL, "%s: head_dim must be a multiple of 8, at most 512", what);
  if (d->dtype == NJ_BF16 && d->head_dim != 128) return !set_last_error(NJ_EINVAL, "%s: bf16 path needs head_dim 128", what);
  if (d->n_heads > 1024) return !set_last_error(NJ_EINVAL, "%s: more than 1024 heads", what);
  return true;
}

bool batch_sizes(const char* what, int32_t B, int32_t rows, int32_t max_chunk) {
  if (B < 1 || rows < 1 || max_chunk < 1 || max_chunk > rows)
    return !set_last_error(NJ_EINVAL, "%s: need B >= 1, rows >= 1 and 1 <= max_chunk <= rows", what);
  if (B > (1 << 20) || rows > (1 << 24)) return !set_last_error(NJ_EINVAL, "%s: more than 2^20 sequences or 2^24 rows", what);
  return true;
}

bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  return (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}
bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The checks that the chunk calls share; fills the kernels' view of the batch.
bool chunk_args(const char* what, const nj_model_desc* d, const nj_kv_layer* kv, const nj_chunk_batch* bt, void* ws,
                size_t ws_bytes, size_t need, ChunkK* out) {
  if (!kv || !bt) return !set_last_error(NJ_EINVAL, "%s: NULL cache or batch", what);
  if (!batch_sizes(what, bt->B, bt->rows, bt->max_chunk)) return false;
  if (bt->max_blocks < 1 || kv->num_blocks < 1)
    return !set_last_error(NJ_EINVAL, "%s: max_blocks and num_blocks must be >= 1", what);
  if (bt->max_blocks > (1 << 21)) return !set_last_error(NJ_EINVAL, "%s: max_blocks > 2^21", what);
  if (!bt->starts || !bt->context_lens || !bt->block_table || !kv->k || !kv->v)
    return !set_last_error(NJ_EINVAL, "%s: a required pointer is NULL", what);
  const bool pages_ok = d->dtype == NJ_F32 ? kv->dtype == NJ_F32 : kv->dtype == NJ_BF16 || kv->dtype == NJ_E4M3;
  if (!pages_ok)
    return !set_last_error(NJ_EINVAL, "%s: NJ_F32 pages go with an NJ_F32 descriptor, NJ_BF16 and NJ_E4M3 pages with NJ_BF16", what);
  if (kv->dtype == NJ_E4M3 && (!kv->k_scale || !kv->v_scale))
    return !set_last_error(NJ_EINVAL, "%s: NJ_E4M3 pages need k_scale and v_scale", what);
  if (!al16(kv->k) || !al16(kv->v) || (kv->dtype == NJ_E4M3 && (!al16(kv->k_scale) || !al16(kv->v_scale))))
    return !set_last_error(NJ_EINVAL, "%s: pages and scales must be 16-byte aligned", what);
  if (!ws || ws_bytes < need)
    return !set_last_error(NJ_EINVAL, "%s: workspace NULL or too small (%zu < %zu bytes)", what, ws_bytes, need);
  if (((uintptr_t)ws & 255) != 0) return !set_last_error(NJ_EINVAL, "%s: workspace must be 256-byte aligned", what);
  *out = {bt->starts, bt->context_lens, bt->block_table, bt->max_blocks, bt->B, bt->rows, bt->max_chunk, kv->num_blocks,
          static_cast<int*>(ws)};
  return true;
}

int page_type(const nj_kv_layer* kv) { return kv->dtype == NJ_F32 ? kPageF32 : kv->dtype == NJ_BF16 ? kPageBF16 : kPageE4M3; }

constexpr size_t kErrBytes = 256;

// Workspace of the attention: [error word][parts of the tiles][parts of the streamed pieces].
struct AttnParts {
  bool tiles, stream;
  size_t o[2], ml[2], cnt[2], total;
};
AttnParts attn_parts(const nj_model_desc& d, int max_chunk) {
  AttnParts p{};
  p.total = kErrBytes;
  const int G = d.n_heads / d.n_kv_heads;
  if (d.dtype == NJ_F32 || G > kTileRows) return p;
  p.tiles = (int64_t)max_chunk * G > kStreamRows;
  p.stream = G <= (p.tiles ? 16 : kStreamRows);
  const int rows[2] = {kTileRows, kStreamRows};
  const bool used[2] = {p.tiles, p.stream};
  for (int c = 0; c < 2; ++c)
    if (used[c]) {
      p.o[c] = p.total;
      p.ml[c] = p.o[c] + (size_t)kSlots[c] * rows[c] * kHD * 4;
      p.cnt[c] = p.ml[c] + (size_t)kSlots[c] * rows[c] * 8;
      p.total = p.cnt[c] + (size_t)kSlots[c] * kCounterStride * 4;
    }
  return p;
}

// Which kernels a batch needs.  Batches of short chunks (up to 32 query rows per
// KV head, two of the stream kernel's row tiles) are streamed; where longer ones are
// about, sequences of up to 16 rows are streamed and the others go by tiles.  Where
// the batch can hold no short sequence (or only by padding), the tiles take
// everything, and one launch is saved.
hipError_t launch_chunk_attn(ChunkAttnK& a, const AttnParts& p, int pt, int B, int rows, int max_chunk, hipStream_t s) {
  const int G = a.G;
  if (pt == kPageF32 || G > kTileRows) {
    auto kern = pt == kPageF32    ? chunk_attn_row_kernel<kPageF32, float>
                : pt == kPageBF16 ? chunk_attn_row_kernel<kPageBF16, bf16_t>
                                  : chunk_attn_row_kernel<kPageE4M3, bf16_t>;
    hipLaunchKernelGGL(kern, dim3(rows, a.H), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  const bool all_long = p.tiles && (!p.stream || (int64_t)B * max_chunk <= rows);
  const bool one_tile = p.tiles || max_chunk * G <= 16;  // of the stream kernel's 16-row tiles
  a.threshold = all_long ? 0 : p.tiles ? 16 : INT_MAX;
  a.min_cut[kTiles] = kMinCutTiles;
  a.min_cut[kStream] = kMinCutStream[one_tile ? 0 : 1];
  hipError_t e = hipSuccess;
  if (p.tiles) {
    const int tiles = rows / a.tokens + std::min(B, rows), pieces = tiles + a.pieces[kTiles];
    // Tiles may be cut where they are few and the contexts (as far as the table reaches) long: their parts get a
    // launch of their own.  (A large batch that is mostly padding can hold few tiles too: the last part joins.)
    const bool merge = tiles <= a.pieces[kTiles] && (int64_t)a.c.max_blocks * kBlock > kMinCutTiles;
    a.join_max = merge ? 1 : INT_MAX;
    hipLaunchKernelGGL(pt == kPageE4M3 ? chunk_tile_kernel<kPageE4M3> : chunk_tile_kernel<kPageBF16>, dim3(pieces * a.Hkv),
                       dim3(256), 0, s, a);
    e = hipGetLastError();
    if (e == hipSuccess && merge) {
      hipLaunchKernelGGL(chunk_merge_kernel, dim3(tiles * a.Hkv, kTileRows / 8), dim3(256), 0, s, a);
      e = hipGetLastError();
    }
  }
  if (!all_long && e == hipSuccess) {
    const int pieces = std::min(B, rows) + a.pieces[kStream];
    auto kern = pt == kPageE4M3 ? (one_tile ? chunk_stream_kernel<kPageE4M3, 1> : chunk_stream_kernel<kPageE4M3, 2>)
                                : (one_tile ? chunk_stream_kernel<kPageBF16, 1> : chunk_stream_kernel<kPageBF16, 2>);
    hipLaunchKernelGGL(kern, dim3(pieces * a.Hkv), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

extern "C" {

int nightjar_chunk_store(const nj_model_desc* desc, const nj_kv_layer* kv, const nj_chunk_batch* batch,
                         const float* qkv, int64_t qkv_stride, void* q_out, void* workspace, size_t workspace_bytes,
                         void* stream) {
  ChunkK a;
  if (!chunk_sizes(desc, "chunk_store") ||
      !chunk_args("chunk_store", desc, kv, batch, workspace, workspace_bytes, kErrBytes, &a))
    return NJ_EINVAL;
  const nj_model_desc& d = *desc;
  if (!(d.rope_theta > 0.f)) return set_last_error(NJ_EINVAL, "chunk_store: rope_theta must be > 0");
  if (!qkv) return set_last_error(NJ_EINVAL, "chunk_store: qkv is NULL");
  if (qkv_stride < (int64_t)(d.n_heads + 2 * d.n_kv_heads) * d.head_dim || qkv_stride % 4)
    return set_last_error(NJ_EINVAL, "chunk_store: qkv_stride must be a multiple of 4, at least (H + 2 Hkv) * D");
  if (!al16(qkv) || !al16(q_out)) return set_last_error(NJ_EINVAL, "chunk_store: qkv and q_out must be 16-byte aligned");
  const size_t in_bytes = ((size_t)(batch->rows - 1) * qkv_stride + (d.n_heads + 2 * d.n_kv_heads) * d.head_dim) * 4;
  if (q_out && overlap(qkv, in_bytes, q_out, (size_t)batch->rows * d.n_heads * d.head_dim * (d.dtype == NJ_F32 ? 4 : 2)))
    return set_last_error(NJ_EINVAL, "chunk_store: qkv and q_out overlap");
  const hipError_t e = launch_chunk_store(a, page_type(kv), qkv, qkv_stride, d.n_heads, d.n_kv_heads, d.head_dim,
                                          d.rope_theta, q_out, kv->k, kv->v, kv->k_scale, kv->v_scale, (hipStream_t)stream);
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "chunk_store: %s", hipGetErrorString(e));
}

int nightjar_chunk_load(const nj_model_desc* desc, const nj_kv_layer* kv, const nj_chunk_batch* batch, void* k_out,
                        void* v_out, void* workspace, size_t workspace_bytes, void* stream) {
  ChunkK a;
  if (!chunk_sizes(desc, "chunk_load") ||
      !chunk_args("chunk_load", desc, kv, batch, workspace, workspace_bytes, kErrBytes, &a))
    return NJ_EINVAL;
  if (!k_out || !v_out || !al16(k_out) || !al16(v_out))
    return set_last_error(NJ_EINVAL, "chunk_load: k_out and v_out must be 16-byte aligned and not NULL");
  const size_t out_bytes = (size_t)batch->rows * desc->n_kv_heads * desc->head_dim * (desc->dtype == NJ_F32 ? 4 : 2);
  if (overlap(k_out, out_bytes, v_out, out_bytes)) return set_last_error(NJ_EINVAL, "chunk_load: k_out and v_out overlap");
  const hipError_t e = launch_chunk_load(a, page_type(kv), desc->n_kv_heads, desc->head_dim, kv->k, kv->v, kv->k_scale,
                                         kv->v_scale, k_out, v_out, (hipStream_t)stream);
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "chunk_load: %s", hipGetErrorString(e));
}

size_t nightjar_chunk_attn_workspace_bytes(const nj_model_desc* desc, int32_t B, int32_t rows, int32_t max_chunk) {
  if (!chunk_sizes(desc, "chunk_attn") || !batch_sizes("chunk_attn", B, rows, max_chunk)) return 0;
  return attn_parts(*desc, max_chunk).total;
}

int nightjar_chunk_attn(const nj_model_desc* desc, const nj_kv_layer* kv, const nj_chunk_batch* batch, const void* q,
                        void* out, void* workspace, size_t workspace_bytes, void* stream) {
  ChunkK c;
  if (!chunk_sizes(desc, "chunk_attn")) return NJ_EINVAL;
  if (!batch) return set_last_error(NJ_EINVAL, "chunk_attn: NULL cache or batch");
  const size_t need = nightjar_chunk_attn_workspace_bytes(desc, batch->B, batch->rows, batch->max_chunk);
  if (!need || !chunk_args("chunk_attn", desc, kv, batch, workspace, workspace_bytes, need, &c)) return NJ_EINVAL;
  if (!q || !out || !al16(q) || !al16(out))
    return set_last_error(NJ_EINVAL, "chunk_attn: q and out must be 16-byte aligned and not NULL");
  const nj_model_desc& d = *desc;
  const size_t row_bytes = (size_t)batch->rows * d.n_heads * d.head_dim * (d.dtype == NJ_F32 ? 4 : 2);
  if (overlap(q, row_bytes, out, row_bytes))
    return set_last_error(NJ_EINVAL, "chunk_attn: q and out overlap");
  const AttnParts p = attn_parts(d, batch->max_chunk);
  ChunkAttnK a{};
  a.c = c;
  a.q = q;
  a.kp = kv->k;
  a.vp = kv->v;
  a.ks = static_cast<const uint8_t*>(kv->k_scale);
  a.vs = static_cast<const uint8_t*>(kv->v_scale);
  a.out = out;
  a.H = d.n_heads;
  a.Hkv = d.n_kv_heads;
  a.D = d.head_dim;
  a.G = d.n_heads / d.n_kv_heads;
  a.tokens = kTileRows / a.G;
  a.inv_tokens = a.tokens ? 1.0f / (float)a.tokens : 0.f;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)d.head_dim);
  for (int k = 0; k < 2; ++k) {
    a.part_o[k] = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.o[k]);
    a.part_ml[k] = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.ml[k]);
    a.counters[k] = reinterpret_cast<int*>(static_cast<char*>(workspace) + p.cnt[k]);
    a.pieces[k] = std::max(1, kPieces[k] / d.n_kv_heads);
  }
  const hipError_t e = launch_chunk_attn(a, p, page_type(kv), batch->B, batch->rows, batch->max_chunk, (hipStream_t)stream);
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "chunk_attn: %s", hipGetErrorString(e));
}

}  // extern "C"
