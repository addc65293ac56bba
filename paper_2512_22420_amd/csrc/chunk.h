// Ragged chunk batches (nj_chunk_batch) on the device, shared by the kernels
// that write a chunk to the paged cache, read it back and attend over it.
#pragma once

#include "common.h"

namespace nj {

// KV page element types (NJ_F32, NJ_BF16, NJ_E4M3 of the public headers).
constexpr int kPageF32 = 0, kPageBF16 = 1, kPageE4M3 = 2;

struct ChunkK {
  const int32_t* starts;  // [B+1]
  const int32_t* ctx;     // [B]
  const int32_t* table;   // [B][max_blocks]
  int max_blocks, B, rows, max_chunk, num_blocks;
  int* err;
};

// Sequence b's rows s0 .. s0+n-1 at positions c ..; n = 0 if it has none or
// breaks the batch's rules (bad).
struct ChunkSeq {
  int s0, n, c;
  bool bad;
};
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkK& a, int b) {
  const int s0 = a.starts[b], s1 = a.starts[b + 1], c = a.ctx[b];
  const bool order = s0 >= 0 && s0 <= s1 && s1 <= a.rows;
  const int n = order ? s1 - s0 : 0;
  const bool bad = !order || (n > 0 && (n > a.max_chunk || c < 0 || (int64_t)c + n > (int64_t)a.max_blocks * kBlock));
  return {s0, bad ? 0 : n, c, bad};
}

// The last b in [0, B) with f(b) <= u, f not decreasing; -1 if there is none.
// Run by whole waves, u uniform: each round the 64 lanes probe 64 places.
template <typename F>
__device__ __forceinline__ int chunk_find(int B, int u, F f) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = B;
  while (true) {
    const int step = (len + kWave - 1) / kWave, at = lo + lane * step;
    const bool in = lane * step < len && f(at) <= u;
    const int cnt = __popcll(__ballot(in));
    if (cnt == 0) return -1;  // only in the first round (f not decreasing), or on a batch that breaks the rules
    lo += (cnt - 1) * step;
    if (step == 1) return lo;
    len = min(step, len - (cnt - 1) * step);
  }
}

// Cutting sequences into page blocks without a plan: sequence b takes units
// chunk_unit0(b) .. chunk_unit0(b+1)-1, at least as many as the 16-token blocks
// that its rows touch ((n + 14) / 16 + 1 at most), and chunk_units() in all.
__device__ __forceinline__ int chunk_unit0(const ChunkK& a, int b) { return max(0, min(a.starts[b], a.rows)) / kBlock + 2 * b; }
inline int chunk_units(int B, int rows) { return rows / kBlock + 2 * B; }

// One page block of a sequence's chunk: rows row0 .. row0+nt-1 at slots
// slot0 .. of logical block blk; nt = 0: nothing to do.
struct ChunkUnit {
  int b, row0, nt, slot0, pos0;
  int phys;  // physical block, -1 if the table's entry is bad
};
__device__ __forceinline__ ChunkUnit chunk_unit(const ChunkK& a, int u) {
  ChunkUnit r{0, 0, 0, 0, 0, -1};
  const int b = chunk_find(a.B, u, [&](int i) { return chunk_unit0(a, i); });
  if (b < 0) return r;
  const ChunkSeq s = chunk_seq(a, b);
  if (s.n == 0) return r;
  const int blk = s.c / kBlock + (u - chunk_unit0(a, b));
  const int64_t p0 = (int64_t)blk * kBlock;
  const int i0 = (int)max((int64_t)0, p0 - s.c), i1 = (int)min((int64_t)s.n, p0 + kBlock - s.c);
  if (i0 >= i1) return r;  // a unit behind the sequence's last block
  const int id = a.table[(size_t)b * a.max_blocks + blk];
  return {b, s.s0 + i0, i1 - i0, (int)(s.c + i0 - p0), s.c + i0, id >= 0 && id < a.num_blocks ? id : -1};
}

// Flags sequences that break the batch's rules (one workgroup per launch).
__device__ __forceinline__ void chunk_check(const ChunkK& a) {
  bool bad = false;
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) bad |= chunk_seq(a, b).bad;
  if (__ballot(bad) && (threadIdx.x & 63) == 0) flag_error(a.err, kErrContext);
}

// e4m3 with a power-of-two scale per head row: the smallest 2^e with
// amax <= 448 2^e = 1.75 * 2^(e+8), so e follows from amax's exponent and
// whether its mantissa passes 1.75.  Clamped to [-112, 119]: below it the
// smallest code (2^-9) would leave bf16's normal numbers, above it 448 2^e would
// overflow.
constexpr int kE4m3ScaleMin = -112, kE4m3ScaleMax = 119;
__device__ __forceinline__ int e4m3_scale_exp(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kE4m3ScaleMin), kE4m3ScaleMax);
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ bool finite_f(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// x * 2^-e for a code: saturated at 448, NaN where x is not finite
__device__ __forceinline__ float e4m3_arg(float x, float inv) {
  return finite_f(x) ? fminf(fmaxf(x * inv, -448.f), 448.f) : __uint_as_float(0x7fc00000u);
}
// four codes, the first in the low byte (v_cvt_pk_fp8_f32, round to nearest even)
__device__ __forceinline__ uint32_t e4m3_pack4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}

}  // namespace nj
