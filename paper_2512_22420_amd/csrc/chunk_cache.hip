// A chunk's queries and keys rotated, its keys and values written to the paged
// cache (fp32, bf16, or e4m3 with a scale per token and KV head), and read back.
//
// Both directions move bytes: per token (H + 2 Hkv) D fp32 in, q and the codes
// out.  Work is cut at page blocks, so that a workgroup holds the 16 tokens
// whose values lie side by side in a V block ([D][16]) and writes whole lines of
// it.
#include <math.h>

#include "../../include/nightjar_serve.h"
#include "chunk.h"
#include "kernels.h"

namespace nj {
namespace {

constexpr int kD = 128;  // head dim of the bf16 path

struct RopeFreq64 {
  double inv_freq[64];  // theta^(-2j/128)
};

// sin and cos of position * inv_freq in 64 bits (ocml reduces any argument).
__device__ __forceinline__ double2 rope_angle(int pos, double inv_freq) {
  double s, c;
  sincos((double)pos * inv_freq, &s, &c);
  return {c, s};
}

// grid (chunk_units, head groups of kStoreHeads): one page block of one
// sequence, some heads.  16 lanes hold a (token, head) row, lane l the rotation
// pairs (4l + e, 64 + 4l + e).  Bound by memory: a prompt of 8000 (8B layout, e4m3) with
// its read back 77 us, 4.3 TB/s (81 with 8 heads a workgroup, 83 with 2, whose angles are
// computed as often as they are used); 20 chunks of 100: 24.6, 26.7 and 25.8; 64 single
// tokens, bound by their two launches: 9.7, 9.4 and 11.5.
constexpr int kStoreHeads = 4;
template <int PT>
__global__ __launch_bounds__(256) void chunk_store_kernel(ChunkK a, const float* __restrict__ qkv, int64_t stride, int H,
                                                          int Hkv, RopeFreq64 f, bf16_t* __restrict__ q_out,
                                                          void* __restrict__ kp, void* __restrict__ vp,
                                                          uint8_t* __restrict__ ks, uint8_t* __restrict__ vs) {
  __shared__ double2 s_cs[kBlock][64];
  __shared__ __attribute__((aligned(16))) char s_v[kD * kBlock * 2];
  if (blockIdx.x == 0 && blockIdx.y == 0) chunk_check(a);
  const ChunkUnit u = chunk_unit(a, blockIdx.x);
  if (u.nt == 0) return;
  if (u.phys < 0 && blockIdx.y == 0 && threadIdx.x == 0) flag_error(a.err, kErrBlock);
  const int nh = H + 2 * Hkv, h0 = blockIdx.y * kStoreHeads, h1 = min(h0 + kStoreHeads, nh), nt = u.nt;
  if (h0 < H + Hkv) {
    for (int e = threadIdx.x; e < nt * 64; e += 256) s_cs[e >> 6][e & 63] = rope_angle(u.pos0 + (e >> 6), f.inv_freq[e & 63]);
  }
  __syncthreads();
  const int j0 = 4 * (threadIdx.x & 15);
  const int items = nt * (h1 - h0);
  const bool whole = nt == kBlock;  // a pass is then one head's 16 tokens
  for (int base = 0; base < items; base += 16) {
    const int it = base + (threadIdx.x >> 4);
    const bool on = it < items;
    const int hd = h0 + min(it, items - 1) / nt, i = min(it, items - 1) % nt;
    const float* src = qkv + (size_t)(u.row0 + i) * stride + (size_t)hd * kD;
    const f32x4 lo = *reinterpret_cast<const f32x4*>(src + j0), hi = *reinterpret_cast<const f32x4*>(src + 64 + j0);
    float x[8];
    if (hd < H + Hkv) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double2 cs = s_cs[i][j0 + e];
        const double p = lo[e], q = hi[e];
        x[e] = (float)(p * cs.x - q * cs.y);
        x[4 + e] = (float)(q * cs.x + p * cs.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = lo[e];
        x[4 + e] = hi[e];
      }
    }
    if (hd < H) {
      if (on && q_out) {
        bf16_t* dst = q_out + ((size_t)(u.row0 + i) * H + hd) * kD;
        *reinterpret_cast<u32x2*>(dst + j0) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
        *reinterpret_cast<u32x2*>(dst + 64 + j0) = u32x2{pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
      }
      continue;  // (whole blocks: the same for every thread of a pass)
    }
    const bool is_k = hd < H + Hkv;
    const int g = is_k ? hd - H : hd - H - Hkv, slot = u.slot0 + i;
    const size_t head = ((size_t)max(u.phys, 0) * Hkv + g) * kBlock;  // token slots before this head's block
    uint32_t w[4] = {};  // bf16: 2 + 2 words; e4m3: 1 + 1
    if constexpr (PT == kPageE4M3) {
      float am = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) am = fmaxf(am, finite_f(x[e]) ? fabsf(x[e]) : 0.f);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor(am, o));
      const int e = e4m3_scale_exp(am);
      const float inv = pow2i(-e);
      w[0] = e4m3_pack4(e4m3_arg(x[0], inv), e4m3_arg(x[1], inv), e4m3_arg(x[2], inv), e4m3_arg(x[3], inv));
      w[1] = e4m3_pack4(e4m3_arg(x[4], inv), e4m3_arg(x[5], inv), e4m3_arg(x[6], inv), e4m3_arg(x[7], inv));
      if (on && u.phys >= 0 && (threadIdx.x & 15) == 0) (is_k ? ks : vs)[head + slot] = (uint8_t)(e + 127);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
    }
    if (is_k) {
      if (on && u.phys >= 0) {
        if constexpr (PT == kPageE4M3) {
          uint8_t* dst = static_cast<uint8_t*>(kp) + (head + slot) * kD;
          *reinterpret_cast<uint32_t*>(dst + j0) = w[0];
          *reinterpret_cast<uint32_t*>(dst + 64 + j0) = w[1];
        } else {
          bf16_t* dst = static_cast<bf16_t*>(kp) + (head + slot) * kD;
          *reinterpret_cast<u32x2*>(dst + j0) = u32x2{w[0], w[1]};
          *reinterpret_cast<u32x2*>(dst + 64 + j0) = u32x2{w[2], w[3]};
        }
      }
      continue;
    }
    // V: dim-major in the block, [D][16]
    if (whole) {
      __syncthreads();  // the previous head's reads
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = (e < 4 ? 0 : 64) + j0 + (e & 3);
        if constexpr (PT == kPageE4M3)
          reinterpret_cast<uint8_t*>(s_v)[d * kBlock + i] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
        else
          reinterpret_cast<bf16_t*>(s_v)[d * kBlock + i] = (bf16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
      __syncthreads();
      constexpr int kBytes = kD * kBlock * (PT == kPageE4M3 ? 1 : 2);
      char* dst = static_cast<char*>(vp) + ((size_t)max(u.phys, 0) * Hkv + g) * kBytes;
      if (u.phys >= 0 && (int)threadIdx.x * 16 < kBytes)
        *reinterpret_cast<u32x4*>(dst + threadIdx.x * 16) = *reinterpret_cast<const u32x4*>(s_v + threadIdx.x * 16);
    } else if (on && u.phys >= 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const size_t d = (e < 4 ? 0 : 64) + j0 + (e & 3);
        const size_t at = (head * kD) + d * kBlock + slot;
        if constexpr (PT == kPageE4M3)
          static_cast<uint8_t*>(vp)[at] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
        else
          static_cast<bf16_t*>(vp)[at] = (bf16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// The fp32 path: any head dim; one thread per (row, head, rotation pair).
// grid (rows, pieces of nh * D/2).
__global__ __launch_bounds__(256) void chunk_store_f32_kernel(ChunkK a, const float* __restrict__ qkv, int64_t stride,
                                                              int H, int Hkv, int D, RopeFreq f, float* __restrict__ q_out,
                                                              float* __restrict__ kp, float* __restrict__ vp) {
  if (blockIdx.x == 0 && blockIdx.y == 0) chunk_check(a);
  const int row = blockIdx.x;
  const int b = chunk_find(a.B, row, [&](int i) { return a.starts[i]; });
  if (b < 0) return;
  const ChunkSeq s = chunk_seq(a, b);
  const int i = row - s.s0;
  if (i < 0 || i >= s.n) return;  // (before it: where starts decrease)
  const int half = D / 2, t = blockIdx.y * 256 + threadIdx.x;
  if (t >= (H + 2 * Hkv) * half) return;
  const int hd = t / half, j = t % half, pos = s.c + i;
  const float* src = qkv + (size_t)row * stride + (size_t)hd * D;
  float lo = src[j], hi = src[j + half];
  if (hd < H + Hkv) {
    const double2 cs = rope_angle(pos, f.inv_freq[j]);
    const double p = lo, q = hi;
    lo = (float)(p * cs.x - q * cs.y);
    hi = (float)(q * cs.x + p * cs.y);
  }
  if (hd < H) {
    if (q_out) {
      q_out[((size_t)row * H + hd) * D + j] = lo;
      q_out[((size_t)row * H + hd) * D + j + half] = hi;
    }
    return;
  }
  const int id = a.table[(size_t)b * a.max_blocks + pos / kBlock], slot = pos % kBlock;
  if (id < 0 || id >= a.num_blocks) {
    if (j == 0) flag_error(a.err, kErrBlock);
    return;
  }
  if (hd < H + Hkv) {
    float* dst = kp + (((size_t)id * Hkv + (hd - H)) * kBlock + slot) * D;
    dst[j] = lo;
    dst[j + half] = hi;
  } else {
    float* dst = vp + ((size_t)id * Hkv + (hd - H - Hkv)) * D * kBlock + slot;
    dst[(size_t)j * kBlock] = lo;
    dst[(size_t)(j + half) * kBlock] = hi;
  }
}

// Eight e4m3 codes (two words) times a power of two as bf16, exact.
__device__ __forceinline__ u32x4 e4m3_to_bf16x8(u32x2 c, const float (&sc)[8]) {
  u32x4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
    o[2 * h] = pack_bf16x2(lo[0] * sc[4 * h], lo[1] * sc[4 * h + 1]);
    o[2 * h + 1] = pack_bf16x2(hi[0] * sc[4 * h + 2], hi[1] * sc[4 * h + 3]);
  }
  return o;
}

// grid (chunk_units, ceil(Hkv / NH)): one page block of one sequence, NH heads, whose
// loads are all in flight together.  K rows are contiguous; V is turned to rows through
// LDS.
constexpr int kLoadMany = 512;  // workgroups
constexpr int kLoadRow = kD + 8;  // LDS row stride in elements
template <int PT, int NH>
__global__ __launch_bounds__(256) void chunk_load_kernel(ChunkK a, int Hkv, const void* __restrict__ kp,
                                                         const void* __restrict__ vp, const uint8_t* __restrict__ ks,
                                                         const uint8_t* __restrict__ vs, bf16_t* __restrict__ k_out,
                                                         bf16_t* __restrict__ v_out) {
  __shared__ __attribute__((aligned(16))) bf16_t s_v[NH][kBlock][kLoadRow];
  if (blockIdx.x == 0 && blockIdx.y == 0) chunk_check(a);
  const ChunkUnit u = chunk_unit(a, blockIdx.x);
  if (u.nt == 0) return;
  if (u.phys < 0) {
    if (blockIdx.y == 0 && threadIdx.x == 0) flag_error(a.err, kErrBlock);
    return;
  }
  const int g0 = blockIdx.y * NH, t = threadIdx.x;
  const int tok = t >> 4, e0 = 8 * (t & 15);  // K: this thread's row and dims
  const int d = t >> 1, t0 = 8 * (t & 1);     // V: this thread's dim and slots
  const int i = tok - u.slot0;
  const bool on = i >= 0 && i < u.nt;
  u32x4 kx[NH], vx[NH];
  if constexpr (PT == kPageE4M3) {
    u32x2 kc[NH], vc[NH], vb[NH];
    uint8_t kb[NH];
#pragma unroll
    for (int q = 0; q < NH; ++q) {
      const size_t head = ((size_t)u.phys * Hkv + min(g0 + q, Hkv - 1)) * kBlock;
      kc[q] = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(kp) + (head + tok) * kD + e0);
      vc[q] = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(vp) + head * kD + d * kBlock + t0);
      vb[q] = *reinterpret_cast<const u32x2*>(vs + head + t0);
      kb[q] = ks[head + tok];
    }
#pragma unroll
    for (int q = 0; q < NH; ++q) {
      const float kscale = __uint_as_float((uint32_t)kb[q] << 23);
      float sk[8], sv[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sk[e] = kscale;
        sv[e] = __uint_as_float(((vb[q][e >> 2] >> (8 * (e & 3))) & 0xffu) << 23);
      }
      kx[q] = e4m3_to_bf16x8(kc[q], sk);
      vx[q] = e4m3_to_bf16x8(vc[q], sv);
    }
  } else {
#pragma unroll
    for (int q = 0; q < NH; ++q) {
      const size_t head = ((size_t)u.phys * Hkv + min(g0 + q, Hkv - 1)) * kBlock;
      kx[q] = *reinterpret_cast<const u32x4*>(static_cast<const bf16_t*>(kp) + (head + tok) * kD + e0);
      vx[q] = *reinterpret_cast<const u32x4*>(static_cast<const bf16_t*>(vp) + head * kD + d * kBlock + t0);
    }
  }
#pragma unroll
  for (int q = 0; q < NH; ++q)
#pragma unroll
    for (int e = 0; e < 8; ++e) s_v[q][t0 + e][d] = (bf16_t)(vx[q][e >> 1] >> (16 * (e & 1)));
  __syncthreads();
  if (!on) return;
#pragma unroll
  for (int q = 0; q < NH; ++q) {
    if (g0 + q >= Hkv) break;
    const size_t at = ((size_t)(u.row0 + i) * Hkv + g0 + q) * kD + e0;
    *reinterpret_cast<u32x4*>(k_out + at) = kx[q];
    *reinterpret_cast<u32x4*>(v_out + at) = *reinterpret_cast<const u32x4*>(&s_v[q][tok][e0]);
  }
}

// The fp32 path: one thread per (row, KV head, dim).  grid (rows, pieces of Hkv * D).
__global__ __launch_bounds__(256) void chunk_load_f32_kernel(ChunkK a, int Hkv, int D, const float* __restrict__ kp,
                                                             const float* __restrict__ vp, float* __restrict__ k_out,
                                                             float* __restrict__ v_out) {
  if (blockIdx.x == 0 && blockIdx.y == 0) chunk_check(a);
  const int row = blockIdx.x;
  const int b = chunk_find(a.B, row, [&](int i) { return a.starts[i]; });
  if (b < 0) return;
  const ChunkSeq s = chunk_seq(a, b);
  const int i = row - s.s0, t = blockIdx.y * 256 + threadIdx.x;
  if (i < 0 || i >= s.n || t >= Hkv * D) return;
  const int g = t / D, d = t % D, pos = s.c + i;
  const int id = a.table[(size_t)b * a.max_blocks + pos / kBlock], slot = pos % kBlock;
  if (id < 0 || id >= a.num_blocks) {
    if (t == 0) flag_error(a.err, kErrBlock);
    return;
  }
  const size_t head = ((size_t)id * Hkv + g) * kBlock;
  k_out[(size_t)row * Hkv * D + t] = kp[(head + slot) * D + d];
  v_out[(size_t)row * Hkv * D + t] = vp[head * D + (size_t)d * kBlock + slot];
}

}  // namespace

hipError_t launch_chunk_store(const ChunkK& a, int pages, const float* qkv, int64_t stride, int H, int Hkv, int D,
                              float theta, void* q_out, void* k, void* v, void* ks, void* vs, hipStream_t s) {
  const int nh = H + 2 * Hkv;
  if (pages == kPageF32) {
    RopeFreq f;
    for (int j = 0; j < D / 2; ++j) f.inv_freq[j] = pow((double)theta, -2.0 * j / D);
    hipLaunchKernelGGL(chunk_store_f32_kernel, dim3(a.rows, (nh * (D / 2) + 255) / 256), dim3(256), 0, s, a, qkv, stride,
                       H, Hkv, D, f, static_cast<float*>(q_out), static_cast<float*>(k), static_cast<float*>(v));
    return hipGetLastError();
  }
  RopeFreq64 f;
  for (int j = 0; j < 64; ++j) f.inv_freq[j] = pow((double)theta, -2.0 * j / kD);
  auto kern = pages == kPageE4M3 ? chunk_store_kernel<kPageE4M3> : chunk_store_kernel<kPageBF16>;
  hipLaunchKernelGGL(kern, dim3(chunk_units(a.B, a.rows), (nh + kStoreHeads - 1) / kStoreHeads), dim3(256), 0, s, a, qkv,
                     stride, H, Hkv, f, static_cast<bf16_t*>(q_out), k, v, static_cast<uint8_t*>(ks),
                     static_cast<uint8_t*>(vs));
  return hipGetLastError();
}

hipError_t launch_chunk_load(const ChunkK& a, int pages, int Hkv, int D, const void* k, const void* v, const void* ks,
                             const void* vs, void* k_out, void* v_out, hipStream_t s) {
  if (pages == kPageF32) {
    hipLaunchKernelGGL(chunk_load_f32_kernel, dim3(a.rows, (Hkv * D + 255) / 256), dim3(256), 0, s, a, Hkv, D,
                       static_cast<const float*>(k), static_cast<const float*>(v), static_cast<float*>(k_out),
                       static_cast<float*>(v_out));
    return hipGetLastError();
  }
  // Four heads a workgroup where that leaves two a CU (32 contexts of 1500, 7B layout, e4m3: 35 us, 4.2 TB/s, one
  // head a workgroup 44; a context of 8000, 8B layout: 10.7 and 11.7), else one (a context of 2000: 5.2 us, four 5.6).
  const int units = chunk_units(a.B, a.rows), nh = units * ((Hkv + 3) / 4) >= kLoadMany ? 4 : 1;
  auto kern = nh == 4 ? (pages == kPageE4M3 ? chunk_load_kernel<kPageE4M3, 4> : chunk_load_kernel<kPageBF16, 4>)
                      : (pages == kPageE4M3 ? chunk_load_kernel<kPageE4M3, 1> : chunk_load_kernel<kPageBF16, 1>);
  hipLaunchKernelGGL(kern, dim3(units, (Hkv + nh - 1) / nh), dim3(256), 0, s, a, Hkv, k, v,
                     static_cast<const uint8_t*>(ks), static_cast<const uint8_t*>(vs), static_cast<bf16_t*>(k_out),
                     static_cast<bf16_t*>(v_out));
  return hipGetLastError();
}

}  // namespace nj
