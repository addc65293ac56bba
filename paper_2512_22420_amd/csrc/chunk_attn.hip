// Attention of a chunk of new tokens over a paged cache: row i of a sequence
// sees positions 0 .. c + i, all of them in the pages.
#include <algorithm>

#include "../../include/nightjar_serve.h"
#include "chunk.h"
#include "kernels.h"

namespace nj {
namespace {

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
};

// Element i of an array of page type PT (e4m3: the code's value, without its scale).
template <int PT>
__device__ __forceinline__ float page_at(const void* p, size_t i) {
  if constexpr (PT == kPageF32) return static_cast<const float*>(p)[i];
  if constexpr (PT == kPageBF16) return bf2f(static_cast<const bf16_t*>(p)[i]);
  if constexpr (PT == kPageE4M3) return __builtin_amdgcn_cvt_f32_fp8((int)static_cast<const uint8_t*>(p)[i], 0);
}

// One workgroup per (row, head), 256 keys at a time: a thread scores one key,
// then sums one output dim (any head dim up to 512).
constexpr int kMaxD = 512;
template <int PT, typename T>
__global__ __launch_bounds__(256) void chunk_attn_row_kernel(ChunkAttnK a) {
  __shared__ float s_q[kMaxD], s_p[256], s_red[4];
  __shared__ int s_id[16];
  if (blockIdx.x == 0 && blockIdx.y == 0) chunk_check(a.c);
  const int row = blockIdx.x, h = blockIdx.y, t = threadIdx.x, D = a.D, g = h / (a.H / a.Hkv);
  const int b = chunk_find(a.c.B, row, [&](int i) { return a.c.starts[i]; });
  if (b < 0) return;
  const ChunkSeq s = chunk_seq(a.c, b);
  const int i = row - s.s0;
  if (i >= s.n) return;
  const T* q = static_cast<const T*>(a.q) + ((size_t)row * a.H + h) * D;
  for (int d = t; d < D; d += 256) s_q[d] = to_f(q[d]);
  const int n = s.c + i + 1;
  float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
  bool bad = false;
  for (int k0 = 0; k0 < n; k0 += 256) {
    __syncthreads();
    if (t < 16) {
      const int blk = k0 / kBlock + t;
      int id = blk * kBlock < n ? a.c.table[(size_t)b * a.c.max_blocks + blk] : 0;
      if (id < 0 || id >= a.c.num_blocks) {
        bad = true;
        id = -1;
      }
      s_id[t] = id;
    }
    __syncthreads();
    const int k = k0 + t, id = s_id[t / kBlock];
    float sc = -INFINITY;
    if (k < n && id >= 0) {
      const size_t slot = ((size_t)id * a.Hkv + g) * kBlock + t % kBlock;
      float dot = 0.f;
      for (int d = 0; d < D; ++d) dot = fmaf(s_q[d], page_at<PT>(a.kp, slot * D + d), dot);
      if constexpr (PT == kPageE4M3) dot *= __uint_as_float((uint32_t)a.ks[slot] << 23);
      sc = dot * a.scale_log2;
    }
    const float mn = fmaxf(m, block_max<256>(sc, s_red));
    const float p = sc == -INFINITY ? 0.f : exp2f(sc - mn), al = m == -INFINITY ? 0.f : exp2f(m - mn);
    m = mn;
    l = l * al + block_sum<256>(p, s_red);
    s_p[t] = p;
    __syncthreads();
    for (int e = 0; e < 2; ++e) {
      const int d = t + 256 * e;
      if (d >= D) break;
      float acc = o[e] * al;
      for (int j = 0; j < 256 && k0 + j < n; ++j) {
        const int jd = s_id[j / kBlock];
        if (jd < 0) continue;
        const size_t head = ((size_t)jd * a.Hkv + g) * kBlock;
        float v = page_at<PT>(a.vp, head * D + (size_t)d * kBlock + j % kBlock);
        if constexpr (PT == kPageE4M3) v *= __uint_as_float((uint32_t)a.vs[head + j % kBlock] << 23);
        acc = fmaf(s_p[j], v, acc);
      }
      o[e] = acc;
    }
  }
  if (bad) flag_error(a.c.err, kErrBlock);
  for (int e = 0; e < 2; ++e) {
    const int d = t + 256 * e;
    if (d < D) static_cast<T*>(a.out)[((size_t)row * a.H + h) * D + d] = from_f<T>(o[e] / l);
  }
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

bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The checks that the chunk calls share; fills the kernels' view of the batch.
bool chunk_args(const char* what, const nj_model_desc* d, const nj_kv_layer* kv, const nj_chunk_batch* bt, void* ws,
                size_t ws_bytes, size_t need, ChunkK* out) {
  if (!kv || !bt) return !set_last_error(NJ_EINVAL, "%s: NULL cache or batch", what);
  if (!batch_sizes(what, bt->B, bt->rows, bt->max_chunk)) return false;
  if (bt->max_blocks < 1 || kv->num_blocks < 1)
    return !set_last_error(NJ_EINVAL, "%s: max_blocks and num_blocks must be >= 1", what);
  if (bt->max_blocks > (1 << 26)) return !set_last_error(NJ_EINVAL, "%s: max_blocks > 2^26", what);
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
  const hipError_t e = launch_chunk_load(a, page_type(kv), desc->n_kv_heads, desc->head_dim, kv->k, kv->v, kv->k_scale,
                                         kv->v_scale, k_out, v_out, (hipStream_t)stream);
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "chunk_load: %s", hipGetErrorString(e));
}

size_t nightjar_chunk_attn_workspace_bytes(const nj_model_desc* desc, int32_t B, int32_t rows, int32_t max_chunk) {
  if (!chunk_sizes(desc, "chunk_attn") || !batch_sizes("chunk_attn", B, rows, max_chunk)) return 0;
  return kErrBytes;
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
  if ((uintptr_t)q < (uintptr_t)out + row_bytes && (uintptr_t)out < (uintptr_t)q + row_bytes)
    return set_last_error(NJ_EINVAL, "chunk_attn: q and out overlap");
  ChunkAttnK a{c, q, kv->k, kv->v, static_cast<const uint8_t*>(kv->k_scale), static_cast<const uint8_t*>(kv->v_scale),
               out, d.n_heads, d.n_kv_heads, d.head_dim, 1.4426950408889634f / sqrtf((float)d.head_dim)};
  const int pt = page_type(kv);
  auto kern = pt == kPageF32    ? chunk_attn_row_kernel<kPageF32, float>
              : pt == kPageBF16 ? chunk_attn_row_kernel<kPageBF16, bf16_t>
                                : chunk_attn_row_kernel<kPageE4M3, bf16_t>;
  hipLaunchKernelGGL(kern, dim3(batch->rows, d.n_heads), dim3(256), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? NJ_OK : set_last_error(NJ_EHIP, "chunk_attn: %s", hipGetErrorString(e));
}

}  // extern "C"
