// C entry points of the streaming operators (include/vp.h): argument checks and launches.
#include <cuda_runtime.h>
#include <math.h>

#include "internal.h"
#include "seq.h"
#include "vp.h"

using namespace vp;

namespace {

constexpr int kMaxQueryHeads = 128;
constexpr int32_t kMaxTokens = 1 << 30;

#define VP_TRY(x)               \
  do {                          \
    vp_status _s = (x);         \
    if (_s != VP_OK) return _s; \
  } while (0)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// Of 32-bit values read one by one, which may be slices of longer arrays.
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

vp_status check_attn_dims(const vp_attn_dims* dm) {
  if (!dm) return VP_ERR_INVALID_ARG;
  if (dm->dtype != VP_DTYPE_BF16 && dm->dtype != VP_DTYPE_FP16) return VP_ERR_INVALID_ARG;
  if (dm->block < 0 || !isfinite(dm->scale)) return VP_ERR_INVALID_ARG;
  if (dm->d != 64 && dm->d != 128) return VP_ERR_UNSUPPORTED_SHAPE;
  if (dm->Hkv < 1 || dm->Hq < dm->Hkv || dm->Hq > kMaxQueryHeads || dm->Hq % dm->Hkv)
    return VP_ERR_UNSUPPORTED_SHAPE;
  return VP_OK;
}

vp_status check_counts(int32_t T, int32_t B) {
  if (T < 0 || B < 0) return VP_ERR_INVALID_ARG;
  if (T > kMaxTokens || B > kMaxTokens || (T > 0 && B == 0)) return VP_ERR_UNSUPPORTED_SHAPE;
  return VP_OK;
}

// A [T][heads][d] tensor with a token stride.
vp_status check_rows(const void* p, int64_t stride, int heads, int d) {
  if (!p) return VP_ERR_INVALID_ARG;
  if (!aligned16(p)) return VP_ERR_ALIGNMENT;
  if (stride < (int64_t)heads * d || stride > ((int64_t)1 << 36)) return VP_ERR_UNSUPPORTED_SHAPE;
  return stride % 8 ? VP_ERR_ALIGNMENT : VP_OK;
}

vp_status check_kv(const vp_paged_kv* kv) {
  if (!kv || !kv->k || !kv->v || !kv->page_table) return VP_ERR_INVALID_ARG;
  if (!aligned16(kv->k) || !aligned16(kv->v) || !aligned4(kv->page_table)) return VP_ERR_ALIGNMENT;
  const int ps = kv->page_size;
  if (ps < 16 || ps > 1024 || (ps & (ps - 1)) || kv->n_pages < 1 || kv->table_width < 1)
    return VP_ERR_UNSUPPORTED_SHAPE;
  return VP_OK;
}

PagedKv make_kv(const vp_paged_kv* kv) {
  PagedKv p{};
  if (!kv) return p;
  p.k = static_cast<uint16_t*>(kv->k);
  p.v = static_cast<uint16_t*>(kv->v);
  p.table = kv->page_table;
  p.n_pages = kv->n_pages;
  p.page_size = kv->page_size;
  while ((1 << p.log2_page) < kv->page_size) ++p.log2_page;
  p.width = kv->table_width;
  return p;
}

vp_status from_cuda(cudaError_t e) { return e == cudaSuccess ? VP_OK : VP_ERR_CUDA; }

SeqAttnArgs make_args(const vp_attn_dims* dm, int32_t T, int32_t B, const void* q,
                      int64_t q_stride, const int32_t* cu, void* out, int64_t out_stride,
                      float* lse, void* ws) {
  SeqAttnArgs a{};
  a.T = T;
  a.B = B;
  a.Hq = dm->Hq;
  a.Hkv = dm->Hkv;
  a.group = dm->Hq / dm->Hkv;
  a.d = dm->d;
  a.fp16 = dm->dtype == VP_DTYPE_FP16;
  a.block = dm->block;
  a.chain_tokens = 128 / a.group;
  // Chains start anew at every mask block where at most a sixteenth of their rows stays empty: rows
  // of one block see the same keys, and a chain across two blocks would take the masked path
  // for a whole block of keys (8 views of 1,374 tokens, 16 heads: 352 us with chains across the
  // views).
  if (dm->block > a.chain_tokens) {
    const int64_t n = (dm->block + a.chain_tokens - 1) / a.chain_tokens;
    if (16 * (n * a.chain_tokens - dm->block) <= dm->block && n < (1 << 20)) a.block_chains = (int)n;
  }
  a.by_group = FastDiv(a.group);
  a.by_block = FastDiv(a.block);
  a.by_chain_tokens = FastDiv(a.chain_tokens);
  a.by_block_chains = FastDiv(a.block_chains);
  a.scale_log2 = dm->scale * 1.4426950408889634f;
  const float cs = fmaxf(fabsf(a.scale_log2), kLeastScale);
  int e;
  const bool power = frexpf(cs, &e) == 0.5f;  // cs in [2^(e - 1), 2^e)
  a.far_scale = power ? cs : ldexpf(1.f, e < 127 ? e : 127);
  a.far_unit = cs / a.far_scale;
  a.far_from = (float)(kFarScore * (1. - 0x1p-20) / cs);
  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.cu = cu;
  a.out = static_cast<uint16_t*>(out);
  a.out_stride = out_stride;
  a.lse = lse;
  a.err = static_cast<unsigned int*>(ws);
  return a;
}

}  // namespace

extern "C" {

vp_status vp_attn_workspace_size(const vp_attn_dims* dims, int32_t T, int32_t B, size_t* bytes) {
  VP_TRY(check_attn_dims(dims));
  VP_TRY(check_counts(T, B));
  if (!bytes) return VP_ERR_INVALID_ARG;
  *bytes = seq_scratch_bytes(dims->d);
  return VP_OK;
}

vp_status vp_rope_append(const vp_attn_dims* dims, const vp_rope_options* rope, int32_t T, int32_t B,
                         const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, const int32_t* cu, const int32_t* kv_len,
                         const int32_t* positions, const vp_paged_kv* kv, void* q_out,
                         int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* ws,
                         size_t ws_bytes, void* stream) {
  VP_TRY(check_attn_dims(dims));
  VP_TRY(check_counts(T, B));
  if (!rope) return VP_ERR_INVALID_ARG;
  if (rope->rot_dim < 0 || rope->rot_dim > dims->d || rope->rot_dim % 16) return VP_ERR_UNSUPPORTED_SHAPE;
  if (rope->rot_dim && !rope->turns) return VP_ERR_INVALID_ARG;
  if ((rope->interleaved != 0 && rope->interleaved != 1) || !isfinite(rope->scale))
    return VP_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(rope->turns) & 7u) return VP_ERR_ALIGNMENT;
  if (T == 0) return VP_OK;  // empty tensors have no address
  if (!cu || !q != !q_out) return VP_ERR_INVALID_ARG;
  if (!aligned4(cu) || !aligned4(kv_len) || !aligned4(positions)) return VP_ERR_ALIGNMENT;
  if (q) {
    VP_TRY(check_rows(q, q_stride, dims->Hq, dims->d));
    VP_TRY(check_rows(q_out, q_out_stride, dims->Hq, dims->d));
  }
  VP_TRY(check_rows(k, k_stride, dims->Hkv, dims->d));
  if (kv) {
    VP_TRY(check_kv(kv));
    VP_TRY(check_rows(v, v_stride, dims->Hkv, dims->d));
    if (!kv_len) return VP_ERR_INVALID_ARG;
  } else if (!k_out) {
    return VP_ERR_INVALID_ARG;
  }
  if (k_out) VP_TRY(check_rows(k_out, k_out_stride, dims->Hkv, dims->d));
  // In place: every token where it was.
  if ((q && q == q_out && q_stride != q_out_stride) || (k == k_out && k_stride != k_out_stride))
    return VP_ERR_INVALID_ARG;
  if (ws && ws_bytes < 256) return VP_ERR_WORKSPACE;
  if (!aligned16(ws)) return VP_ERR_ALIGNMENT;
  if (!device_is_sm103()) return VP_ERR_UNSUPPORTED_DEVICE;
  RopeAppendArgs a{};
  a.T = T;
  a.B = B;
  a.Hq = dims->Hq;
  a.Hkv = dims->Hkv;
  a.d = dims->d;
  a.fp16 = dims->dtype == VP_DTYPE_FP16;
  a.rot = rope->rot_dim;
  a.interleaved = rope->interleaved;
  a.scale = rope->scale;
  a.turns = rope->turns;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = kv ? static_cast<const uint16_t*>(v) : nullptr;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.cu = cu;
  a.kv_len = kv_len;
  a.positions = positions;
  a.kv = make_kv(kv);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_out = static_cast<uint16_t*>(k_out);
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.err = static_cast<unsigned int*>(ws);
  return from_cuda(launch_rope_append(a, device_sm_count(), static_cast<cudaStream_t>(stream)));
}

vp_status vp_prompt_attention(const vp_attn_dims* dims, int32_t T, int32_t B, const void* q,
                              int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                              int64_t v_stride, const int32_t* cu, void* out, int64_t out_stride,
                              float* lse, void* ws, size_t ws_bytes, void* stream) {
  VP_TRY(check_attn_dims(dims));
  VP_TRY(check_counts(T, B));
  if (T == 0) return VP_OK;
  if (!cu) return VP_ERR_INVALID_ARG;
  if (!aligned4(cu) || !aligned4(lse)) return VP_ERR_ALIGNMENT;
  VP_TRY(check_rows(q, q_stride, dims->Hq, dims->d));
  VP_TRY(check_rows(k, k_stride, dims->Hkv, dims->d));
  VP_TRY(check_rows(v, v_stride, dims->Hkv, dims->d));
  VP_TRY(check_rows(out, out_stride, dims->Hq, dims->d));
  if (!ws || ws_bytes < seq_scratch_bytes(dims->d)) return VP_ERR_WORKSPACE;
  if (!aligned16(ws)) return VP_ERR_ALIGNMENT;
  if (!device_is_sm103()) return VP_ERR_UNSUPPORTED_DEVICE;
  SeqAttnArgs a = make_args(dims, T, B, q, q_stride, cu, out, out_stride, lse, ws);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  return from_cuda(launch_seq_attention(a, carve_seq_scratch(ws, dims->d), device_sm_count(),
                                        static_cast<cudaStream_t>(stream)));
}

vp_status vp_paged_attention(const vp_attn_dims* dims, int32_t T, int32_t B, const void* q,
                             int64_t q_stride, const int32_t* cu, const int32_t* kv_len,
                             const vp_paged_kv* kv, void* out, int64_t out_stride, float* lse,
                             void* ws, size_t ws_bytes, void* stream) {
  VP_TRY(check_attn_dims(dims));
  VP_TRY(check_counts(T, B));
  if (T == 0) return VP_OK;
  if (!cu || !kv_len) return VP_ERR_INVALID_ARG;
  if (!aligned4(cu) || !aligned4(kv_len) || !aligned4(lse)) return VP_ERR_ALIGNMENT;
  VP_TRY(check_rows(q, q_stride, dims->Hq, dims->d));
  VP_TRY(check_rows(out, out_stride, dims->Hq, dims->d));
  VP_TRY(check_kv(kv));
  if (!ws || ws_bytes < seq_scratch_bytes(dims->d)) return VP_ERR_WORKSPACE;
  if (!aligned16(ws)) return VP_ERR_ALIGNMENT;
  if (!device_is_sm103()) return VP_ERR_UNSUPPORTED_DEVICE;
  SeqAttnArgs a = make_args(dims, T, B, q, q_stride, cu, out, out_stride, lse, ws);
  a.kv_len = kv_len;
  a.kv = make_kv(kv);
  return from_cuda(launch_seq_attention(a, carve_seq_scratch(ws, dims->d), device_sm_count(),
                                        static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
