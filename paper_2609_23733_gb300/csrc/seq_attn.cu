// Softmax attention of packed sequences, over themselves (vp_prompt_attention) or over the paged
// cache (vp_paged_attention): o = sum_j p_j v_j / sum_j p_j over the keys j < lim(i) that
// row (token i, head h) sees, p_j = 2^(s_j - m), s_j = scale log2(e) q . k_j, m the running maximum.
//
// One warp per row: a lane scores one of 32 keys, then all lanes accumulate the values of the 32,
// a few channels each.  In 32 bits throughout.
#include "common.cuh"
#include "seq.h"

namespace vp {

namespace {

constexpr int kRowWarps = 4;

template <int D, bool F16>
__global__ void __launch_bounds__(32 * kRowWarps) seq_attn_rows_kernel(SeqAttnArgs a) {
  __shared__ float s_q[kRowWarps][D];
  const int warp = warp_id(), lane = lane_id();
  const long long r = (long long)blockIdx.x * kRowWarps + warp;
  if (r >= (long long)a.T * a.Hq) return;
  const int t = (int)(r / a.Hq), h = (int)(r - (long long)t * a.Hq), hk = h / a.group;
  const int b = seq_of_token(a.cu, a.B, t);
  const Seq sq = load_seq(a, b);
  const int i = t - sq.q0;
  if (i < 0 || i >= sq.ql) return;
  const int lim = row_limit(i, sq.ql, sq.kl, a.block);
  for (int c = lane; c < D; c += 32) s_q[warp][c] = to_float<F16>(a.q[t * a.q_stride + h * D + c]);
  __syncwarp();
  float m = -INFINITY, l = 0.f, o[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) o[c] = 0.f;
  for (int j0 = 0; j0 < lim; j0 += 32) {
    const int j = j0 + lane;
    const bool seen = j < lim;
    long long ko = 0, vo = 0;  // offsets of the key's and the value's row
    bool held = seen;
    if (a.kv.k) {
      if (seen) {
        const int page = a.kv.table[(size_t)b * a.kv.width + (j >> a.kv.log2_page)];
        held = (unsigned)page < (unsigned)a.kv.n_pages;
        ko = (((((long long)page * a.Hkv + hk) << a.kv.log2_page)) + (j & (a.kv.page_size - 1))) * D;
        vo = ko;
        if (!held && a.err) atomicOr(a.err, VP_DEVERR_PAGE);
      }
    } else {
      ko = (long long)(sq.q0 + j) * a.k_stride + hk * D;
      vo = (long long)(sq.q0 + j) * a.v_stride + hk * D;
    }
    const uint16_t* kp = a.kv.k ? a.kv.k : a.k;
    const uint16_t* vp = a.kv.k ? a.kv.v : a.v;
    float s = -INFINITY;
    if (seen) {
      s = 0.f;
      if (held)
        for (int c = 0; c < D; ++c) s = fmaf(s_q[warp][c], to_float<F16>(kp[ko + c]), s);
      s *= a.scale_log2;
    }
    float mx = s;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
    mx = fmaxf(m, mx);
    const float alpha = exp2f(m - mx);
    m = mx;
    const float p = seen ? exp2f(s - m) : 0.f;
    float ps = p;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, k);
    l = l * alpha + ps;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[c] *= alpha;
    const int n = min(32, lim - j0);
    for (int k = 0; k < n; ++k) {
      const float pk = __shfl_sync(0xffffffffu, p, k);
      const long long vk = __shfl_sync(0xffffffffu, vo, k);
      if (!__shfl_sync(0xffffffffu, (int)held, k)) continue;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[c] = fmaf(pk, to_float<F16>(vp[vk + lane + 32 * c]), o[c]);
    }
  }
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const float y = lim > 0 ? o[c] / l : 0.f;
    a.out[t * a.out_stride + h * D + lane + 32 * c] = (uint16_t)pack2<F16>(y, 0.f);
  }
  if (a.lse && lane == 0)
    a.lse[(size_t)t * a.Hq + h] = lim > 0 ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

}  // namespace

cudaError_t launch_seq_attention(const SeqAttnArgs& a, int num_sms, cudaStream_t st) {
  const long long rows = (long long)a.T * a.Hq;
  const unsigned grid = (unsigned)((rows + kRowWarps - 1) / kRowWarps);
  prof_before(VP_KERNEL_SEQ_ATTN, st);
  if (a.d == 64) {
    if (a.fp16)
      seq_attn_rows_kernel<64, true><<<grid, 32 * kRowWarps, 0, st>>>(a);
    else
      seq_attn_rows_kernel<64, false><<<grid, 32 * kRowWarps, 0, st>>>(a);
  } else {
    if (a.fp16)
      seq_attn_rows_kernel<128, true><<<grid, 32 * kRowWarps, 0, st>>>(a);
    else
      seq_attn_rows_kernel<128, false><<<grid, 32 * kRowWarps, 0, st>>>(a);
  }
  prof_after(st);
  return cudaGetLastError();
}

}  // namespace vp
