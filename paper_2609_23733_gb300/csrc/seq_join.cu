// Joins the parts of items cut between the CTAs of the attention kernels (seq_attn.cu, seq_rows.cu):
// per row, with parts (m_i, l_i, o_i), m = max m_i, l = sum 2^(m_i - m) l_i, o = sum 2^(m_i - m) o_i / l,
// always in the parts' order, so that results do not depend on timing.
//
// Launched as a programmatic dependent of the kernel ahead, so that its CTAs are in place when that
// ends; a CTA whose entry of the list is empty returns at once.  D / 4 threads per row, 16
// bytes each; the kernel for few rows may cut an item hundreds of times (one sequence, one kv
// head), so there kSub groups of threads share a row's parts.
#include <float.h>
#include <math.h>

#include "seq.h"

namespace vp {

namespace {

constexpr int kThreads = 256;
constexpr float kUnset = -FLT_MAX;

template <int D, bool F16, bool kTiles>
__global__ void __launch_bounds__(kThreads)
    seq_join_kernel(const __grid_constant__ SeqAttnArgs a, const SeqScratch sc) {
  constexpr int kAtOnce = 4;
  constexpr int kLanes = D / 4, kSub = kTiles ? 1 : 256 / D;
  constexpr int kRowsCta = kThreads / (kLanes * kSub);       // rows of a CTA at a time
  constexpr int kRows = kTiles ? seq_chains(D) * 128 : kSmallRows;  // rows of a slot
  __shared__ __align__(16) float s_o[kTiles ? 1 : kThreads][4];
  __shared__ __align__(16) uint2 s_out[kTiles ? kRowsCta : 1][kLanes + 1];  // rows of outputs, padded
  __shared__ uint16_t* s_dst[kTiles ? kRowsCta : 1];                        // where they go
  __shared__ __align__(8) float2 s_ml[kTiles ? 1 : kThreads];
  pdl_launch_dependents();
  pdl_wait();
  const int cta = blockIdx.x;
  const int4 x = sc.recs[2 * cta], y = sc.recs[2 * cta + 1];
  const int np = x.x;
  if (np == 0) return;
  // Threads of a row: kSub groups of D / 4.  The tile kernel's parts have a row's neighbours side by
  // side, the other's its channels.
  const int tid = threadIdx.x;
  const int c = (kTiles ? tid / kRowsCta : tid % kLanes) * 4, sub = kTiles ? 0 : tid / kLanes % kSub;
  auto slot = [&](int i) { return (size_t)(i == 0 ? y.w : 2 * (cta + i)); };
  for (int base = blockIdx.y * kRowsCta; base < kRows; base += gridDim.y * kRowsCta) {
    const int r = base + (kTiles ? tid % kRowsCta : tid / (kLanes * kSub));
    int tok, sub_head;
    bool valid;
    if (kTiles) {  // chain, row of the chain
      const int chain = x.z + r / 128, row = r % 128, t = a.by_group(row);
      valid = chain < count_chains(a, y.y) && t < a.chain_tokens;
      tok = (valid ? chain_start(a, chain) : 0) + t;
      sub_head = row - t * a.group;
      valid = valid && tok < chain_end(a, chain, y.y);
    } else {
      const int row = x.z * kSmallRows + r;
      tok = a.by_group(row);
      sub_head = row - tok * a.group;
      valid = tok < y.y;
    }
    float m = kUnset, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    if (valid) {
      // kAtOnce parts' loads in flight, then joined to what there is.
      for (int i0 = sub; i0 < np; i0 += kAtOnce * kSub) {
        float2 ml[kAtOnce];
        float4 v[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const int i = i0 + k * kSub;
          ml[k] = make_float2(kUnset, 0.f);
          v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (i < np) {
            const size_t row = slot(i) * kRows + r;
            ml[k] = sc.part_ml[row];
            v[k] = *reinterpret_cast<const float4*>(
                sc.part_o +
                (kTiles ? ((slot(i) * (kRows / 128) + r / 128) * (D / 4) + c / 4) * 512 + (r % 128) * 4
                        : row * D + c));
          }
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, ml[k].x);
        const float f0 = fast_exp2(m - top);
        m = top;
        l *= f0;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] *= f0;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          const float f = fast_exp2(ml[k].x - top);
          l = fmaf(f, ml[k].y, l);
          o[0] = fmaf(f, v[k].x, o[0]);
          o[1] = fmaf(f, v[k].y, o[1]);
          o[2] = fmaf(f, v[k].z, o[2]);
          o[3] = fmaf(f, v[k].w, o[3]);
        }
      }
    }
    if (kSub > 1) {
      __syncthreads();
      *reinterpret_cast<float4*>(s_o[tid]) = make_float4(o[0], o[1], o[2], o[3]);
      s_ml[tid] = make_float2(m, l);
      __syncthreads();
      if (sub == 0) {
        const float mine = m;
        float top = m;
#pragma unroll
        for (int k = 1; k < kSub; ++k) top = fmaxf(top, s_ml[tid + k * kLanes].x);
        m = top;
        const float f0 = fast_exp2(mine - top);
        l *= f0;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= f0;
#pragma unroll
        for (int k = 1; k < kSub; ++k) {
          const float2 ml = s_ml[tid + k * kLanes];
          const float f = fast_exp2(ml.x - top);
          l = fmaf(f, ml.y, l);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = fmaf(f, s_o[tid + k * kLanes][i], o[i]);
        }
      }
    }
    const int lim = valid ? row_limit(a, tok, y.y, y.z) : 0, head = x.y * a.group + sub_head;
    const float inv = 1.f / l;
    const uint2 packed = lim > 0 ? make_uint2(pack2<F16>(o[0] * inv, o[1] * inv),
                                              pack2<F16>(o[2] * inv, o[3] * inv))
                                 : make_uint2(0u, 0u);
    uint16_t* dst = a.out + (int64_t)(y.x + tok) * a.out_stride + head * D;
    if (valid && sub == 0 && c == 0 && a.lse)
      a.lse[(size_t)(y.x + tok) * a.Hq + head] =
          lim > 0 ? ((kTiles ? near_units(a, m) : m) + log2f(l)) * 0.69314718055994531f : -INFINITY;
    if (kTiles) {  // rows written whole, by neighbouring threads
      if (base != (int)blockIdx.y * kRowsCta) __syncthreads();
      s_out[tid % kRowsCta][tid / kRowsCta] = packed;
      if (c == 0) s_dst[tid % kRowsCta] = valid ? dst : nullptr;
      __syncthreads();
      uint16_t* to = s_dst[tid / kLanes];
      if (to) *reinterpret_cast<uint2*>(to + (tid % kLanes) * 4) = s_out[tid / kLanes][tid % kLanes];
    } else if (valid && sub == 0) {
      *reinterpret_cast<uint2*>(dst + c) = packed;
    }
  }
}

}  // namespace

cudaError_t launch_seq_join(const SeqAttnArgs& a, const SeqScratch& sc, bool tiles, int ctas,
                            cudaStream_t st) {
  static const void* table[2][2][2] = {
      {{reinterpret_cast<const void*>(seq_join_kernel<64, false, false>),
        reinterpret_cast<const void*>(seq_join_kernel<64, false, true>)},
       {reinterpret_cast<const void*>(seq_join_kernel<64, true, false>),
        reinterpret_cast<const void*>(seq_join_kernel<64, true, true>)}},
      {{reinterpret_cast<const void*>(seq_join_kernel<128, false, false>),
        reinterpret_cast<const void*>(seq_join_kernel<128, false, true>)},
       {reinterpret_cast<const void*>(seq_join_kernel<128, true, false>),
        reinterpret_cast<const void*>(seq_join_kernel<128, true, true>)}}};
  SeqAttnArgs aa = a;
  SeqScratch ss = sc;
  void* args[] = {&aa, &ss};
  prof_extra_launch();
  return launch_pdl(table[a.d == 128][a.fp16 != 0][tiles], dim3(ctas, tiles ? 12 : 4), kThreads, 0, st, args);
}

}  // namespace vp
