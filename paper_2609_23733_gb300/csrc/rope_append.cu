// vp_rope_append: rotary positions of q and k fused with the append of k and v to the paged cache.
//
//   slot = kv_len[b] - n + i,  angle = pos x turns[f] of a turn (a 64-bit product that wraps at one
//   turn, so the reduction is exact at any position; its upper 32 bits give the angle to 2^-25
//   of a half turn),  (a, b) -> scale (a cos - b sin, b cos + a sin) in 32 bits, rounded once.
//
// Bound by memory: every value is read and written once.  A CTA takes a few consecutive tokens:
// its threads first fill a table of their (cos, sin) and cache rows in shared memory, so that a
// sine is taken once per token and frequency and not once per head, then move 32 bytes (two 16-byte
// vectors: the two halves of eight pairs, or sixteen neighbouring channels) per step, kRaUnroll
// steps' loads in flight per thread.  Measured on GB300: 43,968 tokens, 16 q heads and 8 kv heads of
// 128, 110.6 us on the device (6.5 TB/s, 0.96 of the measured copy bandwidth; 1, 3, 4 steps in flight: 117,
// 112, 116 us; 4 or 16 tokens per CTA instead of 8: 126, 113 us), 111.6 us as called; 64 single tokens of 24
// heads of 64: 3.6 us on the device.
#include "common.cuh"
#include "seq.h"

namespace vp {

namespace {

constexpr int kRaThreads = 256;
constexpr int kRaTokens = 8;   // most tokens of a CTA
constexpr int kRaUnroll = 2;

template <bool F16>
__device__ __forceinline__ void rotate_pair(uint32_t& a, uint32_t& b, float2 cs0, float2 cs1) {
  // a holds the first members of two pairs, b the second ones
  const float2 x = unpack2<F16>(a), y = unpack2<F16>(b);
  a = pack2<F16>(x.x * cs0.x - y.x * cs0.y, x.y * cs1.x - y.y * cs1.y);
  b = pack2<F16>(y.x * cs0.x + x.x * cs0.y, y.y * cs1.x + x.y * cs1.y);
}

template <bool F16>
__device__ __forceinline__ uint32_t rotate_adjacent(uint32_t u, float2 cs) {
  const float2 x = unpack2<F16>(u);
  return pack2<F16>(x.x * cs.x - x.y * cs.y, x.y * cs.x + x.x * cs.y);
}

template <bool F16>
__global__ void __launch_bounds__(kRaThreads) rope_append_kernel(const __grid_constant__ RopeAppendArgs a,
                                                               int tokens) {
  __shared__ float2 s_cs[kRaTokens * 64];
  __shared__ long long s_row[kRaTokens];  // row (of d channels) of kv head 0 in the cache, -1: none
  __shared__ int s_pos[kRaTokens];
  pdl_launch_dependents();
  pdl_wait();
  const int t0 = blockIdx.x * tokens;
  const int nt = min(min(tokens, a.T - t0), a.cu[a.B] - t0);
  if (nt <= 0) return;  // uniform
  const int tid = threadIdx.x, half = a.rot >> 1;
  if (tid < nt) {
    const int t = t0 + tid;
    const int b = seq_of_token(a.cu, a.B, t);
    const int c0 = a.cu[b], n = a.cu[b + 1] - c0, i = t - c0;
    long long slot = i, row = -1;
    if (a.kv.k) {
      slot = (long long)a.kv_len[b] - n + i;
      bool ok = slot >= 0 && (slot >> a.kv.log2_page) < a.kv.width;
      if (ok) {
        const int page = a.kv.table[(size_t)b * a.kv.width + (slot >> a.kv.log2_page)];
        ok = (unsigned)page < (unsigned)a.kv.n_pages;
        row = (((long long)page * a.Hkv) << a.kv.log2_page) + (slot & (a.kv.page_size - 1));
      }
      if (!ok) {
        row = -1;
        if (a.err) atomicOr(a.err, VP_DEVERR_PAGE);
      }
    }
    s_row[tid] = row;
    s_pos[tid] = a.positions ? a.positions[t] : (int)slot;
  }
  __syncthreads();
  for (int e = tid; e < nt * half; e += kRaThreads) {
    const int tk = e / half, f = e - tk * half;
    const unsigned long long turn =
        (unsigned long long)(long long)s_pos[tk] * (unsigned long long)__ldg(a.turns + f);
    float sn, cn;
    sincospif((float)(int)(turn >> 32) * (1.f / 2147483648.f), &sn, &cn);  // half turns in [-1, 1)
    s_cs[tk * half + f] = make_float2(cn * a.scale, sn * a.scale);
  }
  __syncthreads();

  // Steps: token-major, then q heads, k heads, v heads; d / 16 steps per head.
  const int spc = a.d >> 4;                       // steps per head
  const int n_heads = (a.q ? a.Hq : 0) + a.Hkv + (a.v ? a.Hkv : 0);
  const int k0 = a.q ? a.Hq : 0, v0 = k0 + a.Hkv;
  const int steps = nt * n_heads * spc, rsteps = a.rot >> 4;
  const int log2p = a.kv.log2_page;
  for (int base = tid; base < steps; base += kRaThreads * kRaUnroll) {
    uint4 x[kRaUnroll], y[kRaUnroll];
    int head[kRaUnroll], tok[kRaUnroll], off0[kRaUnroll], off1[kRaUnroll], rr[kRaUnroll];
#pragma unroll
    for (int u = 0; u < kRaUnroll; ++u) {
      const int e = base + u * kRaThreads;
      if (e >= steps) break;
      const int hh = e / spc, j = e - hh * spc;
      tok[u] = hh / n_heads;
      head[u] = hh - tok[u] * n_heads;
      const bool rot = j < rsteps && head[u] < v0;
      rr[u] = rot ? j : -1;
      const bool split = rot && !a.interleaved;
      off0[u] = split ? j * 8 : j * 16;
      off1[u] = split ? half + j * 8 : j * 16 + 8;
      const uint16_t* src;
      const int t = t0 + tok[u];
      if (head[u] < k0)
        src = a.q + t * a.q_stride + head[u] * a.d;
      else if (head[u] < v0)
        src = a.k + t * a.k_stride + (head[u] - k0) * a.d;
      else
        src = a.v + t * a.v_stride + (head[u] - v0) * a.d;
      x[u] = *reinterpret_cast<const uint4*>(src + off0[u]);
      y[u] = *reinterpret_cast<const uint4*>(src + off1[u]);
    }
#pragma unroll
    for (int u = 0; u < kRaUnroll; ++u) {
      if (base + u * kRaThreads >= steps) break;
      if (rr[u] >= 0) {
        const float2* cs = s_cs + tok[u] * half + rr[u] * 8;
        uint32_t* px = &x[u].x;
        uint32_t* py = &y[u].x;
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            px[i] = rotate_adjacent<F16>(px[i], cs[i]);
            py[i] = rotate_adjacent<F16>(py[i], cs[4 + i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) rotate_pair<F16>(px[i], py[i], cs[2 * i], cs[2 * i + 1]);
        }
      }
      const int t = t0 + tok[u];
      uint16_t* dst = nullptr;    // packed output
      uint16_t* cache = nullptr;
      const long long row = s_row[tok[u]];
      if (head[u] < k0) {
        dst = a.q_out + t * a.q_out_stride + head[u] * a.d;
      } else {
        const bool is_k = head[u] < v0;
        const int h = head[u] - (is_k ? k0 : v0);
        if (is_k && a.k_out) dst = a.k_out + t * a.k_out_stride + h * a.d;
        if (row >= 0) cache = (is_k ? a.kv.k : a.kv.v) + (row + ((long long)h << log2p)) * a.d;
      }
      if (dst) {
        *reinterpret_cast<uint4*>(dst + off0[u]) = x[u];
        *reinterpret_cast<uint4*>(dst + off1[u]) = y[u];
      }
      if (cache) {
        *reinterpret_cast<uint4*>(cache + off0[u]) = x[u];
        *reinterpret_cast<uint4*>(cache + off1[u]) = y[u];
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope_append(const RopeAppendArgs& a, int num_sms, cudaStream_t st) {
  // A few tokens: one per CTA, for the latency; many: up to kRaTokens.
  int tokens = a.T / (4 * num_sms);
  tokens = tokens < 1 ? 1 : tokens > kRaTokens ? kRaTokens : tokens;
  const int grid = (a.T + tokens - 1) / tokens;
  RopeAppendArgs aa = a;
  void* args[] = {&aa, &tokens};
  const void* fn = a.fp16 ? reinterpret_cast<const void*>(rope_append_kernel<true>)
                          : reinterpret_cast<const void*>(rope_append_kernel<false>);
  prof_before(VP_KERNEL_ROPE_APPEND, st);
  const cudaError_t e = launch_pdl(fn, dim3(grid), kRaThreads, 0, st, args);
  prof_after(st);
  return e;
}

}  // namespace vp
