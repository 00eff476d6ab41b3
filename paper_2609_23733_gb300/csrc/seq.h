// Streaming operators (rotary append, prompt attention, attention over the paged cache):
// launch arguments and device helpers shared by their kernels (not part of the ABI).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include "common.cuh"
#include "internal.h"

namespace vp {

// The paged cache (vp_paged_kv, vp_paged_kv8) as the kernels see it.
struct PagedKv {
  uint16_t* k;
  uint16_t* v;
  const int32_t* table;
  int32_t n_pages, page_size, log2_page, width;
  uint8_t* k8;  // 8-bit cache: codes and scales (k and v are then NULL); else NULL
  uint8_t* v8;
  uint8_t* k_scale;
  uint8_t* v_scale;
  // Whether there is a cache, by what both kinds have (by k or k8: 12 mixed chunks in 16 bits 130.8 against 129.4 us).
  __host__ __device__ bool any() const { return table != nullptr; }
};

struct RopeAppendArgs {
  int T, B, Hq, Hkv, d, fp16;
  int rot, interleaved;
  float scale;
  const int64_t* turns;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t* cu;
  const int32_t* kv_len;     // NULL: no cache
  const int32_t* positions;  // NULL: the slot
  PagedKv kv;                // kv.k NULL: no cache
  uint16_t* q_out;
  uint16_t* k_out;
  int64_t q_out_stride, k_out_stride;
  unsigned int* err;         // NULL: not recorded
};
cudaError_t launch_rope_append(const RopeAppendArgs& a, int num_sms, cudaStream_t st);

constexpr int kMaxAxes = 4;
struct NormAppendArgs {
  int T, B, Hq, Hkv, d, fp16;
  int rot, pair_block, n_axes;
  float scale;
  const int64_t* turns;
  int q_kind, k_kind;
  float eps;
  int per_head;
  const float* q_g;          // NULL: 1
  const float* q_b;          // NULL: 0
  const float* k_g;
  const float* k_b;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t* cu;
  const int32_t* kv_len;     // NULL: no cache
  const int32_t* positions;  // [T][n_axes]; NULL: the slot
  PagedKv kv;
  uint16_t* q_out;
  uint16_t* k_out;
  int64_t q_out_stride, k_out_stride;
  unsigned int* err;         // NULL: not recorded
};
cudaError_t launch_norm_append(const NormAppendArgs& a, int num_sms, cudaStream_t st);

struct ReadCacheArgs {
  int T, B, Hkv, d, fp16;
  PagedKv kv;
  const int32_t* cu;
  const int32_t* first;      // NULL: 0
  uint16_t* k_out;           // either may be NULL
  uint16_t* v_out;
  int64_t k_out_stride, v_out_stride;
  unsigned int* err;         // NULL: not recorded
};
cudaError_t launch_read_cache(const ReadCacheArgs& a, int num_sms, cudaStream_t st);

// Division of 0 <= n < 2^31 by a number the host knows, as a multiplication (round-up method: with s =
// ceil(log2 d) and mul = ceil(2^(31 + s) / d) < 2^32, floor(n mul / 2^(31 + s)) = floor(n / d) for all
// such n, since mul d - 2^(31 + s) < d <= 2^s).
struct FastDiv {
  uint32_t mul = 0, shift = 0;  // mul 0: d = 1
  FastDiv() = default;
  explicit FastDiv(uint32_t d) {
    if (d <= 1) return;
    while ((1u << shift) < d && shift < 31) ++shift;  // d <= 2^31
    mul = (uint32_t)(((1ull << (31 + shift)) + d - 1) / d);
    --shift;  // the product's upper word is shifted by 31 + s - 32
  }
  __device__ __forceinline__ int operator()(int n) const {
    return mul ? (int)(__umulhi((uint32_t)n, mul) >> shift) : n;
  }
};

struct SeqAttnArgs {
  int T, B, Hq, Hkv, group, d, fp16;
  int block;
  int chain_tokens;          // tokens of a chain (128 / group rows each)
  int block_chains;          // > 0: chains start anew at every mask block, this many per block
  FastDiv by_group, by_block, by_chain_tokens, by_block_chains;
  float scale_log2;          // scale x log2(e)
  float far_from, far_scale, far_unit;  // the tile kernel's scores past kFarScore (see there)
  const uint16_t* q;
  int64_t q_stride;
  const uint16_t* k;         // prompts: packed keys and values; paged: NULL (in kv)
  const uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* cu;
  const int32_t* kv_len;     // paged only
  PagedKv kv;                // neither kv.k nor kv.k8: prompts
  uint16_t* out;
  int64_t out_stride;
  float* lse;                // [T][Hq] or NULL
  unsigned int* err;
};

// Attention's scratch inside the caller's workspace, after the error word.
struct SeqScratch {
  int4* recs;       // [CTAs][2] items cut between CTAs: {parts (0: none), kv head, first chain or
                    // row tile, sequence}, {q0, ql, kl, first part's slot}; part i > 0 lies in slot
                    // 2 (cta + i)
  float* part_o;    // partial outputs, unnormalised: [slot][kSmallRows][d], or, of the tile kernel (written
                    // row by row in parallel), [slot][chain][d / 4][128 rows][4]
  float2* part_ml;  // [slot][rows] (m, l)
};
constexpr int kMaxCtas = 160;            // CTAs of the tile kernel, at most (one per SM)
constexpr int kMaxSlots = 2 * kMaxCtas;  // a CTA's run has at most two items in part
// Chains of 128 query rows of an item of the tile kernel.
__host__ __device__ constexpr int seq_chains(int d) { return d == 64 ? 3 : 2; }
size_t seq_scratch_bytes(int d);
SeqScratch carve_seq_scratch(void* ws, int d);

// Few rows per sequence (seq_rows.cu): items of kSmallRows rows.
constexpr int kSmallRows = 16;
__host__ __device__ constexpr int small_rows_ctas_per_sm(int d) { return d == 64 ? 3 : 2; }
// Over the 8-bit cache, by an item's rows.
__host__ __device__ constexpr int rows8_ctas_per_sm(int d, int rows) {
  return rows == 8 ? (d == 64 ? 4 : 3) : small_rows_ctas_per_sm(d);
}
constexpr int kMaxRecs = 4 * kMaxCtas;   // CTAs of any of the kernels, at most
// Most keys of a sequence, as far as the host knows.
inline long long most_keys(const SeqAttnArgs& a) {
  return a.kv.any() ? (long long)a.kv.width << a.kv.log2_page : a.T;
}
// Items of `rows` rows (token x head of a kv head's group), for sequences of about the mean length.
inline long long count_items(const SeqAttnArgs& a, int rows) {
  const long long n = (a.T + a.B - 1) / a.B;
  return (long long)a.B * a.Hkv * ((n * a.group + rows - 1) / rows);
}
// Short items of 16 rows are not cut between CTAs, which saves the join: all of at most 256 keys, and
// of 512 if there are enough of them for the SMs (us, cut / whole; heads of 64, 4 kv heads,
// single tokens: 8 x 256: 7.3 / 6.2; 64 x 512: 11.6 / 9.2; 1 x 512: 6.6 / 7.4; 8 x 1,024: 8.2 / 11.8).
inline bool rows_whole(const SeqAttnArgs& a, int ctas) {
  const long long keys = most_keys(a);
  return keys <= 256 || (keys <= 512 && 2 * count_items(a, kSmallRows) >= ctas);
}
static_assert(2 * kMaxRecs * kSmallRows <= kMaxSlots * 2 * 128, "its parts fit the scratch");
cudaError_t launch_seq_rows(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st);
// The same over the 8-bit cache (seq_rows8.cu): items of 8 or 16 rows.
cudaError_t launch_seq_rows8(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st);

// Joins the items cut between the `ctas` CTAs of the kernel ahead (seq_join.cu): of `rows` rows each, or the
// tile kernel's (rows 0).
cudaError_t launch_seq_join(const SeqAttnArgs& a, const SeqScratch& sc, int rows, int ctas, cudaStream_t st);

// Where keys and values are: packed rows, 16-bit pages, 8-bit pages.
enum class Keys { packed, paged, paged8 };

// Tensor maps of the keys and values, boxes of 64 channels x min(page, tile_keys) keys.
cudaError_t make_kv_maps(const SeqAttnArgs& a, int tile_keys, CUtensorMap* mk, CUtensorMap* mv);
// The same of 8-bit pages: boxes of a row's d codes x min(page, tile_keys) keys, d-byte swizzle.
cudaError_t make_kv8_maps(const SeqAttnArgs& a, int tile_keys, CUtensorMap* mk, CUtensorMap* mv);
// A launch whose kernel may start before the one ahead of it in the stream has ended.
cudaError_t launch_pdl(const void* fn, dim3 grid, int threads, int smem, cudaStream_t st, void** args);

cudaError_t launch_seq_attention(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms,
                                 cudaStream_t st);

// 4-D tensor map of 16-bit values with a 64-element (128-byte) inner box, 128-byte swizzle, zero
// fill out of bounds; strides in elements (dims 1..3).
cudaError_t make_tmap_16bit_4d(CUtensorMap* map, const void* base, bool fp16,
                               const uint64_t dims[4], const uint64_t strides[3],
                               const uint32_t box[4]);

// 4-D tensor map of bytes, zero fill out of bounds; strides in bytes; swizzle 64 or 128 bytes, the box's
// inner extent.
cudaError_t make_tmap_8bit_4d(CUtensorMap* map, const void* base, const uint64_t dims[4],
                              const uint64_t strides[3], const uint32_t box[4]);

// The tile kernel takes 2^(s cs - m) in one fused multiply and add, whose product is exact while m has 24
// bits.  What m's rounding leaves is common to all of a row's weights, and far out it would make all of
// them 0 or infinite (a unit in m's last place is 64 at 2^29).  Where a tile's largest score is past
// kFarScore, s far_scale is taken instead, far_scale the power of two from cs up: a product with 24 bits, so
// m = mx far_scale is exact.  Two different scores lie at least 16 apart there, so a weight w < 1 is below
// 2^-16 and comes out between w^2 and w.  The log-sum is put back into units of cs.
constexpr float kFarScore = 1 << 28;
// Of the tile kernel's |cs|, so that a hidden score, -inf, stays -inf; the least there is, since scores (of bf16) may be
// as large as cs is small.
constexpr float kLeastScale = FLT_TRUE_MIN;
// m in units of cs: a near tile's m is below kFarScore (far_from is a little below kFarScore / cs), a far
// one's that is below it too has far_unit = 1 to 2^-19.
__device__ __forceinline__ float near_units(const SeqAttnArgs& a, float m) {
  return fabsf(m) < kFarScore ? m : m * a.far_unit;
}

// One sequence: its new tokens [q0, q0 + ql) among the T packed ones, and the keys [0, kl).
struct Seq {
  int q0, ql, kl;
};

// Sequence b, clamped so that nothing outside the T tokens or the page table is touched.
__device__ __forceinline__ Seq load_seq(const SeqAttnArgs& a, int b) {
  Seq s;
  const int c0 = a.cu[b], c1 = a.cu[b + 1];
  s.q0 = min(max(c0, 0), a.T);
  s.ql = min(max(c1, s.q0), a.T) - s.q0;
  if (a.kv.any()) {
    const long long cap = min((long long)a.kv.width << a.kv.log2_page, 1ll << 30);
    const int n = a.kv_len[b];
    s.kl = (int)min((long long)max(n, 0), cap);
    if (s.kl != n && a.err) atomicOr(a.err, VP_DEVERR_PAGE);
  } else {
    s.kl = s.ql;
  }
  return s;
}

// Weights are 2^(score - m); m for a running maximum x (in log2 units: x = mx cs).  bf16: x.  fp16: 2^7
// below it, since its smallest normal number is 2^-14 and a weight below 2^-24 of the largest would be
// lost, and those of many keys beside one heavy one add up; with 2^8 for a maximum not yet moved, none
// passes 2^15.  Rounded up there: 2^(s cs - m) by a fused multiply and add keeps what m's rounding cut
// off, a factor common to the row's weights, which then only lowers them (2^-16 at most, see kFarScore) and
// cannot make them overflow.
template <bool F16>
__device__ __forceinline__ float reference_point(float mx, float cs) {
  return F16 ? __fmaf_ru(mx, cs, -7.f) : mx * cs;
}

// Keys [0, lim) are visible to new token i (0 <= i < ql).  lim <= 0: none.
__device__ __forceinline__ int row_limit(const SeqAttnArgs& a, int i, int ql, int kl) {
  if (a.block == 0) return kl;
  if (a.block == 1) return kl - ql + i + 1;
  const int rest = ql - i, step = a.block - (i - a.by_block(i) * a.block);  // both at least 1
  return kl - ql + i + min(rest, step);
}

// The new tokens of a sequence in chains of up to chain_tokens.  Where that wastes little, chains
// do not run across mask blocks, so that all rows of a chain see the same keys.
__device__ __forceinline__ int count_chains(const SeqAttnArgs& a, int ql) {
  const int n = a.chain_tokens;
  if (a.block_chains == 0) return a.by_chain_tokens(ql + n - 1);  // ql <= 2^30
  const int full = a.by_block(ql);
  return full * a.block_chains + a.by_chain_tokens(ql - full * a.block + n - 1);
}
__device__ __forceinline__ int chain_start(const SeqAttnArgs& a, int chain) {
  if (a.block_chains == 0) return chain * a.chain_tokens;
  const int full = a.by_block_chains(chain);
  return full * a.block + (chain - full * a.block_chains) * a.chain_tokens;
}
// One past the chain's last token.
__device__ __forceinline__ int chain_end(const SeqAttnArgs& a, int chain, int ql) {
  if (a.block_chains == 0) return min((chain + 1) * a.chain_tokens, ql);
  const int full = a.by_block_chains(chain);
  const int start = full * a.block + (chain - full * a.block_chains) * a.chain_tokens;
  return min(min(start + a.chain_tokens, (full + 1) * a.block), ql);
}

// The last sequence b < B with cu[b] <= t (0 if there is none): the owner of token t where cu
// is ascending; always a valid index.
__device__ __forceinline__ int seq_of_token(const int32_t* cu, int B, int t) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= t)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// 16-bit storage types.
template <bool F16>
__device__ __forceinline__ float to_float(uint16_t u) {
  if constexpr (F16)
    return __half2float(__ushort_as_half(u));
  else
    return __uint_as_float((uint32_t)u << 16);
}
template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t u) {
  if constexpr (F16) {
    __half2 h = *reinterpret_cast<__half2*>(&u);
    return __half22float2(h);
  } else {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
  }
}
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (F16) {
    __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
  } else {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
  }
}

// ------------------------------------------------------------------ 8-bit cache
// A row is e4m3 codes and a scale 2^e, e in [kLeastScaleExp, kMostScaleExp], as the byte e + 127.  The range
// makes 2^e a normal fp16 number and every value code x 2^e (2^-23 .. 57,344) an fp16 and a bf16 number, so
// that a product in fp16 gives it exactly.
constexpr int kLeastScaleExp = -14, kMostScaleExp = 7;
constexpr uint32_t kLeastScaleByte = 127 + kLeastScaleExp, kMostScaleByte = 127 + kMostScaleExp;
constexpr uint32_t kBadScaleByte = 255;

__device__ __forceinline__ bool bad_scale(uint32_t byte) {
  return byte - kLeastScaleByte > kMostScaleByte - kLeastScaleByte;
}
// 2^e as fp16 bits; NaN for a byte that stands for none.
__device__ __forceinline__ uint32_t scale_half(uint32_t byte) {
  return bad_scale(byte) ? 0x7E00u : (byte - kLeastScaleByte + 1) << 10;
}
// The fp16 pairs of codes 0, 1 and of codes 2, 3 of u (NaN for a code 0x7F or 0xFF).
__device__ __forceinline__ void codes_to_half(uint32_t u, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(u));
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Codes of four values, rounded to the nearest (ties to even), at most 448 in magnitude.
__device__ __forceinline__ uint32_t to_codes(float x0, float x1, float x2, float x3) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
      "mov.b32 %0, {a, b};\n\t}"
      : "=r"(r)
      : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
  return r;
}

// A bf16 row of Q as fp16, the type of the products over the 8-bit cache: times a power of two that brings
// its largest value to 2^14 .. 2^15, so that what lies within 2^-31 of it keeps its 8 bits, and the rest is at
// most 2^-39 of it off (a score by 2^-39 max |q| sum |k|, where its 32-bit sum may be 2^-24 sum |q k| off).
// top: the largest magnitude as fp32 bits; an infinity or a NaN stays one.
struct HalfRow {
  float up, back;  // scores are multiplied by `back`
  __device__ __forceinline__ explicit HalfRow(uint32_t top) {
    const uint32_t e = min(127u + 141u - (top >> 23), 253u);
    up = __uint_as_float(e << 23);
    back = __uint_as_float((254u - e) << 23);
  }
  __device__ __forceinline__ uint32_t convert(uint32_t u) const {
    const float2 f = unpack2<false>(u);
    return pack2<true>(f.x * up, f.y * up);
  }
};

__device__ __forceinline__ void tma_load_4d(void* smem_dst, const void* tmap, uint64_t* bar, int x,
                                            int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(smem_dst)),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}

// Copies `bytes` (a multiple of 16; both addresses too) and counts them at bar.
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(smem_dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

__device__ __forceinline__ void pdl_launch_dependents() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Whether a pair of 16-bit values holds an infinity or a NaN (all exponent bits set): adding one
// to the exponent field carries into the sign place exactly then.
template <bool F16>
__device__ __forceinline__ bool nonfinite2(uint32_t u) {
  if constexpr (F16)
    return (((u & 0x7C007C00u) + 0x04000400u) & 0x80008000u) != 0;
  else
    return (((u & 0x7F807F80u) + 0x00800080u) & 0x80008000u) != 0;
}
// The pair with its infinities and NaNs replaced by 0.
template <bool F16>
__device__ __forceinline__ uint32_t finite2(uint32_t u) {
  const uint32_t t = F16 ? (((u & 0x7C007C00u) + 0x04000400u) & 0x80008000u)
                         : (((u & 0x7F807F80u) + 0x00800080u) & 0x80008000u);
  if (t & 0x8000u) u &= 0xFFFF0000u;
  if (t & 0x80000000u) u &= 0x0000FFFFu;
  return u;
}

}  // namespace vp
