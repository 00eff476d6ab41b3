// Attention of few query rows per sequence over the 8-bit paged cache: o = sum_j p_j v_j / sum_j p_j over
// the keys j < lim(i) that row (token i, head h) sees, k_j and v_j being codes times 2^e.
//
// Bound by memory like the kernel for 16-bit keys (seq_rows.cu), with half the bytes and the codes to
// unpack, so instructions count.  mma.sync m16n8k16 takes the keys as its M and the rows as its N, which
// are 8 (single tokens of grouped heads) or 16: with the rows as M, 8 rows would waste half of all
// products, exponentials and registers.
//   S^T = K Q^T    a lane's four bytes of a row of codes are the k indices of one operand, once Q's
//                  channels lie the same way; the scores are multiplied by the keys' scales.
//   O^T += V^T P^T  transposed by ldmatrix, a lane has two neighbouring channels of two neighbouring keys:
//                  even channels are rows 0-7 of the operand, odd ones rows 8-15; each value is code x 2^e,
//                  exact in fp16.  P^T comes from S^T by movmatrix.
// Products are of fp16 for both types: bf16 rows of Q are brought into its range (HalfRow), and P has 11 bits.
// The work is cut as seq_rows.cuh says, in units of kRows rows and 128 keys.
//   warp 4      TMA: codes of K and V page by page through a ring, and their scales (16 bytes and more of
//               a page) by bulk copies; page ids read 32 ahead.
//   warps 0-3   32 keys of every tile each, with a running maximum of their own (moved when it grows by more
//               than 2^8); the four warps' results are joined at the end of an item.
// Measured on GB300: 4 single tokens over 130,003 to 137,400 keys, 32 heads of 128 on 4 kv heads, pages of 16: 93.3 us as
// called (5.9 TB/s, 0.88 of the measured copy bandwidth; 127 us with the rows as M); 64 tokens over 97 to 16,381
// keys, 16 heads of 64 on 4: 27.7 us (40.6 with the rows as M; the first 2.6 us find the place, the last 4 join the
// parts; the units in between run at 0.8 of the copy bandwidth, a warp's chain of steps in the way: 4 CTAs of 96
// registers an SM).
// Keys that some row does not see: scores become -inf by selection; V codes that stand for NaN are taken out
// of the tile (0 x NaN would reach all rows) and added to the rows that see them.
#include "seq_rows.cuh"

namespace vp {

namespace {

constexpr int kBN = 128;  // keys of a unit
static_assert(kBN == 32 * kWarps, "a scale per lane");

template <int D, int kRows>
struct Rows8Cfg {
  static constexpr int kStages = D == 64 ? 3 : 2;
  static constexpr int kJoin = D == 64 && kRows == 8 ? 32 : 64;  // channels of O joined at a time
  static constexpr int kPerSm = rows8_ctas_per_sm(D, kRows);
};

template <int D, int kRows>
struct Rows8Smem {
  using C = Rows8Cfg<D, kRows>;
  uint8_t k[C::kStages][kBN * D];  // rows of codes, D-byte swizzle
  uint8_t v[C::kStages][kBN * D];
  uint8_t k_scale[C::kStages][kBN];
  uint8_t v_scale[C::kStages][kBN];
  struct Scales {  // of a warp's keys: K's, V's as fp16
    float k[32];
    uint16_t v[32];
  } scales[kWarps];
  uint2 q[kRows == 16 ? kRows / 8 : 1][kRows == 16 ? D / 16 : 1][32];  // 16 rows: Q's operands (too many registers)
  float o[2][kRows][C::kJoin + 4];  // channels of two warps' O, padded
  float2 ml[kWarps][kRows];
  uint64_t full[C::kStages], empty[C::kStages];
  int abort_flag;
};

// Offset of a byte of a key's row of codes in a tile.
template <int D>
__device__ __forceinline__ uint32_t swizzled(int key, int byte) {
  return key * D + ((((byte >> 4) ^ (D == 64 ? (key >> 1) & 3 : key & 7)) << 4) | (byte & 15));
}
__device__ __forceinline__ bool nan_codes(uint32_t u) {
  return (((u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
}
__device__ __forceinline__ uint32_t finite_codes(uint32_t u) {  // with 0 in their place
  uint32_t r = u;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (((u >> (8 * k)) & 0x7Fu) == 0x7Fu) r &= ~(0xFFu << (8 * k));
  return r;
}

// The 8 x 8 matrix of 16-bit values that the warp holds, transposed.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t u) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(u));
  return r;
}

// V codes that stand for NaN, and those of keys without a legal scale, among a warp's 32 keys (from key0 on):
// replaced by 0, and NaN put into the outputs of the rows that see them.  Keys past the sequence's last, kl (slots that
// nobody has written, or what the last tile left), are cleared ahead, so that the search for the rows is rare
// (16 rows over 400 keys in pages of 16: 67 us with the search in every last tile).
template <int D, int kNB>
__device__ __forceinline__ void take_out_nan(uint8_t* v, uint8_t* scale, int key0, int kl, const int (&lim)[kNB][2],
                                             int lane, float (&o)[kNB][D / 16][4]) {
  uint4* vv = reinterpret_cast<uint4*>(v);
  if (key0 + 32 > kl) {
    if (key0 + lane >= kl) {
      scale[lane] = kLeastScaleByte;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) vv[lane * (D / 16) + i] = make_uint4(0, 0, 0, 0);
    }
    __syncwarp();
  }
  const bool lost = bad_scale(scale[lane]);
  bool bad = lost;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const uint4 x = vv[lane + 32 * i];
    bad |= nan_codes(x.x) || nan_codes(x.y) || nan_codes(x.z) || nan_codes(x.w);
  }
  if (!__any_sync(0xffffffffu, bad)) return;
#pragma unroll 1
  for (int key = 0; key < 32; ++key) {
    const bool all = bad_scale(scale[key]);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
      const uint32_t two = *reinterpret_cast<const uint16_t*>(v + swizzled<D>(key, 16 * n + 2 * (lane >> 2)));
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // channel 16 n + 2 (lane / 4) + k
        if (!all && ((two >> (8 * k)) & 0x7Fu) != 0x7Fu) continue;
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (key0 + key < lim[b][i]) o[b][n][2 * k + i] = __int_as_float(0x7FC00000);
      }
    }
  }
  __syncwarp();
  if (lost) {
    scale[lane] = kLeastScaleByte;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) vv[lane * (D / 16) + i] = make_uint4(0, 0, 0, 0);
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const uint4 x = vv[lane + 32 * i];
    vv[lane + 32 * i] = make_uint4(finite_codes(x.x), finite_codes(x.y), finite_codes(x.z), finite_codes(x.w));
  }
  __syncwarp();
}

template <int D, bool F16, int kRows>
__global__ void __launch_bounds__(kThreads, Rows8Cfg<D, kRows>::kPerSm)
    seq_rows8_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                     const __grid_constant__ SeqAttnArgs prm, const SeqScratch sc, const int cost, const bool whole) {
  using C = Rows8Cfg<D, kRows>;
  constexpr int kStages = C::kStages, kNB = kRows / 8;
  extern __shared__ unsigned char smem_raw[];
  Rows8Smem<D, kRows>& sm = *reinterpret_cast<Rows8Smem<D, kRows>*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ long long scratch[33];
  const int P = gridDim.x, cta = blockIdx.x, tid = threadIdx.x;
  const int warp = warp_uniform_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  unsigned int* err = prm.err;
  pdl_launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], kWarps);
    }
    sm.abort_flag = 0;
    fence_mbarrier_init();
    fence_proxy_async_smem();
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  const int Hkv = prm.Hkv, group = prm.group;
  pdl_wait();  // what is ahead in the stream: the inputs are there, and the last call's join is over
  Place pl;
  const long long total = find_place<kBN, kRows>(prm, cost, &pl, scratch);  // also publishes the mbarriers
  const long long per = units_per_cta(total, P);
  long long begin = min(cta * per, total);
  const long long end = min(begin + per, total);
  // Nothing cut, until the producer knows better (one writer, since no barrier lies between the two).
  if (tid == 32 * kWarps) sc.recs[2 * cta] = make_int4(0, 0, 0, 0);
  if (begin >= end) return;  // uniform
  if (whole) {  // from the next item's start on
    const int ext = pl.item(), in = (int)((begin - pl.base) % ext);
    if (in > 0) begin += ext - in;
    if (begin >= end) return;  // uniform
    if (begin - pl.base >= pl.extent(Hkv)) advance<kBN, kRows>(prm, &pl);
  }
  bool ok = true;

  if (warp == kWarps) {
    // ------------------------------------------------------------ TMA producer
    const int log2p = prm.kv.log2_page, ps = prm.kv.page_size;
    const int ppt = ps < kBN ? kBN / ps : 1;  // pages (boxes) of a tile
    const int box_rows = ps < kBN ? ps : kBN;
    uint32_t lc = 0;
    for (long long u = begin; u < end && ok;) {
      Segment sg;
      if (!segment_at(pl, u, end, whole, &sg)) break;
      const int h = sg.h;
      const int n_pages = (pl.s.kl + ps - 1) >> log2p;
      const int32_t* table = prm.kv.table + (size_t)pl.b * prm.kv.width;
      int first = (sg.t0 * kBN) >> log2p, window = 0, next = 0;
      if (first + lane < n_pages) window = table[first + lane];
      if (first + 32 + lane < n_pages) next = table[first + 32 + lane];
      for (int j = sg.t0; j < sg.t1; ++j, ++lc) {
        const int st = lc % kStages, p0 = (j * kBN) >> log2p;
        if (p0 >= first + 32) {
          first += 32;
          window = next;
          next = first + 32 + lane < n_pages ? table[first + 32 + lane] : 0;
        }
        const int n_box = min(ppt, n_pages - p0);  // the pages that exist; the rest of the tile is masked
        const int at = p0 - first, y = (j * kBN) & (ps - 1);
        ok = mbar_wait_warp(&sm.empty[st], ((lc / kStages) & 1) ^ 1, err, abort_flag);
        if (!ok) break;
        // The scales of a page outside the pool, whose codes the copy fills with 0, are set here.
        const bool mine = lane >= at && lane < at + n_box, out = (unsigned)window >= (unsigned)prm.kv.n_pages;
        const unsigned lost = __ballot_sync(0xffffffffu, mine && out);
        if (lost) {
          if (mine && out)
            for (int i = 0; i < box_rows; ++i) {
              sm.k_scale[st][(lane - at) * box_rows + i] = kLeastScaleByte;
              sm.v_scale[st][(lane - at) * box_rows + i] = kLeastScaleByte;
            }
          if (lane == 0) atomicOr(err, VP_DEVERR_PAGE);
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (elect_one())
          mbar_arrive_expect_tx(&sm.full[st], 2 * box_rows * (n_box * D + n_box - __popc(lost)));
        __syncwarp();
        // One elected lane copies page after page: coordinates that differ between lanes would cost
        // the copies' issue more than twice as much.
        for (int i = 0; i < n_box; ++i) {
          const int page = __shfl_sync(0xffffffffu, window, at + i);
          if (elect_one()) {
            tma_load_4d(sm.k[st] + i * box_rows * D, &tmap_k, &sm.full[st], 0, y, h, page);
            tma_load_4d(sm.v[st] + i * box_rows * D, &tmap_v, &sm.full[st], 0, y, h, page);
            if ((unsigned)page < (unsigned)prm.kv.n_pages) {
              const long long row = (((long long)page * Hkv + h) << log2p) + y;
              bulk_load(sm.k_scale[st] + i * box_rows, prm.kv.k_scale + row, box_rows, &sm.full[st]);
              bulk_load(sm.v_scale[st] + i * box_rows, prm.kv.v_scale + row, box_rows, &sm.full[st]);
            }
          }
          __syncwarp();
        }
      }
      // This CTA's entry of the list of cut items: one whose first part ends this run.  The cuts k per
      // of the item that stay: item0 + kItemCost < k per < item0 + its extent.
      if (sg.t1 < pl.n_kv && sg.t0 == 0 && lane == 0) {
        const int last = (int)((sg.item0 + pl.item() - 1) / per);
        sc.recs[2 * cta] = make_int4(last - cta + 1, h, sg.rt, pl.b);
        sc.recs[2 * cta + 1] = make_int4(pl.s.q0, pl.s.ql, pl.s.kl, 2 * cta + (u > begin));
      }
      u = sg.item0 + pl.item();
      if (u < end && u - pl.base >= pl.extent(Hkv)) advance<kBN, kRows>(prm, &pl);
    }
    // The copies land before the CTA releases its shared memory (after a timeout nobody else
    // may be waiting for them).
    if (!ok && lane == 0)
      for (int s = 0; s < kStages; ++s)
        if (lc > (uint32_t)s) {
          const uint32_t last = (lc - 1 - s) / kStages * kStages + s;
          for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.full[s], (last / kStages) & 1); ++t) {}
        }
    return;
  }

  // -------------------------------------------------------------- compute
  const int r0 = lane >> 2, tq = lane & 3;
  const int ld_key = lane & 15, ld_chunk = lane >> 4;  // ldmatrix: 16 keys at two neighbouring chunks of 16 bytes
  auto& scales = sm.scales[warp];
  uint32_t lc = 0;
  for (long long u = begin; u < end && ok;) {
    Segment sg;
    if (!segment_at(pl, u, end, whole, &sg)) break;
    const int h = sg.h, rt = sg.rt;
    const Seq s = pl.s;
    // Q: row r0 of each block of 8, channels 16 kk + 4 tq .. + 3.  Scores and outputs: rows 2 tq + i.
    uint32_t qf[kNB][D / 16][2];
    int tok[kNB][2], head[kNB][2], lim[kNB][2];
    float back[kNB][2];
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int row = rt * kRows + 8 * b + r0, t = prm.by_group(row);
      const uint16_t* q = prm.q + (int64_t)(s.q0 + t) * prm.q_stride + (h * group + row - t * group) * D + 4 * tq;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint2 x = t < s.ql ? *reinterpret_cast<const uint2*>(q + kk * 16) : make_uint2(0u, 0u);
        qf[b][kk][0] = x.x;
        qf[b][kk][1] = x.y;
      }
      float mine = 1.f;
      if constexpr (!F16) {
        uint32_t top = 0;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            top = max(top, max(qf[b][kk][x] << 16 & 0x7FFF0000u, qf[b][kk][x] & 0x7FFF0000u));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const HalfRow r(top);
        mine = r.back;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
          for (int x = 0; x < 2; ++x) qf[b][kk][x] = r.convert(qf[b][kk][x]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int mr = rt * kRows + 8 * b + 2 * tq + i;
        tok[b][i] = prm.by_group(mr);
        head[b][i] = h * group + mr - tok[b][i] * group;
        lim[b][i] = tok[b][i] < s.ql ? row_limit(prm, tok[b][i], s.ql, s.kl) : 0;
        back[b][i] = F16 ? 1.f : __shfl_sync(0xffffffffu, mine, 4 * (2 * tq + i));
      }
    }
    if constexpr (kRows == 16) {  // (the last item's reads are behind the join's barriers)
      if (warp == 0) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) sm.q[b][kk][lane] = make_uint2(qf[b][kk][0], qf[b][kk][1]);
      }
      compute_barrier();
    }
    auto q_at = [&](int b, int kk) {
      return kRows == 16 ? sm.q[b][kk][lane] : make_uint2(qf[b][kk][0], qf[b][kk][1]);
    };
    const int masked_from = max(row_limit(prm, prm.by_group(rt * kRows), s.ql, s.kl), 0) / kBN;
    float m[kNB][2], l[kNB][2], o[kNB][D / 16][4];
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      m[b][0] = m[b][1] = kUnset;
      l[b][0] = l[b][1] = 0.f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[b][n][i] = 0.f;
    }

    for (int j = sg.t0; j < sg.t1; ++j, ++lc) {
      const int st = lc % kStages, key0 = j * kBN + 32 * warp;
      ok = mbar_wait_warp(&sm.full[st], (lc / kStages) & 1, err, abort_flag);
      if (!ok) break;
      const bool masked = j >= masked_from;
      uint8_t* vt = sm.v[st] + 32 * warp * D;
      const uint32_t kb = smem_u32(sm.k[st]) + 32 * warp * D, vb = smem_u32(vt);
      if (masked) take_out_nan<D, kNB>(vt, sm.v_scale[st] + 32 * warp, key0, s.kl, lim, lane, o);
      // The keys' scales, a key per lane; NaN where there is none.
      {
        const uint32_t ke = sm.k_scale[st][32 * warp + lane];
        scales.k[lane] = __uint_as_float(bad_scale(ke) ? 0x7FC00000u : ke << 23);
        scales.v[lane] = (uint16_t)scale_half(sm.v_scale[st][32 * warp + lane]);
        __syncwarp();
      }
      // c[b][g][2 k + i]: key 16 g + 8 k + r0 of the warp's, row 2 tq + i of block b.
      float c[kNB][2][4];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) c[b][g][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < D / 16; kk += 2) {
          uint32_t x[4], a[2][4];
          ldmatrix4(x, kb + g * 16 * D + swizzled<D>(ld_key, 16 * (kk + ld_chunk)));
#pragma unroll
          for (int y = 0; y < 4; ++y) codes_to_half(x[y], a[y >> 1][y & 1], a[y >> 1][2 + (y & 1)]);
#pragma unroll
          for (int b = 0; b < kNB; ++b) {
            const uint2 q0 = q_at(b, kk), q1 = q_at(b, kk + 1);
            mma16816<true>(c[b][g], a[0], q0.x, q0.y);
            mma16816<true>(c[b][g], a[1], q1.x, q1.y);
          }
        }
      }
      float mx[kNB][2];
#pragma unroll
      for (int b = 0; b < kNB; ++b) mx[b][0] = mx[b][1] = kUnset;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float f = scales.k[16 * g + 8 * k + r0];
#pragma unroll
          for (int b = 0; b < kNB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              // q . k first, by powers of two, then the scale: their product ahead of it may be past 32 bits
              // where the score is not (0 x inf; q of 2^-125 under a scale of 2^125).
              float& x = c[b][g][2 * k + i];
              x *= F16 ? f : f * back[b][i];
              x *= prm.scale_log2;
              if (masked && key0 + 16 * g + 8 * k + r0 >= lim[b][i]) x = -INFINITY;
              mx[b][i] = fmaxf(mx[b][i], x);
            }
        }
      bool need = false;
#pragma unroll
      for (int b = 0; b < kNB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) mx[b][i] = fmaxf(mx[b][i], __shfl_xor_sync(0xffffffffu, mx[b][i], k));
          mx[b][i] = reference_point<true>(mx[b][i], 1.f);
          need = need || mx[b][i] - m[b][i] > kRescaleThreshold;  // (a difference: m + 8 could round up to mx)
        }
      if (__any_sync(0xffffffffu, need)) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float to = fmaxf(m[b][i], mx[b][i]), alpha = fast_exp2(m[b][i] - to);
            m[b][i] = to;
            l[b][i] *= alpha;
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
              o[b][n][i] *= alpha;
              o[b][n][2 + i] *= alpha;
            }
          }
      }
      uint32_t p[kNB][2][2];
#pragma unroll
      for (int b = 0; b < kNB; ++b)
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float x = fast_exp2(c[b][g][2 * k] - m[b][0]), y = fast_exp2(c[b][g][2 * k + 1] - m[b][1]);
            l[b][0] += x;
            l[b][1] += y;
            p[b][g][k] = transpose8x8(pack2<true>(x, y));
          }
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t scale[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) scale[k] = *reinterpret_cast<const uint32_t*>(scales.v + 16 * g + 8 * k + 2 * tq);
#pragma unroll
        for (int n = 0; n < D / 16; n += 2) {
          uint32_t x[4], a[2][4];
          ldmatrix4_trans(x, vb + g * 16 * D + swizzled<D>(ld_key, 16 * (n + ld_chunk)));
#pragma unroll
          for (int y = 0; y < 4; ++y) {  // keys 8 (y & 1) .. + 7 of the group, chunk n + y / 2
            uint32_t even, odd;
            codes_to_half(__byte_perm(x[y], 0, 0x3120), even, odd);
            a[y >> 1][2 * (y & 1)] = mul_half2(even, scale[y & 1]);
            a[y >> 1][2 * (y & 1) + 1] = mul_half2(odd, scale[y & 1]);
          }
#pragma unroll
          for (int b = 0; b < kNB; ++b) {
            mma16816<true>(o[b][n], a[0], p[b][g][0], p[b][g][1]);
            mma16816<true>(o[b][n + 1], a[1], p[b][g][0], p[b][g][1]);
          }
        }
      }
      if (masked) fence_proxy_async_smem();  // the zeros written above, before the next copy
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.empty[st]);
    }
    // Join the four warps: common maximum, sums, then O through shared memory (2, 3 into 0, 1;
    // 1 into 0: always in this order).  A warp that gave up waiting takes all along.
    float L[kNB][2], M[kNB][2];
#pragma unroll
    for (int b = 0; b < kNB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) l[b][i] += __shfl_xor_sync(0xffffffffu, l[b][i], k);
        if (r0 == 0) sm.ml[warp][8 * b + 2 * tq + i] = make_float2(m[b][i], l[b][i]);
      }
    if (compute_any(!ok)) break;
#pragma unroll
    for (int b = 0; b < kNB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        M[b][i] = kUnset;
        L[b][i] = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M[b][i] = fmaxf(M[b][i], sm.ml[w][8 * b + 2 * tq + i].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 x = sm.ml[w][8 * b + 2 * tq + i];
          L[b][i] = fmaf(x.y, fast_exp2(x.x - M[b][i]), L[b][i]);
        }
        const float f = fast_exp2(m[b][i] - M[b][i]);
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
          o[b][n][i] *= f;
          o[b][n][2 + i] *= f;
        }
      }
    // o[b][n][i], o[b][n][2 + i]: channels 16 n + 2 r0 and the next of row 2 tq + i.
#pragma unroll
    for (int n0 = 0; n0 < D / 16; n0 += C::kJoin / 16) {
      auto put = [&](float (*dst)[C::kJoin + 4]) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int n = 0; n < C::kJoin / 16; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              *reinterpret_cast<float2*>(&dst[8 * b + 2 * tq + i][16 * n + 2 * r0]) =
                  make_float2(o[b][n0 + n][i], o[b][n0 + n][2 + i]);
      };
      auto add = [&](float (*src)[C::kJoin + 4]) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int n = 0; n < C::kJoin / 16; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float2 x = *reinterpret_cast<const float2*>(&src[8 * b + 2 * tq + i][16 * n + 2 * r0]);
              o[b][n0 + n][i] += x.x;
              o[b][n0 + n][2 + i] += x.y;
            }
      };
      if (n0 > 0) compute_barrier();  // warp 0 has read the channels before
      if (warp >= 2) put(sm.o[warp - 2]);
      compute_barrier();
      if (warp < 2) add(sm.o[warp]);
      if (warp == 1) put(sm.o[1]);
      compute_barrier();
      if (warp == 0) add(sm.o[1]);
    }
    if (warp == 0) {
#pragma unroll
      for (int b = 0; b < kNB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (tok[b][i] >= s.ql) continue;
          if (!sg.part) {  // the whole item
            const float inv = 1.f / L[b][i];
            uint16_t* out = prm.out + (int64_t)(s.q0 + tok[b][i]) * prm.out_stride + head[b][i] * D + 2 * r0;
#pragma unroll
            for (int n = 0; n < D / 16; ++n)
              *reinterpret_cast<uint32_t*>(out + 16 * n) =
                  lim[b][i] > 0 ? pack2<F16>(o[b][n][i] * inv, o[b][n][2 + i] * inv) : 0u;
            if (prm.lse && r0 == 0)
              prm.lse[(size_t)(s.q0 + tok[b][i]) * prm.Hq + head[b][i]] =
                  lim[b][i] > 0 ? (M[b][i] + log2f(L[b][i])) * 0.69314718055994531f : -INFINITY;
          } else {
            const size_t r = (2 * (size_t)cta + (u == begin ? 0 : 1)) * kSmallRows + 8 * b + 2 * tq + i;
#pragma unroll
            for (int n = 0; n < D / 16; ++n)
              *reinterpret_cast<float2*>(sc.part_o + r * D + 16 * n + 2 * r0) =
                  make_float2(o[b][n][i], o[b][n][2 + i]);
            if (r0 == 0) sc.part_ml[r] = make_float2(M[b][i], L[b][i]);
          }
        }
    }
    u = sg.item0 + pl.item();
    if (u < end && u - pl.base >= pl.extent(Hkv)) advance<kBN, kRows>(prm, &pl);
  }
}

template <int D, bool F16, int kRows>
cudaError_t launch_rows8(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st) {
  using C = Rows8Cfg<D, kRows>;
  CUtensorMap mk, mv;
  cudaError_t e = make_kv8_maps(a, kBN, &mk, &mv);
  if (e != cudaSuccess) return e;
  const int P = C::kPerSm * (num_sms < kMaxCtas ? num_sms : kMaxCtas);
  constexpr int smem = (int)sizeof(Rows8Smem<D, kRows>) + 1024;
  static_assert(C::kPerSm * (smem + 1024 + 512) <= 228 * 1024, "shared memory of an SM");
  const void* fn = reinterpret_cast<const void*>(seq_rows8_kernel<D, F16, kRows>);
  e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  SeqAttnArgs aa = a;
  SeqScratch ss = sc;
  bool whole = rows_whole(a, P);
  int cost = whole && count_items(a, kRows) <= P ? kWholeCost : kItemCost;
  void* args[] = {&mk, &mv, &aa, &ss, &cost, &whole};
  e = launch_pdl(fn, dim3(P), kThreads, smem, st, args);
  if (e != cudaSuccess || whole) return e;
  return launch_seq_join(a, sc, kRows, P, st);
}

}  // namespace

cudaError_t launch_seq_rows8(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st) {
  using Launch = cudaError_t (*)(const SeqAttnArgs&, const SeqScratch&, int, cudaStream_t);
  static const Launch table[2][2][2] = {{{launch_rows8<64, false, 8>, launch_rows8<64, false, 16>},
                                         {launch_rows8<64, true, 8>, launch_rows8<64, true, 16>}},
                                        {{launch_rows8<128, false, 8>, launch_rows8<128, false, 16>},
                                         {launch_rows8<128, true, 8>, launch_rows8<128, true, 16>}}};
  // Sequences of up to 8 rows, on average: items of 8.
  const bool few = (long long)a.T * a.group <= 8ll * a.B;
  return table[a.d == 128][a.fp16 != 0][few ? 0 : 1](a, sc, num_sms, st);
}

}  // namespace vp
