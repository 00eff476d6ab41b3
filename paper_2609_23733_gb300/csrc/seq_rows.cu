// Attention of few query rows per sequence (single tokens and short chunks) over long keys:
// o = sum_j p_j v_j / sum_j p_j over the keys j < lim(i) that row (token i, head h) sees.
//
// Bound by memory: every key and value is read once per 16 rows (token x head of a kv head's
// group), 4 d flop per row and key beside 4 d bytes per key, far below the tensor cores' rate;
// mma.sync m16n8k16 with the rows padded to 16 keeps up with HBM and needs no TMEM round
// trip per tile.  What counts is bytes in flight on every SM and an even cut of the work.
//
// The work is the sequence of units (sequence, kv head, 16 rows, 64 keys), each item (16 rows of a kv
// head) with kItemCost added; CTA c of P takes the c-th of P equal runs, whatever items they belong
// to, so that all CTAs end together for any mix of lengths.  An item that a CTA holds in part leaves a
// partial result, and seq_join_kernel (a programmatic dependent launch) joins the parts in order.
// Each CTA finds its place by a scan over the sequences' lengths.  Short items are kept whole (see
// rows_whole) and nothing is joined.
//   warp 4      TMA: K / V tiles through a ring, page by page (page ids read 32 ahead).
//   warps 0-3   16 keys of every tile each: S = Q K^T (16 x 16), softmax against the warp's own
//               running maximum (moved when it grows by more than 2^8), O += P V in registers;
//               the four warps' results are joined at the end of an item.
// Scores, maxima, sums and outputs are held in 32 bits; P is rounded to the storage type.
// Measured on GB300: 4 single tokens over 130,003 to 137,400 keys, 32 heads of 128 on 4 kv heads, pages
// of 16: 169 us as called (6.5 TB/s, 0.95 of the measured copy bandwidth); 64 tokens over 97 to 16,381 keys,
// 16 heads of 64 on 4: 41.7 us (5.1 TB/s; the first 2.6 us find the place, the last 4 join the parts).
// V values that are not finite and not seen by every row are taken out of the tile (0 x inf
// would reach all rows) and added to the rows that see them.
#include <float.h>
#include <math.h>

#include "seq.h"

namespace vp {

namespace {

constexpr int kRows = kSmallRows;  // rows of an item (an MMA's M)
constexpr int kBN = 64;            // keys of a unit
constexpr int kWarps = 4;          // compute warps
constexpr int kThreads = 32 * (kWarps + 1);
constexpr float kUnset = -FLT_MAX;
constexpr float kRescaleThreshold = 8.f;  // log2 units
// An item costs about as much as this many units on top of its own (its rows' q, the join of the warps):
// the extent of an item is kItemCost + its units, and cuts within the first kItemCost move to its start.
// (64 single tokens over 97 to 16,381 keys, on the device: 47.4 us without, 43.0 with 1, 40.6 with 2 to 5.)
constexpr int kItemCost = 4;
// The same where items are kept whole and there are no more of them than CTAs: runs of one item, so that
// none has two while another has none (prompts of 1, 16, 261, 4 and 65 tokens, 16 heads of 64: 10.8 ->
// 9.1 us; with more items than CTAs runs of equal work are better: prompts of 3, 5, 400 and 90
// tokens, 4 kv heads, 12.2 against 17.2 us).
constexpr int kWholeCost = 32;

template <int D>
struct RowsCfg {
  static constexpr int kHalves = D / 64;
  static constexpr int kStages = D == 64 ? 4 : 3;   // 64 / 96 KB of K and V
  static constexpr int kPerSm = small_rows_ctas_per_sm(D);
};

template <int D>
struct RowsSmem {
  using C = RowsCfg<D>;
  uint16_t k[C::kStages][C::kHalves][kBN * 64];
  uint16_t v[C::kStages][C::kHalves][kBN * 64];
  float o[2][kRows][64 + 8];  // a 64-channel half of two warps' O, padded
  float2 ml[kWarps][kRows];
  uint64_t full[C::kStages], empty[C::kStages];
  int abort_flag;
};

// A sequence's place in the order of items.
struct Place {
  int b;             // a.B: past the end
  long long base;    // the extent of all items before it
  Seq s;
  int n_kv, n_rt;    // key tiles, 16-row tiles per kv head
  int cost;          // kItemCost or kWholeCost
  __device__ __forceinline__ int item() const { return n_kv + cost; }
  __device__ __forceinline__ long long extent(int Hkv) const { return (long long)Hkv * n_rt * item(); }
};

__device__ __forceinline__ void fill_place(const SeqAttnArgs& a, int b, Place* p) {
  p->b = b;
  p->s = load_seq(a, b);
  p->n_kv = max(1, (int)(((long long)p->s.kl + kBN - 1) / kBN));  // one even without keys: for the zeros
  p->n_rt = (int)(((long long)p->s.ql * a.group + kRows - 1) / kRows);
}

// Units per CTA.
__device__ __forceinline__ long long units_per_cta(long long total, int P) {
  const long long x = total + P - 1;
  return x >> 32 ? x / P : (long long)((uint32_t)x / (uint32_t)P);
}

// The units of all sequences, and the place of this CTA's first one (if it has any): a scan of the
// lengths by all threads, once where there are no more sequences than threads, else once for
// the total and once for the place.  scratch: a value per warp.
__device__ __forceinline__ long long find_place(const SeqAttnArgs& a, int cost, Place* place,
                                                long long* scratch) {
  __shared__ Place s_place;
  const int tid = threadIdx.x, n = blockDim.x, n_warps = n / 32, lane = lane_id(), w = warp_id();
  if (tid == 0) {
    s_place.b = 0;  // there always is one, but for sequences that change under the call
    s_place.base = 0;
    s_place.s = Seq{0, 0, 0};
    s_place.n_kv = s_place.n_rt = 1;
    s_place.cost = cost;
  }
  long long all = 0;
  for (int pass = a.B <= n ? 1 : 0; pass < 2; ++pass) {
    long long before = 0;
    for (int b0 = 0; b0 < a.B; b0 += n) {
      Place p;
      long long mine = 0;
      if (b0 + tid < a.B) {
        p.cost = cost;
        fill_place(a, b0 + tid, &p);
        mine = p.extent(a.Hkv);
      }
      long long v = mine;
#pragma unroll
      for (int k = 1; k < 32; k <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, v, k);
        if (lane >= k) v += x;
      }
      __syncthreads();
      if (lane == 31) scratch[w] = v;
      __syncthreads();
      long long lead = before, total = before;
      for (int i = 0; i < n_warps; ++i) {
        if (i < w) lead += scratch[i];
        total += scratch[i];
      }
      before = total;
      if (pass == 0) continue;
      if (a.B <= n) all = total;
      const long long u = (long long)blockIdx.x * units_per_cta(all, gridDim.x), end = lead + v;
      if (mine > 0 && end - mine <= u && u < end) {
        p.base = end - mine;
        s_place = p;
      }
    }
    if (pass == 0) all = before;
  }
  __syncthreads();
  *place = s_place;
  return all;
}

// The next sequence with items.
__device__ __forceinline__ void advance(const SeqAttnArgs& a, Place* p) {
  long long base = p->base + p->extent(a.Hkv);
  int b = p->b + 1;
  for (; b < a.B; ++b) {
    fill_place(a, b, p);
    if (p->extent(a.Hkv) > 0) break;
  }
  p->b = b;
  p->base = base;
}

// What a CTA's run [begin, end) holds of one item.
struct Segment {
  int h, rt;        // kv head, row tile
  int t0, t1;       // key tiles
  bool part;        // not all of the item's
  long long item0;  // where the item begins
};

// The segment at u; false if the run holds none of the item (a cut within its first p.cost).
// whole: an item belongs to the run that it begins in.
__device__ __forceinline__ bool segment_at(const Place& p, long long u, long long end, bool whole,
                                           Segment* s) {
  const long long rel = u - p.base;
  const int ext = p.item();
  const int item = rel >> 32 ? (int)(rel / ext) : (int)((uint32_t)rel / (uint32_t)ext);
  s->item0 = p.base + (long long)item * ext;
  const int from = (int)(u - s->item0), to = whole ? ext : (int)min((long long)ext, end - s->item0);
  if (to < ext && to <= p.cost) return false;
  s->h = item / p.n_rt;
  s->rt = item - s->h * p.n_rt;
  s->t0 = max(from - p.cost, 0);
  s->t1 = to - p.cost;
  s->part = s->t0 > 0 || s->t1 < p.n_kv;
  return true;
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// c += a b, 16 x 8 x 16, fp32 accumulators.
template <bool F16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// compute_barrier that also tells every thread whether `v` was true on any of them.
__device__ __forceinline__ bool compute_any(bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)v), "n"(32 * kWarps)
      : "memory");
  return r != 0;
}

__device__ __forceinline__ void compute_barrier() {
  asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
}

template <int D, bool F16, bool kPaged>
__global__ void __launch_bounds__(kThreads, RowsCfg<D>::kPerSm)
    seq_rows_kernel(const __grid_constant__ CUtensorMap tmap_k,
                    const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ SeqAttnArgs prm, const SeqScratch sc, const int cost,
                    const bool whole) {
  using C = RowsCfg<D>;
  constexpr int kStages = C::kStages, kHalves = C::kHalves;
  extern __shared__ unsigned char smem_raw[];
  RowsSmem<D>& sm = *reinterpret_cast<RowsSmem<D>*>(
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
  const long long total = find_place(prm, cost, &pl, scratch);  // its barriers also publish the mbarriers
  const long long per = units_per_cta(total, P);
  long long begin = min(cta * per, total);
  const long long end = min(begin + per, total);
  // Nothing cut, until the producer knows better: cleared by the thread that writes the entry below, since
  // no barrier lies between the two.
  if (tid == 32 * kWarps) sc.recs[2 * cta] = make_int4(0, 0, 0, 0);
  if (begin >= end) return;  // uniform
  if (whole) {  // from the next item's start on
    const int ext = pl.item(), in = (int)((begin - pl.base) % ext);
    if (in > 0) begin += ext - in;
    if (begin >= end) return;  // uniform
    if (begin - pl.base >= pl.extent(Hkv)) advance(prm, &pl);
  }
  bool ok = true;

  if (warp == kWarps) {
    // ------------------------------------------------------------ TMA producer
    const int log2p = prm.kv.log2_page, ps = prm.kv.page_size;
    const int ppt = kPaged && ps < kBN ? kBN / ps : 1;  // pages (boxes) of a tile
    const uint32_t box_bytes = (kPaged && ps < kBN ? ps : kBN) * 128;
    uint32_t lc = 0;
    for (long long u = begin; u < end && ok;) {
      Segment sg;
      if (!segment_at(pl, u, end, whole, &sg)) break;
      const int h = sg.h;
      const int n_pages = kPaged ? (pl.s.kl + ps - 1) >> log2p : 0;
      const int32_t* table = kPaged ? prm.kv.table + (size_t)pl.b * prm.kv.width : nullptr;
      int first = kPaged ? (sg.t0 * kBN) >> log2p : 0, window = 0, next = 0;
      if (kPaged) {
        if (first + lane < n_pages) window = table[first + lane];
        if (first + 32 + lane < n_pages) next = table[first + 32 + lane];
      }
      for (int j = sg.t0; j < sg.t1; ++j, ++lc) {
        const int st = lc % kStages;
        int y = pl.s.q0 + j * kBN, at = 0, n_box = 1;
        if (kPaged) {
          const int p0 = (j * kBN) >> log2p;
          if (p0 >= first + 32) {
            first += 32;
            window = next;
            next = first + 32 + lane < n_pages ? table[first + 32 + lane] : 0;
          }
          n_box = min(ppt, n_pages - p0);  // the pages that exist; the rest of the tile is masked
          at = p0 - first;
          y = (j * kBN) & (ps - 1);
        }
        ok = mbar_wait_warp(&sm.empty[st], ((lc / kStages) & 1) ^ 1, err, abort_flag);
        if (!ok) break;
        if (elect_one()) mbar_arrive_expect_tx(&sm.full[st], 2 * n_box * kHalves * box_bytes);
        __syncwarp();
        // One elected lane copies page after page: coordinates that differ between lanes would cost
        // the copies' issue 800 clocks a tile, more than twice as much.
        for (int i = 0; i < n_box; ++i) {
          const int page = kPaged ? __shfl_sync(0xffffffffu, window, at + i) : 0;
          if (kPaged && (unsigned)page >= (unsigned)prm.kv.n_pages && lane == 0) atomicOr(err, VP_DEVERR_PAGE);
          const int off = i * (box_bytes / 2);
          if (elect_one()) {
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) {
              tma_load_4d(sm.k[st][hf] + off, &tmap_k, &sm.full[st], hf * 64, y, h, page);
              tma_load_4d(sm.v[st][hf] + off, &tmap_v, &sm.full[st], hf * 64, y, h, page);
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
      if (u < end && u - pl.base >= pl.extent(Hkv)) advance(prm, &pl);
    }
    // The copies land before the CTA releases its shared memory (after a timeout nobody else
    // may be waiting for them).
    if (!ok && lane == 0)
      for (int s = 0; s < kStages; ++s)
        if (lc > (uint32_t)s) {
          const uint32_t last = (lc - 1 - s) / kStages * kStages + s;
          for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.full[s], (last / kStages) & 1); ++t) {}
        }
  } else {
    // ------------------------------------------------------------ compute
    const float cs = prm.scale_log2;
    const int r0 = lane >> 2, tq = lane & 3;
    // ldmatrix rows of this lane: K, keys (lane & 7) + 8 (lane >> 4) at channel chunk (lane >> 3) & 1;
    // V (transposed), keys (lane & 15) at channel chunk lane >> 4.
    const int k_key = (lane & 7) + ((lane >> 4) << 3), k_chunk = (lane >> 3) & 1;
    const int v_key = lane & 15, v_chunk = lane >> 4;
    uint32_t lc = 0;
    for (long long u = begin; u < end && ok;) {
      Segment sg;
      if (!segment_at(pl, u, end, whole, &sg)) break;
      const int h = sg.h, rt = sg.rt;
      const Seq s = pl.s;
      int tok[2], head[2], lim[2];
      bool valid[2];
      uint32_t qf[D / 16][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = rt * kRows + r0 + 8 * i;
        tok[i] = prm.by_group(row);
        head[i] = h * group + row - tok[i] * group;
        valid[i] = tok[i] < s.ql;
        lim[i] = valid[i] ? row_limit(prm, tok[i], s.ql, s.kl) : 0;
        const uint16_t* q = prm.q + (int64_t)(s.q0 + tok[i]) * prm.q_stride + head[i] * D + 2 * tq;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          qf[kk][i] = valid[i] ? *reinterpret_cast<const uint32_t*>(q + kk * 16) : 0u;
          qf[kk][2 + i] = valid[i] ? *reinterpret_cast<const uint32_t*>(q + kk * 16 + 8) : 0u;
        }
      }
      const int masked_from = max(row_limit(prm, prm.by_group(rt * kRows), s.ql, s.kl), 0) / kBN;
      float m[2] = {kUnset, kUnset}, l[2] = {0.f, 0.f}, o[D / 8][4];
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = 0.f;

      for (int j = sg.t0; j < sg.t1; ++j, ++lc) {
        const int st = lc % kStages;
        ok = mbar_wait_warp(&sm.full[st], (lc / kStages) & 1, err, abort_flag);
        if (!ok) break;
        const uint32_t kb = smem_u32(sm.k[st][0]) + warp * 16 * 128;
        const uint32_t vb = smem_u32(sm.v[st][0]) + warp * 16 * 128;
        const int key0 = j * kBN + warp * 16;
        float c[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) c[n][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          uint32_t b[4];
          const int chunk = 2 * (kk & 3) + k_chunk;
          ldmatrix4(b, kb + (kk >> 2) * (kBN * 128) + k_key * 128 + ((chunk ^ (k_key & 7)) << 4));
          mma16816<F16>(c[0], qf[kk], b[0], b[1]);
          mma16816<F16>(c[1], qf[kk], b[2], b[3]);
        }
        const bool masked = j >= masked_from;
        float mx[2] = {kUnset, kUnset};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            c[n][i] *= cs;
            if (masked && key0 + n * 8 + 2 * tq + (i & 1) >= lim[i >> 1]) c[n][i] = -INFINITY;
            mx[i >> 1] = fmaxf(mx[i >> 1], c[n][i]);
          }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
          mx[i] = reference_point<F16>(fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2)), 1.f);
        }
        // (A difference: m + 8 could round up to mx.)
        const bool need = mx[0] - m[0] > kRescaleThreshold || mx[1] - m[1] > kRescaleThreshold;
        if (__any_sync(0xffffffffu, need)) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float to = fmaxf(m[i], mx[i]), alpha = fast_exp2(m[i] - to);
            m[i] = to;
            l[i] *= alpha;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
              o[n][2 * i] *= alpha;
              o[n][2 * i + 1] *= alpha;
            }
          }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            c[n][i] = fast_exp2(c[n][i] - m[i >> 1]);
            l[i >> 1] += c[n][i];
          }
        const uint32_t p[4] = {pack2<F16>(c[0][0], c[0][1]), pack2<F16>(c[0][2], c[0][3]),
                               pack2<F16>(c[1][0], c[1][1]), pack2<F16>(c[1][2], c[1][3])};
        if (masked) {
          bool bad = false;
          uint4* vv[kHalves];
#pragma unroll
          for (int hf = 0; hf < kHalves; ++hf) {
            vv[hf] = reinterpret_cast<uint4*>(sm.v[st][hf] + warp * 16 * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint4 x = vv[hf][lane + 32 * i];
              bad |= nonfinite2<F16>(x.x) || nonfinite2<F16>(x.y) || nonfinite2<F16>(x.z) || nonfinite2<F16>(x.w);
            }
          }
          if (__any_sync(0xffffffffu, bad)) {
#pragma unroll 1
            for (int key = 0; key < 16; ++key) {
#pragma unroll
              for (int n = 0; n < D / 8; ++n) {
                const uint32_t at = vb + (n >> 3) * (kBN * 128) + key * 128 + (((n & 7) ^ (key & 7)) << 4) + 4 * tq;
                uint32_t w;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
                const float2 x = unpack2<F16>(w);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  if (key0 + key >= lim[i]) continue;
                  if (!isfinite(x.x)) o[n][2 * i] += x.x;
                  if (!isfinite(x.y)) o[n][2 * i + 1] += x.y;
                }
              }
            }
            __syncwarp();
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint4 x = vv[hf][lane + 32 * i];
                x.x = finite2<F16>(x.x);
                x.y = finite2<F16>(x.y);
                x.z = finite2<F16>(x.z);
                x.w = finite2<F16>(x.w);
                vv[hf][lane + 32 * i] = x;
              }
            __syncwarp();
          }
        }
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
          uint32_t b[4];
          const int chunk = 2 * (n & 3) + v_chunk;
          ldmatrix4_trans(b, vb + (n >> 2) * (kBN * 128) + v_key * 128 + ((chunk ^ (v_key & 7)) << 4));
          mma16816<F16>(o[2 * n], p, b[0], b[1]);
          mma16816<F16>(o[2 * n + 1], p, b[2], b[3]);
        }
        if (masked) fence_proxy_async_smem();  // the zeros written above, before the next copy
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.empty[st]);
      }
      // Join the four warps: common maximum, sums, then O through shared memory (2, 3 into 0, 1;
      // 1 into 0: always in this order).  A warp that gave up waiting takes all along.
      float f[2], L[2] = {0.f, 0.f}, M[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        if (tq == 0) sm.ml[warp][r0 + 8 * i] = make_float2(m[i], l[i]);
      }
      if (compute_any(!ok)) break;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        M[i] = kUnset;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M[i] = fmaxf(M[i], sm.ml[w][r0 + 8 * i].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 x = sm.ml[w][r0 + 8 * i];
          L[i] = fmaf(x.y, fast_exp2(x.x - M[i]), L[i]);
        }
        f[i] = fast_exp2(m[i] - M[i]);
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][2 * i] *= f[i];
          o[n][2 * i + 1] *= f[i];
        }
      }
#pragma unroll
      for (int hf = 0; hf < kHalves; ++hf) {
        auto put = [&](float (*dst)[64 + 8]) {
#pragma unroll
          for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              *reinterpret_cast<float2*>(&dst[r0 + 8 * i][8 * n + 2 * tq]) =
                  make_float2(o[8 * hf + n][2 * i], o[8 * hf + n][2 * i + 1]);
        };
        auto add = [&](float (*src)[64 + 8]) {
#pragma unroll
          for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float2 x = *reinterpret_cast<const float2*>(&src[r0 + 8 * i][8 * n + 2 * tq]);
              o[8 * hf + n][2 * i] += x.x;
              o[8 * hf + n][2 * i + 1] += x.y;
            }
        };
        if (hf > 0) compute_barrier();  // warp 0 has read the first half
        if (warp >= 2) put(sm.o[warp - 2]);
        compute_barrier();
        if (warp < 2) add(sm.o[warp]);
        if (warp == 1) put(sm.o[1]);
        compute_barrier();
        if (warp == 0) add(sm.o[1]);
      }
      if (warp == 0) {
        if (!sg.part) {  // the whole item
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!valid[i]) continue;
            const float inv = 1.f / L[i];
            uint16_t* out = prm.out + (int64_t)(s.q0 + tok[i]) * prm.out_stride + head[i] * D + 2 * tq;
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
              *reinterpret_cast<uint32_t*>(out + 8 * n) =
                  lim[i] > 0 ? pack2<F16>(o[n][2 * i] * inv, o[n][2 * i + 1] * inv) : 0u;
            if (prm.lse && tq == 0)
              prm.lse[(size_t)(s.q0 + tok[i]) * prm.Hq + head[i]] =
                  lim[i] > 0 ? (M[i] + log2f(L[i])) * 0.69314718055994531f : -INFINITY;
          }
        } else {
          const size_t slot = 2 * cta + (u == begin ? 0 : 1);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const size_t r = slot * kRows + r0 + 8 * i;
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
              *reinterpret_cast<float2*>(sc.part_o + r * D + 8 * n + 2 * tq) =
                  make_float2(o[n][2 * i], o[n][2 * i + 1]);
            if (tq == 0) sc.part_ml[r] = make_float2(M[i], L[i]);
          }
        }
      }
      u = sg.item0 + pl.item();
      if (u < end && u - pl.base >= pl.extent(Hkv)) advance(prm, &pl);
    }
  }
}

template <int D, bool F16, bool kPaged>
cudaError_t launch_rows(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st) {
  using C = RowsCfg<D>;
  CUtensorMap mk, mv;
  cudaError_t e = make_kv_maps(a, kBN, &mk, &mv);
  if (e != cudaSuccess) return e;
  const int P = C::kPerSm * (num_sms < kMaxCtas ? num_sms : kMaxCtas);
  constexpr int smem = (int)sizeof(RowsSmem<D>) + 1024;
  const void* fn = reinterpret_cast<const void*>(seq_rows_kernel<D, F16, kPaged>);
  e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  SeqAttnArgs aa = a;
  SeqScratch ss = sc;
  bool whole = rows_whole(a, P);
  int cost = whole && count_items(a, kRows) <= P ? kWholeCost : kItemCost;
  void* args[] = {&mk, &mv, &aa, &ss, &cost, &whole};
  e = launch_pdl(fn, dim3(P), kThreads, smem, st, args);
  if (e != cudaSuccess || whole) return e;
  return launch_seq_join(a, sc, false, P, st);
}

}  // namespace

cudaError_t launch_seq_rows(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st) {
  using Launch = cudaError_t (*)(const SeqAttnArgs&, const SeqScratch&, int, cudaStream_t);
  static const Launch table[2][2][2] = {
      {{launch_rows<64, false, false>, launch_rows<64, false, true>},
       {launch_rows<64, true, false>, launch_rows<64, true, true>}},
      {{launch_rows<128, false, false>, launch_rows<128, false, true>},
       {launch_rows<128, true, false>, launch_rows<128, true, true>}}};
  return table[a.d == 128][a.fp16 != 0][a.kv.k != nullptr](a, sc, num_sms, st);
}

}  // namespace vp
