// Softmax attention of packed sequences, over themselves (vp_prompt_attention) or over the paged
// cache (vp_paged_attention), on the sm_103a tensor cores: o = sum_j p_j v_j / sum_j p_j over the
// keys j < lim(i) that row (token i, head h) sees, p_j = 2^(s_j - m), s_j = scale log2(e) q . k_j.
//
// Three kernels, chained by programmatic dependent launch:
//   seq_plan_kernel     one CTA reads the lengths and lists the work.  A tile is kChains x (128 /
//       group) tokens of a sequence with all heads of one kv head's group (row = token x group +
//       head, so K and V are read once for the group).  Tiles whose keys are more than an even
//       share (half of the total over the CTAs) are cut along the keys into pieces of
//       at most that, and the list is ordered by length, longest first.
//   seq_tile_kernel     persistent CTAs, one per SM, take items of the list (x kv heads) back and
//       forth: CTA c the items c, 2 P - 1 - c, 2 P + c, ... of P CTAs, which evens out a list in
//       descending order without a counter.
//   seq_combine_kernel  joins the pieces of cut tiles, one warp per row, in the pieces' order.
//
// The tile kernel.  The kChains 128-row tiles of an item run as independent chains that share the
// K / V ring (64 keys per tile): the tensor core works for one chain while another's softmax runs.
//   warp 0               TMA: Q once per item; K / V tiles, page by page, page ids read a window of
//                        32 ahead by the lanes.
//   warps 1 .. kChains   one elected lane issues a chain's tcgen05.mma: S = Q K^T (128 x 64, fp32 in
//                        TMEM), O += P V (P read from TMEM as 16-bit pairs).
//   warps 4 ..           four softmax warps per chain, a row per thread; the running maximum
//                        is moved only when it grows by more than 2^8 (exact either way).
// A chain stops at its own last visible key; the tiles after it are only released.  A tile that
// some row of the item sees in part takes the masked path: scores past a row's limit become -inf
// by selection, and V values that are not finite are replaced by 0 in shared memory, since
// 0 x inf would reach rows that do not see them; rows that do see them get them added back in
// the epilogue (a flag says whether there were any).
// Scores, maxima, sums and outputs are held in 32 bits; P is rounded to the storage type, as the
// tensor core needs.  Every wait is bounded; a CTA that gives up lets its copies and MMAs land.
#include <math.h>

#include "seq.h"

namespace vp {

namespace {

constexpr int kBM = 128;   // rows of a chain
constexpr int kBN = 64;    // keys of a tile
constexpr float kUnset = -1e30f;           // running maximum before the first visible key
constexpr float kRescaleThreshold = 8.f;   // log2 units

// Counts in SeqScratch::head.
constexpr int kPlanItems = 0, kPlanSplits = 1;
constexpr int kPlanThreads = 1024;
constexpr int kBuckets = 512;

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// The sequence's keys that rows up to the last of [t0, t0 + n) see, in tiles.
__device__ __forceinline__ int tiles_seen(int last_token, const Seq& s, int block) {
  const int lim = row_limit(last_token, s.ql, s.kl, block);
  return lim > 0 ? ceil_div(lim, kBN) : 0;
}

// Inclusive scan over the CTA's kPlanThreads values; *total: their sum.
__device__ __forceinline__ int block_scan(int v, int* s_warp, int* total) {
  const int lane = lane_id(), w = warp_id();
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, k);
    if (lane >= k) v += u;
  }
  __syncthreads();
  if (lane == 31) s_warp[w] = v;
  __syncthreads();
  if (w == 0) {
    int x = s_warp[lane];
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, x, k);
      if (lane >= k) x += u;
    }
    s_warp[lane] = x;
  }
  __syncthreads();
  *total = s_warp[31];
  return v + (w ? s_warp[w - 1] : 0);
}

// tokens: of a tile (all chains); ctas: of the tile kernel; min_piece: a piece's least key tiles.
__global__ void __launch_bounds__(kPlanThreads) seq_plan_kernel(SeqAttnArgs a, SeqScratch sc,
                                                                int tokens, int ctas,
                                                                int min_piece) {
  __shared__ int s_warp[32], s_hist[kBuckets], s_slots, s_splits;
  __shared__ unsigned long long s_work;
  pdl_launch_dependents();
  const int tid = threadIdx.x;
  if (tid == 0) {
    s_work = 0;
    s_slots = s_splits = 0;
    sc.tile_off[0] = 0;
  }
  if (tid < kBuckets) s_hist[tid] = 0;
  int n_tiles = 0;
  for (int base = 0; base < a.B; base += kPlanThreads) {
    const int b = base + tid;
    const int n = b < a.B ? ceil_div(load_seq(a, b).ql, tokens) : 0;
    int total;
    const int before = block_scan(n, s_warp, &total);
    if (b < a.B) sc.tile_off[b + 1] = n_tiles + before;
    n_tiles += total;
  }
  __syncthreads();
  // Tile w: sequence b, first token t0, key tiles nk.
  auto tile = [&](int w, int* b, int* t0, Seq* s) {
    *b = seq_of_token(sc.tile_off, a.B, w);
    *s = load_seq(a, *b);
    *t0 = (w - sc.tile_off[*b]) * tokens;
    return tiles_seen(min(*t0 + tokens, s->ql) - 1, *s, a.block);
  };
  int b, t0;
  Seq s;
  unsigned long long work = 0;
  for (int w = tid; w < n_tiles; w += kPlanThreads) work += tile(w, &b, &t0, &s);
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) work += __shfl_xor_sync(0xffffffffu, work, k);
  if (lane_id() == 0) atomicAdd(&s_work, work);
  __syncthreads();
  const unsigned long long share = (s_work * a.Hkv + 2 * ctas - 1) / (2 * ctas);
  const int piece = (int)max((unsigned long long)min_piece, share);
  // Pieces of n tiles each (or one less), longest first.
  auto bucket = [&](int nk, int np) {
    return kBuckets - 1 - (int)((long long)ceil_div(nk, np) * (kBuckets - 1) / piece);
  };
  for (int w = tid; w < n_tiles; w += kPlanThreads) {
    const int nk = tile(w, &b, &t0, &s), np = max(1, ceil_div(nk, piece));
    atomicAdd(&s_hist[bucket(nk, np)], np);
  }
  __syncthreads();
  int total;
  const int mine = tid < kBuckets ? s_hist[tid] : 0;
  const int before = block_scan(mine, s_warp, &total) - mine;
  __syncthreads();
  if (tid < kBuckets) s_hist[tid] = before;
  __syncthreads();
  for (int w = tid; w < n_tiles; w += kPlanThreads) {
    const int nk = tile(w, &b, &t0, &s), np = max(1, ceil_div(nk, piece));
    const int at = atomicAdd(&s_hist[bucket(nk, np)], np);
    int slot = -1;
    if (np > 1) {
      slot = atomicAdd(&s_slots, np);
      const int r = atomicAdd(&s_splits, 1);
      sc.splits[2 * r] = make_int4(s.q0, t0, s.ql, s.kl);
      sc.splits[2 * r + 1] = make_int4(slot, np, 0, 0);
    }
    for (int i = 0; i < np; ++i) {
      const int j0 = (int)((long long)i * nk / np), j1 = (int)((long long)(i + 1) * nk / np);
      sc.items[2 * (at + i)] = make_int4(b, t0, j0, j1 - j0);
      sc.items[2 * (at + i) + 1] = make_int4(slot < 0 ? -1 : slot + i, s.q0, s.ql, s.kl);
    }
  }
  __syncthreads();
  if (tid == 0) {
    sc.head[kPlanItems] = total;
    sc.head[kPlanSplits] = s_splits;
  }
}

// ------------------------------------------------------------------ tile kernel
template <int D>
struct Cfg {
  static constexpr int kChains = seq_chains(D);
  static constexpr int kHalves = D / 64;               // 64-channel (128-byte) column blocks
  static constexpr int kStages = 512 / kBN / kHalves;  // 64 KB of K and 64 KB of V
  static constexpr int kThreads = 128 + 128 * kChains;
  static constexpr int kCtrlRegs = kChains == 3 ? 56 : 80;
  static constexpr int kSoftRegs = kChains == 3 ? 152 : 208;
  static_assert(128 * kCtrlRegs + 128 * kChains * kSoftRegs <= 65536, "register split");
  // TMEM columns: S_c (fp32), O_c (fp32), P_c (16-bit pairs) of every chain.
  static constexpr uint32_t kColS = 0, kColO = kChains * kBN, kColP = kColO + kChains * D;
  static_assert(kColP + kChains * kBN / 2 <= 512, "TMEM columns");
};

template <int D>
struct TileSmem {
  using C = Cfg<D>;
  uint16_t q[C::kChains][C::kHalves][kBM * 64];
  uint16_t k[C::kStages][C::kHalves][kBN * 64];
  uint16_t v[C::kStages][C::kHalves][kBN * 64];
  uint64_t q_full, q_empty;
  uint64_t k_full[C::kStages], v_full[C::kStages], kv_empty[C::kStages];
  uint64_t s_full[C::kChains], s_empty[C::kChains], p_full[C::kChains], o_bar[C::kChains],
      o_empty[C::kChains], drain[C::kChains];
  uint32_t tmem_base;
  int abort_flag;
  int nonfinite;  // some visible V of a masked tile was not finite
};

struct Item {
  int b, t0, j0, nk, slot, q0, ql, kl, h;
};

__device__ __forceinline__ Item load_item(const SeqScratch& sc, int idx, int Hkv) {
  const int e = idx / Hkv;
  const int4 x = sc.items[2 * e], y = sc.items[2 * e + 1];
  Item it;
  it.b = x.x;
  it.t0 = x.y;
  it.j0 = x.z;
  it.nk = x.w;
  it.slot = y.x;
  it.q0 = y.y;
  it.ql = y.z;
  it.kl = y.w;
  it.h = idx - e * Hkv;
  return it;
}

// The n-th item of this CTA (see the top): c, 2 P - 1 - c, 2 P + c, 4 P - 1 - c, ...
__device__ __forceinline__ int item_index(int n, int cta, int P) {
  return n * P + ((n & 1) ? P - 1 - cta : cta);
}

// Key tiles [j0, j0 + n) of an item that chain c takes (tpt tokens per chain).
__device__ __forceinline__ int chain_tiles(const Item& it, int c, int tpt, int block) {
  const int first = it.t0 + c * tpt, last = min(first + tpt, it.ql) - 1;
  if (last < first) return 0;
  const Seq s{it.q0, it.ql, it.kl};
  return min(max(tiles_seen(last, s, block) - it.j0, 0), it.nk);
}

template <bool F16>
__host__ __device__ constexpr uint32_t idesc_16bit(int M, int N, int b_mn) {
  // D fp32; A and B bf16 (1) or fp16 (0); A K-major, B K-major or MN-major
  return (1u << 4) | ((F16 ? 0u : 1u) << 7) | ((F16 ? 0u : 1u) << 10) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Replaces what is not finite in the 64 V rows of a tile by 0 (the chain's 128 threads, 16 bytes
// each in turn); sets *flag if a row below n_valid held any.
template <int D, bool F16>
__device__ __forceinline__ void scrub_v(uint16_t* v, int n_valid, int tid, volatile int* flag) {
  uint4* p = reinterpret_cast<uint4*>(v);
#pragma unroll
  for (int i = 0; i < kBN * D / 8 / 128; ++i) {
    const int e = tid + 128 * i;
    uint4 x = p[e];
    if (nonfinite2<F16>(x.x) || nonfinite2<F16>(x.y) || nonfinite2<F16>(x.z) || nonfinite2<F16>(x.w)) {
      if (((e >> 3) & (kBN - 1)) < n_valid) *flag = 1;  // rows of 8 vectors, kBN rows a half
      __threadfence_block();
      x.x = finite2<F16>(x.x);
      x.y = finite2<F16>(x.y);
      x.z = finite2<F16>(x.z);
      x.w = finite2<F16>(x.w);
      p[e] = x;
    }
  }
  fence_proxy_async_smem();
}

// o[0 .. 32) += the values that are not finite among channels [c0, c0 + 32) of the keys [j0, j1).
template <int D, bool F16, bool kPaged>
__device__ __forceinline__ void add_nonfinite(const SeqAttnArgs& a, int b, int q0, int h, int c0,
                                              int j0, int j1, float (&o)[32]) {
#pragma unroll 1
  for (int j = j0; j < j1; ++j) {
    const uint16_t* row;
    if constexpr (kPaged) {
      const int page = a.kv.table[(size_t)b * a.kv.width + (j >> a.kv.log2_page)];
      if ((unsigned)page >= (unsigned)a.kv.n_pages) continue;
      row = a.kv.v + (((((long long)page * a.Hkv + h) << a.kv.log2_page)) + (j & (a.kv.page_size - 1))) * D;
    } else {
      row = a.v + (long long)(q0 + j) * a.v_stride + h * D;
    }
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      const float2 x = unpack2<F16>(*reinterpret_cast<const uint32_t*>(row + c0 + c));
      if (!isfinite(x.x)) o[c] += x.x;
      if (!isfinite(x.y)) o[c + 1] += x.y;
    }
  }
}

template <int D, bool F16, bool kPaged>
__global__ void __launch_bounds__(Cfg<D>::kThreads, 1)
    seq_tile_kernel(const __grid_constant__ CUtensorMap tmap_q,
                    const __grid_constant__ CUtensorMap tmap_k,
                    const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ SeqAttnArgs prm, const SeqScratch sc) {
  using C = Cfg<D>;
  constexpr int kChains = C::kChains, kStages = C::kStages, kHalves = C::kHalves;
  extern __shared__ unsigned char smem_raw[];
  TileSmem<D>& sm = *reinterpret_cast<TileSmem<D>*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int P = gridDim.x, cta = blockIdx.x;
  const int warp = warp_uniform_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  unsigned int* err = prm.err;
  pdl_launch_dependents();

  if (threadIdx.x == 0) {
    mbar_init(&sm.q_full, 1);
    mbar_init(&sm.q_empty, kChains);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.kv_empty[s], kChains);
    }
    for (int c = 0; c < kChains; ++c) {
      mbar_init(&sm.s_full[c], 1);
      mbar_init(&sm.s_empty[c], 128);
      mbar_init(&sm.p_full[c], 128);
      mbar_init(&sm.o_bar[c], 1);
      mbar_init(&sm.o_empty[c], 128);
      mbar_init(&sm.drain[c], 1);
    }
    sm.abort_flag = 0;
    sm.nonfinite = 0;
    fence_mbarrier_init();
    fence_proxy_async_smem();
    tma_prefetch_desc(&tmap_q);
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem_base, 0);

  pdl_wait();  // the plan
  const int Hkv = prm.Hkv, group = prm.group, block = prm.block;
  const int tpt = kBM / group;  // tokens of a chain
  const int n_items = sc.head[kPlanItems] * Hkv;

  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kCtrlRegs));
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    uint32_t lc = 0, ic = 0;
    bool ok = true;
    const int log2p = prm.kv.log2_page, ps = prm.kv.page_size;
    const int ppt = kPaged ? (ps >= kBN ? 1 : kBN / ps) : 1;  // pages (boxes) of a tile
    const uint32_t box_bytes = (kPaged && ps < kBN ? ps : kBN) * 128;
    for (int idx; ok && (idx = item_index(ic, cta, P)) < n_items; ++ic) {
      const Item it = load_item(sc, idx, Hkv);
      ok = mbar_wait_warp(&sm.q_empty, (ic & 1) ^ 1, err, abort_flag);
      if (!ok) break;
      const int chains = min(kChains, ceil_div(it.ql - it.t0, tpt));
      if (elect_one()) {
        mbar_arrive_expect_tx(&sm.q_full, chains * kHalves * tpt * group * 128);
        for (int c = 0; c < chains; ++c)
#pragma unroll
          for (int hf = 0; hf < kHalves; ++hf)
            tma_load_4d(sm.q[c][hf], &tmap_q, &sm.q_full, hf * 64, 0, it.h, it.q0 + it.t0 + c * tpt);
      }
      __syncwarp();
      // Page ids: lane l holds that of page first + l; `next` the 32 after them.
      const int n_pages = kPaged ? (it.kl + ps - 1) >> log2p : 0;
      const int32_t* table = kPaged ? prm.kv.table + (size_t)it.b * prm.kv.width : nullptr;
      int first = kPaged ? (it.j0 * kBN) >> log2p : 0, window = 0, next = 0;
      if (kPaged) {
        if (first + lane < n_pages) window = table[first + lane];
        if (first + 32 + lane < n_pages) next = table[first + 32 + lane];
      }
      for (int jj = 0; jj < it.nk; ++jj, ++lc) {
        const int j = it.j0 + jj, st = lc % kStages;
        int y = it.q0 + j * kBN, page = 0, n_box = 1;
        if (kPaged) {
          const int p0 = (j * kBN) >> log2p;
          if (p0 >= first + 32) {
            first += 32;
            window = next;
            next = first + 32 + lane < n_pages ? table[first + 32 + lane] : 0;
          }
          n_box = min(ppt, n_pages - p0);  // the pages that exist; the rest of the tile is masked
          page = __shfl_sync(0xffffffffu, window, (p0 - first + lane) & 31);
          y = (j * kBN) & (ps - 1);
          if (lane < n_box && (unsigned)page >= (unsigned)prm.kv.n_pages) atomicOr(err, VP_DEVERR_PAGE);
        }
        ok = mbar_wait_warp(&sm.kv_empty[st], ((lc / kStages) & 1) ^ 1, err, abort_flag);
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&sm.k_full[st], n_box * kHalves * box_bytes);
          mbar_arrive_expect_tx(&sm.v_full[st], n_box * kHalves * box_bytes);
        }
        __syncwarp();
        if (lane < n_box) {
          const int off = lane * (box_bytes / 2);
#pragma unroll
          for (int hf = 0; hf < kHalves; ++hf)
            tma_load_4d(sm.k[st][hf] + off, &tmap_k, &sm.k_full[st], hf * 64, y, it.h, page);
#pragma unroll
          for (int hf = 0; hf < kHalves; ++hf)
            tma_load_4d(sm.v[st][hf] + off, &tmap_v, &sm.v_full[st], hf * 64, y, it.h, page);
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) {
      // Let the copies this warp issued land before the CTA releases its shared memory.
      if (ic > 0)
        for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.q_full, (ic - 1) & 1); ++t) {}
      for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.q_full, ic & 1); ++t) {}
      for (int s = 0; s < kStages; ++s) {
        if (lc > (uint32_t)s) {
          const uint32_t last = (lc - 1 - s) / kStages * kStages + s;  // last use of stage s
          const uint32_t par = (last / kStages) & 1;
          for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.k_full[s], par); ++t) {}
          for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.v_full[s], par); ++t) {}
        }
      }
    }
  } else if (warp <= kChains) {
    // ------------------------------------------------------------ MMA issuers (chain c)
    const int c = warp - 1;
    const uint32_t id_s = idesc_16bit<F16>(kBM, kBN, 0);  // Q (K-major) x K^T (K-major)
    const uint32_t id_o = idesc_16bit<F16>(kBM, 64, 1);   // P (TMEM) x V (MN-major)
    const uint64_t dq = sdesc_sw128(smem_u32(sm.q[c][0]));
    const uint32_t t_s = tmem + C::kColS + c * kBN;
    const uint32_t t_o = tmem + C::kColO + c * D;
    const uint32_t t_p = tmem + C::kColP + c * (kBN / 2);
    uint32_t lc = 0, ic = 0, g = 0, oc = 0;  // ring tiles, items, this chain's tiles, its items
    bool ok = true;
    Item it;
    int idx = item_index(0, cta, P);
    if (idx < n_items) it = load_item(sc, idx, Hkv);
    for (; ok && idx < n_items; ++ic) {
      const int nk = it.nk, n = chain_tiles(it, c, tpt, block);
      idx = item_index(ic + 1, cta, P);
      if (idx < n_items) it = load_item(sc, idx, Hkv);  // ahead of its use
      ok = mbar_wait_warp(&sm.q_full, ic & 1, err, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint32_t lc0 = lc, g0 = g;
      auto issue_s = [&](int j) -> bool {
        const uint32_t l = lc0 + j, gg = g0 + j;
        const int st = l % kStages;
        if (!mbar_wait_warp(&sm.k_full[st], (l / kStages) & 1, err, abort_flag)) return false;
        if (!mbar_wait_warp(&sm.s_empty[c], (gg & 1) ^ 1, err, abort_flag)) return false;
        tc_fence_after();
        const uint64_t dk = sdesc_sw128(smem_u32(sm.k[st][0]));
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)  // K = 16 per step: +32 bytes, +1 block per 64
            tc_mma_ss(t_s, dq + (kk >> 2) * (kBM * 128 / 16) + 2 * (kk & 3),
                      dk + (kk >> 2) * (kBN * 128 / 16) + 2 * (kk & 3), id_s, kk > 0);
          tc_commit(&sm.s_full[c]);
          if (j == n - 1) tc_commit(&sm.q_empty);
        }
        __syncwarp();
        return true;
      };
      if (n > 0) {
        ok = issue_s(0);
      } else if (lane == 0) {
        mbar_arrive(&sm.q_empty);
      }
      for (int j = 0; j < n && ok; ++j) {
        if (j + 1 < n) {
          ok = issue_s(j + 1);  // as soon as the softmax has read S_c(j)
          if (!ok) break;
        }
        const uint32_t l = lc0 + j, gg = g0 + j;
        const int st = l % kStages;
        ok = mbar_wait_warp(&sm.p_full[c], gg & 1, err, abort_flag) &&
             mbar_wait_warp(&sm.v_full[st], (l / kStages) & 1, err, abort_flag) &&
             (j > 0 || mbar_wait_warp(&sm.o_empty[c], (oc & 1) ^ 1, err, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint64_t dv = sdesc_sw128(smem_u32(sm.v[st][0]));
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kBN / 16; ++kk)  // 16 keys per step: 8 TMEM columns, 2 KB of V
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf)
              tc_mma_ts(t_o + 64 * hf, t_p + 8 * kk, dv + hf * (kBN * 128 / 16) + (uint64_t)(kk * 128),
                        id_o, (j > 0 || kk > 0) ? 1u : 0u);
          tc_commit(&sm.o_bar[c]);
          tc_commit(&sm.kv_empty[st]);
        }
        __syncwarp();
      }
      // The item's tiles past this chain's last visible key: released once they have landed.
      for (int j = n; j < nk && ok; ++j) {
        const uint32_t l = lc0 + j;
        const int st = l % kStages;
        ok = mbar_wait_warp(&sm.k_full[st], (l / kStages) & 1, err, abort_flag) &&
             mbar_wait_warp(&sm.v_full[st], (l / kStages) & 1, err, abort_flag);
        if (ok && lane == 0) mbar_arrive(&sm.kv_empty[st]);
      }
      lc = lc0 + nk;
      g = g0 + n;
      oc += n > 0;
    }
    if (!ok) {
      if (elect_one()) {
        tc_commit(&sm.drain[c]);
        for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.drain[c], 0); ++t) {}
      }
      __syncwarp();
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ softmax / epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftRegs));
    const int c = (warp - 4) >> 2;  // chain
    const int quarter = warp & 3;   // TMEM lane quarter this warp may access
    const int row = quarter * 32 + lane;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem + lane_off + C::kColS + c * kBN;
    const uint32_t t_o = tmem + lane_off + C::kColO + c * D;
    const uint32_t t_p = tmem + lane_off + C::kColP + c * (kBN / 2);
    const int row_tok = row / group, row_head = row - row_tok * group;
    const bool flip = prm.scale_log2 < 0.f;  // scores are negated, so that the maximum is the scores'
    const float cs = fmaxf(fabsf(prm.scale_log2), 1e-30f);
    uint32_t g = 0, lc = 0;
    bool ok = true;
    for (int n_it = 0, idx; ok && (idx = item_index(n_it, cta, P)) < n_items; ++n_it) {
      const Item it = load_item(sc, idx, Hkv);
      const int n = chain_tiles(it, c, tpt, block);
      const int tok = it.t0 + c * tpt + row_tok;  // this thread's token in its sequence
      const bool valid = row_tok < tpt && tok < it.ql;
      const int lim = valid ? row_limit(tok, it.ql, it.kl, block) : 0;
      // Tiles from here on hide something from some row of the item (any chain).
      const int masked_from = max(row_limit(it.t0, it.ql, it.kl, block), 0) / kBN;
      const bool active = __any_sync(0xffffffffu, valid);
      float m = kUnset, lsum = 0.f;
      for (int jj = 0; jj < n; ++jj, ++g) {
        const int j = it.j0 + jj;
        const bool masked = j >= masked_from;  // uniform over the chain
        ok = mbar_wait_warp(&sm.s_full[c], g & 1, err, abort_flag);
        if (!ok) break;
        if (masked) {
          const uint32_t l = lc + jj;
          const int st = l % kStages;
          ok = mbar_wait_warp(&sm.v_full[st], (l / kStages) & 1, err, abort_flag);
          if (!ok) break;
          scrub_v<D, F16>(sm.v[st][0], it.kl - j * kBN, row, &sm.nonfinite);
        }
        tc_fence_after();
        if (!active) {  // no row of this warp exists: its lanes of P and O are never read
          tc_fence_before();
          mbar_arrive(&sm.s_empty[c]);
          if (g > 0) ok = mbar_wait_warp(&sm.o_bar[c], (g - 1) & 1, err, abort_flag);
          if (!ok) break;
          mbar_arrive(&sm.p_full[c]);
          continue;
        }
        float s[kBN], pmx[kBN / 32];
#pragma unroll
        for (int cc = 0; cc < kBN / 32; ++cc) tmem_ld32_max(t_s + 32 * cc, s + 32 * cc, pmx[cc]);
        tmem_wait_ld();
        tc_fence_before();
        mbar_arrive(&sm.s_empty[c]);  // the MMA warp may overwrite S_c now
        float mx = fmaxf(pmx[0], pmx[1]);
        if (masked || flip) {
          const int n_seen = lim - j * kBN;
#pragma unroll
          for (int i = 0; i < kBN; ++i) {
            if (flip) s[i] = -s[i];
            if (i >= n_seen) s[i] = -INFINITY;
          }
          float t[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = fmaxf(s[k], s[8 + k]);
#pragma unroll
          for (int i = 16; i < kBN; i += 16) {
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = fmax3(t[k], s[i + k], s[i + 8 + k]);
          }
          mx = fmaxf(fmax3(t[0], t[1], t[2]), fmax3(t[3], t[4], fmax3(t[5], t[6], t[7])));
        }
        const float mx2 = mx * cs;
        float alpha = 1.f;
        bool need = false;
        if (jj == 0) {
          m = fmaxf(mx2, kUnset);
        } else if (mx2 > m + kRescaleThreshold) {
          need = true;
          alpha = fast_exp2(m - mx2);
          m = mx2;
        }
        const float2 c2 = make_float2(cs, cs), nm = make_float2(-m, -m);
        float2 acc0 = make_float2(0.f, 0.f), acc1 = make_float2(0.f, 0.f);
        uint32_t pk[kBN / 2];
#pragma unroll
        for (int i = 0; i < kBN / 2; ++i) {
          float2 x = ffma2(make_float2(s[2 * i], s[2 * i + 1]), c2, nm);
          x.x = fast_exp2(x.x);
          x.y = fast_exp2(x.y);
          pk[i] = pack2<F16>(x.x, x.y);
          if (i & 1)
            acc1 = fadd2(acc1, x);
          else
            acc0 = fadd2(acc0, x);
        }
        const float2 at = fadd2(acc0, acc1);
        lsum = lsum * alpha + (at.x + at.y);
        // P_c and O_c are free once P_c(g-1) V has completed.
        if (g > 0) {
          ok = mbar_wait_warp(&sm.o_bar[c], (g - 1) & 1, err, abort_flag);
          if (!ok) break;
          tc_fence_after();
        }
#pragma unroll
        for (int cc = 0; cc < kBN / 32; ++cc) tmem_st16(t_p + 16 * cc, pk + 16 * cc);
        if (__any_sync(0xffffffffu, need)) {
#pragma unroll
          for (int q = 0; q < D / 32; ++q) {
            float o[32];
            tmem_ld32(t_o + 32 * q, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= alpha;
            tmem_st32(t_o + 32 * q, o);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sm.p_full[c]);
      }
      if (!ok) break;
      lc += it.nk;
      if (n > 0) {
        ok = mbar_wait_warp(&sm.o_bar[c], (g - 1) & 1, err, abort_flag);
        if (!ok) break;
        tc_fence_after();
        __threadfence_block();
      }
      const bool refill = n > 0 && *(volatile int*)&sm.nonfinite != 0;
      const int head = it.h * group + row_head;
      if (it.slot >= 0) {  // a piece: unnormalised O, m and l
        const size_t r = ((size_t)(it.slot * Hkv + it.h) * kChains + c) * kBM + row;
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          if (n == 0) break;
          float o[32];
          tmem_ld32(t_o + 32 * q, o);
          tmem_wait_ld();
          if (q == D / 32 - 1) {
            tc_fence_before();
            mbar_arrive(&sm.o_empty[c]);
          }
          if (!valid) continue;
          if (refill)
            add_nonfinite<D, F16, kPaged>(prm, it.b, it.q0, it.h, 32 * q, max(it.j0, masked_from) * kBN,
                                          min(lim, (it.j0 + n) * kBN), o);
          float4* dst = reinterpret_cast<float4*>(sc.part_o + r * D + 32 * q);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
        if (valid) sc.part_ml[r] = make_float2(m, lsum);
      } else {
        const float inv = 1.f / lsum;
        uint16_t* out = prm.out + (int64_t)(it.q0 + tok) * prm.out_stride + head * D;
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          float o[32];
          if (n > 0) {
            tmem_ld32(t_o + 32 * q, o);
            tmem_wait_ld();
            if (q == D / 32 - 1) {
              tc_fence_before();
              mbar_arrive(&sm.o_empty[c]);
            }
          }
          if (!valid) continue;
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = lim > 0 ? o[i] * inv : 0.f;
          if (refill)
            add_nonfinite<D, F16, kPaged>(prm, it.b, it.q0, it.h, 32 * q, max(it.j0, masked_from) * kBN,
                                          min(lim, (it.j0 + n) * kBN), o);
          uint4* dst = reinterpret_cast<uint4*>(out + 32 * q);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            dst[i] = make_uint4(pack2<F16>(o[8 * i], o[8 * i + 1]), pack2<F16>(o[8 * i + 2], o[8 * i + 3]),
                                pack2<F16>(o[8 * i + 4], o[8 * i + 5]),
                                pack2<F16>(o[8 * i + 6], o[8 * i + 7]));
        }
        if (valid && prm.lse)
          prm.lse[(size_t)(it.q0 + tok) * prm.Hq + head] =
              lim > 0 ? (m + log2f(lsum)) * 0.69314718055994531f : -INFINITY;
      }
      __syncwarp();
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------ pieces joined
constexpr int kCombineThreads = 256;

// One warp per row of a cut tile: M = max m_i, o = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i.
template <int D, bool F16>
__global__ void __launch_bounds__(kCombineThreads) seq_combine_kernel(SeqAttnArgs a, SeqScratch sc) {
  constexpr int kChains = seq_chains(D), kRows = kChains * kBM, kPer = D / 32;
  pdl_wait();
  const int n_splits = sc.head[kPlanSplits], Hkv = a.Hkv, tpt = kBM / a.group;
  const int lane = lane_id();
  const long long rows = (long long)n_splits * Hkv * kRows;
  const long long step = (long long)gridDim.x * (kCombineThreads / 32);
  for (long long w = (long long)blockIdx.x * (kCombineThreads / 32) + warp_id(); w < rows; w += step) {
    const int r = (int)(w % kRows), sh = (int)(w / kRows), h = sh % Hkv, sp = sh / Hkv;
    const int row = r % kBM, row_tok = row / a.group;
    const int4 x = sc.splits[2 * sp], y = sc.splits[2 * sp + 1];
    const int tok = x.y + (r / kBM) * tpt + row_tok;
    if (row_tok >= tpt || tok >= x.z) continue;
    const size_t pitch = (size_t)Hkv * kRows;  // rows between pieces
    const size_t r0 = ((size_t)y.x * Hkv + h) * kRows + r;
    const int np = y.y;
    float M = kUnset;
    for (int i = lane; i < np; i += 32) M = fmaxf(M, sc.part_ml[r0 + i * pitch].x);
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, k));
    float L = 0.f, o[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[c] = 0.f;
    for (int i0 = 0; i0 < np; i0 += 32) {
      float2 ml = make_float2(kUnset, 0.f);
      if (i0 + lane < np) ml = sc.part_ml[r0 + (i0 + lane) * pitch];
      const float wgt = fast_exp2(ml.x - M);
      const int n = min(32, np - i0);
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const float l = __shfl_sync(0xffffffffu, ml.y, i), f = __shfl_sync(0xffffffffu, wgt, i);
        if (l == 0.f) continue;  // nothing visible in this piece (its O may be unwritten)
        L = fmaf(f, l, L);
        const float* src = sc.part_o + (r0 + (i0 + i) * pitch) * D + lane * kPer;
#pragma unroll
        for (int c = 0; c < kPer; ++c) o[c] = fmaf(f, src[c], o[c]);
      }
    }
    const int lim = row_limit(tok, x.z, x.w, a.block);
    const float inv = 1.f / L;
    const int head = h * a.group + row - row_tok * a.group;
    uint16_t* out = a.out + (int64_t)(x.x + tok) * a.out_stride + head * D + lane * kPer;
#pragma unroll
    for (int c = 0; c < kPer; c += 2)
      *reinterpret_cast<uint32_t*>(out + c) =
          lim > 0 ? pack2<F16>(o[c] * inv, o[c + 1] * inv) : 0u;
    if (a.lse && lane == 0)
      a.lse[(size_t)(x.x + tok) * a.Hq + head] =
          lim > 0 ? (M + log2f(L)) * 0.69314718055994531f : -INFINITY;
  }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct ScratchLayout {
  size_t items, splits, tile_off, part_ml, part_o, end;
};
ScratchLayout scratch_layout(int d, int Hq, int Hkv, int64_t T, int64_t B) {
  const int chains = seq_chains(d), tokens = chains * (kBM / (Hq / Hkv));
  const int64_t tiles = T / tokens + B;  // sum of ceil(n / tokens)
  ScratchLayout l;
  l.items = 512;  // after the error word and the counts
  l.splits = l.items + align256((size_t)(tiles + kMaxSlots) * 2 * sizeof(int4));
  l.tile_off = l.splits + align256((size_t)kMaxSlots * 2 * sizeof(int4));
  l.part_ml = l.tile_off + align256((size_t)(B + 1) * sizeof(int));
  l.part_o = l.part_ml + align256((size_t)kMaxSlots * chains * kBM * sizeof(float2));
  l.end = l.part_o + align256((size_t)kMaxSlots * chains * kBM * d * sizeof(float));
  return l;
}

template <int D, bool F16, bool kPaged>
cudaError_t launch_tiles(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st) {
  using C = Cfg<D>;
  CUtensorMap mq, mk, mv;
  const uint64_t g = a.group, H = a.Hkv;
  const int tpt = kBM / a.group;
  const uint64_t qd[4] = {D, g, H, (uint64_t)a.T};
  const uint64_t qs[3] = {D, g * D, (uint64_t)a.q_stride};
  const uint32_t qb[4] = {64, (uint32_t)g, 1, (uint32_t)tpt};
  cudaError_t e = make_tmap_16bit_4d(&mq, a.q, F16, qd, qs, qb);
  if (e != cudaSuccess) return e;
  e = make_kv_maps(a, kBN, &mk, &mv);
  if (e != cudaSuccess) return e;
  const int P = num_sms < kMaxCtas ? num_sms : kMaxCtas;
  constexpr int smem = (int)sizeof(TileSmem<D>) + 1024;
  const void* tile = reinterpret_cast<const void*>(seq_tile_kernel<D, F16, kPaged>);
  e = cudaFuncSetAttribute(tile, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  // A piece has at least 16 tiles (1,024 keys): below that its start and its join outweigh it.
  seq_plan_kernel<<<1, kPlanThreads, 0, st>>>(a, sc, C::kChains * tpt, P, 16);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  SeqAttnArgs aa = a;
  SeqScratch ss = sc;
  void* targs[] = {&mq, &mk, &mv, &aa, &ss};
  e = launch_pdl(tile, P, C::kThreads, smem, st, targs);
  if (e != cudaSuccess) return e;
  void* cargs[] = {&aa, &ss};
  prof_extra_launch();
  prof_extra_launch();
  return launch_pdl(reinterpret_cast<const void*>(seq_combine_kernel<D, F16>), 2 * P, kCombineThreads, 0,
                    st, cargs);
}

}  // namespace

cudaError_t launch_pdl(const void* fn, int grid, int threads, int smem, cudaStream_t st, void** args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelExC(&cfg, fn, args);
}

cudaError_t make_kv_maps(const SeqAttnArgs& a, int tile_keys, CUtensorMap* mk, CUtensorMap* mv) {
  const uint64_t d = a.d, H = a.Hkv;
  if (a.kv.k) {
    const uint64_t ps = a.kv.page_size;
    const uint64_t dims[4] = {d, ps, H, (uint64_t)a.kv.n_pages};
    const uint64_t strides[3] = {d, ps * d, H * ps * d};
    const uint32_t box[4] = {64, ps < (uint64_t)tile_keys ? (uint32_t)ps : (uint32_t)tile_keys, 1, 1};
    const cudaError_t e = make_tmap_16bit_4d(mk, a.kv.k, a.fp16 != 0, dims, strides, box);
    return e != cudaSuccess ? e : make_tmap_16bit_4d(mv, a.kv.v, a.fp16 != 0, dims, strides, box);
  }
  // Packed keys: one page of T rows.
  const uint64_t dims[4] = {d, (uint64_t)a.T, H, 1};
  const uint64_t ks[3] = {(uint64_t)a.k_stride, d, H * d}, vs[3] = {(uint64_t)a.v_stride, d, H * d};
  const uint32_t box[4] = {64, (uint32_t)tile_keys, 1, 1};
  const cudaError_t e = make_tmap_16bit_4d(mk, a.k, a.fp16 != 0, dims, ks, box);
  return e != cudaSuccess ? e : make_tmap_16bit_4d(mv, a.v, a.fp16 != 0, dims, vs, box);
}

size_t seq_scratch_bytes(int d, int Hq, int Hkv, int64_t T, int64_t B) {
  return scratch_layout(d, Hq, Hkv, T, B).end;
}

SeqScratch carve_seq_scratch(void* ws, int d, int Hq, int Hkv, int64_t T, int64_t B) {
  const ScratchLayout l = scratch_layout(d, Hq, Hkv, T, B);
  char* p = static_cast<char*>(ws);
  SeqScratch s;
  s.head = reinterpret_cast<int*>(p + 256);
  s.items = reinterpret_cast<int4*>(p + l.items);
  s.splits = reinterpret_cast<int4*>(p + l.splits);
  s.tile_off = reinterpret_cast<int*>(p + l.tile_off);
  s.part_ml = reinterpret_cast<float2*>(p + l.part_ml);
  s.part_o = reinterpret_cast<float*>(p + l.part_o);
  return s;
}

cudaError_t launch_seq_attention(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms,
                                 cudaStream_t st) {
  using Launch = cudaError_t (*)(const SeqAttnArgs&, const SeqScratch&, int, cudaStream_t);
  static const Launch table[2][2][2] = {
      {{launch_tiles<64, false, false>, launch_tiles<64, false, true>},
       {launch_tiles<64, true, false>, launch_tiles<64, true, true>}},
      {{launch_tiles<128, false, false>, launch_tiles<128, false, true>},
       {launch_tiles<128, true, false>, launch_tiles<128, true, true>}}};
  prof_before(VP_KERNEL_SEQ_ATTN, st);
  // Up to 16 rows per sequence on average: the keys are read once by either kernel, and the one for
  // few rows has more of them in flight and no TMEM round trip; above, it would read them again
  // for every 16 rows.
  const bool few = (long long)a.T * a.group <= (long long)kSmallRows * a.B;
  const cudaError_t e = few ? launch_seq_rows(a, sc, num_sms, st)
                            : table[a.d == 128][a.fp16 != 0][a.kv.k != nullptr](a, sc, num_sms, st);
  prof_after(st);
  return e;
}

}  // namespace vp
