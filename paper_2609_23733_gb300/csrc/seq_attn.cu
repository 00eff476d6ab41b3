// Softmax attention of packed sequences, over themselves (vp_prompt_attention) or over the paged
// cache (vp_paged_attention), on the sm_103a tensor cores: o = sum_j p_j v_j / sum_j p_j over the
// keys j < lim(i) that row (token i, head h) sees, p_j = 2^(s_j - m), s_j = scale log2(e) q . k_j.
//
// Work.  A tile is kChains chains of 128 / group tokens of a sequence with all heads of one kv head's
// group (row = token x group + head, so K and V are read once for the group).  The work is the
// sequence of units (tile, kv head, kBN keys that the tile's last row sees), an item's (tile, kv
// head) with kItemCost added for its start and end; CTA c of P (one per SM) takes the c-th of P
// equal runs, whatever items they belong to, so that all CTAs end together for any mix of
// lengths (a cut very near an item's end moves there).  Each CTA finds its run by a scan of the
// lengths.  An item that a CTA holds in part leaves its unnormalised output, and seq_join_kernel
// (a programmatic dependent launch) joins the parts in order.  A list of whole items in descending
// order, the long ones halved, was 1.4 to 1.6 times slower for chunks over a cache (few,
// long items: 374 against 229 us for 1,374 tokens over 43,968 keys) and needed a kernel ahead.
//
// The tile kernel.  The chains (128 rows each) of an item share the K / V ring; the tensor core works
// for one chain while another's softmax runs.  d 64: three chains, 64-key tiles, S, P and O of a
// chain in TMEM columns of their own, S of the next tile issued as soon as S has been read.  d 128:
// two chains, 128-key tiles (S at the full rate with both operands in shared memory; 64-key tiles,
// whose S runs at two thirds of it, measured 1,400 against 1,550 TFLOP/s), P in the first
// columns of S, the chains' products issued by turns.
//   warp 0               TMA: Q once per item; K / V tiles, page by page, page ids read a window of
//                        32 ahead by the lanes; it walks the run and publishes the items.
//   warps 1 .. kChains   one elected lane issues a chain's tcgen05.mma: S = Q K^T (fp32 in TMEM),
//                        O += P V (P read from TMEM as 16-bit pairs).
//   warps 4 ..           four softmax warps per chain, a row per thread; the running maximum
//                        is moved only when it grows by more than 2^8 (exact either way).
// A chain stops at its own last visible key; the tiles after it are only released.  A tile that
// some row of the chain does not see in full takes the masked path: scores past a row's limit
// become -inf by selection, and V values that are not finite are replaced by 0 in shared
// memory, since 0 x inf would reach rows that do not see them.  Rows that do see them get
// them added back in the epilogue (a flag says whether there were any), those of the other
// chains too: adding an infinity or a NaN to a sum that has it already changes nothing.
// Scores, maxima, sums and outputs are held in 32 bits; P is rounded to the storage type, as the
// tensor core needs (A and B of one MMA have one type).  Every wait is bounded; a CTA that gives up
// lets its copies and MMAs land.
//
// Bounds: 4 d flop and one exponential per row and visible key.  Measured on GB300, as called: 43,968
// causal tokens, 16 heads of 64 on 4 kv heads, 3.01 ms (1,315 TFLOP/s, 0.70 of the burst bf16 peak; the
// latency of a chain's steps bounds d 64, the exponentials' pipe is busy 47 % of the time); 32,768
// tokens, 16 heads of 128, no mask, 5.5 ms in bf16 (1,600 TFLOP/s, 0.85 of burst; the tensor pipe), 6.0 ms
// in fp16.  Between two items of a CTA lie about 7,000 clocks of drain, epilogue and fill (3.7 us),
// which is what short prompts pay.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "seq.h"

namespace vp {

namespace {

constexpr int kBM = 128;   // rows of a chain
constexpr float kUnset = -FLT_MAX;         // reference point before the first visible key
constexpr float kRescaleThreshold = 8.f;   // log2 units

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

template <int D>
struct Cfg {
  static constexpr int kChains = seq_chains(D);
  static constexpr int kBN = D == 64 ? 64 : 128;       // keys of a tile
  static constexpr bool kAlias = D == 128;             // P lies in the first columns of S
  static constexpr int kHalves = D / 64;               // 64-channel (128-byte) column blocks
  static constexpr int kStages = D == 64 ? 8 : 2;      // 128 KB of K and V, beside 48 / 64 KB of Q
  static constexpr int kThreads = 128 + 128 * kChains;
  static constexpr int kCtrlRegs = kChains == 3 ? 56 : 80;
  static constexpr int kSoftRegs = kChains == 3 ? 152 : 208;
  static_assert(128 * kCtrlRegs + 128 * kChains * kSoftRegs <= 65536, "register split");
  // TMEM columns: S_c (fp32), O_c (fp32), P_c (16-bit pairs) of every chain.
  static constexpr uint32_t kColS = 0, kColO = kChains * kBN, kColP = kAlias ? kColS : kColO + kChains * D;
  static constexpr uint32_t kPitchP = kAlias ? kBN : kBN / 2;
  static_assert((kAlias ? kColO + kChains * D : kColP + kChains * kBN / 2) <= 512, "TMEM columns");
  // An item costs about as much as this many units on top of its own (its Q, first scores and
  // epilogue, which the other chains hide only in part).
  // (Measured on packed prompts of d 128: 2: 351, 3: 337, 4: 347 us; of 8 views, d 64: 5: 261, 6: 255, 8: 257 us.)
  static constexpr int kItemCost = D == 64 ? 6 : 3;
};

// A value that is the same on all lanes, in a form that lets the compiler see it: what tcgen05 and TMA
// instructions, and the branches around them, are given stays in uniform registers.
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// Key tiles that a token sees.
template <int kBN>
__device__ __forceinline__ int tiles_seen(const SeqAttnArgs& a, int token, const Seq& s) {
  const int lim = row_limit(a, token, s.ql, s.kl);
  return lim > 0 ? ceil_div(lim, kBN) : 0;
}

// Key tiles (units) of the tile that begins with chain c0, kChains at most; at least one, in which
// rows that see nothing get their zeros.
template <class C>
__device__ __forceinline__ int tile_units(const SeqAttnArgs& a, int c0, const Seq& s) {
  const int last = min(c0 + C::kChains, count_chains(a, s.ql)) - 1;
  return max(1, tiles_seen<C::kBN>(a, chain_end(a, last, s.ql) - 1, s));
}

// ------------------------------------------------------------------ runs of units
// A CTA's run: the first segment, and its extent in units, kItemCost for every item begun included.
struct Run {
  int b, c0, h, j0, q0, ql, kl;
  long long units;
};

// A segment of a run: key tiles [j0, j0 + nk), of `all`, of the tile at chain c0 of sequence b and kv
// head h; the part-th of the run.  nk < 0: no more.
struct Item {
  int b, c0, h, j0, nk, all, q0, ql, kl, part;
};
// Chain c of an item: its tokens [t0, t1) (none: t0 == t1), the key tiles [j0, j0 + n) it takes,
// and the first key that is hidden from some row of it (from its first token's).
struct Chain {
  int t0, t1, n, hidden_from;
};
template <int kBN>
__device__ __forceinline__ Chain chain_of(const SeqAttnArgs& a, const Item& it, int c, int n_chains) {
  Chain x{0, 0, 0, 0};
  if (it.c0 + c < n_chains) {
    x.t0 = chain_start(a, it.c0 + c);
    x.t1 = chain_end(a, it.c0 + c, it.ql);
    const Seq s{it.q0, it.ql, it.kl};
    x.n = min(max(tiles_seen<kBN>(a, x.t1 - 1, s) - it.j0, 0), it.nk);
    x.hidden_from = max(row_limit(a, x.t0, s.ql, s.kl), 0);
  }
  return x;
}

// Items in flight between the producer and the epilogues: the producer writes item i + 4 when all
// softmax warps have begun item i + 2 (the first chain's i + 3), i.e. after item i's epilogue.
constexpr int kItemRing = 4;

// The segments of a run, one after another.
template <class C>
struct Walk {
  static constexpr int kChains = C::kChains, kItemCost = C::kItemCost;
  Item it;
  long long left;  // extent from this segment on
  int here;        // this segment's extent, were its item not cut
  int n_chains;    // of the sequence

  __device__ __forceinline__ void take(const SeqAttnArgs& a, const Seq& s) {
    it.q0 = uniform(s.q0);
    it.ql = uniform(s.ql);
    it.kl = uniform(s.kl);
    n_chains = count_chains(a, it.ql);
  }
  __device__ __forceinline__ void load(const SeqAttnArgs& a) { take(a, load_seq(a, it.b)); }
  __device__ __forceinline__ void set(const SeqAttnArgs& a) {
    it.all = tile_units<C>(a, it.c0, Seq{it.q0, it.ql, it.kl});
    const int cost = it.j0 == 0 ? kItemCost : 0;
    here = it.all - it.j0 + cost;
    it.nk = left >= here ? it.all - it.j0 : (int)left - cost;
  }
  __device__ __forceinline__ void start(const SeqAttnArgs& a, const Run& r) {
    it.b = uniform(r.b);
    it.c0 = uniform(r.c0);
    it.h = uniform(r.h);
    it.j0 = uniform(r.j0);
    it.part = 0;
    left = __shfl_sync(0xffffffffu, r.units, 0);
    if (left > 0) {
      take(a, Seq{r.q0, r.ql, r.kl});
      set(a);
      if (it.nk == 0) {  // from the next item on
        next(a);
        it.part = 0;
      }
    }
  }
  // The next segment: next kv head, next tile, next sequence that has new tokens.
  __device__ __forceinline__ void next(const SeqAttnArgs& a) {
    left -= here;
    ++it.part;
    if (left <= 0) return;
    it.j0 = 0;
    if (++it.h == a.Hkv) {
      it.h = 0;
      it.c0 += kChains;
      if (it.c0 >= n_chains) {
        it.c0 = 0;
        do {
          ++it.b;
          load(a);
        } while (it.ql == 0);
      }
    }
    set(a);
  }
};

// ------------------------------------------------------------------ tile kernel
template <int D>
struct TileSmem {
  using C = Cfg<D>;
  uint16_t q[C::kChains][C::kHalves][kBM * 64];
  uint4 out[C::kChains][4][32 * 8];  // of each softmax warp: 64 channels of its 32 rows, on their way out
  uint16_t k[C::kStages][C::kHalves][C::kBN * 64];
  uint16_t v[C::kStages][C::kHalves][C::kBN * 64];
  uint64_t q_full[C::kChains], q_empty[C::kChains];
  uint64_t k_full[C::kStages], v_full[C::kStages], k_empty[C::kStages], v_empty[C::kStages];
  uint64_t s_full[C::kChains], s_empty[C::kChains], p_full[C::kChains], o_bar[C::kChains],
      o_empty[C::kChains], drain[C::kChains], turn[C::kChains];
  uint32_t tmem_base;
  int abort_flag;
  int nonfinite[2];  // V values of masked tiles replaced by 0: any, and any that some row sees
  Run run;
  Item item[kItemRing];  // published by the producer with q_full, and their chains
  Chain chain[kItemRing][C::kChains];
};

// Inclusive scan of v over the CTA's 32 kWarps threads; *total: the sum.  v < 2^26, so that a warp's sum
// fits 32 bits.  s_warp: one value per warp.
template <int kWarps>
__device__ __forceinline__ long long cta_scan(int v, int* s_warp, long long* total) {
  const int lane = lane_id(), w = warp_id();
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, k);
    if (lane >= k) v += u;
  }
  __syncthreads();
  if (lane == 31) s_warp[w] = v;
  __syncthreads();
  long long t = 0, before = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    if (i == w) before = t;
    t += s_warp[i];
  }
  *total = t;
  return before + v;
}

// x / y of non-negative values; 64-bit division only where it takes it.
__device__ __forceinline__ long long div64(long long x, long long y) {
  return (x | y) >> 32 ? x / y : (long long)((uint32_t)x / (uint32_t)y);
}

// The extents of all tiles in order: on_total(sum of them), then fn(b, c0, seq, extent of an item, extent
// before the tile) for every tile, each on one thread.  One pass over the tiles where there are
// no more sequences and tiles than threads, else two.  Called by all threads; s_seq: scratch of 16 bytes
// per thread and 4 per warp.
template <class C, class Total, class Fn>
__device__ __forceinline__ void scan_tiles(const SeqAttnArgs& a, int4* s_seq, Total on_total, Fn fn) {
  constexpr int kChains = C::kChains, n = C::kThreads, kWarps = n / 32;
  const int tid = threadIdx.x;
  int* s_warp = reinterpret_cast<int*>(s_seq + n);
  bool last = false;  // the pass that calls fn
  for (int pass = 0; pass < 2; ++pass) {
    long long before = 0;
    for (int b0 = 0; b0 < a.B; b0 += n) {
      Seq s{0, 0, 0};
      int tiles;
      if (a.B == 1) {  // no search
        s = load_seq(a, 0);
        tiles = ceil_div(count_chains(a, s.ql), kChains);
      } else {
        if (b0 + tid < a.B) s = load_seq(a, b0 + tid);
        const int n_tiles = ceil_div(count_chains(a, s.ql), kChains);
        long long all;  // (2^26 tiles of queries would not fit the GPU's memory)
        const long long end = cta_scan<kWarps>(min(n_tiles, (1 << 26) - 1), s_warp, &all);
        tiles = (int)all;
        s_seq[tid] = make_int4(s.q0, s.ql, s.kl, (int)end);  // .w: tiles up to this sequence's last
        __syncthreads();
      }
      const bool once = a.B <= n && tiles <= n;
      for (int w0 = 0; w0 < tiles; w0 += n) {
        const int w = w0 + tid;
        int lo = 0, c0 = 0;
        int u = 0;  // < 2^26: key tiles of at most 2^30 keys
        if (w < tiles) {
          if (a.B == 1) {
            c0 = w * kChains;
          } else {
            int hi = min(n, a.B - b0) - 1;  // the first sequence with .w > w
            while (lo < hi) {
              const int mid = (lo + hi) >> 1;
              if (s_seq[mid].w > w)
                hi = mid;
              else
                lo = mid + 1;
            }
            const int4 x = s_seq[lo];
            s = Seq{x.x, x.y, x.z};
            c0 = (w - (x.w - ceil_div(count_chains(a, s.ql), kChains))) * kChains;
          }
          u = tile_units<C>(a, c0, s) + C::kItemCost;
        }
        long long total;
        const long long upto = cta_scan<kWarps>(u, s_warp, &total) * a.Hkv;
        total *= a.Hkv;
        if (once) {
          on_total(total);
          last = true;
        }
        if (last && u > 0) fn(b0 + lo, c0, s, u, before + upto - (long long)u * a.Hkv);
        before += total;
      }
      __syncthreads();
    }
    if (last) return;
    on_total(before);
    if (before == 0) return;
    last = true;
  }
}

// Cut x of the units moved to the end of the item [first, first + n) it lies in, if that is near.
__device__ __forceinline__ long long snap(long long x, long long first, int n, long long near) {
  return x - first < near ? first : first + n - x < near ? first + n : x;
}

template <bool F16>
__host__ __device__ constexpr uint32_t idesc_16bit(int M, int N, int b_mn) {
  // D fp32; A and B bf16 (1) or fp16 (0); A K-major, B K-major or MN-major
  return (1u << 4) | ((F16 ? 0u : 1u) << 7) | ((F16 ? 0u : 1u) << 10) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Replaces what is not finite in the rows [first, kBN) of a V tile by 0 (the chain's 128 threads,
// 16 rows at a time).  flags[0]: there was something to replace; flags[1]: in a row below n_valid.
template <int D, int kBN, bool F16>
__device__ __forceinline__ void scrub_v(uint16_t* v, int first, int n_valid, int tid, volatile int* flags) {
  constexpr int kHalves = D / 64;
  uint4* p = reinterpret_cast<uint4*>(v);
  // In pairs of passes, so that two loads or more are in flight.
#pragma unroll 1
  for (int r0 = first / 32 * 32; r0 < kBN; r0 += 32) {
    uint4 x[2 * kHalves];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 2 * kHalves; ++i) {
      x[i] = p[(i >> 1) * (kBN * 8) + (r0 + 16 * (i & 1)) * 8 + tid];
      bad |= nonfinite2<F16>(x[i].x) || nonfinite2<F16>(x[i].y) || nonfinite2<F16>(x[i].z) ||
             nonfinite2<F16>(x[i].w);
    }
    if (bad) {
#pragma unroll
      for (int i = 0; i < 2 * kHalves; ++i) {
        const int row = r0 + 16 * (i & 1) + (tid >> 3);
        if (!(nonfinite2<F16>(x[i].x) || nonfinite2<F16>(x[i].y) || nonfinite2<F16>(x[i].z) ||
              nonfinite2<F16>(x[i].w)))
          continue;
        flags[0] = 1;
        if (row < n_valid) flags[1] = 1;
        __threadfence_block();
        p[(i >> 1) * (kBN * 8) + (r0 + 16 * (i & 1)) * 8 + tid] =
            make_uint4(finite2<F16>(x[i].x), finite2<F16>(x[i].y), finite2<F16>(x[i].z), finite2<F16>(x[i].w));
      }
    }
  }
  // Zeros written here, or by another chain's threads and read here: before this chain's MMA.
  __threadfence_block();
  if (flags[0]) fence_proxy_async_smem();
}

// Adds to a row of outputs in memory the V values that are not finite among the keys [j0, j1).
// at(c): reads channel c; put(c, x): writes it.
template <int D, bool F16, bool kPaged, class At, class Put>
__device__ __forceinline__ void add_nonfinite(const SeqAttnArgs& a, const Item& it, int j0, int j1, At at,
                                              Put put) {
#pragma unroll 1
  for (int j = j0; j < j1; ++j) {
    const uint16_t* row;
    if constexpr (kPaged) {
      const int page = a.kv.table[(size_t)it.b * a.kv.width + (j >> a.kv.log2_page)];
      if ((unsigned)page >= (unsigned)a.kv.n_pages) continue;
      row = a.kv.v +
            (((((long long)page * a.Hkv + it.h) << a.kv.log2_page)) + (j & (a.kv.page_size - 1))) * D;
    } else {
      row = a.v + (long long)(it.q0 + j) * a.v_stride + it.h * D;
    }
#pragma unroll 1
    for (int c = 0; c < D; ++c) {
      const float x = to_float<F16>(row[c]);
      if (!isfinite(x)) put(c, at(c) + x);
    }
  }
}
template <int D, bool F16, bool kPaged>
__device__ __noinline__ void refill_out(const SeqAttnArgs& a, const Item& it, int j0, int j1, uint16_t* out) {
  add_nonfinite<D, F16, kPaged>(
      a, it, j0, j1, [&](int c) { return to_float<F16>(out[c]); },
      [&](int c, float x) { out[c] = (uint16_t)pack2<F16>(x, 0.f); });
}
template <int D, bool F16, bool kPaged>
__device__ __noinline__ void refill_part(const SeqAttnArgs& a, const Item& it, int j0, int j1, float* part) {
  auto addr = [&](int c) { return part + (c >> 2) * (4 * kBM) + (c & 3); };
  add_nonfinite<D, F16, kPaged>(
      a, it, j0, j1, [&](int c) { return *addr(c); }, [&](int c, float x) { *addr(c) = x; });
}

// This CTA's run, into *run (visible after the next barrier), and its entry of the list of cut
// items: an item whose first part is this run's end.
template <class C>
__device__ __forceinline__ void find_run(const SeqAttnArgs& a, const SeqScratch& sc, int4* s_seq,
                                         Run* run) {
  constexpr int kItemCost = C::kItemCost;
  __shared__ long long s_begin, s_end, s_first;
  __shared__ int4 s_rec[2];
  const int P = gridDim.x, cta = blockIdx.x;
  long long per = 0, near = 0, x0 = 0, x1 = 0;
  auto on_total = [&](long long total) {
    per = div64(total + P - 1, P);
    near = max(per / 128, kItemCost + 4ll);
    x0 = cta * per;
    x1 = x0 + per;
    if (threadIdx.x == 0) {
      s_begin = min(x0, total);
      s_end = min(x1, total);
      s_rec[0] = make_int4(0, 0, 0, 0);
      run->b = run->c0 = run->h = run->j0 = 0;
    }
    __syncthreads();
  };
  scan_tiles<C>(a, s_seq, on_total, [&](int b, int c0, const Seq& s, int n, long long before) {
    const long long end = before + (long long)n * a.Hkv;
    if (before <= x0 && x0 < end) {
      const int h = (int)div64(x0 - before, n);
      const long long first = before + (long long)h * n, x = snap(x0, first, n, near);
      s_begin = x;
      run->b = b;
      run->c0 = c0;
      run->q0 = s.q0;
      run->ql = s.ql;
      run->kl = s.kl;
      run->h = h;
      run->j0 = x == first ? 0 : (int)(x - first) - kItemCost;  // all: from the next item on
    }
    if (before <= x1 && x1 < end) {
      const int h = (int)div64(x1 - before, n);
      const long long first = before + (long long)h * n, x = snap(x1, first, n, near);
      s_end = x;
      if (x > first && x < first + n && x0 - first < near) {
        // The cuts k per of this item that stay: first + near <= k per <= first + n - near.
        const int last = (int)div64(first + n - near, per);
        s_rec[0] = make_int4(last - cta + 1, h, c0, b);
        s_rec[1] = make_int4(s.q0, s.ql, s.kl, 0);
        s_first = first;
      }
    }
  });
  if (threadIdx.x == 0) {
    run->units = s_end - s_begin;
    if (s_rec[0].x) s_rec[1].w = 2 * cta + (s_first > s_begin);  // the first part's slot
    sc.recs[2 * cta] = s_rec[0];
    sc.recs[2 * cta + 1] = s_rec[1];
  }
}

template <int D, bool F16, bool kPaged>
__global__ void __launch_bounds__(Cfg<D>::kThreads, 1)
    seq_tile_kernel(const __grid_constant__ CUtensorMap tmap_q,
                    const __grid_constant__ CUtensorMap tmap_k,
                    const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ SeqAttnArgs prm, const SeqScratch sc) {
  using C = Cfg<D>;
  constexpr int kChains = C::kChains, kStages = C::kStages, kHalves = C::kHalves, kBN = C::kBN;
  constexpr bool kAlias = C::kAlias;
  extern __shared__ unsigned char smem_raw[];
  TileSmem<D>& sm = *reinterpret_cast<TileSmem<D>*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int P = gridDim.x, cta = blockIdx.x;
  const int warp = warp_uniform_id(), lane = lane_id();
  volatile int* abort_flag = &sm.abort_flag;
  unsigned int* err = prm.err;
  pdl_launch_dependents();

  if (threadIdx.x == 0) {
    for (int c = 0; c < kChains; ++c) {
      mbar_init(&sm.q_full[c], 1);
      mbar_init(&sm.q_empty[c], 5);  // the chain's last scores; its softmax warps have begun the item
    }
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.k_empty[s], kChains);
      mbar_init(&sm.v_empty[s], kChains);
    }
    for (int c = 0; c < kChains; ++c) {
      mbar_init(&sm.s_full[c], 1);
      mbar_init(&sm.s_empty[c], 128);
      mbar_init(&sm.p_full[c], 128);
      mbar_init(&sm.o_bar[c], 1);
      mbar_init(&sm.o_empty[c], 128);
      mbar_init(&sm.drain[c], 1);
      mbar_init(&sm.turn[c], 1);
    }
    sm.abort_flag = 0;
    sm.nonfinite[0] = sm.nonfinite[1] = 0;
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
  pdl_wait();  // what is ahead in the stream: the inputs are there, and the last call's join is over
  find_run<C>(prm, sc, reinterpret_cast<int4*>(sm.q), &sm.run);
  fence_proxy_async_smem();  // sm.q was scratch: before the copies into it
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem_base, 0);

  const int group = prm.group, tpt = prm.chain_tokens;

  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kCtrlRegs));
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    uint32_t lc = 0, ic = 0, k_ahead = 0;  // tiles, items; 1: K of tile lc is on its way
    int q_last = -1;  // the last Q tile asked for: item x kChains + chain
    bool ok = true;
    const int log2p = prm.kv.log2_page, ps = prm.kv.page_size;
    const int ppt = kPaged ? (ps >= kBN ? 1 : kBN / ps) : 1;  // pages (boxes) of a tile
    const uint32_t box_bytes = (kPaged && ps < kBN ? ps : kBN) * 128;
    Walk<C> walk;
    for (walk.start(prm, sm.run);; walk.next(prm), ++ic) {
      const Item& it = walk.it;
      // Q of chains c .. c_end - 1 (nothing to load for a chain without tokens), in turn.
      auto load_q = [&](int c, int c_end) {
        for (; c < c_end && ok; ++c) {
          ok = mbar_wait_warp(&sm.q_empty[c], (ic & 1) ^ 1, err, abort_flag);
          if (!ok) return;
          if (c == 0) {  // the item's first Q tile: publish it
            if (lane == 0) {
              sm.item[ic % kItemRing] = it;
              if (walk.left <= 0) sm.item[ic % kItemRing].nk = -1;  // the end of the run
            }
            if (lane < kChains && walk.left > 0)
              sm.chain[ic % kItemRing][lane] = chain_of<kBN>(prm, it, lane, walk.n_chains);
            __syncwarp();
          }
          if (elect_one()) {
            if (walk.left > 0 && it.c0 + c < walk.n_chains) {
              mbar_arrive_expect_tx(&sm.q_full[c], kHalves * tpt * group * 128);
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf)
                tma_load_4d(sm.q[c][hf], &tmap_q, &sm.q_full[c], hf * 64, 0, it.h,
                            it.q0 + chain_start(prm, it.c0 + c));
            } else {
              mbar_arrive(&sm.q_full[c]);
            }
          }
          __syncwarp();
          q_last = ic * kChains + c;
        }
      };
      // Page ids: lane l holds that of page first + l; `next` the 32 after them.
      const int n_pages = kPaged && walk.left > 0 ? (it.kl + ps - 1) >> log2p : 0;
      const int32_t* table = kPaged ? prm.kv.table + (size_t)it.b * prm.kv.width : nullptr;
      int first = kPaged ? (it.j0 * kBN) >> log2p : 0, window = 0, next = 0;
      if (kPaged) {
        if (first + lane < n_pages) window = table[first + lane];
        if (first + 32 + lane < n_pages) next = table[first + 32 + lane];
      }
      load_q(0, 1);
      if (!ok) break;
      if (walk.left <= 0) {
        load_q(1, kChains);
        break;
      }
      for (int jj = 0; jj < it.nk; ++jj, ++lc) {
        const int j = it.j0 + jj, st = lc % kStages;
        int y = it.q0 + j * kBN, at = 0, n_box = 1;
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
        const uint32_t par = ((lc / kStages) & 1) ^ 1, bytes = n_box * kHalves * box_bytes;
        // Page after page by one elected lane, with coordinates that are the same on all lanes.
        auto copy = [&](uint16_t (*dst)[kBN * 64], const CUtensorMap* map, uint64_t* bar) {
          for (int i = 0; i < n_box; ++i) {
            const int page = kPaged ? __shfl_sync(0xffffffffu, window, at + i) : 0;
            if (kPaged && (unsigned)page >= (unsigned)prm.kv.n_pages && lane == 0)
              atomicOr(err, VP_DEVERR_PAGE);
            if (elect_one()) {
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf)
                tma_load_4d(dst[hf] + i * (box_bytes / 2), map, bar, hf * 64, y, it.h, page);
            }
            __syncwarp();
          }
        };
        // K and V of a tile are released apart with 128-key tiles, together with 64-key ones.
        ok = mbar_wait_warp(kAlias ? &sm.k_empty[st] : &sm.v_empty[st], par, err, abort_flag);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(&sm.k_full[st], bytes);
          if (!kAlias) mbar_arrive_expect_tx(&sm.v_full[st], bytes);
        }
        __syncwarp();
        copy(sm.k[st], &tmap_k, &sm.k_full[st]);
        if (kAlias) {
          ok = mbar_wait_warp(&sm.v_empty[st], par, err, abort_flag);
          if (!ok) {
            k_ahead = 1;
            break;
          }
          if (elect_one()) mbar_arrive_expect_tx(&sm.v_full[st], bytes);
          __syncwarp();
        }
        copy(sm.v[st], &tmap_v, &sm.v_full[st]);
        if (jj == 0) {  // the other chains' Q behind the first keys
          load_q(1, kChains);
          if (!ok) {
            ++lc;
            break;
          }
        }
      }
      if (!ok) break;
    }
    if (!ok && lane == 0) {
      // Let the copies this warp issued land before the CTA releases its shared memory: the last use
      // of slot s of a ring of n after `count` uses.
      auto wait_last = [&](uint64_t* bar, uint32_t s, uint32_t n, uint32_t count) {
        if (count <= s) return;
        const uint32_t last = (count - 1 - s) / n * n + s;
        for (int t = 0; t < 1000000 && !mbar_try_wait(bar, (last / n) & 1); ++t) {}
      };
      for (uint32_t c = 0; c < (uint32_t)kChains; ++c) wait_last(&sm.q_full[c], c, kChains, q_last + 1);
      for (uint32_t s = 0; s < (uint32_t)kStages; ++s) {
        wait_last(&sm.k_full[s], s, kStages, lc + k_ahead);
        wait_last(&sm.v_full[s], s, kStages, lc);
      }
    }
  } else if (kAlias && warp <= kChains) {
    // ------------------------------------------------------------ MMA issuers (chain c), by turns
    // A chain's products of a step, P_c V of this tile and S_c of the next, are issued in one go and
    // the chains take turns, so that one chain's softmax runs while the other's MMAs do; without
    // turns the two interleave and both softmaxes run at once (3,880 clocks for 2 x 128 rows x
    // 128 keys of d 128, against 2,048 of MMAs).  A warp per chain: the waits of one (a couple of
    // hundred clocks even when there is nothing to wait for) pass during the other's turn.
    const int c = warp - 1;
    const uint32_t id_s = idesc_16bit<F16>(kBM, kBN, 0);  // Q (K-major) x K^T (K-major)
    const uint32_t id_o = idesc_16bit<F16>(kBM, 64, 1);   // P (TMEM) x V (MN-major)
    const uint32_t t_s = tmem + C::kColS + c * kBN;
    const uint32_t t_o = tmem + C::kColO + c * D;
    const uint32_t t_p = tmem + C::kColP + c * C::kPitchP;
    uint32_t lc = 0, g = 0, oc = 0, turn = 0;  // ring tiles, this chain's tiles, its items, its turns
    bool ok = true;
    // Three barriers at once (lanes 0-10, 11-21, 22-31).
    auto wait3 = [&](uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1, uint64_t* b2, uint32_t p2) {
      const int grp = lane / 11;
      uint64_t* bar = grp == 0 ? b0 : grp == 1 ? b1 : b2;
      const uint32_t par = grp == 0 ? p0 : grp == 1 ? p1 : p2;
      return (bool)__all_sync(0xffffffffu, mbar_wait(bar, par, err, abort_flag));
    };
    auto my_turn = [&] { return c == 0 ? (turn & 1) ^ 1 : turn & 1; };
    for (uint32_t ic = 0;; ++ic) {
      ok = mbar_wait_warp(&sm.q_full[c], ic & 1, err, abort_flag);
      if (!ok) break;
      const int nk = uniform(sm.item[ic % kItemRing].nk);
      const int n = uniform(sm.chain[ic % kItemRing][c].n);
      if (nk < 0) break;
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q[c][0]));
      // Step -1: S_c(0); step j: P_c(j) V and S_c(j + 1).
      for (int j = -1; j < nk && ok; ++j) {
        const uint32_t l = lc + j;  // the ring's tile of P V; l + 1 that of S
        const int st = l % kStages, st1 = (l + 1) % kStages;
        const bool pv = j >= 0 && j < n, sc_next = j + 1 < n;
        uint64_t* k_bar = &sm.k_full[st1];
        const uint32_t k_par = ((l + 1) / kStages) & 1, v_par = (l / kStages) & 1;
        if (pv)
          ok = wait3(&sm.p_full[c], g & 1, &sm.v_full[st], v_par, sc_next ? k_bar : &sm.p_full[c],
                     sc_next ? k_par : g & 1);
        else if (sc_next)
          ok = mbar_wait_warp(k_bar, k_par, err, abort_flag);
        else if (j >= 0)  // past the chain's last visible key: released once it has landed
          ok = mbar_wait_warp(&sm.k_full[st], v_par, err, abort_flag) &&
               mbar_wait_warp(&sm.v_full[st], v_par, err, abort_flag);
        if (ok && pv && j == 0) ok = mbar_wait_warp(&sm.o_empty[c], (oc & 1) ^ 1, err, abort_flag);
        ok = ok && mbar_wait_warp(&sm.turn[c], my_turn(), err, abort_flag);
        if (!ok) break;
        ++turn;
        tc_fence_after();
        const uint64_t dv = sdesc_sw128(smem_u32(sm.v[st][0]));
        const uint64_t dk = sdesc_sw128(smem_u32(sm.k[st1][0]));
        if (elect_one()) {
          if (pv) {
#pragma unroll
            for (int kk = 0; kk < kBN / 16; ++kk)  // 16 keys per step: 8 TMEM columns, 2 KB of V
#pragma unroll
              for (int hf = 0; hf < kHalves; ++hf)
                tc_mma_ts(t_o + 64 * hf, t_p + 8 * kk,
                          dv + hf * (kBN * 128 / 16) + (uint64_t)(kk * 128), id_o,
                          (j > 0 || kk > 0) ? 1u : 0u);
            tc_commit(&sm.v_empty[st]);
            if (j == n - 1) tc_commit(&sm.o_bar[c]);
          } else if (j >= 0) {
            mbar_arrive(&sm.k_empty[st]);
            mbar_arrive(&sm.v_empty[st]);
          }
          if (sc_next) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)  // K = 16 per step: +32 bytes, +1 block per 64
              tc_mma_ss(t_s, dq + (kk >> 2) * (kBM * 128 / 16) + 2 * (kk & 3),
                        dk + (kk >> 2) * (kBN * 128 / 16) + 2 * (kk & 3), id_s, kk > 0);
            tc_commit(&sm.s_full[c]);
            tc_commit(&sm.k_empty[st1]);
            if (j + 1 == n - 1) tc_commit(&sm.q_empty[c]);
          }
          if (j < 0 && n == 0) mbar_arrive(&sm.q_empty[c]);
          mbar_arrive(&sm.turn[c ^ 1]);
        }
        __syncwarp();
        if (pv) ++g;
      }
      if (!ok) break;
      lc += nk;
      oc += n > 0;
    }
    if (!ok) {
      if (elect_one()) {
        tc_commit(&sm.drain[c]);
        for (int t = 0; t < 1000000 && !mbar_try_wait(&sm.drain[c], 0); ++t) {}
      }
      __syncwarp();
    }
  } else if (!kAlias && warp <= kChains) {
    // ------------------------------------------------------------ MMA issuers (chain c)
    const int c = warp - 1;
    const uint32_t id_s = idesc_16bit<F16>(kBM, kBN, 0);  // Q (K-major) x K^T (K-major)
    const uint32_t id_o = idesc_16bit<F16>(kBM, 64, 1);   // P (TMEM) x V (MN-major)
    const uint32_t t_s = tmem + C::kColS + c * kBN;
    const uint32_t t_o = tmem + C::kColO + c * D;
    const uint32_t t_p = tmem + C::kColP + c * C::kPitchP;
    uint32_t lc = 0, ic = 0, g = 0, oc = 0;  // ring tiles, items, this chain's tiles, its items
    bool ok = true;
    for (;; ++ic) {
      ok = mbar_wait_warp(&sm.q_full[c], ic & 1, err, abort_flag);
      if (!ok) break;
      const int nk = uniform(sm.item[ic % kItemRing].nk);
      const int n = uniform(sm.chain[ic % kItemRing][c].n);
      if (nk < 0) break;
      const uint64_t dq = sdesc_sw128(smem_u32(sm.q[c][0]));
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
          if (j == n - 1) tc_commit(&sm.q_empty[c]);
        }
        __syncwarp();
        return true;
      };
      if (n > 0) {
        ok = issue_s(0);
      } else if (lane == 0) {
        mbar_arrive(&sm.q_empty[c]);
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
          tc_commit(&sm.v_empty[st]);
        }
        __syncwarp();
      }
      // The item's tiles past this chain's last visible key: released once they have landed.
      for (int j = n; j < nk && ok; ++j) {
        const uint32_t l = lc0 + j;
        const int st = l % kStages;
        ok = mbar_wait_warp(&sm.k_full[st], (l / kStages) & 1, err, abort_flag) &&
             mbar_wait_warp(&sm.v_full[st], (l / kStages) & 1, err, abort_flag);
        if (ok && lane == 0) mbar_arrive(&sm.v_empty[st]);  // of K and V
      }
      if (!ok) break;
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
    const uint32_t t_p = tmem + lane_off + C::kColP + c * C::kPitchP;
    const int row_tok = prm.by_group(row), row_head = row - row_tok * group;
    const bool flip = prm.scale_log2 < 0.f;  // scores are negated, so that the maximum is the scores'
    const float cs = fmaxf(fabsf(prm.scale_log2), kLeastScale);
    uint32_t g = 0, lc = 0, oc = 0;  // the chain's tiles, ring tiles, the chain's items
    bool ok = true;
    for (uint32_t ic = 0;; ++ic) {
      ok = mbar_wait_warp(&sm.q_full[c], ic & 1, err, abort_flag);
      if (!ok) break;
      const Item& it = sm.item[ic % kItemRing];
      if (it.nk < 0) break;
      if (lane == 0) mbar_arrive(&sm.q_empty[c]);
      const Chain ch = sm.chain[ic % kItemRing][c];
      const int n = ch.n, tok = ch.t0 + row_tok;  // this thread's token in its sequence
      const bool valid = row_tok < tpt && tok < ch.t1;
      const int lim = valid ? row_limit(prm, tok, it.ql, it.kl) : 0;
      const int masked_from = ch.hidden_from / kBN;  // the first tile with a hidden key
      const bool active = __any_sync(0xffffffffu, valid);
      float m = kUnset, lsum = 0.f;
      // One key tile; kMasked: some row of the chain may not see all of it, or the scores are negated.
      auto tile = [&](auto masked_const, int jj) -> bool {
        constexpr bool kMasked = decltype(masked_const)::value;
        if (!mbar_wait_warp(&sm.s_full[c], g & 1, err, abort_flag)) return false;
        if (kMasked) {
          const uint32_t l = lc + jj;
          const int st = l % kStages;
          if (!mbar_wait_warp(&sm.v_full[st], (l / kStages) & 1, err, abort_flag)) return false;
          if (it.j0 + jj >= masked_from)
            scrub_v<D, kBN, F16>(sm.v[st][0], max(ch.hidden_from - (it.j0 + jj) * kBN, 0),
                                 it.kl - (it.j0 + jj) * kBN, row, sm.nonfinite);
        }
        tc_fence_after();
        float s[kBN], pmx[kBN / 32];
#pragma unroll
        for (int cc = 0; cc < kBN / 32; ++cc) tmem_ld32_max(t_s + 32 * cc, s + 32 * cc, pmx[cc]);
        tmem_wait_ld();
        tc_fence_before();
        if (!kAlias) mbar_arrive(&sm.s_empty[c]);  // the MMA warp may overwrite S_c now
        float mx = pmx[0];
#pragma unroll
        for (int cc = 1; cc < kBN / 32; ++cc) mx = fmaxf(mx, pmx[cc]);
        const int n_seen = valid ? lim - (it.j0 + jj) * kBN : kBN;
        if (kMasked && __any_sync(0xffffffffu, flip || n_seen < kBN)) {
          if (flip) {
#pragma unroll
            for (int i = 0; i < kBN; ++i) s[i] = -s[i];
          }
#pragma unroll
          for (int b = 0; b < kBN; b += 32) {  // a bit per column
            const int k = min(max(n_seen - b, 0), 32);
            const uint32_t bits = k == 32 ? 0xffffffffu : (1u << k) - 1u;
#pragma unroll
            for (int i = 0; i < 32; ++i) s[b + i] = (bits >> i) & 1u ? s[b + i] : -INFINITY;
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
        const float mul = fabsf(mx) < prm.far_from ? cs : prm.far_scale;
        const float to = reference_point<F16>(mx, mul);
        float alpha = 1.f;
        bool need = false;
        if (jj == 0) {
          m = fmaxf(to, kUnset);
        } else if (to - m > kRescaleThreshold) {  // (m + 8 could round up to `to`)
          need = true;
          alpha = fast_exp2(m - to);
          m = to;
        }
        const float2 c2 = make_float2(mul, mul), nm = make_float2(-m, -m);
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
        // P_c and O_c are free once P_c(g-1) V has completed (before S_c(g), where P_c lies in it).
        if (!kAlias && g > 0) {
          if (!mbar_wait_warp(&sm.o_bar[c], (g - 1) & 1, err, abort_flag)) return false;
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
        ++g;
        return true;
      };
      if (active) {
        const int clear = flip ? 0 : min(max(masked_from - it.j0, 0), n);
        int jj = 0;
        for (; jj < clear && ok; ++jj) ok = tile(std::false_type{}, jj);
        for (; jj < n && ok; ++jj) ok = tile(std::true_type{}, jj);
      } else {
        // No row of this warp exists: its lanes of P and O are never read.
        for (int jj = 0; jj < n && ok; ++jj, ++g) {
          const uint32_t l = lc + jj;
          const int st = l % kStages, j = it.j0 + jj;
          ok = mbar_wait_warp(&sm.s_full[c], g & 1, err, abort_flag);
          if (ok && j >= masked_from) {
            ok = mbar_wait_warp(&sm.v_full[st], (l / kStages) & 1, err, abort_flag);
            if (ok)
              scrub_v<D, kBN, F16>(sm.v[st][0], max(ch.hidden_from - j * kBN, 0), it.kl - j * kBN, row,
                                   sm.nonfinite);
          }
          if (!ok) break;
          if (!kAlias) {
            mbar_arrive(&sm.s_empty[c]);
            if (g > 0) ok = mbar_wait_warp(&sm.o_bar[c], (g - 1) & 1, err, abort_flag);
          }
          if (ok) mbar_arrive(&sm.p_full[c]);
        }
      }
      lc += it.nk;
      if (n > 0 && ok)  // one o_bar per tile, or (kAlias) per item
        ok = mbar_wait_warp(&sm.o_bar[c], (kAlias ? oc : g - 1) & 1, err, abort_flag);
      oc += n > 0;
      if (!ok) break;
      tc_fence_after();
      const bool part = it.nk < it.all;
      const float inv = part ? 1.f : lim > 0 ? 1.f / lsum : 0.f;
      const size_t slot_chain = (size_t)(2 * cta + (it.part > 0)) * kChains + c;
      float* to_part = sc.part_o + (slot_chain * (D / 4) * kBM + row) * 4;  // [D / 4][128 rows][4]
      uint16_t* to = prm.out + (int64_t)(it.q0 + tok) * prm.out_stride + (it.h * group + row_head) * D;
      const unsigned rows = __ballot_sync(0xffffffffu, valid);
      uint4* out = sm.out[c][quarter];
#pragma unroll 1
      for (int hf = 0; hf < kHalves; ++hf) {
        float o[64];
        if (n > 0) {
          tmem_ld32(t_o + 64 * hf, o);
          tmem_ld32(t_o + 64 * hf + 32, o + 32);
          tmem_wait_ld();
          if (hf == kHalves - 1) {
            tc_fence_before();
            mbar_arrive(&sm.o_empty[c]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 64; ++i) o[i] = 0.f;
        }
        if (part) {
          if (valid)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              *reinterpret_cast<float4*>(to_part + (16 * hf + i) * (4 * kBM)) =
                  make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          continue;
        }
        const float2 inv2 = make_float2(inv, inv);
        auto scaled = [&](int i) {
          const float2 x = fmul2(make_float2(o[i], o[i + 1]), inv2);
          return pack2<F16>(x.x, x.y);
        };
        // Through shared memory (16-byte chunks swizzled by the row), so that eight lanes write a
        // row's 128 bytes and not every lane 16 of its own row.
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i)
          out[lane * 8 + (i ^ (lane & 7))] = make_uint4(scaled(8 * i), scaled(8 * i + 2), scaled(8 * i + 4),
                                                        scaled(8 * i + 6));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = 4 * i + (lane >> 3), ch8 = lane & 7;
          uint16_t* dst = reinterpret_cast<uint16_t*>(
              __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), r));
          if (rows >> r & 1)
            *reinterpret_cast<uint4*>(dst + 64 * hf + 8 * ch8) = out[r * 8 + (ch8 ^ (r & 7))];
        }
      }
      __syncwarp();
      if (n > 0 && valid && *(volatile int*)&sm.nonfinite[1] != 0) {
        // Chains may have taken values out of V from the item's first hidden key on.
        const int j0 = max(it.j0, sm.chain[ic % kItemRing][0].hidden_from / kBN) * kBN;
        const int j1 = min(lim, (it.j0 + n) * kBN);
        __threadfence_block();  // the row was written by other lanes
        if (part)
          refill_part<D, F16, kPaged>(prm, it, j0, j1, to_part);
        else
          refill_out<D, F16, kPaged>(prm, it, j0, j1, to);
      }
      if (valid && part) sc.part_ml[slot_chain * kBM + row] = make_float2(m, lsum);
      if (valid && !part && prm.lse)
        prm.lse[(size_t)(it.q0 + tok) * prm.Hq + it.h * group + row_head] =
            lim > 0 ? (near_units(prm, m) + log2f(lsum)) * 0.69314718055994531f : -INFINITY;
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

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct ScratchLayout {
  size_t part_ml, part_o, end;
};
ScratchLayout scratch_layout(int d) {
  const size_t rows = (size_t)kMaxSlots * seq_chains(d) * kBM;
  ScratchLayout l;
  l.part_ml = 256 + align256((size_t)kMaxRecs * 2 * sizeof(int4));  // after the error word and the list
  l.part_o = l.part_ml + align256(rows * sizeof(float2));
  l.end = l.part_o + align256(rows * d * sizeof(float));
  return l;
}

template <int D, bool F16, bool kPaged>
cudaError_t launch_tiles(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms, cudaStream_t st) {
  using C = Cfg<D>;
  CUtensorMap mq, mk, mv;
  const uint64_t g = a.group, H = a.Hkv;
  const uint64_t qd[4] = {D, g, H, (uint64_t)a.T};
  const uint64_t qs[3] = {D, g * D, (uint64_t)a.q_stride};
  const uint32_t qb[4] = {64, (uint32_t)g, 1, (uint32_t)a.chain_tokens};
  cudaError_t e = make_tmap_16bit_4d(&mq, a.q, F16, qd, qs, qb);
  if (e != cudaSuccess) return e;
  e = make_kv_maps(a, C::kBN, &mk, &mv);
  if (e != cudaSuccess) return e;
  const int P = num_sms < kMaxCtas ? num_sms : kMaxCtas;
  constexpr int smem = (int)sizeof(TileSmem<D>) + 1024;
  const void* tile = reinterpret_cast<const void*>(seq_tile_kernel<D, F16, kPaged>);
  e = cudaFuncSetAttribute(tile, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  SeqAttnArgs aa = a;
  SeqScratch ss = sc;
  void* args[] = {&mq, &mk, &mv, &aa, &ss};
  e = launch_pdl(tile, dim3(P), C::kThreads, smem, st, args);
  // Items of at most kItemCost + 7 key tiles are never cut (find_run): nothing to join.
  if (e != cudaSuccess || most_keys(a) <= (C::kItemCost + 7) * C::kBN) return e;
  return launch_seq_join(a, sc, true, P, st);
}

}  // namespace

cudaError_t launch_pdl(const void* fn, dim3 grid, int threads, int smem, cudaStream_t st, void** args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
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

size_t seq_scratch_bytes(int d) { return scratch_layout(d).end; }

SeqScratch carve_seq_scratch(void* ws, int d) {
  const ScratchLayout l = scratch_layout(d);
  char* p = static_cast<char*>(ws);
  SeqScratch s;
  s.recs = reinterpret_cast<int4*>(p + 256);
  s.part_ml = reinterpret_cast<float2*>(p + l.part_ml);
  s.part_o = reinterpret_cast<float*>(p + l.part_o);
  return s;
}

namespace {

// Which kernel: the one for few rows reads a sequence's keys again (from L2) for every 16 rows, but
// starts sooner and spreads a small call over all SMs; the tile kernel reads them once for 384
// or 256 rows.  The host knows the token and sequence counts and the cache's capacity, not the
// lengths, so the rules go by averages (a batch of single tokens with one long chunk among
// them is better sent as two calls).  Measured (us, few rows / tiles; 16 heads of 64 on 4 kv heads
// unless stated):
//   cache: rows of a kv head per sequence, sequences x keys
//     8, 16 x 4,096, 16 kv heads: 49 / 86    32, 16 x 4,096: 19 / 35    32, 64 x 4,096: 57 / 87
//     64, 1 x 2,048: 9.3 / 22    64, 16 x 4,096: 30 / 36    64, 16 x 4,096, 16 kv heads: 137 / 89
//     128, 1 x 32,768: 28 / 28   128, 16 x 4,096: 51 / 36   128, 4 x 8,192, 2 kv heads of 128: 25 / 36
//   prompts x tokens, 16 kv heads
//     1 x 256: 8.4 / 10.8   1 x 400: 11.1 / 12.4   1 x 512: 19.2 / 13.3   8 x 64: 8.4 / 10.3
//     8 x 128: 15.1 / 13.9  64 x 16: 13.1 / 39.4   64 x 64: 29 / 39 (4 kv heads: 29 / 17)
bool takes_few_rows(const SeqAttnArgs& a, int num_sms) {
  if (a.kv.k) {
    const long long rows = (long long)a.T * a.group;            // of a kv head
    const long long tiles = (long long)a.T * a.Hq / kSmallRows;  // 16-row tiles of all kv heads
    return rows <= 32ll * a.B || (rows <= 128ll * a.B && tiles * (most_keys(a) / 64) <= 20000);
  }
  // Prompts: both kernels' times in us, from the units (16 rows x 64 keys; a tile's rows x its keys) of
  // all items, or of the items of a CTA where they are not cut.
  const int ctas = small_rows_ctas_per_sm(a.d) * num_sms, kBN = a.d == 64 ? Cfg<64>::kBN : Cfg<128>::kBN;
  const int cost = a.d == 64 ? Cfg<64>::kItemCost : Cfg<128>::kItemCost;
  const long long n = (a.T + a.B - 1) / a.B, items = count_items(a, kSmallRows);
  const long long tiles = count_items(a, 128 * seq_chains(a.d)), waves = (tiles + num_sms - 1) / num_sms;
  const double row_units = 4. + (n + 63) / 64, tile_units = cost + (double)((n + kBN - 1) / kBN);
  const double unit = a.d == 64 ? 0.55 : 0.74, tile_unit = a.d == 64 ? 0.64 : 1.5;
  const double few = rows_whole(a, ctas) ? 4.5 + unit * row_units * ((items + ctas - 1) / ctas)
                                         : 7.8 + unit * row_units * items / ctas;
  const double whole = tile_units < cost + 11. ? tile_units : cost + 11.;  // longer ones are cut
  const double cut = tile_units * tiles / num_sms;
  return few <= 6. + tile_unit * (tile_units <= cost + 11. ? whole * waves : cut > whole ? cut : whole);
}

}  // namespace

cudaError_t launch_seq_attention(const SeqAttnArgs& a, const SeqScratch& sc, int num_sms,
                                 cudaStream_t st) {
  using Launch = cudaError_t (*)(const SeqAttnArgs&, const SeqScratch&, int, cudaStream_t);
  static const Launch table[2][2][2] = {
      {{launch_tiles<64, false, false>, launch_tiles<64, false, true>},
       {launch_tiles<64, true, false>, launch_tiles<64, true, true>}},
      {{launch_tiles<128, false, false>, launch_tiles<128, false, true>},
       {launch_tiles<128, true, false>, launch_tiles<128, true, true>}}};
  prof_before(VP_KERNEL_SEQ_ATTN, st);
  const cudaError_t e = takes_few_rows(a, num_sms) ? launch_seq_rows(a, sc, num_sms, st)
                                          : table[a.d == 128][a.fp16 != 0][a.kv.k != nullptr](a, sc, num_sms, st);
  prof_after(st);
  return e;
}

}  // namespace vp
