// Attention of packed tokens over a cache in pages, on the tensor cores: the prefill (causal, sliding window, sinks) and the
// part of a decode step over a prefix that many sequences share.
//
//   S = Q K^T,  P = exp2(scale2 S - m),  O = sum P V,  l = sum P;  out = O / l,  lse = (m + log2 l) ln 2
//
// An item is up to 256 query rows of a (sequence, kv head), tokens times the G heads of the group, so that a tile of K and V
// serves the whole group, against a range of steps, each a tile of 128 keys.  paged_plan_kernel makes the list of items from the
// lengths, which are on the device; items that are long against the mean share of an SM are cut along the keys (few tokens on a long
// cache), and the list is in falling order of cost, dealt to the persistent CTAs forwards and backwards in turn.  What was cut is
// joined by paged_combine_kernel, or by the decode kernel.
//
// A CTA works on two streams of 128 rows; while one stream has its softmax the other has the tensor cores.  A stream is two
// warpgroups, two threads to a row, 64 of a tile's keys each.  Tensor memory: S of the streams at columns 0 and 128, O at 256 and
// 384.  P, rounded to 16 bits, overwrites S, the first 32 of the 64 columns of each warpgroup.  One warp issues all MMAs, and those of
// an issuing thread run in order, so
//   * S(j+1) may be issued behind P V(j), which reads P from the same columns;
//   * a stream that has been told of S(j) also knows that its P V(j-1) is done, and may rescale O itself.
// P is handed over in two halves, so that P V begins while the second is worked on.
// O is rescaled only when a row's maximum has grown by more than 2^8 over its reference, which on real logits is a few times a
// row; until then terms are at most 2^8, and the sums and O hold that in 32 bits.
#include <algorithm>

#include "exp2.cuh"
#include "paged_common.cuh"

namespace calidrop {

bool paged_kv_map(CUtensorMap* out, const void* base, const PagedGeom& g, int rows, int halves);

namespace {

using namespace tc;

constexpr int kSoftmaxWarps = 16;                 // two streams of two warpgroups
constexpr int kProducerWarp = 16, kMmaWarp = 17, kQWarp = 18;
constexpr int kThreads = 640;
constexpr int kSlots = 5;                         // K and V tiles in one ring, in the order in which they are used
constexpr int kTileBytes = kKvTileBytes;          // 32 KB
// What is in shared memory beside the two query blocks and the ring.
struct Tail {
  unsigned long long bars[2 * kSlots + 12];
  float max[2][2][128];                           // [stream][half][row]: maxima of a tile's halves, and at the end the sums
  uint32_t tmem;
  Ctl ctl;
};
constexpr int kSmemBytes = (2 + kSlots) * kTileBytes + sizeof(Tail);
static_assert(kSmemBytes <= 227 * 1024, "all of it: there is no static shared memory, so that the tiles begin at a multiple of 1024");
constexpr uint32_t kColO = 256;
constexpr int kPlanThreads = 1024;
constexpr int kBuckets = 256;

struct PlanArgs {
  PagedGeom g;
  const int *q_start, *kv_len;
  int n_seqs, causal, partial, grid;
  int item_tokens;                // tokens of an item: 2 * (128 / G)
  PagedPlanHeader* head;
  PagedItem* items;
  PagedTile* tiles;
  int max_tiles, max_items, max_split;
  long long max_rows;
};

// 0..255, growing with c: eight steps to a factor of two
__device__ __forceinline__ int cost_bucket(int c) {
  if (c < 16) return c;
  const int lg = 31 - __clz(c);
  return min(kBuckets - 1, (lg - 3) * 8 + 8 + ((c >> (lg - 3)) & 7));
}

__global__ void __launch_bounds__(kPlanThreads) paged_plan_kernel(const PlanArgs a) {
  __shared__ int tb[kMaxSequences + 1];      // first tile of each sequence
  __shared__ int warp_sum[32];
  __shared__ unsigned long long s_steps;
  __shared__ int s_hist[kBuckets];
  __shared__ unsigned long long s_rows;
  __shared__ int s_split, s_carry;
  const PagedGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  if (tid == 0) { s_steps = 0; s_rows = 0; s_split = 0; s_carry = 0; }
  if (tid < kBuckets) s_hist[tid] = 0;
  pdl_wait();
  const int cap = g.max_pages << g.lg_page;
  auto lengths = [&](int b, int& s0, int& n, int& kv) {
    s0 = __ldg(a.q_start + b);
    const int s1 = __ldg(a.q_start + b + 1);
    kv = __ldg(a.kv_len + b);
    const bool bad = s0 < 0 || s1 < s0 || s1 > g.n_tokens;
    n = bad ? 0 : s1 - s0;
    const bool bad_kv = kv < 0 || kv > cap;
    kv = min(max(kv, 0), cap);
    return bad || bad_kv;
  };
  // tiles of the sequences
  for (int base = 0; base < a.n_seqs; base += kPlanThreads) {
    const int b = base + tid;
    int nt = 0;
    if (b < a.n_seqs) {
      int s0, n, kv;
      if (lengths(b, s0, n, kv)) paged_flag(g.status, kBadLength);
      nt = (n + a.item_tokens - 1) / a.item_tokens;
    }
    int incl = nt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    if (warp == 0) {
      int v = warp_sum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
      }
      warp_sum[lane] = v;
    }
    __syncthreads();
    const int carry = s_carry;
    incl += carry + (warp ? warp_sum[warp - 1] : 0);
    if (b < a.n_seqs) tb[b + 1] = min(incl, a.max_tiles);   // (more than that only with a q_start that falls)
    __syncthreads();
    if (tid == 0) s_carry = min(carry + warp_sum[31], a.max_tiles);
  }
  if (tid == 0) tb[0] = 0;
  if (a.partial)
    for (int t = tid; t < g.n_tokens; t += kPlanThreads) a.tiles[t] = PagedTile{0, 0, 0, 0};
  __syncthreads();
  const int n_tiles = tb[a.n_seqs];
  auto tile_of = [&](int e, PagedItem& it) {
    int lo = 0, hi = a.n_seqs;             // tb[lo] <= e < tb[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tb[mid] <= e) lo = mid; else hi = mid;
    }
    int s0, n, kv;
    lengths(lo, s0, n, kv);
    const int t = e - tb[lo], first_tok = t * a.item_tokens;
    it.seq = lo;
    it.tok0 = s0 + first_tok;
    it.n_tok = min(a.item_tokens, n - first_tok);
    it.pos0 = a.causal ? kv - n + first_tok : 1 << 30;
    it.kv_end = a.causal ? max(0, min(kv, it.pos0 + it.n_tok)) : kv;
    it.win_lo = a.causal && g.window ? max(0, it.pos0 - g.window + 1) : 0;
    const int last = (it.kv_end + kPagedTileKeys - 1) / kPagedTileKeys, first = min(it.win_lo / kPagedTileKeys, last);
    it.near_tiles = (int)min((long long)first, ((long long)g.n_sink + kPagedTileKeys - 1) / kPagedTileKeys);
    it.skip = first - it.near_tiles;
    it.step0 = 0;
    it.n_steps = max(1, it.near_tiles + last - first);
    it.part_row = -1;
    it.rows = it.n_tok * g.G;
  };
  // how much work there is
  unsigned long long steps = 0;
  for (int e = tid; e < n_tiles; e += kPlanThreads) {
    PagedItem it;
    tile_of(e, it);
    steps += (unsigned)it.n_steps;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) steps += __shfl_xor_sync(0xffffffffu, steps, o);
  if (lane == 0 && steps) atomicAdd(&s_steps, steps);
  __syncthreads();
  const unsigned long long all = s_steps * (unsigned long long)g.Hkv;
  // A tile of rows is cut into as many chunks as it has times the mean share of an SM, rounded down: all chunks of cut tiles together are no more than the
  // SMs, and tiles of less than twice the share stay whole.
  auto chunks_of = [&](const PagedItem& it) {
    const unsigned long long k = (unsigned long long)it.n_steps * a.grid / all;
    return (int)max(1ull, min(k, (unsigned long long)it.n_steps));
  };
  for (int e = tid; e < n_tiles; e += kPlanThreads) {
    PagedItem it;
    tile_of(e, it);
    const int k = chunks_of(it), len = (it.n_steps + k - 1) / k;
    atomicAdd(&s_hist[cost_bucket(len)], (it.n_steps + len - 1) / len);
  }
  __syncthreads();
  if (warp == 0) {      // places of the buckets in the list, the costliest first
    int carry = 0;
    for (int base = kBuckets - 32; base >= 0; base -= 32) {
      const int i = base + 31 - lane, n = s_hist[i];
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
      }
      s_hist[i] = carry + incl - n;
      carry += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) { a.head->n_items = min(carry, a.max_items); a.head->n_tiles = n_tiles; }
  }
  __syncthreads();
  for (int e = tid; e < n_tiles; e += kPlanThreads) {
    PagedItem it;
    tile_of(e, it);
    int k = chunks_of(it);
    const int len = (it.n_steps + k - 1) / k;
    k = (it.n_steps + len - 1) / len;
    const int slot = atomicAdd(&s_hist[cost_bucket(len)], k);
    const bool parts = a.partial || k > 1;
    int row = -1;
    if (parts) {
      // (which rows a tile gets is a matter of who comes first; what is written there is not)
      const unsigned long long at = atomicAdd(&s_rows, (unsigned long long)k * g.Hkv * it.rows);
      if ((long long)(at + (unsigned long long)k * g.Hkv * it.rows) > a.max_rows) {
        paged_flag(g.status, kBadLength);    // (cannot be, but for a q_start that falls)
        row = -2;
      } else {
        row = (int)at;
      }
      if (!a.partial && row >= 0) {
        const int i = atomicAdd(&s_split, 1);
        if (i < a.max_split) a.tiles[i] = PagedTile{row, k, it.rows, it.tok0};
      }
      if (a.partial && row >= 0)
        for (int i = 0; i < it.n_tok; ++i) a.tiles[it.tok0 + i] = PagedTile{row + i * g.G, k, it.rows, 0};
    }
    for (int c = 0; c < k; ++c) {
      if (slot + c >= a.max_items) break;
      PagedItem x = it;
      x.step0 = c * len;
      x.n_steps = min(len, it.n_steps - x.step0);
      x.part_row = row < 0 ? row : row + c * g.Hkv * it.rows;
      a.items[slot + c] = x;
    }
  }
  __syncthreads();
  if (tid == 0) a.head->n_split = min(s_split, a.max_split);
}

struct KernelArgs {
  PagedGeom g;
  const int* block_table;
  const PagedPlanHeader* head;
  const PagedItem* items;
  float* parts;
  void* out;
  float* lse;
  int tokens;                 // of a stream: 128 / G
  int box_rows, lg_box;
};

__device__ __forceinline__ PagedItem load_item(const PagedItem* items, int e) {
  PagedItem it;
  const int4* s = reinterpret_cast<const int4*>(items + e);
  int4* d = reinterpret_cast<int4*>(&it);
  d[0] = __ldg(s); d[1] = __ldg(s + 1); d[2] = __ldg(s + 2);
  return it;
}

// The CTA's items: of every `grid` places of the list the CTA's own, from the front and from the back in turn.
struct Deal {
  int round, n;
  __device__ __forceinline__ explicit Deal(int n_) : round(0), n(n_) {}
  __device__ __forceinline__ int next() {
    const int i = (round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x;
    const long long w = (long long)round * gridDim.x + i;
    ++round;
    return w < n ? (int)w : -1;
  }
};

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1)
paged_attention_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                       const __grid_constant__ CUtensorMap v_map, const KernelArgs a) {
  extern __shared__ __align__(1024) unsigned char smem_al[];
  Tail& tail = *reinterpret_cast<Tail*>(smem_al + (2 + kSlots) * kTileBytes);
  Ctl& ctl = tail.ctl;

  const PagedGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t q_base = smem_u32(smem_al), ring = q_base + 2 * kTileBytes;
  const uint32_t bar0 = smem_u32(tail.bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (kSlots + s); };
  auto q_full = [&](int s) { return bar0 + 8u * (2 * kSlots + s); };
  auto q_empty = [&](int s) { return bar0 + 8u * (2 * kSlots + 2 + s); };
  auto s_full = [&](int s) { return bar0 + 8u * (2 * kSlots + 4 + s); };
  auto p_full = [&](int s, int part) { return bar0 + 8u * (2 * kSlots + 6 + (part ? 4 : 0) + s); };
  auto o_full = [&](int s) { return bar0 + 8u * (2 * kSlots + 8 + s); };

  if (tid == 0) {
    ctl.abort = 0;
    ctl.status = g.status;
    for (int s = 0; s < kSlots; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(q_full(s), 1); mbar_init(q_empty(s), 1);
      mbar_init(s_full(s), 1); mbar_init(p_full(s, 0), 256); mbar_init(p_full(s, 1), 256); mbar_init(o_full(s), 1);
    }
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(&tail.tmem), 512);
    tmem_relinquish();
  }
  // rows of the query blocks that no copy writes (128 is not a multiple of G) hold zeros
  for (int i = tid; i < 2 * kTileBytes / 16; i += kThreads) reinterpret_cast<uint4*>(smem_al)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = tail.tmem;
  pdl_wait();
  const int n_work = a.head->n_items * g.Hkv;
  const int R = a.tokens;

  if (warp == kProducerWarp) {
    // ------------------------------------------------------------ K and V, a copy per page box and half of the columns
    if (lane == 0) { tma_prefetch_desc(&k_map); tma_prefetch_desc(&v_map); }
    const int copies = 2 * (kTileKeys >> a.lg_box);
    const uint32_t box_bytes = (uint32_t)a.box_rows * kLineBytes;
    const int box = lane >> 1, half = lane & 1;
    int slot = 0;
    uint32_t ph = 1;                         // parity of a slot's emptiness
    bool ok = true;
    Deal deal(n_work);
    for (int w; ok && (w = deal.next()) >= 0;) {
      const int e = w / g.Hkv, h = w - e * g.Hkv;
      const PagedItem it = load_item(a.items, e);
      const int* table = a.block_table + (size_t)it.seq * g.max_pages;
      int ids = 0, ids_at = -1;
      for (int j = it.step0; ok && j < it.step0 + it.n_steps; ++j) {
        const int row0 = (j < it.near_tiles ? j : j + it.skip) * kTileKeys;
        const int pg = row0 >> g.lg_page, pg_last = (row0 + kTileKeys - 1) >> g.lg_page;
        if (ids_at < 0 || pg < ids_at || pg_last >= ids_at + 32) {
          ids_at = pg;
          ids = pg + lane < g.max_pages ? __ldg(table + pg + lane) : -1;
        }
        const int r = row0 + (box << a.lg_box);
        const bool need = lane < copies && r < it.kv_end && (r + a.box_rows > it.win_lo || r < g.n_sink);
        int page = __shfl_sync(0xffffffffu, ids, ((r >> g.lg_page) - ids_at) & 31);
        if (need && (page < 0 || page >= g.n_pages)) {
          paged_flag(g.status, kBadPage);
          page = g.n_pages;                   // outside the pool: the copy brings zeros
        }
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, need)) * box_bytes;
        const int in_page = r & (g.page - 1);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          ok = __all_sync(0xffffffffu, mbar_wait_far(&ctl, empty(slot), ph, 0x100u));
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(full(slot), bytes);
          __syncwarp();
          if (need)
            tma_load_4d(ring + slot * kTileBytes + half * (kTileBytes / 2) + (uint32_t)box * box_bytes, kv ? &v_map : &k_map,
                        full(slot), half * kHalfCols, in_page, h, page);
          if (++slot == kSlots) { slot = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == kQWarp) {
    // ------------------------------------------------------------ the query blocks of the streams
    if (lane == 0) {
      tma_prefetch_desc(&q_map);
      uint32_t ph[2] = {1u, 1u};
      bool ok = true;
      Deal deal(n_work);
      for (int w; ok && (w = deal.next()) >= 0;) {
        const int e = w / g.Hkv, h = w - e * g.Hkv;
        const PagedItem it = load_item(a.items, e);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (s * R >= it.n_tok) break;
          ok = ok && mbar_wait_far(&ctl, q_empty(s), ph[s], 0x200u);
          if (!ok) break;
          ph[s] ^= 1u;
          mbar_arrive_expect_tx(q_full(s), 2u * (uint32_t)(R * g.G) * kLineBytes);
          for (int half = 0; half < 2; ++half)
            tma_load_4d(q_base + s * kTileBytes + half * (kTileBytes / 2), &q_map, q_full(s), half * kHalfCols, 0, h, it.tok0 + s * R);
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------ all MMAs, the warp as a whole with one lane issuing
    constexpr uint32_t kTypes = kF16 ? ~((7u << 7) | (7u << 10)) : ~0u;    // f16 operands are type 0
    const uint32_t idesc_s = umma_idesc(128, 128, false, false) & kTypes;   // A = Q, B = K tile, both K-major
    const uint32_t idesc_o = umma_idesc(128, 128, false, true) & kTypes;    // A = P (tensor memory), B = V tile, MN-major
    const uint64_t dq = smem_desc_sw128(q_base, 16u, 1024u);
    const uint64_t dk = smem_desc_sw128(ring, 16u, 1024u);
    const uint64_t dv = smem_desc_sw128(ring, kTileBytes / 2, 1024u);
    const bool leader = elect_one();
    int slot = 0;
    uint32_t ph = 0, qph[2] = {0u, 0u}, pph[2] = {0u, 0u};
    bool ok = true;
    auto take = [&](int& sl) {              // the next tile of the ring, landed
      sl = slot;
      ok = ok && __all_sync(0xffffffffu, mbar_wait_far(&ctl, full(slot), ph, 0x300u));
      if (++slot == kSlots) { slot = 0; ph ^= 1u; }
    };
    auto issue_s = [&](int s, int k_slot) {
      if (leader) {
        const uint32_t d = tmem_base + (uint32_t)(s * 128);
        const uint64_t qd = desc_advance(dq, (uint32_t)s * kTileBytes), kd = desc_advance(dk, (uint32_t)k_slot * kTileBytes);
        umma_ss_imm<0>(d, qd, kd, idesc_s);
#pragma unroll
        for (int kk = 1; kk < kD / 16; ++kk)
          umma_ss_imm<1>(d, desc_advance(qd, kmajor_step_bytes(kTileBytes / 2, kk)),
                         desc_advance(kd, kmajor_step_bytes(kTileBytes / 2, kk)), idesc_s);
        umma_commit(s_full(s));
      }
      __syncwarp();
    };
    // P V of the keys of part 0 (0..31 and 64..95 of the tile) or 1; the P of keys 64.. sits at columns 64..
    auto issue_pv = [&](int s, int v_slot, int part, bool first) {
      if (leader) {
        const uint32_t d = tmem_base + kColO + (uint32_t)(s * 128), p = tmem_base + (uint32_t)(s * 128);
        const uint64_t vd = desc_advance(dv, (uint32_t)v_slot * kTileBytes);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int kk = (i >> 1) * 4 + (i & 1);           // the step of part 0; that of part 1 is two on
          const uint32_t col = p + (uint32_t)((kk >> 2) * 64 + (kk & 3) * 8) + (part ? 16u : 0u);
          const uint64_t v = desc_advance(vd, ((uint32_t)kk + (part ? 2u : 0u)) * 16u * kLineBytes);
          if (i == 0) umma_ts(d, col, v, idesc_o, first ? 0u : 1u);
          else umma_ts_imm<1>(d, col, v, idesc_o);
        }
      }
      __syncwarp();
    };
    auto commit = [&](uint32_t bar) {
      if (leader) umma_commit(bar);
      __syncwarp();
    };
    Deal deal(n_work);
    for (int w; ok && (w = deal.next()) >= 0;) {
      const PagedItem it = load_item(a.items, w / g.Hkv);
      const bool dual = it.n_tok > R;
      const int n = it.n_steps;
      int ks, vs;
      for (int s = 0; s < 2; ++s) {
        if (s == 1 && !dual) break;
        ok = ok && __all_sync(0xffffffffu, mbar_wait_far(&ctl, q_full(s), qph[s], 0x400u));
        qph[s] ^= 1u;
        if (s == 0) take(ks);
        if (!ok) break;
        tc_fence_after_sync();
        issue_s(s, ks);
        if (n == 1) commit(q_empty(s));
      }
      if (!ok) break;
      commit(empty(ks));
      for (int j = 0; j < n; ++j) {
        take(vs);
        if (!ok) break;
        // rows of V that none of the tokens sees may hold anything (or have not been loaded), and zero times that could be
        // a NaN: they become zeros
        const int row0 = (it.step0 + j < it.near_tiles ? it.step0 + j : it.step0 + j + it.skip) * kTileKeys;
        if (row0 + kTileKeys > it.kv_end || (row0 < it.win_lo && row0 + kTileKeys > g.n_sink)) {
          unsigned char* const vt = smem_al + 2 * kTileBytes + vs * kTileBytes;
          for (int r = lane >> 4; r < kTileKeys; r += 2) {
            const int t = row0 + r;
            if (t >= it.kv_end || (t < it.win_lo && t >= g.n_sink))
              *reinterpret_cast<uint4*>(vt + ((lane >> 3) & 1) * (kTileBytes / 2) + r * kLineBytes + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        const bool more = j + 1 < n;
        for (int s = 0; s < 2; ++s) {
          if (s == 1 && !dual) break;
          ok = ok && __all_sync(0xffffffffu, mbar_wait_far(&ctl, p_full(s, 0), pph[s], 0x500u));
          if (!ok) break;
          tc_fence_after_sync();
          issue_pv(s, vs, 0, j == 0);
          ok = __all_sync(0xffffffffu, mbar_wait_far(&ctl, p_full(s, 1), pph[s], 0x580u));
          pph[s] ^= 1u;
          if (!ok) break;
          tc_fence_after_sync();
          issue_pv(s, vs, 1, false);
          if (!more) {
            commit(o_full(s));
          } else {
            if (s == 0) take(ks);
            if (!ok) break;
            tc_fence_after_sync();
            issue_s(s, ks);
            if (j + 2 == n) commit(q_empty(s));
          }
        }
        if (!ok) break;
        commit(empty(vs));
        if (more) commit(empty(ks));
      }
    }
  } else if (warp < kSoftmaxWarps) {
    // ------------------------------------------------------------ softmax: two threads to a row
    constexpr float kBias = kF16 ? 7.f : 0.f;     // (see pack16; with the 2^8 of the lazy rescaling below the largest fp16)
    constexpr float kLazy = 8.f;
    const int s = warp >> 3, half = (warp >> 2) & 1, r = tid & 127;
    const uint32_t lane_bits = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_bits + (uint32_t)(s * 128 + half * 64), o_addr = s_addr + kColO;
    const int i_tok = s * R + r / g.G, head = r - (r / g.G) * g.G;
    const bool in_block = r < R * g.G;
    const f32x2 sc = pack2(g.scale2);
    // (read by the other warpgroup before it hands over its P: whoever sees the next S may write again)
    volatile float* const my_max = &tail.max[s][half][r];
    const volatile float* const other_max = &tail.max[s][half ^ 1][r];
    auto meet = [&]() { asm volatile("barrier.cta.sync %0, 256;" ::"r"(1 + s) : "memory"); };   // the stream's two warpgroups
    uint32_t sph = 0, oph = 0;
    bool ok = true;
    Deal deal(n_work);
    for (int w; ok && (w = deal.next()) >= 0;) {
      const int e = w / g.Hkv, h = w - e * g.Hkv;
      const PagedItem it = load_item(a.items, e);
      if (s * R >= it.n_tok) continue;
      const int pos = it.pos0 + i_tok;
      const int tok_last = min(it.n_tok, (s + 1) * R) - 1;
      // the keys from clear_lo (or from the first, as far as the sinks go) up to clear_hi are seen by all rows of the stream
      const int clear_hi = min(it.kv_end, it.pos0 + s * R + 1);
      const int clear_lo = g.window ? it.pos0 + tok_last - g.window + 1 : 0;
      float ref = -INFINITY, l = 0.f;       // reference of the row's terms (log2 domain), the sum of this thread's
#pragma unroll 1
      for (int j = 0; j < it.n_steps; ++j) {
        const int row0 = (it.step0 + j < it.near_tiles ? it.step0 + j : it.step0 + j + it.skip) * kTileKeys;
        // (a wait that runs out leaves the loop together with the other warps of the stream, or they would wait at `meet`: both
        // see the same barrier, and none of the phases behind it will complete)
        ok = __all_sync(0xffffffffu, mbar_wait(&ctl, s_full(s), sph, 0x600u));
        sph ^= 1u;
        tc_fence_after_sync();
        uint32_t x[2][32];
        tmem_ld32_issue(s_addr, x[0]);
        tmem_ld32_issue(s_addr + 32, x[1]);
        tmem_ld_wait(x[0]);
        tmem_ld_wait(x[1]);
        if (row0 + kTileKeys > clear_hi || (row0 < clear_lo && row0 + kTileKeys > g.n_sink)) {
          const int key0 = row0 + half * 64;
          auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };   // the n lowest bits
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int k0 = key0 + 32 * q;
            uint32_t seen = below(min(it.kv_end, pos + 1) - k0);
            if (g.window) seen &= ~below(pos - g.window + 1 - k0) | below(g.n_sink - k0);
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!((seen >> c) & 1u)) x[q][c] = 0xff800000u;
          }
        }
        float mx[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          mx[q] = __uint_as_float(x[q >> 1][(q & 1) * 16]);
#pragma unroll
          for (int c = 1; c < 16; ++c) mx[q] = fmaxf(mx[q], __uint_as_float(x[q >> 1][(q & 1) * 16 + c]));
        }
        float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        *my_max = top;
        meet();
        top = fmaxf(top, *other_max) * g.scale2 - kBias;
        const bool grow = top > ref + kLazy;             // (from -inf on the first key that is seen)
        if (__any_sync(0xffffffffu, grow)) {
          const float f = grow ? ex2_approx(ref - top) : 1.f;
          const bool had = __any_sync(0xffffffffu, grow && ref > -INFINITY);
          if (grow) { l *= f; ref = top; }
          if (had && j > 0) {                            // this half of O's columns
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              uint32_t o[16];
              tmem_ld16(o_addr + 16 * q, o);
#pragma unroll
              for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
              tmem_st16(o_addr + 16 * q, o);
            }
          }
        }
        const f32x2 nref = pack2(ref == -INFINITY ? 0.f : -ref);
        f32x2 sum0 = 0ull, sum1 = 0ull;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t packed[16];
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const f32x2 y = exp2_pair<false>(fma2(pack2(x[q][c], x[q][c + 1]), sc, nref), c / 2);
            if (c & 2) sum1 = add2(sum1, y);
            else sum0 = add2(sum0, y);
            const float2 p = unpack2(y);
            packed[c >> 1] = pack16<kF16>(p.x, p.y);
          }
          tmem_st16(s_addr + 16 * q, packed);
          tmem_st_wait();
          tc_fence_before_sync();
          mbar_arrive(p_full(s, q));
        }
        const float2 t = unpack2(add2(sum0, sum1));
        l += t.x + t.y;
        if (!ok) break;
      }
      if (!ok) break;
      ok = __all_sync(0xffffffffu, mbar_wait(&ctl, o_full(s), oph, 0x700u));
      oph ^= 1u;
      tc_fence_after_sync();
      // the row's sum, of the lower keys and the upper ones in this order
      *my_max = l;
      meet();
      const float l_other = *other_max;
      l = half ? l_other + l : l + l_other;
      meet();                                            // (the next item writes there)
      if (!ok) break;
      const bool valid = in_block && i_tok < it.n_tok;
      if (it.part_row < 0) {
        const float inv = l == 0.f ? 0.f : 1.f / l;        // no key seen: zeros
        const size_t row = (size_t)(it.tok0 + i_tok) * g.Hq + h * g.G + head;
        uint4* const dst = reinterpret_cast<uint4*>(a.out) + row * (kD / 8) + half * 8;
        const bool store = valid && it.part_row == -1;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t o[32];
          tmem_ld32(o_addr + 32 * q, o);
          if (store) {
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
              uint4 v;
              v.x = pack16<kF16>(__uint_as_float(o[c]) * inv, __uint_as_float(o[c + 1]) * inv);
              v.y = pack16<kF16>(__uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv);
              v.z = pack16<kF16>(__uint_as_float(o[c + 4]) * inv, __uint_as_float(o[c + 5]) * inv);
              v.w = pack16<kF16>(__uint_as_float(o[c + 6]) * inv, __uint_as_float(o[c + 7]) * inv);
              dst[q * 4 + c / 8] = v;
            }
          }
        }
        if (store && a.lse && half == 0) a.lse[row] = l == 0.f ? -INFINITY : (ref + log2f(l)) * kLn2;
      } else {
        float* const dst = a.parts + ((size_t)it.part_row + (size_t)h * it.rows + (size_t)i_tok * g.G + head) * kPagedPartStride;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t o[32];
          tmem_ld32(o_addr + 32 * q, o);
          if (valid) {
#pragma unroll
            for (int c = 0; c < 32; c += 4)
              *reinterpret_cast<uint4*>(dst + half * 64 + 32 * q + c) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
          }
        }
        if (valid && half == 0) *reinterpret_cast<float2*>(dst + kD) = make_float2(ref, l);
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  pdl_trigger();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
}

// Rows of the tiles that were cut along the keys: a warp to a row, four outputs a lane, the chunks in their order.
template <bool kF16>
__global__ void __launch_bounds__(256) paged_combine_kernel(const KernelArgs a, const PagedTile* tiles) {
  pdl_trigger();
  pdl_wait();
  const PagedGeom& g = a.g;
  const int lane = threadIdx.x & 31;
  const long long n = (long long)a.head->n_split * g.Hkv * kPagedRows;
  for (long long w = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; w < n; w += (long long)gridDim.x * (blockDim.x >> 5)) {
    const int r = (int)(w % kPagedRows), h = (int)((w / kPagedRows) % g.Hkv);
    const int4 t = __ldg(reinterpret_cast<const int4*>(tiles) + w / kPagedRows / g.Hkv);   // {row, chunks, rows, first token}
    if (r >= t.z) continue;
    Partial p;
    p.o[0] = p.o[1] = p.o[2] = p.o[3] = 0.f; p.m = -INFINITY; p.l = 0.f;
    join_rows(p, t.y, lane, [&](int i) { return a.parts + ((size_t)t.x + ((size_t)i * g.Hkv + h) * t.z + r) * kPagedPartStride; });
    const size_t row = (size_t)(t.w + r / g.G) * g.Hq + h * g.G + r % g.G;
    const float inv = p.l == 0.f ? 0.f : 1.f / p.l;
    uint2 v;
    v.x = pack16<kF16>(p.o[0] * inv, p.o[1] * inv);
    v.y = pack16<kF16>(p.o[2] * inv, p.o[3] * inv);
    reinterpret_cast<uint2*>(a.out)[row * (kD / 4) + lane] = v;
    if (a.lse && lane == 0) a.lse[row] = p.l == 0.f ? -INFINITY : (p.m + log2f(p.l)) * kLn2;
  }
}

bool paged_q_map(CUtensorMap* out, const void* q, const PagedGeom& g, int tokens) {
  const uint64_t dims[3] = {(uint64_t)g.G, (uint64_t)g.Hkv, (uint64_t)g.n_tokens};
  const uint64_t strides[3] = {kRowBytes, (uint64_t)g.G * kRowBytes, (uint64_t)g.q_stride * 2};
  const uint32_t box[3] = {(uint32_t)g.G, 1, (uint32_t)tokens};
  return make_tensor_map_bf16(out, q, 4, dims, strides, box);
}

template <bool kF16>
cudaError_t launch(const PagedAttnArgs& d, const PagedWs& ws, cudaStream_t st) {
  static OncePerDevice granted;
  cudaError_t e = grant_smem(paged_attention_kernel<kF16>, kSmemBytes, granted);
  if (e != cudaSuccess) return e;
  PlanArgs p{};
  p.g = d.g;
  p.q_start = d.q_start; p.kv_len = d.kv_len;
  p.n_seqs = d.n_seqs; p.causal = d.causal; p.partial = d.partial; p.grid = kSms;
  const int tokens = 128 / d.g.G;
  p.item_tokens = 2 * tokens;
  p.head = (PagedPlanHeader*)(d.wsp + kPagedPlan);
  p.items = (PagedItem*)(d.wsp + ws.items);
  p.tiles = (PagedTile*)(d.wsp + ws.tiles);
  p.max_tiles = ws.max_tiles; p.max_items = ws.max_items; p.max_split = ws.max_split; p.max_rows = ws.max_rows;
  KernelArgs a{};
  a.g = d.g;
  a.block_table = d.block_table; a.head = p.head; a.items = p.items;
  a.parts = (float*)(d.wsp + ws.part_o);
  a.out = d.out; a.lse = d.lse;
  a.tokens = tokens;
  a.box_rows = std::min(d.g.page, kTileKeys);
  while ((1 << a.lg_box) < a.box_rows) ++a.lg_box;
  CUtensorMap qm, km, vm;
  if (!paged_q_map(&qm, d.q, d.g, tokens) || !paged_kv_map(&km, d.K, d.g, a.box_rows, 0) || !paged_kv_map(&vm, d.V, d.g, a.box_rows, 0))
    return cudaErrorInvalidValue;
  e = launch_pdl(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
  if (e == cudaSuccess) e = launch_pdl(paged_attention_kernel<kF16>, dim3(kSms), dim3(kThreads), kSmemBytes, st, qm, km, vm, a);
  if (e != cudaSuccess) return e;
  count_launch(2);
  if (!d.partial) {
    e = launch_pdl(paged_combine_kernel<kF16>, dim3(4 * kSms), dim3(256), 0, st, a, (const PagedTile*)p.tiles);
    if (e == cudaSuccess) count_launch(1);
  }
  return e;
}

}  // namespace

// K or V as [page][kv head][row][128], in boxes of `rows` rows: 64 columns, or (halves = 2) both halves of the columns behind one
// another.
bool paged_kv_map(CUtensorMap* out, const void* base, const PagedGeom& g, int rows, int halves) {
  const uint64_t dims[3] = {(uint64_t)g.page, (uint64_t)g.Hkv, (uint64_t)g.n_pages};
  const uint64_t strides[3] = {kRowBytes, (uint64_t)g.page * kRowBytes, (uint64_t)g.page_stride * 2};
  const uint32_t box[3] = {(uint32_t)rows, 1, 1};
  return halves ? make_tile_map_bf16(out, base, 4, dims, strides, box, halves) : make_tensor_map_bf16(out, base, 4, dims, strides, box);
}

PagedWs paged_ws(int B, int Hq, int Hkv, int n_tokens, int n_groups) {
  PagedWs w{};
  const int G = Hq / Hkv, item_tokens = 2 * (128 / G);
  w.max_tiles = n_tokens / item_tokens + std::max(B, n_groups);
  w.max_split = kSms;
  w.max_items = w.max_tiles + kSms;
  // chunks of cut tiles are no more than the SMs; with a shared prefix every token has a row in any case
  w.max_rows = (long long)kSms * std::min((long long)kPagedRows, (long long)n_tokens * G) + (n_groups ? (long long)B * Hq : 0);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t off = kPagedPlan + 256;
  w.items = off;  off = up(off + (size_t)w.max_items * sizeof(PagedItem));
  w.tiles = off;  off = up(off + (size_t)std::max(w.max_split, n_groups ? B : 0) * sizeof(PagedTile));
  w.part_o = off; off = up(off + (size_t)w.max_rows * kPagedPartStride * 4);
  w.total = off;
  return w;
}

cudaError_t launch_paged_attention(const PagedAttnArgs& a, const PagedWs& ws, cudaStream_t st) {
  return a.g.f16 ? launch<true>(a, ws, st) : launch<false>(a, ws, st);
}

}  // namespace calidrop
