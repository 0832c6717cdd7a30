// Attention of packed tokens over a cache in pages, on the tensor cores: the prefill (causal, sliding window, sinks) and the
// part of a decode step over a prefix that many sequences share.
//
//   S = Q K^T,  P = exp2(scale2 S - m),  O = sum P V,  l = sum P;  out = O / l,  lse = (m + log2 l) ln 2
//
// A tile is up to 256 query rows of a (sequence, kv head), tokens times the G heads of the group, so that a tile of K and V serves
// the whole group; its work is a number of steps, each 128 keys.  The lengths are on the device and may be anything, so the work is
// dealt there: every CTA sums the steps of all tiles, lists the heavy ones (half an SM's mean share or more: few) from the
// heaviest down, cuts those of twice the share or more along the keys, and takes one piece after another from a common counter, the
// heavy tiles ahead of the others, which come sequence by sequence, the last tokens (which see the most keys) first.  Of a tile that is
// cut each CTA leaves partial rows and the last to arrive joins them, in the order of the keys; those of a shared prefix are
// joined by the decode kernel.
//
// A CTA works on two streams of 128 rows; while one stream has its softmax the other has the tensor cores.  A stream is two
// warpgroups, two threads to a row, 64 of a tile's keys each.  Tensor memory: S of the streams at columns 0 and 128, O at 256 and
// 384.  P, rounded to 16 bits, overwrites S, the first 32 of the 64 columns of each warpgroup.  One warp issues all MMAs, and those of an
// issuing thread run in order, so
//   * S(j+1) may be issued behind P V(j), which reads P from the same columns;
//   * a stream that has been told of S(j) also knows that its P V(j-1) is done, and may rescale O itself.
// P is handed over in two parts, of 48 keys and 16, so that little of P V is left when the last is done.
//
// What bounds it: for long prompts the power limit, behind it the chain of a stream's step (S, its way to the registers, the exponentials, P,
// P V: 3000 cycles for two streams where the tensor cores need 2048); causal, 32 heads x 8192 tokens take 501 to 516 us from box to box
// (1.08 PFLOP/s; 567 with a thread to a row, which held 128 logits and worked on few exponentials at a time).  For short prompts the longest
// tile (1024 tokens: eight steps where the mean of an SM is four) and the launch: 6 us of start, list and first loads, and 3 at the end.  For a prefix
// shared by few rows the memory (64 KB a step and SM in 1.4 us) and shares that are rounded down (pieces of 15 steps for a mean of 10).
#include <algorithm>

#include "exp2.cuh"
#include "paged_common.cuh"

namespace calidrop {

bool paged_kv_map(CUtensorMap* out, const void* base, const PagedGeom& g, int rows, int halves);

namespace {

using namespace tc;

constexpr int kSoftmaxWarps = 16;                 // two streams of two warpgroups
constexpr int kProducerWarp = 16, kStewardWarp = 17, kMmaWarp = 18;
constexpr int kThreads = 640;
constexpr int kSlots = 5;                         // K and V tiles in one ring, in the order in which they are used
constexpr int kTileBytes = kKvTileBytes;          // 32 KB
constexpr uint32_t kColO = 256;
constexpr int kMaxHeavy = 2 * kSms;               // tiles of at least half an SM's mean share
constexpr int kItemReaders = kSoftmaxWarps + 2;   // warps that take a piece from the producer

// A piece of work: a tile of rows of one kv head against a range of steps.
struct Piece {
  int tok0, n_tok;       // its tokens
  int seq;               // whose row of the block table
  int head;              // kv head
  int pos0;              // position of the first token
  int kv_end;            // keys at and beyond it are seen by none of the tokens
  int win_lo;            // keys in [n_sink, win_lo) neither
  int near_tiles, skip;  // step j is tile j, or j + skip from step near_tiles on
  int step0, n_steps;    // n_steps 0: there is no more work
  int part_row;          // of a tile that is cut, its first partial row for this head and chunk; or -1
  int part_step;         // rows from a chunk's partial rows to the next chunk's
  int n_chunks, counter; // chunks, and which arrival counter of them
  int chunk_steps;
};
static_assert(sizeof(Piece) == 64, "four 16-byte vectors");

// A heavy tile.
struct Heavy {
  int seq, t;            // tile t of a sequence
  int n_chunks, chunk_steps;
  int first_piece;       // chunks ahead of its own, over the list
  int part_row;          // first partial row, if it is cut
  int counter;           // first arrival counter, if it is cut
  int pad;
};

// What is in shared memory beside the two query blocks and the ring.
struct Tail {
  unsigned long long bars[2 * kSlots + 14];
  Piece piece[2];
  float max[2][2][128];                           // [stream][half][row]: maxima of a tile's halves, and at the end the sums
  uint32_t tmem;
  int last[2];
  Ctl ctl;
};
constexpr int kSmemBytes = (2 + kSlots) * kTileBytes + sizeof(Tail);
static_assert(kSmemBytes <= 227 * 1024, "all of it: there is no static shared memory, so that the tiles begin at a multiple of 1024");
static_assert((kMaxSequences + 1 + 63) * 4 + kMaxHeavy * 16 <= kSlots * kTileBytes, "the list of work is made where the ring will be");

struct KernelArgs {
  PagedGeom g;
  const int *block_table, *q_start, *kv_len;
  int n_seqs, causal, partial;
  int tokens;                 // of a stream: 128 / G
  int g_inv;                  // row / G = row * g_inv >> 16 for a row of a stream
  int box_rows, lg_box;
  unsigned* sched;            // [0] next piece, [1] CTAs that are done, then the arrival counters; all zero between launches
  Heavy* heavy;               // a list for each CTA
  PagedToken* token_parts;    // partial: where the decode kernel finds its rows
  float* parts;
  long long max_rows;
  void* out;
  float* lse;
};

// Whether the tokens [s0, s1) are those of a sequence: else it is taken to have none.
__device__ __forceinline__ bool good_starts(const KernelArgs& a, int s0, int s1) { return s0 >= 0 && s1 >= s0 && s1 <= a.g.n_tokens; }

// Sequence b: its first token, number of tokens and cached rows, held to what the buffers allow.
__device__ __forceinline__ bool lengths(const KernelArgs& a, int b, int& s0, int& n, int& kv) {
  const int cap = a.g.max_pages << a.g.lg_page;
  s0 = __ldg(a.q_start + b);
  const int s1 = __ldg(a.q_start + b + 1);
  kv = __ldg(a.kv_len + b);
  const bool bad = !good_starts(a, s0, s1), bad_kv = kv < 0 || kv > cap;
  n = bad ? 0 : s1 - s0;
  kv = min(max(kv, 0), cap);
  return bad || bad_kv;
}

// Tile t of a sequence (the last tokens first), all of its steps.
__device__ __forceinline__ void tile_piece(const KernelArgs& a, int seq, int s0, int n, int kv, int t, Piece& p) {
  const PagedGeom& g = a.g;
  const int size = 2 * a.tokens, n_tiles = (n + size - 1) / size;
  const int first_tok = (n_tiles - 1 - t) * size;
  p.seq = seq;
  p.tok0 = s0 + first_tok;
  p.n_tok = min(size, n - first_tok);
  p.pos0 = a.causal ? kv - n + first_tok : 1 << 30;
  p.kv_end = a.causal ? max(0, min(kv, p.pos0 + p.n_tok)) : kv;
  p.win_lo = a.causal && g.window ? max(0, p.pos0 - g.window + 1) : 0;
  const int last = (p.kv_end + kPagedTileKeys - 1) / kPagedTileKeys, first = min(p.win_lo / kPagedTileKeys, last);
  p.near_tiles = (int)min((long long)first, ((long long)g.n_sink + kPagedTileKeys - 1) / kPagedTileKeys);
  p.skip = first - p.near_tiles;
  p.step0 = 0;
  p.n_steps = max(1, p.near_tiles + last - first);
  p.part_row = -1; p.part_step = 0; p.n_chunks = 1; p.counter = 0; p.chunk_steps = 1;
}

// Half the mean share of an SM or more.
__device__ __forceinline__ bool is_heavy(int n, unsigned long long all) { return 2ull * n * gridDim.x >= all; }

// Into how many chunks a tile of n steps is cut, `all` being the steps of all tiles and heads.  Twice the mean share of an SM or more is cut into as many
// pieces as it has shares, so that all pieces of cut tiles together are no more than the SMs.  Joining k chunks of `rows` rows costs the
// last CTA about 8 cycles a row and chunk, and a chunk less takes n / k steps of 3000 cycles off: beyond sqrt(375 n / rows) chunks
// the joining costs more than it gives, and so it does for chunks of less than 8 steps (a shared prefix is joined elsewhere, by many).
__device__ __forceinline__ int chunks_of(const KernelArgs& a, int n, int rows, unsigned long long all) {
  const unsigned shares = all >> 31 ? 0u : (unsigned)n * gridDim.x / (unsigned)all;     // (n is below 2^23)
  if (shares < 2) return 1;
  int k = min((int)shares, n);
  if (!a.partial) k = max(1, min(min(k, n / 8), (int)sqrtf(375.f * n / rows)));
  const int len = (n + k - 1) / k;
  return (n + len - 1) / len;
}

// exp2(scale2 x - ref) of keys kFrom..kTo - 1, rounded in pairs, and their sum.  All on the special-function unit: with 2, 3, 4, 5 of 16 pairs on
// the FMA pipe (see exp2.cuh) an 8192-token prompt takes 510, 509, 512, 518 us instead of 501.
template <bool kF16, int kFrom, int kTo>
__device__ __forceinline__ void terms(const uint32_t (&x)[32], f32x2 scale2, float ref, uint32_t (&packed)[16], f32x2& sum) {
  const f32x2 nref = pack2(ref == -INFINITY ? 0.f : -ref);
#pragma unroll
  for (int c = kFrom; c < kTo; c += 2) {
    const f32x2 y = exp2_unit2(fma2(pack2(x[c], x[c + 1]), scale2, nref));
    sum = add2(sum, y);
    const float2 p = unpack2(y);
    packed[(c - kFrom) >> 1] = pack16<kF16>(p.x, p.y);
  }
}

// The list of work: heavy tiles, in falling order of their chunks, at a.heavy; made by all threads of the CTA in `scratch`, or for a few
// tiles by one warp.
struct WorkList {
  int n_tiles, n_heavy_pieces;
  unsigned long long all_steps;    // of all tiles and heads
};

// Up to 32 sequences: their tiles are counted by every warp for itself, lane b holding sequence b.
struct Few {
  int s0, n, kv, nt, incl;
  __device__ __forceinline__ int load(const KernelArgs& a, int lane, bool tell) {    // returns the number of tiles
    const int size = 2 * a.tokens;
    s0 = n = kv = nt = 0;
    if (lane < a.n_seqs) {
      if (lengths(a, lane, s0, n, kv) && tell) paged_flag(a.g.status, kBadLength);
      nt = (n + size - 1) / size;
    }
    incl = nt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if ((threadIdx.x & 31) >= o) incl += u;
    }
    return __shfl_sync(0xffffffffu, incl, 31);
  }
  // Tile e of each lane (any number for lanes that have none): all lanes call.
  __device__ __forceinline__ int tile(const KernelArgs& a, int e, Piece& p) const {
    int own = 0;                         // sequences whose tiles all lie ahead of e
#pragma unroll
    for (int step = 16; step > 0; step >>= 1) {
      const int v = __shfl_sync(0xffffffffu, incl, (own + step - 1) & 31);
      if (v <= e) own += step;
    }
    own = min(own, 31);
    const int first = __shfl_sync(0xffffffffu, incl - nt, own);
    const int b0 = __shfl_sync(0xffffffffu, s0, own), bn = __shfl_sync(0xffffffffu, n, own), bkv = __shfl_sync(0xffffffffu, kv, own);
    tile_piece(a, own, b0, bn, bkv, e - first, p);
    return e - first;
  }
};

// The list for up to 32 tiles, a lane to a tile; by one warp.
__device__ __forceinline__ WorkList make_short_list(const KernelArgs& a, const Few& few, int n_tiles, int lane) {
  const PagedGeom& g = a.g;
  Heavy* const heavy = a.heavy + (size_t)blockIdx.x * kMaxHeavy;
  WorkList r{n_tiles, 0, 0};
  Piece p;
  const int t = few.tile(a, min(lane, n_tiles - 1), p);
  const bool mine = lane < n_tiles;
  r.all_steps = (unsigned long long)__reduce_add_sync(0xffffffffu, mine ? (unsigned)p.n_steps : 0u) * g.Hkv;   // (32 tiles of less than 2^23 steps)
  const int rows = p.n_tok * g.G;
  int k = mine ? chunks_of(a, p.n_steps, rows, r.all_steps) : 0;
  if (a.n_seqs == 1 && !__any_sync(0xffffffffu, k > 1)) {       // the tiles of one sequence are in order
    r.all_steps = ~0ull;                 // (none is heavy)
    return r;
  }
  const bool is = mine && is_heavy(p.n_steps, r.all_steps);
  const int len = is ? (p.n_steps + k - 1) / k : 0;
  if (!is) k = 0;
  const int part_rows = k > 1 ? k * g.Hkv * rows : 0;
  int rank = 0, pieces = 0, rows_at = a.partial ? g.n_tokens * g.Hq : 0, cut_ahead = 0;
  for (int j = 0; j < n_tiles; ++j) {
    const int lj = __shfl_sync(0xffffffffu, len, j), kj = __shfl_sync(0xffffffffu, k, j), rj = __shfl_sync(0xffffffffu, part_rows, j);
    if (lj > len || (lj == len && j < lane)) {
      rank += kj > 0;
      pieces += kj;
      rows_at += rj;
      cut_ahead += kj > 1;
    }
  }
  if (is) heavy[rank] = Heavy{p.seq, t, k, len, pieces, rows_at, 2 * g.Hkv * cut_ahead, 0};
  r.n_heavy_pieces = __reduce_add_sync(0xffffffffu, (unsigned)k);
  __syncwarp();
  return r;
}

__device__ __noinline__ WorkList make_list(const KernelArgs& a, const Few& few, int few_tiles, unsigned char* scratch, int tid) {
  const PagedGeom& g = a.g;
  constexpr int kN = kThreads, kWarps = kN / 32;
  const int lane = tid & 31, warp = tid >> 5;
  const int size = 2 * a.tokens;
  int* const tb = reinterpret_cast<int*>(scratch);                    // [n_seqs + 1]: first tiles of the sequences
  int* const sums = tb + kMaxSequences + 1;                           // [63]
  int2* const found = reinterpret_cast<int2*>(sums + 63);             // [kMaxHeavy] {tile, steps of a chunk}
  int2* const order = found + kMaxHeavy;                              // by rank: {chunks, rows of a head}
  Heavy* const heavy = a.heavy + (size_t)blockIdx.x * kMaxHeavy;
  auto scan = [&](int v, int& all) {       // what lies ahead of this thread, and the sum
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const int u = sums[w];
      if (w < warp) before += u;
      all += u;
    }
    return before + incl - v;
  };
  WorkList r{0, 0, 0};
  const bool is_few = a.n_seqs <= 32;
  if (is_few) r.n_tiles = few_tiles;
  const int most_tiles = g.n_tokens / size + a.n_seqs;     // of starts that do not fall
  for (int base = 0; !is_few && base < a.n_seqs; base += kN) {
    const int b = base + tid;
    int nt = 0, all;
    if (b < a.n_seqs) {
      int s0, n, kv;
      if (lengths(a, b, s0, n, kv) && blockIdx.x == 0) paged_flag(g.status, kBadLength);
      nt = (n + size - 1) / size;
    }
    const int before = scan(nt, all);
    if (b < a.n_seqs) tb[b] = r.n_tiles + before;
    if (all > most_tiles - r.n_tiles) return WorkList{0, 0, 0};   // (flagged above; the sums could overflow)
    r.n_tiles += all;
  }
  if (!is_few) {
    if (tid == 0) tb[a.n_seqs] = r.n_tiles;
    __syncthreads();
  }
  auto tile_of = [&](int e, Piece& p) {      // all lanes of a warp call; returns the tile's place in its sequence
    if (is_few) return few.tile(a, e, p);
    int lo = 0, hi = a.n_seqs;             // tb[lo] <= e < tb[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tb[mid] <= e) lo = mid; else hi = mid;
    }
    int s0, n, kv;
    lengths(a, lo, s0, n, kv);
    tile_piece(a, lo, s0, n, kv, e - tb[lo], p);
    return e - tb[lo];
  };
  unsigned long long steps = 0;
  int my_steps = 0;             // of tile tid
  for (int base = 0; base < r.n_tiles; base += kN) {
    const int e = base + tid;
    Piece p;
    tile_of(min(e, r.n_tiles - 1), p);
    if (e < r.n_tiles) steps += (unsigned)p.n_steps;
    if (base == 0) my_steps = p.n_steps;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) steps += __shfl_xor_sync(0xffffffffu, steps, o);
  unsigned long long* const wide = reinterpret_cast<unsigned long long*>(found);
  if (lane == 0) wide[warp] = steps;
  __syncthreads();
  steps = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) steps += wide[w];
  __syncthreads();
  r.all_steps = steps * (unsigned long long)g.Hkv;
  // heavy tiles, in the order of the tiles
  int n_heavy = 0;
  for (int base = 0; base < r.n_tiles; base += kN) {
    const int e = base + tid;
    if (base) {
      Piece p;
      tile_of(min(e, r.n_tiles - 1), p);
      my_steps = p.n_steps;
    }
    const bool is = e < r.n_tiles && is_heavy(my_steps, r.all_steps);
    int all;
    const int i = n_heavy + scan(is ? 1 : 0, all);
    if (is && i < kMaxHeavy) found[i] = make_int2(e, 0);
    n_heavy += all;
  }
  n_heavy = min(n_heavy, kMaxHeavy);   // (there are no more)
  if (n_heavy == 0) return r;
  // ... the heaviest first
  __syncthreads();
  static_assert(kMaxHeavy <= kN, "a thread to a tile of the list");
  Piece p;
  const bool mine = tid < n_heavy;
  const int e = found[min(tid, n_heavy - 1)].x;
  const int t = tile_of(e, p);
  const int k = chunks_of(a, p.n_steps, p.n_tok * g.G, r.all_steps), len = (p.n_steps + k - 1) / k;
  if (mine) found[tid].y = len;
  __syncthreads();
  if (mine) {
    int rank = tid;
    if (a.n_seqs > 1) {                // (one sequence's are in order)
      rank = 0;
      for (int j = 0; j < n_heavy; ++j) {
        const int l = found[j].y;
        rank += l > len || (l == len && j < tid);
      }
    }
    order[rank] = make_int2(k, p.n_tok * g.G);
    heavy[rank] = Heavy{p.seq, t, k, len, 0, 0, 0, 0};
  }
  __syncthreads();
  int pieces = 0, rows = a.partial ? g.n_tokens * g.Hq : 0, counters = 0;
  for (int base = 0; base < n_heavy; base += kN) {
    const int i = base + tid;
    const int2 o = i < n_heavy ? order[i] : make_int2(0, 0);
    const bool cut = o.x > 1;
    int all_pieces, all_rows, all_counters;
    const int p0 = scan(o.x, all_pieces), r0 = scan(cut ? o.x * g.Hkv * o.y : 0, all_rows), c0 = scan(cut ? 2 * g.Hkv : 0, all_counters);
    if (i < n_heavy) {
      heavy[i].first_piece = pieces + p0;
      heavy[i].part_row = rows + r0;
      heavy[i].counter = counters + c0;
    }
    pieces += all_pieces; rows += all_rows; counters += all_counters;
  }
  r.n_heavy_pieces = pieces;
  __syncthreads();
  return r;
}

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
  auto s_full = [&](int s) { return bar0 + 8u * (2 * kSlots + 2 + s); };
  auto p_full = [&](int s, int part) { return bar0 + 8u * (2 * kSlots + 4 + 2 * part + s); };
  auto o_full = [&](int s) { return bar0 + 8u * (2 * kSlots + 8 + s); };
  auto piece_full = [&](int i) { return bar0 + 8u * (2 * kSlots + 10 + i); };
  auto piece_empty = [&](int i) { return bar0 + 8u * (2 * kSlots + 12 + i); };

  if (tid == 0) {
    ctl.abort = 0;
    ctl.status = g.status;
    for (int s = 0; s < kSlots; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(q_full(s), 1);
      mbar_init(s_full(s), 1); mbar_init(p_full(s, 0), 256 + 1); mbar_init(p_full(s, 1), 256); mbar_init(o_full(s), 1);
      mbar_init(piece_full(s), 1); mbar_init(piece_empty(s), kItemReaders);
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
  const int R = a.tokens;

  // ---- the list of work, the same in every CTA; only the producer needs it
  const int size = 2 * R;
  WorkList work{};
  bool is_short = false;
  Few few{};
  int few_tiles = 0;
  if (a.n_seqs <= 32) {
    few_tiles = few.load(a, lane, blockIdx.x == 0 && warp == 0);
    is_short = few_tiles <= 32;
    if (is_short && warp == kProducerWarp && few_tiles > 0) work = make_short_list(a, few, few_tiles, lane);
  }
  if (!is_short) work = make_list(a, few, few_tiles, smem_al + 2 * kTileBytes, tid);
  if (a.partial)      // tokens of no group, or of one that is not taken, have no partial rows; the workspace may hold anything there
    for (int t0 = blockIdx.x * kThreads + warp * 32; t0 < g.n_tokens; t0 += gridDim.x * kThreads) {
      bool good = (a.n_seqs <= 32 ? few_tiles : work.n_tiles) > 0;
      for (int b = lane; b < a.n_seqs; b += 32) good = good && good_starts(a, __ldg(a.q_start + b), __ldg(a.q_start + b + 1));
      good = __all_sync(0xffffffffu, good);
      const int t = t0 + lane;
      if (t >= g.n_tokens) continue;
      bool none = !good || t < __ldg(a.q_start) || t >= __ldg(a.q_start + a.n_seqs);
      if (!good && (a.n_seqs <= 32 || work.n_tiles > 0))
        for (int b = 0; none && b < a.n_seqs; ++b) {
          int s0, n, kv;
          lengths(a, b, s0, n, kv);
          none = t < s0 || t >= s0 + n;
        }
      if (none) a.token_parts[t] = PagedToken{0, 0, 0, 0};
    }
  if (!is_short) {
    fence_proxy_async_smem();    // the ring's copies come after what was written there
    __syncthreads();
  }

  // The next piece of work; false: there is none, or a wait has run out.
  uint32_t n_taken = 0;
  auto take_piece = [&](Piece& p) {
    const int i = n_taken & 1;
    if (!__all_sync(0xffffffffu, mbar_wait_far(&ctl, piece_full(i), (n_taken >> 1) & 1u, 0x800u))) return false;
    p = tail.piece[i];
    __syncwarp();
    if (lane == 0) mbar_arrive(piece_empty(i));
    ++n_taken;
    return p.n_steps != 0;
  };
  auto step_row = [](const Piece& p, int j) { return (p.step0 + j < p.near_tiles ? p.step0 + j : p.step0 + j + p.skip) * kTileKeys; };
  // whether a tile of keys has rows that none of the tokens sees
  auto unseen_rows = [&](const Piece& p, int row0) {
    return row0 + kTileKeys > p.kv_end || (row0 < p.win_lo && row0 + kTileKeys > g.n_sink);
  };

  if (warp == kProducerWarp) {
    // ------------------------------------------------------------ the pieces of work, and their K and V: a copy per page box and half of
    // the columns
    if (lane == 0) { tma_prefetch_desc(&k_map); tma_prefetch_desc(&v_map); }
    const int copies = 2 * (kTileKeys >> a.lg_box);
    const uint32_t box_bytes = (uint32_t)a.box_rows * kLineBytes;
    const int box = lane >> 1, half = lane & 1;
    int slot = 0;
    uint32_t ph = 1;                         // parity of a slot's emptiness
    const Heavy* const heavy = a.heavy + (size_t)blockIdx.x * kMaxHeavy;
    const long long heavy_work = (long long)work.n_heavy_pieces * g.Hkv, total = heavy_work + (long long)work.n_tiles * g.Hkv;
    long long w = blockIdx.x;
    int at_heavy = 0;
    int strip = -32, strip_first = 0, strip_all = 0, incl = 0, nt = 0, s0 = 0, n = 0, kv = 0;   // 32 sequences, one a lane
    uint32_t n_given = 0;
    bool ok = true;
    while (ok) {
      const bool more = w < total;
      Piece p;
      p.n_steps = 0;
      long long next = 0;
      if (more) {
        if (lane == 0) next = (long long)atomicAdd(a.sched, 1u) + gridDim.x;
        if (w < heavy_work) {
          const int piece = (int)(w / g.Hkv);
          p.head = (int)(w - (long long)piece * g.Hkv);
          Heavy x;
          for (; at_heavy < kMaxHeavy; ++at_heavy) {
            const int4* src = reinterpret_cast<const int4*>(heavy + at_heavy);
            *reinterpret_cast<int4*>(&x) = __ldcg(src);
            *(reinterpret_cast<int4*>(&x) + 1) = __ldcg(src + 1);
            if (piece < x.first_piece + x.n_chunks) break;
          }
          int b0, bn, bkv;
          lengths(a, x.seq, b0, bn, bkv);
          const int h = p.head;
          tile_piece(a, x.seq, b0, bn, bkv, x.t, p);
          p.head = h;
          const int c = piece - x.first_piece, rows = p.n_tok * g.G;
          p.step0 = c * x.chunk_steps;
          p.n_steps = min(x.chunk_steps, p.n_steps - p.step0);
          if (x.n_chunks > 1) {
            p.n_chunks = x.n_chunks;
            p.chunk_steps = x.chunk_steps;
            p.part_step = g.Hkv * rows;
            p.part_row = x.part_row + c * p.part_step + h * rows;
            p.counter = x.counter + 2 * h;
          }
        } else {
          const int e = (int)((w - heavy_work) / g.Hkv);
          p.head = (int)(w - heavy_work - (long long)e * g.Hkv);
          while (e >= strip_first + strip_all) {
            strip += 32;
            strip_first += strip_all;
            nt = 0;
            if (strip + lane < a.n_seqs) {
              lengths(a, strip + lane, s0, n, kv);
              nt = (n + size - 1) / size;
            }
            incl = nt;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
              const int v = __shfl_up_sync(0xffffffffu, incl, o);
              if (lane >= o) incl += v;
            }
            strip_all = __shfl_sync(0xffffffffu, incl, 31);
          }
          const int own = __popc(__ballot_sync(0xffffffffu, strip_first + incl <= e));
          const int h = p.head, t = e - strip_first - __shfl_sync(0xffffffffu, incl - nt, own);
          tile_piece(a, strip + own, __shfl_sync(0xffffffffu, s0, own), __shfl_sync(0xffffffffu, n, own), __shfl_sync(0xffffffffu, kv, own), t, p);
          p.head = h;
          if (is_heavy(p.n_steps, work.all_steps)) {     // it was among those
            w = __shfl_sync(0xffffffffu, next, 0);
            continue;
          }
        }
        if (a.partial) {
          const bool whole = p.n_chunks == 1;
          if (p.head == 0 && p.step0 == 0)
            for (int i = lane; i < p.n_tok; i += 32)
              a.token_parts[p.tok0 + i] = whole ? PagedToken{(p.tok0 + i) * g.Hq, 1, 0, g.G}
                                                : PagedToken{p.part_row + i * g.G, p.n_chunks, p.part_step, p.n_tok * g.G};
        }
      }
      const int i = n_given & 1;
      if (!__all_sync(0xffffffffu, mbar_wait_far(&ctl, piece_empty(i), ((n_given >> 1) & 1u) ^ 1u, 0x900u))) break;
      if (lane == 0) {
        tail.piece[i] = p;
        mbar_arrive(piece_full(i));
      }
      __syncwarp();
      ++n_given;
      if (!more) {
        // the last CTA that finds nothing leaves the counter ready for the next launch
        if (lane == 0 && atomicAdd(a.sched + 1, 1u) == gridDim.x - 1) { a.sched[0] = 0u; a.sched[1] = 0u; }
        break;
      }
      w = __shfl_sync(0xffffffffu, next, 0);
      const Piece& it = p;
      const int h = it.head;
      const int* table = a.block_table + (size_t)it.seq * g.max_pages;
      int ids = 0, ids_at = -1;
      for (int j = 0; ok && j < it.n_steps; ++j) {
        const int row0 = step_row(it, j);
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
  } else if (warp == kStewardWarp) {
    // ------------------------------------------------------------ steward: the query blocks, unseen rows of V, and all that the warp which
    // issues the MMAs would otherwise wait for or report: it shares its scheduler with busy warps, and each of those waits and commits
    // cost it 100 cycles and more, during which the tensor cores ran dry (3600 cycles a step with all of them).
    // For step j it answers for V(j) and K(j+1) having landed by being one of those that hand over P.  It waits for nothing that could
    // go on without it, so that no phase of a barrier can pass it by: a tile of the ring is given back (by the softmax of the last
    // stream, which is told of S(j) when K(j) and V(j-1) have been read) only after a product that needed its answer.
    if (lane == 0) tma_prefetch_desc(&q_map);
    uint32_t rph = 0, pph = 3u;              // parities: of the ring; a bit for each stream
    int slot = 0;                            // of the next tile to land
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity, unsigned code) {
      ok = ok && __all_sync(0xffffffffu, mbar_wait_far(&ctl, bar, parity, code));
    };
    auto advance = [&]() { if (++slot == kSlots) { slot = 0; rph ^= 1u; } };
    auto load_q = [&](const Piece& p) {
      if (lane == 0)
        for (int s = 0; s < 2 && s * R < p.n_tok; ++s) {
          mbar_arrive_expect_tx(q_full(s), 2u * (uint32_t)(R * g.G) * kLineBytes);
          for (int half = 0; half < 2; ++half)
            tma_load_4d(q_base + s * kTileBytes + half * (kTileBytes / 2), &q_map, q_full(s), half * kHalfCols, 0, p.head, p.tok0 + s * R);
        }
      __syncwarp();
    };
    Piece it;
    while (ok && take_piece(it)) {
      load_q(it);                            // (all products with the queries of the piece before are done: see below)
      const int n = it.n_steps, last = it.n_tok > R ? 1 : 0;
      advance();                             // K(0): the issuing warp waits for it itself
      for (int j = 0; ok && j < n; ++j) {
        const int vs = slot;
        wait(full(vs), rph, 0x280u);
        advance();
        const int row0 = step_row(it, j);
        if (ok && unseen_rows(it, row0)) {
          // Rows of V that none of the tokens sees may hold anything (or have not been loaded), and zero times that could be a NaN: they
          // become zeros before the product.
          unsigned char* const mine = smem_al + (2 + vs) * kTileBytes + ((lane >> 3) & 1) * (kTileBytes / 2) + (lane & 7) * 16;
          auto clear = [&](int r0, int r1) {
#pragma unroll 4
            for (int r = max(r0, 0) + (lane >> 4); r < min(r1, kTileKeys); r += 2)
              *reinterpret_cast<uint4*>(mine + r * kLineBytes) = make_uint4(0u, 0u, 0u, 0u);
          };
          clear(it.kv_end - row0, kTileKeys);
          clear(g.n_sink - row0, min(it.win_lo, it.kv_end) - row0);
        }
        if (j + 1 < n) {
          wait(full(slot), rph, 0x290u);
          advance();
        }
        fence_proxy_async_smem();
        __syncwarp();
        for (int s = 0; s <= last; ++s) {
          wait(p_full(s, 0), (pph >> s) & 1u, 0x220u);      // (that of the step before, so that this arrival counts for its own)
          if (ok && lane == 0) mbar_arrive(p_full(s, 0));
          pph ^= 1u << s;
        }
      }
      // the last stream hands over the P of the last step when its S, and so all S, are done: the queries may be replaced
      wait(p_full(last, 0), (pph >> last) & 1u, 0x230u);
    }
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------ all MMAs, the warp as a whole with one lane issuing.  The streams take
    // turns, which also keeps one half a step behind the other (with a warp each they fell into step, both at their softmax and then both
    // waiting for the tensor cores: 4000 cycles a step instead of 2970).
    constexpr uint32_t kTypes = kF16 ? ~((7u << 7) | (7u << 10)) : ~0u;    // f16 operands are type 0
    const uint32_t idesc_s = umma_idesc(128, 128, false, false) & kTypes;   // A = Q, B = K tile, both K-major
    const uint32_t idesc_o = umma_idesc(128, 128, false, true) & kTypes;    // A = P (tensor memory), B = V tile, MN-major
    const uint64_t dq = smem_desc_sw128(q_base, 16u, 1024u);
    const uint64_t dk = smem_desc_sw128(ring, 16u, 1024u);
    const uint64_t dv = smem_desc_sw128(ring, kTileBytes / 2, 1024u);
    const bool leader = elect_one();
    int slot = 0;
    uint32_t ph = 0, qph = 0, pph = 0;       // parities: of the ring; a bit for each stream
    auto advance = [&]() { if (++slot == kSlots) { slot = 0; ph ^= 1u; } };
    auto wait = [&](uint32_t bar, uint32_t parity, unsigned code) {
      const bool ok = __any_sync(0xffffffffu, mbar_try_wait(bar, parity)) || __all_sync(0xffffffffu, mbar_wait_poll_far(&ctl, bar, parity, code));
      tc_fence_after_sync();
      return ok;
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
    // P V of 16 keys of each half of the tile: steps kk and kk + 4; the P of keys 64.. sits at columns 64..
    auto pv = [&](int s, uint64_t vd, int kk, uint32_t acc) {
      const uint32_t p = tmem_base + (uint32_t)(s * 128 + kk * 8), d = tmem_base + (uint32_t)(s * 128) + kColO;
      umma_ts(d, p, desc_advance(vd, (uint32_t)kk * 16u * kLineBytes), idesc_o, acc);
      umma_ts_imm<1>(d, p + 64u, desc_advance(vd, (uint32_t)(kk + 4) * 16u * kLineBytes), idesc_o);
    };
    Piece it;
    while (take_piece(it)) {
      const int n = it.n_steps, n_streams = it.n_tok > R ? 2 : 1;
      if (!wait(full(slot), ph, 0x300u)) break;
      bool ok = true;
      for (int s = 0; ok && s < n_streams; ++s) {
        ok = wait(q_full(s), (qph >> s) & 1u, 0x400u);
        qph ^= 1u << s;
        if (ok) issue_s(s, slot);
      }
      advance();
      for (int j = 0; ok && j < n; ++j) {
        const uint64_t vd = desc_advance(dv, (uint32_t)slot * kTileBytes);
        advance();
        const bool more = j + 1 < n;
        for (int s = 0; s < n_streams; ++s) {
          const uint32_t parity = (pph >> s) & 1u;
          if (!(ok = wait(p_full(s, 0), parity, 0x500u))) break;
          if (leader) {
            pv(s, vd, 0, j ? 1u : 0u);
            pv(s, vd, 1, 1u);
            pv(s, vd, 2, 1u);
          }
          __syncwarp();
          if (!(ok = wait(p_full(s, 1), parity, 0x510u))) break;
          if (leader) {
            pv(s, vd, 3, 1u);
            if (!more) umma_commit(o_full(s));
          }
          __syncwarp();
          if (more) issue_s(s, slot);
          pph ^= 1u << s;
        }
        if (more) advance();
      }
      if (!ok) break;
    }
  } else if (warp < kSoftmaxWarps) {
    // ------------------------------------------------------------ softmax: two threads to a row
    // O is rescaled when a row's maximum has grown by more than 2^kLazy over its reference.  In bf16 the terms are kept 2^-8 lower than
    // they are, so that one that has grown is 1 at most and the sums of P V have the range that they have with the maximum itself
    // (with a growth of 2^40 let pass, values of V beyond 2^87 became infinite); a factor costs no bits.  In fp16 terms have to stay
    // below 2^16 (and are kept 2^kBias higher than they are, see pack16).
    constexpr float kLazy = 8.f, kBias = kF16 ? 7.f : -kLazy;
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
    auto any_of_stream = [&](bool x) {
      uint32_t r;
      asm volatile(
          "{\n"
          ".reg .pred p, q;\n"
          "setp.ne.u32 p, %1, 0;\n"
          "barrier.cta.red.or.pred q, %2, 256, p;\n"
          "selp.u32 %0, 1, 0, q;\n"
          "}\n"
          : "=r"(r) : "r"((uint32_t)x), "r"(1 + s) : "memory");
      return r != 0;
    };
    auto max_of = [](const uint32_t (&x)[32]) {
      float m[2] = {__uint_as_float(x[0]), __uint_as_float(x[1])};
#pragma unroll
      for (int c = 2; c < 30; c += 4) {
        m[0] = max3(m[0], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
        m[1] = max3(m[1], __uint_as_float(x[c + 2]), __uint_as_float(x[c + 3]));
      }
      return max3(fmaxf(m[0], m[1]), __uint_as_float(x[30]), __uint_as_float(x[31]));
    };
    uint32_t sph = 0, oph = 0;
    int ring_at = 0;
    // The warps of a stream meet at barriers, so they leave the loop together, and a wait that runs out (after which all others
    // of the CTA return at once) takes none of them out of a piece.
    for (;;) {
      const int slot = n_taken & 1;
      const bool there = mbar_wait_far(&ctl, piece_full(slot), (n_taken >> 1) & 1u, 0x800u);
      const Piece& it = tail.piece[slot];              // read where it lies, and given back at the end
      const int n_steps = there ? it.n_steps : 0;
      if (any_of_stream(n_steps == 0)) break;
      ++n_taken;
      auto give_back = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(piece_empty(slot));
      };
      int ks = ring_at;                                // ring slot of K(j); V(j - 1) lies ahead of it
      ring_at = (ring_at + 2 * n_steps) % kSlots;
      if (s * R >= it.n_tok) { give_back(); continue; }
      const bool releases = (tid & 255) == 0 && (s + 1) * R >= it.n_tok;     // a thread of the last stream
      auto release = [&](int sl) { mbar_arrive(empty(sl < 0 ? sl + kSlots : sl)); };
      const int pos = it.pos0 + i_tok;
      const int tok_last = min(it.n_tok, (s + 1) * R) - 1;
      // the keys from clear_lo (or from the first, as far as the sinks go) up to clear_hi are seen by all rows of the stream
      const int clear_hi = min(it.kv_end, it.pos0 + s * R + 1);
      const int clear_lo = g.window ? it.pos0 + tok_last - g.window + 1 : 0;
      float ref = -INFINITY, l = 0.f;       // reference of the row's terms (log2 domain), the sum of this thread's
#pragma unroll 1
      for (int j = 0; j < n_steps; ++j) {
        const int row0 = step_row(it, j);
        mbar_wait(&ctl, s_full(s), sph, 0x600u);
        __syncwarp();
        sph ^= 1u;
        tc_fence_after_sync();
        if (releases) {                                  // S(j) is done, and with it all MMAs issued before
          release(ks);
          if (j > 0) release(ks - 1);
        }
        ks = ks + 2 >= kSlots ? ks + 2 - kSlots : ks + 2;
        if (row0 + kTileKeys > clear_hi || (row0 < clear_lo && row0 + kTileKeys > g.n_sink)) {
          // keys that the row does not see become -inf where they lie, 16 columns at a time: in the registers, all unrolled, it was
          // code of 4 KB that few tiles need, and took 1500 cycles of each
          const int key0 = row0 + half * 64, hi = min(it.kv_end, pos + 1), lo = pos - g.window + 1;
          auto below = [](int n) { return n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << n) - 1u; };   // the n lowest bits
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            const int k0 = key0 + 16 * q;
            uint32_t seen = below(hi - k0);
            if (g.window) seen &= ~below(lo - k0) | below(g.n_sink - k0);
            if (__all_sync(0xffffffffu, seen == 0xffffu)) continue;
            uint32_t y[16];
            tmem_ld16(s_addr + 16 * q, y);
#pragma unroll
            for (int c = 0; c < 16; ++c)
              if (!(seen & (1u << c))) y[c] = 0xff800000u;
            tmem_st16(s_addr + 16 * q, y);
          }
          tmem_st_wait();
        }
        // (The upper 32 keys are read twice, first for their maximum alone: with 64 logits held, a thread's 96 registers leave no room
        // for more than a few exponentials at a time, and these took 700 cycles instead of the unit's 420 for 32 keys.)
        uint32_t x[32], packed[16];
        tmem_ld32(s_addr + 32, x);
        float top = max_of(x);
        tmem_ld32(s_addr, x);
        top = fmaxf(top, max_of(x));
        if (any_of_stream(top * g.scale2 - kBias > ref + kLazy)) {       // (from -inf on the first key that is seen)
          *my_max = top;
          meet();
          const float t = fmaxf(top, *other_max) * g.scale2 - kBias;
          const bool grow = t > ref + kLazy;
          const float f = grow ? ex2_approx(ref - t) : 1.f;
          const bool had = __any_sync(0xffffffffu, grow && ref > -INFINITY);
          if (grow) { l *= f; ref = t; }
          if (had && j > 0) {                            // this half of O's columns
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              tmem_ld16(o_addr + 16 * q, packed);
#pragma unroll
              for (int c = 0; c < 16; ++c) packed[c] = __float_as_uint(__uint_as_float(packed[c]) * f);
              tmem_st16(o_addr + 16 * q, packed);
            }
          }
        }
        f32x2 sum = 0ull;
        terms<kF16, 0, 32>(x, sc, ref, packed, sum);
        tmem_st16(s_addr, packed);
        tmem_ld32(s_addr + 32, x);
        terms<kF16, 0, 16>(x, sc, ref, packed, sum);
        tmem_st8(s_addr + 16, packed);
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(p_full(s, 0));
        terms<kF16, 16, 32>(x, sc, ref, packed, sum);
        tmem_st8(s_addr + 24, packed);
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(p_full(s, 1));
        const float2 t = unpack2(sum);
        l += t.x + t.y;
      }
      mbar_wait(&ctl, o_full(s), oph, 0x700u);
      __syncwarp();
      if (releases) release(ks - 1);                     // V of the last step
      oph ^= 1u;
      tc_fence_after_sync();
      // the row's sum, of the lower keys and the upper ones in this order
      *my_max = l;
      meet();
      const float l_other = *other_max;
      l = half ? l_other + l : l + l_other;
      meet();                                            // (the next item writes there)
      // O comes out of tensor memory with a row in a quad of lanes, eight columns of each of its groups of 32 bits, and is stored as
      // it comes (partial rows) or after the lanes of a quad have traded for 16 bytes in a row: a store of a warp then touches eight
      // rows.  (With a thread to a row each touched 32, and an item's end took 8000 cycles.)
      const float inv = l == 0.f ? 0.f : 1.f / l;        // no key seen: zeros
      const bool cut = it.n_chunks > 1, final = !a.partial && !cut;
      const int n_tok = it.n_tok;
      const size_t head_row = (size_t)it.tok0 * g.Hq + it.head * g.G;     // output row of the first token and the group's first head
      const size_t part_at = cut ? (size_t)it.part_row : head_row;         // and its partial row
      const int tok_step = cut ? g.G : g.Hq;                               // (of partial rows, from a token to the next)
#pragma unroll 1
      for (int e = 0; e < 2; ++e) {                      // 16 rows each
        uint32_t o[32];
        tmem_ld_16x64(o_addr + ((uint32_t)(16 * e) << 16), o);
#pragma unroll
        for (int u = 0; u < 2; ++u) {                    // the upper and the lower eight of them
          const int in_warp = 16 * e + 8 * u + (lane >> 2);
          const int row = (warp & 3) * 32 + in_warp;
          const int i = s * R + (row * a.g_inv >> 16), hd = row - (row * a.g_inv >> 16) * g.G;
          const bool valid = row < R * g.G && i < n_tok;
          if (final) {
            const float f = __shfl_sync(0xffffffffu, inv, in_warp);
            uint4* const dst = reinterpret_cast<uint4*>(a.out) + (head_row + (uint32_t)(i * g.Hq + hd)) * (kD / 8) + half * 8 + (lane & 3);
#pragma unroll
            for (int b = 0; b < 2; ++b) {                // 32 columns each
              uint32_t v[4];
#pragma unroll
              for (int c = 0; c < 4; ++c)
                v[c] = pack16<kF16>(__uint_as_float(o[16 * b + 4 * c + 2 * u]) * f, __uint_as_float(o[16 * b + 4 * c + 2 * u + 1]) * f);
              const uint4 t = quad_transpose(v, lane);
              if (valid) dst[4 * b] = t;
            }
          } else {
            const size_t to = part_at + (uint32_t)(i * tok_step + hd);
            float* const dst = a.parts + to * kPagedPartStride + half * 64 + 2 * (lane & 3);
            if (valid && (long long)to < a.max_rows) {
#pragma unroll
              for (int c = 0; c < 8; ++c)
                __stcg(reinterpret_cast<float2*>(dst + 8 * c), make_float2(__uint_as_float(o[4 * c + 2 * u]), __uint_as_float(o[4 * c + 2 * u + 1])));
            }
          }
        }
      }
      if (in_block && i_tok < n_tok && half == 0) {
        if (final) {
          if (a.lse) a.lse[head_row + (uint32_t)(i_tok * g.Hq + head)] = l == 0.f ? -INFINITY : (ref + __log2f(l)) * kLn2;
        } else {
          const size_t to = part_at + (uint32_t)(i_tok * tok_step + head);
          if ((long long)to < a.max_rows) __stcg(reinterpret_cast<float2*>(a.parts + to * kPagedPartStride + kD), make_float2(ref, l));
        }
      }
      if (final || a.partial) { give_back(); continue; }
      // the last of the tile's chunks to arrive joins them all
      __threadfence();
      meet();
      if ((tid & 255) == 0) {
        unsigned* const count = a.sched + 16 + it.counter + s;
        const bool last = atomicAdd(count, 1u) == (unsigned)(it.n_chunks - 1);
        if (last) *count = 0u;                           // ready for the next launch
        __threadfence();
        tail.last[s] = last;
      }
      meet();
      if (*reinterpret_cast<volatile int*>(&tail.last[s])) {
        const int n_rows = min(R, n_tok - s * R) * g.G, n_chunks = it.n_chunks, step = it.part_step;
        const size_t first_row = part_at - (size_t)(it.step0 / it.chunk_steps) * step + s * R * g.G;
        // four rows of a warp at a time: first their chunks' weights, a lane to a row and chunk, then the sums, whose loads wait for nothing
        for (int r0 = (warp & 7) * 4; r0 < n_rows; r0 += 32) {
          const float* const src = a.parts + (first_row + r0) * kPagedPartStride;
          const size_t chunk_at = (size_t)step * kPagedPartStride;
          const int my_row = lane >> 3;
          const bool there = r0 + my_row < n_rows;
          float top = -INFINITY, sum = 0.f;
          for (int c0 = 0; c0 < n_chunks; c0 += 8) {
            const int c = c0 + (lane & 7);
            const float2 ml = there && c < n_chunks ? __ldcg(reinterpret_cast<const float2*>(src + c * chunk_at + my_row * kPagedPartStride + kD))
                                                    : make_float2(-INFINITY, 0.f);
            float m = ml.x;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            m = fmaxf(m, top);
            const float at = m == -INFINITY ? 0.f : m;
            float l_sum = ml.y * ex2_approx(ml.x - at);
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) l_sum += __shfl_xor_sync(0xffffffffu, l_sum, o);
            sum = sum * ex2_approx(top - at) + l_sum;
            top = m;
          }
          const float at = top == -INFINITY ? 0.f : top, f_row = sum == 0.f ? 0.f : 1.f / sum;
          float4 acc[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int c0 = 0; c0 < n_chunks; c0 += 8) {
            const int c = c0 + (lane & 7);
            const float m = there && c < n_chunks ? __ldcg(src + c * chunk_at + my_row * kPagedPartStride + kD) : -INFINITY;
            const float weight = ex2_approx(m - at) * f_row;
            const int n_c = min(8, n_chunks - c0);
#pragma unroll 4
            for (int i = 0; i < n_c; ++i) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float w = __shfl_sync(0xffffffffu, weight, k * 8 + i);
                const float* x = src + (c0 + i) * chunk_at + (r0 + k < n_rows ? k : 0) * kPagedPartStride;
                const float4 o = __ldcg(reinterpret_cast<const float4*>(x) + lane);
                acc[k].x = fmaf(o.x, w, acc[k].x); acc[k].y = fmaf(o.y, w, acc[k].y);
                acc[k].z = fmaf(o.z, w, acc[k].z); acc[k].w = fmaf(o.w, w, acc[k].w);
              }
            }
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int row = r0 + k;
            const float lse = __shfl_sync(0xffffffffu, sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2, k * 8);
            if (row >= n_rows) continue;
            const int i = s * R + (row * a.g_inv >> 16), hd = row - (row * a.g_inv >> 16) * g.G;
            const size_t out_row = head_row + (uint32_t)(i * g.Hq + hd);
            reinterpret_cast<uint2*>(a.out)[out_row * (kD / 4) + lane] =
                make_uint2(pack16<kF16>(acc[k].x, acc[k].y), pack16<kF16>(acc[k].z, acc[k].w));
            if (a.lse && lane == 0) a.lse[out_row] = lse;
          }
        }
      }
      give_back();
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (paged_aborted(ctl)) {      // copies and MMAs may still be under way, and need this CTA's memory for a few microseconds
    const long long t0 = clock64();
    while (clock64() - t0 < 400000) {}
  }
  pdl_trigger();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
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
  KernelArgs a{};
  a.g = d.g;
  a.block_table = d.block_table; a.q_start = d.q_start; a.kv_len = d.kv_len;
  a.n_seqs = d.n_seqs; a.causal = d.causal; a.partial = d.partial;
  a.tokens = 128 / d.g.G;
  a.g_inv = 65536 / d.g.G + 1;
  a.box_rows = std::min(d.g.page, kTileKeys);
  while ((1 << a.lg_box) < a.box_rows) ++a.lg_box;
  a.sched = (unsigned*)(d.wsp + ws.sched);
  a.heavy = (Heavy*)(d.wsp + ws.heavy);
  a.token_parts = (PagedToken*)(d.wsp + ws.tokens);
  a.parts = (float*)(d.wsp + ws.part_o);
  a.max_rows = ws.max_rows;
  a.out = d.out; a.lse = d.lse;
  CUtensorMap qm, km, vm;
  if (!paged_q_map(&qm, d.q, d.g, a.tokens) || !paged_kv_map(&km, d.K, d.g, a.box_rows, 0) || !paged_kv_map(&vm, d.V, d.g, a.box_rows, 0))
    return cudaErrorInvalidValue;
  e = launch_pdl(paged_attention_kernel<kF16>, dim3(kSms), dim3(kThreads), kSmemBytes, st, qm, km, vm, a);
  if (e == cudaSuccess) count_launch(1);
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
  const int G = Hq / Hkv;
  // chunks of cut tiles are no more than the SMs; with a shared prefix every token has rows of its own in any case
  w.max_rows = (long long)kSms * std::min((long long)kPagedRows, (long long)n_tokens * G) + (n_groups ? (long long)n_tokens * Hq : 0);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t off = kPagedPlan;
  w.sched = off;  off = up(off + (16 + 2 * kSms) * 4);
  w.heavy = off;  off = up(off + (size_t)kSms * kMaxHeavy * sizeof(Heavy));
  w.tokens = off; off = up(off + (size_t)(n_groups ? B : 0) * sizeof(PagedToken));
  w.part_o = off; off = up(off + (size_t)w.max_rows * kPagedPartStride * 4);
  w.total = off;
  return w;
}

cudaError_t launch_paged_attention(const PagedAttnArgs& a, const PagedWs& ws, cudaStream_t st) {
  return a.g.f16 ? launch<true>(a, ws, st) : launch<false>(a, ws, st);
}

}  // namespace calidrop
