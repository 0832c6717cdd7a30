// Attention of one new token a sequence over a cache in pages, with a sliding window and sinks, and optionally joined
// with the attention over a prefix that the sequence shares with others.
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp2(scale2 q.k_t - m),  t over the visible rows;  lse = (m + log2 sum p) ln 2
//
// Bound by memory: every visible row of K and V is read once for the G heads of its group, about 2G operations a byte.
// The lengths are on the device and may be anything, so the work is dealt there: all visible rows of all (sequence, kv
// head) units, in blocks of 64 rows, form one line that is cut into equal parts, one per CTA.  Every CTA sums the lengths itself
// (a launch ahead of this one would cost more than the sum).  A unit that lies in one part is finished there; of a unit
// that is cut each CTA leaves its partial (outputs, maximum, sum), and the last of them to arrive joins these, in the order of
// the parts, so that the result does not depend on who is last.
//
// A CTA is a producer warp and four stream warps: K and V come through a ring of three slots of 64 rows by TMA, a copy per page and
// slot, and a slot is consumed by the four warps, 16 rows each, with mma.sync, keys on the 16-row side (as in decode.cu).  The
// producer runs ahead over the borders of units, so that the memory does not wait for a unit's end, and two CTAs share an SM, so that
// one streams while the other ends a unit.  (One CTA of eight stream warps and six slots: 768 units of 24 to 600 rows, joined with
// a shared prefix, 87 us, now 40.)  32 caches of 600 to 16000 rows, 0.9 GB: 140 us, 98 % of the copy bandwidth; 48 with a window of 4064 rows, 0.66 GB:
// 108 us, 94 %; one cache of 512 visible rows: 8 us, a chain of lengths, table, rows, partials, ticket and join.
#include <algorithm>

#include "paged_common.cuh"

namespace calidrop {

bool paged_kv_map(CUtensorMap* out, const void* base, const PagedGeom& g, int rows, int halves);

namespace {

constexpr int kSlots = 3, kSlotRows = 64, kLgRows = 6;
constexpr int kStreamWarps = 4, kThreads = (kStreamWarps + 1) * 32;
constexpr int kCtas = 2 * kSms;                        // two to an SM
constexpr int kPartBytes = kSlotRows * kRowBytes;      // K or V of a slot: 16 KB
constexpr int kSlotBytes = 2 * kPartBytes;
constexpr int kStride = kPagedPartStride;              // floats of a warp's partial row: heads land in distinct banks
// What a unit costs beside its rows, in blocks.  With 1, 2, 3: 768 short units and their prefix 78, 73, 73 us, 64 of them 27.5, 26.0, 27.7, 256 long units
// 140, 141, 140.
constexpr int kUnitCost = 2;
constexpr int kMinShare = 2;                           // of a CTA's part of the line, which may hold nothing but the places of a unit that have no rows
// What is in shared memory behind the ring.
struct Tail {
  float part[kStreamWarps][kMaxG][kStride];            // of the warps, at the end of a unit
  unsigned long long full[kSlots], empty[kSlots];
  long long scan[kStreamWarps + 1], unit0;             // unit0: where the first unit of this CTA begins on the line
  int b, h, abort, last;
};
constexpr int kSmemBytes = kSlots * kSlotBytes + sizeof(Tail);
static_assert(2 * (kSmemBytes + 1024) <= 228 * 1024, "two CTAs to an SM (and no static shared memory: the ring begins at a multiple of 1024)");
static_assert(kCtas <= kPagedMaxCtas, "");
constexpr long long kWaitLimitCycles = 2000000000ll;   // about a second: a wait this long has failed

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// A wait that runs out raises the CTA's flag and the workspace's error word; all later waits return at once and the CTA
// walks to its end, with undefined results.
__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned* status) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  long long t0 = 0;
  unsigned polls = 0;
  while (!tc::mbar_try_wait(bar, parity)) {
    if ((++polls & 255u) == 0u) {
      if (*abort_flag) return false;
      const long long now = clock64();
      if (t0 == 0) t0 = now;
      if (now - t0 > kWaitLimitCycles) {
        *abort_flag = 1;
        atomicOr(status, 0x100u);
        return false;
      }
    }
  }
  return true;
}

struct KernelArgs {
  PagedGeom g;
  const void* q;
  const int *block_table, *kv_len;
  void* out;
  float* lse;
  unsigned* counters;
  float* parts;                // [CTA][2][8][kStride]
  const PagedToken* tokens;     // partial rows of the shared prefix, per sequence; null: none
  const float* prefix_rows;
  long long max_rows;
  int box_rows, lg_box;
};

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 2)
paged_decode_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const KernelArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Tail& tail = *reinterpret_cast<Tail*>(smem + kSlots * kSlotBytes);

  const PagedGeom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t ring = smem_u32(smem);
  volatile int* abort_flag = &tail.abort;
  auto full = [&](int s) { return smem_u32(&tail.full[s]); };
  auto empty = [&](int s) { return smem_u32(&tail.empty[s]); };

  pdl_trigger();
  if (tid == 0) {
    for (int s = 0; s < kSlots; ++s) {
      tc::mbar_init(full(s), 1);
      tc::mbar_init(empty(s), kStreamWarps);
    }
    tc::fence_mbar_init();
    tail.abort = 0;
  }
  if (tid == kStreamWarps * 32) {
    tc::tma_prefetch_desc(&k_map);
    tc::tma_prefetch_desc(&v_map);
  }
  pdl_wait();

  const int cap = g.max_pages << g.lg_page;
  auto view = [&](int kv) { return paged_view<kLgRows>(min(max(kv, 0), cap), g.window, g.n_sink); };
  auto length_of = [&](int b) { return b < g.B ? __ldg(a.kv_len + b) : 0; };

  // ---- the line: its length, and the unit at this CTA's start.  A unit's blocks come behind kUnitCost places without rows.
  long long total = 0;
  auto scan = [&](int base, long long& incl, int& places) {   // inclusive sums over the sequences base + tid; their sum
    const int b = base + tid;
    places = 0;
    if (b < g.B) {
      const int kv = length_of(b);
      if ((kv < 0 || kv > cap) && blockIdx.x == 0) paged_flag(g.status, kBadLength);
      places = view(kv).n_blocks + kUnitCost;
    }
    incl = places;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) tail.scan[warp] = incl;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w <= kStreamWarps; ++w) {
      const long long v = tail.scan[w];
      if (w < warp) incl += v;
      all += v;
    }
    return all;
  };
  long long incl = 0;
  int places = 0;
  for (int base = 0; base < g.B; base += kThreads) total += scan(base, incl, places);
  const long long line = total * g.Hkv;
  const long long share = max((line + gridDim.x - 1) / gridDim.x, (long long)kMinShare);
  const long long begin = blockIdx.x * share, end = min(line, begin + share);
  if (begin >= line) return;
  long long before = 0;
  for (int base = 0; base < g.B; base += kThreads) {
    const long long all = g.B > kThreads ? scan(base, incl, places) : total;
    const long long u0 = (before + incl - places) * g.Hkv;
    if (places && begin >= u0 && begin < u0 + (long long)places * g.Hkv) {
      const long long h = (begin - u0) / places;
      tail.b = base + tid;
      tail.h = (int)h;
      tail.unit0 = u0 + h * places;
    }
    before += all;
  }
  __syncthreads();
  int b = tail.b, h = tail.h;
  long long unit0 = tail.unit0;
  PagedView v = view(length_of(b));
  int kv_next = length_of(b + 1);
  // The unit's blocks [blk, blk + n) lie in this CTA's part.
  auto segment = [&](int& blk) {
    const long long first = unit0 + kUnitCost, lo = max(begin, first);
    blk = (int)(lo - first);
    return (int)max(0ll, min(end, first + v.n_blocks) - lo);
  };
  auto next_unit = [&]() {
    unit0 += v.n_blocks + kUnitCost;
    if (++h == g.Hkv) {
      h = 0;
      ++b;
      v = view(kv_next);
      kv_next = length_of(b + 1);
    }
    return unit0 < end;
  };

  if (warp == kStreamWarps) {
    // ---------------------------------------------------------------- producer
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    const int boxes = kSlotRows >> a.lg_box;               // copies of a slot's K
    const uint32_t box_bytes = (uint32_t)a.box_rows * kRowBytes;
    int ids = 0, ids_at = -1, ids_b = -1;                   // lane i holds the page of rows (ids_at + i) * page.. of sequence ids_b
    int slot = 0;
    uint32_t ph = 1;
    bool ok = true;
    do {
      int blk;
      const int n = segment(blk);
      for (int i = 0; ok && i < n; ++i) {
        const int row0 = v.block(blk + i) << kLgRows;
        const int pg = row0 >> g.lg_page, pg_last = (row0 + kSlotRows - 1) >> g.lg_page;
        if (ids_b != b || pg < ids_at || pg_last >= ids_at + 32) {
          ids_b = b;
          ids_at = pg;
          ids = pg + lane < g.max_pages ? __ldg(a.block_table + (size_t)b * g.max_pages + pg + lane) : -1;
        }
        const int r = row0 + (lane << a.lg_box);
        const bool need = lane < boxes && r < v.kv && (r + a.box_rows > v.lo || r < g.n_sink);
        int page = __shfl_sync(0xffffffffu, ids, ((r >> g.lg_page) - ids_at) & 31);
        if (need && (page < 0 || page >= g.n_pages)) {
          paged_flag(g.status, kBadPage);
          page = g.n_pages;                                   // outside the pool: the copy brings zeros
        }
        const int n_boxes = __popc(__ballot_sync(0xffffffffu, need));
        ok = __all_sync(0xffffffffu, wait_bounded(empty(slot), ph, abort_flag, g.status));
        if (!ok) break;
        if (lane == 0) tc::mbar_arrive_expect_tx(full(slot), 2u * box_bytes * (uint32_t)n_boxes);
        __syncwarp();
        if (need) {
          const uint32_t dst = ring + slot * kSlotBytes + (uint32_t)lane * box_bytes;
          const int in_page = r & (g.page - 1);
          tma_load_5d(dst, &k_map, full(slot), 0, in_page, h, page, 0, pol);
          tma_load_5d(dst + kPartBytes, &v_map, full(slot), 0, in_page, h, page, 0, pol);
        }
        if (++slot == kSlots) { slot = 0; ph ^= 1u; }
      }
    } while (next_unit());
    if (*abort_flag) {      // a wait has run out: copies may still be under way, and need this CTA's memory for a few microseconds
      const long long t0 = clock64();
      while (clock64() - t0 < 400000) {}
    }
    return;
  }

  // ------------------------------------------------------------------ stream warps
  constexpr float kBias = kF16 ? 12.f : 0.f;   // (see pack16)
  const int gq = lane >> 2, tq = lane & 3;     // MMA fragment coordinates
  const int mid = lane >> 3;
  const uint32_t plane = (uint32_t)a.box_rows * 128u;   // from the first half of a box's columns to the second
  // this warp's 16 rows of a slot
  const uint32_t blk_off = (uint32_t)((warp * 16) >> a.lg_box) * 2u * plane + (uint32_t)((warp * 16) & (a.box_rows - 1)) * 128u;
  auto off = [&](int row, int chunk) { return (uint32_t)(chunk >> 3) * plane + (uint32_t)(row * 128 + (((chunk & 7) ^ (row & 7)) << 4)); };
  auto load_q = [&](int b, int h, uint32_t (&qa)[kD / 16][2]) {
    const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q) + ((size_t)b * g.q_stride + (size_t)(h * g.G + min(gq, g.G - 1)) * kD) / 2 + tq;
#pragma unroll
    for (int kk = 0; kk < kD / 16; ++kk) { qa[kk][0] = __ldg(src + kk * 8); qa[kk][1] = __ldg(src + kk * 8 + 4); }
  };
  auto meet = [&]() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(kStreamWarps * 32) : "memory"); };

  uint32_t q_next[kD / 16][2];     // the next unit's queries are on their way while this one streams
  load_q(b, h, q_next);
  int slot = 0;
  uint32_t ph = 0;
  do {
    int blk;
    const int n_blk = segment(blk);
    uint32_t qa[kD / 16][2];
#pragma unroll
    for (int kk = 0; kk < kD / 16; ++kk) { qa[kk][0] = q_next[kk][0]; qa[kk][1] = q_next[kk][1]; }
    {
      const bool wrap = h + 1 == g.Hkv;
      load_q(min(b + (wrap ? 1 : 0), g.B - 1), wrap ? 0 : h + 1, q_next);
    }
    if (n_blk == 0) continue;
    int4 prefix = make_int4(0, 0, 0, 0);
    if (a.tokens) prefix = __ldg(reinterpret_cast<const int4*>(a.tokens) + b);   // {row, chunks, rows to the next chunk, and to the next head}
    float o[kD / 16][4];
#pragma unroll
    for (int n = 0; n < kD / 16; ++n) { o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f; }
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;   // heads 2tq and 2tq+1

    for (int i = 0; i < n_blk; ++i) {
      const int r0 = (v.block(blk + i) << kLgRows) + warp * 16;
      const bool ok = wait_bounded(full(slot), ph, abort_flag, g.status);
      if (ok && r0 < v.kv && (r0 + 16 > v.lo || r0 < g.n_sink)) {
        const uint32_t sK = ring + slot * kSlotBytes + blk_off, sV = sK + kPartBytes;
        float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};   // two accumulators halve the chain
#pragma unroll
        for (int kk = 0; kk < kD / 16; ++kk) {
          uint32_t a0, a1, a2, a3;
          ldmatrix_x4(sK + off((lane & 7) + (mid & 1) * 8, kk * 2 + (mid >> 1)), a0, a1, a2, a3);
          if (kk & 1) mma_16816<kF16>(sb, a0, a1, a2, a3, qa[kk][0], qa[kk][1]);
          else mma_16816<kF16>(sa, a0, a1, a2, a3, qa[kk][0], qa[kk][1]);
        }
        auto seen = [&](int r) { return r < v.kv && (r >= v.lo || r < g.n_sink); };
        const bool v0 = seen(r0 + gq), v1 = seen(r0 + gq + 8);
        const float x00 = v0 ? (sa[0] + sb[0]) * g.scale2 : -INFINITY, x01 = v0 ? (sa[1] + sb[1]) * g.scale2 : -INFINITY;
        const float x10 = v1 ? (sa[2] + sb[2]) * g.scale2 : -INFINITY, x11 = v1 ? (sa[3] + sb[3]) * g.scale2 : -INFINITY;
        float bm0 = fmaxf(x00, x10), bm1 = fmaxf(x01, x11);
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) {
          bm0 = fmaxf(bm0, __shfl_xor_sync(0xffffffffu, bm0, w));
          bm1 = fmaxf(bm1, __shfl_xor_sync(0xffffffffu, bm1, w));
        }
        const float mn0 = fmaxf(m0, bm0 - kBias), mn1 = fmaxf(m1, bm1 - kBias);
        const float rf0 = mn0 == -INFINITY ? 0.f : mn0, rf1 = mn1 == -INFINITY ? 0.f : mn1;   // (logits may be -inf)
        const float c0 = ex2_approx(m0 - rf0), c1 = ex2_approx(m1 - rf1);
        const float p00 = ex2_approx(x00 - rf0), p01 = ex2_approx(x01 - rf1);
        const float p10 = ex2_approx(x10 - rf0), p11 = ex2_approx(x11 - rf1);
        l0 = l0 * c0 + (p00 + p10);   // over this thread's keys, summed over gq at the end
        l1 = l1 * c1 + (p01 + p11);
        m0 = mn0; m1 = mn1;
#pragma unroll
        for (int n = 0; n < kD / 16; ++n) { o[n][0] *= c0; o[n][1] *= c1; o[n][2] *= c0; o[n][3] *= c1; }
        const uint32_t pb0 = movmatrix_trans(pack16<kF16>(p00, p01)), pb1 = movmatrix_trans(pack16<kF16>(p10, p11));
        // rows that are not seen may hold anything, and zero times that could be a NaN: they become zeros
        const bool all = r0 + 16 <= v.kv && (r0 >= v.lo || r0 + 16 <= g.n_sink);
        uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
        if (!all) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            keep[e] = (seen(r0 + 2 * tq + 8 * e) ? 0xffffu : 0u) | (seen(r0 + 2 * tq + 8 * e + 1) ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int n = 0; n < kD / 16; ++n) {
          uint32_t a0, a1, a2, a3;
          ldmatrix_x4_trans(sV + off((lane & 7) + (mid >> 1) * 8, n * 2 + (mid & 1)), a0, a1, a2, a3);
          if (!all) { a0 &= keep[0]; a1 &= keep[0]; a2 &= keep[1]; a3 &= keep[1]; }
          mma_16816<kF16>(o[n], a0, a1, a2, a3, pb0, pb1);
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(empty(slot));
      if (++slot == kSlots) { slot = 0; ph ^= 1u; }
    }
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, w);
      l1 += __shfl_xor_sync(0xffffffffu, l1, w);
    }
    // ---- the warps' partials, then a warp per head with four outputs a lane
    meet();                        // (those of the unit before have been read)
    if (2 * tq < g.G) {
      float* w0 = tail.part[warp][2 * tq];
#pragma unroll
      for (int n = 0; n < kD / 16; ++n) {
        w0[n * 16 + gq] = o[n][0]; w0[n * 16 + gq + 8] = o[n][2];
        w0[kStride + n * 16 + gq] = o[n][1]; w0[kStride + n * 16 + gq + 8] = o[n][3];
      }
      if (gq == 0) {
        w0[kD] = m0; w0[kD + 1] = l0;
        w0[kStride + kD] = m1; w0[kStride + kD + 1] = l1;
      }
    }
    meet();
    auto own = [&](int head) {
      Partial p;
      p.clear();
      float mw[kStreamWarps];
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) { mw[w] = tail.part[w][head][kD]; p.m = fmaxf(p.m, mw[w]); }
      const float ref = p.m == -INFINITY ? 0.f : p.m;
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) {
        const float* r = tail.part[w][head];
        const float f = ex2_approx(mw[w] - ref);
        const float4 x = *reinterpret_cast<const float4*>(r + 4 * lane);
        p.l = fmaf(r[kD + 1], f, p.l);
        p.o[0] = fmaf(x.x, f, p.o[0]); p.o[1] = fmaf(x.y, f, p.o[1]);
        p.o[2] = fmaf(x.z, f, p.o[2]); p.o[3] = fmaf(x.w, f, p.o[3]);
      }
      return p;
    };
    auto finish = [&](Partial& p, int head) {
      const long long last_row = prefix.x + (long long)(prefix.y - 1) * prefix.z + (long long)h * prefix.w + head;
      // (not so only where groups overlap after a group_start that falls, whose records may be a mixture)
      if (prefix.y > 0 && prefix.y <= kSms && prefix.x >= 0 && prefix.z >= 0 && prefix.w >= 0 && last_row < a.max_rows)
        join_rows(p, prefix.y, lane, [&](int i) { return a.prefix_rows + ((size_t)prefix.x + (size_t)i * prefix.z + (size_t)h * prefix.w + head) * kStride; });
      const int hq = h * g.G + head;
      const float inv = p.l == 0.f ? 0.f : 1.f / p.l;    // no visible row: zeros
      uint2 w;
      w.x = pack16<kF16>(p.o[0] * inv, p.o[1] * inv);
      w.y = pack16<kF16>(p.o[2] * inv, p.o[3] * inv);
      reinterpret_cast<uint2*>(a.out)[((size_t)b * g.Hq + hq) * (kD / 4) + lane] = w;
      if (a.lse && lane == 0) a.lse[(size_t)b * g.Hq + hq] = p.l == 0.f ? -INFINITY : (p.m + log2f(p.l)) * kLn2;
    };
    const long long first = unit0 + kUnitCost;
    if (first >= begin && first + v.n_blocks <= end) {
      for (int head = warp; head < g.G; head += kStreamWarps) {
        Partial p = own(head);
        finish(p, head);
      }
    } else {
      const int c_first = (int)(first / share), c_last = (int)((first + v.n_blocks - 1) / share);
      for (int head = warp; head < g.G; head += kStreamWarps) {
        const Partial p = own(head);
        float* r = a.parts + (((size_t)blockIdx.x * 2 + ((int)blockIdx.x == c_first ? 1 : 0)) * kMaxG + head) * kStride;
        __stcg(reinterpret_cast<float4*>(r) + lane, make_float4(p.o[0], p.o[1], p.o[2], p.o[3]));
        if (lane == 0) __stcg(reinterpret_cast<float2*>(r + kD), make_float2(p.m, p.l));
      }
      __threadfence();
      meet();
      if (tid == 0) {
        const unsigned n = atomicAdd(a.counters + c_first, 1u);
        const bool last = n == (unsigned)(c_last - c_first);
        if (last) a.counters[c_first] = 0u;     // everybody has arrived: ready for the next launch
        __threadfence();
        tail.last = last;
      }
      meet();
      if (*reinterpret_cast<volatile int*>(&tail.last))
        for (int head = warp; head < g.G; head += kStreamWarps) {
          Partial p;
          p.clear();
          join_rows(p, c_last - c_first + 1, lane, [&](int i) {
            return a.parts + (((size_t)(c_first + i) * 2 + (i == 0 ? 1 : 0)) * kMaxG + head) * kStride;
          });
          finish(p, head);
        }
    }
  } while (next_unit());
}

template <bool kF16>
cudaError_t launch(const PagedDecodeArgs& d, const PagedWs& ws, cudaStream_t st) {
  static OncePerDevice granted;
  cudaError_t e = grant_smem(paged_decode_kernel<kF16>, kSmemBytes, granted);
  if (e != cudaSuccess) return e;
  KernelArgs a{};
  a.g = d.g;
  a.q = d.q; a.block_table = d.block_table; a.kv_len = d.kv_len; a.out = d.out; a.lse = d.lse;
  a.counters = (unsigned*)(d.wsp + kPagedCounters);
  a.parts = (float*)(d.wsp + kPagedDecodeParts);
  a.tokens = d.n_groups ? (const PagedToken*)(d.wsp + ws.tokens) : nullptr;
  a.prefix_rows = (const float*)(d.wsp + ws.part_o);
  a.max_rows = ws.max_rows;
  a.box_rows = std::min(d.g.page, kSlotRows);
  while ((1 << a.lg_box) < a.box_rows) ++a.lg_box;
  CUtensorMap km, vm;
  if (!paged_kv_map(&km, d.K, d.g, a.box_rows, 2) || !paged_kv_map(&vm, d.V, d.g, a.box_rows, 2)) return cudaErrorInvalidValue;
  e = launch_pdl(paged_decode_kernel<kF16>, dim3(kCtas), dim3(kThreads), kSmemBytes, st, km, vm, a);
  if (e == cudaSuccess) count_launch(1);
  return e;
}

}  // namespace

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, const PagedWs& ws, cudaStream_t st) {
  return a.g.f16 ? launch<true>(a, ws, st) : launch<false>(a, ws, st);
}

}  // namespace calidrop
