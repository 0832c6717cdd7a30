// Rotation and append: queries and keys of the new tokens are turned by their positions, keys and values go to their pages.
//
//   (x1, x2) -> (x1 c - x2 s, x2 c + x1 s),  c, s = cos_sin[pos][i], cos_sin[pos][rot/2 + i]
//
// Bound by memory: every row of q, k and v is read once and written once.  A warp has one token: it finds the token's
// sequence, place and page once, eight lanes take a row of 256 bytes, two 16-byte vectors each, and the vectors of a lane are
// the partners of a rotation by halves (elements 8j.. and rot/2 + 8j..), so no value crosses lanes.  The angles of a lane are
// the same for all heads and stay in registers.  Few tokens (a decode step) take a warp per four rows, so that nothing waits for
// a second row; many take four rows a lane, whose loads are in flight together: 16284 tokens of 36 heads out of a fused projection, 308 MB, 57 us
// (82 % of the copy bandwidth; written rows of 256 bytes are scattered over the heads' pages).  A step of 8 tokens takes 3.2 to 3.8 us, the
// pace at which the host calls, one of 256 tokens 3.7 to 4.2.  Rows asked for ahead of the look-up: no gain.
#include "paged_common.cuh"

namespace calidrop {

namespace {

// one 16-byte vector of each half of the rotated elements
template <bool kF16>
__device__ __forceinline__ void turn_halves(uint4& x, uint4& y, const float (&c)[8], const float (&s)[8]) {
  uint32_t* a = &x.x;
  uint32_t* b = &y.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 u = unpack16<kF16>(a[i]), w = unpack16<kF16>(b[i]);
    a[i] = pack16<kF16>(u.x * c[2 * i] - w.x * s[2 * i], u.y * c[2 * i + 1] - w.y * s[2 * i + 1]);
    b[i] = pack16<kF16>(w.x * c[2 * i] + u.x * s[2 * i], w.y * c[2 * i + 1] + u.y * s[2 * i + 1]);
  }
}
// neighbouring pairs: four angles for a vector
template <bool kF16>
__device__ __forceinline__ void turn_pairs(uint4& x, const float* c, const float* s) {
  uint32_t* a = &x.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 u = unpack16<kF16>(a[i]);
    a[i] = pack16<kF16>(u.x * c[i] - u.y * s[i], u.y * c[i] + u.x * s[i]);
  }
}

// kRows: rows of a lane group.  Warps of a token: as many as its rows need.
template <bool kF16, int kRows>
__global__ void __launch_bounds__(256) paged_append_kernel(const PagedAppendArgs a, int warps_per_token) {
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long w = ((long long)(blockIdx.x - 1) * blockDim.x + threadIdx.x) >> 5;
  const PagedGeom& g = a.g;
  const int t = (int)(w / warps_per_token), part = (int)(w - (long long)t * warps_per_token);
  pdl_wait();
  const int cap = g.max_pages << g.lg_page;
  if (blockIdx.x == 0) {       // a block of its own, the first to run: the starts and lengths of all sequences, with tokens or without
#pragma unroll 4
    for (int b = threadIdx.x; b < g.B; b += blockDim.x) {
      const int s0 = __ldg(a.q_start + b), s1 = __ldg(a.q_start + b + 1), kv = __ldg(a.kv_len + b);
      if (s0 < 0 || s1 < s0 || s1 > g.n_tokens || kv < 0 || kv > cap) paged_flag(g.status, kBadLength);
    }
    return;
  }
  if (t >= g.n_tokens || t >= __ldg(a.q_start + g.B)) return;
  const int b = paged_find(a.q_start, g.B, t, lane);
  if (b < 0) { if (lane == 0) paged_flag(g.status, kBadLength); return; }
  const int s0 = __ldg(a.q_start + b), s1 = __ldg(a.q_start + b + 1), kv = __ldg(a.kv_len + b);
  const long long at = (long long)kv - s1 + t;     // place in the cache (64 bits: the lengths may be anything)
  if (s0 < 0 || s1 <= t || s1 > g.n_tokens || kv < 0 || kv > cap || at < 0) {
    if (lane == 0) paged_flag(g.status, kBadLength);
    return;
  }
  const int pos = a.positions ? __ldg(a.positions + t) : (int)at;
  if (a.rot_dim && (pos < 0 || pos >= a.max_pos)) { if (lane == 0) paged_flag(g.status, kBadPosition); return; }
  const int page = __ldg(a.block_table + (size_t)b * g.max_pages + (at >> g.lg_page));
  if (page < 0 || page >= g.n_pages) { if (lane == 0) paged_flag(g.status, kBadPage); return; }

  const int j = lane & 7;                          // lane of the row
  const int rc = a.rot_dim >> 4;                   // vectors of half of the rotated elements
  const bool rot = j < rc;
  const int c0 = rot ? j : 2 * rc + 2 * (j - rc), c1 = rot ? j + rc : c0 + 1;   // the lane's two vectors
  alignas(16) float cs[8], sn[8];
  if (rot) {
    const float* base = a.cos_sin + (size_t)pos * a.rot_dim;
    const float4 *pc, *ps, *pc2, *ps2;
    // halves: angles 8j..8j+7; pairs: 4 c0.. for the first vector and 4 c1.. for the second
    pc = reinterpret_cast<const float4*>(base) + (a.interleaved ? c0 : 2 * j);
    pc2 = a.interleaved ? reinterpret_cast<const float4*>(base) + c1 : pc + 1;
    ps = pc + (a.rot_dim >> 3);
    ps2 = pc2 + (a.rot_dim >> 3);
    *reinterpret_cast<float4*>(cs) = __ldg(pc); *reinterpret_cast<float4*>(cs + 4) = __ldg(pc2);
    *reinterpret_cast<float4*>(sn) = __ldg(ps); *reinterpret_cast<float4*>(sn + 4) = __ldg(ps2);
  }
  const int n_q = a.q ? g.Hq : 0, n_rows = n_q + 2 * g.Hkv;
  const size_t page_at = (size_t)page * (g.page_stride >> 3) + (size_t)(at & (g.page - 1)) * 16;
  const uint4* src[kRows];
  uint4* dst[kRows];
  uint4 x[kRows], y[kRows];
  const int r0 = part * 4 * kRows + (lane >> 3);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + 4 * i;
    if (r < n_q) {
      src[i] = a.q + (size_t)t * (g.q_stride >> 3) + r * 16;
      dst[i] = a.q_out + ((size_t)t * g.Hq + r) * 16;
    } else if (r < n_q + g.Hkv) {
      src[i] = a.k + (size_t)t * (g.k_stride >> 3) + (r - n_q) * 16;
      dst[i] = a.K + page_at + (size_t)(r - n_q) * g.page * 16;
    } else {
      src[i] = a.v + (size_t)t * (g.v_stride >> 3) + (r - n_q - g.Hkv) * 16;
      dst[i] = a.V + page_at + (size_t)(r - n_q - g.Hkv) * g.page * 16;
    }
    if (r < n_rows) {
      x[i] = src[i][c0];       // (not through the read-only path: q_out may be q)
      y[i] = src[i][c1];
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + 4 * i;
    if (r >= n_rows) break;
    if (rot && r < n_q + g.Hkv) {
      if (a.interleaved) {
        turn_pairs<kF16>(x[i], cs, sn);
        turn_pairs<kF16>(y[i], cs + 4, sn + 4);
      } else {
        turn_halves<kF16>(x[i], y[i], cs, sn);
      }
    }
    dst[i][c0] = x[i];
    dst[i][c1] = y[i];
  }
}

template <bool kF16, int kRows>
cudaError_t launch(const PagedAppendArgs& a, cudaStream_t st) {
  const int n_rows = (a.q ? a.g.Hq : 0) + 2 * a.g.Hkv;
  const int warps = (n_rows + 4 * kRows - 1) / (4 * kRows);
  const long long blocks = ((long long)a.g.n_tokens * warps + 7) / 8 + 1;   // (the first looks the starts over)
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const cudaError_t e = launch_pdl(paged_append_kernel<kF16, kRows>, dim3((unsigned)blocks), dim3(256), 0, st, a, warps);
  if (e == cudaSuccess) count_launch(1);
  return e;
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st) {
  // One row a lane or four: the former while its warps are all resident at once (40 registers: 48 warps an SM).  Measured, us, one / four,
  // a token a sequence: 48 rows a token, 500 tokens 4.7 / 4.9, 583 4.7 / 4.7, 666 6.0 / 5.3, 833 7.0 / 6.1; 36 rows, 666 tokens 4.5 / 4.5, 888
  // 6.0 / 5.1; 10 rows, 2100 tokens 4.5 / 4.4, 2400 5.7 / 4.6, 3200 7.0 / 5.0.  In long appends of 48 rows a token 12 thousand rows 3.5 / 4.1,
  // 24 thousand 4.1 / 4.6, 28 thousand 5.0 / 4.7, 128 thousand 15.7 / 13.2.  (Two rows a lane: 586 thousand rows 60, four 57.)
  const int n_rows = (a.q ? a.g.Hq : 0) + 2 * a.g.Hkv;
  const bool many = (long long)a.g.n_tokens * ((n_rows + 3) / 4) > 48 * kSms;
  if (a.g.f16) return many ? launch<true, 4>(a, st) : launch<true, 1>(a, st);
  return many ? launch<false, 4>(a, st) : launch<false, 1>(a, st);
}

}  // namespace calidrop
