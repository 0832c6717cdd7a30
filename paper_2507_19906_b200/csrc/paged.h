// What the kernels over a cache in pages share: the geometry of a call, the layout of its workspace, and the launchers.
#pragma once

#include "internal.h"

namespace calidrop {

constexpr int kMaxSequences = 4096;
constexpr int kPagedTileKeys = 128;   // keys of a tile of the tensor-core attention
constexpr int kPagedRows = 256;       // query rows of an item of it: two streams of 128

// bits of the workspace's error word.  kWaitRanOut: beside the code of the wait, which is stored only where the word was 0
constexpr unsigned kBadLength = 1u, kBadPage = 2u, kBadPosition = 4u, kWaitRanOut = 0x1000u;

struct PagedGeom {
  int B, Hq, Hkv, G, n_tokens;
  int page, lg_page, n_pages, max_pages;
  int window, n_sink;
  float scale2;                // softmax scale * log2(e)
  long long q_stride, k_stride, v_stride, page_stride;   // elements
  int f16;
  unsigned* status;
};

// Workspace of a call: the fixed part first, so that calls of different sizes may share a workspace.
constexpr int kPagedMaxCtas = 2 * kSms;                         // of the decode kernel
constexpr size_t kPagedCounters = 256;                          // arrival counters, one per CTA
constexpr size_t kPagedDecodeParts = kPagedCounters + 4096;     // [CTA][2][8][132] f32
constexpr int kPagedPartStride = kD + 4;                        // floats of a partial row: 128 outputs, maximum, sum
constexpr size_t kPagedPlan = kPagedDecodeParts + (size_t)kPagedMaxCtas * 2 * kMaxG * kPagedPartStride * 4;
static_assert(kPagedMaxCtas * 4 <= 4096 && kPagedPlan % 256 == 0, "");

struct PagedWs {
  size_t sched, heavy, tokens, part_o, total;
  long long max_rows;          // partial rows
};

// Where the attention of a sequence's query token over a shared prefix lies: chunk c of head g of kv head h is partial row
// part_row + c * chunk_rows + h * head_rows + g.
struct PagedToken {
  int part_row, n_chunks, chunk_rows, head_rows;
};

// paged_append.cu
struct PagedAppendArgs {
  PagedGeom g;
  const uint4 *q, *k, *v;
  const int *positions, *block_table, *q_start, *kv_len;
  const float* cos_sin;
  uint4 *K, *V, *q_out;
  int rot_dim, interleaved, max_pos;
};
cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st);

// paged_prefill.cu: attention of packed tokens over pages.  With `partial` every tile of rows leaves partial rows (which
// the decode kernel joins), `causal` off every token sees the keys [0, kv_len) of its sequence.
struct PagedAttnArgs {
  PagedGeom g;
  const void *q, *K, *V;
  const int *block_table, *q_start, *kv_len;
  int n_seqs;
  int causal, partial;
  void* out;
  float* lse;
  char* wsp;
};
PagedWs paged_ws(int B, int Hq, int Hkv, int n_tokens, int n_groups);
cudaError_t launch_paged_attention(const PagedAttnArgs& a, const PagedWs& ws, cudaStream_t st);

// paged_decode.cu: one token a sequence.  n_groups > 0: joined with the partial rows of launch_paged_attention over the groups' prefixes.
struct PagedDecodeArgs {
  PagedGeom g;
  const void *q, *K, *V;
  const int *block_table, *kv_len;
  void* out;
  float* lse;
  char* wsp;
  int n_groups;
  const int* group_start;
};
cudaError_t launch_paged_decode(const PagedDecodeArgs& a, const PagedWs& ws, cudaStream_t st);

#ifdef __CUDACC__
__device__ __forceinline__ void paged_flag(unsigned* status, unsigned bit) { atomicOr(status, bit); }

// The largest b in [0, n) with start[b] <= t, for a non-decreasing start of n + 1 entries with start[0] <= t; -1 if there is
// none.  All lanes of a warp ask for the same t: each round they look at 32 places of the range at once, so that a batch of a
// thousand sequences costs two rounds and not ten dependent loads.
__device__ __forceinline__ int paged_find(const int* start, int n, int t, int lane) {
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 31) >> 5;
    const int i = lo + lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, lane * step < len && __ldg(start + i) <= t);
    const int k = max(0, __popc(m) - 1);
    const int end = lo + len;
    lo += k * step;
    len = min(step, end - lo);
  }
  return __ldg(start + lo) <= t ? lo : -1;
}
#endif

}  // namespace calidrop
