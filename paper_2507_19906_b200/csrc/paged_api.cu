// C-ABI layer of the entry points over a cache in pages: argument validation and launch sequencing.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "../../include/calidrop.h"
#include "common.cuh"
#include "paged.h"

using namespace calidrop;

namespace {

static_assert(CALIDROP_MAX_SEQUENCES == kMaxSequences, "");

bool bad_ptr(const void* p) { return !p || (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool bad_ptr4(const void* p) { return !p || (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }   // i32 arrays

int check_stride(int64_t stride, int64_t least) {
  return stride == 0 || (stride >= least && (stride & 7) == 0 && stride < (1ll << 38)) ? CALIDROP_OK : CALIDROP_INVALID_ARG;
}

int check_paged(const calidrop_paged_params* p) {
  if (!p) return CALIDROP_INVALID_ARG;
  if (p->B < 1 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0) return CALIDROP_INVALID_ARG;
  if (p->n_pages < 1 || p->max_pages < 1 || p->window < 0 || p->n_sink < 0) return CALIDROP_INVALID_ARG;
  if (!(p->softmax_scale >= 0.f) || !std::isfinite(p->softmax_scale)) return CALIDROP_INVALID_ARG;
  if (p->D != kD || p->Hq / p->Hkv > kMaxG || p->B > kMaxSequences) return CALIDROP_UNSUPPORTED;
  if (p->dtype != CALIDROP_BF16 && p->dtype != CALIDROP_FP16) return CALIDROP_UNSUPPORTED;
  if (p->page_size < 16 || p->page_size > 256 || (p->page_size & (p->page_size - 1))) return CALIDROP_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page_size > (1ll << 30) || (int64_t)p->max_prefix_pages * p->page_size > (1ll << 30))
    return CALIDROP_INVALID_ARG;   // positions are 32-bit
  if (p->Hq > 4096) return CALIDROP_UNSUPPORTED;
  if (p->rot_dim < 0 || p->rot_dim > kD || p->rot_dim % 16 || (p->interleaved & ~1)) return CALIDROP_UNSUPPORTED;
  if (p->rot_dim && p->max_pos < 1) return CALIDROP_INVALID_ARG;
  if (p->n_groups < 0 || p->n_groups > p->B || (p->n_groups && p->max_prefix_pages < 1)) return CALIDROP_INVALID_ARG;
  int rc = check_stride(p->q_stride, (int64_t)p->Hq * kD);
  if (rc == CALIDROP_OK) rc = check_stride(p->k_stride, (int64_t)p->Hkv * kD);
  if (rc == CALIDROP_OK) rc = check_stride(p->v_stride, (int64_t)p->Hkv * kD);
  if (rc == CALIDROP_OK) rc = check_stride(p->page_stride, (int64_t)p->Hkv * p->page_size * kD);
  return rc;
}

constexpr int32_t kMaxTokens = 1 << 25;

PagedWs ws_of(const calidrop_paged_params* p, int32_t n_tokens) {
  return paged_ws(p->B, p->Hq, p->Hkv, n_tokens, p->n_groups);
}

PagedGeom geom_of(const calidrop_paged_params* p, int32_t n_tokens, void* workspace) {
  PagedGeom g{};
  g.B = p->B; g.Hq = p->Hq; g.Hkv = p->Hkv; g.G = p->Hq / p->Hkv; g.n_tokens = n_tokens;
  g.page = p->page_size;
  while ((1 << g.lg_page) < g.page) ++g.lg_page;
  g.n_pages = p->n_pages; g.max_pages = p->max_pages;
  g.window = std::min(p->window, 1 << 30); g.n_sink = std::min(p->n_sink, 1 << 30);   // (more rows than a sequence has)
  g.scale2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)kD)) * kLog2e;
  g.q_stride = p->q_stride ? p->q_stride : (int64_t)p->Hq * kD;
  g.k_stride = p->k_stride ? p->k_stride : (int64_t)p->Hkv * kD;
  g.v_stride = p->v_stride ? p->v_stride : (int64_t)p->Hkv * kD;
  g.page_stride = p->page_stride ? p->page_stride : (int64_t)p->Hkv * p->page_size * kD;
  g.f16 = p->dtype == CALIDROP_FP16;
  g.status = (unsigned*)workspace;
  return g;
}

// What all calls check of their workspace, and of the device; the last checks ahead of a launch.
int check_run(const calidrop_paged_params* p, int32_t n_tokens, void* workspace, size_t workspace_bytes) {
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return CALIDROP_INVALID_ARG;
  if (workspace_bytes < ws_of(p, n_tokens).total) return CALIDROP_WORKSPACE_TOO_SMALL;
  return device_supported() ? CALIDROP_OK : CALIDROP_UNSUPPORTED;
}

}  // namespace

extern "C" {

size_t calidrop_paged_workspace_bytes(const calidrop_paged_params* p, int32_t n_tokens) {
  if (check_paged(p) != CALIDROP_OK || n_tokens < 0 || n_tokens > kMaxTokens) return 0;
  return ws_of(p, n_tokens).total;
}

int calidrop_paged_append(const calidrop_paged_params* p, int32_t n_tokens, const void* q, const void* k, const void* v,
                          const int32_t* positions, const float* cos_sin, void* K_pages, void* V_pages,
                          const int32_t* block_table, const int32_t* q_start, const int32_t* kv_len, void* q_out,
                          void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_paged(p);
  if (rc != CALIDROP_OK) return rc;
  if (n_tokens < 0 || n_tokens > kMaxTokens) return CALIDROP_INVALID_ARG;
  if (bad_ptr(K_pages) || bad_ptr(V_pages) || bad_ptr4(block_table) || bad_ptr4(q_start) || bad_ptr4(kv_len)) return CALIDROP_INVALID_ARG;
  if (n_tokens && (bad_ptr(k) || bad_ptr(v))) return CALIDROP_INVALID_ARG;
  if (positions && bad_ptr4(positions)) return CALIDROP_INVALID_ARG;
  if (q && (bad_ptr(q) || bad_ptr(q_out))) return CALIDROP_INVALID_ARG;
  if (q && q == q_out && p->q_stride && p->q_stride != (int64_t)p->Hq * kD) return CALIDROP_INVALID_ARG;
  if (p->rot_dim && bad_ptr(cos_sin)) return CALIDROP_INVALID_ARG;
  rc = check_run(p, n_tokens, workspace, workspace_bytes);
  if (rc != CALIDROP_OK || n_tokens == 0) return rc;
  PagedAppendArgs a{};
  a.g = geom_of(p, n_tokens, workspace);
  a.q = (const uint4*)q; a.k = (const uint4*)k; a.v = (const uint4*)v;
  a.positions = positions; a.block_table = block_table; a.q_start = q_start; a.kv_len = kv_len;
  a.cos_sin = cos_sin;
  a.K = (uint4*)K_pages; a.V = (uint4*)V_pages; a.q_out = (uint4*)q_out;
  a.rot_dim = p->rot_dim; a.interleaved = p->interleaved; a.max_pos = p->max_pos;
  const cudaError_t e = launch_paged_append(a, (cudaStream_t)stream);
  return e == cudaSuccess ? CALIDROP_OK : cuda_fail(e);
}

int calidrop_paged_prefill(const calidrop_paged_params* p, int32_t n_tokens, const void* q, const void* K_pages,
                           const void* V_pages, const int32_t* block_table, const int32_t* q_start,
                           const int32_t* kv_len, void* out, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream) {
  int rc = check_paged(p);
  if (rc != CALIDROP_OK) return rc;
  if (n_tokens < 0 || n_tokens > kMaxTokens) return CALIDROP_INVALID_ARG;
  if (bad_ptr(K_pages) || bad_ptr(V_pages) || bad_ptr4(block_table) || bad_ptr4(q_start) || bad_ptr4(kv_len)) return CALIDROP_INVALID_ARG;
  if (n_tokens && (bad_ptr(q) || bad_ptr(out))) return CALIDROP_INVALID_ARG;
  if (lse && bad_ptr4(lse)) return CALIDROP_INVALID_ARG;
  rc = check_run(p, n_tokens, workspace, workspace_bytes);
  if (rc != CALIDROP_OK || n_tokens == 0) return rc;
  PagedAttnArgs a{};
  a.g = geom_of(p, n_tokens, workspace);
  a.q = q; a.K = K_pages; a.V = V_pages;
  a.block_table = block_table; a.q_start = q_start; a.kv_len = kv_len;
  a.n_seqs = p->B; a.causal = 1; a.partial = 0;
  a.out = out; a.lse = lse; a.wsp = (char*)workspace;
  const cudaError_t e = launch_paged_attention(a, ws_of(p, n_tokens), (cudaStream_t)stream);
  return e == cudaSuccess ? CALIDROP_OK : cuda_fail(e);
}

int calidrop_paged_decode(const calidrop_paged_params* p, const void* q, const void* K_pages, const void* V_pages,
                          const int32_t* block_table, const int32_t* kv_len, void* out, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream) {
  int rc = check_paged(p);
  if (rc != CALIDROP_OK) return rc;
  if (bad_ptr(q) || bad_ptr(K_pages) || bad_ptr(V_pages) || bad_ptr4(block_table) || bad_ptr4(kv_len) || bad_ptr(out)) return CALIDROP_INVALID_ARG;
  if (lse && bad_ptr4(lse)) return CALIDROP_INVALID_ARG;
  rc = check_run(p, p->B, workspace, workspace_bytes);
  if (rc != CALIDROP_OK) return rc;
  PagedDecodeArgs a{};
  a.g = geom_of(p, p->B, workspace);
  a.q = q; a.K = K_pages; a.V = V_pages; a.block_table = block_table; a.kv_len = kv_len;
  a.out = out; a.lse = lse; a.wsp = (char*)workspace;
  const cudaError_t e = launch_paged_decode(a, ws_of(p, p->B), (cudaStream_t)stream);
  return e == cudaSuccess ? CALIDROP_OK : cuda_fail(e);
}

int calidrop_paged_prefix_decode(const calidrop_paged_params* p, const void* q, const void* K_pages, const void* V_pages,
                                 const int32_t* group_start, const int32_t* prefix_table, const int32_t* prefix_len,
                                 const int32_t* block_table, const int32_t* kv_len, void* out, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_paged(p);
  if (rc != CALIDROP_OK) return rc;
  if (p->n_groups < 1) return CALIDROP_INVALID_ARG;
  if (p->window) return CALIDROP_UNSUPPORTED;
  if (bad_ptr(q) || bad_ptr(K_pages) || bad_ptr(V_pages) || bad_ptr4(block_table) || bad_ptr4(kv_len) || bad_ptr(out)) return CALIDROP_INVALID_ARG;
  if (bad_ptr4(group_start) || bad_ptr4(prefix_table) || bad_ptr4(prefix_len)) return CALIDROP_INVALID_ARG;
  if (lse && bad_ptr4(lse)) return CALIDROP_INVALID_ARG;
  rc = check_run(p, p->B, workspace, workspace_bytes);
  if (rc != CALIDROP_OK) return rc;
  const PagedWs ws = ws_of(p, p->B);
  PagedAttnArgs a{};
  a.g = geom_of(p, p->B, workspace);
  a.g.max_pages = p->max_prefix_pages;
  a.q = q; a.K = K_pages; a.V = V_pages;
  a.block_table = prefix_table; a.q_start = group_start; a.kv_len = prefix_len;
  a.n_seqs = p->n_groups; a.causal = 0; a.partial = 1;
  a.wsp = (char*)workspace;
  cudaError_t e = launch_paged_attention(a, ws, (cudaStream_t)stream);
  if (e != cudaSuccess) return cuda_fail(e);
  PagedDecodeArgs d{};
  d.g = geom_of(p, p->B, workspace);
  d.q = q; d.K = K_pages; d.V = V_pages; d.block_table = block_table; d.kv_len = kv_len;
  d.out = out; d.lse = lse; d.wsp = (char*)workspace;
  d.n_groups = p->n_groups; d.group_start = group_start;
  e = launch_paged_decode(d, ws, (cudaStream_t)stream);
  return e == cudaSuccess ? CALIDROP_OK : cuda_fail(e);
}

}  // extern "C"
