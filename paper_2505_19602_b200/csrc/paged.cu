// Host runtime and C ABI of the paged token cache (see include/scalekv.h for the contract): checks arguments, cuts launches.
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <string>

#include "../../include/scalekv.h"
#include "paged_attend.cuh"
#include "paged_store.cuh"

using namespace scalekv;
using namespace scalekv::paged;

namespace scalekv {
namespace paged {
extern const cudaLaunchAttributeID kBehindTheOneBefore = cudaLaunchAttributeProgrammaticStreamSerialization;
}  // namespace paged
}  // namespace scalekv

namespace {

scalekv_status make_layout(const scalekv_paged_config *c, Layout &y, std::string &err) {
  if (!c) { err = "null config"; return SCALEKV_ERR_INVALID_ARG; }
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1) { err = "n_layers, n_pages and n_kv_heads must be >= 1"; return SCALEKV_ERR_INVALID_ARG; }
  if (c->page_tokens < 16 || (c->page_tokens & (c->page_tokens - 1))) { err = "page_tokens must be a power of two >= 16"; return SCALEKV_ERR_INVALID_ARG; }
  if (c->head_dim != 64 && c->head_dim != 128) { err = "unsupported head_dim: 64 and 128 are built"; return SCALEKV_ERR_UNSUPPORTED; }
  if (c->store != SCALEKV_STORE_BF16 && c->store != SCALEKV_STORE_Q8) { err = "unknown store"; return SCALEKV_ERR_INVALID_ARG; }
  const double rows = (double)c->n_layers * c->n_pages * c->n_kv_heads * c->page_tokens;
  if (rows > 1e14 || (long long)c->n_pages * c->page_tokens > 0x7fffffffLL || (long long)c->n_layers * c->n_pages > 0x7fffffffLL ||
      (long long)c->n_kv_heads * c->page_tokens > 0x7fffffffLL) {
    err = "more than 2^31 - 1 tokens in a layer's pages, pages in all layers or rows in a page";
    return SCALEKV_ERR_CAPACITY;
  }
  const size_t n = (size_t)c->n_layers * c->n_pages * c->n_kv_heads * c->page_tokens;
  y.rows_bytes = n * c->head_dim * (c->store == SCALEKV_STORE_Q8 ? 1 : 2);
  y.scale_bytes = c->store == SCALEKV_STORE_Q8 ? n * 4 : 0;
  y.pool_bytes = 2 * (y.rows_bytes + y.scale_bytes);
  y.ws_bytes = kStatusBytes + kMaxCounts * 4 + (size_t)kPartRows * (c->head_dim + 2) * 4;
  return SCALEKV_OK;
}

template <bool kWrite, typename T, int D, bool kQ8>
void launch_store(Moves &mv, int n_sm, cudaStream_t stream) {
  // as many tokens to a block as give its threads four pieces (read: one, two, four, eight of them, 84 168 tokens of 8 heads: 106 / 96 / 92 / 92 us;
  // written and read back, two, four, eight, 24 646 tokens of 16 heads: 116 / 112 / 112), unless the blocks then leave SMs idle
  mv.per_token = Divisor::of(2 * mv.s.heads * (D / 16));
  const int n = mv.bt.n_tokens, full = (4 * kStoreThreads + mv.per_token.d - 1) / mv.per_token.d;
  mv.tokens = std::max(1, std::min(std::min(full, kMostTokens), n / (2 * n_sm)));
  const dim3 grid((n + mv.tokens - 1) / mv.tokens);
  if constexpr (kWrite) launch(paged_write_kernel<T, D, kQ8>, grid, kStoreThreads, 0, stream, mv);
  else launch(paged_read_kernel<T, D, kQ8>, grid, kStoreThreads, 0, stream, mv);
}

template <bool kWrite>
scalekv_status move_rows(scalekv_paged *c, int layer, const scalekv_paged_batch *batch, scalekv_rows K, scalekv_rows V, int dtype, void *stream) {
  if (!c) return SCALEKV_ERR_INVALID_ARG;
  Range range(kWrite ? "scalekv.paged_write" : "scalekv.paged_read");
  Batch bt;
  if (scalekv_status st = check_batch(c, layer, batch, bt)) return st;
  if (dtype != SCALEKV_BF16 && dtype != SCALEKV_F32) return fail(c, SCALEKV_ERR_UNSUPPORTED, "rows are bf16 or f32");
  if (bt.n_tokens == 0) return SCALEKV_OK;
  const int esize = dtype == SCALEKV_BF16 ? 2 : 4;
  if (!rows_ok(K, esize) || !rows_ok(V, esize)) return fail(c, SCALEKV_ERR_INVALID_ARG, "K/V null or rows not 16-byte aligned");
  if (c->cfg.n_kv_heads > 65535) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 65535 kv heads");
  Moves mv;
  mv.s = layer_store(c, layer);
  mv.bt = bt;
  mv.K = view(K, esize); mv.V = view(V, esize);
  mv.wide = rows_ok(K, esize, 32) && rows_ok(V, esize, 32);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    if (c->cfg.store == SCALEKV_STORE_Q8) launch_store<kWrite, T, D, true>(mv, c->n_sm, st);
    else launch_store<kWrite, T, D, false>(mv, c->n_sm, st);
  };
  auto typed = [&](auto t) {
    if (c->cfg.head_dim == 128) go(t, std::integral_constant<int, 128>{});
    else go(t, std::integral_constant<int, 64>{});
  };
  if (dtype == SCALEKV_BF16) typed(__nv_bfloat16{}); else typed(float{});
  return launched(c, kWrite ? "paged_write" : "paged_read");
}

}  // namespace

extern "C" {

scalekv_status scalekv_paged_query_sizes(const scalekv_paged_config *cfg, size_t *pool_bytes, size_t *workspace_bytes) {
  Layout y;
  std::string err;
  if (scalekv_status st = make_layout(cfg, y, err)) return st;
  if (pool_bytes) *pool_bytes = y.pool_bytes;
  if (workspace_bytes) *workspace_bytes = y.ws_bytes;
  return SCALEKV_OK;
}

scalekv_status scalekv_paged_init(const scalekv_paged_config *cfg, scalekv_paged **out) {
  if (!out) return SCALEKV_ERR_INVALID_ARG;
  *out = nullptr;
  Layout y;
  std::string err;
  scalekv_status st = make_layout(cfg, y, err);
  if (st) { fprintf(stderr, "scalekv_paged_init: %s\n", err.c_str()); return st; }
  if (!cfg->pool || !cfg->workspace || (reinterpret_cast<uintptr_t>(cfg->pool) & 255) || (reinterpret_cast<uintptr_t>(cfg->workspace) & 255)) {
    fprintf(stderr, "scalekv_paged_init: pool and workspace must be 256-byte aligned device pointers\n");
    return SCALEKV_ERR_INVALID_ARG;
  }
  if (cfg->pool_bytes < y.pool_bytes || cfg->workspace_bytes < y.ws_bytes) {
    fprintf(stderr, "scalekv_paged_init: pool needs %zu bytes, workspace %zu\n", y.pool_bytes, y.ws_bytes);
    return SCALEKV_ERR_CAPACITY;
  }
  scalekv_paged *c = new (std::nothrow) scalekv_paged;
  if (!c) return SCALEKV_ERR_CAPACITY;
  c->cfg = *cfg;
  c->lay = y;
  while ((1 << c->page_shift) < cfg->page_tokens) ++c->page_shift;
  if (cudaSetDevice(cfg->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&c->n_sm, cudaDevAttrMultiProcessorCount, cfg->device) != cudaSuccess ||
      cudaDeviceSynchronize() != cudaSuccess ||            // (whoever had this memory before may still be at work, on any stream)
      cudaMemset(cfg->workspace, 0, kStatusBytes + kMaxCounts * 4) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    fprintf(stderr, "scalekv_paged_init: %s\n", cudaGetErrorString(cudaGetLastError()));
    delete c;
    return SCALEKV_ERR_CUDA;
  }
  const bool q8 = cfg->store == SCALEKV_STORE_Q8;
  if (!(cfg->head_dim == 128 ? (q8 ? room_for_attend<128, true, false>() : room_for_attend<128, false, false>()) : (q8 ? room_for_attend<64, true, false>() : room_for_attend<64, false, false>())) ||
      !room_for_tree(cfg->head_dim, q8) || !room_for_weigh(cfg->head_dim, q8) || !room_for_evict()) {
    fprintf(stderr, "scalekv_paged_init: cannot raise the dynamic shared memory limit\n");
    cudaGetLastError();
    delete c;
    return SCALEKV_ERR_CUDA;
  }
  if (!c->maps.make(cfg->pool, static_cast<char *>(cfg->pool) + y.rows_bytes, (long long)cfg->n_layers * cfg->n_pages, cfg->n_kv_heads, cfg->page_tokens,
                    cfg->head_dim, cfg->store == SCALEKV_STORE_Q8, err)) {
    fprintf(stderr, "scalekv_paged_init: %s\n", err.c_str());
    delete c;
    return SCALEKV_ERR_CUDA;
  }
  *out = c;
  return SCALEKV_OK;
}

scalekv_status scalekv_paged_destroy(scalekv_paged *kv) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  delete kv;
  return SCALEKV_OK;
}

scalekv_status scalekv_paged_write(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, scalekv_rows K, scalekv_rows V, int32_t dtype,
                                   void *stream) {
  return move_rows<true>(kv, layer, batch, K, V, dtype, stream);
}

scalekv_status scalekv_paged_read(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, scalekv_rows K, scalekv_rows V, int32_t dtype,
                                  void *stream) {
  return move_rows<false>(kv, layer, batch, K, V, dtype, stream);
}

scalekv_status scalekv_paged_attend(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, int32_t n_heads, scalekv_rows Q, scalekv_rows O,
                                    float *lse, const scalekv_paged_mask *mask, float softmax_scale, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_attend");
  AttendArgs a;
  if (scalekv_status st = check_batch(c, layer, batch, a.bt)) return st;
  if (scalekv_status st = check_heads(c, n_heads, softmax_scale)) return st;
  if (!mask || mask->window < 0 || mask->n_sink < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "mask null, or a negative size in it");
  a.mask = {mask->causal != 0, std::min(mask->window, kMaxLength), mask->n_sink};
  a.tree = nullptr;
  a.tree_words = 0;
  return attend_over<false>(c, layer, batch, n_heads, Q, O, lse, a, softmax_scale, stream);
}

scalekv_status scalekv_paged_sync(scalekv_paged *kv, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  int status = 0;
  cudaError_t e = cudaMemcpyAsync(&status, kv->cfg.workspace, sizeof status, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return fail(kv, SCALEKV_ERR_CUDA, "sync: %s", cudaGetErrorString(e));
  if (status == 0) return SCALEKV_OK;
  return fail(kv, (scalekv_status)status, status == SCALEKV_ERR_TIMEOUT ? "a device-side wait gave up"
                                                                        : "a page, length or start of a batch was out of range: its rows were left out");
}

scalekv_status scalekv_paged_launch_count(scalekv_paged *kv, int64_t *count) {
  if (!kv || !count) return SCALEKV_ERR_INVALID_ARG;
  *count = kv->launches;
  return SCALEKV_OK;
}

const char *scalekv_paged_error_string(scalekv_paged *kv) { return kv ? kv->err.c_str() : "null handle"; }

}  // extern "C"
