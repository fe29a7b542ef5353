// What the host side of the paged token cache's calls shares: the handle, the checks of their arguments, the launch.
#pragma once
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>

#include "../../include/scalekv.h"
#include "paged_tile.cuh"

namespace scalekv {
namespace paged {

constexpr size_t kStatusBytes = 256;
constexpr int kMaxLength = 1 << 30;      // tokens that a sequence's pages may hold: sums of a position and a window stay in 32 bits

struct Layout {
  size_t rows_bytes, scale_bytes;        // of K, and of V, over all layers
  size_t pool_bytes, ws_bytes;
};

}  // namespace paged
}  // namespace scalekv

struct scalekv_paged {
  scalekv_paged_config cfg;
  scalekv::paged::Layout lay;
  int n_sm = 148, page_shift = 0;
  int64_t launches = 0;
  scalekv::paged::TileMaps maps;
  std::string err = "ok";
};

namespace scalekv {
namespace paged {

inline scalekv_status fail(scalekv_paged *c, scalekv_status st, const char *fmt, ...) {
  char buf[512];
  va_list ap; va_start(ap, fmt); vsnprintf(buf, sizeof buf, fmt, ap); va_end(ap);
  if (c) c->err = buf;
  return st;
}

inline Store layer_store(const scalekv_paged *c, int layer) {
  const scalekv_paged_config &g = c->cfg;
  const size_t rows = c->lay.rows_bytes / g.n_layers, scales = c->lay.scale_bytes / g.n_layers;
  char *pool = static_cast<char *>(g.pool);
  Store s;
  s.k_rows = pool + rows * layer;
  s.v_rows = pool + c->lay.rows_bytes + rows * layer;
  s.k_scales = reinterpret_cast<float *>(pool + 2 * c->lay.rows_bytes + scales * layer);
  s.v_scales = reinterpret_cast<float *>(pool + 2 * c->lay.rows_bytes + c->lay.scale_bytes + scales * layer);
  s.n_pages = g.n_pages; s.heads = g.n_kv_heads; s.page_shift = c->page_shift;
  s.status = static_cast<int *>(g.workspace);
  return s;
}

inline bool rows_ok(const scalekv_rows &x, int esize, int align = 16) {
  return x.ptr != nullptr && !(reinterpret_cast<uintptr_t>(x.ptr) & (align - 1)) && (x.stride_t * esize) % align == 0 && (x.stride_h * esize) % align == 0;
}

inline Rows view(const scalekv_rows &x, int esize) { return {static_cast<char *>(const_cast<void *>(x.ptr)), x.stride_t * esize, x.stride_h * esize}; }

inline scalekv_status check_batch(scalekv_paged *c, int layer, const scalekv_paged_batch *b, Batch &out) {
  if (layer < 0 || layer >= c->cfg.n_layers) return fail(c, SCALEKV_ERR_INVALID_ARG, "layer %d out of range", layer);
  if (!b || b->n_seqs < 0 || b->n_tokens < 0 || b->max_new < 0 || b->max_length < 0)
    return fail(c, SCALEKV_ERR_INVALID_ARG, "batch null, or a negative size in it");
  if (b->n_seqs == 0 && b->n_tokens > 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "tokens without sequences");
  if (b->n_tokens > 0 && (!b->page_table || !b->lengths || !b->starts)) return fail(c, SCALEKV_ERR_INVALID_ARG, "batch array null");
  if (b->n_tokens > 0 && b->max_new < 1) return fail(c, SCALEKV_ERR_INVALID_ARG, "max_new must be >= 1 when there are tokens");
  if (b->table_stride < 0 || b->table_pages < 0 || ((long long)b->table_pages << c->page_shift) > kMaxLength)
    return fail(c, SCALEKV_ERR_INVALID_ARG, "table_stride or table_pages negative, or a sequence's pages hold more than 2^30 tokens");
  out = {b->page_table, b->lengths, b->starts, b->table_stride, b->table_pages, b->n_seqs, b->n_tokens};
  return SCALEKV_OK;
}

inline scalekv_status check_heads(scalekv_paged *c, int n_heads, float softmax_scale) {
  const int H = c->cfg.n_kv_heads;
  if (n_heads < 1 || n_heads % H) return fail(c, SCALEKV_ERR_INVALID_ARG, "%d query heads are not a multiple of %d kv heads", n_heads, H);
  if (!std::isfinite(softmax_scale) || softmax_scale < 0.f) return fail(c, SCALEKV_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  return SCALEKV_OK;
}

inline scalekv_status launched(scalekv_paged *c, const char *what) {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(c, SCALEKV_ERR_CUDA, "launch of %s failed: %s", what, cudaGetErrorString(e));
  ++c->launches;
  return SCALEKV_OK;
}

struct Range {  // an NVTX range around one call
  explicit Range(const char *name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
};

// How the kernels here are launched: every one may be set up while the one before it in the stream is finishing, and waits for that one's end
// (griddepcontrol.wait) before it reads or writes anything.
extern const cudaLaunchAttributeID kBehindTheOneBefore;
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  attr.id = kBehindTheOneBefore;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
  cfg.attrs = &attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// Lets the kernels of the calls that have a file of their own have the shared memory they ask for.
bool room_for_tree(int head_dim, bool q8);
bool room_for_evict();
bool room_for_weigh(int head_dim, bool q8);

}  // namespace paged
}  // namespace scalekv
