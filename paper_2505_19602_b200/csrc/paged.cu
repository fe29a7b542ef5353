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
#include "paged_store.cuh"
#include "paged_stream.cuh"
#include "paged_tile.cuh"

using namespace scalekv;
using namespace scalekv::paged;

namespace {

constexpr size_t kStatusBytes = 256;
constexpr int kMaxLength = 1 << 30;      // tokens that a sequence's pages may hold: sums of a position and a window stay in 32 bits

struct Layout {
  size_t rows_bytes, scale_bytes;        // of K, and of V, over all layers
  size_t pool_bytes, ws_bytes;
};

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

}  // namespace

struct scalekv_paged {
  scalekv_paged_config cfg;
  Layout lay;
  int n_sm = 148, page_shift = 0;
  int64_t launches = 0;
  TileMaps maps;
  std::string err = "ok";
};

namespace {

scalekv_status fail(scalekv_paged *c, scalekv_status st, const char *fmt, ...) {
  char buf[512];
  va_list ap; va_start(ap, fmt); vsnprintf(buf, sizeof buf, fmt, ap); va_end(ap);
  if (c) c->err = buf;
  return st;
}

Store layer_store(const scalekv_paged *c, int layer) {
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

bool rows_ok(const scalekv_rows &x, int esize, int align = 16) {
  return x.ptr != nullptr && !(reinterpret_cast<uintptr_t>(x.ptr) & (align - 1)) && (x.stride_t * esize) % align == 0 && (x.stride_h * esize) % align == 0;
}

Rows view(const scalekv_rows &x, int esize) { return {static_cast<char *>(const_cast<void *>(x.ptr)), x.stride_t * esize, x.stride_h * esize}; }

scalekv_status check_batch(scalekv_paged *c, int layer, const scalekv_paged_batch *b, Batch &out) {
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

scalekv_status launched(scalekv_paged *c, const char *what) {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(c, SCALEKV_ERR_CUDA, "launch of %s failed: %s", what, cudaGetErrorString(e));
  ++c->launches;
  return SCALEKV_OK;
}

struct Range {  // an NVTX range around one call
  explicit Range(const char *name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
};

// Every kernel here may be set up while the one before it in the stream is finishing: all of them wait for that one's end (griddepcontrol.wait)
// before they read or write anything.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
  cfg.attrs = &attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
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

template <int D, bool kQ8, int kN>
scalekv_status launch_stream(scalekv_paged *c, const AttendArgs &a, int tiles, long long keys, cudaStream_t stream) {
  using Y = StreamLayout<D, kQ8, kN>;
  const int slots = c->n_sm * Y::kCtas;
  const StreamCut cut = cut_stream(c->n_sm, slots, a.bt.n_seqs, (long long)a.bt.n_seqs * a.s.heads * tiles, (long long)a.bt.n_tokens * a.n_heads, keys);
  launch(paged_stream_kernel<D, kQ8, kN>, cut.most_parts > 0 ? dim3((unsigned)slots) : dim3(a.bt.n_seqs, a.s.heads * tiles, (unsigned)cut.split), kStreamThreads, Y::kSmem,
         stream, a, cut.most_parts, tiles);
  return launched(c, "paged_attend");
}

template <int D, bool kQ8>
scalekv_status launch_tile(scalekv_paged *c, int layer, const AttendArgs &a, int items, long long keys, cudaStream_t stream) {
  using Y = TileLayout<D, kQ8>;
  // An item and kv head to a CTA.  Those that do not fill the SMs are shared by as many CTAs as find one, each with two key tiles or more (us, 20 tokens behind
  // 8 192 entries, 8 kv heads in codes, 1 / 2 / 4 / 8 / 16 / 32 CTAs an item: 202 / 108 / 60 / 35 / 25 / 26), and so are those of the last, partial wave (2 x 16 heads, bf16, 1 400
  // queries over 1 500 / 3 000 / 5 000 entries, alone: 82 / 127 / 187, shared: 77 / 108 / 151).  Not with fewer than 16 key tiles: of a causal chunk the last wave are the items that see least, and
  // the launch that joins them can cost more than it gives (us, alone / shared: chunks beside single tokens under a window of 700 56 / 61; 2 x 1 400 causal queries of 16 heads behind 100 entries,
  // 44 of 192 items, in bf16 58 / 69, in codes 63 / 77; behind 800, 18 tiles, 84 / 86 and 94 / 98, behind 1 600 105 / 101 and 124 / 119).  What that leaves out: 12 last items with 10 CTAs each,
  // 10 x 256 queries of 16 heads behind 444 / 944 entries, in bf16 64 / 61 and 79 / 69, in codes 67 / 63 and 88 / 75.
  const int n = items * a.s.heads, sms = (int)std::min<long long>(c->n_sm, kPartRows / kItemRows), last = n % sms;
  const long long tiles = (keys + kTileKeys - 1) / kTileKeys;
  int parts = last ? (int)std::min<long long>(sms / last, tiles / 2) : 1;
  if (n > sms && tiles < 16) parts = 1;
  const int n_full = parts > 1 ? n - last : n;
  const Cut cut = {Divisor::of(a.s.heads), Divisor::of(std::max(parts, 1)), items, n_full};
  launch(paged_tile_kernel<D, kQ8>, dim3((unsigned)(n_full + (n - n_full) * parts)), Y::kThreads, Y::kSmem, stream, c->maps.k, c->maps.v, a, cut,
         layer * c->cfg.n_pages);
  if (scalekv_status st = launched(c, "paged_attend")) return st;
  if (n_full == n) return SCALEKV_OK;
  launch(paged_join_kernel<D>, dim3((unsigned)((n - n_full) * (kItemRows / kJoinRows))), 32 * kJoinRows, 0, stream, a, cut);
  return launched(c, "paged_join");
}

// Lets the attention kernels of a handle have the shared memory they ask for.
template <int D, bool kQ8>
bool room_for_attend() {
  auto ask = [](auto kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess; };
  return ask(paged_stream_kernel<D, kQ8, 1>, StreamLayout<D, kQ8, 1>::kSmem) && ask(paged_stream_kernel<D, kQ8, 2>, StreamLayout<D, kQ8, 2>::kSmem) &&
         ask(paged_tile_kernel<D, kQ8>, TileLayout<D, kQ8>::kSmem);
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
  if (!(cfg->head_dim == 128 ? (q8 ? room_for_attend<128, true>() : room_for_attend<128, false>()) : (q8 ? room_for_attend<64, true>() : room_for_attend<64, false>()))) {
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
  const int H = c->cfg.n_kv_heads, D = c->cfg.head_dim;
  if (n_heads < 1 || n_heads % H) return fail(c, SCALEKV_ERR_INVALID_ARG, "%d query heads are not a multiple of %d kv heads", n_heads, H);
  if (!mask || mask->window < 0 || mask->n_sink < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "mask null, or a negative size in it");
  if (!std::isfinite(softmax_scale) || softmax_scale < 0.f) return fail(c, SCALEKV_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  if (a.bt.n_tokens == 0) return SCALEKV_OK;
  if (!rows_ok(Q, 2) || !rows_ok(O, 2)) return fail(c, SCALEKV_ERR_INVALID_ARG, "Q/O null or rows not 16-byte aligned");
  const long long all_rows = (long long)a.bt.n_tokens * n_heads;
  const int G = n_heads / H;
  const long long max_rows = (long long)std::min(batch->max_new, a.bt.n_tokens) * G;      // query rows of a sequence and kv head
  if (all_rows > kMaxLength) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 2^30 query rows in a call");
  if (H > 32767) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 32767 kv heads");
  a.s = layer_store(c, layer);
  a.Q = view(Q, 2); a.O = view(O, 2);
  a.lse = lse;
  a.counts = reinterpret_cast<int *>(static_cast<char *>(c->cfg.workspace) + kStatusBytes);
  a.part_o = reinterpret_cast<float *>(a.counts + kMaxCounts);
  a.part_ml = a.part_o + (size_t)kPartRows * D;
  a.mask = {mask->causal != 0, std::min(mask->window, kMaxLength), mask->n_sink};
  a.group = Divisor::of(G);
  a.n_heads = n_heads;
  a.max_new = batch->max_new;
  a.scale_log2e = (softmax_scale > 0.f ? softmax_scale : 1.f / std::sqrt((float)D)) * kLog2e;
  long long keys = std::max(batch->max_length, 1);
  if (a.mask.window > 0) keys = std::min<long long>(keys, (long long)a.mask.window + batch->max_new + a.mask.n_sink);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool q8 = c->cfg.store == SCALEKV_STORE_Q8;
  // Up to 32 query rows stream.  (us, 64 heads, 8 kv heads of 128, 8 000 entries, streamed / on the tensor cores' tiles, one / 8 / 32 sequences.  Codes: 16 rows 23.7 / 23.5, 54 / 117, 149 / 420; 24 rows
  // 24.9 / 23.6, 86 / 117, 268 / 420; 32 rows 25.0 / 23.7, 87 / 117, 270 / 420; 40 rows 29.4 / 24.0, 121 / 118, 394 / 421; 64 rows 32 / 25, 148 / 119, 519 / 423.  bf16: 16 rows 25.8 / 20.8, 61 / 63, 189 / 202;
  // 24 rows 27.1 / 21.2, 96 / 64, 370 / 203; 32 rows 27.2 / 21.6, 96 / 65, 370 / 204; 64 rows 34 / 26, 191 / 69, 700 / 211.  By time alone bf16 rows would stream up to 16; up to 32 they do for the
  // sake of P, which the tiles round to bf16.)
  if (max_rows <= kStreamRows) {
    auto go = [&](auto dim, auto codes) {
      constexpr int kD = decltype(dim)::value;
      constexpr bool kQ8 = decltype(codes)::value;
      const int row_tiles = (int)((max_rows + kTileRows - 1) / kTileRows);
      return max_rows <= 8 ? launch_stream<kD, kQ8, 1>(c, a, 1, keys, st) : launch_stream<kD, kQ8, 2>(c, a, row_tiles, keys, st);
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (D == 128) return q8 ? go(D128{}, std::true_type{}) : go(D128{}, std::false_type{});
    return q8 ? go(D64{}, std::true_type{}) : go(D64{}, std::false_type{});
  }
  // no more items than this, whatever the starts say
  const long long items = std::min<long long>((long long)a.bt.n_tokens * G / kItemRows + a.bt.n_seqs, (max_rows + kItemRows - 1) / kItemRows * a.bt.n_seqs);
  if (items * H > 0x3fffffffLL) return fail(c, SCALEKV_ERR_UNSUPPORTED, "too many row tiles in a call");
  if (D == 128) return q8 ? launch_tile<128, true>(c, layer, a, (int)items, keys, st) : launch_tile<128, false>(c, layer, a, (int)items, keys, st);
  return q8 ? launch_tile<64, true>(c, layer, a, (int)items, keys, st) : launch_tile<64, false>(c, layer, a, (int)items, keys, st);
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
