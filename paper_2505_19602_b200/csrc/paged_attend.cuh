// The launches of the attention of new tokens, under a mask of positions (kTree: false) or under a draft's own.
#pragma once
#include "paged_host.cuh"

namespace scalekv {
namespace paged {

template <int D, bool kQ8, int kN, bool kTree>
scalekv_status launch_stream(scalekv_paged *c, const AttendArgs &a, int tiles, long long keys, cudaStream_t stream) {
  using Y = StreamLayout<D, kQ8, kN>;
  const int slots = c->n_sm * Y::kCtas;
  const StreamCut cut = cut_stream(c->n_sm, slots, a.bt.n_seqs, (long long)a.bt.n_seqs * a.s.heads * tiles, (long long)a.bt.n_tokens * a.n_heads, keys);
  launch(paged_stream_kernel<D, kQ8, kN, kTree>, cut.most_parts > 0 ? dim3((unsigned)slots) : dim3(a.bt.n_seqs, a.s.heads * tiles, (unsigned)cut.split), kStreamThreads, Y::kSmem,
         stream, a, cut.most_parts, tiles);
  return launched(c, kTree ? "paged_attend_tree" : "paged_attend");
}

template <int D, bool kQ8, bool kTree>
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
  launch(paged_tile_kernel<D, kQ8, kTree>, dim3((unsigned)(n_full + (n - n_full) * parts)), Y::kThreads, Y::kSmem, stream, c->maps.k, c->maps.v, a, cut,
         layer * c->cfg.n_pages);
  if (scalekv_status st = launched(c, kTree ? "paged_attend_tree" : "paged_attend")) return st;
  if (n_full == n) return SCALEKV_OK;
  launch(paged_join_kernel<D>, dim3((unsigned)((n - n_full) * (kItemRows / kJoinRows))), 32 * kJoinRows, 0, stream, a, cut);
  return launched(c, "paged_join");
}

// Lets the attention kernels of a handle have the shared memory they ask for.
template <int D, bool kQ8, bool kTree>
bool room_for_attend() {
  auto ask = [](auto kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess; };
  return ask(paged_stream_kernel<D, kQ8, 1, kTree>, StreamLayout<D, kQ8, 1>::kSmem) && ask(paged_stream_kernel<D, kQ8, 2, kTree>, StreamLayout<D, kQ8, 2>::kSmem) &&
         ask(paged_tile_kernel<D, kQ8, kTree>, TileLayout<D, kQ8>::kSmem);
}

// An attend behind the checks of its mask: a has the batch, and the mask or the draft.
template <bool kTree>
scalekv_status attend_over(scalekv_paged *c, int layer, const scalekv_paged_batch *batch, int n_heads, const scalekv_rows &Q, const scalekv_rows &O, float *lse, AttendArgs &a,
                           float softmax_scale, void *stream) {
  if (a.bt.n_tokens == 0) return SCALEKV_OK;
  if (!rows_ok(Q, 2) || !rows_ok(O, 2)) return fail(c, SCALEKV_ERR_INVALID_ARG, "Q/O null or rows not 16-byte aligned");
  const int H = c->cfg.n_kv_heads, D = c->cfg.head_dim;
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
      return max_rows <= 8 ? launch_stream<kD, kQ8, 1, kTree>(c, a, 1, keys, st) : launch_stream<kD, kQ8, 2, kTree>(c, a, row_tiles, keys, st);
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (D == 128) return q8 ? go(D128{}, std::true_type{}) : go(D128{}, std::false_type{});
    return q8 ? go(D64{}, std::true_type{}) : go(D64{}, std::false_type{});
  }
  // no more items than this, whatever the starts say
  const long long items = std::min<long long>((long long)a.bt.n_tokens * G / kItemRows + a.bt.n_seqs, (max_rows + kItemRows - 1) / kItemRows * a.bt.n_seqs);
  if (items * H > 0x3fffffffLL) return fail(c, SCALEKV_ERR_UNSUPPORTED, "too many row tiles in a call");
  if (D == 128) return q8 ? launch_tile<128, true, kTree>(c, layer, a, (int)items, keys, st) : launch_tile<128, false, kTree>(c, layer, a, (int)items, keys, st);
  return q8 ? launch_tile<64, true, kTree>(c, layer, a, (int)items, keys, st) : launch_tile<64, false, kTree>(c, layer, a, (int)items, keys, st);
}

}  // namespace paged
}  // namespace scalekv
