// Attention of drafted tokens over the paged token cache (see include/scalekv.h for the contract).
//
// The draft's tokens are new tokens like others, and the kernels are those of paged_stream.cuh and paged_tile.cuh: everything before the draft is seen whole, by all rows, and
// what bounds them is the same.  Only the last key tiles, in which the draft lies, are masked, by bits: 32 positions' worth are taken from two words of the row's token (tree_bits).
// us, 32 heads on 8 of 128, codes: 8 tokens behind 1 991 entries 15.2, 64 tokens of 16 sequences of up to 10 521 entries 236 (128 items of up to 83 key tiles, one to an SM: the longest takes 2.8 us for each of its
// tiles).  Equal shares of all items' tiles, a CTA with one item after the other, took 235 to 245: 52 tiles an SM at 3.3 us, which is what a tile takes with all SMs at work, are 173, the join of the
// parts is 23, and what the other 40 were was not found.
#include "paged_attend.cuh"

using namespace scalekv;
using namespace scalekv::paged;

bool scalekv::paged::room_for_tree(int head_dim, bool q8) {
  if (head_dim == 128) return q8 ? room_for_attend<128, true, true>() : room_for_attend<128, false, true>();
  return q8 ? room_for_attend<64, true, true>() : room_for_attend<64, false, true>();
}

extern "C" {

scalekv_status scalekv_paged_attend_tree(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, int32_t n_heads, scalekv_rows Q, scalekv_rows O, float *lse,
                                         const int32_t *tree, int32_t tree_words, float softmax_scale, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_attend_tree");
  AttendArgs a;
  if (scalekv_status st = check_batch(c, layer, batch, a.bt)) return st;
  if (scalekv_status st = check_heads(c, n_heads, softmax_scale)) return st;
  if (tree_words < 0 || (long long)tree_words * 32 < batch->max_new)
    return fail(c, SCALEKV_ERR_INVALID_ARG, "%d words hold no bit for each of %d new tokens", tree_words, batch->max_new);
  if (a.bt.n_tokens > 0 && !tree) return fail(c, SCALEKV_ERR_INVALID_ARG, "tree null");
  a.mask = {0, 0, 0};
  a.tree = tree;
  a.tree_words = tree_words;
  return attend_over<true>(c, layer, batch, n_heads, Q, O, lse, a, softmax_scale, stream);
}

}  // extern "C"
