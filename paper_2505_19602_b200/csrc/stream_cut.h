// How the keys of sequences are cut for the streaming attention: apart, so that it compiles without CUDA.  What the host decides by the sizes of a call, and
// what the CTAs of a launch decide by the lengths.
#pragma once
#include <algorithm>

#ifdef __CUDACC__
#define SCALEKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define SCALEKV_HOST_DEVICE inline
#endif

namespace scalekv {
namespace paged {

// Rows of partial results that a launch may leave (rows of the call times CTAs that share a row's keys).
constexpr long long kPartRows = 148 * 256;
constexpr int kMaxCounts = 4096;                  // sequences times kv heads of a launch whose keys are shared
constexpr int kMostParts = 256;                   // of a sequence and head: what the last CTA's shared memory has room for
constexpr int kStreamWarps = 4;                   // of a CTA
// What a share that begins in one sequence and ends in the next costs a CTA beyond a whole part, in steps.  (us, 8 kv heads in codes, n sequences of two fifths of L to L entries, equal
// parts / equal shares: 32 x 10 521 131.1 / 105.6, 32 x 6 000 80.2 / 68.4, 64 x 6 000 141.9 / 119.6, 64 x 3 000 75.2 / 71.3, 100 x 3 000 107.0 / 102.9, and the other way round 64 x 1 500
// 42.2 / 47.3, 64 all of 2 000 60.2 / 67.7.  Not the better side: 32 x 3 000 46.6 / 43.6 has parts, 100 x 1 500 60.4 / 64.6 and 200 x 1 500 104.5 / 118.4 shares.)
constexpr int kSecond = 40;

// CTAs that an SM has room for: n: n-tiles of eight query rows
constexpr int stream_ctas(int head_dim, bool q8, int n) { return head_dim * (q8 ? 1 : 2) >= 256 ? 2 : n == 2 && head_dim == 128 ? 3 : 4; }

struct StreamCut {
  int split;                       // CTAs that share a sequence's keys, or
  int most_parts;                  // > 0: the parts are dealt out on the device, no more than this to a sequence and head
};
// items: sequences times heads (and rows beyond the first 16); slots: CTAs that the device has room for; rows: query rows of the call; keys: of the longest sequence.
inline StreamCut cut_stream(int n_sm, int slots, int n_seqs, long long items, long long rows, long long keys) {
  const long long steps = (keys + 15) / 16;
  const long long room = std::min<long long>(kPartRows / rows, kMostParts);      // parts that the workspace holds
  // CTAs that share a sequence's keys: one for every SM, down to two steps of 16 keys for each of its warps; two where that leaves them four; as many as
  // fit where it leaves them 16.  (us, one sequence with 8 kv heads in codes, 4 / 8 / 16 / 32 / 74 CTAs a head: 1 999 entries 12.8 / 10.3 / 8.6 / 10.6 / 18.5, 8 000
  // 31.7 / 19.8 / 13.4 / 13.3 / 17.9, 32 000 107.7 / 58.9 / 34.1 / 26.7 / 28.9.)  Then no more of them than the longest warp's number of steps asks for.
  long long split = std::max(n_sm / items, std::max(std::min(2 * n_sm / items, steps / 16), std::min(slots / items, steps / 64)));
  split = std::max<long long>(1, std::min(split, (steps + 7) / 8));
  const long long each = ((steps + split - 1) / split + kStreamWarps - 1) / kStreamWarps * kStreamWarps;
  split = std::max<long long>(1, std::min((steps + each - 1) / each, room));
  // Sequences of different lengths have their parts dealt out on the device, where that gives a CTA 64 steps or more (32 of up to 10 521 entries: 117 us in equal parts of
  // each, 108 so).
  const bool by_length = n_seqs > 1 && n_seqs <= 512 && items <= std::min<long long>(kMaxCounts, 3 * slots) && room >= 3 && items * steps >= slots * 64LL;
  if (items > kMaxCounts) split = 1;
  return {(int)split, by_length ? (int)room : 0};
}

struct StreamDeal {
  int split;                       // equal parts of every sequence and head, or
  int share;                       // > 0: steps of a CTA, of all sequences and heads one behind the other
};
// total: steps of all items; longest: of the longest one; ctas: of the launch.
SCALEKV_HOST_DEVICE StreamDeal deal_steps(long long total, int longest, int items, int ctas, int most_parts) {
  int split = ctas / items < longest / 8 ? ctas / items : longest / 8;
  split = split < most_parts ? split : most_parts;
  split = split > 1 ? split : 1;
  const int equal = (int)((total + ctas - 1) / ctas), least = (longest + most_parts - 2) / (most_parts - 1);
  const int share = equal > least ? equal : least;
  return {split, share + kSecond >= (items + ctas - 1) / ctas * ((longest + split - 1) / split) ? 0 : share};
}

}  // namespace paged
}  // namespace scalekv
