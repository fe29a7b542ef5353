// What stays of a sequence in the paged token cache: the accepted tokens of a draft, and the entries that attention has paid most to (see include/scalekv.h for the contract).
#include <math_constants.h>

#include <type_traits>

#include "paged_host.cuh"

using namespace scalekv;
using namespace scalekv::paged;

namespace scalekv {
namespace paged {

// ---- accept: row first + path[i] of a sequence moves to first + i, in every layer, of K and V and their scales.
//
// A draft's rows move to places at or below their own, in ascending order, so a thread that has a column of the rows (16 bytes of a head's, or a scale) to itself takes them in that
// order, four loads and then their stores: what a store puts down lies below everything that is still to be loaded.  Few bytes; what bounds it is the look-up of a path's places, three trips to memory one behind the other, and
// the rows' own.  us, up to 8 of 64 drafted tokens of 32 sequences in 32 layers, 8 kv heads of 128 in codes: 6.6 (24.6 MB; eight loads at once, in 64 registers: 7.8); one sequence in 16 layers 3.0.
constexpr int kAcceptThreads = 256, kAcceptRows = 64;      // at most; of a block's paths

struct Accept {
  Store s;                                       // of the first layer
  size_t layer_rows, layer_scales;               // from a layer to the next: bytes, floats
  Batch bt;
  const int *path, *counts;
  int path_stride, path_len;
  int row_pieces, q8;                            // 16-byte pieces of a row
};

__global__ void __launch_bounds__(kAcceptThreads, 5) paged_accept_kernel(const __grid_constant__ Accept a) {
  __shared__ long long src[kAcceptRows], dst[kAcceptRows];
  __shared__ int stop;
  wait_for_grid();
  next_grid();
  const int b = blockIdx.x;
  const int start = a.bt.starts[b], end = a.bt.starts[b + 1], length = a.bt.lengths[b], count = a.counts[b];
  const int *path = a.path + (size_t)b * a.path_stride;
  // (a path's first entries are asked for beside these, not behind them)
  int j = 0, before = -1;
  if ((int)threadIdx.x < min(kAcceptRows, a.path_len)) {
    j = path[threadIdx.x];
    if (threadIdx.x > 0) before = path[threadIdx.x - 1];
  }
  const bool wrong = starts_wrong(a.bt, b, start, end) || count < 0 || count > a.path_len || count > end - start;
  if (wrong && threadIdx.x == 0) report(a.s.status);
  if (wrong || count == 0) return;
  const int first = length - (end - start);
  const int half = a.s.heads * a.row_pieces, columns = 2 * half + (a.q8 ? 2 * a.s.heads : 0), column = blockIdx.y * blockDim.x + threadIdx.x;
  for (int i0 = 0; i0 < count; i0 += kAcceptRows) {
    if (threadIdx.x == 0) stop = min(kAcceptRows, count - i0);
    __syncthreads();
    if ((int)threadIdx.x < kAcceptRows && i0 + (int)threadIdx.x < count) {
      const int i = i0 + threadIdx.x;
      if (i0 > 0) { j = path[i]; before = path[i - 1]; }
      bool ok = j > before && j < end - start && before >= -1;
      if (!ok) report(a.s.status);
      const int from = ok ? page_of(a.s, a.bt, b, first + j) : -1, to = ok ? page_of(a.s, a.bt, b, first + i) : -1;
      ok = from >= 0 && to >= 0;
      src[threadIdx.x] = ok ? (long long)store_row(a.s, from, 0, first + j) : 0;
      dst[threadIdx.x] = ok ? (long long)store_row(a.s, to, 0, first + i) : 0;
      if (!ok) atomicMin(&stop, (int)threadIdx.x);
    }
    __syncthreads();
    const int n = stop;
    if (column < columns) {
      if (column < 2 * half) {
        const bool v = column >= half;
        const int c = v ? column - half : column, head = c / a.row_pieces, piece = c - head * a.row_pieces;
        uint4 *rows = reinterpret_cast<uint4 *>((v ? a.s.v_rows : a.s.k_rows) + blockIdx.z * a.layer_rows) + ((size_t)head << a.s.page_shift) * a.row_pieces + piece;
        for (int i = 0; i < n; i += 4) {
          uint4 x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + k < n) x[k] = rows[(size_t)src[i + k] * a.row_pieces];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + k < n) rows[(size_t)dst[i + k] * a.row_pieces] = x[k];
        }
      } else {
        const bool v = column >= 2 * half + a.s.heads;
        const int head = column - 2 * half - (v ? a.s.heads : 0);
        float *scales = (v ? a.s.v_scales : a.s.k_scales) + blockIdx.z * a.layer_scales + ((size_t)head << a.s.page_shift);
        for (int i = 0; i < n; i += 4) {
          float x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + k < n) x[k] = scales[src[i + k]];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + k < n) scales[dst[i + k]] = x[k];
        }
      }
    }
    if (n < min(kAcceptRows, count - i0)) return;          // (the same for the whole block: what is behind a wrong one stays where it is)
    __syncthreads();
  }
}

// ---- evict: of the L entries of a sequence and kv head k stay, in their order: the first n_sink, the last n_recent and of those between them the heaviest, of equal ones
// the first.
//
// (1) paged_choose_kernel finds them: the weights as whole numbers of the same order, the k'th largest of them by three histograms of 11, 11 and 10 bits from the top, each of the keys that agree with
// it so far, in two copies, as the lanes of a warp often mean the same bin.  A long sequence's head is shared by a cluster of CTAs; every CTA holds its stretch of the keys in shared memory (those
// that find no room are read again), four of them to a load, and the histograms are summed over the cluster, a share of the bins by each.  Then every warp counts what it keeps of a stretch of
// its own and puts it down behind what lies before it.
// Up to 256 keys need no histogram: each counts those ahead of it (us, 24 items of 190 keys 14.2 so, 15.7 with histograms, 320 items of 490 keys 30.8 and 24.2, with one event's 10 us).
// (2) paged_gather_kernel moves the rows, which is most of the bytes, over all SMs whatever the heads and sequences are.
// us, (1) and (2), from cold caches: one sequence of 170 521 entries, 16 heads, bf16, to 17 052: 31 and 46 (6.0 TB/s); 8 of 10 521 entries, 8 heads in codes, to 1 052: 14 and 11.  (1) is bound by its chain: length, table, weights, and two
// or three histograms; an entry's weight is little to read.  (First built, a weight to a load and its page looked up ahead of each, 66 and 22; 1 024 threads 40 and 13; a cluster of two for 10 521 entries 17.  (2) with 32 / 64 / 128 entries
// a block: 49 / 46 / 45.5 and 16 / 14 / 11.)
constexpr int kChooseThreads = 512, kChooseWarps = kChooseThreads / 32, kBins = 2048, kMostCluster = 8;
constexpr int kFewKeys = 256;
constexpr int kCopies = 2;                       // of the histogram (so small that two CTAs with 21 000 keys each find room on an SM: clusters of eight need eight places near one another)
constexpr int kMostHeld = 40960;                 // keys that a CTA's shared memory holds, 160 KB

struct Evict {
  Store s;
  Batch bt;
  const int *keep;
  int *kept;                                     // [n_seqs][heads][kept_stride]
  int kept_stride, kept_len;
  const int *to;                                 // [n_seqs][to_stride], to_pages of them in use
  int to_stride, to_pages;
  float *weights;                                // [page][head][row of the page]
  int n_sink, n_recent;
  int held;                                      // keys that the launch gave shared memory for
  int moves;                                     // whoever chooses moves the rows, too
  int row_pieces, q8;
  Divisor heads, blocks;
};

// How many entries of sequence b stay, of `length`: none, where what it is told makes no sense, which whoever asks first tells.
__device__ __forceinline__ int kept_of(const Evict &a, int b, int &length, bool tell) {
  length = a.bt.lengths[b];
  const int keep = a.keep[b], room = a.bt.table_pages << a.s.page_shift, k = min(keep, length);
  const long long to_room = (long long)a.to_pages << a.s.page_shift;
  const bool wrong = (unsigned)length > (unsigned)room || keep < 0 || k > a.kept_len || k > to_room;
  if (wrong && tell) report(a.s.status);
  return wrong ? 0 : k;
}

// A weight as a whole number of the same order; -0 is 0, a NaN counts as -infinity.
__device__ __forceinline__ uint32_t key_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0x007fffffu : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The address of `at`, a place in this CTA's shared memory, in that of another CTA of the cluster.
__device__ __forceinline__ uint32_t peer_at(uint32_t at, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
  return r;
}
__device__ __forceinline__ uint2 peer_load2(uint32_t at) {
  uint2 r;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ void peer_store(uint32_t at, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void cluster_meet() {
  tc::cluster_arrive();
  tc::cluster_wait();
}

constexpr int kGatherThreads = 256, kGatherRows = 128, kGatherBatch = 4;
// With so few entries to move at most, whoever chooses them moves them.  (us, 10 521 entries of 64 / 2 heads to 128: 19.9 / 18.7 so, 21.3 / 20.5 in two launches; to 300 of 256 heads 32.5 / 31.5, to 1 052 of 2 heads 36.8 / 20.3; one
// event's 10 us in each.)
constexpr int kMostMoved = kGatherRows;

// Moves the entries numbers r0 .. r0 + n - 1, n <= kGatherRows, of those of a sequence and head that stay.  All threads of a block.
template <int kThreads>
__device__ __forceinline__ void gather_rows(const Evict &a, int b, int head, int r0, int n, long long *src, long long *dst) {
  if ((int)threadIdx.x < n) {
    const int i = r0 + threadIdx.x, pos = __ldcg(a.kept + ((size_t)b * a.s.heads + head) * a.kept_stride + i), to = a.to[(size_t)b * a.to_stride + (i >> a.s.page_shift)];
    const int from = page_of(a.s, a.bt, b, pos);
    const bool ok = (unsigned)to < (unsigned)a.s.n_pages;
    if (!ok) report(a.s.status);
    src[threadIdx.x] = from >= 0 && ok ? (long long)store_row(a.s, from, head, pos) : -1;
    dst[threadIdx.x] = ok ? (long long)store_row(a.s, to, head, i) : 0;
  }
  __syncthreads();
  const int both = 2 * a.row_pieces, shift = 31 - __clz(both);      // (a power of two)
  for (int i0 = threadIdx.x; i0 < n * both; i0 += kGatherBatch * kThreads) {
    uint4 x[kGatherBatch], *to[kGatherBatch];
#pragma unroll
    for (int j = 0; j < kGatherBatch; ++j) {
      const int i = i0 + j * kThreads, r = i >> shift, c = i & (both - 1);
      to[j] = nullptr;
      if (i < n * both && src[r] >= 0) {
        const bool v = c >= a.row_pieces;
        uint4 *rows = reinterpret_cast<uint4 *>(v ? a.s.v_rows : a.s.k_rows) + (v ? c - a.row_pieces : c);
        to[j] = rows + (size_t)dst[r] * a.row_pieces;
        x[j] = __ldcg(rows + (size_t)src[r] * a.row_pieces);
      }
    }
#pragma unroll
    for (int j = 0; j < kGatherBatch; ++j)
      if (to[j]) *to[j] = x[j];
  }
  if ((int)threadIdx.x < n && src[threadIdx.x] >= 0) {
    const size_t from = (size_t)src[threadIdx.x], to = (size_t)dst[threadIdx.x];
    a.weights[to] = __ldcg(a.weights + from);
    if (a.q8) {
      a.s.k_scales[to] = __ldcg(a.s.k_scales + from);
      a.s.v_scales[to] = __ldcg(a.s.v_scales + from);
    }
  }
}

__device__ __forceinline__ void choose_entries(const Evict &a, int cluster, int rank, int b, int head, int length, int k) {
  extern __shared__ __align__(16) uint32_t held[];
  __shared__ __align__(16) uint32_t bins[kBins * kCopies];
  __shared__ uint32_t total[kBins], warp_sum[kChooseWarps], found[3], counted[2 * kMostCluster], warp_before[2 * kChooseWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sinks = min(a.n_sink, k), recent = min(a.n_recent, k - sinks), end = length - recent;
  int need = k - sinks - recent;                 // of the entries sinks .. end - 1
  int *kept = a.kept + ((size_t)b * a.s.heads + head) * a.kept_stride;
  if (rank == 0) {
    for (int i = threadIdx.x; i < sinks; i += kChooseThreads) kept[i] = i;
    for (int i = threadIdx.x; i < recent; i += kChooseThreads) kept[k - recent + i] = end + i;
  }
  if (need == 0) return;                         // (all of the cluster)
  if (cluster > 1) cluster_meet();               // (all of them are there: from here on they look into each other's shared memory)
  // This CTA's stretch, in fours of positions: they lie together in a page.  A key of 0, which no weight has, is no entry to choose from.
  const int four0 = sinks >> 2, fours = ((end + 3) >> 2) - four0, per = (fours + cluster - 1) / cluster, from = min(rank * per, fours), mine = min(from + per, fours) - from;
  const bool in_shared = mine <= a.held >> 2;
  auto to_keys = [&](int i, const float4 &w) {
    const int pos = (four0 + from + i) << 2;
    uint4 x = make_uint4(key_of(w.x), key_of(w.y), key_of(w.z), key_of(w.w));
    if (pos < sinks || pos + 4 > end) {
      auto inside = [&](int p) { return p >= sinks && p < end; };
      x = make_uint4(inside(pos) ? x.x : 0u, inside(pos + 1) ? x.y : 0u, inside(pos + 2) ? x.z : 0u, inside(pos + 3) ? x.w : 0u);
    }
    return x;
  };
  const float4 least_w = make_float4(-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F);      // of entries without a page
  auto load_keys = [&](int i) {
    const int pos = (four0 + from + i) << 2, page = page_of(a.s, a.bt, b, pos);
    return to_keys(i, page >= 0 ? __ldcg(reinterpret_cast<const float4 *>(a.weights + store_row(a.s, page, head, pos))) : least_w);
  };
  uint4 *held4 = reinterpret_cast<uint4 *>(held);
  auto keys_at = [&](int i) { return in_shared ? held4[i] : load_keys(i); };
  const bool few = cluster == 1 && mine <= kFewKeys / 4 && in_shared;
  if (!few)
    for (int i = threadIdx.x; i < kBins * kCopies / 4; i += kChooseThreads) reinterpret_cast<uint4 *>(bins)[i] = make_uint4(0u, 0u, 0u, 0u);
  if (in_shared) {
    // (look-ups side by side, and then what they lead to: with one behind the other a thread's five fours of 10 521 entries took ten trips to memory)
    constexpr int kAtOnce = 6;
    const int *table = a.bt.table + (size_t)b * a.bt.table_ld;
    bool lost = false;
    for (int i0 = threadIdx.x; i0 < mine; i0 += kAtOnce * kChooseThreads) {
      int page[kAtOnce];
      float4 w[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int i = min(i0 + j * kChooseThreads, mine - 1);      // (within the length, so within the table)
        page[j] = table[((four0 + from + i) << 2) >> a.s.page_shift];
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int i = min(i0 + j * kChooseThreads, mine - 1);
        const bool there = (unsigned)page[j] < (unsigned)a.s.n_pages;
        lost = lost || !there;
        w[j] = least_w;
        if (there) w[j] = __ldcg(reinterpret_cast<const float4 *>(a.weights + store_row(a.s, page[j], head, (four0 + from + i) << 2)));
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (i0 + j * kChooseThreads < mine) held4[i0 + j * kChooseThreads] = to_keys(i0 + j * kChooseThreads, w[j]);
    }
    if (lost) report(a.s.status);
  }
  __syncthreads();
  if (few) {
    // a thread to each key, which counts those ahead of it: the larger ones, and the equal ones before it
    const uint32_t key = (int)threadIdx.x < 4 * mine ? held[threadIdx.x] : 0u;
    const int own = threadIdx.x >> 2;
    uint32_t ahead = 0;
    auto count = [&](const uint4 &x, uint32_t least) { ahead += (x.x >= least) + (x.y >= least) + (x.z >= least) + (x.w >= least); };
    for (int i = 0; i < min(own, mine); ++i) count(held4[i], key);
    for (int i = own + 1; i < mine; ++i) count(held4[i], key + 1u);
    if (own < mine) {
#pragma unroll
      for (int j = 0; j < 4; ++j) ahead += held[own * 4 + j] >= key + (j < (int)(threadIdx.x & 3) ? 0u : 1u);
    }
    const bool stays = key != 0u && ahead < (uint32_t)need;
    const unsigned vote = __ballot_sync(0xffffffffu, stays);
    if (lane == 0) warp_sum[warp] = __popc(vote);
    __syncthreads();
    const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane & (kChooseWarps - 1)] : 0u);
    if (stays) kept[sinks + before + __popc(vote & ((1u << lane) - 1u))] = (four0 << 2) + (int)threadIdx.x;
    return;
  }
  const uint32_t bins_at = tc::smem_u32(bins), total_at = tc::smem_u32(total), counted_at = tc::smem_u32(counted);
  uint32_t prefix = 0;                           // of the k'th largest key, below which bits are zeros that are not known
  bool ties = false;                             // some of the entries that have that key leave
  // (keys of 0 are counted in bin 0, which no other key has, or not at all: nobody comes down to them)
  auto narrow = [&](auto shift_, auto n_bins_) {
    constexpr int shift = decltype(shift_)::value, n_bins = decltype(n_bins_)::value;
    constexpr uint32_t known = shift == 21 ? 0u : ~0u << (shift == 0 ? 10 : shift + 11);
    auto count = [&](uint32_t key) {
      if (((key ^ prefix) & known) == 0u)
        atomicAdd(&bins[((key >> shift) & (n_bins - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
    };
    for (int i = threadIdx.x; i < mine; i += kChooseThreads) {
      const uint4 x = keys_at(i);
      count(x.x); count(x.y); count(x.z); count(x.w);
    }
    if (cluster > 1) cluster_meet(); else __syncthreads();
    const int share = n_bins / cluster;
    for (int i = threadIdx.x; i < share; i += kChooseThreads) {
      const int bin = rank * share + i;
      if (cluster == 1) {
        const uint2 x = reinterpret_cast<const uint2 *>(bins)[bin];
        total[bin] = x.x + x.y;
      } else {
        uint2 x[kMostCluster];
        uint32_t sum = 0;
#pragma unroll
        for (int c = 0; c < kMostCluster; ++c) x[c] = c < cluster ? peer_load2(peer_at(bins_at + 8 * bin, c)) : make_uint2(0u, 0u);
#pragma unroll
        for (int c = 0; c < kMostCluster; ++c) sum += x[c].x + x[c].y;
#pragma unroll
        for (int c = 0; c < kMostCluster; ++c)
          if (c < cluster) peer_store(peer_at(total_at + 4 * bin, c), sum);
      }
    }
    if (cluster > 1) cluster_meet(); else __syncthreads();
    if (shift > 0) {
      for (int i = threadIdx.x; i < kBins * kCopies / 4; i += kChooseThreads) reinterpret_cast<uint4 *>(bins)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    // the bin of the need'th largest: threads from the top bin down, two bins each or one
    constexpr int each = n_bins / kChooseThreads;
    const int top = n_bins - 1 - (int)threadIdx.x * each;
    uint32_t own = 0;
    for (int e = 0; e < each; ++e) own += total[top - e];
    uint32_t incl = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += up;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane & (kChooseWarps - 1)] : 0u);
    uint32_t above = before + incl - own;
    if (above < (uint32_t)need && above + own >= (uint32_t)need) {
      int e = 0;
      while (above + total[top - e] < (uint32_t)need) above += total[top - e++];
      found[0] = (uint32_t)(top - e);
      found[1] = above;
      found[2] = total[top - e];
    }
    __syncthreads();
    prefix |= found[0] << shift;
    need -= (int)found[1];
    ties = (uint32_t)need < found[2];
  };
  if (need < end - sinks) {
    narrow(std::integral_constant<int, 21>{}, std::integral_constant<int, kBins>{});
    if (ties) narrow(std::integral_constant<int, 10>{}, std::integral_constant<int, kBins>{});
    if (ties) narrow(std::integral_constant<int, 0>{}, std::integral_constant<int, 1024>{});
  } else {
    prefix = 1;
  }
  // Now every entry with a key of `prefix` or more stays or, where there are ties, those above it and the first `need` of those that have it.  A warp takes a stretch of the CTA's.
  const int warp_per = (mine + kChooseWarps - 1) / kChooseWarps, w0 = min(warp * warp_per, mine), w1 = min(w0 + warp_per, mine);
  const uint32_t least = ties ? prefix + 1u : prefix;      // (no key is 2^32 - 1)
  auto is_larger = [&](uint32_t key) { return key >= least ? 1u : 0u; };
  auto is_equal = [&](uint32_t key) { return key == prefix ? 1u : 0u; };
  uint32_t larger = 0, equal = 0;
  for (int i = w0 + lane; i < w1; i += 32) {
    const uint4 x = keys_at(i);
    larger += is_larger(x.x) + is_larger(x.y) + is_larger(x.z) + is_larger(x.w);
    if (ties) equal += is_equal(x.x) + is_equal(x.y) + is_equal(x.z) + is_equal(x.w);
  }
  larger = __reduce_add_sync(0xffffffffu, larger);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) { warp_before[2 * warp] = larger; warp_before[2 * warp + 1] = equal; }
  __syncthreads();
  static_assert(kChooseWarps <= 32, "a lane for each warp's counts");
  const uint32_t l_all = lane < kChooseWarps ? warp_before[2 * lane] : 0u, e_all = lane < kChooseWarps ? warp_before[2 * lane + 1] : 0u;
  uint32_t l = __reduce_add_sync(0xffffffffu, lane < warp ? l_all : 0u), e = __reduce_add_sync(0xffffffffu, lane < warp ? e_all : 0u);
  if (cluster > 1) {
    if (warp == 0) {
      const uint32_t l_sum = __reduce_add_sync(0xffffffffu, l_all), e_sum = __reduce_add_sync(0xffffffffu, e_all);
      if (lane < cluster) {
        peer_store(peer_at(counted_at + 8 * rank, lane), l_sum);
        peer_store(peer_at(counted_at + 8 * rank + 4, lane), e_sum);
      }
    }
    cluster_meet();                              // (nobody reads another's shared memory behind this)
    for (int c = 0; c < rank; ++c) { l += counted[2 * c]; e += counted[2 * c + 1]; }
  }
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const uint4 x = i0 + lane < w1 ? keys_at(i0 + lane) : make_uint4(0u, 0u, 0u, 0u);
    const uint32_t key[4] = {x.x, x.y, x.z, x.w};
    const int pos = (four0 + from + i0 + lane) << 2;
    uint32_t own = 0;                            // larger ones in the low half, equal ones in the high one: 128 at most
#pragma unroll
    for (int j = 0; j < 4; ++j) own += is_larger(key[j]) + (ties ? is_equal(key[j]) << 16 : 0u);
    uint32_t incl = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += up;
    }
    const uint32_t sum = __shfl_sync(0xffffffffu, incl, 31);
    int *to = kept + sinks + l + ((incl - own) & 0xffffu);
    if (!ties) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (key[j] >= least) *to++ = pos + j;
    } else {
      uint32_t e_here = e + ((incl - own) >> 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool larger_j = key[j] >= least, equal_j = key[j] == prefix;
        if (larger_j || (equal_j && e_here < (uint32_t)need)) to[min(e_here, (uint32_t)need)] = pos + j;
        to += larger_j;
        e_here += equal_j;
      }
      e += sum >> 16;
    }
    l += sum & 0xffffu;
  }
}

__global__ void __launch_bounds__(kChooseThreads) paged_choose_kernel(const __grid_constant__ Evict a, int cluster) {
  __shared__ long long src[kGatherRows], dst[kGatherRows];
  const int rank = cluster > 1 ? (int)cluster_rank() : 0, item = blockIdx.x / cluster, b = a.heads.div(item), head = item - b * a.heads.d;
  wait_for_grid();
  next_grid();
  int length;
  const int k = kept_of(a, b, length, head == 0 && rank == 0 && threadIdx.x == 0);
  if (k > 0) choose_entries(a, cluster, rank, b, head, length, k);
  if (!a.moves) return;
  // (a cluster of one: its own writes are there)
  for (int r0 = 0; r0 < k; r0 += kGatherRows) {
    __syncthreads();
    gather_rows<kChooseThreads>(a, b, head, r0, min(k - r0, kGatherRows), src, dst);
  }
}

__global__ void __launch_bounds__(kGatherThreads) paged_gather_kernel(const __grid_constant__ Evict a) {
  __shared__ long long src[kGatherRows], dst[kGatherRows];
  wait_for_grid();
  next_grid();
  const int item = a.blocks.div(blockIdx.x), block = blockIdx.x - item * a.blocks.d, b = a.heads.div(item), head = item - b * a.heads.d;
  int length;
  const int k = kept_of(a, b, length, false), r0 = block * kGatherRows, n = min(k - r0, kGatherRows);
  if (n > 0) gather_rows<kGatherThreads>(a, b, head, r0, n, src, dst);
}

}  // namespace paged
}  // namespace scalekv

bool scalekv::paged::room_for_evict() {
  return cudaFuncSetAttribute(paged_choose_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostHeld * 4) == cudaSuccess;
}

extern "C" {

scalekv_status scalekv_paged_accept(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, const int32_t *path, int32_t path_stride, int32_t path_len,
                                    const int32_t *counts, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_accept");
  Accept a;
  if (scalekv_status st = check_batch(c, layer == -1 ? 0 : layer, batch, a.bt)) return st;
  if (path_stride < 0 || path_len < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "path_stride or path_len negative");
  // (without tokens, or places in a path, all counts have to be 0, which the device looks at; a batch without tokens may come without its arrays)
  if (a.bt.n_seqs == 0 || (a.bt.n_tokens == 0 && (!a.bt.starts || !a.bt.lengths || !counts))) return SCALEKV_OK;
  if ((!path && path_len > 0) || !counts) return fail(c, SCALEKV_ERR_INVALID_ARG, "path or counts null");
  const int layers = layer == -1 ? c->cfg.n_layers : 1;
  a.s = layer_store(c, layer == -1 ? 0 : layer);
  a.layer_rows = c->lay.rows_bytes / c->cfg.n_layers;
  a.layer_scales = c->lay.scale_bytes / c->cfg.n_layers / 4;
  a.path = path; a.counts = counts; a.path_stride = path_stride; a.path_len = path_len;
  a.q8 = c->cfg.store == SCALEKV_STORE_Q8;
  a.row_pieces = c->cfg.head_dim * (a.q8 ? 1 : 2) / 16;
  const long long columns = 2LL * c->cfg.n_kv_heads * (a.row_pieces + a.q8), blocks = (columns + kAcceptThreads - 1) / kAcceptThreads;
  if (blocks > 65535 || layers > 65535) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 65535 layers, or too many kv heads");
  // (blocks of as many threads as there are columns for, and enough for a stretch of a path)
  const int threads = std::max(kAcceptRows, (int)((columns + blocks - 1) / blocks + 31) & ~31);
  launch(paged_accept_kernel, dim3((unsigned)a.bt.n_seqs, (unsigned)blocks, (unsigned)layers), threads, 0, static_cast<cudaStream_t>(stream), a);
  return launched(c, "paged_accept");
}

scalekv_status scalekv_paged_evict(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, const int32_t *to_table, int32_t to_stride, int32_t to_pages,
                                   const int32_t *keep, float *weights, int32_t n_sink, int32_t n_recent, int32_t *kept, int32_t kept_stride, int32_t kept_len, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_evict");
  Evict a;
  if (scalekv_status st = check_batch(c, layer, batch, a.bt)) return st;
  if (n_sink < 0 || n_recent < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "n_sink or n_recent negative");
  if (to_stride < 0 || to_pages < 0 || kept_stride < 0 || kept_len < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "a size of to_table or kept negative");
  const int H = c->cfg.n_kv_heads;
  const long long items = (long long)a.bt.n_seqs * H;
  if ((a.bt.n_seqs > 1 && to_stride < to_pages) || (items > 1 && kept_stride < kept_len)) return fail(c, SCALEKV_ERR_INVALID_ARG, "rows of to_table or kept overlap");
  if (a.bt.n_seqs == 0) return SCALEKV_OK;
  // (places for nothing need no memory, but what should stay all the same is told)
  if ((!a.bt.table && a.bt.table_pages > 0) || !a.bt.lengths || (!to_table && to_pages > 0) || !keep || !weights || (!kept && kept_len > 0)) return fail(c, SCALEKV_ERR_INVALID_ARG, "an array null");
  if (reinterpret_cast<uintptr_t>(weights) & 15) return fail(c, SCALEKV_ERR_INVALID_ARG, "weights not 16-byte aligned");
  // what the tables have room for, whatever the caller's bounds say
  const long long room = (long long)a.bt.table_pages << c->page_shift, most = std::min<long long>(std::min<long long>(kept_len, room), (long long)to_pages << c->page_shift);
  const long long blocks = std::max(1ll, (most + kGatherRows - 1) / kGatherRows);
  if (items * std::max<long long>(blocks, kMostCluster) > 0x7fffffffLL) return fail(c, SCALEKV_ERR_UNSUPPORTED, "too many sequences, kv heads and entries in a call");
  a.s = layer_store(c, layer);
  a.keep = keep; a.kept = kept; a.kept_stride = kept_stride; a.kept_len = kept_len;
  a.to = to_table; a.to_stride = to_stride; a.to_pages = to_pages;
  a.weights = weights;
  a.n_sink = n_sink; a.n_recent = n_recent;
  a.q8 = c->cfg.store == SCALEKV_STORE_Q8;
  a.row_pieces = c->cfg.head_dim * (a.q8 ? 1 : 2) / 16;
  a.heads = Divisor::of(H);
  a.blocks = Divisor::of((int)blocks);
  const int length = (int)std::max(1ll, std::min<long long>(batch->max_length, room));      // (at most kMaxLength)
  // as many CTAs to a sequence and head as find an SM, with more than 16 384 entries for each (us, one sequence to 1 000 entries, with one event's 7.  16 heads: 12 000 entries with 1 / 2 / 4 CTAs 25.9 / 26.4 / 25.5;
  // 20 000 with 1 / 2 / 4 / 8 31.9 / 28.8 / 26.0 / 29.9; 40 000 with 2 / 4 / 8 32.8 / 25.7 / 29.5; 80 000 with 4 / 8 34.6 / 32.0.  4 heads, 40 000 with 2 / 4 / 8 33.9 / 28.8 / 27.6.  One head, 20 000 with 1 / 2 / 4 / 8 29.2 / 24.2 / 22.2 / 22.0.
  // What the rule leaves out: four instead of two for 16 385 to 32 768 entries, a tenth.)
  int cluster = 1;
  while (cluster < kMostCluster && items * cluster <= c->n_sm && length > cluster * 16384) cluster *= 2;
  a.held = std::min((length + cluster - 1) / cluster + 8, kMostHeld) & ~3;      // (fours that begin and end inside)
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = kBehindTheOneBefore;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(items * cluster)); cfg.blockDim = dim3(kChooseThreads); cfg.dynamicSmemBytes = (size_t)a.held * 4; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = 2;
  a.moves = cluster == 1 && most <= kMostMoved;
  cudaLaunchKernelEx(&cfg, paged_choose_kernel, a, cluster);
  if (scalekv_status s = launched(c, "paged_choose")) return s;
  if (a.moves) return SCALEKV_OK;
  launch(paged_gather_kernel, dim3((unsigned)(items * blocks)), kGatherThreads, 0, st, a);
  return launched(c, "paged_gather");
}

}  // extern "C"
