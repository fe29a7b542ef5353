// What stays of a sequence in the paged token cache: the accepted tokens of a draft, and the entries that attention has paid most to (see include/scalekv.h for the contract).
#include <math_constants.h>

#include "paged_host.cuh"

using namespace scalekv;
using namespace scalekv::paged;

namespace scalekv {
namespace paged {

// ---- accept: row first + path[i] of a sequence moves to first + i, in every layer, of K and V and their scales.
//
// A draft's rows move to places at or below their own, in ascending order, so a thread that has a column of the rows (16 bytes of a head's, or a scale) to itself takes them in that
// order, eight loads and then their stores: what a store puts down lies below everything that is still to be loaded.  Few bytes; what bounds it is the look-up of a path's places, four trips to memory one behind the other.
constexpr int kAcceptThreads = 128, kAcceptRows = 64;

struct Accept {
  Store s;                                       // of the first layer
  size_t layer_rows, layer_scales;               // from a layer to the next: bytes, floats
  Batch bt;
  const int *path, *counts;
  int path_stride, path_len;
  int row_pieces, q8;                            // 16-byte pieces of a row
};

__global__ void __launch_bounds__(kAcceptThreads) paged_accept_kernel(const __grid_constant__ Accept a) {
  __shared__ long long src[kAcceptRows], dst[kAcceptRows];
  __shared__ int stop;
  wait_for_grid();
  next_grid();
  const int b = blockIdx.x;
  const int start = a.bt.starts[b], end = a.bt.starts[b + 1], length = a.bt.lengths[b];
  int count = a.counts[b];
  const bool wrong = starts_wrong(a.bt, b, start, end) || count < 0 || count > a.path_len || count > end - start;
  if (wrong && threadIdx.x == 0) report(a.s.status);
  if (wrong || count == 0) return;
  const int first = length - (end - start);
  const int half = a.s.heads * a.row_pieces, columns = 2 * half + (a.q8 ? 2 * a.s.heads : 0), column = blockIdx.y * kAcceptThreads + threadIdx.x;
  for (int i0 = 0; i0 < count; i0 += kAcceptRows) {
    if (threadIdx.x == 0) stop = min(kAcceptRows, count - i0);
    __syncthreads();
    if ((int)threadIdx.x < kAcceptRows && i0 + (int)threadIdx.x < count) {
      const int i = i0 + threadIdx.x;
      const int *path = a.path + (size_t)b * a.path_stride + i;
      const int j = path[0], before = i > 0 ? path[-1] : -1;
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
        for (int i = 0; i < n; i += 8) {
          uint4 x[8];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i + k < n) x[k] = rows[(size_t)src[i + k] * a.row_pieces];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i + k < n) rows[(size_t)dst[i + k] * a.row_pieces] = x[k];
        }
      } else {
        const bool v = column >= 2 * half + a.s.heads;
        const int head = column - 2 * half - (v ? a.s.heads : 0);
        float *scales = (v ? a.s.v_scales : a.s.k_scales) + blockIdx.z * a.layer_scales + ((size_t)head << a.s.page_shift);
        for (int i = 0; i < n; i += 8) {
          float x[8];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i + k < n) x[k] = scales[src[i + k]];
#pragma unroll
          for (int k = 0; k < 8; ++k)
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
// it so far.  A cluster of CTAs shares a sequence and head; every CTA holds its stretch of the keys in shared memory (those that find no room are read again), and the histograms
// are summed over the cluster, a share of the bins by each.  Then every warp counts what it keeps of a stretch of its own and puts it down behind what lies before it.
// (2) paged_gather_kernel moves the rows, which is most of the bytes, over all SMs whatever the heads and sequences are.
constexpr int kChooseThreads = 512, kChooseWarps = kChooseThreads / 32, kBins = 2048, kMostCluster = 8;
constexpr int kMostHeld = 49152;                 // keys that a CTA's shared memory holds, 192 KB

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
  if (w != w) w = -CUDART_INF_F;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
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
__device__ __forceinline__ uint32_t peer_load(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ void peer_store(uint32_t at, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void cluster_meet() {
  tc::cluster_arrive();
  tc::cluster_wait();
}

__global__ void __launch_bounds__(kChooseThreads) paged_choose_kernel(const __grid_constant__ Evict a, int cluster) {
  extern __shared__ __align__(16) uint32_t held[];
  __shared__ uint32_t bins[kBins], total[kBins];
  __shared__ uint32_t warp_sum[kChooseWarps], found[2], counted[2 * kMostCluster], warp_before[2 * kChooseWarps];
  const int rank = cluster > 1 ? (int)cluster_rank() : 0, item = blockIdx.x / cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int b = a.heads.div(item), head = item - b * a.heads.d;
  wait_for_grid();
  next_grid();
  int length;
  const int k = kept_of(a, b, length, head == 0 && rank == 0 && threadIdx.x == 0);
  if (k == 0) return;                            // (all of the cluster)
  const int sinks = min(a.n_sink, k), recent = min(a.n_recent, k - sinks), middle = length - sinks - recent;
  int need = k - sinks - recent;                 // of the entries sinks .. sinks + middle - 1
  int *kept = a.kept + ((size_t)b * a.s.heads + head) * a.kept_stride;
  if (rank == 0) {
    for (int i = threadIdx.x; i < sinks; i += kChooseThreads) kept[i] = i;
    for (int i = threadIdx.x; i < recent; i += kChooseThreads) kept[k - recent + i] = length - recent + i;
  }
  if (need == 0) return;
  if (cluster > 1) cluster_meet();               // (all of them are there: from here on they look into each other's shared memory)
  const int per = (middle + cluster - 1) / cluster, from = min(rank * per, middle), mine = min(from + per, middle) - from;      // this CTA's stretch
  const bool in_shared = mine <= a.held;
  auto load_key = [&](int i) {
    const int pos = sinks + from + i, page = page_of(a.s, a.bt, b, pos);
    return page < 0 ? key_of(-CUDART_INF_F) : key_of(__ldcg(a.weights + store_row(a.s, page, head, pos)));
  };
  auto key_at = [&](int i) { return in_shared ? held[i] : load_key(i); };
  if (in_shared) {
#pragma unroll 4
    for (int i = threadIdx.x; i < mine; i += kChooseThreads) held[i] = load_key(i);
  }
  const uint32_t bins_at = tc::smem_u32(bins), total_at = tc::smem_u32(total), counted_at = tc::smem_u32(counted);
  uint32_t prefix = 0, known = 0;                // of the k'th largest key, and which bits of it
  const bool all = need == middle;
  for (int pass = 0; pass < 3 && !all; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, n_bins = pass == 2 ? 1024 : kBins;
    for (int i = threadIdx.x; i < n_bins; i += kChooseThreads) bins[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < mine; i += kChooseThreads) {
      const uint32_t key = key_at(i);
      if ((key & known) == prefix) atomicAdd(&bins[(key >> shift) & (n_bins - 1)], 1u);
    }
    if (cluster > 1) cluster_meet(); else __syncthreads();
    const int share = n_bins / cluster;
    for (int i = threadIdx.x; i < share; i += kChooseThreads) {
      const int bin = rank * share + i;
      uint32_t sum = 0;
      for (int c = 0; c < cluster; ++c) sum += cluster > 1 ? peer_load(peer_at(bins_at + 4 * bin, c)) : bins[bin];
      for (int c = 0; c < cluster; ++c) {
        if (cluster > 1) peer_store(peer_at(total_at + 4 * bin, c), sum);
        else total[bin] = sum;
      }
    }
    if (cluster > 1) cluster_meet(); else __syncthreads();
    // the bin of the need'th largest: threads from the top bin down, four or two bins each
    const int each = n_bins / kChooseThreads, top = n_bins - 1 - (int)threadIdx.x * each;
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
    uint32_t above = incl - own;
    for (int w = 0; w < warp; ++w) above += warp_sum[w];
    if (above < (uint32_t)need && above + own >= (uint32_t)need) {
      int e = 0;
      while (above + total[top - e] < (uint32_t)need) above += total[top - e++];
      found[0] = (uint32_t)(top - e);
      found[1] = above;
    }
    __syncthreads();
    prefix |= found[0] << shift;
    known |= (uint32_t)(n_bins - 1) << shift;
    need -= (int)found[1];
    __syncthreads();                             // (found is read before the next pass writes it)
  }
  // Now `prefix` is the key, and `need` of the entries that have it stay (all: everything does).  A warp takes a stretch of the CTA's.
  const int warp_per = (mine + kChooseWarps - 1) / kChooseWarps, w0 = min(warp * warp_per, mine), w1 = min(w0 + warp_per, mine);
  uint32_t larger = 0, equal = 0;
  for (int i = w0 + lane; i < w1; i += 32) {
    const uint32_t key = all ? 0u : key_at(i);
    larger += all || key > prefix;
    equal += !all && key == prefix;
  }
  larger = __reduce_add_sync(0xffffffffu, larger);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) { warp_before[2 * warp] = larger; warp_before[2 * warp + 1] = equal; }
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t l = 0, e = 0;
    for (int w = 0; w < kChooseWarps; ++w) {
      const uint32_t lw = warp_before[2 * w], ew = warp_before[2 * w + 1];
      warp_before[2 * w] = l; warp_before[2 * w + 1] = e;
      l += lw; e += ew;
    }
    for (int c = 0; c < cluster; ++c) {
      if (cluster > 1) { peer_store(peer_at(counted_at + 8 * rank, c), l); peer_store(peer_at(counted_at + 8 * rank + 4, c), e); }
      else { counted[0] = l; counted[1] = e; }
    }
  }
  if (cluster > 1) cluster_meet(); else __syncthreads();      // (nobody reads another's shared memory behind this)
  uint32_t l = warp_before[2 * warp], e = warp_before[2 * warp + 1];
  for (int c = 0; c < rank; ++c) { l += counted[2 * c]; e += counted[2 * c + 1]; }
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t key = i < w1 && !all ? key_at(i) : 0u;
    const unsigned is_larger = __ballot_sync(0xffffffffu, i < w1 && (all || key > prefix)), is_equal = __ballot_sync(0xffffffffu, i < w1 && !all && key == prefix);
    const unsigned below = (1u << lane) - 1u;
    const uint32_t l_here = l + __popc(is_larger & below), e_here = e + __popc(is_equal & below);
    const bool stays = ((is_larger >> lane) & 1u) || (((is_equal >> lane) & 1u) && e_here < (uint32_t)need);
    if (stays) kept[sinks + l_here + min(e_here, (uint32_t)need)] = sinks + from + i;
    l += __popc(is_larger);
    e += __popc(is_equal);
  }
}

constexpr int kGatherThreads = 256, kGatherRows = 32;

__global__ void __launch_bounds__(kGatherThreads) paged_gather_kernel(const __grid_constant__ Evict a) {
  __shared__ long long src[kGatherRows], dst[kGatherRows];
  wait_for_grid();
  next_grid();
  const int item = a.blocks.div(blockIdx.x), block = blockIdx.x - item * a.blocks.d, b = a.heads.div(item), head = item - b * a.heads.d;
  int length;
  const int k = kept_of(a, b, length, false), r0 = block * kGatherRows, n = min(k - r0, kGatherRows);
  if (n <= 0) return;
  if ((int)threadIdx.x < n) {
    const int i = r0 + threadIdx.x, pos = a.kept[((size_t)b * a.s.heads + head) * a.kept_stride + i], from = page_of(a.s, a.bt, b, pos);
    const int to = a.to[(size_t)b * a.to_stride + (i >> a.s.page_shift)];
    const bool ok = (unsigned)to < (unsigned)a.s.n_pages;
    if (!ok) report(a.s.status);
    src[threadIdx.x] = from >= 0 && ok ? (long long)store_row(a.s, from, head, pos) : -1;
    dst[threadIdx.x] = ok ? (long long)store_row(a.s, to, head, i) : 0;
  }
  __syncthreads();
  const int both = 2 * a.row_pieces;
  for (int i = threadIdx.x; i < n * both; i += kGatherThreads) {
    const int r = i / both, c = i - r * both;
    if (src[r] < 0) continue;
    const bool v = c >= a.row_pieces;
    uint4 *rows = reinterpret_cast<uint4 *>(v ? a.s.v_rows : a.s.k_rows) + (v ? c - a.row_pieces : c);
    rows[(size_t)dst[r] * a.row_pieces] = __ldcg(rows + (size_t)src[r] * a.row_pieces);
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
  if (a.bt.n_tokens == 0 || path_len == 0) return SCALEKV_OK;
  if (!path || !counts) return fail(c, SCALEKV_ERR_INVALID_ARG, "path or counts null");
  const int layers = layer == -1 ? c->cfg.n_layers : 1;
  a.s = layer_store(c, layer == -1 ? 0 : layer);
  a.layer_rows = c->lay.rows_bytes / c->cfg.n_layers;
  a.layer_scales = c->lay.scale_bytes / c->cfg.n_layers / 4;
  a.path = path; a.counts = counts; a.path_stride = path_stride; a.path_len = path_len;
  a.q8 = c->cfg.store == SCALEKV_STORE_Q8;
  a.row_pieces = c->cfg.head_dim * (a.q8 ? 1 : 2) / 16;
  const long long columns = 2LL * c->cfg.n_kv_heads * (a.row_pieces + a.q8), blocks = (columns + kAcceptThreads - 1) / kAcceptThreads;
  if (blocks > 65535 || layers > 65535) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 65535 layers, or too many kv heads");
  launch(paged_accept_kernel, dim3((unsigned)a.bt.n_seqs, (unsigned)blocks, (unsigned)layers), kAcceptThreads, 0, static_cast<cudaStream_t>(stream), a);
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
  if (a.bt.n_seqs == 0 || kept_len == 0) return SCALEKV_OK;
  if (!a.bt.table || !a.bt.lengths || !to_table || !keep || !weights || !kept) return fail(c, SCALEKV_ERR_INVALID_ARG, "an array null");
  const int H = c->cfg.n_kv_heads;
  const long long items = (long long)a.bt.n_seqs * H, blocks = (kept_len + kGatherRows - 1) / kGatherRows;
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
  const int length = std::max(batch->max_length, 1);
  int cluster = 1;
  while (cluster < kMostCluster && items * cluster <= c->n_sm && length > cluster * 2048) cluster *= 2;
  a.held = std::min((length + cluster - 1) / cluster, kMostHeld);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = kBehindTheOneBefore;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(items * cluster)); cfg.blockDim = dim3(kChooseThreads); cfg.dynamicSmemBytes = (size_t)a.held * 4; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = 2;
  cudaLaunchKernelEx(&cfg, paged_choose_kernel, a, cluster);
  if (scalekv_status s = launched(c, "paged_choose")) return s;
  launch(paged_gather_kernel, dim3((unsigned)(items * blocks)), kGatherThreads, 0, st, a);
  return launched(c, "paged_gather");
}

}  // extern "C"
