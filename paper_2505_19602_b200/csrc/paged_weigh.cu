// What attention the entries of the paged token cache get, summed up entry by entry (see include/scalekv.h for the contract).
//
//   w_j <- (j before the new tokens ? decay w_j : 0) + sum over the rows that see j of exp(scale <q, k_j> - lse_row)
//
// A kv head's query rows, the group's heads of every new token, pay their attention to the same keys.  The rows' log-sum-exps are known, so every key's sum stands by itself: keys are
// cut over CTAs and warps at will, each is one warp's alone, and sums have one order.
#include "paged_host.cuh"

using namespace scalekv;
using namespace scalekv::paged;

namespace scalekv {
namespace paged {

struct WeighArgs {
  AttendArgs a;                                  // without outputs; a.lse is read
  float *weights;                                // [page][head][row of the page]
  float decay;
};

__device__ __forceinline__ int key_of(const Span &sp, int step) { return (step < sp.sink_steps ? step : step - sp.sink_steps + sp.lo_step) << 4; }
// Whether some row sees position pos of a step.
__device__ __forceinline__ bool some_see(const Span &sp, int pos) { return pos < sp.hi && (pos >= sp.lo || pos < sp.n_sink); }

// ---- few rows: keys stream past queries that stay in registers, as in paged_stream.cuh: products are m16n8k16 with the rows as n-tiles of eight (there is the layout).
template <int D, bool kQ8, int kN>
struct WeighLayout {
  static constexpr int kRowBytes = D * (kQ8 ? 1 : 2);
  static constexpr int kStages = kRowBytes >= 256 ? 3 : 4;
  static constexpr int kScales = 16 * kRowBytes, kOld = kScales + (kQ8 ? 64 : 0), kStage = kOld + 64;      // offsets in a stage: the keys' scales, their weights
  static constexpr int kSmem = kStreamWarps * kStages * kStage;
  static __device__ __forceinline__ int piece(int r, int x) { return StreamLayout<D, kQ8, 1>::piece(r, x); }
};
constexpr int kWeighRows = 32;                   // query rows of a sequence and kv head that go this way
constexpr int kWeighSteps = 16;                  // of a warp, in a row

template <int D, bool kQ8, int kN>
__global__ void __launch_bounds__(kStreamThreads) paged_weigh_stream_kernel(const __grid_constant__ WeighArgs w) {
  using Y = WeighLayout<D, kQ8, kN>;
  constexpr int kRowBytes = Y::kRowBytes, kStages = Y::kStages;
  extern __shared__ __align__(16) char smem[];
  const AttendArgs &a = w.a;
  const Store &s = a.s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, oct = lane >> 2, seq = blockIdx.x, head = blockIdx.y;
  wait_for_grid();
  next_grid();
  const Span sp(a, seq, 0x7fffffff, blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0);
  // a warp's stretches of kWeighSteps: stretch number z * warps + warp, and as many behind it as the grid has CTAs for
  const int stride = gridDim.z * kStreamWarps;
  if ((long long)(blockIdx.z * kStreamWarps) * kWeighSteps >= sp.steps) return;
  const int rows = min(sp.rows, 8 * kN), start = sp.start, first = sp.first, length = sp.length;
  int stretch = blockIdx.z * kStreamWarps + warp;
  // step number i of this warp; -1: there are no more
  auto step_of = [&](int i) {
    const long long at = ((long long)stretch + (long long)(i / kWeighSteps) * stride) * kWeighSteps + i % kWeighSteps;
    return at < sp.steps ? (int)at : -1;
  };
  auto page_at = [&](int step) { return step >= 0 ? page_of(s, a.bt, seq, key_of(sp, step)) : -1; };
  char *ring = smem + warp * kStages * Y::kStage;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  auto fetch = [&](int step, int page, int stage) {
    if (page >= 0) {
      constexpr int kRowPieces = kRowBytes / 16, kRowsAtOnce = 32 / kRowPieces;
      const int key0 = key_of(sp, step), x = lane % kRowPieces, r0 = lane / kRowPieces;
      const size_t row = store_row(s, page, head, key0);
      const uint32_t to = ring_at + stage * Y::kStage;
      const char *k = s.k_rows + (row + r0) * kRowBytes + x * 16;
#pragma unroll
      for (int i = 0; i < 16 / kRowsAtOnce; ++i) copy16(to + Y::piece(r0 + i * kRowsAtOnce, x), k + i * kRowsAtOnce * kRowBytes, true);
      if (kQ8 && lane < 4) copy16(to + Y::kScales + lane * 16, s.k_scales + row + lane * 4, true);
      if (lane >= 28) copy16(to + Y::kOld + (lane & 3) * 16, w.weights + row + (lane & 3) * 4, true);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int steps[kStages], pages[kStages];
#pragma unroll
  for (int i = 0; i < kStages; ++i) { steps[i] = step_of(i); pages[i] = page_at(steps[i]); }
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(steps[i], pages[i], i);

  uint2 q[kN][D / 16];
  float lse[kN][2];                              // of rows 2 quad, 2 quad + 1 of every n-tile, in base 2; +inf: the row counts for nothing
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    int t, h;
    const int r = n * 8 + oct;
    place_row(a, start, head, min(r, rows - 1), t, h);
    const char *row = a.Q.ptr + t * a.Q.st + h * a.Q.sh;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int dim = kQ8 ? (k >> 2) * 64 + quad * 16 + (k & 3) * 4 : (k >> 1) * 32 + quad * 8 + (k & 1) * 4;
      q[n][k] = r < rows ? *reinterpret_cast<const uint2 *>(row + dim * 2) : make_uint2(0u, 0u);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = n * 8 + 2 * quad + e;
      place_row(a, start, head, min(i, rows - 1), t, h);
      const float x = a.lse[(size_t)t * a.n_heads + h] * kLog2e;
      lse[n][e] = i < rows && x != -INFINITY ? x : INFINITY;
    }
  }
  // a step all of whose keys every row sees: [lo_full, hi_full)
  const int lo_full = seen_lo(a.mask, first + a.group.div(rows - 1)), hi_full = seen_hi(a.mask, first, length);

  for (int i = 0, stage = 0; steps[0] >= 0; ++i) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();
    fetch(steps[kStages - 1], pages[kStages - 1], stage == 0 ? kStages - 1 : stage - 1);
    const int key0 = key_of(sp, steps[0]), page = pages[0];
#pragma unroll
    for (int k = 0; k + 1 < kStages; ++k) { steps[k] = steps[k + 1]; pages[k] = pages[k + 1]; }
    steps[kStages - 1] = step_of(i + kStages);
    pages[kStages - 1] = page_at(steps[kStages - 1]);
    const char *k_at = ring + stage * Y::kStage;
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (page < 0) continue;
    float sum[2] = {0.f, 0.f};                   // of keys oct and oct + 8, over this lane's rows
    float x[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll
    for (int c = 0; c < kRowBytes / 64; ++c) {
      const uint4 lo = *reinterpret_cast<const uint4 *>(k_at + Y::piece(oct, c * 4 + quad)), hi = *reinterpret_cast<const uint4 *>(k_at + Y::piece(oct + 8, c * 4 + quad));
      if constexpr (kQ8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w0 = turn_signs(word(lo, e)), w1 = turn_signs(word(hi, e));
          const uint32_t f[4] = {codes_low(w0), codes_low(w1), codes_high(w0), codes_high(w1)};
#pragma unroll
          for (int n = 0; n < kN; ++n) mma_16816(x[n], f, q[n][4 * c + e].x, q[n][4 * c + e].y);
        }
      } else {
        const uint32_t f0[4] = {lo.x, hi.x, lo.y, hi.y}, f1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          mma_16816(x[n], f0, q[n][2 * c].x, q[n][2 * c].y);
          mma_16816(x[n], f1, q[n][2 * c + 1].x, q[n][2 * c + 1].y);
        }
      }
    }
    float ks0 = a.scale_log2e, ks1 = a.scale_log2e;
    if constexpr (kQ8) {
      const float *scales = reinterpret_cast<const float *>(k_at + Y::kScales) + oct;
      ks0 *= kCodeUnit * scales[0];
      ks1 *= kCodeUnit * scales[8];
    }
    const bool whole = key0 >= lo_full && key0 + 16 <= hi_full;
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float p = tc::ex2(x[n][e] * (e < 2 ? ks0 : ks1) - lse[n][e & 1]);
        if (lse[n][e & 1] == INFINITY) p = 0.f;                   // (whatever the product is)
        if (!whole) {
          const int r = first + a.group.div(min(n * 8 + 2 * quad + (e & 1), rows - 1)), pos = key0 + oct + 8 * (e >> 1);
          if (pos >= seen_hi(a.mask, r, length) || (pos < seen_lo(a.mask, r) && pos >= sp.n_sink)) p = 0.f;
        }
        sum[e >> 1] += p;
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
      sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
    }
    if (quad < 2) {
      const int pos = key0 + oct + 8 * quad;
      const float old = reinterpret_cast<const float *>(k_at + Y::kOld)[oct + 8 * quad];
      if (some_see(sp, pos)) w.weights[store_row(s, page, head, pos)] = (pos < first ? w.decay * old : 0.f) + sum[quad];
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// ---- many rows: a warp's 16 keys stay in registers, queries pass through shared memory, 64 rows at a time.
constexpr int kQueryRows = 64, kManyWarps = 8;

template <int D, bool kQ8>
__global__ void __launch_bounds__(32 * kManyWarps) paged_weigh_kernel(const __grid_constant__ WeighArgs w) {
  __shared__ __align__(16) uint2 q_smem[kQueryRows * D / 4 + kQueryRows];
  __shared__ float lse_smem[kQueryRows];
  const AttendArgs &a = w.a;
  const Store &s = a.s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, oct = lane >> 2, seq = blockIdx.x, head = blockIdx.y;
  constexpr int kPitch = D * 2 + 8;              // bytes of a row of queries
  wait_for_grid();
  next_grid();
  const Span sp(a, seq, 0x7fffffff, blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0);
  const int rows = sp.rows, start = sp.start, first = sp.first, length = sp.length;
  for (int step0 = blockIdx.z * kManyWarps; step0 < sp.steps; step0 += gridDim.z * kManyWarps) {
    const int step = step0 + warp, key0 = step < sp.steps ? key_of(sp, step) : 0, page = step < sp.steps ? page_of(s, a.bt, seq, key0) : -1;
    const bool on = page >= 0;
    uint32_t k[D / 16][4];
    float ks[2] = {a.scale_log2e, a.scale_log2e};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const size_t row = store_row(s, max(page, 0), head, key0 + oct + 8 * e);
      if constexpr (kQ8) {
        if (on) ks[e] *= kCodeUnit * s.k_scales[row];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          uint4 x = on ? *reinterpret_cast<const uint4 *>(s.k_rows + row * D + (c * 4 + quad) * 16) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t u = turn_signs(word(x, i));
            k[4 * c + i][e] = codes_low(u);
            k[4 * c + i][2 + e] = codes_high(u);
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint4 x = on ? *reinterpret_cast<const uint4 *>(s.k_rows + row * D * 2 + (c * 4 + quad) * 16) : make_uint4(0u, 0u, 0u, 0u);
          k[2 * c][e] = x.x; k[2 * c][2 + e] = x.y;
          k[2 * c + 1][e] = x.z; k[2 * c + 1][2 + e] = x.w;
        }
      }
    }
    float sum[2] = {0.f, 0.f};
    for (int r0 = 0; r0 < rows; r0 += kQueryRows) {
      __syncthreads();
      for (int i = threadIdx.x; i < kQueryRows * D / 4; i += 32 * kManyWarps) {
        const int r = i / (D / 4), x = i % (D / 4);
        int t, h;
        place_row(a, start, head, min(r0 + r, rows - 1), t, h);
        *reinterpret_cast<uint2 *>(reinterpret_cast<char *>(q_smem) + r * kPitch + x * 8) = *reinterpret_cast<const uint2 *>(a.Q.ptr + t * a.Q.st + h * a.Q.sh + x * 8);
        if (x == 0) {
          const float l = a.lse[(size_t)t * a.n_heads + h] * kLog2e;
          lse_smem[r] = r0 + r < rows && l != -INFINITY ? l : INFINITY;
        }
      }
      __syncthreads();
      if (!on) continue;
#pragma unroll 1
      for (int n = 0; n < kQueryRows; n += 8) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        const char *row = reinterpret_cast<const char *>(q_smem) + (n + oct) * kPitch;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const int dim = kQ8 ? (i >> 2) * 64 + quad * 16 + (i & 3) * 4 : (i >> 1) * 32 + quad * 8 + (i & 1) * 4;
          const uint2 b = *reinterpret_cast<const uint2 *>(row + dim * 2);
          mma_16816(x, k[i], b.x, b.y);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l = lse_smem[n + 2 * quad + (e & 1)];
          const int i = r0 + n + 2 * quad + (e & 1), t = first + a.group.div(min(i, rows - 1)), pos = key0 + oct + 8 * (e >> 1);
          float p = tc::ex2(x[e] * ks[e >> 1] - l);
          if (l == INFINITY || pos >= seen_hi(a.mask, t, length) || (pos < seen_lo(a.mask, t) && pos >= sp.n_sink)) p = 0.f;
          sum[e >> 1] += p;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
      sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
    }
    if (quad < 2 && on) {
      const int pos = key0 + oct + 8 * quad;
      if (some_see(sp, pos)) {
        float *at = w.weights + store_row(s, page, head, pos);
        *at = (pos < first ? w.decay * *at : 0.f) + sum[quad];
      }
    }
  }
}

template <int D, bool kQ8>
bool room() {
  auto ask = [](auto kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess; };
  return ask(paged_weigh_stream_kernel<D, kQ8, 1>, WeighLayout<D, kQ8, 1>::kSmem) && ask(paged_weigh_stream_kernel<D, kQ8, 2>, WeighLayout<D, kQ8, 2>::kSmem) &&
         ask(paged_weigh_stream_kernel<D, kQ8, 4>, WeighLayout<D, kQ8, 4>::kSmem);
}

}  // namespace paged
}  // namespace scalekv

bool scalekv::paged::room_for_weigh(int head_dim, bool q8) {
  if (head_dim == 128) return q8 ? room<128, true>() : room<128, false>();
  return q8 ? room<64, true>() : room<64, false>();
}

extern "C" scalekv_status scalekv_paged_weigh(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, int32_t n_heads, scalekv_rows Q, const float *lse,
                                              const scalekv_paged_mask *mask, float softmax_scale, float *weights, float decay, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_weigh");
  WeighArgs w;
  AttendArgs &a = w.a;
  if (scalekv_status st = check_batch(c, layer, batch, a.bt)) return st;
  if (scalekv_status st = check_heads(c, n_heads, softmax_scale)) return st;
  if (!mask || mask->window < 0 || mask->n_sink < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "mask null, or a negative size in it");
  if (!(decay >= 0.f && decay <= 1.f)) return fail(c, SCALEKV_ERR_INVALID_ARG, "decay must lie in [0, 1]");
  if (a.bt.n_tokens == 0) return SCALEKV_OK;
  if (!rows_ok(Q, 2) || !lse || !weights || (reinterpret_cast<uintptr_t>(weights) & 15))
    return fail(c, SCALEKV_ERR_INVALID_ARG, "Q, lse or weights null, or not 16-byte aligned");
  const int H = c->cfg.n_kv_heads, D = c->cfg.head_dim, G = n_heads / H;
  if ((long long)a.bt.n_tokens * n_heads > kMaxLength) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 2^30 query rows in a call");
  if (H > 32767) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 32767 kv heads");
  a.s = layer_store(c, layer);
  a.Q = view(Q, 2);
  a.O = {};
  a.lse = const_cast<float *>(lse);
  a.part_o = a.part_ml = nullptr;
  a.counts = nullptr;
  a.tree = nullptr;
  a.tree_words = 0;
  a.mask = {mask->causal != 0, std::min(mask->window, kMaxLength), mask->n_sink};
  a.group = Divisor::of(G);
  a.n_heads = n_heads;
  a.max_new = batch->max_new;
  a.scale_log2e = (softmax_scale > 0.f ? softmax_scale : 1.f / std::sqrt((float)D)) * kLog2e;
  w.weights = weights;
  w.decay = decay;
  const long long max_rows = (long long)std::min(batch->max_new, a.bt.n_tokens) * G;      // query rows of a sequence and kv head
  long long keys = std::max(batch->max_length, 1);
  if (a.mask.window > 0) keys = std::min<long long>(keys, (long long)a.mask.window + batch->max_new + a.mask.n_sink + 32);
  const int steps = (int)((keys + 15) / 16);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto dim, auto codes) {
    constexpr int kD = decltype(dim)::value;
    constexpr bool kQ8 = decltype(codes)::value;
    if (max_rows <= kWeighRows) {
      const dim3 grid(a.bt.n_seqs, H, (unsigned)std::min(65535, (steps + kStreamWarps * kWeighSteps - 1) / (kStreamWarps * kWeighSteps)));
      if (max_rows <= 8) launch(paged_weigh_stream_kernel<kD, kQ8, 1>, grid, kStreamThreads, WeighLayout<kD, kQ8, 1>::kSmem, st, w);
      else if (max_rows <= 16) launch(paged_weigh_stream_kernel<kD, kQ8, 2>, grid, kStreamThreads, WeighLayout<kD, kQ8, 2>::kSmem, st, w);
      else launch(paged_weigh_stream_kernel<kD, kQ8, 4>, grid, kStreamThreads, WeighLayout<kD, kQ8, 4>::kSmem, st, w);
    } else {
      const dim3 grid(a.bt.n_seqs, H, (unsigned)std::min(65535, (steps + kManyWarps - 1) / kManyWarps));
      launch(paged_weigh_kernel<kD, kQ8>, grid, 32 * kManyWarps, 0, st, w);
    }
    return launched(c, "paged_weigh");
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  const bool q8 = c->cfg.store == SCALEKV_STORE_Q8;
  if (D == 128) return q8 ? go(D128{}, std::true_type{}) : go(D128{}, std::false_type{});
  return q8 ? go(D64{}, std::true_type{}) : go(D64{}, std::false_type{});
}
