// What attention the entries of the paged token cache get, summed up entry by entry (see include/scalekv.h for the contract).
//
//   w_j <- (j before the new tokens ? decay w_j : 0) + sum over the rows that see j of exp(scale <q, k_j> - lse_row)      for every j that some row sees,
//   w_j <- decay w_j                                                                                                     for those that a window hides from all of them, in a call of its own.
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
  double scale_log2e;                            // the factor of an exponent: a key's has it, and its scale, rounded once
};

constexpr double kLog2eExact = 1.4426950408889634074;

__device__ __forceinline__ int key_of(const Span &sp, int step) { return (step < sp.sink_steps ? step : step - sp.sink_steps + sp.lo_step) << 4; }
// Whether some row sees position pos of a step.
__device__ __forceinline__ bool some_see(const Span &sp, int pos) { return pos < sp.hi && (pos >= sp.lo || pos < sp.n_sink); }

// ---- few rows: keys stream past queries that stay in registers, as in paged_stream.cuh: products are m16n8k16 with the rows as n-tiles of eight (there is the layout).  A warp takes stretches of
// eight steps of 16 keys, whose pages it looks up at once, a lane to each.  What bounds it: reading K and the sums once, and with codes the instructions that turn them into bf16.  us, 32 sequences of up to 10 521
// entries, 32 heads on 8 of 128: codes 59.3 (4.5 TB/s; 72 of 100 issue slots; with one sum for all products 57.5, then stretches of 16 / 32 steps 61 / 69, pages looked up step by step 63), bf16 85 (5.9 TB/s).
template <int D, bool kQ8, int kN>
struct WeighLayout {
  static constexpr int kRowBytes = D * (kQ8 ? 1 : 2);
  static constexpr int kStages = 3;              // (codes of 128: four take 61.4 us where three take 60.0)
  static constexpr int kScales = 16 * kRowBytes, kOld = kScales + (kQ8 ? 64 : 0), kStage = kOld + 64;      // offsets in a stage: the keys' scales, their weights
  static constexpr int kSmem = kStreamWarps * kStages * kStage;
  static __device__ __forceinline__ int piece(int r, int x) { return StreamLayout<D, kQ8, 1>::piece(r, x); }
};
// Query rows of a sequence and kv head that go this way.  (us, four sequences of 8 192 entries, 8 heads of 128 in codes, with one event's 5: 64 rows in two such launches 51, on tcgen05 40; one of 2 000 entries 25 and 15; 53 sequences
// of 70 entries, 16 heads, 66 rows in three 71 and 36.)
constexpr int kWeighRows = 32;
constexpr int kWeighSteps = 8;                   // of a warp, in a row

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
  const int stride = gridDim.z * kStreamWarps;   // a warp's stretches of kWeighSteps: number z * warps + warp, and those a grid further
  if (blockIdx.z * kStreamWarps * kWeighSteps >= sp.steps) return;
  const int rows = min(sp.rows, 8 * kN), start = sp.start, first = sp.first, length = sp.length;
  char *ring = smem + warp * kStages * Y::kStage;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);

  // What fills the tile up is the last row once more, with a log-sum-exp of kNever: whatever a key holds, its power is 0 or what that row's own is, infinite or no number.  (Of zeros an infinite key would make NaN.)
  constexpr float kNever = FLT_MAX;
  uint2 q[kN][D / 16];
  // of rows 2 quad, 2 quad + 1 of every n-tile, in base 2, and what the rounding leaves of it; kNever: the row counts for nothing.  (An exponent of 20 in one float is off by 2^-21, and so is its power of two:
  // with log-sum-exps and factors in two floats a sum's relative error, one heavy key's mostly, was 2e-7 where it was 1.7e-6.)
  float lse[kN][2], lse_rest[kN][2];
  bool nothing = false;                          // some row counts for nothing
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    int t, h;
    const int r = n * 8 + oct;
    place_row(a, start, head, min(r, rows - 1), t, h);
    const char *row = a.Q.ptr + t * a.Q.st + h * a.Q.sh;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int dim = kQ8 ? (k >> 2) * 64 + quad * 16 + (k & 3) * 4 : (k >> 1) * 32 + quad * 8 + (k & 1) * 4;
      q[n][k] = *reinterpret_cast<const uint2 *>(row + dim * 2);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = n * 8 + 2 * quad + e;
      place_row(a, start, head, min(i, rows - 1), t, h);
      const float l = a.lse[(size_t)t * a.n_heads + h], x = (float)((double)l * kLog2eExact);
      const bool never = i >= rows || fabsf(x) == INFINITY;
      lse[n][e] = never ? kNever : x;
      lse_rest[n][e] = never ? 0.f : (float)((double)l * kLog2eExact - (double)x);
      nothing = nothing || (i < rows && never);
    }
  }
  nothing = __any_sync(0xffffffffu, nothing);
  // (the factor's parts have one sign: an infinite product stays what it is in both)
  const float scale_hi = __double2float_rd(w.scale_log2e), scale_lo = fmaxf((float)(w.scale_log2e - (double)scale_hi), FLT_TRUE_MIN);
  // a step all of whose keys every row sees: [lo_full, hi_full)
  const int lo_full = seen_lo(a.mask, first + a.group.div(rows - 1)), hi_full = seen_hi(a.mask, first, length);

  for (int stretch = blockIdx.z * kStreamWarps + warp; stretch < (sp.steps + kWeighSteps - 1) / kWeighSteps; stretch += stride) {
    const int step0 = stretch * kWeighSteps, n_steps = min(kWeighSteps, sp.steps - step0);
    // a lane for each step's page
    static_assert(kWeighSteps <= 32, "a lane for each step");
    const int own_page = lane < n_steps ? page_of(s, a.bt, seq, key_of(sp, step0 + lane)) : -1;
    auto fetch = [&](int i, int stage) {
      if (i < n_steps) {
        const int page = __shfl_sync(0xffffffffu, own_page, i);
        if (page >= 0) {
          constexpr int kRowPieces = kRowBytes / 16, kRowsAtOnce = 32 / kRowPieces;
          const int x = lane % kRowPieces, r0 = lane / kRowPieces;
          const size_t row = store_row(s, page, head, key_of(sp, step0 + i));
          const uint32_t to = ring_at + stage * Y::kStage;
          const char *k = s.k_rows + (row + r0) * kRowBytes + x * 16;
#pragma unroll
          for (int j = 0; j < 16 / kRowsAtOnce; ++j) copy16(to + Y::piece(r0 + j * kRowsAtOnce, x), k + j * kRowsAtOnce * kRowBytes, true);
          // (the scales by lanes 0-3, the weights by lanes 4-7)
          if (lane < 8 && (kQ8 || lane >= 4)) copy16(to + (lane < 4 ? Y::kScales : Y::kOld) + (lane & 3) * 16, (lane < 4 ? s.k_scales : w.weights) + row + (lane & 3) * 4, true);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i, i);
    auto one = [&](int i, int stage) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      __syncwarp();
      fetch(i + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
      const int key0 = key_of(sp, step0 + i), page = __shfl_sync(0xffffffffu, own_page, i);
      if (page < 0) return;
      const char *k_at = ring + stage * Y::kStage;
      float x[kN][4];
#pragma unroll
      for (int n = 0; n < kN; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
      // (Products of two steps are summed by themselves: of a step's 16 products and the sum so far the tensor core cuts each at 2^-25 of the largest, and the result at 2^-23 of itself (measured), 1.25 x 2^-21 at most; an exponent's error
      // is a relative one of its power.  A sum that one key dominates is off by 2.5e-6 with a single sum, by 7e-7 so; at worst 8 steps in one sum make 80 x 2^-24, four sums of two and their three additions 23 x 2^-24.)
      float y[kN][4];
      auto fresh = [&]() {
#pragma unroll
        for (int n = 0; n < kN; ++n) y[n][0] = y[n][1] = y[n][2] = y[n][3] = 0.f;
      };
      auto gather = [&]() {
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n][e] += y[n][e];
      };
#pragma unroll
      for (int c = 0; c < kRowBytes / 64; ++c) {
        const uint4 lo = *reinterpret_cast<const uint4 *>(k_at + Y::piece(oct, c * 4 + quad)), hi = *reinterpret_cast<const uint4 *>(k_at + Y::piece(oct + 8, c * 4 + quad));
        if constexpr (kQ8) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w0 = turn_signs(word(lo, e)), w1 = turn_signs(word(hi, e));
            const uint32_t f[4] = {codes_low(w0), codes_low(w1), codes_high(w0), codes_high(w1)};
            if (!(e & 1)) fresh();
#pragma unroll
            for (int n = 0; n < kN; ++n) mma_16816(y[n], f, q[n][4 * c + e].x, q[n][4 * c + e].y);
            if (e & 1) gather();
          }
        } else {
          const uint32_t f0[4] = {lo.x, hi.x, lo.y, hi.y}, f1[4] = {lo.z, hi.z, lo.w, hi.w};
          fresh();
#pragma unroll
          for (int n = 0; n < kN; ++n) {
            mma_16816(y[n], f0, q[n][2 * c].x, q[n][2 * c].y);
            mma_16816(y[n], f1, q[n][2 * c + 1].x, q[n][2 * c + 1].y);
          }
          gather();
        }
      }
      float ks[2] = {scale_hi, scale_hi}, ks_rest[2] = {scale_lo, scale_lo};
      if constexpr (kQ8) {
        const float *scales = reinterpret_cast<const float *>(k_at + Y::kScales) + oct;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float s = kCodeUnit * scales[8 * e];
          ks[e] = __fmul_rd(scale_hi, s);
          ks_rest[e] = fmaf(scale_lo, s, fmaf(scale_hi, s, -ks[e]));
        }
      }
      float sum[2] = {0.f, 0.f};                 // of keys oct and oct + 8, over this lane's rows
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = tc::ex2(fmaf(x[n][e], ks[e >> 1], -lse[n][e & 1]) + fmaf(x[n][e], ks_rest[e >> 1], -lse_rest[n][e & 1]));
      const bool whole = key0 >= lo_full && key0 + 16 <= hi_full;
      if (!whole || nothing) {
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = first + a.group.div(min(n * 8 + 2 * quad + (e & 1), rows - 1)), pos = key0 + oct + 8 * (e >> 1);
            if (lse[n][e & 1] == kNever || pos >= seen_hi(a.mask, r, length) || (pos < seen_lo(a.mask, r) && pos >= sp.n_sink)) x[n][e] = 0.f;      // (whatever the product is)
          }
      }
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e >> 1] += x[n][e];
      // lanes of even quads put the first key's sum together, those of odd quads the second's
      const float give = quad & 1 ? sum[0] : sum[1], keep = quad & 1 ? sum[1] : sum[0];
      float all = keep + __shfl_xor_sync(0xffffffffu, give, 1);
      all += __shfl_xor_sync(0xffffffffu, all, 2);
      if (quad < 2) {
        const int pos = key0 + oct + 8 * quad;
        const float old = reinterpret_cast<const float *>(k_at + Y::kOld)[oct + 8 * quad];
        if (whole || some_see(sp, pos)) w.weights[store_row(s, page, head, pos)] = (pos < first ? w.decay * old : 0.f) + all;
      }
    };
#pragma unroll 1
    for (int i = 0; i < n_steps; i += kStages) {
#pragma unroll
      for (int j = 0; j < kStages; ++j)
        if (i + j < n_steps) one(i + j, j);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();                                // (the ring is free)
  }
}

// ---- many rows: products on tcgen05 with the keys for rows, so that a key's sum is a thread's own.
//
// An item is 256 keys of a sequence and kv head, two tiles A and B of 128, whose rows lie in TMEM as the products' first operand for as long as queries pass: read from shared memory for every
// product they took as much of its data path as the queries.  Query rows come 128 at a time through a ring in shared memory.  S^T = K Q^T is formed in units of 64 query rows, A's and B's
// side by side, in three buffers that go round; units go to two pairs of softmax warpgroups in turn, half of a unit's columns to a warpgroup, a thread to each key of A and the same of B: a row's
// log-sum-exp, which is a column's here, is loaded once for both.  A CTA takes items one after the other, as many as there are CTAs apart.
//   warp 0        : tcgen05.mma issuer
//   warp 1        : finds the items, ahead of the others
//   warps 4-7     : the queries, by asynchronous copies of 16 bytes (rows are a token's heads, in any strides), and their log-sum-exps; the next item's keys, scales and weights
//   warps 8-23    : keys from shared memory into TMEM (codes become bf16 exactly), then p = 2^(x ks - lse) and its sums
// Every wait is bounded, as in paged_tile.cuh.  A product's sum is the tensor core's, with its cut-off at each of D / 16 steps (see above): 2.5e-6 of a sum that one key of four times the others' length dominates.
// What bounds it: exponentials, of which the special function unit does 16 a cycle (a tile of 128 x 128 takes it twice as long as the tensor core its product; it is busy for 80 of 100 cycles while a
// CTA has work), and the power that both draw: 2 048 queries of 4 x 32 heads behind 6 144 entries in codes take 577 us from a cool start, 0.83 PFLOP/s, and 596 to 615 in a row.  (One exponential in
// four by a polynomial on the FMA pipe: 555 us from a cool start, 597 in a row; half of them 658.  A key tile's rows in shared memory and eight softmax warps: 715; products issued one by one: 621; a CTA for
// each block of keys, its rows fetched when it begins: 600.  16 columns at a time, the next ones on their way: 643.)
constexpr int kKeyRows = 256, kQueryTile = 128, kUnit = 64, kUnits = 3, kSumGroups = 4, kItems = 3;

template <int D, bool kQ8>
struct WeighTile {
  static constexpr int kThreads = 256 + 128 * kSumGroups;
  static constexpr int kRegs0 = 40, kRegs1 = 56, kRegsS = 96;
  static_assert(kRegs0 + kRegs1 + kSumGroups * kRegsS <= 80 * 6, "a share would wait for registers that nobody returns");
  static constexpr int kStages = 4, kSlots = 2 * kStages;      // of queries; of their log-sum-exps: a stage is free when its products are through, whose sums may still be under way
  static constexpr int kRowBytes = D * (kQ8 ? 1 : 2), kPitch = kRowBytes + 16;      // of keys as they are held (a thread reads a row of its own: eight of them meet all banks)
  static constexpr uint32_t kTile = kQueryTile * D * 2, kHalf = kQueryTile * 128;
  static constexpr uint32_t kOffLse = kStages * kTile, kOffVoid = kOffLse + kSlots * kQueryTile * 4, kOffKeys = kOffVoid + kSlots * 16;
  static constexpr uint32_t kOffScale = kOffKeys + kKeyRows * kPitch, kOffOld = kOffScale + kKeyRows * 4, kOffRow = kOffOld + kKeyRows * 4;      // and of every key: scale, weight, row
  static constexpr uint32_t kOffSum = kOffRow + kKeyRows * 8;  // sums of the other warpgroups, for the first
  static constexpr uint32_t kOffItem = kOffSum + (kSumGroups - 1) * kKeyRows * 4;
  static constexpr uint32_t kOffBar = kOffItem + kItems * 64;
  enum { bQFull = 0, bQEmpty = bQFull + kStages, bSFull = bQEmpty + kStages, bSFree = bSFull + kUnits, bKeys = bSFree + kUnits, bRaw, bRawFree, bItem, bItemFree = bItem + kItems,
         bCount = bItemFree + kItems };
  static_assert(bCount <= 32, "one lane of a warp initialises each barrier");
  static constexpr uint32_t kOffWord = kOffBar + 8 * bCount;   // TMEM address, abort flag
  static constexpr uint32_t kSmem = kOffWord + 16;
  static_assert(kSmem <= 232448, "more shared memory than a CTA can have");
  static_assert(kOffBar % 8 == 0 && kOffRow % 8 == 0 && kOffKeys % 16 == 0 && kOffItem % 16 == 0, "alignment");
};

// Whether all threads of the softmax warpgroups bring true.  A named barrier, which knows no limit: whoever has given up comes, too, and all of them hear of it.
__device__ __forceinline__ bool all_agree(bool mine) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 3, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(mine ? 1u : 0u), "n"(128 * kSumGroups)
      : "memory");
  return all != 0;
}

// D/16 steps of a product, by one thread: A in TMEM (16 dims = 8 columns a step), B in shared memory, K-major (32 bytes a step inside a half of 64 dims).
template <int D> __device__ __forceinline__ void mma_ts_k(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc) {
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem + 8 * k), "r"(b_lo + (uint32_t)((k >> 2) * 1024 + (k & 3) * 2)), "r"(hi), "r"(idesc), "r"(k > 0 ? 1u : 0u)
        : "memory");
}

// What an item is: key0 < 0: there are no more.
struct KeyItem {
  int seq, head, key0, tile0, tiles;             // the tiles of 128 rows that see some of its keys
  int start, rows, length, first, n_sink, lo, hi;
};

template <int D, bool kQ8>
__global__ void __launch_bounds__(WeighTile<D, kQ8>::kThreads, 1) paged_weigh_tile_kernel(const __grid_constant__ WeighArgs w) {
  using Y = WeighTile<D, kQ8>;
  constexpr int kStages = Y::kStages;
  constexpr uint32_t kTile = Y::kTile, kHalf = Y::kHalf, kColK = kUnits * 2 * kUnit;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  auto bar = [&](int i) { return base + Y::kOffBar + 8u * (uint32_t)i; };
  volatile int *words = reinterpret_cast<volatile int *>(smem_raw + Y::kOffWord);
  volatile int *abort_flag = words + 1;
  const AttendArgs &a = w.a;
  const Store &s = a.s;
  int *status = s.status;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x & 127, G = a.group.d;
  if (warp == 1) {
    if (lane < Y::bCount) {
      // arrivals a phase: one lane of every warp that hands something over, or a commit
      const uint32_t readers = 1 + 4 + 4 * kSumGroups;         // of an item
      mbar_init(bar(lane), lane < Y::bQEmpty ? 4u : lane < Y::bSFree ? 1u : lane < Y::bKeys ? 8u : lane < Y::bRaw ? 4u * kSumGroups : lane < Y::bRawFree ? 4u : lane < Y::bItem ? 4u * kSumGroups
                           : lane < Y::bItemFree ? 1u : readers);
    }
    if (lane == 0) words[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + Y::kOffWord), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  wait_for_grid();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)words[0];
  // Item number k of this CTA, as warp 1 has left it.
  auto read_item = [&](int k, KeyItem &it) {
    const bool there = mbar_wait_warp(bar(Y::bItem + k % kItems), (k / kItems) & 1, abort_flag, status);
    const volatile int *v = reinterpret_cast<const volatile int *>(smem_raw + Y::kOffItem + (k % kItems) * 64);
    it = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], v[10], v[11]};
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(Y::bItemFree + k % kItems));
    return there && it.key0 >= 0;
  };

  if (warp < 4) {
    registers_down<Y::kRegs0>();
    if (warp == 0) {
      constexpr uint32_t idesc = tile_desc(false, kUnit), dhi = desc_hi(1024);
      const bool leader = elect_one();
      int q = 0, u = 0;                          // query tiles and units so far
      uint32_t latest = 0, latest_parity = 0;      // barrier and phase of the commit that stands behind all products so far
      KeyItem it;
      bool ok = true;
      for (int n = 0; ok && read_item(n, it); ++n) {
        ok = mbar_wait_warp(bar(Y::bKeys), n & 1, abort_flag, status);
        if (!ok) break;
        tc_fence_after();
        for (int j = 0; j < it.tiles && ok; ++j, ++q) {
          ok = mbar_wait_warp(bar(Y::bQFull + q % kStages), (q / kStages) & 1, abort_flag, status);
          if (!ok) break;
          const uint32_t qd = desc_lo(base + (q % kStages) * kTile, 16);
#pragma unroll 1
          for (int h = 0; h < 2; ++h, ++u) {
            const int buf = u % kUnits;
            ok = mbar_wait_warp(bar(Y::bSFree + buf), ((u / kUnits) & 1) ^ 1, abort_flag, status);
            if (!ok) break;
            tc_fence_after();
            if (leader) {
#pragma unroll
              for (int t = 0; t < 2; ++t) mma_ts_k<D>(tmem + buf * 2 * kUnit + t * kUnit, tmem + kColK + t * (D / 2), qd + h * (kUnit * 128 / 16), dhi, idesc);
              tc_commit(bar(Y::bSFull + buf));
              if (h == 1) tc_commit(bar(Y::bQEmpty + q % kStages));
            }
            latest = bar(Y::bSFull + buf);
            latest_parity = (u / kUnits) & 1;
            __syncwarp();
          }
        }
      }
      next_grid();
      // (whoever has given up: no product may be under way when TMEM is freed and the tiles that it reads are gone)
      if (latest) drain(latest, latest_parity);
    } else if (warp == 1) {
      // Items are counted through the sequences, and in one through the blocks of 256 keys that some row sees, the sinks' and those of [lo, hi), all heads of a block together.
      const bool dead = (base & 1023u) || *reinterpret_cast<volatile int *>(status) == kDevTimeout;      // (an earlier CTA gave up: do not pile on)
      if ((base & 1023u) && lane == 0) report(status);
      auto blocks_of = [&](const Span &sp, int &lo_block, int &sink_blocks) {
        lo_block = sp.lo >> 8;
        sink_blocks = min((min(sp.n_sink, sp.hi) + 255) >> 8, lo_block);
        return sp.rows > 0 ? sink_blocks + max((sp.hi + 255) >> 8, lo_block) - lo_block : 0;
      };
      bool ok = true;
      long long before = 0, want = blockIdx.x;   // items ahead of sequence b0; the one that is looked for
      int n = 0;
      for (int b0 = 0; b0 < a.bt.n_seqs && ok && !dead; b0 += 32) {
        int blocks = 0, lo_block, sink_blocks;
        if (b0 + lane < a.bt.n_seqs) {
          const Span sp(a, b0 + lane, 0x7fffffff, blockIdx.x == 0);
          blocks = blocks_of(sp, lo_block, sink_blocks);
        }
        long long incl = (long long)blocks * s.heads;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const long long up = __shfl_up_sync(0xffffffffu, incl, d);
          if (lane >= d) incl += up;
        }
        const long long all = __shfl_sync(0xffffffffu, incl, 31);
        while (ok && want < before + all) {
          const int src = __ffs(__ballot_sync(0xffffffffu, before + incl > want)) - 1;
          const long long i = want - before - __shfl_sync(0xffffffffu, incl - (long long)blocks * s.heads, src);
          const int block = (int)(i / s.heads);
          const Span sp(a, b0 + src, 0x7fffffff, false);
          blocks_of(sp, lo_block, sink_blocks);
          const int key0 = (block < sink_blocks ? block : block - sink_blocks + lo_block) << 8, last = (key0 < sp.n_sink ? key0 : min(key0 + kKeyRows, sp.length) - 1);
          // the rows that see key0, and those that see the last key: [.., end)
          const int begin = a.mask.causal ? (int)min((long long)sp.rows, (long long)max(key0 - sp.first, 0) * G) : 0;
          const int end = a.mask.window > 0 && last >= sp.n_sink ? (int)min((long long)sp.rows, max((long long)last - sp.first + a.mask.window, 0ll) * G) : sp.rows;
          const int tile0 = begin / kQueryTile, tiles = (end + kQueryTile - 1) / kQueryTile - tile0;
          if (tiles > 0) {
            ok = mbar_wait_warp(bar(Y::bItemFree + n % kItems), ((n / kItems) & 1) ^ 1, abort_flag, status);
            if (lane == 0 && ok) {
              volatile int *v = reinterpret_cast<volatile int *>(smem_raw + Y::kOffItem + (n % kItems) * 64);
              v[0] = b0 + src; v[1] = (int)(i - (long long)block * s.heads); v[2] = key0; v[3] = tile0; v[4] = tiles; v[5] = sp.start; v[6] = sp.rows;
              v[7] = sp.length; v[8] = sp.first; v[9] = sp.n_sink; v[10] = sp.lo; v[11] = sp.hi;
              mbar_arrive(bar(Y::bItem + n % kItems));
            }
            ++n;
          }
          want += gridDim.x;
          __syncwarp();
        }
        before += all;
      }
      if (ok) ok = mbar_wait_warp(bar(Y::bItemFree + n % kItems), ((n / kItems) & 1) ^ 1, abort_flag, status);
      if (lane == 0 && ok) {
        volatile int *v = reinterpret_cast<volatile int *>(smem_raw + Y::kOffItem + (n % kItems) * 64);
        v[2] = -1;
        mbar_arrive(bar(Y::bItem + n % kItems));
      }
    }
  } else if (warp < 8) {
    registers_down<Y::kRegs1>();
    constexpr int kPieces = D / 8, kAtOnce = 32 / kPieces, kAhead = 2;      // (a warp has 32 rows of a tile; tiles whose copies are under way beside the one that is waited for)
    const int piece = lane % kPieces, sub = lane / kPieces, wq = warp & 3;
    KeyItem it, next;
    // An item's keys, by this warp 64 of them: a lane knows where two lie, and the others ask it.
    int page[2];
    auto find_keys = [&](const KeyItem &of) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int pos = of.key0 + wq * 64 + half * 32 + lane;
        const bool seen = pos < of.hi && (pos >= of.lo || pos < of.n_sink);
        page[half] = seen ? page_of(s, a.bt, of.seq, pos) : -1;
      }
    };
    auto fetch_keys = [&](const KeyItem &of) {
      constexpr int kRowPieces = Y::kRowBytes / 16, kRowsAtOnce = 32 / kRowPieces;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        const int own = wq * 64 + half * 32 + lane, pg = half ? page[1] : page[0];
        const unsigned long long row = store_row(s, max(pg, 0), of.head, of.key0 + own);
        asm volatile("st.shared.b64 [%0], %1;" ::"r"(base + Y::kOffRow + own * 8), "l"(pg >= 0 ? row : ~0ull) : "memory");
        auto copy4 = [&](uint32_t to, const float *from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(pg >= 0 ? 4 : 0) : "memory"); };
        if (kQ8) copy4(base + Y::kOffScale + own * 4, s.k_scales + row);
        copy4(base + Y::kOffOld + own * 4, w.weights + row);
#pragma unroll 4
        for (int i = 0; i < kRowPieces; ++i) {
          const int from = i * kRowsAtOnce + lane / kRowPieces;
          const unsigned long long r = __shfl_sync(0xffffffffu, row, from);
          copy16(base + Y::kOffKeys + (wq * 64 + half * 32 + from) * Y::kPitch + (lane % kRowPieces) * 16, s.k_rows + r * Y::kRowBytes + (lane % kRowPieces) * 16, __shfl_sync(0xffffffffu, pg, from) >= 0);
        }
      }
    };
    bool ok = true, more = read_item(0, it);
    if (more) {
      find_keys(it);
      fetch_keys(it);
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Y::bRaw));
    }
    int q = 0;
    for (int n = 0; more && ok; ++n) {
      more = false;
      const int keys_at = min(kStages, it.tiles) - 1;          // behind this tile the next item's keys are asked for
      float lse[kAhead + 1];
#pragma unroll
      for (int k = 0; k <= kAhead; ++k) lse[k] = 0.f;
      for (int j = 0; j < it.tiles + kAhead && ok; ++j) {
        if (j < it.tiles) {
          const int at = q + j;
          ok = mbar_wait_warp(bar(Y::bQEmpty + at % kStages), ((at / kStages) & 1) ^ 1, abort_flag, status);
          if (!ok) break;
          const int r = (it.tile0 + j) * kQueryTile + tid, row = min(r, it.rows - 1), t = a.group.div(row), h = it.head * G + row - t * G;
          const char *mine = a.Q.ptr + (it.start + t) * a.Q.st + h * a.Q.sh;
          const uint32_t to = base + (at % kStages) * kTile + (piece >> 3) * kHalf + wq * 32 * 128;
#pragma unroll
          for (int k = 0; k < kPieces; ++k) {
            const int from = k * kAtOnce + sub;
            const char *src = reinterpret_cast<const char *>(__shfl_sync(0xffffffffu, (unsigned long long)mine, from));
            copy16(to + from * 128 + (((piece & 7) ^ (from & 7)) << 4), src + piece * 16, r - tid + wq * 32 + from < it.rows);
          }
          const float x = (float)((double)a.lse[(size_t)(it.start + t) * a.n_heads + h] * kLog2eExact);
          lse[kAhead] = r < it.rows && x != -INFINITY ? x : INFINITY;
        }
        if (j == keys_at) {
          more = read_item(n + 1, next);
          if (more) find_keys(next);               // (while the softmax warps still have this item's: 848 items of one query tile 34.3 us where behind them it was 35.5)
          if (more) ok = mbar_wait_warp(bar(Y::bRawFree), n & 1, abort_flag, status);
          if (!ok) break;
          if (more) fetch_keys(next);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (j >= kAhead) {
          const int at = q + j - kAhead, slot = at % Y::kSlots;
          const float x = lse[0];
          const uint32_t nothing = __ballot_sync(0xffffffffu, x == INFINITY);
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(base + Y::kOffLse + (slot * kQueryTile + tid) * 4), "f"(-x) : "memory");
          if (lane == 0) asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + Y::kOffVoid + slot * 16 + wq * 4), "r"(nothing) : "memory");
          asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
          fence_async_proxy();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(Y::bQFull + at % kStages));
            if (more && j == keys_at + kAhead) mbar_arrive(bar(Y::bRaw));
          }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) lse[k] = lse[k + 1];
      }
      q += it.tiles;
      it = next;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    registers_up<Y::kRegsS>();
    const int wg = (warp - 8) >> 2, quarter = warp & 3, row = quarter * 32 + lane, col0 = (wg & 1) * (kUnit / 2);
    const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
    int q = 0;
    float total[2];
    // This warpgroup's columns of unit u, rows r0 .. of the sequence's.
    auto unit = [&](int u, int r0, int all_lo, int all_hi, const int *lo, const int *hi, const uint64_t *k2) {
      const bool there = mbar_wait_warp(bar(Y::bSFull + u % kUnits), (u / kUnits) & 1, abort_flag, status);
      if (!there) return there;
      tc_fence_after();
      float x[2][32];
      const uint32_t s_addr = lane_addr + (u % kUnits) * 2 * kUnit + col0;
      tc_ld32(s_addr, x[0]);
      tc_ld32(s_addr + kUnit, x[1]);
      const int slot = (u >> 1) % Y::kSlots, col = (u & 1) * kUnit + col0;      // (column of the query tile)
      const uint32_t lse_at = base + Y::kOffLse + (slot * kQueryTile + col) * 4;
      uint32_t nothing;
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(nothing) : "r"(base + Y::kOffVoid + slot * 16 + (col >> 5) * 4) : "memory");
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Y::bSFree + u % kUnits));
      uint64_t sum[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
      if (nothing == 0 && all_lo <= r0 && all_hi >= r0 + 32) {
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 l = load_shared4(lse_at + e * 4);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float y[4];
            unpack2(fma2(pack2(x[t][e], x[t][e + 1]), k2[t], pack2(l.x, l.y)), y[0], y[1]);
            unpack2(fma2(pack2(x[t][e + 2], x[t][e + 3]), k2[t], pack2(l.z, l.w)), y[2], y[3]);
            sum[t] = add2(sum[t], add2(pack2(ex2(y[0]), ex2(y[1])), pack2(ex2(y[2]), ex2(y[3]))));
          }
        }
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t seen = lowest_bits(hi[t] - r0) & ~lowest_bits(lo[t] - r0) & ~nothing;
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 l = load_shared4(lse_at + e * 4);
            float y[4];
            unpack2(fma2(pack2(x[t][e], x[t][e + 1]), k2[t], pack2(l.x, l.y)), y[0], y[1]);
            unpack2(fma2(pack2(x[t][e + 2], x[t][e + 3]), k2[t], pack2(l.z, l.w)), y[2], y[3]);
#pragma unroll
            for (int f = 0; f < 4; ++f) y[f] = (seen >> (e + f)) & 1u ? ex2(y[f]) : 0.f;
            sum[t] = add2(sum[t], add2(pack2(y[0], y[1]), pack2(y[2], y[3])));
          }
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float s0, s1;
        unpack2(sum[t], s0, s1);
        total[t] += s0 + s1;
      }
      return there;
    };
    KeyItem it;
    bool ok = true;
    for (int n = 0;; ++n) {
      const bool there = read_item(n, it);
      if (!all_agree(there)) break;              // (a warp whose wait gave up comes here, too; and the last item's sums have been read)
      ok = ok && mbar_wait_warp(bar(Y::bRaw), n & 1, abort_flag, status);
      // keys into TMEM: warpgroups 0 and 1 have halves of A's dims, 2 and 3 of B's (what reads them is through: its results have been waited for)
      {
        const int tile = wg >> 1, half = wg & 1;
        const uint32_t from = base + Y::kOffKeys + (tile * 128 + row) * Y::kPitch + half * (Y::kRowBytes / 2);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {       // 32 dims, 16 columns
          uint32_t k[16];
#pragma unroll
          for (int x = 0; x < (kQ8 ? 2 : 4); ++x) {
            const uint4 v = load_shared16(from + (c * (kQ8 ? 2 : 4) + x) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if constexpr (kQ8) {
                const uint32_t u = turn_signs(word(v, e));
                k[x * 8 + 2 * e] = codes_low(u);
                k[x * 8 + 2 * e + 1] = codes_high(u);
              } else {
                k[x * 4 + e] = word(v, e);
              }
            }
          }
          tc_st16(lane_addr + kColK + tile * (D / 2) + half * (D / 4) + c * 16, k);
        }
      }
      unsigned long long at_row[2];
      float old[2];
      uint64_t k2[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = t * 128 + row;
        float scale = 1.f;
        asm volatile("ld.shared.b64 %0, [%1];" : "=l"(at_row[t]) : "r"(base + Y::kOffRow + key * 8) : "memory");
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(old[t]) : "r"(base + Y::kOffOld + key * 4) : "memory");
        if constexpr (kQ8) {
          asm volatile("ld.shared.f32 %0, [%1];" : "=f"(scale) : "r"(base + Y::kOffScale + key * 4) : "memory");
          scale *= kCodeUnit;
        }
        const float ks = (float)(w.scale_log2e * (double)scale);
        k2[t] = pack2(ks, ks);
      }
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(Y::bKeys));
        mbar_arrive(bar(Y::bRawFree));
      }
      // the rows that see this thread's keys, [lo, hi), and those that see all of the warp's
      int lo[2], hi[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int pos = it.key0 + t * 128 + row;
        lo[t] = a.mask.causal ? (int)min((long long)it.rows, (long long)max(pos - it.first, 0) * G) : 0;
        hi[t] = at_row[t] == ~0ull ? 0 : a.mask.window > 0 && pos >= it.n_sink ? (int)min((long long)it.rows, max((long long)pos - it.first + a.mask.window, 0ll) * G) : it.rows;
      }
      const int all_lo = __reduce_max_sync(0xffffffffu, max(lo[0], lo[1])), all_hi = __reduce_min_sync(0xffffffffu, min(hi[0], hi[1]));
      total[0] = total[1] = 0.f;
      for (int j = 0; j < it.tiles && ok; ++j) ok = unit(2 * (q + j) + (wg >> 1), (it.tile0 + j) * kQueryTile + (wg >> 1) * kUnit + col0, all_lo, all_hi, lo, hi, k2);
      q += it.tiles;
      // the warpgroups' shares of the rows are put together, in their order
      const uint32_t sum_at = base + Y::kOffSum + row * 4;
      if (wg > 0) {
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(sum_at + (wg - 1) * 1024), "f"(total[0]) : "memory");
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(sum_at + (wg - 1) * 1024 + 512), "f"(total[1]) : "memory");
      }
      if (!all_agree(ok)) break;
      if (wg == 0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float sum = total[t];
#pragma unroll
          for (int k = 0; k < kSumGroups - 1; ++k) {
            float other;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(other) : "r"(sum_at + k * 1024 + t * 512) : "memory");
            sum += other;
          }
          if (at_row[t] != ~0ull) w.weights[at_row[t]] = (it.key0 + t * 128 + row < it.first ? w.decay * old[t] : 0.f) + sum;
        }
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ---- what a window hides from all new tokens of a sequence, entries n_sink .. lo - 1: one product each, eight bytes of traffic.  A page that is out of range was given back, as windows do.
// us, 32 sequences of up to 10 521 entries of 8 heads behind a window of 1 024: the weigh 18.4, with this 24.6 (13 MB; a launch and its chain of length, table, sum).
constexpr int kFadeThreads = 256, kFadeFours = 2;      // fours of entries for a thread, or so

__global__ void __launch_bounds__(kFadeThreads) paged_fade_kernel(const __grid_constant__ WeighArgs w) {
  const AttendArgs &a = w.a;
  const Store &s = a.s;
  const int seq = blockIdx.x, head = blockIdx.y;
  wait_for_grid();
  next_grid();
  const Span sp(a, seq, 0x7fffffff, blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0);
  const int from = sp.n_sink, to = sp.rows > 0 ? sp.lo : 0;
  for (int i = (from >> 2) + blockIdx.z * kFadeThreads + threadIdx.x; i < (to + 3) >> 2; i += gridDim.z * kFadeThreads) {
    const int pos = i << 2, page = a.bt.table[(size_t)seq * a.bt.table_ld + (pos >> s.page_shift)];      // (a four lies in one page)
    if ((unsigned)page >= (unsigned)s.n_pages) continue;
    float4 *at = reinterpret_cast<float4 *>(w.weights + store_row(s, page, head, pos));
    auto faded = [&](float x, int p) { return p >= from && p < to ? w.decay * x : x; };
    const float4 x = *at;
    *at = make_float4(faded(x.x, pos), faded(x.y, pos + 1), faded(x.z, pos + 2), faded(x.w, pos + 3));
  }
}

template <int D, bool kQ8>
bool room() {
  auto ask = [](auto kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess; };
  return ask(paged_weigh_stream_kernel<D, kQ8, 1>, WeighLayout<D, kQ8, 1>::kSmem) && ask(paged_weigh_stream_kernel<D, kQ8, 2>, WeighLayout<D, kQ8, 2>::kSmem) &&
         ask(paged_weigh_stream_kernel<D, kQ8, 4>, WeighLayout<D, kQ8, 4>::kSmem) &&
         ask(paged_weigh_tile_kernel<D, kQ8>, WeighTile<D, kQ8>::kSmem);
}

}  // namespace paged
}  // namespace scalekv

bool scalekv::paged::room_for_weigh(int head_dim, bool q8) {
  if (head_dim == 128) return q8 ? room<128, true>() : room<128, false>();
  return q8 ? room<64, true>() : room<64, false>();
}

namespace {

scalekv_status check_sums(scalekv_paged *c, const scalekv_paged_mask *mask, const float *weights, float decay, const Batch &bt) {
  if (!mask || mask->window < 0 || mask->n_sink < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "mask null, or a negative size in it");
  if (!(decay >= 0.f && decay <= 1.f)) return fail(c, SCALEKV_ERR_INVALID_ARG, "decay must lie in [0, 1]");
  if (bt.n_tokens > 0 && (!weights || (reinterpret_cast<uintptr_t>(weights) & 15))) return fail(c, SCALEKV_ERR_INVALID_ARG, "weights null, or not 16-byte aligned");
  if (c->cfg.n_kv_heads > 32767) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 32767 kv heads");
  return SCALEKV_OK;
}

}  // namespace

extern "C" scalekv_status scalekv_paged_fade(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, const scalekv_paged_mask *mask, float *weights, float decay, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_fade");
  WeighArgs w = {};
  AttendArgs &a = w.a;
  if (scalekv_status st = check_batch(c, layer, batch, a.bt)) return st;
  if (scalekv_status st = check_sums(c, mask, weights, decay, a.bt)) return st;
  if (a.bt.n_tokens == 0 || mask->window == 0 || decay == 1.f) return SCALEKV_OK;
  a.s = layer_store(c, layer);
  a.mask = {mask->causal != 0, std::min(mask->window, kMaxLength), mask->n_sink};
  a.group = Divisor::of(1);
  a.max_new = batch->max_new;
  w.weights = weights;
  w.decay = decay;
  const long long entries = std::min<long long>(batch->max_length, (long long)a.bt.table_pages << c->page_shift);
  const dim3 grid(a.bt.n_seqs, c->cfg.n_kv_heads, (unsigned)std::clamp<long long>(entries / (4 * kFadeFours * kFadeThreads), 1, 65535));
  launch(paged_fade_kernel, grid, kFadeThreads, 0, static_cast<cudaStream_t>(stream), w);
  return launched(c, "paged_fade");
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
  if (scalekv_status st = check_sums(c, mask, weights, decay, a.bt)) return st;
  if (a.bt.n_tokens == 0) return SCALEKV_OK;
  if (!rows_ok(Q, 2) || !lse) return fail(c, SCALEKV_ERR_INVALID_ARG, "Q or lse null, or rows not 16-byte aligned");
  const int H = c->cfg.n_kv_heads, D = c->cfg.head_dim, G = n_heads / H;
  if ((long long)a.bt.n_tokens * n_heads > kMaxLength) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 2^30 query rows in a call");
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
  a.scale_log2e = 0.f;
  w.scale_log2e = (softmax_scale > 0.f ? (double)softmax_scale : 1. / std::sqrt((double)D)) * kLog2eExact;
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
      // a CTA to an SM, and no more of them than there may be items
      const long long items = std::min<long long>((keys + 2 * kKeyRows - 2) / kKeyRows * H, c->n_sm) * a.bt.n_seqs;
      launch(paged_weigh_tile_kernel<kD, kQ8>, dim3((unsigned)std::min<long long>(items, c->n_sm)), WeighTile<kD, kQ8>::kThreads, WeighTile<kD, kQ8>::kSmem, st, w);
    }
    return launched(c, "paged_weigh");
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  const bool q8 = c->cfg.store == SCALEKV_STORE_Q8;
  if (D == 128) return q8 ? go(D128{}, std::true_type{}) : go(D128{}, std::false_type{});
  return q8 ? go(D64{}, std::true_type{}) : go(D64{}, std::false_type{});
}
