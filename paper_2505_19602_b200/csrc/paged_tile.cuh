// Attention of many query rows over the paged token cache: chunks of new tokens, on tcgen05.
//
// The query rows of a kv head (row r: head r mod G of the group, token r / G) are cut into items of 256, a pair of 128-row tiles A and B;
// every 128-key tile is brought into shared memory once for both.  An item of 128 rows or fewer is a single: A and B are then the
// same queries against the even and the odd key tiles, combined at the end.  Where items do not fill the SMs, and for the last, partial wave of
// them, several CTAs share an item's key tiles; paged_join_kernel combines what they leave.
//
// Roles in a CTA, by warpgroup (registers dealt out by setmaxnreg):
//   warp 0        : tcgen05.mma issuer.  S_A(0), S_B(0), then per step j  PV_A(j), S_A(j+1), PV_B(j), S_B(j+1): the tensor pipe works
//                   for one tile while the other's softmax runs.
//   warp 1        : TMA producer: the tile's rows, page by page, into a ring of operand tiles K_0, V_0, K_1, V_1, ...  bf16 rows land as the
//                   products read them (128-byte swizzle), codes in the second half of their stage.
//   warps 4-7     : with codes only, converters, which put the codes of a stage back into it as bf16 (exactly: codes_bf16) and bring the scales.
//   the last eight: softmax, a warpgroup for each tile, a thread for each row (TMEM lane): one sweep over its 128 products in
//                   four chunks of 32, exponentials against a lazy reference, which rises when one exceeds it by more than 2^8, P as bf16 over the products already
//                   read (rounded: in two pieces, as few rows have it, its product would be twice as long, half as much again of all products).  With codes
//                   a key's scale is a factor of its column: K's is part of the factor of the exponent's FMA, V's multiplies P before it is rounded; both come from shared memory, four columns to a load.  (A thread with a quarter of the columns of four rows loads a quarter as many
//                   scales, but its sweep was the longer: 1 478 us for what was 1 247.)
// Rows that no query of the item sees (behind the length, ahead of the window, on a page out of range) may hold anything.  Their products are hidden one
// by one; as values codes are numbers whatever they are, and bf16 rows are zeroed by the issuer before the product reads them.
// Every wait is bounded; one that gives up raises the sticky status and all roles fall through to the end, behind the copies and products that are
// under way.
// What bounds it: with bf16 rows the two chains  S -> sweep -> P V, 3 750 cycles a step of a pair (2 048 at the tensor peak, and as many for its
// exponentials): 4 096 queries of 2 x 16 heads over 10 521 entries in 717 us, 0.99 PFLOP/s.  With codes shared memory, too: of a step's 5 000 cycles the
// products read for 1 540 and the threads take 2 860, about 2 050 of these for the scales (a 16-byte load takes a warp four cycles, the same address or not;
// without them 1 230 us were 1 020), the rest for the converters.  2 048 queries of 4 x 32 heads behind 6 144 entries: 1 124 us, 0.86 PFLOP/s; the same in
// bf16 1 000.
#pragma once
#include <string>
#include <type_traits>

#include "paged_stream.cuh"
#include "tc.cuh"

namespace scalekv {
namespace paged {

using namespace scalekv::tc;

constexpr int kItemRows = 256;
constexpr int kTileKeys = 128;
constexpr int kSweepChunks = 4;
constexpr int kEarly = 3;                         // chunks whose part of the PV product is issued under the rest of the sweep

template <int D, bool kQ8>
struct TileLayout {
  static constexpr int kThreads = kQ8 ? 512 : 384, kSoftmaxWarp = kQ8 ? 8 : 4;
  // registers of a thread of the first warpgroup, of the converters, of softmax: shares of what the block was launched with
  static constexpr int kRegs0 = kQ8 ? 56 : 72, kRegs1 = 104, kRegsS = kQ8 ? 176 : 216, kRegsLaunch = kQ8 ? 128 : 168;
  static_assert(kRegs0 + (kQ8 ? kRegs1 : 0) + 2 * kRegsS <= kRegsLaunch * (kThreads / 128), "a share would wait for registers that nobody returns");
  static constexpr int kStages = D == 64 ? (kQ8 ? 6 : 8) : (kQ8 ? 4 : 5);
  // Key tiles whose scales and holes are held.  Tile i + kSlots writes over tile i's when the stage of its K is free, which is when ring tile
  // 2 (i + kSlots) - kStages has been read: K of tile i + 2 or later (or V of i + 1 or later), whose product is issued behind the P of tile i.
  static constexpr int kSlots = D == 64 ? 8 : 4;
  static_assert(2 * kSlots - kStages >= 3, "tile i's scales may still be read");
  static constexpr uint32_t kTile = 128 * D * 2, kHalf = 128 * 128;      // an operand tile; 64 columns of it: one 128-byte swizzle span
  static constexpr uint32_t kOffQ = 0, kOffRing = 2 * kTile, kOffScale = kOffRing + kStages * kTile;
  static constexpr uint32_t kOffHoles = kOffScale + (kQ8 ? kSlots * 2 * 512 : 0);
  static constexpr uint32_t kOffBar = kOffHoles + kSlots * 4;
  enum { bQFull = 0, bFull = 2, bEmpty = bFull + kStages, bSFull = bEmpty + kStages, bPFull = bSFull + 2, bPvDone = bPFull + 2,
         bFinal = bPvDone + 2, bPEarly = bFinal + 2, bPvEarly = bPEarly + 2, bRaw = bPvEarly + 2, bCount = bRaw + (kQ8 ? kStages : 0) };
  static_assert(bCount <= 32, "one lane of a warp initialises each barrier");
  static constexpr uint32_t kOffItem = kOffBar + 8 * bCount;             // TMEM address, abort flag, the item
  static constexpr uint32_t kSmem = kOffItem + 64;
  static_assert(kSmem <= 232448, "more shared memory than a CTA can have");
  static_assert(kOffBar % 8 == 0, "barriers are 8 bytes");
};

// Instruction descriptor: bf16 x bf16 -> fp32, M = 128, N = n, A K-major; B K-major or MN-major.
__host__ __device__ constexpr uint32_t tile_desc(bool b_mn_major, int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// The four products of a K-major operand of 64 columns (tc_mma_ss_x8: of 128).
__device__ __forceinline__ void mma_ss_x4(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred e, pf, pt;\n\t.reg .b64 da, db;\n\t.reg .b32 al, bl;\n\t"
      "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 pf, 0, 0;\n\tsetp.eq.b32 pt, 0, 0;\n\t"
      "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, pf;\n\t"
      "add.u32 al, %1, 2;\n\tadd.u32 bl, %2, 2;\n\tmov.b64 da, {al, %3};\n\tmov.b64 db, {bl, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, pt;\n\t"
      "add.u32 al, %1, 4;\n\tadd.u32 bl, %2, 4;\n\tmov.b64 da, {al, %3};\n\tmov.b64 db, {bl, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, pt;\n\t"
      "add.u32 al, %1, 6;\n\tadd.u32 bl, %2, 6;\n\tmov.b64 da, {al, %3};\n\tmov.b64 db, {bl, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, pt;\n\t"
      "}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc)
      : "memory");
}
template <int kRegs> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void store_shared(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float4 load_shared4(uint32_t at) {
  float4 x;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at));
  return x;
}
__device__ __forceinline__ uint4 load_shared16(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at));
  return x;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *tm, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(tm), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}

// The bounded wait of tc.cuh, without a call: a kernel that deals out its registers by setmaxnreg makes none.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status) {
  bool ok = mbar_try(bar, parity);
  if (!ok) {
    const unsigned long long t0 = globaltimer();
    for (int i = 0;; ++i) {
      if (mbar_try(bar, parity)) { ok = true; break; }
      if ((i & 63) != 63) continue;
      if (*abort_flag || *reinterpret_cast<volatile int *>(status) == kDevTimeout) break;
      if (globaltimer() - t0 > kWaitLimitNs) {
        *abort_flag = 1;
        atomicExch(status, kDevTimeout);
        break;
      }
    }
  }
  return __all_sync(0xffffffffu, ok);
}

// For what a CTA has asked for and must not leave behind, copies into its shared memory and products into its TMEM: waits until it is through, whatever the
// status, a second at most.
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = globaltimer();
  while (!mbar_try(bar, parity) && globaltimer() - t0 < kWaitLimitNs / 2) {}
}

// Whether all 128 threads of the converters bring true.  A named barrier, which knows no limit: whoever has given up comes, too, and all of them hear of it.
__device__ __forceinline__ bool all_converters(bool mine) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 3, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(mine ? 1u : 0u)
      : "memory");
  return all != 0;
}

__device__ __forceinline__ float2 load_shared2(uint32_t at) {
  float2 x;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at));
  return x;
}
// 8 consecutive 32-bit columns of this thread's TMEM lane
__device__ __forceinline__ void tc_ld8(uint32_t at, uint32_t *r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t at, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// Item number `want`, items counted through the sequences: its sequence (-1: there are fewer), its tile, and where the sequence's new tokens lie.  A whole
// warp.  (The length is asked for with the starts: behind them it was one more trip to memory for every item.  us, chunks under a window of 700 55.5 / 55.3, two
// prompts of 64 tokens behind 448 entries 22.7 / 22.5.)
struct Item {
  int seq, tile, start, n_new, length;
};
__device__ __forceinline__ Item find_item(const AttendArgs &a, int want) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int b0 = 0; b0 < a.bt.n_seqs; b0 += 32) {
    const int b = b0 + lane;
    int n = 0, st = 0, en = 0, length = 0;
    if (b < a.bt.n_seqs) {
      st = a.bt.starts[b];
      en = min(a.bt.starts[b + 1], a.bt.n_tokens);
      length = a.bt.lengths[b];
      if (st >= 0 && en > st) n = (int)(((long long)(en - st) * a.group.d + kItemRows - 1) / kItemRows);
    }
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    const unsigned behind = __ballot_sync(0xffffffffu, before + incl > want);
    if (behind) {
      const int src = __ffs(behind) - 1;
      const int first = __shfl_sync(0xffffffffu, incl - n, src), start = __shfl_sync(0xffffffffu, st, src);
      return {b0 + src, want - before - first, start, __shfl_sync(0xffffffffu, en, src) - start, __shfl_sync(0xffffffffu, length, src)};
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return {-1, 0, 0, 0, 0};
}
// CTAs of a launch: the first n_full take an item of a kv head each, the items behind them are shared by `parts`.
struct Cut {
  Divisor heads, parts;
  int n_items, n_full;
};

__device__ __forceinline__ uint32_t lowest_bits(int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; }
// Of 32 columns of a key tile, from position `at`, those that a row with limits [lo, hi) and n_sink does not see, a bit for each; holes: a bit for each 16
// columns whose page is out of range.
__device__ __forceinline__ uint32_t hidden_bits(int at, int lo, int hi, int n_sink, uint32_t holes) {
  const uint32_t seen = lowest_bits(hi - at) & (~lowest_bits(lo - at) | lowest_bits(n_sink - at));
  return ~seen | ((holes & 1u) * 0xffffu) | ((holes & 2u) * 0x7fff8000u);
}

// tmK, tmV: the K and V rows of all layers, [layer * pages + page][kv head * page_tokens + row][head_dim]; page0: layer * pages
template <int D, bool kQ8>
__global__ void __launch_bounds__(TileLayout<D, kQ8>::kThreads, 1)
paged_tile_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ AttendArgs a,
                  const Cut cut, int page0) {
  using Y = TileLayout<D, kQ8>;
  constexpr int kStages = Y::kStages;
  constexpr uint32_t kTile = Y::kTile, kHalf = Y::kHalf;
  constexpr uint32_t kColS = 0, kColO = 256;      // S/P buffers at 0 and 128, O accumulators at 256 and 384
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const uint32_t bars = base + Y::kOffBar;
  auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
  volatile int *item = reinterpret_cast<volatile int *>(smem_raw + Y::kOffItem);
  volatile int *abort_flag = item + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x & 127;
  const Store &s = a.s;
  int *status = s.status;
  const int beyond = (int)blockIdx.x - cut.n_full, shared_item = cut.parts.div(max(beyond, 0));
  const int part = beyond < 0 ? 0 : beyond - shared_item * cut.parts.d, parts = beyond < 0 ? 1 : cut.parts.d;
  const int at_item = beyond < 0 ? (int)blockIdx.x : cut.n_full + shared_item, e = cut.heads.div(at_item), head = at_item - e * cut.heads.d;

  // ---- set-up: barriers, TMEM, and the item.  Items are counted through the sequences, and taken from the end: of a causal chunk the
  // last rows see most.
  if (warp == 0) {
    wait_for_grid();
    Item it = find_item(a, cut.n_items - 1 - e);
    if (lane == 0) {
      if (it.seq >= 0) {
        it.length = max(min(it.length, a.bt.table_pages << s.page_shift), 0);
      }
      if (*reinterpret_cast<volatile int *>(status) == kDevTimeout) it.seq = -1;      // an earlier CTA gave up: do not pile on
      if (base & 1023u) { report(status); it.seq = -1; }
      item[1] = 0;
      item[2] = it.seq; item[3] = it.tile; item[4] = it.start; item[5] = it.n_new; item[6] = it.length;
    }
  } else if (warp == 1) {
    if (lane < Y::bCount) {
      // arrivals a phase: one lane of each of four warps for what a warpgroup hands over, else the producer or a commit
      const bool four = lane < 2 || (kQ8 && lane >= Y::bFull && lane < Y::bFull + kStages) || (lane >= Y::bPFull && lane < Y::bPFull + 2) ||
                        (lane >= Y::bPEarly && lane < Y::bPEarly + 2);
      mbar_init(bar(lane), four ? 4u : 1u);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + Y::kOffItem), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else if (warp == 3 && blockIdx.x == 0) {
    // what is out of range in the batch, of sequences that have no item, too
    wait_for_grid();
    for (int b = lane; b < a.bt.n_seqs; b += 32) {
      const int start_b = a.bt.starts[b], end_b = a.bt.starts[b + 1];
      if (starts_wrong(a.bt, b, start_b, end_b) || end_b - start_b > a.max_new ||
          (unsigned)a.bt.lengths[b] > (unsigned)(a.bt.table_pages << s.page_shift))
        report(status);
    }
  }
  wait_for_grid();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)item[0];
  const int seq = item[2], row0 = item[3] * kItemRows, start = item[4], n_new = item[5], length = item[6];
  const int first = length - n_new, all = n_new * a.group.d, rows = seq < 0 ? 0 : min(kItemRows, all - row0);
  const bool pair = rows > 128;
  // the key tiles that some row of the item sees: the sinks', then those of [lo, hi); this CTA's are lo .. lo + nt - 1 of them
  int lo_all = 0, hi_all = 0;
  if (rows > 0) {
    lo_all = min(seen_lo(a.mask, first + a.group.div(row0)), length);
    hi_all = seen_hi(a.mask, first + a.group.div(row0 + rows - 1), length);
  }
  const int n_sink = a.mask.window > 0 ? a.mask.n_sink : 0;
  const int lo_tile = lo_all >> 7, hi_tile = max((hi_all + 127) >> 7, lo_tile);
  const int sink_tiles = min((min(n_sink, hi_all) + 127) >> 7, lo_tile);
  const int n_tiles = sink_tiles + hi_tile - lo_tile;
  const int lo = (int)((long long)n_tiles * part / parts), nt = (int)((long long)n_tiles * (part + 1) / parts) - lo;
  auto key_of = [&](int i) { i += lo; return (i < sink_tiles ? i : i - sink_tiles + lo_tile) << 7; };     // first position of key tile i of this CTA
  const bool shared = !pair && nt > 1;
  auto n_steps = [&](int qt) { return shared ? (nt + 1 - qt) >> 1 : (pair || qt == 0 ? nt : 0); };
  auto ring_of = [&](int j, int qt) { return shared ? 4 * j + 2 * qt : 2 * j; };      // ring tile of tile qt's K in step j (its V is the next)

  auto in_use = [&](int pos) { return pos < hi_all && (pos >= lo_all || pos < n_sink); };       // some row of the item sees it
  // pages of key tile i: lane g (mod 8) has that of keys 16 g .. of the tile, which lie in one; -1: nobody looks there, or it is out of range
  auto group_in_use = [&](int i) {
    const int pos = key_of(i) + 16 * (lane & 7);
    return pos < hi_all && (pos + 16 > lo_all || pos < n_sink);
  };
  auto pages = [&](int i) { return i < nt && group_in_use(i) ? page_of(s, a.bt, seq, key_of(i) + 16 * (lane & 7)) : -1; };

  if (warp < 4) {
    registers_down<Y::kRegs0>();
    if (warp == 0 && rows > 0) {
      // -------------------------------------------------------------- MMA issuer (the whole warp walks, one elected lane issues)
      constexpr uint32_t idesc_qk = tile_desc(false, 128), idesc_pv = tile_desc(true, D), dhi = desc_hi(1024);
      const bool leader = elect_one();
      // What stands between the arrival of P and the tile's next S product is issue alone: descriptors and barriers' addresses are formed before the wait.
      const uint32_t q_lo[2] = {desc_lo(base + Y::kOffQ, 16), desc_lo(base + Y::kOffQ + (pair ? kTile : 0u), 16)};
      auto k_desc = [&](int kt) { return desc_lo(base + Y::kOffRing + (kt % kStages) * kTile, 16); };
      auto mma_s = [&](uint32_t k, int qt) {
        if constexpr (D == 128) tc_mma_ss_x8(tmem + kColS + qt * 128, qt ? q_lo[1] : q_lo[0], k, dhi, idesc_qk);
        else mma_ss_x4(tmem + kColS + qt * 128, qt ? q_lo[1] : q_lo[0], k, dhi, idesc_qk);
      };
      auto ring_full = [&](int t) { return mbar_wait_warp(bar(Y::bFull + t % kStages), (t / kStages) & 1, abort_flag, status); };
      const int steps[2] = {n_steps(0), n_steps(1)};
      // hidden rows of a tile of bf16 values become zeros before a product reads them: P is 0 there, and 0 x NaN is NaN
      auto clean = [&](int vt) {
        const int key0 = key_of(vt >> 1);
        uint32_t holes;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(holes) : "r"(base + Y::kOffHoles + ((vt >> 1) % Y::kSlots) * 4));
        if (key0 >= lo_all && key0 + kTileKeys <= hi_all && holes == 0) return;
        const uint32_t tile = base + Y::kOffRing + (vt % kStages) * kTile;
        for (int r = lane; r < kTileKeys; r += 32) {
          if (in_use(key0 + r) && !((holes >> (r >> 4)) & 1u)) continue;
#pragma unroll 1
          for (int x = 0; x < D / 8; ++x) store_shared(tile + (x >> 3) * kHalf + r * 128 + (x & 7) * 16, 0u, 0u, 0u, 0u);
        }
        fence_async_proxy();
        __syncwarp();
      };
      bool ok = true;
      uint32_t latest = 0, latest_parity = 0;      // barrier and phase of the commit that stands behind all products so far
      for (int qt = 0; qt < 2 && ok && steps[qt] > 0; ++qt) {
        const int kt = ring_of(0, qt);
        ok = mbar_wait_warp(bar(Y::bQFull + (pair ? qt : 0)), 0, abort_flag, status) && ring_full(kt);
        if (!ok) break;
        tc_fence_after();
        mma_s(k_desc(kt), qt);
        if (leader) {
          tc_commit(bar(Y::bSFull + qt));
          if (!pair || qt == 1) tc_commit(bar(Y::bEmpty + kt % kStages));
        }
        latest = bar(Y::bSFull + qt);
        __syncwarp();
      }
      for (int j = 0; j < steps[0] && ok; ++j) {
#pragma unroll 1
        for (int qt = 0; qt < 2 && ok; ++qt) {
          const int mine = qt ? steps[1] : steps[0];
          if (j >= mine) break;
          const bool more = j + 1 < mine;
          const int vt = ring_of(j, qt) + 1, kt = ring_of(j + 1, qt);
          const uint32_t vd = desc_lo(base + Y::kOffRing + (vt % kStages) * kTile, kHalf), pa = tmem + kColS + qt * 128, oa = tmem + kColO + qt * 128;
          const uint32_t kd = k_desc(kt), v_empty = bar(Y::bEmpty + vt % kStages), k_empty = bar(Y::bEmpty + kt % kStages);
          const uint32_t done = bar((more ? Y::bSFull : Y::bFinal) + qt);
          ok = ring_full(vt);
          if (!ok) break;
          if (!kQ8 && (!pair || qt == 0)) clean(vt);
          ok = mbar_wait_warp(bar(Y::bPEarly + qt), j & 1, abort_flag, status);
          if (!ok) break;
          tc_fence_after();
          tc_mma_ts_n<2 * kEarly>(oa, pa, vd, dhi, idesc_pv, j > 0 ? 1u : 0u);
          if (leader) tc_commit(bar(Y::bPvEarly + qt));
          latest = bar(Y::bPvEarly + qt);
          latest_parity = j & 1;
          __syncwarp();
          ok = (!more || ring_full(kt)) && mbar_wait_warp(bar(Y::bPFull + qt), j & 1, abort_flag, status);
          if (!ok) break;
          tc_fence_after();
          tc_mma_ts_n<8 - 2 * kEarly>(oa, pa + p_col(2 * kEarly), vd + 128 * 2 * kEarly, dhi, idesc_pv, 1u);
          if (more) mma_s(kd, qt);
          if (leader) {
            tc_commit(done);
            if (!pair || qt == 1) {
              tc_commit(v_empty);
              if (more) tc_commit(k_empty);
            }
            tc_commit(bar(Y::bPvDone + qt));
          }
          latest = bar(Y::bPvDone + qt);
          __syncwarp();
        }
      }
      next_grid();
      // (whoever has given up: no product may be under way when TMEM is freed and the tiles that it reads are gone)
      if (latest) drain(latest, latest_parity);
    } else if (warp == 1 && rows > 0) {
      // -------------------------------------------------------------- TMA producer (a lane to each box of rows of a page)
      // Ring tile t holds K (even) or V (odd) of key tile t / 2, which bRaw (codes) or bFull says.  A tile's holes go with its K.  (One lane that issued all boxes,
      // one after the other, needed 245 cycles for each: with pages of 16 tokens that was the larger part of a step.)
      const int box = min(1 << s.page_shift, kTileKeys), in_page = (1 << s.page_shift) - 1;
      constexpr int kLanded = kQ8 ? Y::bRaw : Y::bFull;
      constexpr uint32_t kRowBytes = D * (kQ8 ? 1 : 2);
      const int r0 = lane * box;
      const uint32_t groups = ((1u << (box >> 4)) - 1u) << ((r0 >> 4) & 31);      // of this lane's box
      int page = pages(0), page_next = pages(1), page_after = pages(2), t = 0;
      bool ok = true;
      for (int i = 0; i < nt && ok; ++i) {
        const int key0 = key_of(i);
        const uint32_t there = __ballot_sync(0xffffffffu, page >= 0) & 0xffu, used = __ballot_sync(0xffffffffu, group_in_use(i)) & 0xffu;
        // a box is loaded if one of its groups in use has a page (they share it)
        const uint32_t mine = r0 < kTileKeys ? there & groups : 0u, bytes = __popc(__ballot_sync(0xffffffffu, mine != 0)) * box * kRowBytes;
        const int pg = __shfl_sync(0xffffffffu, page, max(__ffs(mine) - 1, 0));
        const int y = (head << s.page_shift) + ((key0 + r0) & in_page), z = page0 + pg;
        page = page_next;
        page_next = page_after;
        page_after = pages(i + 3);
#pragma unroll
        for (int v = 0; v < 2; ++v, ++t) {
          const int st = t % kStages;
          ok = mbar_wait_warp(bar(Y::bEmpty + st), ((t / kStages) & 1) ^ 1, abort_flag, status);
          if (!ok) break;
          if (lane == 0) {
            if (v == 0) asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + Y::kOffHoles + (i % Y::kSlots) * 4), "r"(used & ~there) : "memory");
            mbar_expect_tx(bar(kLanded + st), bytes);
          }
          __syncwarp();
          if (mine) {
            const CUtensorMap *tm = v ? &tmV : &tmK;
            const uint32_t dst = base + Y::kOffRing + st * kTile + (kQ8 ? kTile - 128 * D : 0u) + r0 * (kQ8 ? D : 128);
            tma_load_3d(dst, tm, 0, y, z, bar(kLanded + st));
            if constexpr (!kQ8 && D == 128) tma_load_3d(dst + kHalf, tm, 64, y, z, bar(kLanded + st));
          }
          __syncwarp();
        }
      }
      // (whoever has given up: nothing may land in this CTA's shared memory once it is gone)
      for (int k = max(t - kStages, 0); k < t; ++k) drain(bar(kLanded + k % kStages), (k / kStages) & 1);
    }
  } else if (kQ8 && warp < 8) {
    registers_down<Y::kRegs1>();
    // ---------------------------------------------------------------- converters
    // The scales of both go with K, into slot (t / 2) mod Y::kSlots; that slot's last readers are done: the stage of this K was
    // released behind a product that was issued after their P.
    const int piece = tid & 3, sub = tid >> 2;      // 16 codes a piece, 64 columns at a time
    float k_scale = 0.f, v_scale = 0.f;
    auto fetch_scales = [&](int i) {
      const int page = __shfl_sync(0xffffffffu, pages(i), tid >> 4), pos = key_of(i) + tid;
      const bool on = page >= 0 && in_use(pos);
      const size_t row = store_row(s, max(page, 0), head, pos);
      k_scale = on ? __ldcg(s.k_scales + row) * (a.scale_log2e * kCodeUnit) : 0.f;
      v_scale = on ? __ldcg(s.v_scales + row) * kCodeUnit : 0.f;
    };
    if (nt > 0 && rows > 0) fetch_scales(0);
    for (int t = 0; t < 2 * nt && rows > 0; ++t) {
      const uint32_t stage = base + Y::kOffRing + (t % kStages) * kTile;
      const bool landed = mbar_wait_warp(bar(Y::bRaw + t % kStages), (t / kStages) & 1, abort_flag, status);
      // 16 codes become two 16-byte pieces of a row's 128-byte span of 64 columns.  Eight lanes' stores, of two
      // neighbouring rows, meet all banks.
      auto convert = [&](const uint4 &raw, uint32_t span, int r) {
        const uint32_t w[4] = {turn_signs(raw.x), turn_signs(raw.y), turn_signs(raw.z), turn_signs(raw.w)};
#pragma unroll
        for (int k = 0; k < 2; ++k)
          store_shared(span + r * 128 + (((piece * 2 + k) ^ (r & 7)) << 4), codes_low(w[2 * k]), codes_high(w[2 * k]), codes_low(w[2 * k + 1]),
                       codes_high(w[2 * k + 1]));
      };
      // The codes lie in the stage's last quarter or half.  What becomes its first half can go there at once; what becomes the half that they
      // lie in is taken out by all threads before any puts it back.
      const uint32_t raw_at = stage + kTile - 128 * D + piece * 16;
      uint4 last[4];
      if (landed) {
        if (!(t & 1)) {
          const uint32_t at = base + Y::kOffScale + ((t >> 1) % Y::kSlots) * 1024 + tid * 4;
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(k_scale) : "memory");
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 512), "f"(v_scale) : "memory");
          if ((t >> 1) + 1 < nt) fetch_scales((t >> 1) + 1);
        }
#pragma unroll
        for (int it = 0; it < 4; ++it) last[it] = load_shared16(raw_at + (it * 32 + sub) * D + (D - 64));
        if constexpr (D == 128) {
#pragma unroll 2
          for (int r = sub; r < 128; r += 32) convert(load_shared16(raw_at + r * D), stage, r);
        }
      }
      if (!all_converters(landed)) break;          // (a warp whose wait gave up comes here, or the others would wait for it for ever)
#pragma unroll
      for (int it = 0; it < 4; ++it) convert(last[it], stage + (D == 128 ? kHalf : 0u), it * 32 + sub);
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Y::bFull + t % kStages));
    }
  } else {
    registers_up<Y::kRegsS>();
    // ---------------------------------------------------------------- softmax
    const int qt = (warp - Y::kSoftmaxWarp) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
    const int tile_row0 = row0 + (pair ? qt * 128 : 0);
    if (rows > 0 && (pair || qt == 0)) {
      // the tile's queries: 16 or 8 pieces of 16 bytes a row, swizzled as the products read them; zeros beyond the last row
      constexpr int kPieces = D / 8, kAtOnce = 128 / kPieces;
      const int piece = tid % kPieces, sub = tid / kPieces;
      const uint32_t to = base + Y::kOffQ + qt * kTile + (piece >> 3) * kHalf;
#pragma unroll 4
      for (int it = 0; it < kPieces; ++it) {
        const int r = it * kAtOnce + sub, i = tile_row0 + r;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (i < all) {
          const int t = a.group.div(i), g = i - t * a.group.d;
          v = reinterpret_cast<const uint4 *>(a.Q.ptr + (start + t) * a.Q.st + (head * a.group.d + g) * a.Q.sh)[piece];
        }
        store_shared(to + r * 128 + (((piece & 7) ^ (r & 7)) << 4), v.x, v.y, v.z, v.w);
      }
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Y::bQFull + qt));
    }
    // this row's limits, and those of the warp's rows together
    const int i_own = tile_row0 + row;                     // this thread's row, of the sequence's
    auto token_of = [&](int i) { return a.group.div(max(min(i, all - 1), 0)); };
    const int t_own = token_of(i_own), p_top = first + token_of(tile_row0 + quarter * 32), p_end = first + token_of(tile_row0 + quarter * 32 + 31);
    const int row_lo = seen_lo(a.mask, first + t_own), row_hi = seen_hi(a.mask, first + t_own, length);
    const int warp_lo = seen_lo(a.mask, p_top), warp_lo_full = seen_lo(a.mask, p_end);
    const int warp_hi = seen_hi(a.mask, p_end, length), warp_hi_full = seen_hi(a.mask, p_top, length);
    const float c = a.scale_log2e;
    const uint64_t c2 = pack2(c, c);
    // the reference starts at the lowest number: differences from it are numbers
    float m = -FLT_MAX, l = 0.f;
    const uint32_t o_addr = lane_addr + kColO + qt * 128, s_addr = lane_addr + kColS + qt * 128;
    const int steps = rows > 0 ? n_steps(qt) : 0;
    bool ok = true;
    for (int j = 0; j < steps && ok; ++j) {
      const int i_tile = shared ? 2 * j + qt : j, key0 = key_of(i_tile);
      ok = mbar_wait_warp(bar(Y::bSFull + qt), j & 1, abort_flag, status);
      if (!ok) break;
      tc_fence_after();
      uint32_t holes;
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(holes) : "r"(base + Y::kOffHoles + (i_tile % Y::kSlots) * 4));
      const uint32_t scales = base + Y::kOffScale + (i_tile % Y::kSlots) * 1024;       // K's, 512 bytes further V's
      auto hand_over = [&](int which) {
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(which + qt));
      };
      // ---- tiles that every row of the warp sees whole.  p = 2^(x - m) of a chunk in place of its products:
      auto front = [&](float *x, int cc) {
        const uint64_t negm2 = pack2(-m, -m);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          uint64_t k0 = c2, k1 = c2;
          if constexpr (kQ8) {
            const float4 k = load_shared4(scales + (cc * 32 + i) * 4);
            k0 = pack2(k.x, k.y);
            k1 = pack2(k.z, k.w);
          }
          unpack2(fma2(pack2(x[i], x[i + 1]), k0, negm2), x[i], x[i + 1]);
          unpack2(fma2(pack2(x[i + 2], x[i + 3]), k1, negm2), x[i + 2], x[i + 3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i + e] = ex2(x[i + e]);
        }
      };
      // P of a chunk, and its sum: 32 values of at most 2^8 sum to at most 2^13; a larger, infinite or NaN sum means that some exponent left the band.
      auto back = [&](const float *x, uint32_t *pk, int cc) {
        uint64_t sum_a = pack2(0.f, 0.f), sum_b = sum_a;
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const uint64_t p0 = pack2(x[i], x[i + 1]), p1 = pack2(x[i + 2], x[i + 3]);
          sum_a = add2(sum_a, p0);
          sum_b = add2(sum_b, p1);
          float y[4] = {x[i], x[i + 1], x[i + 2], x[i + 3]};
          if constexpr (kQ8) {
            const float4 k = load_shared4(scales + 512 + (cc * 32 + i) * 4);
            unpack2(mul2(p0, pack2(k.x, k.y)), y[0], y[1]);
            unpack2(mul2(p1, pack2(k.z, k.w)), y[2], y[3]);
          }
          pk[i / 2] = pack_bf16(y[0], y[1]);
          pk[i / 2 + 1] = pack_bf16(y[2], y[3]);
        }
        float s0, s1;
        unpack2(add2(sum_a, sum_b), s0, s1);
        return s0 + s1;
      };
      int cc = 0;                                  // the first chunk that is not finished
      if (holes == 0 && key0 >= warp_lo_full && key0 + kTileKeys <= warp_hi_full) {
        // Software-pipelined: the exponentials of the next chunk are under way while this one is summed, checked and stored.
        float v[2][32];
        tc_ld32(s_addr, v[0]);
        tc_ld32(s_addr + 32, v[1]);
        tc_wait_ld();
        front(v[0], 0);
        auto finish = [&](int q, const float *x) {         // false: chunk q has to be taken again
          uint32_t pk[16];
          const float sum = back(x, pk, q);
          if (__any_sync(0xffffffffu, !(sum <= 8192.f))) return false;
          tc_st16(s_addr + q * 16, pk);
          l += sum;
          cc = q + 1;
          return true;
        };
#pragma unroll
        for (int q = 0; q < kSweepChunks; q += 2) {
          front(v[1], q + 1);
          if (!finish(q, v[0])) break;
          if (q == 0) {
            tc_ld32(s_addr + 64, v[0]);
            tc_wait_ld();
            front(v[0], 2);
          } else {
            hand_over(Y::bPEarly);
          }
          if (!finish(q + 1, v[1])) break;
          if (q == 0) {
            tc_ld32(s_addr + 96, v[1]);
            tc_wait_ld();
          }
        }
      }
      // ---- chunk by chunk, from the raw products in columns 32 cc .. (P covers columns below 16 cc only): tiles of which some rows see a part, and what is
      // left of a tile once an exponent has left the band.  Where one is more than 2^8 above a row's reference, the references of all the warp's rows rise
      // to their chunk's largest or just above, and what was accumulated under the old one is multiplied by f = 2^(old - new): the sum, P of the chunks that the
      // tensor core has not been given yet, and O, once the last product given to it has landed.
      // (One loop for both, not unrolled: the roles' loops together have to stay in the SM's instruction cache.  With a masked copy of the sweep above and a copy of
      // the raise in each of its chunks a step in codes, which has the converters' loop beside it, missed it 28 times in a hundred: 2 255 us for what was 1 618.)
      int landed = 0;                              // 1: the last step's product has; 2: the early part of this one's, too
#pragma unroll 1
      for (; cc < kSweepChunks && ok; ++cc) {
        const int col0 = cc * 32, at = key0 + col0;
        uint32_t pk[16];
        if (at >= warp_hi || (at + 32 <= warp_lo && at >= n_sink)) {       // no row of the warp sees it
#pragma unroll
          for (int i = 0; i < 16; ++i) pk[i] = 0u;
        } else {
          float x[32], top = -INFINITY;
          tc_ld32(s_addr + col0, x);
          tc_wait_ld();
          const uint32_t hidden = hidden_bits(at, row_lo, row_hi, n_sink, holes >> (2 * cc));
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float2 k = kQ8 ? load_shared2(scales + (col0 + i) * 4) : make_float2(c, c);
            x[i] = (hidden >> i) & 1u ? -INFINITY : x[i] * k.x;
            x[i + 1] = (hidden >> i) & 2u ? -INFINITY : x[i + 1] * k.y;
            top = max3(top, x[i], x[i + 1]);
          }
          if (__any_sync(0xffffffffu, top > m + 8.f)) {
            // (to a whole number, so that f is a power of two and P, scaled, is not rounded again)
            const float raised = fmaxf(m, ceilf(top)), f = __uint_as_float((uint32_t)(max((int)(m - raised), -127) + 127) << 23);
            m = raised;
            l *= f;
            const bool late = cc >= kEarly;
            uint32_t r[8];
            tc_wait_st();
#pragma unroll 1
            for (int e = late ? 2 * kEarly : 0; e < cc * 2; ++e) {
              tc_ld8(s_addr + e * 8, r);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 8; ++i) r[i] = pack_bf16(__uint_as_float(r[i] << 16) * f, __uint_as_float(r[i] & 0xffff0000u) * f);
              tc_st8(s_addr + e * 8, r);
            }
            if (late || j > 0) {
              if (landed < (late ? 2 : 1)) {
                ok = mbar_wait_warp(bar((late ? Y::bPvEarly : Y::bPvDone) + qt), (late ? j : j - 1) & 1, abort_flag, status);
                if (!ok) break;
                tc_fence_after();
                landed = late ? 2 : 1;
              }
#pragma unroll 1
              for (int e = 0; e < D / 8; ++e) {
                tc_ld8(o_addr + e * 8, r);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
                tc_st8(o_addr + e * 8, r);
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float2 k = kQ8 ? load_shared2(scales + 512 + (col0 + i) * 4) : make_float2(1.f, 1.f);
            float p0 = ex2(x[i] - m), p1 = ex2(x[i + 1] - m);
            l += p0 + p1;
            if constexpr (kQ8) {                   // (a hidden value's scale may be no number)
              p0 = (hidden >> i) & 1u ? 0.f : p0 * k.x;
              p1 = (hidden >> i) & 2u ? 0.f : p1 * k.y;
            }
            pk[i / 2] = pack_bf16(p0, p1);
          }
        }
        tc_st16(s_addr + cc * 16, pk);
        if (cc == kEarly - 1) hand_over(Y::bPEarly);
      }
      if (!ok) break;
      hand_over(Y::bPFull);
    }
    // ---- the rows go out: normalised, or, where CTAs share them, as they are with their reference and sum
    if (steps > 0 && ok) ok = mbar_wait_warp(bar(Y::bFinal + qt), 0, abort_flag, status);
    tc_fence_after();
    const bool mine = i_own < all && rows > 0;
    const int g = i_own - a.group.div(max(i_own, 0)) * a.group.d;
    const int h = head * a.group.d + g;
    const size_t out_row = mine ? (size_t)(start + t_own) * a.n_heads + h : 0;
    const bool split = parts > 1;
    const size_t part_row = ((size_t)shared_item * parts + part) * kItemRows + (tile_row0 - row0) + row;
    auto put = [&](float *o, int col0, float f) {          // 32 columns of this row
      if (!mine) return;
      if (split) {
        float4 *to = reinterpret_cast<float4 *>(a.part_o + part_row * D + col0);
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i] = make_float4(o[4 * i] * f, o[4 * i + 1] * f, o[4 * i + 2] * f, o[4 * i + 3] * f);
      } else {
        uint4 *to = reinterpret_cast<uint4 *>(a.O.ptr + (start + t_own) * a.O.st + h * a.O.sh + col0 * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          to[i] = make_uint4(pack_bf16(o[8 * i] * f, o[8 * i + 1] * f), pack_bf16(o[8 * i + 2] * f, o[8 * i + 3] * f),
                             pack_bf16(o[8 * i + 4] * f, o[8 * i + 5] * f), pack_bf16(o[8 * i + 6] * f, o[8 * i + 7] * f));
      }
    };
    auto put_sums = [&](float mr, float lr) {
      if (!mine) return;
      if (split) *reinterpret_cast<float2 *>(a.part_ml + part_row * 2) = make_float2(lr == 0.f ? -INFINITY : mr, lr);
      else if (a.lse != nullptr) a.lse[out_row] = lr == 0.f ? -INFINITY : (mr + log2f(lr)) * kLn2;
    };
    if (rows > 0 && ok && !shared && (pair || qt == 0)) {
      // (a row that saw nothing has a sum of 0 and an accumulator of zeros, or none at all)
      const float f = split ? 1.f : (l == 0.f ? 0.f : 1.f / l);
#pragma unroll 1
      for (int cc = 0; cc < D / 32; ++cc) {
        float o[32];
        if (steps > 0) {
          tc_ld32(o_addr + cc * 32, o);
          tc_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0.f;
        }
        put(o, cc * 32, f);
      }
      put_sums(m, l);
    } else if (shared) {
      // the two halves of the keys: both accumulators lie in the same lanes, so only references and sums are handed over (through the
      // second query tile's place, which a single does not use); each warpgroup finishes half of the columns
      const uint32_t stat = base + Y::kOffQ + kTile + (uint32_t)row * 8;
      if (!ok) l = -1.f;                                   // (no sum is negative)
      asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(stat + (uint32_t)qt * 1024), "f"(m), "f"(l) : "memory");
      tc_fence_before();
      asm volatile("bar.sync 2, 256;" ::: "memory");
      tc_fence_after();
      float m2, l2;
      asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(m2), "=f"(l2) : "r"(stat + (uint32_t)(qt ^ 1) * 1024) : "memory");
      const float top = fmaxf(m, m2);
      const float f1 = l == 0.f ? 0.f : ex2(m - top), f2 = l2 == 0.f ? 0.f : ex2(m2 - top), sum = l * f1 + l2 * f2;
      const float f = split ? 1.f : (sum == 0.f ? 0.f : 1.f / sum);
      if (__all_sync(0xffffffffu, !(l < 0.f || l2 < 0.f))) {
#pragma unroll 1
        for (int cc = 0; cc < D / 64; ++cc) {
          const int col = qt * (D / 2) + cc * 32;
          float x[32], y[32];
          tc_ld32(o_addr + col, x);
          tc_ld32(lane_addr + kColO + (qt ^ 1) * 128 + col, y);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = x[i] * f1 + y[i] * f2;
          put(x, col, f);
        }
        if (qt == 0) put_sums(top, sum);
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

// O = sum_e 2^(m_e - M) O_e / sum_e 2^(m_e - M) l_e, M the largest reference, of the items that several CTAs share: a warp to each row.  Once a wait has given
// up (ever: the status is sticky), parts may be missing and old ones lie in their places: nothing is stored then.
constexpr int kJoinRows = 8;
template <int D>
__global__ void __launch_bounds__(32 * kJoinRows) paged_join_kernel(const __grid_constant__ AttendArgs a, const Cut cut) {
  constexpr int kPer = D / 32, kBlocks = kItemRows / kJoinRows;
  const int lane = threadIdx.x & 31, r = blockIdx.x % kBlocks * kJoinRows + (threadIdx.x >> 5), shared_item = blockIdx.x / kBlocks, parts = cut.parts.d;
  const int at_item = cut.n_full + shared_item, e0 = cut.heads.div(at_item), head = at_item - e0 * cut.heads.d;
  wait_for_grid();
  next_grid();
  const bool complete = __ldcg(a.s.status) != kDevTimeout;
  const size_t row0 = (size_t)shared_item * parts * kItemRows + r;
  float m = -INFINITY;
  for (int e = lane; e < parts; e += 32) m = fmaxf(m, __ldcg(a.part_ml + (row0 + (size_t)e * kItemRows) * 2));
  const Item it = find_item(a, cut.n_items - 1 - e0);
  if (it.seq < 0) return;
  const int start = it.start, all = it.n_new * a.group.d, i = it.tile * kItemRows + r;
  if (i >= all) return;
  float sum = 0.f, acc[kPer];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
  for (int c = 0; c < kPer; ++c) acc[c] = 0.f;
#pragma unroll 8
  for (int e = 0; e < parts; ++e) {
    const size_t at = row0 + (size_t)e * kItemRows;
    const float2 ml = __ldcg(reinterpret_cast<const float2 *>(a.part_ml + at * 2));
    const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - m);
    sum += f * ml.y;
    float v[kPer];
    if constexpr (kPer == 4) *reinterpret_cast<float4 *>(v) = __ldcg(reinterpret_cast<const float4 *>(a.part_o + at * D + lane * kPer));
    else *reinterpret_cast<float2 *>(v) = __ldcg(reinterpret_cast<const float2 *>(a.part_o + at * D + lane * kPer));
#pragma unroll
    for (int c = 0; c < kPer; ++c) acc[c] += f * v[c];
  }
  if (!complete) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int t = a.group.div(i), h = head * a.group.d + i - t * a.group.d;
  char *out = a.O.ptr + (start + t) * a.O.st + h * a.O.sh + lane * kPer * 2;
#pragma unroll
  for (int c = 0; c < kPer; c += 2) *reinterpret_cast<uint32_t *>(out + c * 2) = pack_bf16(acc[c] * inv, acc[c + 1] * inv);
  if (lane == 0 && a.lse != nullptr) a.lse[(size_t)(start + t) * a.n_heads + h] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
}

// The tensor maps of a pool's rows, made once.
struct TileMaps {
  CUtensorMap k, v;
  bool make(void *k_rows, void *v_rows, long long pages, int heads, int page_tokens, int head_dim, bool q8, std::string &err) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || !fn) {
      err = "cuTensorMapEncodeTiled not available";
      return false;
    }
    const auto encode = reinterpret_cast<CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                                      const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill)>(fn);
    const size_t row = (size_t)head_dim * (q8 ? 1 : 2);
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads * page_tokens, (cuuint64_t)pages};
    const cuuint64_t strides[2] = {row, row * heads * page_tokens};
    const cuuint32_t box[3] = {(cuuint32_t)(q8 ? head_dim : 64), (cuuint32_t)(page_tokens < kTileKeys ? page_tokens : kTileKeys), 1}, step[3] = {1, 1, 1};
    for (int i = 0; i < 2; ++i) {
      const CUresult r = encode(i ? &v : &k, q8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, i ? v_rows : k_rows, dims, strides, box,
                                step, CU_TENSOR_MAP_INTERLEAVE_NONE, q8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
      if (r != CUDA_SUCCESS) {
        err = "cuTensorMapEncodeTiled(pool) failed with code " + std::to_string((int)r);
        return false;
      }
    }
    return true;
  }
};

}  // namespace paged
}  // namespace scalekv
