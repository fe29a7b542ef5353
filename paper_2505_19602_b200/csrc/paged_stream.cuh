// Attention of few query rows over the paged token cache: single tokens above all.
//
//   y_j = scale <q, k_j>,  lse = log sum_j exp(y_j),  O = sum_j exp(y_j - lse) v_j   over the keys j that the row sees.
//
// A kv head's query rows, the group's heads of every new token, share its keys: row r is head r mod G of token r / G; a CTA has up to 16 of them.
// What bounds it is reading the keys and values once: 2 (d + 4) bytes a key as codes, 4 d as bf16, against 8 d products a key and row.
// So every warp streams its own share of the cache, 16 keys (which lie in one page) at a time, through a ring of stages in shared memory that it
// fills with asynchronous copies and shares with nobody: no barrier before the end, and the loads of a few steps are always under way.
// (With the loads in registers, half a step ahead, a step took a loaded DRAM latency: 32 sequences of up to 10 521 entries, 8 kv heads in codes, 285 us for
// what is 115.)  Products are m16n8k16 with the few query rows as the n-tiles of eight, S^T = K Q^T (keys x rows x dims) and O^T = V^T P^T
// (dims x rows x keys): of an m-tile of query rows most would be padding, in the products and in the exponentials.
//   - A lane has keys r and r + 8 (r = lane / 4) of K, as the A operand does, and since a product's sum may run in any order, it takes the dims that lie in its
//     16-byte pieces; the queries, which stay in registers, are read in the same order.
//   - P is transposed from where the first product leaves it to where the second wants it by movmatrix.
//   - V's pairs of keys are interleaved from two rows' pieces, and its dims are dealt to the m-tiles so that those are 16 bytes long, too.
//   - Pieces are placed in a stage so that eight lanes' loads meet all banks, K's (two rows, four pieces) and V's (four rows, two pieces).
//   - Codes become bf16 exactly (codes_bf16).  The key's scale multiplies the product, the value's scale multiplies P, both in fp32; P goes into its
//     product in two pieces of bf16.
// The running maximum of a row is raised when a step exceeds it by more than 2^3, and the sums with it: P stays below that.
// A CTA's four warps take the steps in turn and are combined in shared memory.  Where a sequence's heads are few, gridDim.z CTAs share its
// keys; each leaves its part in the workspace, and the last one to do so, by a counter that it sets back, combines them in their order.
// 32 sequences of up to 10 521 entries, 32 heads, 8 kv heads in codes: 114 us, 4.4 TB/s of 6.46 measured; SMs that still have work read 21 of 23.6 bytes a cycle and issue in
// 55 of 100; the rest is beginnings, ends and what is left of balance.  One sequence of 170 521 bf16 entries, 16 heads: 228 us, 6.1 TB/s.
#pragma once
#include <cfloat>
#include <cmath>

#include "paged_store.cuh"
#include "stream_cut.h"

namespace scalekv {
namespace paged {

constexpr int kStreamThreads = 32 * kStreamWarps;
constexpr int kStreamRows = 32;                   // query rows of a sequence and kv head that go this way
constexpr int kTileRows = 16;                     // of them a CTA takes so many, at most

// kN: n-tiles of eight query rows
template <int D, bool kQ8, int kN>
struct StreamLayout {
  static constexpr int kRowBytes = D * (kQ8 ? 1 : 2);
  static constexpr int kStages = kRowBytes >= 128 ? 3 : 4;
  static constexpr int kCtas = stream_ctas(D, kQ8, kN);
  static constexpr int kScales = 32 * kRowBytes;                                  // offsets in a stage: K rows, V rows, the scales of both
  static constexpr int kStage = kScales + (kQ8 ? 128 : 0);
  static constexpr int kRing = kStreamWarps * kStages * kStage;
  static constexpr int kParts = kStreamWarps * 8 * kN * (D + 2) * 4;              // the warps' sums, over the ring once that is done with
  // the parts of a sequence and head that the last CTA combines: references and sums of every row, and sums of groups of threads
  static constexpr int kJoin = 8 * kN * (kMostParts + 1) * 8 + 8 + kStreamThreads * 32;
  static constexpr int kSmem = kRing > kParts ? (kRing > kJoin ? kRing : kJoin) : (kParts > kJoin ? kParts : kJoin);
  // where piece x (16 bytes) of row r lies
  static __device__ __forceinline__ int piece(int r, int x) {
    if (kRowBytes == 64) return r * 64 + ((x ^ ((r >> 1) & 3)) << 4);
    return r * kRowBytes + ((x ^ ((r & 6) ^ ((r & 1) << 2))) << 4);
  }
};
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRaise = 3.f;

struct Mask {
  int causal, window, n_sink;      // window 0: none
};

struct AttendArgs {
  Store s;
  Batch bt;
  Rows Q, O;                       // [tokens][heads][head_dim] bf16
  float *lse;                      // [tokens][heads] or null
  float *part_o, *part_ml;         // parts of rows that CTAs share: columns, and base-2 reference and sum
  int *counts;                     // parts left so far, one for each sequence and kv head (and 16 rows) of a launch; zero between launches
  Mask mask;
  Divisor group;                   // query heads of a kv head
  int n_heads;                     // query heads
  int max_new;                     // new tokens of a sequence that the launch was sized for
  float scale_log2e;
};

// Keys that the query at position p of a sequence of `length` entries sees: [lo, hi) and [0, min(n_sink, lo)).
__device__ __forceinline__ int seen_hi(const Mask &m, int p, int length) { return m.causal ? max(min(p + 1, length), 0) : length; }
__device__ __forceinline__ int seen_lo(const Mask &m, int p) { return m.window > 0 ? max(p - m.window + 1, 0) : 0; }

// Codes as bf16, exactly and without a conversion instruction: a byte u = c + 128 (the code with its sign bit turned) alone in 16 bits is the
// subnormal u 2^-133, so one fused multiply-add gives u 2^-133 2^127 - 2 = c 2^-6.  The 2^6 goes into the factor that the scale is anyway.
constexpr float kCodeUnit = 64.f;
__device__ __forceinline__ uint32_t turn_signs(uint32_t w) { return w ^ 0x80808080u; }
__device__ __forceinline__ uint32_t codes_bf16(uint32_t two) {                    // two such bytes, each in 16 bits
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(two), "r"(0x7f007f00u), "r"(0xc000c000u));
  return r;
}
__device__ __forceinline__ uint32_t codes_low(uint32_t w) { return codes_bf16(__byte_perm(w, 0u, 0x4140)); }      // of a word's four the first two
__device__ __forceinline__ uint32_t codes_high(uint32_t w) { return codes_bf16(__byte_perm(w, 0u, 0x4342)); }
template <int kByte> __device__ __forceinline__ uint32_t codes_across(uint32_t a, uint32_t b) {                   // the same byte of two words, signs as they are
  return codes_bf16((__byte_perm(a, b, 0x0400 + kByte * 0x0101) ^ 0x00800080u) & 0x00ff00ffu);
}

__device__ __forceinline__ void mma_16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// What a sequence has to do with a launch: its query rows of a kv head, and the keys that some of them see, in steps of 16: the sinks' steps,
// then those of [lo, hi).
struct Span {
  int start, rows, length, first, lo, hi, n_sink, lo_step, sink_steps, steps;
  __device__ __forceinline__ Span(const AttendArgs &a, int seq, int most_rows, bool tell) {
    start = a.bt.starts[seq];
    length = a.bt.lengths[seq];
    const int end = a.bt.starts[seq + 1], n_new = min(end, a.bt.n_tokens) - start, room = a.bt.table_pages << a.s.page_shift;
    if (tell && (starts_wrong(a.bt, seq, start, end) || n_new > a.max_new || (unsigned)length > (unsigned)room)) report(a.s.status);
    length = max(min(length, room), 0);                    // (what lies behind the table counts as hidden)
    first = length - n_new;                                // position of the sequence's first new token
    rows = start < 0 || n_new <= 0 ? 0 : min(n_new * a.group.d, most_rows);
    const int t_last = a.group.div(max(rows - 1, 0));
    lo = min(seen_lo(a.mask, first), length);
    hi = seen_hi(a.mask, first + t_last, length);
    n_sink = a.mask.window > 0 ? a.mask.n_sink : 0;
    lo_step = lo >> 4;
    sink_steps = min((min(n_sink, hi) + 15) >> 4, lo_step);
    steps = rows > 0 ? sink_steps + max((hi + 15) >> 4, lo_step) - lo_step : 0;
  }
};

// [row of 8][pair of columns] in the lanes -> [column][pair of rows]
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
// 16 bytes from global to shared memory, or zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}

// Token and query head of row r of a sequence and kv head.
__device__ __forceinline__ void place_row(const AttendArgs &a, int start, int head, int r, int &t, int &h) {
  t = a.group.div(r);
  h = head * a.group.d + r - t * a.group.d;
  t += start;
}
// 8 columns of a row, normalised, and with the first of them its log-sum-exp; ml: reference and sum.
__device__ __forceinline__ void put_row(const AttendArgs &a, int t, int h, int piece, const float *acc, float2 ml) {
  const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
  *(reinterpret_cast<uint4 *>(a.O.ptr + t * a.O.st + h * a.O.sh) + piece) =
      make_uint4(tc::pack_bf16(acc[0] * inv, acc[1] * inv), tc::pack_bf16(acc[2] * inv, acc[3] * inv), tc::pack_bf16(acc[4] * inv, acc[5] * inv), tc::pack_bf16(acc[6] * inv, acc[7] * inv));
  if (piece == 0 && a.lse != nullptr) a.lse[(size_t)t * a.n_heads + h] = ml.y == 0.f ? -INFINITY : (ml.x + log2f(ml.y)) * kLn2;
}

// What the last CTA of a sequence and kv head does: references and sums of all parts side by side, a weight for each (a row's by one warp), then the parts'
// columns, dealt to as many groups of threads as there are.  (One part after the other, three loads each, cost 0.2 us a part.)  A function of its own, so that
// the streaming loop is compiled without it: inlined it made that 5 to 10 % longer.
template <int D, int kRows>
__device__ __noinline__ void join_parts(const AttendArgs &a, int start, int row0, int rows, int head, int parts, char *smem) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const size_t all_rows = (size_t)a.bt.n_tokens * a.n_heads;
  float2 *row_ml = reinterpret_cast<float2 *>(smem), *ml = row_ml + kRows;      // [row]; [row][part]
  for (int i = threadIdx.x; i < rows * parts; i += kStreamThreads) {
    const int r = i / parts;
    int t, h;
    place_row(a, start, head, row0 + r, t, h);
    ml[i] = __ldcg(reinterpret_cast<const float2 *>(a.part_ml + ((size_t)(i - r * parts) * all_rows + (size_t)t * a.n_heads + h) * 2));
  }
  __syncthreads();
  for (int r = warp; r < rows; r += kStreamWarps) {
    float top = -INFINITY, sum = 0.f;
    for (int e = lane; e < parts; e += 32) top = fmaxf(top, ml[r * parts + e].x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    for (int e = lane; e < parts; e += 32) {
      const float2 x = ml[r * parts + e];
      const float f = tc::ex2(x.x - top);
      sum += f * x.y;
      ml[r * parts + e].x = f;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    __syncwarp();
    if (lane == 0) row_ml[r] = make_float2(top, sum);
  }
  __syncthreads();
  const int pieces = rows * (D / 8), groups = max(1, kStreamThreads / pieces);
  float4 *sums = reinterpret_cast<float4 *>(ml + rows * parts + (rows * parts & 1));      // [group][piece][2]
  for (int i = threadIdx.x; i < groups * pieces; i += kStreamThreads) {
    const int group = i / pieces, j = i - group * pieces, r = j / (D / 8), piece = j % (D / 8);
    int t, h;
    place_row(a, start, head, row0 + r, t, h);
    const float *columns = a.part_o + ((size_t)t * a.n_heads + h) * D + piece * 8;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int e = group; e < parts; e += groups) {
      const float4 *v = reinterpret_cast<const float4 *>(columns + (size_t)e * all_rows * D);
      const float4 lo = __ldcg(v), hi = __ldcg(v + 1);
      const float f = ml[r * parts + e].x;
      acc[0] += f * lo.x; acc[1] += f * lo.y; acc[2] += f * lo.z; acc[3] += f * lo.w;
      acc[4] += f * hi.x; acc[5] += f * hi.y; acc[6] += f * hi.z; acc[7] += f * hi.w;
    }
    if (groups == 1) {
      put_row(a, t, h, piece, acc, row_ml[r]);
    } else {
      sums[i * 2] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      sums[i * 2 + 1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
  }
  __syncthreads();
  if (groups > 1 && (int)threadIdx.x < pieces) {
    const int r = threadIdx.x / (D / 8), piece = threadIdx.x % (D / 8);
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < groups; ++g) {
      const float4 lo = sums[(g * pieces + threadIdx.x) * 2], hi = sums[(g * pieces + threadIdx.x) * 2 + 1];
      acc[0] += lo.x; acc[1] += lo.y; acc[2] += lo.z; acc[3] += lo.w;
      acc[4] += hi.x; acc[5] += hi.y; acc[6] += hi.z; acc[7] += hi.w;
    }
    int t, h;
    place_row(a, start, head, row0 + r, t, h);
    put_row(a, t, h, piece, acc, row_ml[r]);
  }
  __syncthreads();                                         // (what was the ring may be one again)
}

// One part of rows row0 .. of a sequence and kv head (item: a number of their own): steps step_lo .. step_hi - 1 of it, as part number `part` of `parts`.  All threads of the CTA.
template <int D, bool kQ8, int kN>
__device__ __forceinline__ void stream_part(const AttendArgs &a, const Span &sp, char *smem, int *shared_word, int seq, int head, int row0, int item, int step_lo, int step_hi,
                                            int part, int parts) {
  using Y = StreamLayout<D, kQ8, kN>;
  constexpr int kRowBytes = Y::kRowBytes, kStages = Y::kStages;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, oct = lane >> 2;
  const Store &s = a.s;
  const int start = sp.start, rows = min(sp.rows - row0, 8 * kN), length = sp.length, first = sp.first, n_sink = sp.n_sink;      // (rows row0 .. of the sequence's)
  auto in_use = [&](int pos) { return pos < sp.hi && (pos >= sp.lo || pos < n_sink); };
  auto key_of = [&](int step) { return (step < sp.sink_steps ? step : step - sp.sink_steps + sp.lo_step) << 4; };
  auto page_at = [&](int step) { return step < step_hi ? page_of(s, a.bt, seq, key_of(step)) : -1; };

  // ---- the ring: this warp's steps are step_lo + warp, + 4, ..
  char *ring = smem + warp * kStages * Y::kStage;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  auto fetch = [&](int step, int page, int stage) {
    if (page >= 0) {
      constexpr int kRowPieces = kRowBytes / 16, kRowsAtOnce = 32 / kRowPieces;
      const int key0 = key_of(step), x = lane % kRowPieces, r0 = lane / kRowPieces;
      const size_t row = store_row(s, page, head, key0);
      const char *k = s.k_rows + (row + r0) * kRowBytes + x * 16, *v = s.v_rows + (row + r0) * kRowBytes + x * 16;
      const uint32_t to = ring_at + stage * Y::kStage;
#pragma unroll
      for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
        const int r = r0 + i * kRowsAtOnce;
        // (hidden keys' products are hidden one by one, and codes are numbers whatever they are; hidden rows of bf16 values must be)
        copy16(to + Y::piece(r, x), k + i * kRowsAtOnce * kRowBytes, true);
        copy16(to + 16 * kRowBytes + Y::piece(r, x), v + i * kRowsAtOnce * kRowBytes, kQ8 || in_use(key0 + r));
      }
      if (kQ8 && lane < 8) copy16(to + Y::kScales + lane * 16, (lane < 4 ? s.k_scales : s.v_scales) + row + (lane & 3) * 4, true);
    } else if (!kQ8 && step < step_hi) {
      for (int i = lane; i < 32 * kRowBytes / 16; i += 32) *reinterpret_cast<uint4 *>(ring + stage * Y::kStage + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int step = step_lo + warp, pages[kStages];               // of this step and those behind it
#pragma unroll
  for (int i = 0; i < kStages; ++i) pages[i] = page_at(step + i * kStreamWarps);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(step + i * kStreamWarps, pages[i], i);

  // the queries of row oct of every n-tile, zeros beyond the last one, in the order in which a lane has K's dims: four for each product
  uint2 q[kN][D / 16];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const int r = n * 8 + oct, t = a.group.div(row0 + r), g = row0 + r - t * a.group.d;
    const char *row = a.Q.ptr + (start + t) * a.Q.st + (head * a.group.d + g) * a.Q.sh;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int dim = kQ8 ? (k >> 2) * 64 + quad * 16 + (k & 3) * 4 : (k >> 1) * 32 + quad * 8 + (k & 1) * 4;
      q[n][k] = r < rows ? *reinterpret_cast<const uint2 *>(row + dim * 2) : make_uint2(0u, 0u);
    }
  }
  // a step all of whose keys every row sees: [lo_full, hi_full)
  const int lo_full = seen_lo(a.mask, first + a.group.div(row0 + rows - 1)), hi_full = seen_hi(a.mask, first + a.group.div(row0), length);

  // O^T: rows 2 quad, 2 quad + 1 of every n-tile; references and sums of those rows (the sum over this lane's keys)
  float o[D / 16][kN][4], m[kN][2], l[kN][2];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
    m[n][0] = m[n][1] = -FLT_MAX;                          // (the lowest number: differences from it are numbers)
    l[n][0] = l[n][1] = 0.f;
  }

  for (int stage = 0; step < step_hi; step += kStreamWarps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();                                          // everybody's copies of this step are there, and the stage before it is done with
    fetch(step + (kStages - 1) * kStreamWarps, pages[kStages - 1], stage == 0 ? kStages - 1 : stage - 1);
    const int key0 = key_of(step), page = pages[0];
#pragma unroll
    for (int i = 0; i + 1 < kStages; ++i) pages[i] = pages[i + 1];
    pages[kStages - 1] = page_at(step + kStages * kStreamWarps);
    const char *k_at = ring + stage * Y::kStage, *v_at = k_at + 16 * kRowBytes;
    stage = stage + 1 == kStages ? 0 : stage + 1;
    // S^T = K Q^T
    float x[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll
    for (int i = 0; i < kRowBytes / 64; ++i) {
      const uint4 lo = *reinterpret_cast<const uint4 *>(k_at + Y::piece(oct, i * 4 + quad)), hi = *reinterpret_cast<const uint4 *>(k_at + Y::piece(oct + 8, i * 4 + quad));
      if constexpr (kQ8) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t w0 = turn_signs(word(lo, w)), w1 = turn_signs(word(hi, w));
          const uint32_t f[4] = {codes_low(w0), codes_low(w1), codes_high(w0), codes_high(w1)};
#pragma unroll
          for (int n = 0; n < kN; ++n) mma_16816(x[n], f, q[n][4 * i + w].x, q[n][4 * i + w].y);
        }
      } else {
        const uint32_t f0[4] = {lo.x, hi.x, lo.y, hi.y}, f1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          mma_16816(x[n], f0, q[n][2 * i].x, q[n][2 * i].y);
          mma_16816(x[n], f1, q[n][2 * i + 1].x, q[n][2 * i + 1].y);
        }
      }
    }
    // base-2 exponents; hidden keys at -inf, whatever their rows and scales hold
    float ks0 = a.scale_log2e, ks1 = a.scale_log2e, vs0 = 1.f, vs1 = 1.f;
    if constexpr (kQ8) {
      const float *scales = reinterpret_cast<const float *>(k_at + Y::kScales) + oct;
      ks0 *= kCodeUnit * scales[0]; ks1 *= kCodeUnit * scales[8];
      vs0 = kCodeUnit * scales[16]; vs1 = kCodeUnit * scales[24];
    }
#pragma unroll
    for (int n = 0; n < kN; ++n) { x[n][0] *= ks0; x[n][1] *= ks0; x[n][2] *= ks1; x[n][3] *= ks1; }
    const bool whole = page >= 0 && key0 >= lo_full && key0 + 16 <= hi_full;
    uint32_t hidden = 0;
    if (!whole) {
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = first + a.group.div(row0 + min(n * 8 + 2 * quad + (e & 1), rows - 1)), pos = key0 + oct + 8 * (e >> 1);
          if (page < 0 || pos >= seen_hi(a.mask, t, length) || (pos < seen_lo(a.mask, t) && pos >= n_sink)) {
            x[n][e] = -INFINITY;
            hidden |= 1u << (4 * n + e);
          }
        }
    }
    // the rows' references
    bool rise = false;
#pragma unroll
    for (int n = 0; n < kN; ++n) rise = rise || fmaxf(x[n][0], x[n][2]) > m[n][0] + kRaise || fmaxf(x[n][1], x[n][3]) > m[n][1] + kRaise;
    if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float raised = fmaxf(fmaxf(x[n][e], x[n][2 + e]), m[n][e]);
#pragma unroll
          for (int d = 4; d < 32; d *= 2) raised = fmaxf(raised, __shfl_xor_sync(0xffffffffu, raised, d));
          const float f = tc::ex2(m[n][e] - raised);
          m[n][e] = raised;
          l[n][e] *= f;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) { o[i][n][e] *= f; o[i][n][2 + e] *= f; }
        }
    }
    // P in two pieces, what bf16 has of it and what it leaves: rounded once, it would put as much error into a row of O as O's own rounding does, and the
    // products cost little beside the loads
    uint32_t p[kN][2], rest[kN][2];
#pragma unroll
    for (int n = 0; n < kN; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[n][e] = tc::ex2(x[n][e] - m[n][e & 1]);
        l[n][e & 1] += x[n][e];
      }
      float y[4] = {x[n][0] * vs0, x[n][1] * vs0, x[n][2] * vs1, x[n][3] * vs1};
      if (kQ8 && !whole) {                                 // (a hidden value counts for nothing even where its scale is no number)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((hidden >> (4 * n + e)) & 1u) y[e] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t most = tc::pack_bf16(y[2 * i], y[2 * i + 1]);
        p[n][i] = transpose_8x8(most);
        rest[n][i] = transpose_8x8(tc::pack_bf16(y[2 * i] - __uint_as_float(most << 16), y[2 * i + 1] - __uint_as_float(most & 0xffff0000u)));
      }
    }
    // O^T += V^T P^T
#pragma unroll
    for (int i = 0; i < (kRowBytes >= 128 ? kRowBytes / 128 : 1); ++i) {
      uint4 v[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int r = (n >> 1) * 8 + 2 * quad + (n & 1);
        if constexpr (kRowBytes >= 128) {
          v[n] = *reinterpret_cast<const uint4 *>(v_at + Y::piece(r, i * 8 + oct));
        } else {
          const uint2 two = *reinterpret_cast<const uint2 *>(v_at + Y::piece(r, oct >> 1) + (oct & 1) * 8);
          v[n] = make_uint4(two.x, two.y, 0u, 0u);
        }
      }
      if constexpr (kQ8) {
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          const uint32_t c0 = word(v[0], w), c1 = word(v[1], w), c2 = word(v[2], w), c3 = word(v[3], w);
          const uint32_t f0[4] = {codes_across<0>(c0, c1), codes_across<1>(c0, c1), codes_across<0>(c2, c3), codes_across<1>(c2, c3)};
          const uint32_t f1[4] = {codes_across<2>(c0, c1), codes_across<3>(c0, c1), codes_across<2>(c2, c3), codes_across<3>(c2, c3)};
#pragma unroll
          for (int n = 0; n < kN; ++n) {
            mma_16816(o[2 * w][n], f0, p[n][0], p[n][1]);
            mma_16816(o[2 * w + 1][n], f1, p[n][0], p[n][1]);
            mma_16816(o[2 * w][n], f0, rest[n][0], rest[n][1]);
            mma_16816(o[2 * w + 1][n], f1, rest[n][0], rest[n][1]);
          }
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t c0 = word(v[0], w), c1 = word(v[1], w), c2 = word(v[2], w), c3 = word(v[3], w);
          const uint32_t f[4] = {__byte_perm(c0, c1, 0x5410), __byte_perm(c0, c1, 0x7632), __byte_perm(c2, c3, 0x5410), __byte_perm(c2, c3, 0x7632)};
#pragma unroll
          for (int n = 0; n < kN; ++n) {
            mma_16816(o[4 * i + w][n], f, p[n][0], p[n][1]);
            mma_16816(o[4 * i + w][n], f, rest[n][0], rest[n][1]);
          }
        }
      }
    }
  }

  // ---- the warps' parts, combined over what was the ring
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  constexpr int kRows = 8 * kN;
  float *o_smem = reinterpret_cast<float *>(smem), *ml_smem = o_smem + kStreamWarps * kRows * D;      // [warp][row][dim], [warp][row][2]
#pragma unroll
  for (int n = 0; n < kN; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float sum = l[n][e];
#pragma unroll
      for (int d = 4; d < 32; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      const int r = n * 8 + 2 * quad + e;
      if (oct == 0) *reinterpret_cast<float2 *>(ml_smem + (warp * kRows + r) * 2) = make_float2(m[n][e], sum);
      // an m-tile's rows oct and oct + 8 are neighbouring dims of the lane's piece
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int dim = kQ8 ? oct * (D / 8) + 2 * i : (i >> 2) * 64 + oct * 8 + 2 * (i & 3);
        *reinterpret_cast<float2 *>(o_smem + (warp * kRows + r) * D + dim) = make_float2(o[i][n][e], o[i][n][2 + e]);
      }
    }
  __syncthreads();
  const size_t all_rows = (size_t)a.bt.n_tokens * a.n_heads;
  auto place = [&](int r, int &t, int &h) { place_row(a, start, head, row0 + r, t, h); };
  for (int i = threadIdx.x; i < rows * (D / 8); i += kStreamThreads) {
    const int r = i / (D / 8), piece = i % (D / 8);
    float acc[8], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) top = fmaxf(top, ml_smem[(w * kRows + r) * 2]);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) {
      const float2 x = *reinterpret_cast<const float2 *>(ml_smem + (w * kRows + r) * 2);
      const float f = tc::ex2(x.x - top);
      sum += f * x.y;
      const float4 *v = reinterpret_cast<const float4 *>(o_smem + (w * kRows + r) * D + piece * 8);
      const float4 lo = v[0], hi = v[1];
      acc[0] += f * lo.x; acc[1] += f * lo.y; acc[2] += f * lo.z; acc[3] += f * lo.w;
      acc[4] += f * hi.x; acc[5] += f * hi.y; acc[6] += f * hi.z; acc[7] += f * hi.w;
    }
    const float2 ml = make_float2(top, sum);
    int t, h;
    place(r, t, h);
    if (parts == 1) {
      put_row(a, t, h, piece, acc, ml);
    } else {
      const size_t at = (size_t)part * all_rows + (size_t)t * a.n_heads + h;
      float4 *dst = reinterpret_cast<float4 *>(a.part_o + at * D + piece * 8);
      dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (piece == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = ml;
    }
  }
  if (parts > 1) __threadfence();
  __syncthreads();                                         // (also: what was the ring may be one again)
  if (parts == 1) return;
  if (threadIdx.x == 0) {
    const int last = atomicAdd(a.counts + item, 1) == parts - 1;
    if (last) a.counts[item] = 0;
    *shared_word = last;
  }
  __syncthreads();
  const bool last = *shared_word != 0;
  __syncthreads();
  if (!last) return;
  __threadfence();
  join_parts<D, 8 * kN>(a, start, row0, rows, head, parts, smem);
}

template <int D, bool kQ8, int kN>
__global__ void __launch_bounds__(kStreamThreads, StreamLayout<D, kQ8, kN>::kCtas) paged_stream_kernel(const __grid_constant__ AttendArgs a, int most_parts, int tiles) {
  using Y = StreamLayout<D, kQ8, kN>;
  extern __shared__ __align__(16) char smem[];
  __shared__ int shared_word;
  const int lane = threadIdx.x & 31;
  wait_for_grid();
  // Either a CTA to each part of a sequence and kv head, as the grid says, or (most_parts > 0) by what the lengths turn out to be: as many equal parts of
  // each as there are CTAs for; or, where that would leave the longest ones' parts too long, the steps of all of them one behind the other and an equal share to
  // every CTA, which may begin and end within a sequence.  That costs a CTA a second beginning and end: kSecond steps.  (At least one step to whoever has
  // rows, so that it is met; no more than most_parts shares to a sequence and head.)
  // Rows beyond the first kTileRows are a CTA's of their own, as if they were another head; `tiles` of them to a kv head.
  const int heads = a.s.heads * tiles, most_rows = tiles > 1 ? tiles * kTileRows : 8 * kN;
  auto weight = [&](int b, bool tell) {
    if (b >= a.bt.n_seqs) return 0u;                       // (32 of at most 2^26 steps each: sums of them need all 32 bits)
    const Span sp(a, b, most_rows, tell);
    return sp.rows > 0 ? (unsigned)max(sp.steps, 1) : 0u;
  };
  long long at = 0, end = 1;
  int share = 0, split = gridDim.z;                        // share 0: parts
  int seq = blockIdx.x, head = blockIdx.y, part = blockIdx.z;
  if (most_parts > 0) {
    long long total = 0;
    int longest = 1;
    for (int b0 = 0; b0 < a.bt.n_seqs; b0 += 32) {
      const unsigned w = weight(b0 + lane, blockIdx.x == 0 && threadIdx.x < 32);
      total += __reduce_add_sync(0xffffffffu, w);
      longest = max(longest, (int)__reduce_max_sync(0xffffffffu, w));
    }
    total *= heads;
    const int ctas = gridDim.x, items = a.bt.n_seqs * heads;
    const StreamDeal deal = deal_steps(total, longest, items, ctas, most_parts);
    split = deal.split;
    share = deal.share;
    if (share == 0) {
      at = blockIdx.x;
      end = (long long)items * split;
    } else {
      at = (long long)blockIdx.x * share;
      end = min(at + share, total);
    }
  }
  while (at < end) {
    int parts = split, lo, hi;
    long long next = at + gridDim.x, from = 0;             // where this CTA goes on; of the sequence and head the first step
    if (share > 0) {
      long long before = 0;                                // steps of the sequences ahead of b0
      unsigned w = 0, incl = 0, behind = 0;
      int b0 = 0;
      for (; b0 < a.bt.n_seqs; b0 += 32) {
        incl = w = weight(b0 + lane, false);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned up = __shfl_up_sync(0xffffffffu, incl, d);
          if (lane >= d) incl += up;
        }
        behind = __ballot_sync(0xffffffffu, before + (long long)incl * heads > at);
        if (behind) break;
        before += (long long)__shfl_sync(0xffffffffu, incl, 31) * heads;
      }
      const int src = __ffs(behind) - 1, steps = (int)__shfl_sync(0xffffffffu, w, src);
      from = before + (long long)__shfl_sync(0xffffffffu, incl - w, src) * heads;
      seq = b0 + src;
      head = (int)((at - from) / steps);
      from += (long long)head * steps;
      next = min(from + steps, end);
      part = (int)(at / share - from / share);
      parts = (int)((from + steps - 1) / share - from / share) + 1;
    } else if (most_parts > 0) {
      part = (int)at % split;
      head = (int)at / split % heads;
      seq = (int)at / split / heads;
    }
    const Span sp(a, seq, most_rows, most_parts == 0 && threadIdx.x == 0);
    if (share > 0) {
      lo = (int)(at - from);
      hi = min((int)(next - from), sp.steps);
    } else {
      lo = (int)((long long)sp.steps * part / parts);
      hi = (int)((long long)sp.steps * (part + 1) / parts);
    }
    const int real_head = head / tiles, row0 = (head - real_head * tiles) * kTileRows;
    if (sp.rows > row0) stream_part<D, kQ8, kN>(a, sp, smem, &shared_word, seq, real_head, row0, seq * heads + head, lo, hi, part, parts);
    at = next;
  }
  next_grid();
}

}  // namespace paged
}  // namespace scalekv
