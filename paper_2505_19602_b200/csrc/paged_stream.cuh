// Attention of few query rows over the paged token cache: single tokens above all.
//
//   y_j = scale <q, k_j>,  lse = log sum_j exp(y_j),  O = sum_j exp(y_j - lse) v_j   over the keys j that the row sees.
//
// A kv head's query rows, the group's heads of every new token, share its keys: row r is head r mod G of token r / G, 16 rows a tile.
// What bounds it is reading the keys and values once: 2 (d + 4) bytes a key as codes, 4 d as bf16, against 8 d products a key and row.
// So a warp streams its share of the cache from global memory straight into the registers of the matrix instructions (m16n8k16, rows x keys x
// dims), with nothing staged in shared memory and no barrier before the end:
//   - 16 keys at a time, which lie in one page.  The eight keys of an n-tile are one to each four lanes, as the B operand has them, and
//     since a product's sum may run in any order, a lane takes whichever dims make its loads 16 bytes long; the query operand is read
//     in the same order.
//   - V's pairs of keys are interleaved from rows held by the lane, and its dims are dealt to the n-tiles so that those rows are 16 bytes long, too.
//   - Codes become bf16 exactly (codes_bf16).  The key's scale multiplies the product, the value's scale multiplies P, both in fp32; P is rounded to bf16 for its product with V, as it is where rows are bf16.
//   - While one half (K or V) of a step is computed with, the other half's loads are under way.
// The running maximum of a row is raised when a step exceeds it by more than 2^3, and the sums with it: P stays below 2^8.
// A CTA's four warps take the steps in turn and are combined in shared memory; gridDim.z CTAs share a row tile's keys where there
// are few, and paged_join_kernel combines what they leave.
#pragma once
#include <cfloat>
#include <cmath>

#include "paged_view.cuh"

namespace scalekv {
namespace paged {

constexpr int kStreamThreads = 128, kStreamWarps = kStreamThreads / 32;
constexpr int kTileRows = 16;
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
  float *part_o, *part_ml;         // [split][tokens * heads][head_dim], [split][tokens * heads][2]: base-2 reference and sum
  Mask mask;
  Divisor group;                   // query heads of a kv head
  int n_heads;                     // query heads
  int max_new;                     // new tokens of a sequence that the launch was sized for
  float scale_log2e;
};

// Keys that the query at position p of a sequence of `length` entries sees: [lo, hi) and [0, min(n_sink, lo)).
__device__ __forceinline__ int seen_hi(const Mask &m, int p, int length) { return m.causal ? max(min(p + 1, length), 0) : length; }
__device__ __forceinline__ int seen_lo(const Mask &m, int p) { return m.window > 0 ? max(p - m.window + 1, 0) : 0; }

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

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
template <int kByte> __device__ __forceinline__ uint32_t codes_across(uint32_t a, uint32_t b) {                   // the same byte of two words
  return codes_bf16(__byte_perm(a, b, 0x0400 + kByte * 0x0101) & 0x00ff00ffu);
}

__device__ __forceinline__ void mma_16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint4 load_stream(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int D, bool kQ8>
__global__ void __launch_bounds__(kStreamThreads, 3) paged_stream_kernel(const AttendArgs a, int tiles) {
  constexpr int kRowBytes = D * (kQ8 ? 1 : 2);
  constexpr int kPieces = kRowBytes / 64;                // 16-byte pieces of a K row that a lane holds
  constexpr int kValPieces = kRowBytes >= 128 ? kRowBytes / 128 : 1;   // ... of a V row (half of one: 64 codes)
  constexpr int kQLd = D + 8;                            // a row of queries in shared memory: 16 bytes more against bank conflicts
  __shared__ __align__(16) __nv_bfloat16 q_smem[kTileRows * kQLd];
  __shared__ float o_smem[kStreamWarps][kTileRows][D];
  __shared__ float ml_smem[kStreamWarps][kTileRows][2];

  const int seq = blockIdx.x / tiles, tile = blockIdx.x - seq * tiles, head = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, oct = lane >> 2;
  const Store &s = a.s;
  const int start = __ldg(a.bt.starts + seq), n_new = min(__ldg(a.bt.starts + seq + 1), a.bt.n_tokens) - start;
  const int rows = n_new * a.group.d - tile * kTileRows;   // query rows of this tile (beyond 16: of later ones too)
  if (n_new > a.max_new && threadIdx.x == 0) report(s.status);
  if (rows <= 0 || start < 0) return;
  int length = __ldg(a.bt.lengths + seq);
  if ((unsigned)length > (unsigned)(a.bt.table_pages << s.page_shift)) {       // (what lies behind the table counts as hidden)
    length = length < 0 ? 0 : a.bt.table_pages << s.page_shift;
    report(s.status);
  }
  const int first = length - n_new;                        // position of the sequence's first new token

  // query rows, zeros beyond the last one
  for (int i = threadIdx.x; i < kTileRows * (D / 8); i += kStreamThreads) {
    const int r = i / (D / 8), piece = i % (D / 8);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r < rows) {
      const int t = a.group.div(tile * kTileRows + r), g = tile * kTileRows + r - t * a.group.d;
      v = __ldg(reinterpret_cast<const uint4 *>(a.Q.ptr + (start + t) * a.Q.st + (head * a.group.d + g) * a.Q.sh) + piece);
    }
    *reinterpret_cast<uint4 *>(q_smem + r * kQLd + piece * 8) = v;
  }

  // the keys that some row of the tile sees, in steps of 16: the sinks' steps, then those of [lo, hi)
  const int t_first = a.group.div(tile * kTileRows), t_last = a.group.div(tile * kTileRows + min(rows, kTileRows) - 1);
  const int lo_all = min(seen_lo(a.mask, first + t_first), length), hi_all = seen_hi(a.mask, first + t_last, length);
  const int lo_step = lo_all >> 4, hi_step = max((hi_all + 15) >> 4, lo_step);
  const int sink_steps = a.mask.window > 0 ? min((min(a.mask.n_sink, hi_all) + 15) >> 4, lo_step) : 0;
  const int steps = sink_steps + hi_step - lo_step;
  const int step_lo = (int)((long long)steps * blockIdx.z / gridDim.z), step_hi = (int)((long long)steps * (blockIdx.z + 1) / gridDim.z);
  // a step all of whose keys every row sees: [lo_full, hi_full)
  const int lo_full = seen_lo(a.mask, first + t_last), hi_full = seen_hi(a.mask, first + t_first, length);
  // limits of this lane's rows, oct and oct + 8
  int row_lo[2], row_hi[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = first + a.group.div(tile * kTileRows + min(oct + 8 * i, rows - 1));
    row_lo[i] = seen_lo(a.mask, p);
    row_hi[i] = seen_hi(a.mask, p, length);
  }
  const int n_sink = a.mask.window > 0 ? a.mask.n_sink : 0;
  auto in_use = [&](int pos) { return pos < hi_all && (pos >= lo_all || pos < n_sink); };
  auto key_of = [&](int step) { return (step < sink_steps ? step : step - sink_steps + lo_step) << 4; };

  uint4 kq[2][kPieces], vq[4][kValPieces];
  float ks[4], vs[4];
  auto load_k = [&](int key0, int page) {
    const size_t row0 = store_row(s, max(page, 0), head, key0);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int k = n * 8 + oct;
      const bool on = page >= 0 && in_use(key0 + k);
      const char *p = s.k_rows + (row0 + k) * kRowBytes + quad * 16;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) kq[n][i] = on ? load_stream(p + i * 64) : make_uint4(0u, 0u, 0u, 0u);
      if constexpr (kQ8) {
        const float2 two = __ldg(reinterpret_cast<const float2 *>(s.k_scales + row0 + n * 8 + 2 * quad));
        ks[2 * n] = two.x; ks[2 * n + 1] = two.y;
      }
    }
  };
  auto load_v = [&](int key0, int page) {
    const size_t row0 = store_row(s, max(page, 0), head, key0);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int k = (n >> 1) * 8 + 2 * quad + (n & 1);
      const bool on = page >= 0 && in_use(key0 + k);
      const char *p = s.v_rows + (row0 + k) * kRowBytes;
      if constexpr (kRowBytes >= 128) {
#pragma unroll
        for (int i = 0; i < kValPieces; ++i) vq[n][i] = on ? load_stream(p + i * 128 + oct * 16) : make_uint4(0u, 0u, 0u, 0u);
      } else {
        const uint2 two = on ? __ldg(reinterpret_cast<const uint2 *>(p + oct * 8)) : make_uint2(0u, 0u);
        vq[n][0] = make_uint4(two.x, two.y, 0u, 0u);
      }
    }
    if constexpr (kQ8) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float2 two = __ldg(reinterpret_cast<const float2 *>(s.v_scales + row0 + n * 8 + 2 * quad));
        vs[2 * n] = two.x; vs[2 * n + 1] = two.y;
      }
    }
  };
  auto page_at = [&](int step) { return step < step_hi ? page_of(s, a.bt, seq, key_of(step)) : -1; };

  float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  __syncthreads();

  int step = step_lo + warp, page = page_at(step);
  int next = page_at(step + kStreamWarps);
  if (step < step_hi) {
    load_k(key_of(step), page);
    load_v(key_of(step), page);
  }
  for (; step < step_hi; step += kStreamWarps) {
    const int key0 = key_of(step);
    // S = Q K^T
    float x[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      if constexpr (kQ8) {
        // a piece is 16 dims: four products, each of four of this lane's dims
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const __nv_bfloat16 *q0 = q_smem + oct * kQLd + i * 64 + quad * 16 + h * 8;
          const uint4 a0 = *reinterpret_cast<const uint4 *>(q0), a1 = *reinterpret_cast<const uint4 *>(q0 + 8 * kQLd);
          const uint32_t f0[4] = {a0.x, a1.x, a0.y, a1.y}, f1[4] = {a0.z, a1.z, a0.w, a1.w};
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint32_t w0 = turn_signs(word(kq[n][i], 2 * h)), w1 = turn_signs(word(kq[n][i], 2 * h + 1));
            mma_16816(x[n], f0, codes_low(w0), codes_high(w0));
            mma_16816(x[n], f1, codes_low(w1), codes_high(w1));
          }
        }
      } else {
        const __nv_bfloat16 *q0 = q_smem + oct * kQLd + i * 32 + quad * 8;
        const uint4 a0 = *reinterpret_cast<const uint4 *>(q0), a1 = *reinterpret_cast<const uint4 *>(q0 + 8 * kQLd);
        const uint32_t f0[4] = {a0.x, a1.x, a0.y, a1.y}, f1[4] = {a0.z, a1.z, a0.w, a1.w};
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          mma_16816(x[n], f0, kq[n][i].x, kq[n][i].y);
          mma_16816(x[n], f1, kq[n][i].z, kq[n][i].w);
        }
      }
    }
    // base-2 exponents; hidden keys at -inf, whatever their rows and scales hold
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][e] *= kQ8 ? a.scale_log2e * kCodeUnit * ks[2 * n + (e & 1)] : a.scale_log2e;
    const bool whole = page >= 0 && key0 >= lo_full && key0 + 16 <= hi_full;
    uint32_t hidden = 0;
    if (!whole) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int pos = key0 + n * 8 + 2 * quad + (e & 1), i = e >> 1;
          if (page < 0 || pos >= row_hi[i] || (pos < row_lo[i] && pos >= n_sink)) { x[n][e] = -INFINITY; hidden |= 1u << (4 * n + e); }
        }
    }
    const int page_next = next;
    if (step + kStreamWarps < step_hi) load_k(key_of(step + kStreamWarps), page_next);
    next = page_at(step + 2 * kStreamWarps);
    // the rows' references
    float top[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      top[i] = fmaxf(fmaxf(x[0][2 * i], x[0][2 * i + 1]), fmaxf(x[1][2 * i], x[1][2 * i + 1]));
      top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
      top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
    }
    if (__any_sync(0xffffffffu, top[0] > m[0] + kRaise || top[1] > m[1] + kRaise)) {
      float f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float raised = fmaxf(m[i], top[i]);
        f[i] = raised == -INFINITY ? 1.f : exp2_approx(m[i] - raised);      // (from no reference at all: 0)
        m[i] = raised;
        l[i] *= f[i];
      }
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        o[j][0] *= f[0]; o[j][1] *= f[0];
        o[j][2] *= f[1]; o[j][3] *= f[1];
      }
    }
    const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
    uint32_t p[4];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[n][e] = exp2_approx(x[n][e] - ref[e >> 1]);
        l[e >> 1] += x[n][e];
      }
      if constexpr (kQ8) {
        // (a hidden key counts for nothing even where its scale is no number)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = (hidden >> (4 * n + e)) & 1u ? 0.f : x[n][e] * (kCodeUnit * vs[2 * n + (e & 1)]);
      }
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[2 * n]) : "f"(x[n][1]), "f"(x[n][0]));
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p[2 * n + 1]) : "f"(x[n][3]), "f"(x[n][2]));
    }
    // O += P V
    if constexpr (kQ8) {
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        uint32_t c[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) c[n] = turn_signs(word(vq[n][0], w));
        mma_16816(o[4 * w], p, codes_across<0>(c[0], c[1]), codes_across<0>(c[2], c[3]));
        mma_16816(o[4 * w + 1], p, codes_across<1>(c[0], c[1]), codes_across<1>(c[2], c[3]));
        mma_16816(o[4 * w + 2], p, codes_across<2>(c[0], c[1]), codes_across<2>(c[2], c[3]));
        mma_16816(o[4 * w + 3], p, codes_across<3>(c[0], c[1]), codes_across<3>(c[2], c[3]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < kValPieces; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t sel = (e & 1) ? 0x7632 : 0x5410;
          mma_16816(o[i * 8 + e], p, __byte_perm(word(vq[0][i], e >> 1), word(vq[1][i], e >> 1), sel),
                    __byte_perm(word(vq[2][i], e >> 1), word(vq[3][i], e >> 1), sel));
        }
    }
    if (step + kStreamWarps < step_hi) load_v(key_of(step + kStreamWarps), page_next);
    page = page_next;
  }

  // ---- the warps' parts, combined
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    if (quad == 0) { ml_smem[warp][oct + 8 * i][0] = m[i]; ml_smem[warp][oct + 8 * i][1] = l[i]; }
  }
#pragma unroll
  for (int j = 0; j < D / 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // column n = 2 quad + (e & 1) of n-tile j
      const int n = 2 * quad + (e & 1);
      const int dim = kQ8 ? n * (D / 8) + j : (j >> 3) * 64 + n * 8 + (j & 7);
      o_smem[warp][oct + 8 * (e >> 1)][dim] = o[j][e];
    }
  __syncthreads();
  const size_t all_rows = (size_t)a.bt.n_tokens * a.n_heads;
  for (int i = threadIdx.x; i < min(rows, kTileRows) * (D / 8); i += kStreamThreads) {
    const int r = i / (D / 8), piece = i % (D / 8);
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) top = fmaxf(top, ml_smem[w][r][0]);
    float sum = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) {
      if (ml_smem[w][r][0] == -INFINITY) continue;
      const float f = exp2_approx(ml_smem[w][r][0] - top);
      sum += f * ml_smem[w][r][1];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += f * o_smem[w][r][piece * 8 + e];
    }
    const int t = a.group.div(tile * kTileRows + r), g = tile * kTileRows + r - t * a.group.d;
    const int h = head * a.group.d + g;
    const size_t row = (size_t)(start + t) * a.n_heads + h;
    if (gridDim.z == 1) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint32_t u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[e]) : "f"(acc[2 * e + 1] * inv), "f"(acc[2 * e] * inv));
      *(reinterpret_cast<uint4 *>(a.O.ptr + (start + t) * a.O.st + h * a.O.sh) + piece) = make_uint4(u[0], u[1], u[2], u[3]);
      if (piece == 0 && a.lse != nullptr) a.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    } else {
      const size_t part = (size_t)blockIdx.z * all_rows + row;
      float4 *dst = reinterpret_cast<float4 *>(a.part_o + part * D + piece * 8);
      dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (piece == 0) *reinterpret_cast<float2 *>(a.part_ml + part * 2) = make_float2(top, sum);
    }
  }
}

// O = sum_e 2^(m_e - M) O_e / sum_e 2^(m_e - M) l_e, M the largest reference: a warp to each row.
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(const AttendArgs a, int n_split) {
  constexpr int kPer = D / 32;
  const int lane = threadIdx.x & 31, row = blockIdx.x * 8 + (threadIdx.x >> 5), all_rows = a.bt.n_tokens * a.n_heads;
  if (row >= all_rows) return;
  float m = -INFINITY, sum = 0.f, acc[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
  for (int e = lane; e < n_split; e += 32) m = fmaxf(m, a.part_ml[((size_t)e * all_rows + row) * 2]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  for (int e = 0; e < n_split; ++e) {
    const size_t part = (size_t)e * all_rows + row;
    const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + part * 2);
    if (ml.x == -INFINITY) continue;
    const float f = exp2_approx(ml.x - m);
    sum += f * ml.y;
    float v[kPer];
    if constexpr (kPer == 4) *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(a.part_o + part * D + lane * kPer);
    else *reinterpret_cast<float2 *>(v) = *reinterpret_cast<const float2 *>(a.part_o + part * D + lane * kPer);
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] += f * v[i];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int t = row / a.n_heads, h = row - t * a.n_heads;
  char *out = a.O.ptr + t * a.O.st + h * a.O.sh + lane * kPer * 2;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    uint32_t u;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(acc[i + 1] * inv), "f"(acc[i] * inv));
    *reinterpret_cast<uint32_t *>(out + i * 2) = u;
  }
  if (lane == 0 && a.lse != nullptr) a.lse[row] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
}

}  // namespace paged
}  // namespace scalekv
