// Writing rows into the paged token cache and reading them back.
//
// A row x of head_dim values is held as bf16, or as 8-bit codes with one scale:  a = max |x_i|,  s = a / 127,
// c_i = rint(x_i / s) in [-127, 127],  x_i ~ c_i s.  The scale is rounded to fp32, the quotient to fp32 and then to an integer (half to even):
// a value is off by at most s / 2 and a few units of fp32.  A row of zeros has s = 0; a row that holds an infinity or a NaN has
// s = NaN and codes 0, so it reads back as NaN and is not taken for numbers.
//
// Both kernels move every row once; what bounds them is that.  A lane has 16 values of a row, 8 lanes are a row of 128, 4 one of 64.  A block takes a few
// tokens, all heads of K and V of them: one thread to a token finds its place, then the rows follow one another as they do in a dense tensor.
// us per pass, eight values a lane and every row's place looked up by its own lanes / so: 84 168 tokens of 8 heads in codes read as bf16 118 / 92 (5.7 of 6.46 TB/s
// measured), 24 646 of 16 heads written and read back 228 / 112: writing takes 57 of that for 303 MB,
// bound by its instructions (71 of 100 issue slots).
#pragma once
#include <math_constants.h>

#include "paged_view.cuh"
#include "tc.cuh"

namespace scalekv {
namespace paged {

constexpr int kStoreThreads = 256;
constexpr int kMostTokens = 32;                  // tokens of a block

struct Moves {
  Store s;
  Batch bt;
  Rows K, V;
  Divisor per_token;                             // 16-value pieces of a token: of K's heads, then of V's
  int tokens;                                    // of a block
  int wide;                                      // every 16 values of the dense tensors begin on 32 bytes
};

// The first sequence that ends behind token t (n_seqs: none does).  All threads of the block, same t.  A launch's first block tells of starts that are out of
// order.
__device__ __forceinline__ int block_seq_of(const Batch &bt, int t, int *status) {
  int seq = 0;
  for (int i0 = 0; i0 < bt.n_seqs; i0 += kStoreThreads) {
    const int i = i0 + (int)threadIdx.x;
    bool ended = false;
    if (i < bt.n_seqs) {
      const int end = bt.starts[i + 1];
      if (blockIdx.x == 0 && starts_wrong(bt, i, bt.starts[i], end)) report(status);
      ended = end <= t;
    }
    seq += __syncthreads_count(ended);
  }
  return seq;
}

// Row of head 0 of the block's tokens, in K as in V; -1 (reported) where a token belongs to no sequence or its page is out of range.
__device__ __forceinline__ void place_tokens(const Moves &mv, int t0, int n, long long *row) {
  const Batch &bt = mv.bt;
  int seq = block_seq_of(bt, t0, mv.s.status);
  if ((int)threadIdx.x < n) {
    const int t = t0 + (int)threadIdx.x;
    // (start, end and length side by side: one behind the other they are three trips to memory; us, a token of 8 sequences written and read back 5.4 / 5.2)
    int start = 0, end = 0, length = 0;
    for (; seq < bt.n_seqs; ++seq) {
      start = bt.starts[seq];
      end = bt.starts[seq + 1];
      length = bt.lengths[seq];
      if (end > t) break;
    }
    long long at = -1;
    if (seq >= bt.n_seqs || t < start) {
      report(mv.s.status);
    } else {
      const int pos = length - end + t, page = page_of(mv.s, bt, seq, pos);
      if (page >= 0) at = (long long)store_row(mv.s, page, 0, pos);
    }
    row[threadIdx.x] = at;
  }
  __syncthreads();
}

// (NaN if any of them is)
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// A lane's 16 values are 32 bytes of bf16, a sector: one access where they begin on 32 bytes, or two of 16 bytes, each of which meets every sector of
// the warp's and fills it by half (us, two / one, 24 646 tokens of 16 heads written and read back: f32 204 / 167, bf16 115 / 112).
__device__ __forceinline__ void load32(const void *p, uint4 &a, uint4 &b) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
               : "l"(p));
}
__device__ __forceinline__ void store32(void *p, const uint4 &a, const uint4 &b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y),
               "r"(b.z), "r"(b.w)
               : "memory");
}
// 16 values as they lie in memory, and as numbers
template <typename T> struct Raw16 {
  uint4 w[sizeof(T)];
  __device__ __forceinline__ void load(const T *p, bool wide) {
    if (wide) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T); i += 2) load32(reinterpret_cast<const uint4 *>(p) + i, w[i], w[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T); ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
  }
  __device__ __forceinline__ void numbers(float *x) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
      const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) {
          x[4 * i + k] = __uint_as_float(u[k]);
        } else {
          x[8 * i + 2 * k] = __uint_as_float(u[k] << 16);
          x[8 * i + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        }
      }
    }
  }
};
__device__ __forceinline__ void store16(__nv_bfloat16 *p, const float *x, bool wide) {
  uint4 w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = make_uint4(tc::pack_bf16(x[8 * i], x[8 * i + 1]), tc::pack_bf16(x[8 * i + 2], x[8 * i + 3]), tc::pack_bf16(x[8 * i + 4], x[8 * i + 5]),
                      tc::pack_bf16(x[8 * i + 6], x[8 * i + 7]));
  if (wide) {
    store32(p, w[0], w[1]);
  } else {
    reinterpret_cast<uint4 *>(p)[0] = w[0];
    reinterpret_cast<uint4 *>(p)[1] = w[1];
  }
}
__device__ __forceinline__ void store16(float *p, const float *x, bool wide) {
  auto four = [&](int i) { return make_uint4(__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]), __float_as_uint(x[i + 3])); };
#pragma unroll
  for (int i = 0; i < 16; i += 8) {
    if (wide) {
      store32(p + i, four(i), four(i + 4));
    } else {
      reinterpret_cast<uint4 *>(p + i)[0] = four(i);
      reinterpret_cast<uint4 *>(p + i)[1] = four(i + 4);
    }
  }
}

// The scale of a row whose largest value is a: a / 127, by the same step as below from the rounded reciprocal (all 2^23 significands give the division's quotient).
__device__ __forceinline__ float scale_of(float a) {
  if (a < 0x1p-60f) return __fdiv_rn(a, 127.f);
  const float r = 1.f / 127.f, q = __fmul_rn(a, r);
  return __fmaf_rn(__fmaf_rn(-q, 127.f, a), r, q);
}
// Codes of 16 values: x / s rounded to fp32 and then to an integer, half to even.  The quotient by Markstein's theorem (IBM J. Res. Dev. 34, 1990): with r the
// rounded reciprocal, q within a unit in the last place of the quotient and e = x - q s, which a fused multiply-add gives exactly, q + e r is the rounded
// quotient.  x r is within two units, one such step makes that one, a second the result.  Rows of bf16 need no second: with 8 bits of significand in x and in the
// row's largest value there are few enough quotients to go through all of them: none of 14 507 841 gives another code than a division (614 592 at scales as they
// are, where 72 do without the first step, and 13 893 249 at lifted ones).  (A division for each of them took the larger part of the kernel's time.)  Adding 1.5 2^23 rounds to an integer and leaves its low byte in the sum's.  A small scale is lifted first, so that nothing underflows, and its values
// are cut off where the codes end, which a rounded subnormal scale leaves below the largest of them.
template <int kSteps> __device__ __forceinline__ uint4 codes_of(float *x, float s) {
  if (!(s > 0.f)) return make_uint4(0u, 0u, 0u, 0u);
  if (s < 0x1p-60f) {
    s *= 0x1p64f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = fmaxf(-127.f * s, fminf(127.f * s, x[i] * 0x1p64f));
  }
  using namespace scalekv::tc;                     // (two values to an instruction)
  const float r = __frcp_rn(s);
  const uint64_t r2 = pack2(r, r), minus_s2 = pack2(-s, -s), unit2 = pack2(12582912.f, 12582912.f);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    float c[4];
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const uint64_t x2 = pack2(x[i + k], x[i + k + 1]);
      uint64_t q = mul2(x2, r2);
#pragma unroll
      for (int step = 0; step < kSteps; ++step) q = fma2(fma2(q, minus_s2, x2), r2, q);
      unpack2(add2(q, unit2), c[k], c[k + 1]);
    }
    w[i / 4] = __byte_perm(__byte_perm(__float_as_uint(c[0]), __float_as_uint(c[1]), 0x0040), __byte_perm(__float_as_uint(c[2]), __float_as_uint(c[3]), 0x0040), 0x5410);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The numbers of four codes: 2^23 + (c + 128) as fp32 has c + 128 for its last byte, and the difference is exact.
__device__ __forceinline__ void numbers_of(uint32_t w, float *c) {
  w ^= 0x80808080u;
#pragma unroll
  for (int k = 0; k < 4; ++k) c[k] = __fsub_rn(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + k)), 8388736.f);
}

// A thread's piece of the dense tensors and of the store.
struct Piece {
  int t, head;                                   // token of the block
  bool is_v;
  __device__ __forceinline__ Piece(const Moves &mv, int i, int lanes) {
    t = mv.per_token.div(i);
    const int e = (i - t * mv.per_token.d) / lanes;
    is_v = e >= mv.s.heads;
    head = is_v ? e - mv.s.heads : e;
  }
  template <typename T> __device__ __forceinline__ T *dense(const Moves &mv, int t0) const {
    const Rows &X = is_v ? mv.V : mv.K;
    return reinterpret_cast<T *>(X.ptr + (t0 + t) * X.st + head * X.sh);
  }
  __device__ __forceinline__ size_t row(const Moves &mv, long long row0) const { return (size_t)row0 + ((size_t)head << mv.s.page_shift); }
};

template <typename T, int D, bool kQ8>
__global__ void __launch_bounds__(kStoreThreads) paged_write_kernel(const __grid_constant__ Moves mv) {
  constexpr int kLanes = D / 16;
  __shared__ long long row0[kMostTokens];
  wait_for_grid();
  next_grid();
  const Store &s = mv.s;
  const int t0 = blockIdx.x * mv.tokens, n = min(mv.tokens, mv.bt.n_tokens - t0), pieces = n * mv.per_token.d, x = threadIdx.x % kLanes;
  // (the lanes of a row take every branch together, and the reduction names them alone)
  const unsigned mask = ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);
  Raw16<T> raw;
  Piece p(mv, threadIdx.x, kLanes);
  if ((int)threadIdx.x < pieces) raw.load(p.dense<T>(mv, t0) + x * 16, mv.wide);       // (under the look-up)
  place_tokens(mv, t0, n, row0);
  for (int i = threadIdx.x; i < pieces; i += kStoreThreads) {
    float v[16];
    raw.numbers(v);
    const Piece next(mv, i + kStoreThreads, kLanes);
    if (i + kStoreThreads < pieces) raw.load(next.dense<T>(mv, t0) + x * 16, mv.wide);
    if (row0[p.t] >= 0) {
      const size_t row = p.row(mv, row0[p.t]);
      char *rows = p.is_v ? s.v_rows : s.k_rows;
      if constexpr (!kQ8) {
        store16(reinterpret_cast<__nv_bfloat16 *>(rows) + row * D + x * 16, v, true);
      } else {
        float a = fabsf(v[0]);
#pragma unroll
        for (int j = 1; j < 15; j += 2) a = max_nan(a, fabsf(v[j]), fabsf(v[j + 1]));
        a = max_nan(a, fabsf(v[15]), 0.f);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(mask, a, o), 0.f);
        const float scale = a < CUDART_INF_F ? scale_of(a) : CUDART_NAN_F;
        *reinterpret_cast<uint4 *>(rows + row * D + x * 16) = codes_of<sizeof(T) == 2 ? 1 : 2>(v, scale);
        if (x == 0) (p.is_v ? s.v_scales : s.k_scales)[row] = scale;
      }
    }
    p = next;
  }
}

template <typename T, int D, bool kQ8>
__global__ void __launch_bounds__(kStoreThreads) paged_read_kernel(const __grid_constant__ Moves mv) {
  constexpr int kLanes = D / 16;
  __shared__ long long row0[kMostTokens];
  wait_for_grid();
  next_grid();
  const Store &s = mv.s;
  const int t0 = blockIdx.x * mv.tokens, n = min(mv.tokens, mv.bt.n_tokens - t0), pieces = n * mv.per_token.d, x = threadIdx.x % kLanes;
  place_tokens(mv, t0, n, row0);
  for (int i = threadIdx.x; i < pieces; i += kStoreThreads) {
    const Piece p(mv, i, kLanes);
    float y[16];
    if (row0[p.t] < 0) {                         // (a row without a page, which is reported, comes back as zeros)
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = 0.f;
    } else {
      const size_t row = p.row(mv, row0[p.t]);
      const char *rows = p.is_v ? s.v_rows : s.k_rows;
      if constexpr (kQ8) {
        const uint4 w = __ldcg(reinterpret_cast<const uint4 *>(rows + row * D + x * 16));
        const float scale = __ldcg((p.is_v ? s.v_scales : s.k_scales) + row);
        numbers_of(w.x, y);
        numbers_of(w.y, y + 4);
        numbers_of(w.z, y + 8);
        numbers_of(w.w, y + 12);
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] *= scale;
      } else {
        Raw16<__nv_bfloat16> raw;
        raw.load(reinterpret_cast<const __nv_bfloat16 *>(rows) + row * D + x * 16, true);
        raw.numbers(y);
      }
    }
    store16(p.dense<T>(mv, t0) + x * 16, y, mv.wide);
  }
}

}  // namespace paged
}  // namespace scalekv
