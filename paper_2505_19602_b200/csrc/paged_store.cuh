// Writing rows into the paged token cache and reading them back.
//
// A row x of head_dim values is held as bf16, or as 8-bit codes with one scale:  a = max |x_i|,  s = a / 127,
// c_i = rint(x_i / s) in [-127, 127],  x_i ~ c_i s.  The scale is rounded to fp32, the quotient to fp32 and then to an integer (half to even):
// a value is off by at most s / 2 and a few units of fp32.  A row of zeros has s = 0; a row that holds an infinity or a NaN has
// s = NaN and codes 0, so it reads back as NaN and is not taken for numbers.
//
// Both kernels move every row once, eight values a lane: 16 lanes are a row of 128, 8 one of 64.  A block takes kRowsPerLane rows for each of its row
// groups, all loads before all stores.  Rows are numbered token by token, in a token K's heads and then V's.
#pragma once
#include <math_constants.h>

#include "paged_view.cuh"

namespace scalekv {
namespace paged {

constexpr int kStoreThreads = 256;
constexpr int kRowsPerLane = 4;

// The first sequence that ends behind token t (n_seqs: none does).  All threads of the block, same t.
__device__ __forceinline__ int block_seq_of(const Batch &bt, int t) {
  int seq = 0;
  for (int i0 = 0; i0 < bt.n_seqs; i0 += kStoreThreads) {
    const int i = i0 + (int)threadIdx.x;
    seq += __syncthreads_count(i < bt.n_seqs && __ldg(bt.starts + i + 1) <= t);
  }
  return seq;
}

// Position of token t in its sequence, and the sequence, which is `seq` or a later one.  False (reported): t belongs to no sequence.
__device__ __forceinline__ bool locate(const Store &s, const Batch &bt, int t, int &seq, int &pos) {
  while (seq < bt.n_seqs && __ldg(bt.starts + seq + 1) <= t) ++seq;
  if (seq >= bt.n_seqs || t < __ldg(bt.starts + seq)) { report(s.status); return false; }
  pos = __ldg(bt.lengths + seq) - __ldg(bt.starts + seq + 1) + t;
  return true;
}

__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *x) { Vec16<__nv_bfloat16>::load(p, x); }
__device__ __forceinline__ void load8(const float *p, float *x) { Vec16<float>::load(p, x); Vec16<float>::load(p + 4, x + 4); }
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *x) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pair_bf16(x[0], x[1]), pair_bf16(x[2], x[3]), pair_bf16(x[4], x[5]), pair_bf16(x[6], x[7]));
}
__device__ __forceinline__ void store8(float *p, const float *x) {
  *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

template <typename T, int D, bool kQ8>
__global__ void __launch_bounds__(kStoreThreads) paged_write_kernel(const Store s, const Batch bt, const Rows K, const Rows V, const Divisor per_token,
                                                                    int n_rows) {
  constexpr int kLanes = D / 8, kGroups = kStoreThreads / kLanes;
  const int lane = threadIdx.x % kLanes, r0 = blockIdx.x * kGroups * kRowsPerLane + threadIdx.x / kLanes;
  wait_for_grid();
  next_grid();
  float x[kRowsPerLane][8];
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int r = r0 + i * kGroups;
    if (r >= n_rows) break;
    const int t = per_token.div(r), e = r - t * per_token.d;
    const bool v = e >= s.heads;
    const Rows &X = v ? V : K;
    load8(reinterpret_cast<const T *>(X.ptr + t * X.st + (v ? e - s.heads : e) * X.sh) + lane * 8, x[i]);
  }
  int seq = block_seq_of(bt, per_token.div(blockIdx.x * kGroups * kRowsPerLane));
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int r = r0 + i * kGroups;
    // (the lanes of a row take every branch together, and the reduction names them alone)
    if (r >= n_rows) break;
    const int t = per_token.div(r), e = r - t * per_token.d;
    const bool v = e >= s.heads;
    int pos;
    if (!locate(s, bt, t, seq, pos)) break;
    const int page = page_of(s, bt, seq, pos);
    if (page < 0) continue;
    const size_t row = store_row(s, page, v ? e - s.heads : e, pos);
    char *rows = v ? s.v_rows : s.k_rows;
    if constexpr (!kQ8) {
      store8(reinterpret_cast<__nv_bfloat16 *>(rows) + row * D + lane * 8, x[i]);
    } else {
      // the largest magnitude by its bits: an infinity or a NaN is above every number
      unsigned a = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) a = max(a, __float_as_uint(x[i][k]) & 0x7fffffffu);
      const unsigned mask = (kLanes == 32 ? 0xffffffffu : ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes));
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(mask, a, o));
      const bool finite = a < 0x7f800000u;
      const float scale = finite ? __fdiv_rn(__uint_as_float(a), 127.f) : CUDART_NAN_F;
      uint32_t w[2] = {0u, 0u};
      if (scale > 0.f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int c = max(-127, min(127, __float2int_rn(__fdiv_rn(x[i][k], scale))));
          w[k >> 2] |= ((unsigned)c & 0xffu) << (8 * (k & 3));
        }
      }
      *reinterpret_cast<uint2 *>(rows + row * D + lane * 8) = make_uint2(w[0], w[1]);
      if (lane == 0) (v ? s.v_scales : s.k_scales)[row] = scale;
    }
  }
}

template <typename T, int D, bool kQ8>
__global__ void __launch_bounds__(kStoreThreads) paged_read_kernel(const Store s, const Batch bt, const Rows K, const Rows V, const Divisor per_token,
                                                                   int n_rows) {
  constexpr int kLanes = D / 8, kGroups = kStoreThreads / kLanes;
  const int lane = threadIdx.x % kLanes, r0 = blockIdx.x * kGroups * kRowsPerLane + threadIdx.x / kLanes;
  wait_for_grid();
  next_grid();
  int seq = block_seq_of(bt, per_token.div(blockIdx.x * kGroups * kRowsPerLane));
  uint4 w[kRowsPerLane];
  float scale[kRowsPerLane];
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int r = r0 + i * kGroups;
    w[i] = make_uint4(0u, 0u, 0u, 0u);
    scale[i] = 0.f;                                     // (a row without a page, which is reported, comes back as zeros)
    if (r >= n_rows) break;
    const int t = per_token.div(r), e = r - t * per_token.d;
    const bool v = e >= s.heads;
    int pos;
    if (!locate(s, bt, t, seq, pos)) break;
    const int page = page_of(s, bt, seq, pos);
    if (page < 0) continue;
    const size_t row = store_row(s, page, v ? e - s.heads : e, pos);
    const char *rows = v ? s.v_rows : s.k_rows;
    if constexpr (kQ8) {
      const uint2 c = __ldg(reinterpret_cast<const uint2 *>(rows + row * D + lane * 8));
      w[i].x = c.x; w[i].y = c.y;
      scale[i] = __ldg((v ? s.v_scales : s.k_scales) + row);
    } else {
      w[i] = __ldg(reinterpret_cast<const uint4 *>(rows + (row * D + lane * 8) * 2));
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int r = r0 + i * kGroups;
    if (r >= n_rows) break;
    const int t = per_token.div(r), e = r - t * per_token.d;
    const bool v = e >= s.heads;
    const Rows &X = v ? V : K;
    T *out = reinterpret_cast<T *>(X.ptr + t * X.st + (v ? e - s.heads : e) * X.sh) + lane * 8;
    float x[8];
    if constexpr (kQ8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = (float)(int8_t)((k < 4 ? w[i].x : w[i].y) >> (8 * (k & 3))) * scale[i];
    } else {
      const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(u[k] << 16);
        x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
      }
    }
    store8(out, x);
  }
}

}  // namespace paged
}  // namespace scalekv
