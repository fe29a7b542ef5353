// Writing new tokens' rows into the paged token cache with their positions in them (see include/scalekv.h for the contract).
//
// Pair i of a row of Q or K turns by the angle  f = position on the pair's axis x frequency of the pair:
//   (x, y) -> (x cos f - y sin f, x sin f + y cos f)   in fp32;  Q goes out as bf16, K and V join the cache as paged_store.cuh's write puts them there.
// Angles grow far beyond what 32 bits hold of them (position 2^20 of a pair that turns by a radian leaves 2^-4 radians), so they are formed in 64 bits and in turns, less whole ones; what
// is left, at most half a turn, goes into sine and cosine in fp32.  They are the same for all heads: a block works them out once for its tokens, into shared memory.
//
// Every row is moved once; what bounds that is memory, and with bf16 rows the instructions for a lane's 16 values, about 200 (56 of 100 issue slots).  A lane has 16 values of a row, as two pieces of eight:
// where the pairs are a dimension of the first half and one of the second, the pieces are those of eight pairs, so nothing is exchanged between lanes.
// us, 8 192 tokens of 16 heads of 128: bf16 into bf16 41.6 (4.8 TB/s of 6.5 measured), f32 into bf16 54 (5.6), bf16 into codes 64 (168.8 MB, 26 at the copy rate: rows that turn nothing, V's
// above all, go through the same branches and both correction steps of a quotient).  (Five blocks to an SM with bf16 rows, at 28 to 36 bytes of spills, 8 into codes, 48.3 / 66.7 with codes where four take
// 49.5 / 68.9, with one event's 5 us; with f32 rows five were the slower.  Two rounds of loads on their way, or angles behind the look-up of places: the same to 1 us.)
#include "paged_host.cuh"
#include "paged_store.cuh"

using namespace scalekv;
using namespace scalekv::paged;

namespace scalekv {
namespace paged {

constexpr int kMostPairs = 64;

struct Turning {
  Moves mv;
  Rows Q, Q_out;
  Divisor pairs;                                 // of dimensions that turn
  int n_heads, adjacent;
  const int *positions;                          // [axis][token]
  long long axis_stride;
  double turns[kMostPairs];                      // of pair i for each position
  unsigned char axis[kMostPairs];
};

// Eight values as they lie in memory, and as numbers
template <typename T> struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
  }
  __device__ __forceinline__ void numbers(float *x) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) {
          x[4 * i + k] = __uint_as_float(u[k]);
        } else {
          x[2 * k] = __uint_as_float(u[k] << 16);
          x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        }
      }
    }
  }
};
__device__ __forceinline__ uint4 eight_bf16(const float *x) {
  return make_uint4(tc::pack_bf16(x[0], x[1]), tc::pack_bf16(x[2], x[3]), tc::pack_bf16(x[4], x[5]), tc::pack_bf16(x[6], x[7]));
}

// A thread's two pieces of a row: head `head` of Q, K or V of token t of the block, dimensions a .. a + 7 and b .. b + 7.
struct TwoPieces {
  int t, head, a, b;
  bool is_q, is_v, turns;
  __device__ __forceinline__ TwoPieces(const Turning &r, int i, int lanes) {
    t = r.mv.per_token.div(i);
    const int e = (i - t * r.mv.per_token.d) / lanes, x = i % lanes, turning = r.pairs.d >> 3;      // (a token's pieces are a multiple of the lanes of a row)
    is_q = e < r.n_heads;
    is_v = e >= r.n_heads + r.mv.s.heads;
    head = e - (is_q ? 0 : is_v ? r.n_heads + r.mv.s.heads : r.n_heads);
    turns = !is_v && x < turning;
    a = 16 * x;
    b = a + 8;
    if (turns && !r.adjacent) {
      a = 8 * x;
      b = r.pairs.d + 8 * x;
    }
  }
  template <typename T> __device__ __forceinline__ const T *dense(const Turning &r, int t0) const {
    const Rows &X = is_q ? r.Q : is_v ? r.mv.V : r.mv.K;
    return reinterpret_cast<const T *>(X.ptr + (t0 + t) * X.st + head * X.sh);
  }
};

template <typename T, int D, bool kQ8>
__global__ void __launch_bounds__(kStoreThreads, sizeof(T) == 2 ? 5 : 4) paged_rotate_kernel(const __grid_constant__ Turning r) {
  constexpr int kLanes = D / 16;
  __shared__ long long row0[kMostTokens];
  __shared__ __align__(16) float2 table[kMostTokens * (D / 2)];     // cosine and sine: [token][pair of pairs mod 4][pair / 8][pair mod 2], so that neighbouring lanes read neighbouring 16 bytes
  wait_for_grid();
  next_grid();
  const Moves &mv = r.mv;
  const Store &s = mv.s;
  const int t0 = blockIdx.x * mv.tokens, n = min(mv.tokens, mv.bt.n_tokens - t0), pieces = n * mv.per_token.d, x = threadIdx.x % kLanes, turning = r.pairs.d >> 3;
  const unsigned mask = ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);
  Raw8<T> lo, hi;
  TwoPieces p(r, threadIdx.x, kLanes);
  if ((int)threadIdx.x < pieces) {                                  // (under the look-up)
    lo.load(p.dense<T>(r, t0) + p.a);
    hi.load(p.dense<T>(r, t0) + p.b);
  }
  for (int i = threadIdx.x; i < n * r.pairs.d; i += kStoreThreads) {
    const int t = r.pairs.div(i), pair = i - t * r.pairs.d;
    const double turn = (double)r.positions[r.axis[pair] * r.axis_stride + t0 + t] * r.turns[pair];
    float2 cs;
    sincospif(2.f * (float)(turn - rint(turn)), &cs.y, &cs.x);
    table[((t * 4 + ((pair & 7) >> 1)) * turning + (pair >> 3)) * 2 + (pair & 1)] = cs;
  }
  place_tokens(mv, t0, n, row0);                                    // (ends with a barrier)
  for (int i = threadIdx.x; i < pieces; i += kStoreThreads) {
    float v[16];
    lo.numbers(v);
    hi.numbers(v + 8);
    const TwoPieces next(r, i + kStoreThreads, kLanes);
    if (i + kStoreThreads < pieces) {
      lo.load(next.dense<T>(r, t0) + next.a);
      hi.load(next.dense<T>(r, t0) + next.b);
    }
    if (p.turns) {
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const float4 cs = reinterpret_cast<const float4 *>(table)[(p.t * 4 + (j >> 1)) * turning + x];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float c = e ? cs.z : cs.x, sn = e ? cs.w : cs.y;
          if (r.adjacent) {
            const float a = v[2 * (j + e)], b = v[2 * (j + e) + 1];
            v[2 * (j + e)] = a * c - b * sn;
            v[2 * (j + e) + 1] = a * sn + b * c;
          } else {
            const float a = v[j + e], b = v[8 + j + e];
            v[j + e] = a * c - b * sn;
            v[8 + j + e] = a * sn + b * c;
          }
        }
      }
    }
    if (p.is_q) {
      char *out = r.Q_out.ptr + (t0 + p.t) * r.Q_out.st + p.head * r.Q_out.sh;
      *reinterpret_cast<uint4 *>(out + p.a * 2) = eight_bf16(v);
      *reinterpret_cast<uint4 *>(out + p.b * 2) = eight_bf16(v + 8);
    } else if (row0[p.t] >= 0) {
      const size_t row = (size_t)row0[p.t] + ((size_t)p.head << s.page_shift);
      char *rows = (p.is_v ? s.v_rows : s.k_rows) + row * (D * (kQ8 ? 1 : 2));
      if constexpr (!kQ8) {
        *reinterpret_cast<uint4 *>(rows + p.a * 2) = eight_bf16(v);
        *reinterpret_cast<uint4 *>(rows + p.b * 2) = eight_bf16(v + 8);
      } else {
        float a = fabsf(v[0]);
#pragma unroll
        for (int j = 1; j < 15; j += 2) a = max_nan(a, fabsf(v[j]), fabsf(v[j + 1]));
        a = max_nan(a, fabsf(v[15]), 0.f);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(mask, a, o), 0.f);
        const float scale = a < CUDART_INF_F ? scale_of(a) : CUDART_NAN_F;
        const uint4 codes = codes_of<2>(v, scale);                  // (turned, the rows are of fp32 values)
        *reinterpret_cast<uint2 *>(rows + p.a) = make_uint2(codes.x, codes.y);
        *reinterpret_cast<uint2 *>(rows + p.b) = make_uint2(codes.z, codes.w);
        if (x == 0) (p.is_v ? s.v_scales : s.k_scales)[row] = scale;
      }
    }
    p = next;
  }
}

}  // namespace paged
}  // namespace scalekv

extern "C" scalekv_status scalekv_paged_write_rotated(scalekv_paged *kv, int32_t layer, const scalekv_paged_batch *batch, int32_t n_heads, scalekv_rows Q, scalekv_rows Q_out,
                                                      scalekv_rows K, scalekv_rows V, int32_t dtype, const scalekv_rotary *rotary, const int32_t *positions,
                                                      int64_t axis_stride, void *stream) {
  if (!kv) return SCALEKV_ERR_INVALID_ARG;
  scalekv_paged *c = kv;
  Range range("scalekv.paged_write_rotated");
  Turning r;
  if (scalekv_status st = check_batch(c, layer, batch, r.mv.bt)) return st;
  if (dtype != SCALEKV_BF16 && dtype != SCALEKV_F32) return fail(c, SCALEKV_ERR_UNSUPPORTED, "rows are bf16 or f32");
  if (n_heads < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "n_heads negative");
  if (!rotary || rotary->n_axes < 1 || rotary->n_axes > kMostPairs) return fail(c, SCALEKV_ERR_INVALID_ARG, "rotary null, or its n_axes not in 1 .. 64");
  if (rotary->n_pairs < 8 || (rotary->n_pairs & 7) || 2 * rotary->n_pairs > c->cfg.head_dim)
    return fail(c, SCALEKV_ERR_INVALID_ARG, "%d pairs: a multiple of 8 from 8 to half of head_dim turn", rotary->n_pairs);
  for (int i = 0; i < rotary->n_pairs; ++i) {
    if (rotary->axis[i] >= rotary->n_axes) return fail(c, SCALEKV_ERR_INVALID_ARG, "pair %d turns by axis %d of %d", i, rotary->axis[i], rotary->n_axes);
    // (a position is below 2^31 and an angle has to keep some bits behind its whole turns)
    if (!std::isfinite(rotary->frequency[i]) || std::fabs(rotary->frequency[i]) > 1024.) return fail(c, SCALEKV_ERR_INVALID_ARG, "frequency %d not within [-1024, 1024]", i);
    r.turns[i] = rotary->frequency[i] / 6.283185307179586476925;
    r.axis[i] = rotary->axis[i];
  }
  const int n = r.mv.bt.n_tokens;
  if (n == 0) return SCALEKV_OK;
  const int esize = dtype == SCALEKV_BF16 ? 2 : 4;
  if (!positions || axis_stride < 0) return fail(c, SCALEKV_ERR_INVALID_ARG, "positions null, or a negative stride of their axes");
  if (!rows_ok(K, esize) || !rows_ok(V, esize) || (n_heads > 0 && (!rows_ok(Q, esize) || !rows_ok(Q_out, 2))))
    return fail(c, SCALEKV_ERR_INVALID_ARG, "Q, Q_out, K or V null or rows not 16-byte aligned");
  if (c->cfg.n_kv_heads > 65535 || n_heads > 65535) return fail(c, SCALEKV_ERR_UNSUPPORTED, "more than 65535 heads");
  r.mv.s = layer_store(c, layer);
  r.mv.K = view(K, esize); r.mv.V = view(V, esize);
  r.mv.wide = 0;
  r.Q = view(Q, esize); r.Q_out = view(Q_out, 2);
  r.n_heads = n_heads;
  r.adjacent = rotary->adjacent != 0;
  r.pairs = Divisor::of(rotary->n_pairs);
  r.positions = positions;
  r.axis_stride = axis_stride;
  r.mv.per_token = Divisor::of((n_heads + 2 * c->cfg.n_kv_heads) * (c->cfg.head_dim / 16));
  // (as many tokens to a block as paged_store's write takes; twice and four times as many: 51.6 and 56.9 us where it takes 49.5, half as many 48.6 and, into codes, 69.4 for 68.9)
  const int full = (4 * kStoreThreads + r.mv.per_token.d - 1) / r.mv.per_token.d;
  r.mv.tokens = std::max(1, std::min(std::min(full, kMostTokens), n / (2 * c->n_sm)));
  const dim3 grid((n + r.mv.tokens - 1) / r.mv.tokens);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto t, auto dim) {
    using T = decltype(t);
    constexpr int D = decltype(dim)::value;
    if (c->cfg.store == SCALEKV_STORE_Q8) launch(paged_rotate_kernel<T, D, true>, grid, kStoreThreads, 0, st, r);
    else launch(paged_rotate_kernel<T, D, false>, grid, kStoreThreads, 0, st, r);
  };
  auto typed = [&](auto t) {
    if (c->cfg.head_dim == 128) go(t, std::integral_constant<int, 128>{});
    else go(t, std::integral_constant<int, 64>{});
  };
  if (dtype == SCALEKV_BF16) typed(__nv_bfloat16{}); else typed(float{});
  return launched(c, "paged_write_rotated");
}
