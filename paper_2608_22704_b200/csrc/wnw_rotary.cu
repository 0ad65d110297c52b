// wnw_rotate: rotary positions with several axes, forward and inverse, for the queries and keys of a layer in one launch.
//
// (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = positions[axis of the pair][token] * frequency of the pair.  Every element is
// read and written once, so memory bounds it from some thousand tokens on, a launch below that.  The angles of a token are shared by
// all heads: a CTA takes a few tokens, leaves their cosines and sines in shared memory, one thread a pair, and then goes over the
// heads' rows 16 bytes at a time: 15064 tokens of 18 heads of 128 in 27.8 us, 5.0 TB/s (6.5 is the measured copy rate); 16 tokens a CTA 28.1, more
// CTAs an SM with fewer registers each 32 to 42.
#include <algorithm>
#include <cstring>

#include "wnw_pages.cuh"

namespace wnw {
namespace {

constexpr int ROT_THREADS = 256, ROT_HEADS = 2;

struct RotateArgs {
  RotaryView rot;
  RowsView in[2], out[2];            // queries, keys
  int n_heads[2];
  const int32_t *positions;
  long long axis_stride;
  int n_tokens, head_dim, tokens_per_cta, tail;   // tail: elements behind the pairs that have to be copied
};

template <typename T> struct Elems;
template <> struct Elems<float> {
  static __device__ __forceinline__ float get(const float *p) { return *p; }
  static __device__ __forceinline__ void put(float *p, float x) { *p = x; }
};
template <> struct Elems<__nv_bfloat16> {
  static __device__ __forceinline__ float get(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }
};
template <> struct Elems<__half> {
  static __device__ __forceinline__ float get(const __half *p) { return __half2float(*p); }
  static __device__ __forceinline__ void put(__half *p, float x) { *p = __float2half_rn(x); }
};

// 16 bytes as floats and back
template <typename T> struct Vec {
  static constexpr int N = 8;
  float x[8];
  __device__ __forceinline__ void get(uint4 u) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 f = Pair<T>::get(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
  }
  __device__ __forceinline__ uint4 put() const {
    return make_uint4(Pair<T>::put(x[0], x[1]), Pair<T>::put(x[2], x[3]), Pair<T>::put(x[4], x[5]), Pair<T>::put(x[6], x[7]));
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  float x[4];
  __device__ __forceinline__ void get(uint4 u) { x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w); }
  __device__ __forceinline__ uint4 put() const { return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])); }
};

// A unit of work is N pairs of one token in up to U heads, 16 bytes (VEC) or one element each of the pairs' two halves: the angles are
// read once for the U heads, whose elements are on their way together.
template <typename T, bool VEC>
__global__ void __launch_bounds__(ROT_THREADS, 4) wnw_rotate_kernel(const __grid_constant__ RotateArgs a) {
  constexpr int N = VEC ? Vec<T>::N : 1, U = ROT_HEADS;
  extern __shared__ __align__(16) float2 cs[];          // [tokens_per_cta][N / 2][units][2], a unit's angles without bank conflicts; N = 1: [token][pair]
  pg_wait_for_stream();
  const int np = a.rot.n_pairs, units = np / N, t0 = blockIdx.x * a.tokens_per_cta, nt = min(a.tokens_per_cta, a.n_tokens - t0);
  const int pitch = np + 2;
  // Neighbouring lanes take neighbouring tokens, so that they read the same word of the plan: the kernel's parameters are read one address at
  // a time, and a pair a lane made 15064 tokens of 18 heads take 52 us instead of 30.
  for (int i = threadIdx.x; i < nt * np; i += ROT_THREADS) {
    const int p = i / nt, t = i - p * nt;
    float2 c = pg_angle(a.rot.turns[p], a.positions[a.rot.axis[p] * a.axis_stride + t0 + t]);
    c.y *= a.rot.sign;
    cs[t * pitch + (VEC ? ((p % N >> 1) * units + p / N) * 2 + (p & 1) : p)] = c;
  }
  const int heads = a.n_heads[0] + a.n_heads[1], blocks = (heads + U - 1) / U, all = nt * blocks * units;
  const bool nb = a.rot.neighbours;
  const int up = nb ? N : np;                           // from a unit's first half to its second
  bool ready = false;
  for (int i = threadIdx.x; i < all || !ready; i += ROT_THREADS) {
    const int row = i / units, u = i - row * units, t = row / blocks, h0 = (row - t * blocks) * U, n = i < all ? min(U, heads - h0) : 0;
    const T *in[U];
    T *out[U];
    uint4 x[U], y[U];
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (k < n) {
        const int which = h0 + k >= a.n_heads[0], h = h0 + k - (which ? a.n_heads[0] : 0), lo = (nb ? 2 : 1) * N * u;
        in[k] = reinterpret_cast<const T *>(a.in[which].p) + (long long)(t0 + t) * a.in[which].row + h * a.in[which].head + lo;
        out[k] = reinterpret_cast<T *>(a.out[which].p) + (long long)(t0 + t) * a.out[which].row + h * a.out[which].head + lo;
        if constexpr (VEC) {
          x[k] = *reinterpret_cast<const uint4 *>(in[k]);
          y[k] = *reinterpret_cast<const uint4 *>(in[k] + up);
        }
      }
    if (!ready) __syncthreads();                        // (the angles, while the first elements are on their way)
    ready = true;
    if (!n) continue;
    float2 c[N];
    if constexpr (VEC) {
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float4 e = *reinterpret_cast<const float4 *>(cs + t * pitch + ((j >> 1) * units + u) * 2);
        c[j] = make_float2(e.x, e.y);
        c[j + 1] = make_float2(e.z, e.w);
      }
    } else {
      c[0] = cs[t * pitch + u];
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (k >= n) break;
      if constexpr (VEC) {
        Vec<T> p, q;
        p.get(x[k]);
        q.get(y[k]);
        if (nb) {
#pragma unroll
          for (int j = 0; j < N / 2; ++j) {
            const float2 s = pg_turn(p.x[2 * j], p.x[2 * j + 1], c[j]), z = pg_turn(q.x[2 * j], q.x[2 * j + 1], c[N / 2 + j]);
            p.x[2 * j] = s.x; p.x[2 * j + 1] = s.y;
            q.x[2 * j] = z.x; q.x[2 * j + 1] = z.y;
          }
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const float2 s = pg_turn(p.x[j], q.x[j], c[j]);
            p.x[j] = s.x; q.x[j] = s.y;
          }
        }
        *reinterpret_cast<uint4 *>(out[k]) = p.put();
        *reinterpret_cast<uint4 *>(out[k] + up) = q.put();
      } else {
        const float2 s = pg_turn(Elems<T>::get(in[k]), Elems<T>::get(in[k] + up), c[0]);
        Elems<T>::put(out[k], s.x);
        Elems<T>::put(out[k] + up, s.y);
      }
    }
  }
  if (a.tail) {                                          // what the pairs leave, where the output is another tensor
    const int all_tail = nt * heads * a.tail;
    for (int i = threadIdx.x; i < all_tail; i += ROT_THREADS) {
      const int row = i / a.tail, e = 2 * np + i - row * a.tail, t = row / heads, h0 = row - t * heads;
      const int which = h0 >= a.n_heads[0], h = h0 - (which ? a.n_heads[0] : 0);
      const RowsView &in = a.in[which], &out = a.out[which];
      reinterpret_cast<T *>(out.p)[(t0 + t) * out.row + h * out.head + e] = reinterpret_cast<const T *>(in.p)[(t0 + t) * in.row + h * in.head + e];
    }
  }
}

template <typename T> cudaError_t launch(const RotateArgs &a, bool vec, cudaStream_t st) {
  const int grid = (a.n_tokens + a.tokens_per_cta - 1) / a.tokens_per_cta;
  const size_t smem = sizeof(float2) * a.tokens_per_cta * (a.rot.n_pairs + 2);
  return pg_launch(vec ? wnw_rotate_kernel<T, true> : wnw_rotate_kernel<T, false>, dim3(grid), ROT_THREADS, smem, st, 0, a);
}

}  // namespace

wnw_status_t rotary_view(const wnw_rotary_t *r, int head_dim, int inverse, RotaryView *v) {
  if (r->n_pairs < 1 || r->n_pairs > 128 || r->n_axes < 1 || r->n_axes > 4 || (r->neighbours & ~1) || 2 * r->n_pairs > head_dim) return WNW_ERR_INVALID_ARG;
  memset(v, 0, sizeof(*v));
  for (int i = 0; i < r->n_pairs; ++i) {
    if (r->axis[i] >= r->n_axes || !std::isfinite(r->frequency[i])) return WNW_ERR_INVALID_ARG;
    v->turns[i] = r->frequency[i] / 6.283185307179586476925286766559;
    v->axis[i] = r->axis[i];
  }
  v->n_pairs = r->n_pairs;
  v->neighbours = r->neighbours;
  v->sign = inverse ? -1.f : 1.f;
  return WNW_OK;
}

}  // namespace wnw

using namespace wnw;

extern "C" wnw_status_t wnw_rotary_init(wnw_rotary_t *rotary, int32_t n_pairs, double base, const int32_t *sections, int32_t n_axes,
                                        int32_t dealt, int32_t neighbours) {
  if (!rotary || !sections || n_pairs < 1 || n_pairs > 128 || n_axes < 1 || n_axes > 4 || !(base > 0) || !std::isfinite(base)) return WNW_ERR_INVALID_ARG;
  if ((dealt & ~1) || (neighbours & ~1)) return WNW_ERR_INVALID_ARG;
  long long sum = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (sections[a] < 0) return WNW_ERR_INVALID_ARG;
    sum += sections[a];
  }
  if (sum != n_pairs) return WNW_ERR_INVALID_ARG;
  wnw_rotary_t r;
  memset(&r, 0, sizeof(r));
  r.n_pairs = n_pairs;
  r.n_axes = n_axes;
  r.neighbours = neighbours;
  for (int i = 0, a = 0, left = sections[0]; i < n_pairs; ++i) {
    r.frequency[i] = std::pow(base, -(double)i / n_pairs);
    if (dealt) {
      r.axis[i] = (uint8_t)(i / n_axes < sections[i % n_axes] ? i % n_axes : 0);
    } else {
      while (left == 0) left = sections[++a];
      --left;
      r.axis[i] = (uint8_t)a;
    }
  }
  *rotary = r;
  return WNW_OK;
}

extern "C" wnw_status_t wnw_rotate(const wnw_rotate_t *call) {
  if (!call || !call->rotary || !call->k.dev != !call->k_out.dev || call->n_tokens < 0 || (call->inverse & ~1)) return WNW_ERR_INVALID_ARG;
  const int n_tokens = call->n_tokens, head_dim = call->head_dim, dtype = call->dtype;
  if (head_dim < 2 || head_dim > 256 || head_dim % 2 || dtype < WNW_DTYPE_BF16 || dtype > WNW_DTYPE_FP32) return WNW_ERR_UNSUPPORTED;
  RotateArgs a;
  const wnw_status_t rc = rotary_view(call->rotary, head_dim, call->inverse, &a.rot);
  if (rc != WNW_OK) return rc;
  const int size = (int)pg_elem(dtype), n = 16 / size;
  bool vec = a.rot.n_pairs % n == 0;
  a.tail = 0;
  a.n_heads[1] = 0;
  for (int i = 0; i < (call->k.dev ? 2 : 1); ++i) {
    const wnw_rows_t &in = i ? call->k : call->q, &out = i ? call->k_out : call->q_out;
    if (in.n_heads < 1 || in.n_heads > 4096 || in.n_heads != out.n_heads) return WNW_ERR_INVALID_ARG;
    if (n_tokens && (!in.dev || !out.dev || (uintptr_t)in.dev % size || (uintptr_t)out.dev % size)) return WNW_ERR_INVALID_ARG;
    vec = vec && pg_vector_rows(in, dtype) && pg_vector_rows(out, dtype);
    const bool same = in.dev == out.dev && in.row_stride == out.row_stride && in.head_stride == out.head_stride;
    if (!same) a.tail = head_dim - 2 * a.rot.n_pairs;
    a.in[i] = rows_view(in);
    a.out[i] = rows_view(out);
    a.n_heads[i] = in.n_heads;
  }
  if (!n_tokens) return WNW_OK;
  if (!call->positions_dev || (uintptr_t)call->positions_dev % 4) return WNW_ERR_INVALID_ARG;
  a.positions = call->positions_dev;
  a.axis_stride = call->axis_stride;
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  OnDevice on(call->device);
  int n_sm = 0;
  if (!on.ok || pg_sms(call->device, &n_sm) != WNW_OK) return WNW_ERR_CUDA;
  a.tokens_per_cta = std::max(1, std::min(8, n_tokens / (n_sm * 4)));
  const cudaStream_t st = (cudaStream_t)call->cuda_stream;
  const cudaError_t e = dtype == WNW_DTYPE_BF16 ? launch<__nv_bfloat16>(a, vec, st) : dtype == WNW_DTYPE_FP16 ? launch<__half>(a, vec, st)
                                                                                                              : launch<float>(a, vec, st);
  return e == cudaSuccess ? WNW_OK : WNW_ERR_CUDA;
}
