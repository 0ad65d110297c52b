// The paged K/V store of eight bits: quantising rows as they are written (wnw_pages_write) and reading them back (wnw_pages_read).
//
// Power-of-two scales make all of it exact but the one rounding to the code: x / 2^e is x with another exponent, code * 2^e a bf16
// number, and a scale that is raised rounds integers (or subnormal e4m3 numbers) again.  Both directions move each element once, so
// memory bounds them; a CTA takes one page of one KV head, K or V, whose scale it thereby owns: no atomics, one order of everything.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "wnw_pages.cuh"

namespace wnw {
namespace {

// ---- codes ----
template <int FMT> __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (FMT == WNW_PAGES_E4M3) {
    unsigned short lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;\n" : "=h"(lo) : "f"(a), "f"(b));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;\n" : "=h"(hi) : "f"(c), "f"(d));
    return lo | (uint32_t)hi << 16;
  } else {
    const int i = max(-127, min(127, __float2int_rn(a))), j = max(-127, min(127, __float2int_rn(b)));   // not-a-number: 0
    const int k = max(-127, min(127, __float2int_rn(c))), l = max(-127, min(127, __float2int_rn(d)));
    return (i & 255) | (j & 255) << 8 | (k & 255) << 16 | (uint32_t)l << 24;
  }
}
template <int FMT> __device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (FMT == WNW_PAGES_E4M3) {
    uint32_t lo, hi;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(lo) : "h"((unsigned short)w));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(hi) : "h"((unsigned short)(w >> 16)));
    const float2 f = Pair<__half>::get(lo), g = Pair<__half>::get(hi);
    x[0] = f.x; x[1] = f.y; x[2] = g.x; x[3] = g.y;
  } else {
    x[0] = (float)(int)(signed char)w; x[1] = (float)(int)(signed char)(w >> 8);
    x[2] = (float)(int)(signed char)(w >> 16); x[3] = (float)((int)w >> 24);
  }
}
// Four codes times their scale.  int8: code + 128 as the low byte of an fp32 number from 2^23 on, times the scale, less (2^23 + 128) times the
// scale (`from`): one rounding, of a number that fp32 holds.  (As far as it holds `from` too.)
template <int FMT> __device__ __forceinline__ void scaled4(uint32_t w, float scale, float from, float (&x)[4]) {
  if (FMT == WNW_PAGES_E4M3 || from == -INFINITY) {
    decode4<FMT>(w, x);
#pragma unroll
    for (int z = 0; z < 4; ++z) x[z] *= scale;
  } else {
    w ^= 0x80808080u;
#pragma unroll
    for (int z = 0; z < 4; ++z) x[z] = __fmaf_rn(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + z)), scale, from);
  }
}
// the scale's exponent for rows whose largest magnitude has these bits
template <int FMT> __device__ __forceinline__ int exponent_for(uint32_t bits) {
  // 448 = 1.75 * 2^8; 127 = 1.984375 * 2^6
  const int e = (int)(bits >> 23) - 127 - (FMT == WNW_PAGES_E4M3 ? 8 : 6) + ((bits & 0x7fffff) > (FMT == WNW_PAGES_E4M3 ? 0x600000u : 0x7e0000u));
  return max(PG_LOWEST, min(pg_highest(FMT), e));
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Magnitudes of 16-bit numbers as the bits of floats
template <typename T> struct Bits;
template <> struct Bits<__nv_bfloat16> {
  static constexpr uint32_t INF = 0x7f80;
  static __device__ __forceinline__ uint32_t as_float(uint32_t x) { return x << 16; }
};
template <> struct Bits<__half> {
  static constexpr uint32_t INF = 0x7c00;
  static __device__ __forceinline__ uint32_t as_float(uint32_t x) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)x))); }
};

// What of a sequence a call covers: tokens [first, end), rows from row0 on; everything inside the table and the tensors
struct Span { int first, end, row0; };
__device__ __forceinline__ Span span_of(const PagesView &pv, const BatchView &b, int s) {
  int r0 = b.starts[s], r1 = b.starts[s + 1], n = b.lengths[s];
  const int cap = b.stride * pv.T;      // (checked on the host to fit)
  if (r0 < 0 || r1 < r0 || r1 > b.n_rows || n < 0 || n > cap || r1 - r0 > cap - n) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) pg_report(pv, WNW_PAGES_BAD_LENGTH);
    if (r0 < 0 || r1 < r0 || n < 0) return Span{0, 0, 0};
    r1 = min(r1, b.n_rows);
    r0 = min(r0, r1);
    n = min(n, cap);
  }
  return Span{n, n + min(r1 - r0, cap - n), r0};
}

// ---- write ----
struct WriteArgs {
  PagesView pv;
  BatchView bv;
  RowsView in[2];                    // K, V
  RotaryView rot;                    // n_pairs = 0: keys are written as they are
  const int32_t *positions;
  long long axis_stride;
  int heads;                         // of K that share a CTA where keys are turned
  bool values_only;
};

constexpr int TURN_HEADS = 4;
// Keys that are turned: a thread takes 8 elements from `lo` on and 8 from `hi` on, so that the turn of a pair stays with it.
template <int D> __device__ __forceinline__ void unit_offsets(int u, int n_pairs, int neighbours, int *lo, int *hi) {
  const int turned = n_pairs / 8;
  if (u < turned && !neighbours) { *lo = 8 * u; *hi = 8 * u + n_pairs; }
  else { *lo = 16 * u; *hi = 16 * u + 8; }             // also what lies behind the pairs: 2 * n_pairs + 16 * (u - turned)
}
// 16 elements of a row turned by the angles of their eight pairs
template <typename T> __device__ __forceinline__ void turn_unit(bool neighbours, const float2 (&c)[8], uint4 &lo, uint4 &hi) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (neighbours) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float2 f = Pair<T>::get(w[q]), t = pg_turn(f.x, f.y, c[q]);
      w[q] = Pair<T>::put(t.x, t.y);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 f = Pair<T>::get(w[q]), g = Pair<T>::get(w[4 + q]);
      const float2 t = pg_turn(f.x, g.x, c[2 * q]), z = pg_turn(f.y, g.y, c[2 * q + 1]);
      w[q] = Pair<T>::put(t.x, z.x);
      w[4 + q] = Pair<T>::put(t.y, z.y);
    }
  }
  lo = make_uint4(w[0], w[1], w[2], w[3]);
  hi = make_uint4(w[4], w[5], w[6], w[7]);
}

// CTA: (KV head and K|V; pages of a sequence, one at a time; sequence).  Where keys are turned, `heads` heads of K share a CTA: its threads
// keep the angles of their pieces' pairs from one to the next.  A thread keeps its N pieces of eight elements in registers from the
// one pass over the rows to the codes: 194 MB of rows in 55 to 58 us (bytes alone: 44).  (1536 threads an SM instead of 1024 took 53 instead of 59
// when it was done.)
template <typename T, int D, int FMT, int N, int THREADS, bool TURN>
__global__ void __launch_bounds__(THREADS, (TURN && N == 8 ? 512 : TURN || N == 8 ? 1024 : 1536) / THREADS) wnw_pages_write_kernel(const __grid_constant__ WriteArgs a) {
  constexpr int PPR = D / 8;                           // pieces of a row
  __shared__ uint32_t red[THREADS / 32];
  const PagesView &pv = a.pv;
  const int s = blockIdx.z, tid = threadIdx.x, n_turned = TURN ? (pv.H + a.heads - 1) / a.heads : 0;
  const int which = TURN ? blockIdx.x >= n_turned : a.values_only ? 1 : blockIdx.x & 1;
  const int head_0 = TURN ? (which ? blockIdx.x - n_turned : blockIdx.x * a.heads) : a.values_only ? blockIdx.x : blockIdx.x >> 1;
  const int head_1 = TURN && !which ? min(pv.H, head_0 + a.heads) : head_0 + 1;
  pg_wait_for_stream();
  const Span sp = span_of(pv, a.bv, s);
  if (sp.first >= sp.end) return;
  __shared__ double turns[TURN ? 128 : 1];             // the plan: lanes want different pairs, the kernel's parameters are read one at a time
  __shared__ int axis[TURN ? 128 : 1];
  if (TURN && which == 0) {
    for (int p = tid; p < a.rot.n_pairs; p += THREADS) { turns[p] = a.rot.turns[p]; axis[p] = a.rot.axis[p]; }
    __syncthreads();
  }
  const int page0 = sp.first / pv.T, n_touched = (sp.end - 1) / pv.T - page0 + 1;
  // Piece j of the thread: row and element of the page's new rows.  Where keys are turned, pieces 2i and 2i + 1 are the two of a unit.
  auto piece = [&](int j, int *r, int *e) {
    if (TURN) {
      const int u = tid + (j >> 1) * THREADS;
      int lo, hi;
      unit_offsets<D>(u % (PPR / 2), which ? 0 : a.rot.n_pairs, a.rot.neighbours, &lo, &hi);
      *r = u / (PPR / 2);
      *e = j & 1 ? hi : lo;
    } else {
      const int u = tid + j * THREADS;
      *r = u / PPR;
      *e = u % PPR * 8;
    }
  };
  for (int i = blockIdx.y; i < n_touched; i += gridDim.y) {
    const int base = (page0 + i) * pv.T, t0 = max(sp.first, base) - base, t1 = min(sp.end - base, pv.T), rows = t1 - t0;
    const int page = a.bv.table[(long long)s * a.bv.stride + page0 + i];
    const int row0 = sp.row0 + base + t0 - sp.first;
    float2 angles[TURN ? N / 2 : 1][8];
    if (TURN && which == 0) {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const int u = tid + j * THREADS, p0 = 8 * (u % (PPR / 2)), r = u / (PPR / 2);
#pragma unroll
        for (int q = 0; q < 8; ++q)
          angles[j][q] = r < rows && p0 < a.rot.n_pairs ? pg_angle(turns[p0 + q], a.positions[axis[p0 + q] * a.axis_stride + row0 + r]) : make_float2(1.f, 0.f);
      }
    }
    if ((page < 0 || page >= pv.n_pages) && tid == 0) pg_report(pv, WNW_PAGES_BAD_PAGE);
    if (page < 0 || page >= pv.n_pages) continue;
    for (int head = head_0; head < head_1; ++head) {
      const T *in = reinterpret_cast<const T *>(a.in[which].p) + (long long)row0 * a.in[which].row + head * a.in[which].head;
      uint4 x[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int r, e;
        piece(j, &r, &e);
        x[j] = r < rows ? *reinterpret_cast<const uint4 *>(in + r * a.in[which].row + e) : make_uint4(0, 0, 0, 0);
      }
      float *scale = pv.scales + page * pv.scale_stride + head * 2 + which;
      const float old_scale = t0 ? *scale : 0.f;         // needed late, asked for early
      if (TURN && which == 0) {
#pragma unroll
        for (int j = 0; j < N; j += 2)
          if (8 * ((tid + (j >> 1) * THREADS) % (PPR / 2)) < a.rot.n_pairs) turn_unit<T>(a.rot.neighbours, angles[j >> 1], x[j], x[j + 1]);
      }
      // The largest magnitude: as integers, two at a time, while all are finite
      uint32_t both = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        both = __vmaxu2(both, __vmaxu2(__vmaxu2(x[j].x & 0x7fff7fffu, x[j].y & 0x7fff7fffu), __vmaxu2(x[j].z & 0x7fff7fffu, x[j].w & 0x7fff7fffu)));
      }
      const uint32_t top = max(both & 0xffffu, both >> 16);
      const bool odd = top >= Bits<T>::INF;               // the thread's elements are not all finite
      uint32_t most = Bits<T>::as_float(top);
      if (odd) {
        most = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const uint32_t m = w[q >> 1] >> 16 * (q & 1) & 0x7fffu;
            most = max(most, m < Bits<T>::INF ? Bits<T>::as_float(m) : 0u);
          }
        }
      }
      most = __reduce_max_sync(0xffffffffu, most);
      if ((tid & 31) == 0) red[tid >> 5] = most;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) most = max(most, red[w]);
      __syncthreads();                                   // red is free for the next page
      int e_new = exponent_for<FMT>(most);
      unsigned char *block = pv.codes + page * pv.page_stride + (long long)(head * 2 + which) * pv.T * D;
      if (t0) {
        const int had = max(PG_LOWEST, min(pg_highest(FMT), (int)(__float_as_uint(old_scale) >> 23 & 255) - 127));
        if (e_new > had) {                               // rows of before, for the raised scale
          const float down = power(max(-64, had - e_new));   // (codes / 2^64 are 0 already)
          for (int u = tid; u < t0 * (D / 16); u += THREADS) {
            uint4 *p = reinterpret_cast<uint4 *>(block + (long long)u * 16), v = *p;
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float f[4];
              decode4<FMT>(w[q], f);
              w[q] = encode4<FMT>(f[0] * down, f[1] * down, f[2] * down, f[3] * down);
            }
            *p = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
        e_new = max(e_new, had);
      }
      if (tid == 0) *scale = power(e_new);
      const float by = power(-e_new);
      const bool plain = !odd && e_new < pg_highest(FMT);   // no code beyond the largest
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int r, e;
        piece(j, &r, &e);
        if (r < rows) {
          const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
          uint32_t c[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float2 f = Pair<T>::get(w[2 * q]), g = Pair<T>::get(w[2 * q + 1]);
            if (FMT == WNW_PAGES_INT8 && plain) {          // rounded where it is added to 1.5 * 2^23: the integer is the sum's low byte
              const float u = __fmaf_rn(f.x, by, 12582912.f), v = __fmaf_rn(f.y, by, 12582912.f), y = __fmaf_rn(g.x, by, 12582912.f), z = __fmaf_rn(g.y, by, 12582912.f);
              c[q] = __byte_perm(__byte_perm(__float_as_uint(u), __float_as_uint(v), 0x0040), __byte_perm(__float_as_uint(y), __float_as_uint(z), 0x0040), 0x5410);
            } else {
              c[q] = encode4<FMT>(f.x * by, f.y * by, g.x * by, g.y * by);
            }
          }
          *reinterpret_cast<uint2 *>(block + (t0 + r) * D + e) = make_uint2(c[0], c[1]);
        }
      }
    }
  }
}

// ---- read ----
struct ReadArgs {
  PagesView pv;
  BatchView bv;
  RowsView out[2];
};

template <typename T, int D, int FMT>
__global__ void __launch_bounds__(256, 8) wnw_pages_read_kernel(const __grid_constant__ ReadArgs a) {
  constexpr int PPR = D / 8, N = 4;                    // pieces of eight codes of a row; of a thread in flight
  const PagesView &pv = a.pv;
  const int s = blockIdx.z, head = blockIdx.x >> 1, which = blockIdx.x & 1;
  pg_wait_for_stream();
  const Span sp = span_of(pv, a.bv, s);
  if (sp.first >= sp.end) return;
  const int page0 = sp.first / pv.T, n_touched = (sp.end - 1) / pv.T - page0 + 1;
  for (int i = blockIdx.y; i < n_touched; i += gridDim.y) {
    const int base = (page0 + i) * pv.T, t0 = max(sp.first, base) - base, t1 = min(sp.end - base, pv.T);
    const int page = a.bv.table[(long long)s * a.bv.stride + page0 + i];
    const bool there = page >= 0 && page < pv.n_pages;
    if (!there && threadIdx.x == 0) pg_report(pv, WNW_PAGES_BAD_PAGE);
    const float scale = there ? pv.scales[page * pv.scale_stride + head * 2 + which] : 0.f;
    const bool large = std::is_same<T, __half>::value && scale > 128.f;      // beyond fp16: 448 * 2^8 on, 127 * 2^10 on
    const float from = -8388736.f * scale;
    const unsigned char *block = pv.codes + (there ? page : 0) * pv.page_stride + ((long long)(head * 2 + which) * pv.T + t0) * D;
    T *out = reinterpret_cast<T *>(a.out[which].p) + (long long)(sp.row0 + base + t0 - sp.first) * a.out[which].row + head * a.out[which].head;
    const int all = (t1 - t0) * PPR;
    for (int u0 = threadIdx.x; u0 < all; u0 += 256 * N) {
      uint2 v[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int u = u0 + 256 * k;
        v[k] = there && u < all ? *reinterpret_cast<const uint2 *>(block + u * 8) : make_uint2(0, 0);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int u = u0 + 256 * k;
        if (u < all) {
          float f[8];
          scaled4<FMT>(v[k].x, scale, from, reinterpret_cast<float (&)[4]>(f[0]));
          scaled4<FMT>(v[k].y, scale, from, reinterpret_cast<float (&)[4]>(f[4]));
          if (large) {
#pragma unroll
            for (int z = 0; z < 8; ++z)
              if (fabsf(f[z]) > 65504.f) f[z] = copysignf(65504.f, f[z]);
          }
          *reinterpret_cast<uint4 *>(out + (long long)(u / PPR) * a.out[which].row + u % PPR * 8) =
              make_uint4(Pair<T>::put(f[0], f[1]), Pair<T>::put(f[2], f[3]), Pair<T>::put(f[4], f[5]), Pair<T>::put(f[6], f[7]));
        }
      }
    }
  }
}

// CTAs along a sequence's pages: as many as its rows can touch, by what the caller says of the rows, but no more than eight times what the
// sequences touch on average; the kernels' loops cover the rest.
int pages_touched(const wnw_batch_t &b, int T) {
  const int rows = b.max_rows > 0 ? std::min(b.max_rows, b.n_rows) : b.n_rows;
  const long long most = (rows + T - 2ll) / T + 1, mean = ((long long)b.n_rows / T + 2ll * b.n_seqs) / b.n_seqs + 1;
  return (int)std::min({most, 8 * mean, 65535ll});
}

template <typename T, int D, int FMT, bool TURN> cudaError_t launch_write(const WriteArgs &a, dim3 grid, cudaStream_t st) {
  const int pieces = a.pv.T * (D / 8);
  if (pieces <= 512) return pg_launch(wnw_pages_write_kernel<T, D, FMT, 4, 128, TURN>, grid, 128, 0, st, 0, a);
  if (pieces <= 1024) return pg_launch(wnw_pages_write_kernel<T, D, FMT, 4, 256, TURN>, grid, 256, 0, st, 0, a);
  if (pieces <= 2048) return pg_launch(wnw_pages_write_kernel<T, D, FMT, 8, 256, TURN>, grid, 256, 0, st, 0, a);
  return pg_launch(wnw_pages_write_kernel<T, D, FMT, 8, 512, TURN>, grid, 512, 0, st, 0, a);
}
// Angles are the larger part of turning a key, and the same for all heads, so that several share a CTA, and the values go by themselves (the
// kernel that turns has registers for fewer threads): 30000 tokens of 8 heads of 128, a head a CTA 91 us, four 78, the values apart 66, 1024
// threads an SM 57 (53 in e4m3; bytes alone: 28); wnw_rotate and then a write take 60 (58).  A few new rows are done soonest a head a CTA,
// values in the same launch.
template <typename T, int D, int FMT> cudaError_t launch_write(WriteArgs &a, int max_rows, dim3 grid, cudaStream_t st) {
  a.values_only = false;
  if (!a.rot.n_pairs) { grid.x = 2 * a.pv.H; return launch_write<T, D, FMT, false>(a, grid, st); }
  const bool few = max_rows > 0 && max_rows <= 8;
  a.heads = few ? 1 : TURN_HEADS;
  grid.x = (a.pv.H + a.heads - 1) / a.heads + (few ? a.pv.H : 0);
  const cudaError_t e = launch_write<T, D, FMT, true>(a, grid, st);
  if (few || e != cudaSuccess) return e;
  a.values_only = true;
  grid.x = a.pv.H;
  return launch_write<T, D, FMT, false>(a, grid, st);
}
template <typename T> cudaError_t launch_write(WriteArgs &a, int d, int fmt, int max_rows, dim3 grid, cudaStream_t st) {
  if (d == 64) return fmt == WNW_PAGES_E4M3 ? launch_write<T, 64, WNW_PAGES_E4M3>(a, max_rows, grid, st) : launch_write<T, 64, WNW_PAGES_INT8>(a, max_rows, grid, st);
  return fmt == WNW_PAGES_E4M3 ? launch_write<T, 128, WNW_PAGES_E4M3>(a, max_rows, grid, st) : launch_write<T, 128, WNW_PAGES_INT8>(a, max_rows, grid, st);
}
template <typename T> cudaError_t launch_read(const ReadArgs &a, int d, int fmt, dim3 grid, cudaStream_t st) {
  if (d == 64) return pg_launch(fmt == WNW_PAGES_E4M3 ? wnw_pages_read_kernel<T, 64, WNW_PAGES_E4M3> : wnw_pages_read_kernel<T, 64, WNW_PAGES_INT8>, grid, 256, 0, st, 0, a);
  return pg_launch(fmt == WNW_PAGES_E4M3 ? wnw_pages_read_kernel<T, 128, WNW_PAGES_E4M3> : wnw_pages_read_kernel<T, 128, WNW_PAGES_INT8>, grid, 256, 0, st, 0, a);
}

wnw_status_t check_rows_call(const wnw_pages_rows_t *c, PagesView *pv, BatchView *bv) {
  if (!c) return WNW_ERR_INVALID_ARG;
  const wnw_status_t rc = pg_view(c->pages, &c->batch, pv, bv);
  if (rc != WNW_OK) return rc;
  if (c->dtype != WNW_DTYPE_BF16 && c->dtype != WNW_DTYPE_FP16) return WNW_ERR_UNSUPPORTED;
  for (const wnw_rows_t *r : {&c->k, &c->v})
    if (r->n_heads != c->pages->n_kv_heads || (c->batch.n_rows && (!r->dev || !pg_vector_rows(*r, c->dtype)))) return WNW_ERR_INVALID_ARG;
  return WNW_OK;
}

}  // namespace

wnw_status_t pg_view(const wnw_pages_t *p, PagesView *v) {
  if (!p || p->n_pages < 0 || p->page_stride < 0 || p->scale_stride < 0) return WNW_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return WNW_ERR_UNSUPPORTED;
  if (p->page_tokens < PG_GR || p->page_tokens > PG_MAX_PAGE || p->page_tokens % PG_GR) return WNW_ERR_UNSUPPORTED;
  if (p->n_kv_heads < 1 || p->format < WNW_PAGES_E4M3 || p->format > WNW_PAGES_INT8) return WNW_ERR_INVALID_ARG;
  if (p->n_kv_heads > 1024) return WNW_ERR_CAPACITY;
  const long long page = 2ll * p->n_kv_heads * p->page_tokens * p->head_dim, scales = 2ll * p->n_kv_heads;
  if (p->n_pages && (!p->codes_dev || !p->scales_dev || (uintptr_t)p->codes_dev % 16 || (uintptr_t)p->scales_dev % 4)) return WNW_ERR_INVALID_ARG;
  if ((p->page_stride && (p->page_stride < page || p->page_stride % 16 || p->page_stride >= 1ll << 40)) || (p->scale_stride && p->scale_stride < scales)) return WNW_ERR_INVALID_ARG;
  if ((uintptr_t)p->status_dev % 4) return WNW_ERR_INVALID_ARG;
  *v = PagesView{(unsigned char *)p->codes_dev, p->scales_dev, p->page_stride ? (long long)p->page_stride : page, p->scale_stride ? (long long)p->scale_stride : scales,
                 p->n_pages, p->page_tokens, p->n_kv_heads, p->status_dev};
  return WNW_OK;
}

wnw_status_t pg_view(const wnw_pages_t *p, const wnw_batch_t *b, PagesView *pv, BatchView *bv) {
  const wnw_status_t rc = pg_view(p, pv);
  if (rc != WNW_OK) return rc;
  if (!b || b->n_seqs < 0 || b->n_rows < 0 || b->max_rows < 0 || b->table_stride < 0) return WNW_ERR_INVALID_ARG;
  if (b->n_seqs > PG_MAX_SEQS || (long long)b->table_stride * p->page_tokens > 1ll << 30) return WNW_ERR_CAPACITY;
  if (b->n_seqs && (!b->lengths_dev || !b->row_starts_dev || (b->table_stride && !b->page_table_dev))) return WNW_ERR_INVALID_ARG;
  for (const void *q : {(const void *)b->page_table_dev, (const void *)b->lengths_dev, (const void *)b->row_starts_dev})
    if ((uintptr_t)q % 4) return WNW_ERR_INVALID_ARG;
  *bv = BatchView{b->page_table_dev, b->lengths_dev, b->row_starts_dev, b->table_stride, b->n_seqs, b->n_rows};
  return WNW_OK;
}

wnw_status_t pg_sms(int device, int *n) {
  static std::atomic<int> known[64];
  if (device < 0 || device >= 64) return WNW_ERR_INVALID_ARG;
  int v = known[device].load(std::memory_order_relaxed);
  if (!v) {
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) { cudaGetLastError(); return WNW_ERR_CUDA; }
    known[device].store(v, std::memory_order_relaxed);
  }
  *n = v;
  return WNW_OK;
}

}  // namespace wnw

using namespace wnw;

extern "C" wnw_status_t wnw_pages_write(const wnw_pages_rows_t *call) {
  WriteArgs a;
  wnw_status_t rc = check_rows_call(call, &a.pv, &a.bv);
  if (rc != WNW_OK) return rc;
  a.rot.n_pairs = 0;
  if (call->rotary) {
    if ((rc = rotary_view(call->rotary, call->pages->head_dim, 0, &a.rot)) != WNW_OK) return rc;
    if (a.rot.n_pairs % 8) return WNW_ERR_UNSUPPORTED;
    if (call->batch.n_rows && (!call->positions_dev || (uintptr_t)call->positions_dev % 4)) return WNW_ERR_INVALID_ARG;
  }
  a.positions = call->positions_dev;
  a.axis_stride = call->axis_stride;
  a.in[0] = rows_view(call->k);
  a.in[1] = rows_view(call->v);
  if (!call->batch.n_seqs || !call->batch.n_rows) return WNW_OK;
  OnDevice on(call->pages->device);
  if (!on.ok) return WNW_ERR_CUDA;
  const dim3 grid(1, pages_touched(call->batch, a.pv.T), call->batch.n_seqs);            // x: heads (a token's lie beside one another)
  const cudaStream_t st = (cudaStream_t)call->cuda_stream;
  const int d = call->pages->head_dim, fmt = call->pages->format, rows = call->batch.max_rows;
  const cudaError_t e = call->dtype == WNW_DTYPE_BF16 ? launch_write<__nv_bfloat16>(a, d, fmt, rows, grid, st) : launch_write<__half>(a, d, fmt, rows, grid, st);
  return e == cudaSuccess ? WNW_OK : WNW_ERR_CUDA;
}

extern "C" wnw_status_t wnw_pages_read(const wnw_pages_rows_t *call) {
  ReadArgs a;
  const wnw_status_t rc = check_rows_call(call, &a.pv, &a.bv);
  if (rc != WNW_OK) return rc;
  if (call->rotary) return WNW_ERR_INVALID_ARG;
  a.out[0] = rows_view(call->k);
  a.out[1] = rows_view(call->v);
  if (!call->batch.n_seqs || !call->batch.n_rows) return WNW_OK;
  OnDevice on(call->pages->device);
  if (!on.ok) return WNW_ERR_CUDA;
  const dim3 grid(2 * a.pv.H, pages_touched(call->batch, a.pv.T), call->batch.n_seqs);   // (a token's heads lie beside one another)
  const cudaStream_t st = (cudaStream_t)call->cuda_stream;
  const int d = call->pages->head_dim, fmt = call->pages->format;
  const cudaError_t e = call->dtype == WNW_DTYPE_BF16 ? launch_read<__nv_bfloat16>(a, d, fmt, grid, st) : launch_read<__half>(a, d, fmt, grid, st);
  return e == cudaSuccess ? WNW_OK : WNW_ERR_CUDA;
}
