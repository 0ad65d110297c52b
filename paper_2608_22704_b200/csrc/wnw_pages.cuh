// What the operators around the paged eight-bit store share: argument checks, the kernels' view of store and batch, the turn of a
// pair by its position.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/wnw.h"

namespace wnw {

constexpr int PG_GR = 16;            // tokens of a granule; a page is whole granules
constexpr int PG_MAX_SEQS = 1024;
constexpr int PG_MAX_PAGE = 256;
constexpr int PG_LOWEST = -110;      // exponent of the smallest scale: stored values stay normal floats
__host__ __device__ constexpr int pg_highest(int fmt) { return fmt == WNW_PAGES_INT8 ? 121 : 119; }   // ... and finite ones

struct PagesView {
  unsigned char *codes;
  float *scales;
  long long page_stride, scale_stride;
  int n_pages, T, H;
  int32_t *status;
};
struct BatchView {
  const int32_t *table, *lengths, *starts;
  int stride, n_seqs, n_rows;
};
struct RowsView {
  unsigned char *p;
  long long row, head;               // strides in elements
};
struct RotaryView {                  // turns a position and pair, so that the reduction of the angle is a rounding to whole turns
  double turns[128];
  uint8_t axis[128];
  int n_pairs, neighbours;
  float sign;
};

__device__ __forceinline__ void pg_report(const PagesView &pv, int bit) {
  if (pv.status) atomicOr(pv.status, bit);
}

// cos and sin of positions * frequency.  64 bits hold position x turns to 2^-22 of a turn at the farthest int32 position; what is left
// after whole turns is taken in 32.
__device__ __forceinline__ float2 pg_angle(double turns, int position) {
  double t = (double)position * turns;
  t -= rint(t);
  float2 cs;
  sincospif(2.f * (float)t, &cs.y, &cs.x);
  return cs;
}

// The turn of a pair, with its roundings spelled out: wherever it is done, the result is the same bits.
__device__ __forceinline__ float2 pg_turn(float a, float b, float2 cs) {
  return make_float2(__fmaf_rn(-b, cs.y, __fmul_rn(a, cs.x)), __fmaf_rn(a, cs.y, __fmul_rn(b, cs.x)));
}

template <typename T> struct Pair;     // two neighbouring elements of a 16-bit type as floats and back
template <> struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ float2 get(uint32_t x) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t put(float a, float b) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t *>(&v); }
};
template <> struct Pair<__half> {
  static __device__ __forceinline__ float2 get(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2 *>(&x)); }
  static __device__ __forceinline__ uint32_t put(float a, float b) { const __half2 v = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t *>(&v); }
};

struct OnDevice {   // the device is current while this lives
  int prev = -1, dev;
  bool ok;
  explicit OnDevice(int device) : dev(device) {
    ok = cudaGetDevice(&prev) == cudaSuccess && (prev == device || cudaSetDevice(device) == cudaSuccess);
    if (!ok) cudaGetLastError();
  }
  ~OnDevice() { if (ok && prev != dev) cudaSetDevice(prev); }
};

inline size_t pg_elem(int dtype) { return dtype == WNW_DTYPE_FP32 ? 4 : 2; }
inline bool pg_vector_rows(const wnw_rows_t &r, int dtype) {
  const long long m = 16 / pg_elem(dtype);
  return (uintptr_t)r.dev % 16 == 0 && r.row_stride % m == 0 && r.head_stride % m == 0;
}
wnw_status_t pg_view(const wnw_pages_t *p, PagesView *v);
wnw_status_t pg_view(const wnw_pages_t *p, const wnw_batch_t *b, PagesView *pv, BatchView *bv);
wnw_status_t rotary_view(const wnw_rotary_t *r, int head_dim, int inverse, RotaryView *v);
inline RowsView rows_view(const wnw_rows_t &r) { return RowsView{(unsigned char *)r.dev, (long long)r.row_stride, (long long)r.head_stride}; }

// ---- launches that start while their predecessor on the stream ends ----
// The next launch may be brought onto the SMs from here on.  Only where that is this call's own, which waits before it touches anything: a
// layer of a step whose queries are given in advance does not.
__device__ __forceinline__ void pg_let_next_start() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }
// Everything before on the stream has completed.  By every CTA, before its first access to memory: then "completed" holds along chains.
__device__ __forceinline__ void pg_wait_for_stream() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
template <typename... P, typename... A>
cudaError_t pg_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, const A &...args) {   // cluster: CTAs, 0: none
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cluster) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

// SMs of a device, asked for once.
wnw_status_t pg_sms(int device, int *n);

}  // namespace wnw
