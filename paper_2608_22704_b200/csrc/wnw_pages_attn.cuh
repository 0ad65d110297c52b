// What the attention kernels over the paged store share: arguments, partial results of heads that several CTAs work on, codes as fp16.
#pragma once
#include "../../include/wnw_debug.h"
#include "wnw_pages.cuh"

namespace wnw {

constexpr float LAZY = 8.f;          // log2 by which a score may exceed the reference before that follows
constexpr float NOTHING = -3e38f;    // the references before a token is seen: finite, so that differences are numbers

// ---- workspace: per CTA two partial results (0: a head begun in an earlier CTA, 1: a head that ends in a later one) ----
struct PartHead { int r0, n, h, tile, n_parts, pad[3]; };  // of slot 1: rows of its sequence, which head and item, CTAs that share it (0: none)
struct PartRow { float m, big_m, l, pad; };

// A head's query rows come in items of `blocks` blocks: block i of item t holds query tokens [(t * blocks + i) * rt, ... + rt) in its
// rows tok * g + head of the group, and has `rb` rows in a partial result.
struct AttendArgs {
  PagesView pv;
  BatchView bv;
  RowsView q, out;
  float *lse;
  int Hq, g, rt, rb, blocks;
  int dtype, causal;
  int lose;                          // WNW_DEBUG_WAIT_*: waits that are to run out
  uint32_t values_parity;            // 1; 0 where the waits for P V are to run out: not every tile has one, and of a phase that never ends the odd ones are over
  uint32_t wait_clocks;              // after which a wait gives up
  float scale_log2;
  float *part_o;                     // [CTA][2][blocks * rb][D]
  PartRow *part_row;                 // [CTA][2][blocks * rb]
  PartHead *part_head;               // [CTA]
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}
// Four codes as fp16: the lower two in `lo`, the upper two in `hi`.
template <int FMT> __device__ __forceinline__ void to_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
  if constexpr (FMT == WNW_PAGES_E4M3) {
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(lo) : "h"((unsigned short)w));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(hi) : "h"((unsigned short)(w >> 16)));
  } else {   // code + 128 as the low byte of an fp16 number between 1024 and 2048, less 1152: exact
    w ^= 0x80808080u;
    const uint32_t x = __byte_perm(w, 0x64646464u, 0x4140), y = __byte_perm(w, 0x64646464u, 0x4342), off = 0x64806480u;
    const __half2 o = *reinterpret_cast<const __half2 *>(&off);
    const __half2 p = __hsub2(*reinterpret_cast<const __half2 *>(&x), o), q = __hsub2(*reinterpret_cast<const __half2 *>(&y), o);
    lo = *reinterpret_cast<const uint32_t *>(&p);
    hi = *reinterpret_cast<const uint32_t *>(&q);
  }
}


// x / y of numbers that are not negative; a 64-bit division takes some hundred instructions, and hardly ever is one needed
__device__ __forceinline__ long long quotient(long long x, long long y) {
  return ((x | y) >> 32) ? x / y : (long long)((uint32_t)x / (uint32_t)y);
}

// The attention of many query rows (wnw_pages_prompt.cu): 128-row tiles, two at a time.
constexpr int PP_ROWS = 128, PP_BLOCKS = 2;
constexpr uint32_t PP_WAIT_CLOCKS = 2000000000;
cudaError_t launch_prompt(const AttendArgs &a, int head_dim, int format, int n_ctas, int device, cudaStream_t st);

}  // namespace wnw
