// wnw_pages_attend for many query rows of a sequence (a prompt, a piece of one): the same formula and the same two references as the kernel
// for few rows (wnw_pages_attn.cu), on the fifth-generation tensor cores.
//
// What bounds it: two products of 128 x 128 x head_dim per tile of 128 tokens and 128 query rows, 1024 clocks at the tensor cores' rate for a
// head_dim of 128, and one exp2 per score, of which an SM does 16 a clock: 1024 clocks too.  The codes are few beside that, but have to become
// fp16 in shared memory before the tensor cores can take them; so a CTA works on two tiles of query rows at a time and turns each tile of codes
// once.  2049 rows of 32 heads behind 13015 tokens of 8 KV heads take 607 us: 776 TFLOP/s, where a library's large bf16 product reaches 1639.
// A tile of tokens takes 4900 clocks for the two row tiles, not 2048: each row tile's chain of scores, softmax and values is as long as that
// (softmax some 3200), with two of them side by side, for tensor memory holds no third; Q K^T, both of whose operands come from shared memory, takes 680
// to 970 clocks instead of 512 beside the other traffic there.
//
// 16 warps: 0-3 and 4-7 softmax of the two row tiles (a thread a row), 8-11 codes to fp16, 12 issues the products, 13 has the tensor memory.
//   S_i = Q_i K^T         operands in shared memory, 128-byte swizzle, rows of 64 elements; S_i fp32 in tensor memory
//   O_i += P_i V          P_i (fp16) in tensor memory over S_i, V as it lies (its rows are the contracted index)
// Tensor memory: S_0 S_1 O_0 O_1, 128 columns each.  While the products of one row tile run, the other's softmax does.
//
// Work is laid on a line as in the other kernel, in tiles of 128 tokens that the rows of an item see; every CTA takes an equal stretch.
// Not-a-numbers among V codes are zero in the product (a weight of zero would not keep them from rows that do not see them); the first
// token that has one is kept per element, and rows that see it get one.
#include <algorithm>
#include <atomic>
#include <cstring>

#include "wnw_pages_attn.cuh"

namespace wnw {
namespace {

constexpr int PP_THREADS = 512, PP_TOKENS = 128;
constexpr uint32_t COL_S = 0, COL_O = 256;

constexpr uint32_t TILE_EVEN = 1;    // all granules have the same scales
constexpr uint32_t TILE_HOLES = 2;   // a granule is not there, its page missing or the sequence at its end

// Where a warp is on the line: the item and the tiles of it that fall to this CTA.  Every warp walks by itself.
struct Walk {
  long long left;                    // tiles of the CTA's stretch from this segment on
  int s, h, t, n_it;                 // sequence, KV head, item of query rows, items of the head
  int n, len, r0;                    // query tokens and tokens of the sequence, its first row
  int k0, k1, need;                  // the segment's tiles; tiles of the item
};

struct Shared {
  uint64_t k_full[2], k_free[2], v_full[2], v_free[2], q_full[2], s_full[2], p_ready[2], o_done[2], begun;
  uint32_t tmem;
  uint32_t dead;                     // a wait ran out: nobody waits any more, and no product is issued
  float2 scale[4][8];                // per tile and granule: 2^eK, eV; eV = -inf: the granule is not there
  uint32_t flags[4];                 // TILE_* below
  // Not-a-numbers among the V codes, per warp that turns codes (each keeps its own), four segments deep (a slot is used again when the
  // slower row tile has left it): whether there are any, and then the first token that has one, per element.
  int nan_any[4][4], nan_first[4][4][128];
  long long sums[17];
  long long line[PG_MAX_SEQS + 1];   // tiles before each sequence
  uint64_t drained;                  // the products are done, and no more come
  int32_t *status;
  uint32_t clocks;                   // after which a wait gives up
};
template <int D> constexpr size_t tiles_bytes() { return 8 * 128 * D * 2 / 4 * 3; }   // 2 Q + 2 K + 2 V of 128 rows
template <int D> constexpr size_t smem_bytes() { return tiles_bytes<D>() + sizeof(Shared) + 1024; }

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(bar)) : "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_smem() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void commit(uint64_t *bar) { commit(smem_u32(bar)); }
// Bounded waits.  After about a second of SM clocks the CTA gives up for good, and says so: the thread of the products (PRODUCTS) waits for
// those under way and ends; the other warps wait for that, so that nothing they touch is in use, and then go on without waiting; their rows
// become not-a-numbers where they are put out.  All of it lies out of the way of a wait that ends: as branches behind the waits it made 607 us
// 618 where the file's head says 2049 rows.
template <bool PRODUCTS> __device__ __noinline__ void wait_long(uint32_t bar, uint32_t parity, volatile Shared *sh) {
  const long long t0 = clock64();
  while (!try_wait(bar, parity)) {
    if (!sh->dead && clock64() - t0 <= sh->clocks) continue;
    if (!sh->dead && sh->status) atomicOr(sh->status, WNW_PAGES_TIMEOUT);
    sh->dead = 1;
    const uint32_t drained = smem_u32((const void *)&sh->drained);
    if (PRODUCTS) commit(drained);
    for (const long long t1 = clock64(); !try_wait(drained, 0) && clock64() - t1 <= PP_WAIT_CLOCKS;) {}
    if (PRODUCTS) asm volatile("exit;\n");
    return;
  }
}
template <bool PRODUCTS = false> __device__ __forceinline__ void wait(uint64_t *bar, uint32_t parity, Shared &sh) {
  if (!try_wait(smem_u32(bar), parity & 1)) wait_long<PRODUCTS>(smem_u32(bar), parity & 1, &sh);
}
// Operands of 128-byte rows in the 128-byte swizzle, eight rows an atom.  lbo: from 64 elements of the outer index to the next 64, where that
// is the contiguous one (V); not used otherwise.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lbo) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 accumulators, fp16 operands, 128 rows, n columns; the B operand's rows the contracted index or not
constexpr uint32_t shape(int n, bool b_rows_contracted) { return 1u << 4 | (b_rows_contracted ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | 8u << 24; }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// 32 or 16 columns of a thread's row
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&x)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19,"
               " %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
               : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]),
               "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(x[16]), "=r"(x[17]), "=r"(x[18]), "=r"(x[19]),
               "=r"(x[20]), "=r"(x[21]), "=r"(x[22]), "=r"(x[23]), "=r"(x[24]), "=r"(x[25]), "=r"(x[26]), "=r"(x[27]), "=r"(x[28]), "=r"(x[29]),
               "=r"(x[30]), "=r"(x[31])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_loaded(uint32_t (&x)[32]) {   // (the registers go through, so that nothing reads them before)
  asm volatile("tcgen05.wait::ld.sync.aligned;\n" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
               "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]), "+r"(x[16]), "+r"(x[17]),
               "+r"(x[18]), "+r"(x[19]), "+r"(x[20]), "+r"(x[21]), "+r"(x[22]), "+r"(x[23]), "+r"(x[24]), "+r"(x[25]), "+r"(x[26]), "+r"(x[27]),
               "+r"(x[28]), "+r"(x[29]), "+r"(x[30]), "+r"(x[31]) : : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&x)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
               : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]),
               "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_loaded(uint32_t (&x)[16]) {   // (the registers go through, so that nothing reads them before)
  asm volatile("tcgen05.wait::ld.sync.aligned;\n" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
               "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]) : : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&x)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n"
               ::"r"(addr), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]),
               "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]) : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// ---- the softmax of a tile's 128 tokens, by the thread of a query row ----
__device__ __forceinline__ uint64_t two(float x, float y) { return (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float lower(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float upper(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// The largest score (`top`), and the largest with its V scale (`big`).  seen: of the tile's tokens, by the row.  32 tokens at a time, the
// next ones on their way meanwhile; x[0] holds the first ones again afterwards.  (The loops are rolled up to two turns of 32: all 128 laid out
// crowd the instruction cache and the registers, 631 us instead of 596 when it was done, where the file's head says 2049 rows.)
template <bool MASKED>
__device__ __forceinline__ void row_top(uint32_t t_s, uint32_t (&x)[2][32], const float2 *scale, bool even, float f_row, int seen, float &top, float &big) {
  top = -INFINITY;
  big = NOTHING;
#pragma unroll 1
  for (int k0 = 0; k0 < 4; k0 += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + h;
      tmem_loaded(x[h]);
      tmem_load(t_s + 32 * ((k + 1) & 3), x[h ^ 1]);
      float t[2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float y[16];
#pragma unroll
        for (int z = 0; z < 16; ++z) {
          y[z] = __uint_as_float(x[h][16 * g + z]);
          if (MASKED && 32 * k + 16 * g + z >= seen) y[z] = -INFINITY;
        }
        t[g] = fmaxf(max3(max3(y[0], y[1], y[2]), max3(y[3], y[4], y[5]), max3(y[6], y[7], y[8])),
                     max3(max3(y[9], y[10], y[11]), max3(y[12], y[13], y[14]), y[15]));
      }
      if (!MASKED && even) {
        top = max3(top, t[0], t[1]);
      } else {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const float2 sc = scale[2 * k + g];
          const float s = MASKED && (t[g] == -INFINITY || sc.y == -INFINITY) ? -INFINITY : t[g] * (f_row * sc.x);
          top = fmaxf(top, s);
          big = fmaxf(big, s + sc.y);
        }
      }
    }
  }
  if (!MASKED && even) {
    top *= f_row * scale[0].x;
    big = top + scale[0].y;
  }
}
// The weights 2^(s + eV - M), as fp16 to P's columns, and their sum as 2^(s - m) onto l.  They are taken as 2^(s - m - d), d = M - eV - m,
// so that the sum is that of a granule times 2^d; where d is so large that weights that count in the denominator would vanish (a page of
// zeros beside one of large values), d is 60 there and the rest a factor of its own (DEEP).  P's columns lie where S has been read.
template <bool MASKED, bool DEEP>
__device__ __forceinline__ void row_weights(uint32_t t_s, uint32_t (&x)[2][32], const float2 *scale, float f_row, int seen, float m, float big_m, float &l) {
#pragma unroll 1
  for (int k0 = 0; k0 < 4; k0 += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + h;
      tmem_loaded(x[h]);
      if (k < 3) tmem_load(t_s + 32 * (k + 1), x[h ^ 1]);
      uint32_t p[16];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float2 sc = scale[2 * k + g];
        const bool hole = MASKED && sc.y == -INFINITY;
        const int lim = hole ? 0 : seen;
        const float f = f_row * sc.x, d = hole ? 0.f : big_m - sc.y - m, d2 = DEEP ? fminf(d, 60.f) : d, off = -(m + d2), rest = DEEP ? ex2(d2 - d) : 1.f;
        const uint64_t ff = two(f, f), oo = two(off, off);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int z = 0; z < 16; z += 2) {
          const uint64_t y = fma2(two(__uint_as_float(x[h][16 * g + z]), __uint_as_float(x[h][16 * g + z + 1])), ff, oo);
          float u = ex2(lower(y)), v = ex2(upper(y));
          if (MASKED && 32 * k + 16 * g + z >= lim) u = 0.f;
          if (MASKED && 32 * k + 16 * g + z + 1 >= lim) v = 0.f;
          sum[z >> 1 & 1] = add2(sum[z >> 1 & 1], two(u, v));
          p[8 * g + z / 2] = DEEP ? half2_of(u * rest, v * rest) : half2_of(u, v);
        }
        const uint64_t both = add2(sum[0], sum[1]);
        l = __fmaf_rn(lower(both) + upper(both), ex2(d2), l);
      }
      tmem_store(t_s + 16 * k, p);
    }
  }
}

// ---- the line ----
// Query tokens, tokens and first row of a sequence, clipped to what is there; whether they had to be
__device__ __forceinline__ bool sequence(const AttendArgs &a, int s, int *n, int *len, int *r0) {
  int x = a.bv.starts[s], y = a.bv.starts[s + 1], l = a.bv.lengths[s];
  const int cap = a.bv.stride * a.pv.T;
  const bool bad = x < 0 || y < x || y > a.bv.n_rows || l < 0 || l > cap;
  x = max(x, 0);
  *n = max(0, min(y, a.bv.n_rows) - x);
  *r0 = x;
  *len = max(0, min(l, cap));
  return bad;
}
// Tiles of tokens that the rows of item t see; one at least, for rows that see nothing are still to be written
__device__ __forceinline__ int tiles_of(const AttendArgs &a, int t, int n, int len) {
  const int last = min(len, a.causal ? len - n + min((t + 1) * PP_BLOCKS * a.rt, n) : len);
  return last > 0 ? (last + PP_TOKENS - 1) / PP_TOKENS : 1;
}
__device__ __forceinline__ int items_of(const AttendArgs &a, int n) { return (n + PP_BLOCKS * a.rt - 1) / (PP_BLOCKS * a.rt); }
__device__ __forceinline__ long long head_tiles(const AttendArgs &a, int n, int len) {
  long long sum = 0;
  if (!a.causal) return (long long)items_of(a, n) * tiles_of(a, 0, n, len);
  for (int t = 0, e = items_of(a, n); t < e; ++t) sum += tiles_of(a, t, n, len);
  return sum;
}
__device__ long long lay_out(const AttendArgs &a, Shared &sh) {
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, n_seqs = a.bv.n_seqs;
  long long base = 0;
  for (int at = 0; at < n_seqs; at += PP_THREADS) {
    const int s = at + tid;
    long long mine = 0;
    if (s < n_seqs) {
      int n, len, r0;
      if (sequence(a, s, &n, &len, &r0) && blockIdx.x == 0) pg_report(a.pv, WNW_PAGES_BAD_LENGTH);
      mine = head_tiles(a, n, len) * a.pv.H;
    }
    long long run = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += x;
    }
    if (lane == 31) sh.sums[w] = run;
    __syncthreads();
    long long before = base;
    for (int k = 0; k < PP_THREADS / 32; ++k) {
      if (k < w) before += sh.sums[k];
      base += sh.sums[k];
    }
    if (s < n_seqs) sh.line[s] = before + run - mine;
    __syncthreads();
  }
  if (tid == 0) sh.line[n_seqs] = base;
  __syncthreads();
  return base;
}
__device__ __forceinline__ void enter_item(const AttendArgs &a, Walk &w) {
  w.need = tiles_of(a, w.t, w.n, w.len);
  w.k1 = (int)min((long long)w.need, w.k0 + w.left);
}
// The first segment of a stretch that begins at x and holds `left` > 0 tiles
__device__ __forceinline__ void walk_begin(const AttendArgs &a, const Shared &sh, long long x, long long left, Walk &w) {
  int lo = 0, hi = a.bv.n_seqs;
  while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (sh.line[mid] <= x) lo = mid; else hi = mid; }
  w.s = lo;
  w.left = left;
  sequence(a, lo, &w.n, &w.len, &w.r0);
  w.n_it = items_of(a, w.n);
  const long long per = (sh.line[lo + 1] - sh.line[lo]) / a.pv.H;
  x -= sh.line[lo];
  w.h = (int)(x / per);
  x -= w.h * per;
  if (!a.causal) {
    const int one = tiles_of(a, 0, w.n, w.len);
    w.t = (int)(x / one);
    x -= (long long)w.t * one;
  } else {
    w.t = 0;
    for (int one; x >= (one = tiles_of(a, w.t, w.n, w.len)); ++w.t) x -= one;
  }
  w.k0 = (int)x;
  enter_item(a, w);
}
// The next one; false at the stretch's end
__device__ __forceinline__ bool walk_on(const AttendArgs &a, Walk &w) {
  w.left -= w.k1 - w.k0;
  if (w.left <= 0) return false;
  w.k0 = 0;
  if (++w.t == w.n_it) {
    w.t = 0;
    if (++w.h == a.pv.H) {
      w.h = 0;
      do {
        ++w.s;
        sequence(a, w.s, &w.n, &w.len, &w.r0);
      } while (w.n == 0);
      w.n_it = items_of(a, w.n);
    }
  }
  enter_item(a, w);
  return true;
}
__device__ __forceinline__ bool two_blocks(const AttendArgs &a, const Walk &w) { return (w.t * PP_BLOCKS + 1) * a.rt < w.n; }

// 16 codes as fp16: two pieces of 16 bytes
template <int FMT> __device__ __forceinline__ void sixteen(uint4 c, uint4 &lo, uint4 &hi) {
  to_half<FMT>(c.x, lo.x, lo.y);
  to_half<FMT>(c.y, lo.z, lo.w);
  to_half<FMT>(c.z, hi.x, hi.y);
  to_half<FMT>(c.w, hi.z, hi.w);
}

// A tile of codes on its way: what a thread of the four warps that turn codes into fp16 keeps of it.  It takes 16 codes of a row at a time;
// eight neighbouring lanes take four pieces of two rows each, which lie in different banks once swizzled.
template <int D> struct Codes {
  static constexpr int PASSES = D == 128 ? 8 : 4;      // rows of a thread
  uint4 k[PASSES], v[PASSES];
  uint32_t meta;                                       // lanes 0-7: of that granule
};

template <int D, int FMT>
__global__ void __launch_bounds__(PP_THREADS, 1) wnw_pages_prompt_kernel(const __grid_constant__ AttendArgs a) {
  extern __shared__ unsigned char raw[];
  unsigned char *tiles = raw + (1024 - (smem_u32(raw) & 1023)) % 1024;
  constexpr uint32_t TILE = 128 * D * 2, HALF = 128 * 128;   // bytes of an operand, and of 64 elements of its rows
  unsigned char *q_s = tiles, *k_s = tiles + 2 * TILE, *v_s = tiles + 4 * TILE;
  Shared &sh = *reinterpret_cast<Shared *>(tiles + 6 * TILE);
  const PagesView &pv = a.pv;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  if (tid == 0) {
    auto init = [&](uint64_t *bar, int count, int kind) {   // (for arrivals that nothing makes, where a test asks for waits that run out)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_u32(bar)), "r"(count + (a.lose & kind ? 1 << 16 : 0)) : "memory");
    };
    for (int i = 0; i < 2; ++i) {
      init(&sh.k_full[i], 4, WNW_DEBUG_WAIT_K_FULL);
      init(&sh.v_full[i], 4, WNW_DEBUG_WAIT_V_FULL);
      init(&sh.q_full[i], 4, WNW_DEBUG_WAIT_Q_FULL);
      init(&sh.p_ready[i], 4, WNW_DEBUG_WAIT_WEIGHTS);
      init(&sh.k_free[i], 1, WNW_DEBUG_WAIT_K_FREE);
      init(&sh.v_free[i], 1, WNW_DEBUG_WAIT_V_FREE);
      init(&sh.s_full[i], 1, WNW_DEBUG_WAIT_SCORES);
      init(&sh.o_done[i], 1, WNW_DEBUG_WAIT_VALUES);
    }
    init(&sh.begun, 1, WNW_DEBUG_WAIT_BEGUN);
    init(&sh.drained, 1, 0);
    fence_smem();
    sh.status = pv.status;
    sh.clocks = a.wait_clocks;
    sh.dead = 0;
  }
  pg_let_next_start();
  pg_wait_for_stream();
  if (tid == 0) a.part_head[blockIdx.x] = PartHead{};
  const long long total = lay_out(a, sh);              // (its barriers order the above too)
  const long long len_line = (total + gridDim.x - 1) / gridDim.x, x0 = min(total, blockIdx.x * len_line), x1 = min(total, x0 + len_line);
  if (x0 >= x1) return;
  if (wid == 13) {                                     // (the warp that frees it has to be whole: 12 may have lost the thread of the products)
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  Walk w;
  walk_begin(a, sh, x0, x1 - x0, w);

  if (wid < 8) {
    // ---- softmax of row tile i, thread: row ----
    const int i = wid >> 2, row = tid & 127, tok_in = row / a.g, hd = row - tok_in * a.g;
    const uint32_t lanes = (uint32_t)(wid & 3) << 21, t_s = tmem + lanes + COL_S + 128 * i, t_o = tmem + lanes + COL_O + 128 * i;
    uint32_t n_all = 0, n_mine = 0;                    // tiles of the CTA, and of this row tile, so far
    int n_seg = 0, n_idle = 0;
    for (bool more = true; more; more = walk_on(a, w), ++n_seg) {
      const int n_tiles = w.k1 - w.k0;
      if (i && !two_blocks(a, w)) {
        // Nothing to do; but a segment begins only when the one before it is out, and this warp is never two of them ahead.
        n_all += n_tiles;
        __syncwarp();
        if (lane == 0) arrive(&sh.q_full[1]);
        wait(&sh.begun, n_idle++, sh);
        continue;
      }
      const int first = (w.t * PP_BLOCKS + i) * a.rt, tok = first + tok_in;
      const bool real = tok_in < a.rt && tok < w.n;
      // the row of Q: scaled by a power of two to fp16's range, its largest magnitude in [2^14, 2^15)
      float f_row;
      {
        const unsigned char *p = a.q.p + 2 * ((long long)(w.r0 + tok) * a.q.row + (w.h * a.g + hd) * a.q.head);
        float most = 0.f;
        uint4 x[D / 8];
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          x[k] = real ? reinterpret_cast<const uint4 *>(p)[k] : make_uint4(0, 0, 0, 0);
          const uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const float2 y = a.dtype == WNW_DTYPE_BF16 ? Pair<__nv_bfloat16>::get(u[z]) : Pair<__half>::get(u[z]);
            most = fmaxf(most, fmaxf(fabsf(y.x), fabsf(y.y)));
          }
        }
        const int eq = most > 0.f && most < INFINITY ? max(-100, (int)(__float_as_uint(most) >> 23) - 127 - 14) : 0;
        const float down = __uint_as_float((uint32_t)(127 - eq) << 23);
        f_row = a.scale_log2 * __uint_as_float((uint32_t)(eq + 127) << 23);
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const float2 y = a.dtype == WNW_DTYPE_BF16 ? Pair<__nv_bfloat16>::get(u[z]) : Pair<__half>::get(u[z]);
            u[z] = half2_of(y.x * down, y.y * down);
          }
          *reinterpret_cast<uint4 *>(q_s + i * TILE + (k >> 3) * HALF + row * 128 + (((k & 7) ^ (row & 7)) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
        }
      }
      fence_smem();
      __syncwarp();
      if (lane == 0) arrive(&sh.q_full[i]);

      const int end_first = a.causal ? w.len - w.n + first + 1 : w.len;                  // of the row tile's first query token
      const int end = real ? min(w.len, a.causal ? w.len - w.n + tok + 1 : w.len) : w.len;
      float m = NOTHING, big_m = NOTHING, l = 0.f;
      for (int kt = w.k0; kt < w.k1; ++kt, ++n_all, ++n_mine) {
        wait(&sh.s_full[i], n_mine, sh);
        fence_after();
        const float2 *scale = sh.scale[n_all & 3];
        const uint32_t flags = sh.flags[n_all & 3];
        const int seen = end - kt * PP_TOKENS;         // of the tile's tokens
        const bool masked = (flags & TILE_HOLES) || (kt + 1) * PP_TOKENS > end_first;
        uint32_t x[2][32];
        float top, big;
        tmem_load(t_s, x[0]);
        if (masked) row_top<true>(t_s, x, scale, false, f_row, seen, top, big);
        else row_top<false>(t_s, x, scale, flags & TILE_EVEN, f_row, seen, top, big);
        if (__any_sync(0xffffffffu, top > m + LAZY || big > big_m + LAZY)) {
          const float mn = fmaxf(m, top), bn = fmaxf(big_m, big), by = ex2(big_m - bn);
          l *= ex2(m - mn);
          m = mn;
          big_m = bn;
          if (kt > w.k0) {
            wait(&sh.o_done[i], (n_mine - 1) & a.values_parity, sh);
            fence_after();
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              uint32_t o[16];
              tmem_load(t_o + 16 * k, o);
              tmem_loaded(o);
#pragma unroll
              for (int z = 0; z < 16; ++z) o[z] = __float_as_uint(__uint_as_float(o[z]) * by);
              tmem_store(t_o + 16 * k, o);
            }
          }
        }
        bool deep = false;
        if (!(flags & TILE_EVEN) || masked) {
#pragma unroll
          for (int g = 0; g < 8; ++g) deep = deep || (scale[g].y != -INFINITY && big_m - scale[g].y - m > 60.f);
        } else {
          deep = big_m - scale[0].y - m > 60.f;
        }
        if (__any_sync(0xffffffffu, deep)) row_weights<true, true>(t_s, x, scale, f_row, masked ? seen : PP_TOKENS, m, big_m, l);
        else if (masked) row_weights<true, false>(t_s, x, scale, f_row, seen, m, big_m, l);
        else row_weights<false, false>(t_s, x, scale, f_row, seen, m, big_m, l);
        tmem_stored();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(&sh.p_ready[i]);
      }

      // ---- out ----
      wait(&sh.o_done[i], (n_mine - 1) & a.values_parity, sh);
      if (*(volatile uint32_t *)&sh.dead) l = NAN;     // incomplete, and looks it (read last: this wait, too, or another warp's may have run out)
      fence_after();
      const bool whole = w.k0 == 0 && w.k1 == w.need;
      const int slot = w.k0 ? 0 : 1;
      const float by = whole ? (l == 0.f ? 0.f : ex2(big_m - m) / l) : 1.f;              // (no token: zeros)
      const long long at = ((long long)blockIdx.x * 2 + slot) * (PP_BLOCKS * PP_ROWS) + i * PP_ROWS + row;
      const int head = w.h * a.g + hd;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        uint32_t o[32];
        tmem_load(t_o + 32 * k, o);
        tmem_loaded(o);
        if (FMT == WNW_PAGES_E4M3) {
          for (int y = 0; y < 4; ++y)
            if (sh.nan_any[n_seg & 3][y]) {
#pragma unroll
              for (int z = 0; z < 32; ++z)
                if (end > sh.nan_first[n_seg & 3][y][32 * k + z]) o[z] = 0x7fc00000u;
            }
        }
        if (!real) continue;
        if (whole) {
          uint4 *p = reinterpret_cast<uint4 *>(a.out.p + 2 * ((long long)(w.r0 + tok) * a.out.row + head * a.out.head + 32 * k));
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            uint32_t u[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const float f = __uint_as_float(o[8 * z + 2 * y]) * by, g = __uint_as_float(o[8 * z + 2 * y + 1]) * by;
              u[y] = a.dtype == WNW_DTYPE_BF16 ? Pair<__nv_bfloat16>::put(f, g) : Pair<__half>::put(f, g);
            }
            p[z] = make_uint4(u[0], u[1], u[2], u[3]);
          }
        } else {
          uint4 *p = reinterpret_cast<uint4 *>(a.part_o + at * D + 32 * k);
#pragma unroll
          for (int z = 0; z < 8; ++z) p[z] = make_uint4(o[4 * z], o[4 * z + 1], o[4 * z + 2], o[4 * z + 3]);
        }
      }
      if (real && whole && a.lse) a.lse[(long long)(w.r0 + tok) * a.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
      if (real && !whole) a.part_row[at] = PartRow{m, big_m, l, 0.f};
      if (tid == 0 && !whole && slot) {
        // the CTAs that this item runs over: it begins `before` tiles into this stretch
        const long long before = x1 - x0 - w.left;
        a.part_head[blockIdx.x] = PartHead{w.r0, w.n, w.h, w.t, (int)((before + w.need - 1) / len_line + 1), {}};
      }
    }
  } else if (wid < 12) {
    // ---- codes to fp16 ----
    const int wq = wid - 8, ch = lane & 3;
    const int half = D == 128 ? lane >> 3 & 1 : 0;
    const int row_in = D == 128 ? wq * 4 + (lane >> 4) * 2 + (lane >> 2 & 1) : (wq & 1) * 8 + (lane >> 2);   // of the granule
    using Tile = Codes<D>;
    const int gpp = pv.T / PG_GR;
    Walk nx = w;                                       // the tile whose codes are asked for next
    int nx_kt = nx.k0;
    bool nx_more = true;
    int page = -1, page_row = 0;                       // lanes 0-7: of that tile's granules
    auto look_up = [&]() {
      page = -1;
      if (nx_more && lane < 8) {
        const int g = nx_kt * 8 + lane;
        if (g * PG_GR < nx.len) {
          page = a.bv.table[(long long)nx.s * a.bv.stride + g / gpp];
          page_row = g % gpp * PG_GR;
          if (page < 0 || page >= pv.n_pages) {
            if (wq == 0) pg_report(pv, WNW_PAGES_BAD_PAGE);
            page = -1;
          }
        }
      }
    };
    Tile c;
    long long off[8];
    auto ask_meta = [&]() {                            // the scales of the tile that is asked for, and where its granules are
      c.meta = 0;
      long long o = -1;
      if (page >= 0) {
        const float *sc = pv.scales + page * pv.scale_stride + nx.h * 2;
        c.meta = (__float_as_uint(sc[0]) >> 23 & 255) | (__float_as_uint(sc[1]) >> 23 & 255) << 8 | 1u << 16;
        o = page * pv.page_stride + ((long long)nx.h * 2 * pv.T + page_row) * D;
      }
#pragma unroll
      for (int g = 0; g < 8; ++g) off[g] = __shfl_sync(0xffffffffu, o, g);
    };
    auto ask = [&](uint4 (&x)[Tile::PASSES], long long which) {
#pragma unroll
      for (int p = 0; p < Tile::PASSES; ++p) {
        const int g = D == 128 ? p : p * 2 + (wq >> 1);
        long long o = off[0];
#pragma unroll
        for (int k = 1; k < 8; ++k)
          if (D == 128 ? k == p : k == g) o = off[k];
        const bool there = o >= 0 && nx_kt * PP_TOKENS + g * PG_GR + row_in < nx.len;
        x[p] = there ? *reinterpret_cast<const uint4 *>(pv.codes + o + which + row_in * D + half * 64 + ch * 16) : make_uint4(0, 0, 0, 0);
      }
    };
    auto next = [&]() {
      if (nx_more && ++nx_kt == nx.k1) {
        nx_more = walk_on(a, nx);
        nx_kt = nx.k0;
      }
    };
    const long long v_off = (long long)pv.T * D;
    look_up();
    ask_meta();
    ask(c.k, 0);
    ask(c.v, v_off);
    next();
    look_up();
    uint32_t n = 0;
    int n_seg = 0;
    for (bool more = true; more; more = walk_on(a, w), ++n_seg) {
      for (int kt = w.k0; kt < w.k1; ++kt, ++n) {
        const int st = n & 1;
        // scales: four tiles deep, so that the slower row tile's softmax has read them before they are overwritten
        const uint32_t meta = c.meta;
        const uint32_t meta_0 = __shfl_sync(0xffffffffu, meta, 0);
        const bool even = __all_sync(0xffffffffu, lane >= 8 || meta == meta_0), holes = __any_sync(0xffffffffu, lane < 8 && !meta);
        wait(&sh.k_free[st], (n >> 1) + 1, sh);
        if (wq == 0) {
          if (lane < 8) sh.scale[n & 3][lane] = make_float2(__uint_as_float((meta & 255) << 23), meta ? (float)((int)(meta >> 8 & 255) - 127) : -INFINITY);
          if (lane == 0) sh.flags[n & 3] = (even ? TILE_EVEN : 0) | (holes ? TILE_HOLES : 0);
        }
        unsigned char *to = k_s + st * TILE + half * HALF;
        auto put = [&](unsigned char *tile, uint4 codes, int p) {
          const int r = D == 128 ? p * 16 + row_in : p * 32 + (wq >> 1) * 16 + row_in;
          uint4 lo, hi;
          sixteen<FMT>(codes, lo, hi);
          *reinterpret_cast<uint4 *>(tile + r * 128 + ((2 * ch ^ (r & 7)) << 4)) = lo;
          *reinterpret_cast<uint4 *>(tile + r * 128 + (((2 * ch + 1) ^ (r & 7)) << 4)) = hi;
        };
#pragma unroll
        for (int p = 0; p < Tile::PASSES; ++p) put(to, c.k[p], p);
        fence_smem();
        __syncwarp();
        if (lane == 0) arrive(&sh.k_full[st]);
        ask_meta();                                    // (of the next tile: page ids were asked for a tile ago)
        ask(c.k, 0);
        wait(&sh.v_free[st], (n >> 1) + 1, sh);
        if (FMT == WNW_PAGES_E4M3) {                   // 0x7f and 0xff
          uint32_t any = 0;
#pragma unroll
          for (int p = 0; p < Tile::PASSES; ++p)
            any |= ((c.v[p].x & 0x7f7f7f7fu) + 0x01010101u) | ((c.v[p].y & 0x7f7f7f7fu) + 0x01010101u) | ((c.v[p].z & 0x7f7f7f7fu) + 0x01010101u) | ((c.v[p].w & 0x7f7f7f7fu) + 0x01010101u);
          int *nan_any = &sh.nan_any[n_seg & 3][wq], *nan_first = sh.nan_first[n_seg & 3][wq];
          if (kt == w.k0) {
            if (lane == 0) *nan_any = 0;
            __syncwarp();
          }
          if (__any_sync(0xffffffffu, any & 0x80808080u)) {
            const bool begun = *nan_any;
            __syncwarp();
            if (!begun) {
              for (int z = lane; z < 128; z += 32) nan_first[z] = 0x7fffffff;
              if (lane == 0) *nan_any = 1;
              __syncwarp();
            }
#pragma unroll
            for (int p = 0; p < Tile::PASSES; ++p) {
              uint32_t u[4] = {c.v[p].x, c.v[p].y, c.v[p].z, c.v[p].w};
              const int token = kt * PP_TOKENS + (D == 128 ? p * 16 : p * 32 + (wq >> 1) * 16) + row_in;
#pragma unroll
              for (int z = 0; z < 16; ++z)
                if ((u[z >> 2] >> 8 * (z & 3) & 0x7f) == 0x7f) {
                  u[z >> 2] &= ~(0xffu << 8 * (z & 3));
                  atomicMin(nan_first + half * 64 + ch * 16 + z, token);
                }
              c.v[p] = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
        }
        to = v_s + st * TILE + half * HALF;
#pragma unroll
        for (int p = 0; p < Tile::PASSES; ++p) put(to, c.v[p], p);
        fence_smem();
        __syncwarp();
        if (lane == 0) arrive(&sh.v_full[st]);
        ask(c.v, v_off);
        next();
        look_up();
      }
    }
  } else {
    if (wid == 12 && lane == 0) {
      // ---- products ----
      uint32_t n = 0, n_seg = 0, n_of[2] = {0, 0};
      const uint32_t q_u = smem_u32(q_s), k_u = smem_u32(k_s), v_u = smem_u32(v_s);
      auto scores = [&](int i, int st) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_ss(tmem + COL_S + 128 * i, operand(q_u + i * TILE + (k >> 2) * HALF + (k & 3) * 32, 16), operand(k_u + st * TILE + (k >> 2) * HALF + (k & 3) * 32, 16),
                 shape(PP_TOKENS, false), k > 0);
        commit(&sh.s_full[i]);
      };
      auto values = [&](int i, int st, bool add) {
#pragma unroll
        for (int k = 0; k < PP_TOKENS / 16; ++k)
          mma_ts(tmem + COL_O + 128 * i, tmem + COL_S + 128 * i + 8 * k, operand(v_u + st * TILE + k * 2048, HALF), shape(D, true), add || k > 0);
        commit(&sh.o_done[i]);
      };
      for (bool more = true; more; more = walk_on(a, w), ++n_seg) {
        const bool two = two_blocks(a, w);
        wait<true>(&sh.k_full[n & 1], n >> 1, sh);
        for (int i = 0; i < 2; ++i) {
          wait<true>(&sh.q_full[i], n_seg, sh);
          fence_after();
          if (i == 0 || two) scores(i, n & 1);
        }
        if (!two) arrive(&sh.begun);
        commit(&sh.k_free[n & 1]);
        for (int kt = w.k0; kt < w.k1; ++kt, ++n) {
          const int st = n & 1;
          const bool again = kt + 1 < w.k1;
          wait<true>(&sh.v_full[st], n >> 1, sh);
          for (int i = 0; i < (two ? 2 : 1); ++i) {
            wait<true>(&sh.p_ready[i], n_of[i]++, sh);
            fence_after();
            values(i, st, kt > w.k0);
            if (again) {
              if (i == 0) wait<true>(&sh.k_full[st ^ 1], (n + 1) >> 1, sh);
              scores(i, st ^ 1);
            }
          }
          commit(&sh.v_free[st]);
          if (again) commit(&sh.k_free[st ^ 1]);
        }
      }
      commit(&sh.drained);
      wait(&sh.drained, 0, sh);
    }
  }
  if (wid != 12) __syncwarp();
  fence_before();
  __syncthreads();
  if (wid == 13) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
  }
}

template <int D, int FMT> cudaError_t launch(const AttendArgs &a, int n_ctas, int device, cudaStream_t st) {
  static std::atomic<unsigned long long> ready{0};       // devices whose kernel has its shared memory
  if (!(ready.load(std::memory_order_acquire) >> device & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(wnw_pages_prompt_kernel<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>());
    if (e != cudaSuccess) return e;
    ready.fetch_or(1ull << device, std::memory_order_release);
  }
  return pg_launch(wnw_pages_prompt_kernel<D, FMT>, dim3(n_ctas), PP_THREADS, smem_bytes<D>(), st, 0, a);
}

}  // namespace

cudaError_t launch_prompt(const AttendArgs &a, int head_dim, int format, int n_ctas, int device, cudaStream_t st) {
  if (head_dim == 64) return format == WNW_PAGES_E4M3 ? launch<64, WNW_PAGES_E4M3>(a, n_ctas, device, st) : launch<64, WNW_PAGES_INT8>(a, n_ctas, device, st);
  return format == WNW_PAGES_E4M3 ? launch<128, WNW_PAGES_E4M3>(a, n_ctas, device, st) : launch<128, WNW_PAGES_INT8>(a, n_ctas, device, st);
}

}  // namespace wnw
