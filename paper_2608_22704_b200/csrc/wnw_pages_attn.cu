// wnw_pages_attend: attention of a ragged batch of query rows over the paged eight-bit store.
//
//   s = (q . code_k) * 2^eK * scale,   p = softmax of s over the tokens that the row sees,   out = sum p * code_v * 2^eV
//
// What bounds it with few query rows: reading the codes, one byte an element.  So the schedule is even in bytes: the granules (16
// tokens of a KV head) of all sequences lie on one line, every CTA takes an equal stretch of it, found on the device from the lengths,
// and a head's stretches meet again in wnw_pages_join_kernel.  Within a CTA the granules go round the warps, each with a softmax of its
// own, which meet in shared memory where a head ends.
//
// A warp multiplies tokens x head_dim by head_dim x query rows (S^T = K Q^T, O^T = V^T P^T; mma.sync m16n8k16), so that a group of up
// to eight query rows fills an operand.  The order of the contracted index is free as long as both operands agree, so every lane keeps
// to 16 bytes of a row at a time.  A granule comes as one TMA copy (K and V rows, swizzled so that no bank conflicts arise) into the
// warp's own ring in shared memory.  (Copies of 16 bytes a lane, cp.async, moved 5.0 TB/s however many warps and stages there were;
// these 6.4 then.)  Codes become fp16 exactly (e4m3 has 4 significant bits, int8 8); the query is scaled by a power of two to the top of
// fp16's range (elements below 2^-31 of its largest lose bits, below 2^-39 they are zero); weights are fp16 against a reference within 2^8
// of the largest.  Sums, maxima and accumulators are fp32.
//
// The scales 2^eV sit inside the sum over tokens.  A second reference M, the maximum of s + eV in log2, carries them: weights enter the
// product as 2^(s + eV - M), the denominator as 2^(s - m), and out = product * 2^(M - m) / denominator.  No spread of scales over the
// pages can push the weights that matter out of fp16's range.
//
// 16 sequences of 50001 tokens, 8 KV heads of 128, e4m3: 245 to 282 us from box to box, 5.8 to 6.7 TB/s (the measured copy rate is 6.5).  Some 10 us
// of a call on the line go into laying it out, its first copies, and the join; 32 sequences of up to 7500 tokens, 332 MB, take 74 us in int8, 70 in e4m3.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cstring>

#include "wnw_pages_attn.cuh"

namespace wnw {
namespace {

constexpr int PA_ROWS = 16;          // query rows of an item at most
constexpr int PA_SEGS = 64;          // stretches of heads that a CTA prepares at a time

// A head's stretch inside a CTA.
struct Seg {
  int s, h, tile;                    // sequence, KV head, tile of query tokens
  int g0, n, y0;                     // first granule, granules, place of the first on the CTA's line
  int need;                          // granules from the head's first on that some row sees
  int len, row0, nq;                 // tokens of the sequence; first query row and query tokens of the tile
  int r0, n_seq;                     // first query row and query tokens of the sequence
  int end0;                          // tokens that the tile's first query row sees; the next rows see one more each if causal
  int slot, n_parts;                 // slot -1: the whole head; else where the partial result goes
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float4 peer(uint32_t at, uint32_t rank) {   // 16 bytes of another CTA of the cluster
  uint32_t there;
  float4 x;
  asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(there) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];\n" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(there));
  return x;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // an 8 x 8 matrix of 16-bit elements over the warp
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(x));
  return r;
}
// One granule of a KV head: 16 K rows, then 16 V rows (see encode_map).
__device__ __forceinline__ void copy_granule(uint32_t dst, const CUtensorMap *map, int row, int block, int page, uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
  asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];\n"
               ::"r"(dst), "l"(map), "r"(bar), "r"(0), "r"(row), "r"(block), "r"(page) : "memory");
}
// Bounded: gives up after about a second of SM clocks and says so, instead of hanging.
__device__ __forceinline__ bool wait_granule(uint32_t bar, uint32_t parity, const AttendArgs &a) {
  if (try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!try_wait(bar, parity))
    if (clock64() - t0 > a.wait_clocks) { pg_report(a.pv, WNW_PAGES_TIMEOUT); return false; }
  return true;
}

// After a copy that did not arrive: those under way, which nothing may disturb, come to rest, for as long again.  (In line it made 3064 tokens of
// 8 heads take 8.45 us instead of 8.15: code that never runs.)
__device__ __noinline__ void come_to_rest(const uint32_t *scales, uint32_t bars, int from, int to, int n, uint32_t phases, uint32_t clocks) {
  do {
    if (scales[from])
      for (const long long t0 = clock64(); !try_wait(bars + 8 * from, phases >> from & 1) && clock64() - t0 <= clocks;) {}
    if (++from == n) from = 0;
  } while (from != to);
}
// W warps of a CTA, S granules of a warp in the ring.
template <int D, int NT> struct Geo {
  static constexpr int W = D == 64 ? (NT == 1 ? 16 : 12) : NT == 1 ? 12 : 8, S = W == 12 && D == 128 ? 3 : 4, THREADS = 32 * W;
  static constexpr int KC = D / 64;                    // 16-byte pieces of a K row that a lane takes
  static constexpr int VB = D / 8;                     // bytes of a V row that a lane takes
  static constexpr int MT = D / 16;                    // 16-row tiles of V^T
  static constexpr int STAGE = 2 * PG_GR * D;          // bytes of a granule in the ring: K, then V
  static constexpr int PITCH = D + 4;                  // floats of a row where the warps' results meet
};
template <int D, int NT> constexpr size_t smem_bytes() {
  using G = Geo<D, NT>;
  return (size_t)G::W * G::S * (G::STAGE + sizeof(uint32_t) + sizeof(uint64_t)) + (G::W + 1) * NT * 8 * (G::PITCH * 4 + sizeof(PartRow)) +
         PA_SEGS * sizeof(Seg) + (PG_MAX_SEQS + 1) * (sizeof(long long) + sizeof(int));
}

// The line: granules and heads (items) of the sequences before each one.  Returns the granules of all.
template <int W>
__device__ __forceinline__ long long lay_out(const AttendArgs &a, long long *grans, int *items) {
  __shared__ long long wsum[W];
  __shared__ long long isum[W];
  const int n = a.bv.n_seqs, tid = threadIdx.x, lane = tid & 31, w = tid >> 5, cap = a.bv.stride * a.pv.T;
  long long gbase = 0, ibase = 0;
  for (int at = 0; at < n; at += 32 * W) {
    const int s = at + tid;
    long long gr = 0, it = 0;
    if (s < n) {
      int r0 = a.bv.starts[s], r1 = a.bv.starts[s + 1], len = a.bv.lengths[s];
      if (r0 < 0 || r1 < r0 || r1 > a.bv.n_rows || len < 0 || len > cap) {
        if (blockIdx.x == 0) pg_report(a.pv, WNW_PAGES_BAD_LENGTH);
        r0 = max(r0, 0); r1 = min(r1, a.bv.n_rows); len = max(0, min(len, cap));
      }
      it = (long long)(r1 > r0 ? (r1 - r0 + a.rt - 1) / a.rt : 0) * a.pv.H;
      gr = it * max(1, (len + PG_GR - 1) / PG_GR);      // (an empty sequence's rows are still to be written)
    }
    long long gi = gr, ii = it;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, gi, o), y = __shfl_up_sync(0xffffffffu, ii, o);
      if (lane >= o) { gi += x; ii += y; }
    }
    if (lane == 31) { wsum[w] = gi; isum[w] = ii; }
    __syncthreads();
    long long gw = gbase, gt = 0, iw = ibase, itot = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if (k < w) { gw += wsum[k]; iw += isum[k]; }
      gt += wsum[k];
      itot += isum[k];
    }
    if (s < n) { grans[s] = gw + gi - gr; items[s] = (int)(iw + ii - it); }
    gbase += gt;
    ibase += itot;
    __syncthreads();
  }
  if (tid == 0) { grans[n] = gbase; items[n] = (int)ibase; }
  __syncthreads();
  if (ibase > 1ll << 30) {             // (row starts that run over one another)
    if (tid == 0 && blockIdx.x == 0) pg_report(a.pv, WNW_PAGES_BAD_LENGTH);
    return 0;
  }
  return gbase;
}
// Granules that a CTA takes: equal stretches, none shorter than a granule for each warp or than a head.
template <int W> __device__ __forceinline__ long long stretch(long long total, int n_items, int n_ctas) {
  return max(n_items ? min((long long)W, quotient(total, n_items)) : 1, quotient(total + n_ctas - 1, n_ctas));
}

// CLUSTER: no line; cluster i takes KV head i % H of sequence i / H, its CTAs equal shares of the tokens, and their results meet in the
// cluster's shared memory instead of in the workspace.
template <int D, int FMT, int NT, bool CLUSTER>
__global__ void __launch_bounds__(Geo<D, NT>::THREADS, 1) wnw_pages_attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map) {
  using G = Geo<D, NT>;
  constexpr int W = G::W, S = G::S;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char *ring = smem;
  float *meet = reinterpret_cast<float *>(ring + W * S * G::STAGE);            // [warp][row][PITCH]
  float *mine_o = meet + W * NT * 8 * G::PITCH;                                        // the CTA's own, for its cluster: [row][PITCH]
  PartRow *meet_row = reinterpret_cast<PartRow *>(mine_o + NT * 8 * G::PITCH);         // [warp][row]
  PartRow *mine_row = meet_row + W * NT * 8;
  uint64_t *bars = reinterpret_cast<uint64_t *>(mine_row + NT * 8);                           // [warp][stage]
  long long *grans = reinterpret_cast<long long *>(bars + W * S);
  Seg *segs = reinterpret_cast<Seg *>(grans + PG_MAX_SEQS + 1);
  int *items = reinterpret_cast<int *>(segs + PA_SEGS);
  uint32_t *ring_scale = reinterpret_cast<uint32_t *>(items + PG_MAX_SEQS + 1);               // [warp][stage]

  const PagesView &pv = a.pv;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, c = lane & 3, r = lane >> 2;
  const int gpp = pv.T / PG_GR;
  if (lane == 0) {
    const uint32_t count = a.lose & WNW_DEBUG_WAIT_GRANULE ? 2 : 1;     // (an arrival that nothing makes, where a test asks for copies that do not arrive)
    for (int k = 0; k < S; ++k) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"((uint32_t)__cvta_generic_to_shared(bars + w * S + k)), "r"(count) : "memory");
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    if (pv.n_pages) asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map) : "memory");   // (a store of no pages has no map)
  }
  __syncwarp();
  if (!CLUSTER) pg_let_next_start();
  pg_wait_for_stream();
  long long len_line = 0, x0 = 0, x1 = 0;
  int item0 = 0, n_items = 0;                           // CLUSTER: the tile of query tokens
  uint32_t rank = 0, n_ranks = 1;
  if constexpr (CLUSTER) {
    asm("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;\n" : "=r"(n_ranks));
  } else {
    const long long total = lay_out<W>(a, grans, items);
    n_items = items[a.bv.n_seqs];
    len_line = stretch<W>(total, n_items, gridDim.x);
    x0 = min(total, blockIdx.x * len_line);
    x1 = min(total, x0 + len_line);
    if (tid == 0) a.part_head[blockIdx.x] = PartHead{};
    if (x0 >= x1) return;
    // the first head of the line
    int lo = 0, hi = a.bv.n_seqs;                       // the last sequence that begins at or before x0 and is not empty
    while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (grans[mid] <= x0) lo = mid; else hi = mid; }
    const int n_it = items[lo + 1] - items[lo];
    const long long per = quotient(grans[lo + 1] - grans[lo], n_it);
    item0 = items[lo] + (int)quotient(x0 - grans[lo], per);
  }
  // a lane's 16-byte pieces of K row r and V rows 2c, 2c + 1 (and 8 rows on) in a swizzled granule
  int k_at[G::KC], v_at[2];
#pragma unroll
  for (int k = 0; k < G::KC; ++k) k_at[k] = 16 * (D == 128 ? (c + 4 * k) ^ r : c ^ (r >> 1));
#pragma unroll
  for (int k = 0; k < 2; ++k) v_at[k] = D == 128 ? 16 * (r ^ (2 * c + k)) : 16 * ((r >> 1) ^ c) + 8 * (r & 1);
  const uint32_t ring_u = (uint32_t)__cvta_generic_to_shared(ring) + w * S * G::STAGE, bars_u = (uint32_t)__cvta_generic_to_shared(bars + w * S);
  uint32_t phases = 0;                                  // parity of each stage's next copy
  bool lost = false;                                    // a copy did not arrive: the warp asks for no more, and what it has a part in is not a number

  for (bool more = true; more;) {
    // ---- the next stretches ----
    __syncthreads();
    int n_seg;
    if constexpr (CLUSTER) {
      const int seq = blockIdx.x / n_ranks / pv.H, cap = a.bv.stride * pv.T;
      const int y0 = a.bv.starts[seq], y1 = a.bv.starts[seq + 1], y2 = a.bv.lengths[seq];
      const int r0 = max(y0, 0), n = max(0, min(y1, a.bv.n_rows) - r0), len = max(0, min(y2, cap));
      if (tid == 0 && (y0 < 0 || y1 < y0 || y1 > a.bv.n_rows || y2 < 0 || y2 > cap)) pg_report(pv, WNW_PAGES_BAD_LENGTH);
      const int first = item0 * a.rt;                   // query token of the sequence
      if (first >= n) break;                            // (all CTAs of the cluster alike)
      if (tid == 0) {
        Seg &sg = segs[0];
        sg.s = seq; sg.h = blockIdx.x / n_ranks % pv.H; sg.tile = item0;
        sg.len = len;
        sg.r0 = r0; sg.n_seq = n;
        sg.nq = min(a.rt, n - first);
        sg.row0 = r0 + first;
        sg.end0 = a.causal ? len - n + first + 1 : len;
        const int last = min(len, a.causal ? sg.end0 + sg.nq - 1 : len);
        sg.need = last > 0 ? (last + PG_GR - 1) / PG_GR : 0;
        const int share = (sg.need + n_ranks - 1) / n_ranks;
        sg.g0 = min(sg.need, (int)rank * share);
        sg.n = min(sg.need - sg.g0, share);
        sg.y0 = 0;
        sg.slot = -1;
        sg.n_parts = 1;
      }
      __syncthreads();
      n_seg = 1;
      ++item0;
    } else {
      int mine = 0;
      if (tid < PA_SEGS && item0 + tid < n_items) {
        const int item = item0 + tid;
        int lo = 0, hi = a.bv.n_seqs;
        while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (items[mid] <= item) lo = mid; else hi = mid; }
        const int cap = a.bv.stride * pv.T, r0 = max(a.bv.starts[lo], 0), n = max(0, min(a.bv.starts[lo + 1], a.bv.n_rows) - r0);
        const int len = max(0, min(a.bv.lengths[lo], cap)), tiles = n <= a.rt ? 1 : (n + a.rt - 1) / a.rt, it = item - items[lo];
        const int per = max(1, (len + PG_GR - 1) / PG_GR);
        const long long b = grans[lo] + (long long)it * per, e = b + per;
        if (b < x1) {
          mine = 1;
          Seg &sg = segs[tid];
          const long long f = max(b, x0), l = min(e, x1);
          sg.s = lo; sg.h = tiles == 1 ? it : it / tiles; sg.tile = tiles == 1 ? 0 : it % tiles;
          sg.g0 = (int)(f - b); sg.n = (int)(l - f); sg.y0 = (int)(f - x0);
          sg.len = len;
          sg.r0 = r0; sg.n_seq = n;
          sg.nq = min(a.rt, n - sg.tile * a.rt);
          sg.row0 = r0 + sg.tile * a.rt;
          sg.end0 = a.causal ? len - n + sg.tile * a.rt + 1 : len;
          const int last = min(len, a.causal ? sg.end0 + sg.nq - 1 : len);
          sg.need = last > 0 ? (last + PG_GR - 1) / PG_GR : 0;
          sg.slot = b >= x0 && e <= x1 ? -1 : b < x0 ? 0 : 1;
          sg.n_parts = sg.slot == 1 ? (int)quotient(e - 1 - x0, len_line) + 1 : 0;
        }
      }
      n_seg = __syncthreads_count(mine);
      more = n_seg == PA_SEGS;                          // (a last round of none costs nothing)
      item0 += n_seg;
    }

    // ---- copies run ahead of the products by S - 1 granules, over the stretches' ends ----
    int p_seg = lost ? n_seg : -1, p_g = 0, p_end = 0, p_cnt = 0, p_stage = 0;
    int p_page = 0, p_row = 0;                          // lane i: where the stretch's granule 32 * k + i of this warp is,
    uint32_t p_scale = 0;                               //   exponent fields of its scales, K | V << 8 | 1 << 16 where it is there
    auto fetch = [&]() {
      while (p_seg < n_seg && p_g >= p_end) {
        if (++p_seg < n_seg) {
          const Seg &sg = segs[p_seg];
          p_g = sg.g0 + (w + W - sg.y0 % W) % W;
          p_end = min(sg.g0 + sg.n, sg.need);
          p_cnt = 0;
        }
      }
      if (p_seg < n_seg) {
        const Seg &sg = segs[p_seg];
        const int j = p_cnt & 31;
        if (j == 0) {
          const int g = p_g + W * lane;
          p_scale = 0;
          if (g < p_end) {
            p_page = a.bv.table[(long long)sg.s * a.bv.stride + g / gpp];
            p_row = g % gpp * PG_GR;
            if (p_page >= 0 && p_page < pv.n_pages) {
              const float *sc = pv.scales + p_page * pv.scale_stride + sg.h * 2;
              p_scale = (__float_as_uint(sc[0]) >> 23 & 255) | (__float_as_uint(sc[1]) >> 23 & 255) << 8 | 1u << 16;
            } else {
              pg_report(pv, WNW_PAGES_BAD_PAGE);
            }
          }
        }
        // by the lane that knows the granule; the others' reads of the stage are behind a __syncwarp
        if (lane == j) {
          ring_scale[w * S + p_stage] = p_scale;
          if (p_scale) copy_granule(ring_u + p_stage * G::STAGE, &map, p_row, 2 * sg.h, p_page, bars_u + 8 * p_stage, G::STAGE);
        }
        p_g += W;
        ++p_cnt;
        if (++p_stage == S) p_stage = 0;
      }
    };
    // ---- the query rows: lane (r, c) holds row r of each tile of eight, the head_dim elements of its K bytes; asked for ahead ----
    uint4 raw[NT][G::KC * 2];
    auto ask_rows = [&](int si) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int k = 0; k < G::KC * 2; ++k) raw[t][k] = make_uint4(0, 0, 0, 0);
        if (si < n_seg) {
          const Seg &sg = segs[si];
          const int j = t * 8 + r, tok = j / a.g, hd = j - tok * a.g;
          if (j < a.rt * a.g && tok < sg.nq) {
            const unsigned char *p = a.q.p + 2 * ((long long)(sg.row0 + tok) * a.q.row + (sg.h * a.g + hd) * a.q.head);
#pragma unroll
            for (int k = 0; k < G::KC; ++k) {
              raw[t][2 * k] = *reinterpret_cast<const uint4 *>(p + 2 * (64 * k + 16 * c));
              raw[t][2 * k + 1] = *reinterpret_cast<const uint4 *>(p + 2 * (64 * k + 16 * c) + 16);
            }
          }
        }
      }
    };
    ask_rows(0);
#pragma unroll
    for (int k = 0; k < S - 1; ++k) fetch();

    int stage = 0;
    for (int si = 0; si < n_seg; ++si) {
      const Seg sg = segs[si];
      uint32_t qf[NT][G::KC * 8];
      float f_col[NT][2];                               // log2 scale of the scores' two columns 2c, 2c + 1
      int end_col[NT][2];                               // tokens that those rows see
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float most = 0.f;
        float2 x[G::KC * 8];
#pragma unroll
        for (int k = 0; k < G::KC * 2; ++k) {
          const uint32_t u[4] = {raw[t][k].x, raw[t][k].y, raw[t][k].z, raw[t][k].w};
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            x[4 * k + z] = a.dtype == WNW_DTYPE_BF16 ? Pair<__nv_bfloat16>::get(u[z]) : Pair<__half>::get(u[z]);
            most = fmaxf(most, fmaxf(fabsf(x[4 * k + z].x), fabsf(x[4 * k + z].y)));
          }
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        // largest magnitude into [2^14, 2^15); rows of zeros and with infinities as they are
        const int eq = most > 0.f && most < INFINITY ? max(-100, (int)(__float_as_uint(most) >> 23) - 127 - 14) : 0;
        const float down = __uint_as_float((uint32_t)(127 - eq) << 23);
#pragma unroll
        for (int k = 0; k < G::KC * 8; ++k) qf[t][k] = half2_of(x[k].x * down, x[k].y * down);
        const float up = a.scale_log2 * __uint_as_float((uint32_t)(eq + 127) << 23);
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          f_col[t][z] = __shfl_sync(0xffffffffu, up, (2 * c + z) * 4);
          const int jc = t * 8 + 2 * c + z;
          end_col[t][z] = a.causal ? min(sg.len, sg.end0 + jc / a.g) : sg.len;
        }
      }
      const int end_min = a.causal ? sg.end0 : sg.len;   // up to here every row of the tile sees every token

      float o[NT][G::MT][4], m[NT][2], big_m[NT][2], l[NT][2], carry[NT][2];   // carry: 2^(m + e_last - M)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < G::MT; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
        m[t][0] = m[t][1] = big_m[t][0] = big_m[t][1] = NOTHING;
        l[t][0] = l[t][1] = 0.f;
        carry[t][0] = carry[t][1] = 1.f;
      }
      float e_last = 0.f;

      const int g_end = min(sg.g0 + sg.n, sg.need);
      for (int g = sg.g0 + (w + W - sg.y0 % W) % W; g < g_end && !lost; g += W) {
        __syncwarp();
        fetch();
        __syncwarp();
        const uint32_t sc = ring_scale[w * S + stage];
        const unsigned char *src = ring + (w * S + stage) * G::STAGE;
        if (sc) {
          if (__any_sync(0xffffffffu, !wait_granule(bars_u + 8 * stage, phases >> stage & 1, a))) {
            come_to_rest(ring_scale + w * S, bars_u, stage, p_stage, S, phases, a.wait_clocks);
            p_seg = n_seg;
            lost = true;
            break;
          }
          phases ^= 1u << stage;
        }
        if (++stage == S) stage = 0;
        const bool there = sc != 0;                      // a page that is not there: nothing of it is seen
        const float k_scale = __uint_as_float((sc & 255) << 23);
        // S^T: tokens r, r + 8 x columns 2c, 2c + 1
        float s[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
        for (int k = 0; k < G::KC; ++k) {
          const unsigned char *p = src + r * D + k_at[k];
          const uint4 u = *reinterpret_cast<const uint4 *>(p), v = *reinterpret_cast<const uint4 *>(p + 8 * D);
          const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            uint32_t a0, a1, a2, a3;
            to_half<FMT>(uw[z], a0, a2);
            to_half<FMT>(vw[z], a1, a3);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma(s[t], a0, a1, a2, a3, qf[t][8 * k + 2 * z], qf[t][8 * k + 2 * z + 1]);
          }
        }
        const int tok = g * PG_GR + r;
        const bool partly = !there || (g + 1) * PG_GR > end_min;
        const float e_v = (float)((int)(sc >> 8 & 255) - 127);
        uint32_t pb[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float f0 = f_col[t][0] * k_scale, f1 = f_col[t][1] * k_scale;
          s[t][0] *= f0; s[t][1] *= f1; s[t][2] *= f0; s[t][3] *= f1;
          if (partly) {
            if (!there || tok >= end_col[t][0]) s[t][0] = -INFINITY;
            if (!there || tok >= end_col[t][1]) s[t][1] = -INFINITY;
            if (!there || tok + 8 >= end_col[t][0]) s[t][2] = -INFINITY;
            if (!there || tok + 8 >= end_col[t][1]) s[t][3] = -INFINITY;
          }
          float top0 = fmaxf(s[t][0], s[t][2]), top1 = fmaxf(s[t][1], s[t][3]);
          const bool far = top0 > fminf(m[t][0], big_m[t][0] - e_v) + LAZY || top1 > fminf(m[t][1], big_m[t][1] - e_v) + LAZY;
          const bool moved = __any_sync(0xffffffffu, far);
          if (moved) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
              top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, x));
              top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, x));
            }
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const float top = z ? top1 : top0, mn = fmaxf(m[t][z], top), bn = fmaxf(big_m[t][z], top + e_v), by = ex2(big_m[t][z] - bn);
              l[t][z] *= ex2(m[t][z] - mn);
#pragma unroll
              for (int i = 0; i < G::MT; ++i) { o[t][i][z] *= by; o[t][i][2 + z] *= by; }
              m[t][z] = mn;
              big_m[t][z] = bn;
            }
          }
          if (moved || e_v != e_last) {                  // (finite: where scales are that far apart, p is zero)
            carry[t][0] = ex2(fminf(m[t][0] + e_v - big_m[t][0], 126.f));
            carry[t][1] = ex2(fminf(m[t][1] + e_v - big_m[t][1], 126.f));
          }
          const float p0 = ex2(s[t][0] - m[t][0]), p1 = ex2(s[t][1] - m[t][1]), p2 = ex2(s[t][2] - m[t][0]), p3 = ex2(s[t][3] - m[t][1]);
          l[t][0] += p0 + p2;
          l[t][1] += p1 + p3;
          pb[t][0] = transposed(half2_of(p0 * carry[t][0], p1 * carry[t][1]));
          pb[t][1] = transposed(half2_of(p2 * carry[t][0], p3 * carry[t][1]));
        }
        e_last = e_v;
        // O^T: elements VB * r + 2i (c0, c1) and VB * r + 2i + 1 (c2, c3) of the columns 2c, 2c + 1
        uint32_t vw[4][G::VB / 4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const unsigned char *p = src + PG_GR * D + (2 * c + (t & 1) + 8 * (t >> 1)) * D + v_at[t & 1];
          if constexpr (G::VB == 16) { const uint4 u = *reinterpret_cast<const uint4 *>(p); vw[t][0] = u.x; vw[t][1] = u.y; vw[t][2] = u.z; vw[t][3] = u.w; }
          else { const uint2 u = *reinterpret_cast<const uint2 *>(p); vw[t][0] = u.x; vw[t][1] = u.y; }
        }
        if (partly) {                                    // rows behind the last token hold anything
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (!there || g * PG_GR + 2 * c + (t & 1) + 8 * (t >> 1) >= sg.len)
#pragma unroll
              for (int z = 0; z < G::VB / 4; ++z) vw[t][z] = 0;
        }
        bool nan_codes = false;                          // in a granule that some rows see only part of: a tile of one row too, before the sequence's others
        if (FMT == WNW_PAGES_E4M3 && partly && end_min < sg.len) {
          bool mine = false;
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int z = 0; z < G::VB / 4; ++z) mine |= __vcmpeq4(vw[t][z] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
          nan_codes = __any_sync(0xffffffffu, mine);
        }
        if (!nan_codes) {
#pragma unroll
          for (int z = 0; z < G::VB / 4; ++z) {
            uint32_t x0, x1, x2, x3, y0, y1, y2, y3;
            to_half<FMT>(__byte_perm(vw[0][z], vw[1][z], 0x5140), x0, x1);
            to_half<FMT>(__byte_perm(vw[2][z], vw[3][z], 0x5140), x2, x3);
            to_half<FMT>(__byte_perm(vw[0][z], vw[1][z], 0x7362), y0, y1);
            to_half<FMT>(__byte_perm(vw[2][z], vw[3][z], 0x7362), y2, y3);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              mma(o[t][2 * z], x0, x1, x2, x3, pb[t][0], pb[t][1]);
              mma(o[t][2 * z + 1], y0, y1, y2, y3, pb[t][0], pb[t][1]);
            }
          }
        } else {
          // a weight of zero does not keep a not-a-number out: they are taken out of the product, and counted for the rows that see them
#pragma unroll
          for (int z = 0; z < G::VB / 4; ++z) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t x[4], bad[4];
              to_half<FMT>(__byte_perm(vw[0][z], vw[1][z], half ? 0x7362 : 0x5140), x[0], x[1]);
              to_half<FMT>(__byte_perm(vw[2][z], vw[3][z], half ? 0x7362 : 0x5140), x[2], x[3]);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const __half2 h = *reinterpret_cast<const __half2 *>(&x[k]);
                const bool b0 = __hisnan(__low2half(h)), b1 = __hisnan(__high2half(h));
                bad[k] = (b0 ? 0x3c00u : 0u) | (b1 ? 0x3c000000u : 0u);
                x[k] &= (b0 ? 0u : 0xffffu) | (b1 ? 0u : 0xffff0000u);
              }
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                const int end = min(sg.len, sg.end0 + (t * 8 + r) / a.g), t0 = g * PG_GR + 2 * c;    // of column r: the lane's part of P^T
                const uint32_t see0 = (t0 < end ? 0x3c00u : 0u) | (t0 + 1 < end ? 0x3c000000u : 0u);
                const uint32_t see1 = (t0 + 8 < end ? 0x3c00u : 0u) | (t0 + 9 < end ? 0x3c000000u : 0u);
                float n[4] = {0.f, 0.f, 0.f, 0.f};
                mma(o[t][2 * z + half], x[0], x[1], x[2], x[3], pb[t][0], pb[t][1]);
                mma(n, bad[0], bad[1], bad[2], bad[3], see0, see1);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (n[k] > 0.f) o[t][2 * z + half][k] = NAN;
              }
            }
          }
        }
      }

      // ---- the warps' results meet ----
      ask_rows(si + 1);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          if (lost) l[t][z] = NAN;                       // incomplete, and looks it
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) l[t][z] += __shfl_xor_sync(0xffffffffu, l[t][z], x);
          float *p = meet + ((w * NT + t) * 8 + 2 * c + z) * G::PITCH + G::VB * r;
#pragma unroll
          for (int i = 0; i < G::MT; i += 2) *reinterpret_cast<float4 *>(p + 2 * i) = make_float4(o[t][i][z], o[t][i][2 + z], o[t][i + 1][z], o[t][i + 1][2 + z]);
          if (r == 0) meet_row[(w * NT + t) * 8 + 2 * c + z] = PartRow{m[t][z], big_m[t][z], l[t][z], 0.f};
        }
      __syncthreads();
      for (int i = tid; i < NT * 8 * (D / 4); i += G::THREADS) {
        const int j = i / (D / 4), d = i % (D / 4) * 4, tok = j / a.g, hd = j - tok * a.g;
        if (j < a.rt * a.g && tok < sg.nq) {
          float mx = NOTHING, bx = NOTHING, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int k = 0; k < W; ++k) {
            mx = fmaxf(mx, meet_row[k * NT * 8 + j].m);
            bx = fmaxf(bx, meet_row[k * NT * 8 + j].big_m);
          }
#pragma unroll
          for (int k = 0; k < W; ++k) {
            const PartRow pr = meet_row[k * NT * 8 + j];
            const float4 x = *reinterpret_cast<const float4 *>(meet + (k * NT * 8 + j) * G::PITCH + d);
            const float by = ex2(pr.big_m - bx);
            sum += pr.l * ex2(pr.m - mx);
            acc.x += x.x * by; acc.y += x.y * by; acc.z += x.z * by; acc.w += x.w * by;
          }
          if (CLUSTER) {
            *reinterpret_cast<float4 *>(mine_o + j * G::PITCH + d) = acc;
            if (d == 0) mine_row[j] = PartRow{mx, bx, sum, 0.f};
          } else if (sg.slot < 0) {
            const float by = sum == 0.f ? 0.f : ex2(bx - mx) / sum;      // (no token: zeros)
            const long long row = sg.row0 + tok;
            const int head = sg.h * a.g + hd;
            unsigned char *p = a.out.p + 2 * (row * a.out.row + head * a.out.head + d);
            uint2 v;
            if (a.dtype == WNW_DTYPE_BF16) v = make_uint2(Pair<__nv_bfloat16>::put(acc.x * by, acc.y * by), Pair<__nv_bfloat16>::put(acc.z * by, acc.w * by));
            else v = make_uint2(Pair<__half>::put(acc.x * by, acc.y * by), Pair<__half>::put(acc.z * by, acc.w * by));
            *reinterpret_cast<uint2 *>(p) = v;
            if (a.lse && d == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + log2f(sum)) * 0.69314718055994531f;
          } else {
            const long long at = ((long long)blockIdx.x * 2 + sg.slot) * PA_ROWS + j;
            *reinterpret_cast<float4 *>(a.part_o + at * D + d) = acc;
            if (d == 0) a.part_row[at] = PartRow{mx, bx, sum, 0.f};
          }
        }
      }
      if constexpr (CLUSTER) {                          // the CTAs' results meet: each puts together its share of the output
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        const int used = sg.nq * a.g * (D / 4);         // (rows of real query tokens come first)
        for (int i = rank * G::THREADS + tid; i < used; i += n_ranks * G::THREADS) {
          const int j = i / (D / 4), d = i % (D / 4) * 4, tok = j / a.g, head = sg.h * a.g + j - tok * a.g;
          const uint32_t o_at = (uint32_t)__cvta_generic_to_shared(mine_o + j * G::PITCH + d), r_at = (uint32_t)__cvta_generic_to_shared(mine_row + j);
          float mx = NOTHING, bx = NOTHING, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (uint32_t k = 0; k < n_ranks; ++k) {
            const float4 pr = peer(r_at, k);
            mx = fmaxf(mx, pr.x);
            bx = fmaxf(bx, pr.y);
          }
          for (uint32_t k = 0; k < n_ranks; ++k) {
            const float4 pr = peer(r_at, k), x = peer(o_at, k);
            const float by = ex2(pr.y - bx);
            sum += pr.z * ex2(pr.x - mx);
            acc.x += x.x * by; acc.y += x.y * by; acc.z += x.z * by; acc.w += x.w * by;
          }
          const float by = sum == 0.f ? 0.f : ex2(bx - mx) / sum;      // (no token: zeros)
          const long long row = sg.row0 + tok;
          unsigned char *p = a.out.p + 2 * (row * a.out.row + head * a.out.head + d);
          if (a.dtype == WNW_DTYPE_BF16) *reinterpret_cast<uint2 *>(p) = make_uint2(Pair<__nv_bfloat16>::put(acc.x * by, acc.y * by), Pair<__nv_bfloat16>::put(acc.z * by, acc.w * by));
          else *reinterpret_cast<uint2 *>(p) = make_uint2(Pair<__half>::put(acc.x * by, acc.y * by), Pair<__half>::put(acc.z * by, acc.w * by));
          if (a.lse && d == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + log2f(sum)) * 0.69314718055994531f;
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");   // read by all, free again
      }
      if (!CLUSTER && tid == 0 && sg.slot == 1) a.part_head[blockIdx.x] = PartHead{sg.r0, sg.n_seq, sg.h, sg.tile, sg.n_parts, {}};
      __syncthreads();
    }
  }
}

// A head that several CTAs share: CTA (b, y) puts rows of the head together that begins in CTA b of the attention and does not end there.
// Up to FEW partial results are read by every thread for itself, a row by D / 4 of them; more are dealt out over the CTA's threads, which
// then take a row together.
template <int D>
__global__ void __launch_bounds__(128) wnw_pages_join_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int LANES = D / 4, SPLIT = 128 / LANES, FEW = 8;
  __shared__ float4 acc_s[SPLIT][LANES];
  __shared__ float sum_s[SPLIT], red[2][4];
  pg_wait_for_stream();
  const PartHead ph = a.part_head[blockIdx.x];
  if (ph.n_parts < 2) return;
  const int used = a.rt * a.g, all = a.blocks * used, part = threadIdx.x / LANES, d = threadIdx.x % LANES;
  // Row y of the head: its place in the partial results, its row of the batch and query head; false: no such token
  auto place = [&](int y, int *j, long long *row, int *head) {
    const int i = y / used, jj = y - i * used, tok = (ph.tile * a.blocks + i) * a.rt + jj / a.g;
    *j = i * a.rb + jj;
    *row = ph.r0 + tok;
    *head = ph.h * a.g + jj % a.g;
    return tok < ph.n;
  };
  auto at = [&](int k, int j) { return ((long long)(blockIdx.x + k) * 2 + (k == 0)) * (a.blocks * a.rb) + j; };
  auto put = [&](float4 acc, float sum, float mx, float bx, long long row, int head) {
    const float by = sum == 0.f ? 0.f : ex2(bx - mx) / sum;        // (no token: zeros)
    unsigned char *p = a.out.p + 2 * (row * a.out.row + head * a.out.head + 4 * d);
    if (a.dtype == WNW_DTYPE_BF16) *reinterpret_cast<uint2 *>(p) = make_uint2(Pair<__nv_bfloat16>::put(acc.x * by, acc.y * by), Pair<__nv_bfloat16>::put(acc.z * by, acc.w * by));
    else *reinterpret_cast<uint2 *>(p) = make_uint2(Pair<__half>::put(acc.x * by, acc.y * by), Pair<__half>::put(acc.z * by, acc.w * by));
    if (a.lse && d == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + log2f(sum)) * 0.69314718055994531f;
  };
  int j, head;
  long long row;
  if (ph.n_parts <= FEW) {
    for (int y = blockIdx.y * SPLIT + part; y < all; y += gridDim.y * SPLIT) {
      if (!place(y, &j, &row, &head)) continue;
      float4 xs[FEW];
      PartRow rows[FEW];
#pragma unroll
      for (int k = 0; k < FEW; ++k)
        if (k < ph.n_parts) {
          rows[k] = a.part_row[at(k, j)];
          xs[k] = *reinterpret_cast<const float4 *>(a.part_o + at(k, j) * D + 4 * d);
        }
      float mx = NOTHING, bx = NOTHING, sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < FEW; ++k)
        if (k < ph.n_parts) { mx = fmaxf(mx, rows[k].m); bx = fmaxf(bx, rows[k].big_m); }
#pragma unroll
      for (int k = 0; k < FEW; ++k)
        if (k < ph.n_parts) {
          const float by = ex2(rows[k].big_m - bx);
          sum += rows[k].l * ex2(rows[k].m - mx);
          acc.x += xs[k].x * by; acc.y += xs[k].y * by; acc.z += xs[k].z * by; acc.w += xs[k].w * by;
        }
      put(acc, sum, mx, bx, row, head);
    }
    return;
  }
  for (int y = blockIdx.y; y < all; y += gridDim.y) {
    if (!place(y, &j, &row, &head)) continue;
    constexpr int AHEAD = 8;                            // partial results on their way before the maxima are known
    float4 xs[AHEAD];
    PartRow rows[AHEAD];
#pragma unroll
    for (int z = 0; z < AHEAD; ++z) {
      const int k = part + z * SPLIT;
      rows[z] = PartRow{NOTHING, NOTHING, 0.f, 0.f};
      xs[z] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k < ph.n_parts) {
        rows[z] = a.part_row[at(k, j)];
        xs[z] = *reinterpret_cast<const float4 *>(a.part_o + at(k, j) * D + 4 * d);
      }
    }
    float mx = NOTHING, bx = NOTHING;
#pragma unroll
    for (int z = 0; z < AHEAD; ++z) {
      mx = fmaxf(mx, rows[z].m);
      bx = fmaxf(bx, rows[z].big_m);
    }
    for (int k = AHEAD * SPLIT + threadIdx.x; k < ph.n_parts; k += 128) {
      const PartRow pr = a.part_row[at(k, j)];
      mx = fmaxf(mx, pr.m);
      bx = fmaxf(bx, pr.big_m);
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) {
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
      bx = fmaxf(bx, __shfl_xor_sync(0xffffffffu, bx, x));
    }
    if ((threadIdx.x & 31) == 0) { red[0][threadIdx.x >> 5] = mx; red[1][threadIdx.x >> 5] = bx; }
    __syncthreads();
    mx = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    bx = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int z = 0; z < AHEAD; ++z) {
      const float by = ex2(rows[z].big_m - bx);
      sum += rows[z].l * ex2(rows[z].m - mx);
      acc.x += xs[z].x * by; acc.y += xs[z].y * by; acc.z += xs[z].z * by; acc.w += xs[z].w * by;
    }
#pragma unroll 4
    for (int k = part + AHEAD * SPLIT; k < ph.n_parts; k += SPLIT) {
      const PartRow pr = a.part_row[at(k, j)];
      const float4 x = *reinterpret_cast<const float4 *>(a.part_o + at(k, j) * D + 4 * d);
      const float by = ex2(pr.big_m - bx);
      sum += pr.l * ex2(pr.m - mx);
      acc.x += x.x * by; acc.y += x.y * by; acc.z += x.z * by; acc.w += x.w * by;
    }
    acc_s[part][d] = acc;
    if (d == 0) sum_s[part] = sum;
    __syncthreads();
    if (part == 0) {
      sum = 0.f;
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < SPLIT; ++k) {
        const float4 x = acc_s[k][d];
        sum += sum_s[k];
        acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
      }
      put(acc, sum, mx, bx, row, head);
    }
    __syncthreads();
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
// part_o and part_row for the larger of the two forms, part_head
size_t workspace_bytes(int n_ctas, int d, size_t *rows, size_t *heads) {
  *rows = align256((size_t)n_ctas * 2 * PP_BLOCKS * PP_ROWS * d * sizeof(float));
  *heads = *rows + align256((size_t)n_ctas * 2 * PP_BLOCKS * PP_ROWS * sizeof(PartRow));
  return *heads + align256((size_t)n_ctas * sizeof(PartHead));
}

// The store as the tensor [page][head, K|V][row][byte]: a box is the K and V rows of a granule, swizzled by the row's length.
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
bool encode_map(CUtensorMap *map, const PagesView &pv, int d) {
  static std::atomic<EncodeTiled> known{nullptr};   // looked up at run time: the library does not link against the driver
  EncodeTiled fn = known.load(std::memory_order_relaxed);
  if (!fn) {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || !p || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      return false;
    }
    fn = (EncodeTiled)p;
    known.store(fn, std::memory_order_relaxed);
  }
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)pv.T, 2 * (cuuint64_t)pv.H, (cuuint64_t)pv.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)d, (cuuint64_t)pv.T * d, (cuuint64_t)pv.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)d, PG_GR, 2, 1}, each[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, pv.codes, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
            d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int FMT, int NT, bool CLUSTER>
cudaError_t launch_form(const AttendArgs &a, const CUtensorMap &map, int n_ctas, int cluster, int device, cudaStream_t st) {
  static std::atomic<unsigned long long> ready{0};       // devices whose kernel has its shared memory
  const auto kernel = wnw_pages_attend_kernel<D, FMT, NT, CLUSTER>;
  if (!(ready.load(std::memory_order_acquire) >> device & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D, NT>());
    if (e != cudaSuccess) { cudaGetLastError(); return e; }
    ready.fetch_or(1ull << device, std::memory_order_release);
  }
  return pg_launch(kernel, dim3(n_ctas), Geo<D, NT>::THREADS, smem_bytes<D, NT>(), st, cluster, a, map);
}
template <int D, int FMT, int NT> cudaError_t launch(const AttendArgs &a, const CUtensorMap &map, int n_ctas, int cluster, int device, cudaStream_t st) {
  return cluster ? launch_form<D, FMT, NT, true>(a, map, n_ctas, cluster, device, st) : launch_form<D, FMT, NT, false>(a, map, n_ctas, 0, device, st);
}
template <int D, int FMT> cudaError_t launch(const AttendArgs &a, const CUtensorMap &map, int nt, int n_ctas, int cluster, int device, cudaStream_t st) {
  return nt == 1 ? launch<D, FMT, 1>(a, map, n_ctas, cluster, device, st) : launch<D, FMT, 2>(a, map, n_ctas, cluster, device, st);
}

// CTAs of a cluster for each head of each sequence, all at once on the GPU; 0: the line.  The line is even whatever the lengths, but lays
// itself out and joins its heads in a second launch; a cluster does neither.  us a call in clusters / on the line when the rule was made, e4m3, 128 elements: 8 KV
// heads of 1000 tokens 6.8 / 11.8, of 3064 8.2 / 10.4, of 15000 16.0 / 17.1, of 30000 26.3 / 23.4; int8, 64 heads of 1000 8.7 / 13.5, of 3000
// 15.2 / 17.5, of 7500 29.3 / 26.4; 128 heads of 3000 24.5 / 25.9.  What a CTA may have to read decides: the table's width says how much, and
// the tiles of query tokens how often.
constexpr long long CLUSTER_BYTES = 512 << 10;
int cluster_of(const AttendArgs &a, int tiles, int d, int n_sm) {
  const long long heads = (long long)a.bv.n_seqs * a.pv.H;
  const int c = heads <= 16 ? 8 : heads <= 32 ? 4 : heads <= 64 ? 2 : heads <= n_sm ? 1 : 0;
  return c && (long long)a.bv.stride * a.pv.T * 2 * d * tiles <= c * CLUSTER_BYTES ? c : 0;
}

std::atomic<int> lose{0};            // of the calls to come

wnw_status_t check_heads(const wnw_pages_t *p, int n_q_heads) {
  if (n_q_heads < 1 || n_q_heads % p->n_kv_heads) return WNW_ERR_INVALID_ARG;
  return n_q_heads / p->n_kv_heads > 16 ? WNW_ERR_UNSUPPORTED : WNW_OK;
}

}  // namespace
}  // namespace wnw

using namespace wnw;

extern "C" wnw_status_t wnw_pages_attend_workspace(const wnw_pages_t *pages, int32_t n_q_heads, int64_t *bytes) {
  PagesView pv;
  wnw_status_t rc = pg_view(pages, &pv);
  if (rc != WNW_OK || !bytes) return rc != WNW_OK ? rc : WNW_ERR_INVALID_ARG;
  if ((rc = check_heads(pages, n_q_heads)) != WNW_OK) return rc;
  OnDevice on(pages->device);
  int n_sm = 0;
  if (!on.ok || pg_sms(pages->device, &n_sm) != WNW_OK) return WNW_ERR_CUDA;
  size_t r, h;
  *bytes = (int64_t)workspace_bytes(n_sm, pages->head_dim, &r, &h);
  return WNW_OK;
}

extern "C" wnw_status_t wnw_debug_pages_lose(int32_t waits) {
  if (waits & ~WNW_DEBUG_WAIT_ALL) return WNW_ERR_INVALID_ARG;
  lose.store(waits, std::memory_order_relaxed);
  return WNW_OK;
}

extern "C" wnw_status_t wnw_pages_attend(const wnw_pages_attend_t *call) {
  if (!call) return WNW_ERR_INVALID_ARG;
  AttendArgs a;
  memset(&a, 0, sizeof(a));
  const wnw_pages_t *pages = call->pages;
  const wnw_batch_t *batch = &call->batch;
  const wnw_rows_t &q = call->q, &out = call->out;
  const float softmax_scale = call->softmax_scale;
  const int dtype = call->dtype;
  wnw_status_t rc = pg_view(pages, batch, &a.pv, &a.bv);
  if (rc != WNW_OK) return rc;
  if ((call->causal & ~1) || q.n_heads != out.n_heads || !(softmax_scale >= 0.f) || std::isinf(softmax_scale)) return WNW_ERR_INVALID_ARG;
  if (dtype != WNW_DTYPE_BF16 && dtype != WNW_DTYPE_FP16) return WNW_ERR_UNSUPPORTED;
  if ((rc = check_heads(pages, q.n_heads)) != WNW_OK) return rc;
  if (!batch->n_seqs || !batch->n_rows) return WNW_OK;
  if (!q.dev || !out.dev || !pg_vector_rows(q, dtype) || !pg_vector_rows(out, dtype) || (uintptr_t)call->lse_dev % 4) return WNW_ERR_INVALID_ARG;
  OnDevice on(pages->device);
  int n_sm = 0;
  if (!on.ok || pg_sms(pages->device, &n_sm) != WNW_OK) return WNW_ERR_CUDA;
  size_t rows_at, heads_at;
  const size_t need = workspace_bytes(n_sm, pages->head_dim, &rows_at, &heads_at);
  void *const workspace_dev = call->workspace_dev;
  if (!workspace_dev || (uintptr_t)workspace_dev % 256 || call->workspace_bytes < (int64_t)need) return WNW_ERR_INVALID_ARG;
  a.q = rows_view(q);
  a.out = rows_view(out);
  a.lse = call->lse_dev;
  a.Hq = q.n_heads;
  a.g = q.n_heads / pages->n_kv_heads;
  a.dtype = dtype;
  a.causal = call->causal;
  a.lose = lose.load(std::memory_order_relaxed);
  a.wait_clocks = a.lose ? 1 << 20 : PP_WAIT_CLOCKS;
  a.values_parity = a.lose & WNW_DEBUG_WAIT_VALUES ? 0 : 1;
  a.scale_log2 = (float)((softmax_scale > 0.f ? (double)softmax_scale : 1.0 / std::sqrt((double)pages->head_dim)) * 1.4426950408889634);
  a.part_o = (float *)workspace_dev;
  a.part_row = (PartRow *)((char *)workspace_dev + rows_at);
  a.part_head = (PartHead *)((char *)workspace_dev + heads_at);
  const int max_rows = batch->max_rows > 0 ? std::min(batch->max_rows, batch->n_rows) : batch->n_rows, d = pages->head_dim;
  // Rows of a KV head that one call of a sequence brings: up to 16 in a pass over the codes, more in passes (the later ones from L2 as far as the
  // codes fit), from 49 on by the tensor cores' tiles of 128.  us, passes / tiles, 8 KV heads of 128: 32 sequences of up to 7500 tokens and
  // up to so many rows, int8, 20 rows 133 / 251, 32 rows 167 / 252, 48 rows 242 / 254; all of the full length and rows, 20 rows 252 / 327,
  // 32 rows 254 / 329, 48 rows 376 / 330; one of 3064, e4m3, 20 rows 20.2 / 23.1, 32 rows 21.4 / 24.0, 48 rows 31.3 / 24.2.
  const bool prompt = (long long)max_rows * a.g > 48;
  const int nt = (long long)max_rows * a.g <= 8 ? 1 : 2;
  a.blocks = prompt ? PP_BLOCKS : 1;
  a.rb = prompt ? PP_ROWS : PA_ROWS;
  a.rt = prompt ? PP_ROWS / a.g : std::min(nt * 8 / a.g, max_rows);
  // items are counted in 32 bits
  if (((long long)batch->n_rows / a.rt + batch->n_seqs) * pages->n_kv_heads > 1ll << 30) return WNW_ERR_CAPACITY;
  const cudaStream_t st = (cudaStream_t)call->cuda_stream;
  cudaError_t e;
  const int cluster = prompt ? 0 : cluster_of(a, (max_rows + a.rt - 1) / a.rt, d, n_sm), n_ctas = cluster ? cluster * a.bv.n_seqs * a.pv.H : n_sm;
  if (prompt) {
    e = launch_prompt(a, d, pages->format, n_sm, pages->device, st);
  } else {
    CUtensorMap map;
    memset(&map, 0, sizeof(map));
    if (pages->n_pages && !encode_map(&map, a.pv, d)) return WNW_ERR_CUDA;
    if (d == 64) e = pages->format == WNW_PAGES_E4M3 ? launch<64, WNW_PAGES_E4M3>(a, map, nt, n_ctas, cluster, pages->device, st) : launch<64, WNW_PAGES_INT8>(a, map, nt, n_ctas, cluster, pages->device, st);
    else e = pages->format == WNW_PAGES_E4M3 ? launch<128, WNW_PAGES_E4M3>(a, map, nt, n_ctas, cluster, pages->device, st) : launch<128, WNW_PAGES_INT8>(a, map, nt, n_ctas, cluster, pages->device, st);
  }
  if (e != cudaSuccess || cluster) return e == cudaSuccess ? WNW_OK : WNW_ERR_CUDA;
  const dim3 grid(n_sm, prompt ? 32 : a.rt * a.g);
  e = pg_launch(d == 64 ? wnw_pages_join_kernel<64> : wnw_pages_join_kernel<128>, grid, 128, 0, st, 0, a);
  return e == cudaSuccess ? WNW_OK : WNW_ERR_CUDA;
}
