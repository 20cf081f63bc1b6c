// Attention of one new token of every sequence over its cached pairs, in pages.
//
// Bound: HBM reads of the cached pairs (each is used once per head that shares it: one flop a byte for bf16, two for e4m3), if a unit costs few enough instructions
// (e4m3: about 890 for 64 positions of a head of 64) and warps enough are there to hide its chain of products, maximum, exponentials and products.
// Measured on one B200, of 6.55 TB/s, in short runs of calls (SM clock 1.97 GHz): 16 sequences of 12 to 33 thousand pairs, 16 heads, e4m3 138 us (86 %; over seconds the
// power cap takes the clock to 1.7 GHz, and it is 163); 128 of 1000, bf16 87 us (93 %); 40 of 0.5 to 8 thousand, 16 query heads on 4 heads of 128, bf16 67.5 us (84 %); 24 of 0 to
// 4096, 12 heads 33.2 us (72 %: some 7 us of every call are launches, the first trips to memory and the join; one sequence of 1024 takes 7.3 us).
// Far from that: heads that are cut by many warps (173 of 1 to 476, 12 heads, e4m3 32 %), e4m3 heads of 128 in middling calls (30 of 1647 51 %), fp32 pages with shared
// heads (39 to 56 %: a shuffle for every weight), more than 8 query heads on one (54 %: the pairs are read for each 8).
//
// Split.  The work of a call is a line of units: sequence by sequence, head of the cache by head, KT positions a unit.  Every warp of the
// launch takes an equal piece of that line, wherever it begins and ends, so one long sequence among short ones costs no more than its bytes;
// the pieces follow from the lengths alone, which each block adds up itself (no plan from the host, the lengths may change between
// replays of a graph).  A warp writes the heads that it holds whole; of a head that it shares with other warps it leaves maximum, sum
// and output in the workspace, and a second kernel joins them in the order of the positions (the result does not depend on timing).  Joining in the warp that
// comes last, with a counter for each head, was slower: fence, counter and join one after the other end a call 7 us later, the second kernel 3.
//
// Stream.  Each warp runs its own ring of STAGES units in shared memory, filled by 16-byte asynchronous copies that run ahead over the ends of heads and
// sequences.  Rows behind a length and pages that do not exist arrive as zeros, so what lies there never meets a product.
//
// Products.  One query row cannot fill a tensor-core tile, but a tile is the cheapest way to use a staged row for all heads that share it:
// up to 8 query heads are rows 0-7 of the A operand of mma m16n8k16 (registers on both sides: with one row of 16 in use and operands read once, tcgen05's
// shared-memory operands and its accumulators' way through TMEM would cost more than the products).  Rows 8-15 carry the second term of the same heads' fp32 numbers, split
// into 16-bit terms, together 22 bits or more (weights are good to 2^-20, with exp2 and the rounding of its argument).  Positions and dimensions are permuted so that each operand is one 16-byte load of a
// row (an order of the contraction is free, and so is the order of the output's columns as long as the epilogue knows it): no transposition.
//   bf16 pages: bf16 products, queries in 1 (bf16) or 3 terms (fp32), weights in 3 terms.
//   e4m3 pages: codes are exact in fp16; fp16 products, queries (scaled by a power of two) in 1 or 2 terms, weights in 2 terms.  The keys' scales
//   multiply the scores, the values' scales the weights, which are kept relative to the largest scaled weight so far (fp16's range); the exponent of a scale is
//   added to a score less its row's maximum, never to the score itself, whose last bit may be worth more than the exponent.
//   fp32 pages: CUDA cores, fp32 throughout.
#include <cuda_fp16.h>

#include <atomic>

#include "rt_paged.h"

namespace rt {
namespace {

constexpr int kWarps = 4, kRows = 8;      // warps of a block; query heads of a unit
constexpr int kSms = 148;
constexpr float kWeightLog2 = 15.0f, kWeightBack = 1.0f / 32768.0f;      // fp16 weights lie in [0, 2^15], the largest above 2^14: their two terms keep 2^-39 of it

// ---- shapes ------------------------------------------------------------------------------------
template <typename CT, int HD>
struct Shape {
  static constexpr int RB = HD * (int)sizeof(CT), NCH = RB / 16;             // bytes and 16-byte chunks of a row
  static constexpr int KT = HD == 128 || sizeof(CT) == 4 ? 16 : sizeof(CT) == 1 ? 64 : 32;      // positions of a unit
  static constexpr int SUB = KT / 16;                                        // (sixteens of them lie in one page)
  static constexpr int KV = 2 * KT * RB;
  static constexpr int EXP = sizeof(CT) == 1 ? 2 * KT : 0;
  static constexpr int OUT = kRows * (HD + 2) * 4;                           // a used stage also carries a head's results
  static constexpr int STAGE = ((KV + EXP > OUT ? KV + EXP : OUT) + 127) / 128 * 128;
  // Units of a ring, and blocks of an SM (both limited by the SM's 227 KB, and by 65,536 registers).  Twelve warps an SM with two units of 8 KB hide a unit's chain
  // better than eight with three (ragged bf16 batch 32.5 us against 37.9) or twelve and sixteen with units of 4 KB (34.9, 33.1); e4m3 units of 64 positions instead of 32
  // spread what a unit costs besides its products (128 us against 143, both with sums in the tensor core).  Heads of 128 in bf16 need the registers of eight warps.
  static constexpr bool SMALL = HD == 64 && sizeof(CT) <= 2;
  static constexpr int STAGES = KV <= 4096 ? 4 : SMALL ? 2 : 3;
  static constexpr int CTAS = KV <= 4096 || SMALL ? 3 : KV <= 8192 ? 2 : 1;
  static constexpr int SMEM = kWarps * STAGES * STAGE;
  static constexpr int WORKERS = kSms * CTAS * kWarps;
};

// ---- the line of units -------------------------------------------------------------------------
// (units are counted in 32 bits: paged_attn_launch refuses caches that could hold more)
struct Line {
  int per;                      // sequences per thread of the scan
  unsigned total, workers;      // units, and the warps that share them: `more` of them take each + 1 units, the others `each`
  unsigned each, more;
  __device__ __forceinline__ unsigned begin(unsigned w) const { return w * each + min(w, more); }
  __device__ __forceinline__ unsigned worker_of(unsigned u) const {
    const unsigned long_part = more * (each + 1);
    return u < long_part ? u / (each + 1) : more + (u - long_part) / each;
  }
};

__device__ __forceinline__ int clamp_len(const PagedAttnParams& p, int b) {
  const int n = __ldg(p.q.lens + b);
  const long long room = (long long)p.c.max_pages << p.log_page;
  return n > room ? (int)room : n;
}
template <int KT>
__device__ __forceinline__ int tiles_of(int n) { return n < 0 ? 0 : max(1, (n + KT - 1) / KT); }

// Units before each thread's first sequence, in sum[] (THREADS entries), and the line.  All threads of the block call.
template <int KT, int THREADS>
__device__ __forceinline__ Line scan_line(const PagedAttnParams& p, int items, int max_workers, unsigned* sum, unsigned* warp_sums, bool report) {
  Line ln;
  ln.per = (p.c.n_seqs + THREADS - 1) / THREADS;
  const int b0 = threadIdx.x * ln.per;
  unsigned mine = 0;
  const long long room = (long long)p.c.max_pages << p.log_page;
  for (int b = b0; b < min(b0 + ln.per, p.c.n_seqs); ++b) {
    const int n = __ldg(p.q.lens + b);
    if (report && n > room && p.c.status) *p.c.status = RT_ERR_INVALID_ARG;
    mine += (unsigned)tiles_of<KT>(n > room ? (int)room : n) * items;
  }
  unsigned inc = mine;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  unsigned before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    total += warp_sums[w];
  }
  sum[threadIdx.x] = before + inc - mine;
  __syncthreads();
  ln.total = total;
  ln.workers = min(total, (unsigned)max_workers);
  ln.each = ln.workers ? total / ln.workers : 0;
  ln.more = total - ln.each * ln.workers;
  return ln;
}

struct Cursor { int b, item, tile, tiles, n; };      // item = head of the cache * slices + slice of its query heads
__device__ __forceinline__ int head_of(int item, int slices) { return slices == 1 ? item : item / slices; }

template <int KT>
__device__ __forceinline__ void next_unit(const PagedAttnParams& p, int items, Cursor& c) {
  if (++c.tile < c.tiles) return;
  c.tile = 0;
  if (++c.item < items) return;
  c.item = 0;
  do {
    if (++c.b >= p.c.n_seqs) { c.b = p.c.n_seqs - 1; return; }               // (behind the line's end: never used)
    c.n = clamp_len(p, c.b);
  } while (c.n < 0);
  c.tiles = tiles_of<KT>(c.n);
}

// ---- small pieces ------------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {        // 2^x to 2^-22, 0 below 2^-126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float whole_power(float n) {      // 2^n of a whole number below 128; 0 below 2^-126
  return __uint_as_float((unsigned)max(127 + (int)n, 0) << 23);
}
__device__ __forceinline__ float q_at(int dtype, const void* p, size_t i) {
  return dtype == RT_BF16 ? __bfloat162float(((const __nv_bfloat16*)p)[i]) : ((const float*)p)[i];
}
__device__ __forceinline__ void copy16(unsigned dst, const void* src, int bytes) {      // bytes = 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes));
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_bf16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool F16>      // without an accumulator
__device__ __forceinline__ void mma_first(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  if (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ F2 ex2(F2 x) {
  float a, b;
  split(x, a, b);
  return f2(ex2(a), ex2(b));
}
// two numbers rounded to a 16-bit type; take_ leaves what the rounding lost
__device__ __forceinline__ unsigned round_bf16(F2 x) {
  float a, b;
  split(x, a, b);
  return pack2(a, b);
}
__device__ __forceinline__ unsigned round_f16(F2 x) {
  float a, b;
  split(x, a, b);
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ unsigned take_bf16(F2& x) {
  const unsigned w = round_bf16(x);
  x = add(x, f2(__uint_as_float((w << 16) ^ 0x80000000u), __uint_as_float((w & 0xffff0000u) ^ 0x80000000u)));
  return w;
}
__device__ __forceinline__ unsigned take_f16(F2& x) {
  const unsigned w = round_f16(x);
  const float2 f = __half22float2(__hneg2(*reinterpret_cast<const __half2*>(&w)));
  x = add(x, f2(f.x, f.y));
  return w;
}
__device__ __forceinline__ unsigned e4m3x2_to_h2(unsigned v) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xffffu), __NV_E4M3);
  return *reinterpret_cast<const unsigned*>(&h);
}

// Places of 16-byte chunks in a staged array of KT rows, such that neither the copies nor the loads below meet bank conflicts: keys are read by
// (row, chunk c) with two neighbouring rows at a time, values by neighbouring chunks of four rows KT / 4 apart.
template <int NCH> __device__ __forceinline__ int key_place(int row, int ch) { return NCH >= 8 ? row * NCH + (ch ^ ((row & 1) << 2)) : row * NCH + ch; }
template <int NCH, int KT> __device__ __forceinline__ int value_place(int row, int ch) {
  const int x = (row / (KT / 4) & 3) << 1;
  return NCH >= 8 ? row * NCH + (ch ^ x) : (row >> 1) * 8 + ((((row & 1) << 2) + ch) ^ x);
}

// ---- tensor-core consumer ------------------------------------------------------------------------
// Lane (r = lane / 4, c = lane % 4) holds row (query head) r of scores and outputs.  Column n of score tile t is position (n / 2) * KT / 4 + 2 t + n % 2 of the
// unit, so that a lane's KT / 4 positions are neighbours: c * KT / 4 + (0 .. KT / 4).
template <typename CT, int HD, bool QF32>
struct Mma {
  using S = Shape<CT, HD>;
  static constexpr bool F8 = sizeof(CT) == 1;
  static constexpr int KS = HD / 16, NT = S::KT / 8, KPL = S::KT / 4, E = 16 / (int)sizeof(CT), TERMS = QF32 ? (F8 ? 2 : 3) : 1;
  unsigned q[TERMS][KS][2];
  F2 o[HD / 8];                            // columns 2 c and 2 c + 1 of every output tile, both terms of the weights together
  float m, q_scale;                        // running maximum (log2 units)
  float top_v;                             // F8: a whole number, at least every weight times value scale (log2) so far relative to m, and less than 1 above the largest; o is relative to it
  F2 l;                                    // this lane's part of the sum
  float slope;

  // The tensor core cuts what a sum loses instead of rounding it: an accumulator kept over a long piece loses half a step of 2^-23 with every product, always
  // towards zero (16 sequences of 12 to 33 thousand pairs: 1.5e-5, where fp32 sums are off by 1e-7).  So it adds up CHAIN sixteens of positions, and ordinary sums do
  // the rest: two over bf16 pages (their unit; 24 of 0 to 4096 33.2 us, one by one 33.7), one over e4m3 pages (16 of 12 to 33 thousand 138 us; with units of four, whose
  // accumulators all live at once, 141.5; with the whole piece in the tensor core 130), and one for fp32 outputs.
  static constexpr int CHAIN = F8 || QF32 ? 1 : S::SUB;
  __device__ __forceinline__ static F2 joined(const float (&c)[4]) { return add(f2(c[0], c[1]), f2(c[2], c[3])); }

  __device__ __forceinline__ void begin(const PagedAttnParams& p, int b, int h0, int g_in, int lane) {
    const int r = lane >> 2, c = lane & 3;
    const bool in = r < g_in;
    const size_t at = (size_t)b * p.q.q_stride + (size_t)(h0 + (in ? r : 0)) * HD;
    F2 x[HD / 8];
#pragma unroll
    for (int i = 0; i < S::NCH / 4; ++i) {
#pragma unroll
      for (int e = 0; e < E; e += 8) {
        float f[8];
        const size_t d = at + (size_t)(c + 4 * i) * E + e;
        if (p.q.dtype == RT_BF16) load8((const __nv_bfloat16*)p.q.q + d, f);
        else load8((const float*)p.q.q + d, f);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[(i * E + e) / 2 + k] = f2(in ? f[2 * k] : 0.f, in ? f[2 * k + 1] : 0.f);
      }
    }
    q_scale = p.scale_log2;
    if (F8) {                              // the largest of the row to [2^10, 2^11)
      float a = 0.f;
#pragma unroll
      for (int d = 0; d < HD / 8; ++d) {
        float y, z;
        split(x[d], y, z);
        a = fmaxf(a, fmaxf(fabsf(y), fabsf(z)));
      }
      a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
      a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
      const int k = min(137 - (int)(__float_as_uint(a) >> 23), 100);       // 10 - floor(log2 a), at least -118
      const float up = __uint_as_float((unsigned)(127 + k) << 23);
#pragma unroll
      for (int d = 0; d < HD / 8; ++d) x[d] = mul(x[d], f2(up, up));
      q_scale *= __uint_as_float((unsigned)(127 - k) << 23);
    }
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        q[t][s][0] = F8 ? take_f16(x[2 * s]) : take_bf16(x[2 * s]);
        q[t][s][1] = F8 ? take_f16(x[2 * s + 1]) : take_bf16(x[2 * s + 1]);
      }
    slope = p.q.alibi_slopes ? __ldg(p.q.alibi_slopes + h0 + (in ? r : 0)) * kLog2e : 0.f;
    m = top_v = -INFINITY;
    l = f2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < HD / 8; ++j) o[j] = f2(0.f, 0.f);
  }

  // One staged unit: positions j0 .. j0 + KT; the first `live` count, but not the sixteens whose bit is
  // set in `bad`; the query is at position `at`.
  __device__ __forceinline__ void unit(const PagedAttnParams& p, const unsigned char* st, int j0, int at, int live, unsigned bad, int lane) {
    const int r = lane >> 2, c = lane & 3;
    float s[NT][4];
#pragma unroll
    for (int i = 0; i < S::NCH / 4; ++i) {
      unsigned x[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint4 w = reinterpret_cast<const uint4*>(st)[key_place<S::NCH>((r >> 1) * KPL + 2 * t + (r & 1), c + 4 * i)];
        x[t][0] = w.x; x[t][1] = w.y; x[t][2] = w.z; x[t][3] = w.w;
      }
      constexpr int KC = E / 4, T1 = TERMS > 1 ? 1 : 0;        // contraction steps of a chunk; the tiles in turn, so that products do not wait for one another
#pragma unroll
      for (int u = 0; u < KC; ++u) {
        const int k = i * KC + u;
        const unsigned q2 = TERMS > 1 ? q[T1][k][0] : 0u, q3 = TERMS > 1 ? q[T1][k][1] : 0u;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const unsigned b0 = F8 ? e4m3x2_to_h2(x[t][u]) : x[t][(2 * u) & 3], b1 = F8 ? e4m3x2_to_h2(x[t][u] >> 16) : x[t][(2 * u + 1) & 3];
          if (k == 0) mma_first<F8>(s[t], q[0][k][0], q2, q[0][k][1], q3, b0, b1);
          else if (F8) mma_f16(s[t], q[0][k][0], q2, q[0][k][1], q3, b0, b1);
          else mma_bf16(s[t], q[0][k][0], q2, q[0][k][1], q3, b0, b1);
        }
        if (TERMS > 2) {
#pragma unroll
          for (int t = 0; t < NT; ++t) mma_bf16(s[t], q[TERMS - 1][k][0], 0u, q[TERMS - 1][k][1], 0u, x[t][(2 * u) & 3], x[t][(2 * u + 1) & 3]);
        }
      }
    }
    // scores in log2 units, the maximum of the row (for F8 then that of the scaled weights), weights; two positions at a time
    F2 a[NT], av[F8 ? NT : 1];
    unsigned ke[KPL / 4], ve[KPL / 4];       // the exponents of this lane's positions
    if (F8) {
#pragma unroll
      for (int y = 0; y < KPL / 4; ++y) {
        ke[y] = reinterpret_cast<const unsigned*>(st + S::KV + KPL * c)[y];
        ve[y] = reinterpret_cast<const unsigned*>(st + S::KV + S::KT + KPL * c)[y];
      }
    }
    const F2 scale2 = f2(q_scale, q_scale);
#pragma unroll
    for (int t = 0; t < NT; ++t) {           // positions 2 t and 2 t + 1 of the lane's
      F2 x = f2(s[t][0], s[t][1]);
      if (TERMS > 1) x = add(x, f2(s[t][2], s[t][3]));
      if (F8) {
        const unsigned w = ke[t / 2];
        const F2 ks = t & 1 ? f2(__uint_as_float(w << 7 & 0x7f800000u), __uint_as_float(w >> 1 & 0x7f800000u))
                            : f2(__uint_as_float(w << 23 & 0x7f800000u), __uint_as_float(w << 15 & 0x7f800000u));
        a[t] = mul(x, mul(scale2, ks));
      } else {
        a[t] = mul(x, scale2);
      }
    }
    if (p.q.alibi_slopes) {
      const float far = (float)(j0 + KPL * c - at);
#pragma unroll
      for (int t = 0; t < NT; ++t) a[t] = fma(f2(slope, slope), add(f2(far, far), f2((float)(2 * t), (float)(2 * t + 1))), a[t]);
    }
    if (live < S::KT || bad) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int j = KPL * c + 2 * t;
        const bool gone = bad >> (j / 16) & 1;
        const float i0 = gone || j >= live ? -INFINITY : 0.f, i1 = gone || j + 1 >= live ? -INFINITY : 0.f;
        float x, y;
        split(a[t], x, y);
        a[t] = f2(i0 != 0.f ? i0 : x, i1 != 0.f ? i1 : y);
      }
    }
    float top = m;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float x, y;
      split(a[t], x, y);
      top = fmaxf(top, fmaxf(x, y));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const float ref = top == -INFINITY ? 0.f : -top, shift = m == -INFINITY ? 0.f : m - top;
#pragma unroll
    for (int t = 0; t < NT; ++t) a[t] = add(a[t], f2(ref, ref));
    float topv = top_v + shift;
    if (F8) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {         // 2^23 + exponent - (2^23 + 127)
        const unsigned w = ve[t / 2], sel = 0x7550u + 2 * (t & 1);
        av[F8 ? t : 0] = add(a[t], add(f2(__uint_as_float(__byte_perm(w, 0x4b000000u, sel)), __uint_as_float(__byte_perm(w, 0x4b000000u, sel + 1))),
                                       f2(-8388735.f, -8388735.f)));
        float x, y;
        split(av[F8 ? t : 0], x, y);
        topv = fmaxf(topv, fmaxf(x, y));
      }
      topv = fmaxf(topv, __shfl_xor_sync(0xffffffffu, topv, 1));
      topv = fmaxf(topv, __shfl_xor_sync(0xffffffffu, topv, 2));
    }
    if (__any_sync(0xffffffffu, top > m || (F8 && topv > top_v))) {
      const float w = m == -INFINITY ? 0.f : ex2(shift);
      float wo = w;
      if (F8) {                              // w 2^(top_v - to); shift + up is exact where up > 0 (up <= -shift)
        const float to = ceilf(topv), up = top_v - to;
        if (top_v == -INFINITY) wo = 0.f;
        else wo = up > 0.f ? ex2(shift + up) : w * whole_power(up);
        top_v = to;
      }
      l = mul(l, f2(w, w));
#pragma unroll
      for (int j = 0; j < HD / 8; ++j) o[j] = mul(o[j], f2(wo, wo));
      m = top;
    }
    const float refv = top_v == -INFINITY ? 0.f : kWeightLog2 - top_v;
    float acc[F8 ? 1 : HD / 8][4];           // what the tensor core adds up, over bf16 pages
#pragma unroll
    for (int sub = 0; sub < S::SUB; ++sub) {
      unsigned w0[2], w1[2], w2[2];          // terms of the weights of positions 4 sub + (0, 1) and (2, 3) of the lane's
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = 2 * sub + h;
        F2 w = ex2(a[t]);
        l = add(l, w);
        if (F8) {
          w = ex2(add(av[F8 ? t : 0], f2(refv, refv)));
          w0[h] = take_f16(w);
          w1[h] = round_f16(w);
          w2[h] = 0;
        } else {
          w0[h] = take_bf16(w);
          w1[h] = take_bf16(w);
          w2[h] = round_bf16(w);
        }
      }
      const unsigned char* vt = st + S::KT * S::RB;
      const int row0 = KPL * c + 4 * sub;
      if (!F8) {
#pragma unroll
        for (int i = 0; i < S::NCH / 8; ++i) {         // chunk r + 8 i of the four rows: dimensions 64 i + 8 r + (0 .. 7)
          unsigned x[4][4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint4 y = reinterpret_cast<const uint4*>(vt)[value_place<S::NCH, S::KT>(row0 + k, r + 8 * i)];
            x[k][0] = y.x; x[k][1] = y.y; x[k][2] = y.z; x[k][3] = y.w;
          }
#pragma unroll
          for (int half = 0; half < 2; ++half) {       // four products, then the four of the third term
            unsigned b0[4], b1[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int j = 4 * half + y;
              const unsigned sel = (j & 1) ? 0x7632u : 0x5410u;
              b0[y] = __byte_perm(x[0][j / 2], x[1][j / 2], sel);
              b1[y] = __byte_perm(x[2][j / 2], x[3][j / 2], sel);
              if (sub % CHAIN == 0) mma_first<false>(acc[8 * i + j], w0[0], w1[0], w0[1], w1[1], b0[y], b1[y]);
              else mma_bf16(acc[8 * i + j], w0[0], w1[0], w0[1], w1[1], b0[y], b1[y]);
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int t = 8 * i + 4 * half + y;
              mma_bf16(acc[t], w2[0], 0u, w2[1], 0u, b0[y], b1[y]);
              if (sub % CHAIN == CHAIN - 1) o[t] = add(o[t], joined(acc[t]));
            }
          }
        }
      } else {
        constexpr int WD = HD / 32;                    // words of this lane: dimensions 4 WD r + (0 .. 4 WD)
        unsigned x[4][WD];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (WD == 2) {
            const uint2 y = *reinterpret_cast<const uint2*>(vt + value_place<S::NCH, S::KT>(row0 + k, r >> 1) * 16 + (r & 1) * 8);
            x[k][0] = y.x; x[k][1] = y.y;
          } else {
            const uint4 y = reinterpret_cast<const uint4*>(vt)[value_place<S::NCH, S::KT>(row0 + k, r)];
            x[k][0] = y.x; x[k][1] = y.y; x[k][2] = y.z; x[k][3] = y.w;
          }
        }
#pragma unroll
        for (int d = 0; d < WD; ++d) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const unsigned sel = h ? 0x7362u : 0x5140u;
            const unsigned y0 = __byte_perm(x[0][d], x[1][d], sel), y1 = __byte_perm(x[2][d], x[3][d], sel);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int t = 4 * d + 2 * h + e;
              float sixteen[4];
              mma_first<true>(sixteen, w0[0], w1[0], w0[1], w1[1], e4m3x2_to_h2(y0 >> (16 * e)), e4m3x2_to_h2(y1 >> (16 * e)));
              o[t] = add(o[t], joined(sixteen));
            }
          }
        }
      }
    }
  }

  // Maximum, sum and output of every row into shared memory: out[r][HD], ml[r][2].  False if a row of the first g_in is not finite.
  __device__ __forceinline__ bool dump(float* out, int g_in, int lane) {
    const int r = lane >> 2, c = lane & 3;
    float all = 0.f;
    float sum, other;
    split(l, sum, other);
    sum += other;
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    const float back = top_v == -INFINITY ? 0.f : whole_power(top_v);       // (times 2^-15 it may lie below fp32's normal numbers, outputs may not)
#pragma unroll
    for (int j = 0; j < HD / 8; ++j) {
      float y[2];
      split(F8 ? mul(mul(o[j], f2(kWeightBack, kWeightBack)), f2(back, back)) : o[j], y[0], y[1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // column 2 c + e of output tile j
        out[r * HD + (F8 ? (HD / 8) * (2 * c + e) + j : (j / 8) * 64 + 8 * (2 * c + e) + j % 8)] = y[e];
        all = fmaf(y[e], 0.f, all);        // NaN once one is not finite
      }
    }
    if (c == 0) { out[kRows * HD + 2 * r] = m; out[kRows * HD + 2 * r + 1] = sum; }
    return !__any_sync(0xffffffffu, r < g_in && !(all == 0.f && sum < INFINITY));
  }
};

// ---- fp32 pages: CUDA cores ----------------------------------------------------------------------
// LPK = HD / 4 lanes hold a row, 128 / HD rows lie side by side.  The heads' dot products are added up over the lanes together: each step hands half of
// the heads to the other half of the lanes, so that a lane ends with the score of one head (G - 1 shuffles and a few, not 4 or 5 for each head) and
// maxima, exponentials and sums are that head's alone; its weights go to the other lanes one by one for the outputs.
template <int HD, int G>
struct Simt {
  using S = Shape<float, HD>;
  static constexpr int LPK = HD / 4, KPI = 32 / LPK, IT = 16 / KPI, PER = LPK / G;      // PER lanes hold the same head's score
  F2 q[G][2], o[G][2];
  float m, l, slope;                       // of this lane's head

  __device__ __forceinline__ void begin(const PagedAttnParams& p, int b, int h0, int g_in, int lane) {
    const int c = lane % LPK;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const size_t at = (size_t)b * p.q.q_stride + (size_t)(h0 + min(g, g_in - 1)) * HD + c * 4;
      q[g][0] = f2(q_at(p.q.dtype, p.q.q, at), q_at(p.q.dtype, p.q.q, at + 1));
      q[g][1] = f2(q_at(p.q.dtype, p.q.q, at + 2), q_at(p.q.dtype, p.q.q, at + 3));
      o[g][0] = o[g][1] = f2(0.f, 0.f);
    }
    slope = p.q.alibi_slopes ? __ldg(p.q.alibi_slopes + h0 + min(c / PER, g_in - 1)) * kLog2e : 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  // a value of the lane's head from the lane of each head, in turn
  __device__ __forceinline__ float from_head(float x, int g, int lane) const { return __shfl_sync(0xffffffffu, x, (lane & ~(LPK - 1)) + g * PER); }

  __device__ __forceinline__ void unit(const PagedAttnParams& p, const unsigned char* st, int j0, int at, int live, unsigned bad, int lane) {
    const int sub = lane / LPK, c = lane % LPK;
    float s[IT], top = m;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int j = i * KPI + sub;
      const float4 k = reinterpret_cast<const float4*>(st)[key_place<S::NCH>(j, c)];
      const F2 k0 = f2(k.x, k.y), k1 = f2(k.z, k.w);
      float a[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float x, y;
        split(fma(q[g][1], k1, mul(q[g][0], k0)), x, y);
        a[g] = x + y;
      }
#pragma unroll
      for (int off = LPK / 2, n = G; off; off >>= 1) {
        if (n > 1) {
          n >>= 1;
          const bool upper = (lane & off) != 0;
#pragma unroll
          for (int g = 0; g < G / 2; ++g)
            if (g < n) {
              const float send = upper ? a[g] : a[g + n], keep = upper ? a[g + n] : a[g];
              a[g] = keep + __shfl_xor_sync(0xffffffffu, send, off);
            }
        } else {
          a[0] += __shfl_xor_sync(0xffffffffu, a[0], off);
        }
      }
      s[i] = j < live && !bad ? a[0] * p.scale_log2 - slope * (float)(at - j0 - j) : -INFINITY;
      top = fmaxf(top, s[i]);
    }
    if (KPI == 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, LPK));
    if (__any_sync(0xffffffffu, top > m)) {
      const float w = m == -INFINITY ? 0.f : ex2(m - top);
      l *= w;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float x = from_head(w, g, lane);
        o[g][0] = mul(o[g][0], f2(x, x));
        o[g][1] = mul(o[g][1], f2(x, x));
      }
      m = top;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const float4 v = reinterpret_cast<const float4*>(st + 16 * S::RB)[value_place<S::NCH, S::KT>(i * KPI + sub, c)];      // (rows that do not count are zeros)
      const F2 v0 = f2(v.x, v.y), v1 = f2(v.z, v.w);
      const float w = ex2(s[i] - ref);
      l += w;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float x = G == 1 ? w : from_head(w, g, lane);
        o[g][0] = fma(f2(x, x), v0, o[g][0]);
        o[g][1] = fma(f2(x, x), v1, o[g][1]);
      }
    }
  }
  __device__ __forceinline__ bool dump(float* out, int g_in, int lane) {
    const int c = lane % LPK;
    if (KPI == 2) l += __shfl_xor_sync(0xffffffffu, l, LPK);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float4 y;
      split(o[g][0], y.x, y.y);
      split(o[g][1], y.z, y.w);
      if (KPI == 2) {
        y.x += __shfl_xor_sync(0xffffffffu, y.x, LPK); y.y += __shfl_xor_sync(0xffffffffu, y.y, LPK);
        y.z += __shfl_xor_sync(0xffffffffu, y.z, LPK); y.w += __shfl_xor_sync(0xffffffffu, y.w, LPK);
      }
      if (lane < LPK && g < g_in) *reinterpret_cast<float4*>(out + g * HD + c * 4) = y;
    }
    if (lane < LPK && c % PER == 0 && c / PER < g_in) { out[kRows * HD + 2 * (c / PER)] = m; out[kRows * HD + 2 * (c / PER) + 1] = l; }
    return true;
  }
};

// What Mma::dump leaves, position by position from the pages, for heads whose result is not finite: the terms of a split number meet an
// infinity with either sign, or as zeros, so an infinite key or value that counts would come out as NaN.
template <typename CT, int HD>
__device__ __noinline__ void slow_piece(const PagedAttnParams& p, int b, int kvh, int h0, int g_in, int j0, int j1, int at, float* out, int lane) {
  for (int g = 0; g < g_in; ++g) {
    const int h = h0 + g;
    const float slope = p.q.alibi_slopes ? __ldg(p.q.alibi_slopes + h) * kLog2e : 0.f;
    float q[HD / 32], o[HD / 32], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) { q[d] = q_at(p.q.dtype, p.q.q, (size_t)b * p.q.q_stride + (size_t)h * HD + d * 32 + lane); o[d] = 0.f; }
    for (int j = j0; j < j1; ++j) {
      const int page = __ldg(p.c.page_table + (size_t)b * p.c.max_pages + (j >> p.log_page));
      if ((unsigned)page >= (unsigned)p.c.n_pages) continue;
      const size_t row = ((size_t)page * p.c.n_kv_heads + kvh) * p.c.page_size + (j & (p.c.page_size - 1));
      const CT *k = (const CT*)p.c.k + row * HD, *v = (const CT*)p.c.v + row * HD;
      const float ks = sizeof(CT) == 1 ? scale_of(p.c.k_exp[row]) : 1.f, vs = sizeof(CT) == 1 ? scale_of(p.c.v_exp[row]) : 1.f;
      float a = 0.f;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) a += q[d] * ((float)k[d * 32 + lane] * ks);
      a = warp_sum(a) * p.scale_log2 - slope * (float)(at - j);
      const float mn = fmaxf(m, a), ref = mn == -INFINITY ? 0.f : mn, w0 = exp2f(m - ref), w1 = exp2f(a - ref);
      m = mn;
      l = l * w0 + w1;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) o[d] = o[d] * w0 + w1 * ((float)v[d * 32 + lane] * vs);
    }
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) out[g * HD + d * 32 + lane] = o[d];
    if (lane == 0) { out[kRows * HD + 2 * g] = m; out[kRows * HD + 2 * g + 1] = l; }
  }
}

// ---- what both kernels end with: the own pair, the division, out and lse ---------------------------
// The own pair of query head h of sequence b, as its warp holds it: the score and this lane's dimensions d * 32 + lane of the value.
template <int HD>
struct Own {
  float a, v[HD / 32];
  __device__ __forceinline__ void load(const PagedAttnParams& p, int b, int h, int lane) {
    a = -INFINITY;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) v[d] = 0.f;
    if (!p.q.k_own) return;
    const size_t qa = (size_t)b * p.q.q_stride + (size_t)h * HD, kvh = (size_t)(h / p.group) * HD;
    float x = 0.f;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) {
      x += q_at(p.q.dtype, p.q.q, qa + d * 32 + lane) * q_at(p.q.dtype, p.q.k_own, (size_t)b * p.q.k_own_stride + kvh + d * 32 + lane);
      v[d] = q_at(p.q.dtype, p.q.v_own, (size_t)b * p.q.v_own_stride + kvh + d * 32 + lane);
    }
    a = warp_sum(x) * p.scale_log2;
  }
};
// m, l and this lane's dimensions of o over the cached pairs -> out, lse
template <int HD>
__device__ __forceinline__ void finish_head(const PagedAttnParams& p, const Own<HD>& own, int b, int h, int lane, float m, float l, float (&o)[HD / 32]) {
  if (p.q.k_own) {
    const float mn = fmaxf(m, own.a), ref = mn == -INFINITY ? 0.f : mn, w0 = ex2(m - ref), w1 = ex2(own.a - ref);
    m = mn;
    l = l * w0 + w1;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = o[d] * w0 + w1 * own.v[d];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) {
    const float y = l == 0.f ? 0.f : o[d] * inv;
    const size_t i = (size_t)b * p.q.out_stride + (size_t)h * HD + d * 32 + lane;
    if (p.q.dtype == RT_BF16) ((__nv_bfloat16*)p.q.out)[i] = __float2bfloat16_rn(y);
    else ((float*)p.q.out)[i] = y;
  }
  if (p.q.lse && lane == 0) p.q.lse[(size_t)b * p.q.n_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// A warp's partial results: slot 0 for the head that it takes over in its middle, slot 1 for the head that it begins and does not end.
// Of each: rows of o, then (m, l) per row.
__host__ __device__ inline size_t slot_floats(int rows, int hd) { return (size_t)rows * (hd + 2); }

template <typename CT, int HD, typename Consumer>
__global__ void __launch_bounds__(kWarps * 32, Shape<CT, HD>::CTAS) paged_attn_kernel(const __grid_constant__ PagedAttnParams p, float* part, int part_rows) {
  using S = Shape<CT, HD>;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ unsigned sums[kWarps * 32], warp_sums[kWarps];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (p.group + kRows - 1) / kRows, items = p.c.n_kv_heads * slices;
  const Line ln = scan_line<S::KT, kWarps * 32>(p, items, S::WORKERS, sums, warp_sums, blockIdx.x == 0);
  const unsigned me = warp * gridDim.x + blockIdx.x;                           // neighbours on the line sit on different SMs
  if (me >= ln.workers) return;
  const unsigned u0 = ln.begin(me);
  const int count = (int)(ln.begin(me + 1) - u0);

  // where the line stands at u0
  Cursor cc;
  {
    int lo = 0, hi = kWarps * 32 - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sums[mid] <= u0) lo = mid; else hi = mid - 1;
    }
    // (several threads may hold no sequence: the last one whose sum is <= u0 has the unit, or begins behind sequences without units)
    unsigned rest = u0 - sums[lo];
    int b = lo * ln.per;
    for (;; ++b) {
      if (b >= p.c.n_seqs) return;                                             // (only if somebody changes the lengths meanwhile)
      cc.n = clamp_len(p, b);
      cc.tiles = tiles_of<S::KT>(cc.n);
      const unsigned here = (unsigned)cc.tiles * items;
      if (rest < here) break;
      rest -= here;
    }
    cc.b = b;
    cc.item = (int)(rest / (unsigned)cc.tiles);
    cc.tile = (int)(rest - (unsigned)cc.item * cc.tiles);
  }

  // The producer: its cursor, and what changes with the head only.  The table is looked up a unit ahead of the copies.
  Cursor cp = cc;
  unsigned char* ring = smem + (size_t)warp * S::STAGES * S::STAGE;
  const unsigned ring_at = (unsigned)__cvta_generic_to_shared(ring);
  const unsigned page_bytes = (unsigned)p.c.n_kv_heads * p.c.page_size * S::RB;
  const int in_page = p.c.page_size - 1, log_page = p.log_page;
  const unsigned n_pages = p.c.n_pages;
  const int* table;
  const unsigned char *k0, *v0;                                                // this lane's first chunk of the head in page 0
  const uint8_t* e0;                                                           // lanes 0 .. 2 SUB - 1: exponents of keys (even), values (odd) of a sixteen
  unsigned bad = 0;                                                            // SUB bits a stage: sixteens without a page
  auto enter_head = [&]() {
    const size_t kv_row = (size_t)head_of(cp.item, slices) * p.c.page_size;
    table = p.c.page_table + (size_t)cp.b * p.c.max_pages;
    k0 = (const unsigned char*)p.c.k + kv_row * S::RB + lane * 16;
    v0 = (const unsigned char*)p.c.v + kv_row * S::RB + lane * 16;
    e0 = ((lane & 1) ? p.c.v_exp : p.c.k_exp) + kv_row;
  };
  int pages[S::SUB];
  auto fetch_pages = [&]() {
    const int j = cp.tile * S::KT;
#pragma unroll
    for (int s = 0; s < S::SUB; ++s) pages[s] = j + 16 * s < cp.n ? __ldg(table + ((j + 16 * s) >> log_page)) : -1;
  };
  auto produce = [&](int stage) {
    const unsigned dst = ring_at + stage * S::STAGE;
    const int j = cp.tile * S::KT;
    bool full = j + S::KT <= cp.n;
#pragma unroll
    for (int s = 0; s < S::SUB; ++s) full = full && (unsigned)pages[s] < n_pages;
    bad &= ~(((1u << S::SUB) - 1) << (stage * S::SUB));
    if (full) {
      size_t off[S::SUB];
#pragma unroll
      for (int s = 0; s < S::SUB; ++s) {
        off[s] = (size_t)pages[s] * page_bytes + (unsigned)(((j + 16 * s) & in_page) * S::RB);
        const unsigned char *k = k0 + off[s], *v = v0 + off[s];
#pragma unroll
        for (int i = 0; i < S::NCH / 2; ++i) {
          const int row = 16 * s + 32 / S::NCH * i + lane / S::NCH, ch = lane % S::NCH;
          copy16(dst + key_place<S::NCH>(row, ch) * 16, k + i * 512, 16);
          copy16(dst + S::KT * S::RB + value_place<S::NCH, S::KT>(row, ch) * 16, v + i * 512, 16);
        }
      }
      if (S::EXP && lane < 2 * S::SUB) {
        size_t mine = off[0];
#pragma unroll
        for (int s = 1; s < S::SUB; ++s) if (lane >> 1 == s) mine = off[s];
        copy16(dst + S::KV + (lane & 1) * S::KT + (lane >> 1) * 16, e0 + mine / S::RB, 16);
      }
    } else {
#pragma unroll 1
      for (int s = 0; s < S::SUB; ++s) {
        int page = pages[0];
#pragma unroll
        for (int t = 1; t < S::SUB; ++t) if (s == t) page = pages[t];
        const int js = j + 16 * s;
        const bool ok = (unsigned)page < n_pages;
        const int live = ok ? cp.n - js : 0;
        const size_t off = ok ? (size_t)page * page_bytes + (unsigned)((js & in_page) * S::RB) : 0;
        if (!ok) {
          bad |= 1u << (stage * S::SUB + s);
          if (js < cp.n && p.c.status && lane == 0) *p.c.status = RT_ERR_INVALID_ARG;
        }
#pragma unroll 1
        for (int i = 0; i < S::NCH / 2; ++i) {
          const int row = (i * 32 + lane) / S::NCH, ch = lane % S::NCH;
          const bool in = row < live;
          copy16(dst + key_place<S::NCH>(16 * s + row, ch) * 16, in ? k0 + off + i * 512 : (const unsigned char*)p.c.k, in ? 16 : 0);
          copy16(dst + S::KT * S::RB + value_place<S::NCH, S::KT>(16 * s + row, ch) * 16, in ? v0 + off + i * 512 : (const unsigned char*)p.c.v, in ? 16 : 0);
        }
        if (S::EXP && lane < 2) copy16(dst + S::KV + lane * S::KT + 16 * s, ok ? e0 + off / S::RB : (const uint8_t*)p.c.k, ok ? 16 : 0);
      }
    }
    if (++cp.tile == cp.tiles) {
      --cp.tile;
      next_unit<S::KT>(p, items, cp);
      enter_head();
    }
  };

  Consumer con;
  enter_head();
  fetch_pages();
#pragma unroll
  for (int s = 0; s < S::STAGES - 1; ++s) {
    if (s < count) {
      produce(s);
      fetch_pages();
    }
    copy_commit();
  }
  auto begin_head = [&]() {
    const int g0 = (slices == 1 ? 0 : cc.item % slices) * kRows;
    con.begin(p, cc.b, head_of(cc.item, slices) * p.group + g0, min(kRows, p.group - g0), lane);
  };
  begin_head();                                                                // (the first head's queries arrive beside its pairs)
  bool fresh = false;
  int first_tile = cc.tile, stage = 0;
  for (int i = 0; i < count; ++i, stage = stage + 1 == S::STAGES ? 0 : stage + 1) {
    copy_wait<S::STAGES - 2>();
    __syncwarp();
    if (i + S::STAGES - 1 < count) {
      produce(stage == 0 ? S::STAGES - 1 : stage - 1);
      fetch_pages();
    }
    copy_commit();
    if (fresh) {
      begin_head();
      first_tile = cc.tile;
      fresh = false;
    }
    unsigned char* st = ring + stage * S::STAGE;
    con.unit(p, st, cc.tile * S::KT, p.q.k_own ? cc.n : cc.n - 1, cc.n - cc.tile * S::KT, bad >> (stage * S::SUB) & ((1u << S::SUB) - 1), lane);
    const bool ends = cc.tile + 1 == cc.tiles;
    if (ends || i + 1 == count) {
      // the stage is used up: it holds the head's results on their way out
      const int kv_head = head_of(cc.item, slices), g0 = (slices == 1 ? 0 : cc.item % slices) * kRows, g_in = min(kRows, p.group - g0),
                h0 = kv_head * p.group + g0;
      float* out = reinterpret_cast<float*>(st);
      __syncwarp();
      const bool fine = con.dump(out, g_in, lane);
      __syncwarp();
      if (!fine) {
        slow_piece<CT, HD>(p, cc.b, kv_head, h0, g_in, first_tile * S::KT, min(cc.n, (cc.tile + 1) * S::KT), p.q.k_own ? cc.n : cc.n - 1, out, lane);
        __syncwarp();
      }
      if (ends && first_tile == 0) {
        for (int g = 0; g < g_in; ++g) {
          float x[HD / 32];
          Own<HD> own;
          own.load(p, cc.b, h0 + g, lane);
#pragma unroll
          for (int d = 0; d < HD / 32; ++d) x[d] = out[g * HD + d * 32 + lane];
          finish_head<HD>(p, own, cc.b, h0 + g, lane, out[kRows * HD + 2 * g], out[kRows * HD + 2 * g + 1], x);
        }
      } else {
        float* slot = part + ((size_t)me * 2 + (first_tile == 0 ? 1 : 0)) * slot_floats(part_rows, HD);
        for (int g = 0; g < g_in; ++g) {
#pragma unroll
          for (int d = 0; d < HD / 32; ++d) slot[g * HD + d * 32 + lane] = out[g * HD + d * 32 + lane];
        }
        if (lane < 2 * g_in) slot[part_rows * HD + lane] = out[kRows * HD + lane];
      }
      fresh = true;
      next_unit<S::KT>(p, items, cc);
    } else {
      ++cc.tile;
    }
  }
}

// Joins the heads that several warps of the kernel above share: a block takes a query head, its warps every kJoinWarps-th partial result
// (maxima and sums first, one result a lane, then outputs with known weights: two trips to memory for up to 32 a warp).  It
// starts beside that kernel (programmatic launch): all that does not depend on its results is done before the wait.
template <int KT, int HD, int kJoinWarps>
__global__ void __launch_bounds__(kJoinWarps * 32) paged_join_kernel(const __grid_constant__ PagedAttnParams p, const float* part, int part_rows, int max_workers) {
  __shared__ unsigned sums[kJoinWarps * 32], warp_sums[kJoinWarps];
  __shared__ float sm_o[kJoinWarps][HD], sm_m[kJoinWarps], sm_l[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (p.group + kRows - 1) / kRows, items = p.c.n_kv_heads * slices;
  const Line ln = scan_line<KT, kJoinWarps * 32>(p, items, max_workers, sums, warp_sums, false);
  bool waited = false;
  const long long all = ln.total ? (long long)p.c.n_seqs * p.q.n_heads : 0;
  for (long long x = blockIdx.x; x < all; x += gridDim.x) {
    const int b = (int)(x / p.q.n_heads), h = (int)(x - (long long)b * p.q.n_heads);
    const int n = clamp_len(p, b);
    if (n < 0) continue;
    unsigned u = sums[b / ln.per];
    for (int s = b / ln.per * ln.per; s < b; ++s) u += (unsigned)tiles_of<KT>(clamp_len(p, s)) * items;
    const int tiles = tiles_of<KT>(n), g = h % p.group;
    u += (unsigned)(h / p.group * slices + g / kRows) * tiles;
    const unsigned w0 = min(ln.worker_of(u), ln.workers - 1), w1 = min(ln.worker_of(u + tiles - 1), ln.workers - 1);      // (min: as above)
    if (w0 == w1) continue;                                            // written by the warp that held all of it
    const int r = g % kRows;
    Own<HD> own;
    if (warp == 0) own.load(p, b, h, lane);
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    waited = true;
    float m = -INFINITY, l = 0.f, o[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
    auto slot = [&](unsigned w) { return part + ((size_t)w * 2 + (w == w0 ? 1 : 0)) * slot_floats(part_rows, HD); };
    for (unsigned first = w0 + warp; first <= w1; first += 32 * kJoinWarps) {
      const unsigned mine = first + lane * kJoinWarps;
      float ms = -INFINITY, ls = 0.f;
      if (mine <= w1) {
        const float* s = slot(mine) + part_rows * HD + 2 * r;
        ms = s[0]; ls = s[1];
      }
      const float mn = fmaxf(m, warp_max(ms)), ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(m - ref), f = ex2(ms - ref);
      m = mn;
      l = l * f0 + warp_sum(ls * f);
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) o[d] *= f0;
      const int n = (int)min(32u, (w1 - first) / kJoinWarps + 1);
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const float fk = __shfl_sync(0xffffffffu, f, k);
        const float* s = slot(first + k * kJoinWarps) + r * HD + lane;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) o[d] += s[d * 32] * fk;
      }
    }
    __syncthreads();                                                   // (the arrays of the head before are read)
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) sm_o[warp][d * 32 + lane] = o[d];
    if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
    __syncthreads();
    if (warp == 0) {
      float ma = -INFINITY, la = 0.f;
#pragma unroll
      for (int w = 0; w < kJoinWarps; ++w) ma = fmaxf(ma, sm_m[w]);
      const float ref = ma == -INFINITY ? 0.f : ma;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
#pragma unroll
      for (int w = 0; w < kJoinWarps; ++w) {
        const float f = ex2(sm_m[w] - ref);
        la += sm_l[w] * f;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) o[d] += sm_o[w][d * 32 + lane] * f;
      }
      finish_head<HD>(p, own, b, h, lane, ma, la, o);
    }
  }
  if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");      // (this grid must not end before the one it follows)
}

int part_rows_of(int group) { return group < kRows ? group : kRows; }

template <typename CT, int HD, typename Consumer>
cudaError_t launch_split(const PagedAttnParams& p, float* part, cudaStream_t s) {
  using S = Shape<CT, HD>;
  auto* kernel = paged_attn_kernel<CT, HD, Consumer>;
  static std::atomic<unsigned long long> set{0};         // devices on which the kernel has its shared memory
  int dev = 0;
  if (const cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
  if (dev > 63 || !(set.load(std::memory_order_relaxed) >> dev & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess) return e;
    if (dev <= 63) set.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  // units there can be at most: no more warps than that
  const long long slices = ceil_div(p.group, kRows);
  const long long most = (long long)p.c.n_seqs * p.c.n_kv_heads * slices * max(1LL, ((long long)p.c.max_pages * p.c.page_size + S::KT - 1) / S::KT);
  const int grid = (int)(most < kSms * S::CTAS ? most : kSms * S::CTAS);
  if (most > 0x7fffffffLL) return cudaErrorInvalidValue;            // (paged_attn_counts refuses these)
  kernel<<<grid, kWarps * 32, S::SMEM, s>>>(p, part, part_rows_of(p.group));
  const cudaError_t e1 = cudaGetLastError();
  if (e1 != cudaSuccess || most <= (long long)p.c.n_seqs * p.c.n_kv_heads * slices) return e1;
  const long long heads = (long long)p.c.n_seqs * p.q.n_heads;
  // eight warps a head; two where there are more heads than such blocks at once (200 x 12 heads: 25 us against 28)
  const int rows = part_rows_of(p.group);
  if (heads <= kSms * 6) return launch_chained(paged_join_kernel<S::KT, HD, 8>, dim3((unsigned)heads), dim3(256), 0, s, true, p, (const float*)part, rows, S::WORKERS);
  return launch_chained(paged_join_kernel<S::KT, HD, 2>, dim3((unsigned)(heads < kSms * 24 ? heads : kSms * 24)), dim3(64), 0, s, true, p, (const float*)part, rows, S::WORKERS);
}

template <typename CT, int HD>
cudaError_t launch_mma(const PagedAttnParams& p, float* part, cudaStream_t s) {
  return p.q.dtype == RT_F32 ? launch_split<CT, HD, Mma<CT, HD, true>>(p, part, s) : launch_split<CT, HD, Mma<CT, HD, false>>(p, part, s);
}
template <int HD>
cudaError_t launch_simt(const PagedAttnParams& p, float* part, cudaStream_t s) {
  if (p.group == 1) return launch_split<float, HD, Simt<HD, 1>>(p, part, s);
  if (p.group == 2) return launch_split<float, HD, Simt<HD, 2>>(p, part, s);
  if (p.group <= 4) return launch_split<float, HD, Simt<HD, 4>>(p, part, s);
  return launch_split<float, HD, Simt<HD, 8>>(p, part, s);
}

}  // namespace

bool paged_attn_counts(const rt_paged_cache* c, int n_heads) {
  const long long items = (long long)c->n_kv_heads * ceil_div(n_heads / c->n_kv_heads, kRows), units = (long long)c->max_pages * (c->page_size / 16);
  return units <= 0x7fffffffLL / items / c->n_seqs && (long long)c->max_pages * c->page_size <= 1LL << 30;
}

size_t paged_attn_workspace(const rt_paged_cache* c, int n_heads) {
  const int hd = c->head_dim, rows = part_rows_of(n_heads / c->n_kv_heads);
  int workers;
  if (hd == 64) workers = c->dtype == RT_F32 ? Shape<float, 64>::WORKERS : c->dtype == RT_BF16 ? Shape<__nv_bfloat16, 64>::WORKERS : Shape<__nv_fp8_e4m3, 64>::WORKERS;
  else workers = c->dtype == RT_F32 ? Shape<float, 128>::WORKERS : c->dtype == RT_BF16 ? Shape<__nv_bfloat16, 128>::WORKERS : Shape<__nv_fp8_e4m3, 128>::WORKERS;
  return align_up((size_t)workers * 2 * slot_floats(rows, hd) * 4, 256);
}

cudaError_t paged_attn_launch(const PagedAttnParams& p, void* workspace, cudaStream_t s) {
  float* part = (float*)workspace;
  if (p.c.head_dim == 64) {
    if (p.c.dtype == RT_F32) return launch_simt<64>(p, part, s);
    return p.c.dtype == RT_BF16 ? launch_mma<__nv_bfloat16, 64>(p, part, s) : launch_mma<__nv_fp8_e4m3, 64>(p, part, s);
  }
  if (p.c.dtype == RT_F32) return launch_simt<128>(p, part, s);
  return p.c.dtype == RT_BF16 ? launch_mma<__nv_bfloat16, 128>(p, part, s) : launch_mma<__nv_fp8_e4m3, 128>(p, part, s);
}

}  // namespace rt
