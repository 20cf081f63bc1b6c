// qkRMS of queries and keys for each head and the rotation by the position, in one pass, and its backward pass.
//
// Bound: HBM traffic, if the instructions are few.  head_dim / 8 neighbouring lanes hold a row of a head; each holds the two sides a[i], b[i] of four pairs of dimensions, as
// two loads of 4 elements, so the rotation needs no exchange and the norm a few shuffles.  Dimensions that are not rotated make pairs too, which stay as
// they are.  A warp takes the heads of one row side by side: its lanes form the row's angles once, one or two each.  All products are paired fp32
// instructions.
// Measured on one B200, of 6.55 TB/s, in a run of calls: 8 x 4050 rows of 16 + 16 heads of 64 with gains, bf16 44.6 us (91 %); 30000 rows: fp32 89 %, 8 + 8 heads of 128 89 %, 16 + 4 of
// 64 77 %, 16 + 4 of 128 83 %, 4 + 4 of 64 60 % and 3 + 3 46 % in bf16 (angles and addresses of a short row), 4 + 4 in fp32 100 %.  Gradients of 8 x 4050 rows 112 us (90 %); 30000 rows of
// 8 + 8 heads of 128 104 us (90 %), 16 + 4 of 128 89 %; 12000 rows of 4 + 1 heads of 128 54 %.
#include "rt_paged.h"
#include "rt_tc.cuh"

namespace rt {
namespace {

constexpr int kThreads = 256;

// Lane c of a row holds two runs of 4 elements, which begin at first and second.  Neighbouring lanes hold neighbouring runs, so that a warp's access covers whole 32-byte
// sectors (8 elements a lane in one piece take half of every sector with each access: fp32 gradients of 26775 rows of 16 + 16 heads 141 us against 109).
// Halves: a and b of a pair are the i-th elements of the two runs; lane c holds pairs 4 c .. 4 c + 3, and what is not rotated makes pairs across its own halves.
// Neighbours: pairs lie inside the runs; lane c holds pairs 2 c, 2 c + 1 and those HD / 4 further.
struct Lane { int first, second; bool turned[2], part; };      // turned: whether pairs 0, 1 and pairs 2, 3 are rotated (rot is a multiple of 16); part: not all of a head is
template <int LPR, bool NEIGHBOURS>
__device__ __forceinline__ Lane lane_of(const RotateParams& p, int c) {
  constexpr int HD = LPR * 8;
  if (NEIGHBOURS) return {4 * c, 4 * c + HD / 2, {4 * c < p.rot, 4 * c + HD / 2 < p.rot}, p.rot < HD};
  if (8 * c < p.rot) return {4 * c, 4 * c + p.rot / 2, {true, true}, p.rot < HD};
  const int begin = p.rot / 2 + 4 * c;                                 // rot + 4 (c - rot / 8)
  return {begin, begin + (HD - p.rot) / 2, {false, false}, true};
}

// a run of four elements as it lies in memory
template <typename T> struct Run;
template <> struct Run<float> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void ones() { v = make_float4(1.f, 1.f, 1.f, 1.f); }
  __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
};
template <> struct Run<__nv_bfloat16> {
  uint2 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void ones() { v = make_uint2(0x3f803f80u, 0x3f803f80u); }
  __device__ __forceinline__ void get(float (&f)[4]) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
};
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) { *reinterpret_cast<uint2*>(p) = make_uint2(pack2(a, b), pack2(c, d)); }

// asynchronous copies of one run, or one position, of a lane's own
template <int BYTES>
__device__ __forceinline__ void copy_run(unsigned to, const void* from) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A warp's ring of passes in shared memory: a pass is AHEAD places of two runs for each lane, and one position.  Every lane reads what it copied itself, so no lane
// waits for another's, and nothing but the copies' completion is waited for.
template <typename T, int AHEAD, int STAGES> struct Ring {
  static constexpr int RUN = 4 * (int)sizeof(T), PASS = 32 * (AHEAD * 2 * RUN + 4), WARP = STAGES * PASS, BLOCK = kThreads / 32 * WARP;
  unsigned char* mine;
  unsigned at;
  int lane;
  __device__ __forceinline__ Ring(unsigned char* smem, int warp, int lane_) : mine(smem + warp * WARP), at((unsigned)__cvta_generic_to_shared(mine)), lane(lane_) {}
  __device__ __forceinline__ void copy(int stage, int u, const T* x, const T* y) const {
    copy_run<RUN>(at + stage * PASS + ((2 * u) * 32 + lane) * RUN, x);
    copy_run<RUN>(at + stage * PASS + ((2 * u + 1) * 32 + lane) * RUN, y);
  }
  __device__ __forceinline__ void copy_pos(int stage, const int* pos) const { copy_run<4>(at + stage * PASS + 64 * AHEAD * RUN + 4 * lane, pos); }
  __device__ __forceinline__ int& pos(int stage) const { return reinterpret_cast<int*>(mine + stage * PASS + 64 * AHEAD * RUN)[lane]; }
  template <typename R> __device__ __forceinline__ void get(int stage, int u, R& r) const {
    r.x.load(reinterpret_cast<const T*>(mine + stage * PASS + ((2 * u) * 32 + lane) * RUN));
    r.y.load(reinterpret_cast<const T*>(mine + stage * PASS + ((2 * u + 1) * 32 + lane) * RUN));
  }
};

// the two runs of a lane, and its pairs' sides: a[0] = sides a of pairs 0 and 1, a[1] of 2 and 3, b likewise
template <typename T> struct Runs {
  Run<T> x, y;
  __device__ __forceinline__ void load(const T* row, const Lane& l) { x.load(row + l.first); y.load(row + l.second); }
  __device__ __forceinline__ void ones() { x.ones(); y.ones(); }
};
struct Pairs { F2 a[2], b[2]; };
template <bool NEIGHBOURS, typename T>
__device__ __forceinline__ Pairs sides(const Runs<T>& r) {
  float u[4], v[4];
  r.x.get(u);
  r.y.get(v);
  if (NEIGHBOURS) return {{f2(u[0], u[2]), f2(v[0], v[2])}, {f2(u[1], u[3]), f2(v[1], v[3])}};
  return {{f2(u[0], u[1]), f2(u[2], u[3])}, {f2(v[0], v[1]), f2(v[2], v[3])}};
}
template <bool NEIGHBOURS, typename T>
__device__ __forceinline__ void store_sides(T* row, const Lane& l, const Pairs& x) {
  float a[4], b[4];
  split(x.a[0], a[0], a[1]); split(x.a[1], a[2], a[3]); split(x.b[0], b[0], b[1]); split(x.b[1], b[2], b[3]);
  if (NEIGHBOURS) {
    store4(row + l.first, a[0], b[0], a[1], b[1]);
    store4(row + l.second, a[2], b[2], a[3], b[3]);
  } else {
    store4(row + l.first, a[0], a[1], a[2], a[3]);
    store4(row + l.second, b[0], b[1], b[2], b[3]);
  }
}
__device__ __forceinline__ float dot(const Pairs& x, const Pairs& y) {        // of this lane's eight elements
  F2 s = mul(x.a[0], y.a[0]);
  s = fma(x.a[1], y.a[1], s);
  s = fma(x.b[0], y.b[0], s);
  s = fma(x.b[1], y.b[1], s);
  float a, b;
  split(s, a, b);
  return a + b;
}
__device__ __forceinline__ Pairs times(const Pairs& x, const Pairs& y) { return {{mul(x.a[0], y.a[0]), mul(x.a[1], y.a[1])}, {mul(x.b[0], y.b[0]), mul(x.b[1], y.b[1])}}; }
__device__ __forceinline__ Pairs times(const Pairs& x, float y) {
  const F2 f = f2(y, y);
  return {{mul(x.a[0], f), mul(x.a[1], f)}, {mul(x.b[0], f), mul(x.b[1], f)}};
}
__device__ __forceinline__ void add_to(Pairs& s, const Pairs& x, const Pairs& y) {       // s += x y
#pragma unroll
  for (int i = 0; i < 2; ++i) { s.a[i] = fma(x.a[i], y.a[i], s.a[i]); s.b[i] = fma(x.b[i], y.b[i], s.b[i]); }
}

// A row's angles as a lane needs them: cos and sin of its pairs 0, 1 and 2, 3.  Pairs that are not rotated stay as they are: an angle of zero would carry an
// infinity or a NaN into the pair's other side.
struct Turn {
  F2 c[2], s[2], ns[2];
  __device__ __forceinline__ static Pairs turned(const Lane& l, const Pairs& x, const F2 (&c)[2], const F2 (&s)[2], const F2 (&ns)[2]) {
    Pairs y = {{fma(x.a[0], c[0], mul(x.b[0], ns[0])), fma(x.a[1], c[1], mul(x.b[1], ns[1]))}, {fma(x.a[0], s[0], mul(x.b[0], c[0])), fma(x.a[1], s[1], mul(x.b[1], c[1]))}};
    if (l.part) {                                                      // (the same for all lanes: heads that are rotated whole go past the selections; 16 + 4 heads, 7800 rows: 17.8 us, 18.3 with them)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (!l.turned[i]) { y.a[i] = x.a[i]; y.b[i] = x.b[i]; }
    }
    return y;
  }
  __device__ __forceinline__ Pairs forward(const Lane& l, const Pairs& x) const { return turned(l, x, c, s, ns); }
  __device__ __forceinline__ Pairs back(const Lane& l, const Pairs& x) const { return turned(l, x, c, ns, s); }
};

// Pair n's angle is formed by lane n % 32 of the warp and handed to the lanes that hold the pair through 512 bytes of shared memory of the warp's own (two loads a lane,
// where shuffles would be 8 or 16).  Turns are multiplied as 64-bit fractions, whole turns falling off at the top: far positions keep their angles (the turns of one position
// come from fp64, so they are off by 2^-53 of all that has been turned, as a product in fp64 would be; 2^-33 turns from the rounding to 32 bits, 2^-24 of itself in fp32), and it
// takes two integer products where fp64 would take six slow instructions.
struct Angles { float cos[64], sin[64]; };
template <int LPR> struct Turns {                                      // of this lane's pairs
  unsigned long long per[LPR / 8];
  __device__ __forceinline__ Turns(const RotateParams& p, int lane) {
#pragma unroll
    for (int k = 0; k < LPR / 8; ++k) per[k] = p.turns[lane + 32 * k];      // (zero where there is no pair)
  }
  // EXACT: to fp32's rounding; otherwise to 2^-20, for rows that are rounded to bf16 (2^-9): 2^-21.2 of __cosf and 2^-21.7 of an angle near a half turn in fp32
  template <bool EXACT>
  __device__ __forceinline__ void make(int pos, int lane, Angles& buf) const {
#pragma unroll
    for (int k = 0; k < LPR / 8; ++k) {
      const int half_turns = (int)((per[k] * (unsigned)pos + 0x80000000u) >> 32);      // in 2^-31
      float co, si;
      if (EXACT) sincospif((float)half_turns * 4.656612873077392578125e-10f, &si, &co);
      else __sincosf((float)half_turns * (4.656612873077392578125e-10f * 3.14159265358979f), &si, &co);
      buf.cos[lane + 32 * k] = co;
      buf.sin[lane + 32 * k] = si;
    }
  }
  template <bool NEIGHBOURS>
  __device__ __forceinline__ static Turn of(const Angles& buf, int lane) {
    float4 c, s;
    if (NEIGHBOURS) {
      const float2 c0 = reinterpret_cast<const float2*>(buf.cos)[lane % LPR], c1 = reinterpret_cast<const float2*>(buf.cos)[lane % LPR + LPR];
      const float2 s0 = reinterpret_cast<const float2*>(buf.sin)[lane % LPR], s1 = reinterpret_cast<const float2*>(buf.sin)[lane % LPR + LPR];
      c = make_float4(c0.x, c0.y, c1.x, c1.y);
      s = make_float4(s0.x, s0.y, s1.x, s1.y);
    } else {
      c = reinterpret_cast<const float4*>(buf.cos)[lane % LPR];
      s = reinterpret_cast<const float4*>(buf.sin)[lane % LPR];
    }
    return {{f2(c.x, c.y), f2(c.z, c.w)}, {f2(s.x, s.y), f2(s.z, s.w)}, {f2(-s.x, -s.y), f2(-s.z, -s.w)}};
  }
};

// Forward.  The heads of a row, queries' first, then keys', are a line; a warp has AHEAD * 32 / LPR places and goes from row to row.
//   kOneKind: block row y of the grid takes the y-th part of the line, all queries or all keys, and no place is empty (one address and constants)
//   kMixed: the same, whatever the parts hold
//   kSideBySide: the line takes half of the places or less, and rows_per rows lie in them side by side, so that no lane idles and a pass moves bytes enough
// Either way a pass is all that the warp does for its row: its gains stay in registers, its angles are formed once.
enum Places { kOneKind, kMixed, kSideBySide };
template <typename T, Places PLACES> constexpr int kMost = sizeof(T) == 2 && PLACES == kMixed ? 5 : 4;      // places of a lane, by registers
constexpr int kSide = 4;                                                                                     // rows side by side
// Blocks of an SM, and passes of a warp's ring.  Sixteen warps with one pass on its way each are faster than 24, or than two passes (16 + 16 heads of 64, bf16, two
// passes a row: 45.7 us; 24 warps 46.4, 32 47.0; with two on their way 45.9, 49, 55; with the pass in registers instead of the ring 51).  Small passes want two (fp32, 4 + 4 heads: 18.2 us against 21.7).
constexpr int kBlocks = 2;
template <int AHEAD> constexpr int kStages = AHEAD <= 2 ? 3 : 2;
// Backward: two places a lane, one pass on its way (16 + 16 heads of 64, bf16: 111 us; three places 119, four 114; with two passes on their way 120).
constexpr int kBackMost = 2, kBackStages = 2;

// The places of a lane: u is a head of row at_row[u] of the pass, `off` elements into the row of the queries or keys (a place without one repeats the last one's, for
// the shuffles).
template <int LPR, int AHEAD, Places PLACES> struct Line {
  static constexpr bool ONE = PLACES == kOneKind, SIDE = PLACES == kSideBySide;
  static constexpr int HPW = 32 / LPR, HD = LPR * 8;
  int at_row[AHEAD], off[AHEAD];
  bool in_use[AHEAD], is_q[AHEAD], part_q;
  unsigned rows;
  __device__ __forceinline__ Line(const RotateParams& p, int parts_q, int rows_per, int lane) : part_q((int)blockIdx.y < parts_q), rows(p.rows) {
    const int heads = p.n_heads + p.n_kv;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int mine = lane / LPR + u * HPW;
      at_row[u] = 0;
      if (ONE) {
        in_use[u] = true;
        is_q[u] = part_q;
        off[u] = ((part_q ? blockIdx.y : blockIdx.y - parts_q) * AHEAD * HPW + lane / LPR) * HD + u * HPW * HD;
      } else {
        const int place = (SIDE ? 0 : blockIdx.y * AHEAD * HPW) + mine, places = SIDE ? rows_per * heads : heads;
        in_use[u] = place < places;
        const int at = min(place, places - 1), hh = SIDE ? at % heads : at;
        if (SIDE) at_row[u] = at / heads;
        is_q[u] = hh < p.n_heads;
        off[u] = (is_q[u] ? hh : hh - p.n_heads) * HD;
      }
    }
  }
  // the place's head in row r (of the pass that begins with row r)
  template <typename E>
  __device__ __forceinline__ E* head(const void* q, const void* k, size_t q_stride, size_t k_stride, unsigned r, int u) const {
    if (SIDE) return (E*)(is_q[u] ? q : k) + (min(r + at_row[u], rows - 1) * (is_q[u] ? q_stride : k_stride) + off[u]);
    E *to_q = (E*)q + r * q_stride, *to_k = (E*)k + r * k_stride;
    return ONE ? (part_q ? to_q : to_k) + off[0] + u * HPW * HD : (is_q[u] ? to_q : to_k) + off[u];
  }
  template <typename T>
  __device__ __forceinline__ void gains(const RotateParams& p, const Lane& l, Runs<T> (&gr)[AHEAD]) const {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const T* g = (const T*)(is_q[u] ? p.g_q : p.g_k);
      if (p.norm && g) gr[u].load(g + off[u], l);
      else gr[u].ones();
    }
  }
};

template <typename T, int LPR, bool NEIGHBOURS, int AHEAD, Places PLACES>
__global__ void __launch_bounds__(kThreads, kBlocks) rotate_kernel(const __grid_constant__ RotateParams p, int parts_q, int rows_per) {
  constexpr bool SIDE = PLACES == kSideBySide;
  constexpr int HD = LPR * 8, STAGES = kStages<AHEAD>;
  __shared__ __align__(16) Angles bufs[kThreads / 32][SIDE ? kSide : 1];
  Angles* buf = bufs[threadIdx.x >> 5];
  const int lane = threadIdx.x & 31;
  const Lane l = lane_of<LPR, NEIGHBOURS>(p, lane % LPR);
  const unsigned rows = p.rows, step = gridDim.x * (kThreads / 32) * (SIDE ? rows_per : 1);
  unsigned row = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * (SIDE ? rows_per : 1);
  if (row >= rows) return;
  const Line<LPR, AHEAD, PLACES> line(p, parts_q, rows_per, lane);
  const bool gains = p.norm && (p.g_q || p.g_k);
  Runs<T> gr[AHEAD];
  line.gains(p, l, gr);
  extern __shared__ __align__(16) unsigned char smem[];
  const Ring<T, AHEAD, STAGES> ring(smem, threadIdx.x >> 5, lane);
  unsigned from_row = row;
  auto fetch = [&](int stage) {
    if (from_row < rows) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const T* from = line.template head<T>(p.q, p.k, p.q_stride, p.k_stride, from_row, u);
        ring.copy(stage, u, from + l.first, from + l.second);
      }
      if (!SIDE) ring.copy_pos(stage, p.pos + from_row);
      else if (lane < rows_per && from_row + lane < rows) ring.copy_pos(stage, p.pos + from_row + lane);      // lane i: row i of a pass
      else ring.pos(stage) = -1;
      from_row += step;
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) fetch(i);
  const Turns<LPR> turns(p, lane);
  for (int stage = 0; row < rows; row += step, stage = stage + 1 == STAGES ? 0 : stage + 1) {
    copy_wait<STAGES - 2>();
    fetch(stage == 0 ? STAGES - 1 : stage - 1);
    const int pos = ring.pos(stage);
    if (!SIDE && pos < 0) continue;
    Runs<T> x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ring.get(stage, u, x[u]);
    __syncwarp();                                                      // (the angles before are read)
    if (SIDE) {
      for (int i = 0; i < rows_per; ++i) turns.template make<sizeof(T) == 4>(__shfl_sync(0xffffffffu, pos, i), lane, buf[i]);
    } else {
      turns.template make<sizeof(T) == 4>(pos, lane, buf[0]);
    }
    __syncwarp();
    Turn turn;
    if (!SIDE) turn = Turns<LPR>::template of<NEIGHBOURS>(buf[0], lane);
    float r[AHEAD];
    if (p.norm) {                                                      // the heads' sums side by side: a sum alone would wait for each of its shuffles
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const Pairs y = sides<NEIGHBOURS>(x[u]);
        r[u] = dot(y, y);
      }
#pragma unroll
      for (int o = LPR / 2; o; o >>= 1)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) r[u] += __shfl_xor_sync(0xffffffffu, r[u], o);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) r[u] = rsqrtf(r[u] * (1.0f / HD) + p.eps);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      Pairs y = sides<NEIGHBOURS>(x[u]);
      if (p.norm) y = gains ? times(y, times(sides<NEIGHBOURS>(gr[u]), r[u])) : times(y, r[u]);
      if (SIDE) turn = Turns<LPR>::template of<NEIGHBOURS>(buf[line.at_row[u]], lane);
      y = turn.forward(l, y);
      const bool used = !SIDE || __shfl_sync(0xffffffffu, pos, line.at_row[u]) >= 0;
      if (used && line.in_use[u]) store_sides<NEIGHBOURS>(line.template head<T>(p.q_out, p.k_out, p.qo_stride, p.ko_stride, row, u), l, y);
    }
  }
}

// Backward, the same way: w = the output's gradient turned back, y = x / rms;  dx = (w g - y mean(w g y)) / rms,  dg = sum over the rows of w y.  Both of a head's sums
// (x^2 and w g x) go through the shuffles together.  A lane adds up dg of its places over its rows; the block's warps are added up at the end and go to
// part[x][heads * HD], which sum_parts_kernel adds up in the order of x.
template <typename T, int LPR, bool NEIGHBOURS, int AHEAD, Places PLACES>
__global__ void __launch_bounds__(kThreads, kBlocks) rotate_backward_kernel(const __grid_constant__ RotateParams p, int parts_q, int rows_per, float* part) {
  constexpr bool SIDE = PLACES == kSideBySide;
  constexpr int HPW = 32 / LPR, HD = LPR * 8, STAGES = kBackStages, WARPS = kThreads / 32;
  __shared__ __align__(16) Angles bufs[WARPS][SIDE ? kSide : 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, heads = p.n_heads + p.n_kv;
  Angles* buf = bufs[warp];
  const Lane l = lane_of<LPR, NEIGHBOURS>(p, lane % LPR);
  const unsigned rows = p.rows, step = gridDim.x * WARPS * (SIDE ? rows_per : 1);
  unsigned row = (blockIdx.x * WARPS + warp) * (SIDE ? rows_per : 1), from_row = row;
  const Line<LPR, AHEAD, PLACES> line(p, parts_q, rows_per, lane);
  const size_t dq_stride = (size_t)p.n_heads * HD, dk_stride = (size_t)p.n_kv * HD;
  Runs<T> gr[AHEAD];
  line.gains(p, l, gr);
  extern __shared__ __align__(16) unsigned char smem[];
  const Ring<T, AHEAD, STAGES> xs(smem, warp, lane);
  const Ring<float, AHEAD, STAGES> ds(smem + Ring<T, AHEAD, STAGES>::BLOCK, warp, lane);
  auto fetch = [&](int stage) {
    if (from_row < rows) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const T* x = line.template head<T>(p.q, p.k, p.q_stride, p.k_stride, from_row, u);
        const float* d = line.template head<float>(p.dq_out, p.dk_out, dq_stride, dk_stride, from_row, u);
        xs.copy(stage, u, x + l.first, x + l.second);
        ds.copy(stage, u, d + l.first, d + l.second);
      }
      if (!SIDE) xs.copy_pos(stage, p.pos + from_row);
      else if (lane < rows_per && from_row + lane < rows) xs.copy_pos(stage, p.pos + from_row + lane);
      else xs.pos(stage) = -1;
      from_row += step;
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) fetch(i);
  const Turns<LPR> turns(p, lane);
  const F2 zero = f2(0.f, 0.f);
  Pairs dg[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) dg[u] = {{zero, zero}, {zero, zero}};
  for (int stage = 0; row < rows; row += step, stage = stage + 1 == STAGES ? 0 : stage + 1) {
    copy_wait<STAGES - 2>();
    fetch(stage == 0 ? STAGES - 1 : stage - 1);
    const int pos = xs.pos(stage);
    if (!SIDE && pos < 0) continue;
    __syncwarp();                                                      // (the angles before are read)
    if (SIDE) {
      for (int i = 0; i < rows_per; ++i) turns.template make<true>(__shfl_sync(0xffffffffu, pos, i), lane, buf[i]);
    } else {
      turns.template make<true>(pos, lane, buf[0]);
    }
    __syncwarp();
    Turn turn;
    if (!SIDE) turn = Turns<LPR>::template of<NEIGHBOURS>(buf[0], lane);
    Runs<T> x[AHEAD];
    Pairs w[AHEAD];
    float xx[AHEAD], wx[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      Runs<float> d;
      xs.get(stage, u, x[u]);
      ds.get(stage, u, d);
      if (SIDE) turn = Turns<LPR>::template of<NEIGHBOURS>(buf[line.at_row[u]], lane);
      w[u] = turn.back(l, sides<NEIGHBOURS>(d));
      if (p.norm) {
        const Pairs y = sides<NEIGHBOURS>(x[u]);
        xx[u] = dot(y, y);
        wx[u] = dot(times(w[u], sides<NEIGHBOURS>(gr[u])), y);
      }
    }
    if (p.norm) {
#pragma unroll
      for (int o = LPR / 2; o; o >>= 1)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          xx[u] += __shfl_xor_sync(0xffffffffu, xx[u], o);
          wx[u] += __shfl_xor_sync(0xffffffffu, wx[u], o);
        }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const bool used = !SIDE || __shfl_sync(0xffffffffu, pos, line.at_row[u]) >= 0;
      if (!used || !line.in_use[u]) continue;
      if (p.norm) {
        const float r = rsqrtf(xx[u] * (1.0f / HD) + p.eps), mean = -(wx[u] * r) * (1.0f / HD);
        const Pairs y = times(sides<NEIGHBOURS>(x[u]), r), m = {{f2(mean, mean), f2(mean, mean)}, {f2(mean, mean), f2(mean, mean)}};
        add_to(dg[u], w[u], y);
        w[u] = times(w[u], sides<NEIGHBOURS>(gr[u]));
        add_to(w[u], y, m);
        w[u] = times(w[u], r);
      }
      store_sides<NEIGHBOURS>(line.template head<float>(p.dq, p.dk, dq_stride, dk_stride, row, u), l, w[u]);
    }
  }
  if (!part) return;
  copy_wait<0>();
  __syncthreads();                                                     // (the ring is used up: it holds the warps' sums)
  float* red = reinterpret_cast<float*>(smem);
  constexpr int PLACE_FLOATS = AHEAD * HPW * HD;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) store_sides<NEIGHBOURS>(red + warp * PLACE_FLOATS + (u * HPW + lane / LPR) * HD, l, dg[u]);
  __syncthreads();
  const int first = SIDE ? 0 : (int)blockIdx.y * AHEAD * HPW, last = SIDE ? heads : min(heads, first + AHEAD * HPW);
  for (int i = threadIdx.x; i < (last - first) * HD; i += kThreads) {
    float a = 0.f;
    for (int side = 0; side < (SIDE ? rows_per : 1); ++side)
#pragma unroll
      for (int w = 0; w < WARPS; ++w) a += red[w * PLACE_FLOATS + side * heads * HD + i];
    part[(size_t)blockIdx.x * heads * HD + first * HD + i] = a;
  }
}

__global__ void __launch_bounds__(kThreads) sum_parts_kernel(const float* part, int parts, int nq, int n, float* dg_q, float* dg_k) {
  __shared__ float red[8][32];
  const int i = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float a = 0.f;
  if (i < n) for (int x = w; x < parts; x += 8) a += part[(size_t)x * n + i];
  red[w][threadIdx.x & 31] = a;
  __syncthreads();
  if (w == 0 && i < n) {
#pragma unroll
    for (int k = 1; k < 8; ++k) a += red[k][threadIdx.x];
    if (i < nq) { if (dg_q) dg_q[i] = a; }
    else if (dg_k) dg_k[i - nq] = a;
  }
}

// Blocks of the backward pass along the rows, at most: two rows for each warp or more.
int backward_blocks(int rows) { return (int)min(148LL * kBlocks, ((long long)rows + 15) / 16); }

template <typename... P, typename... A>
cudaError_t launch_with_smem(void (*kernel)(P...), dim3 grid, int smem, cudaStream_t s, const A&... args) {
  if (const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem); e != cudaSuccess) return e;
  kernel<<<grid, kThreads, smem, s>>>(args...);
  return cudaGetLastError();
}
template <typename T, int LPR, bool NEIGHBOURS, Places PLACES>
cudaError_t start(const RotateParams& p, int ahead, int parts_q, int parts, int rows_per, cudaStream_t s) {
  const long long warps = ((long long)p.rows + rows_per - 1) / rows_per, blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  // as many blocks as the GPU holds at once: a warp goes on to its next row with that row's loads under way
  const dim3 grid((unsigned)min(blocks, (long long)max(1, 148 * kBlocks / parts)), parts);
  auto go = [&](auto* kernel, int smem) { return launch_with_smem(kernel, grid, smem, s, p, parts_q, rows_per); };
  constexpr int MOST = PLACES == kSideBySide ? 2 : kMost<T, PLACES>;
  if constexpr (MOST >= 5) if (ahead == 5) return go(rotate_kernel<T, LPR, NEIGHBOURS, 5, PLACES>, Ring<T, 5, kStages<5>>::BLOCK);
  if constexpr (MOST >= 4) if (ahead == 4) return go(rotate_kernel<T, LPR, NEIGHBOURS, 4, PLACES>, Ring<T, 4, kStages<4>>::BLOCK);
  if constexpr (MOST >= 3) if (ahead == 3) return go(rotate_kernel<T, LPR, NEIGHBOURS, 3, PLACES>, Ring<T, 3, kStages<3>>::BLOCK);
  if constexpr (PLACES != kSideBySide) if (ahead == 1) return go(rotate_kernel<T, LPR, NEIGHBOURS, 1, PLACES>, Ring<T, 1, kStages<1>>::BLOCK);
  return go(rotate_kernel<T, LPR, NEIGHBOURS, 2, PLACES>, Ring<T, 2, kStages<2>>::BLOCK);
}
template <typename T, int LPR, bool NEIGHBOURS>
cudaError_t forward_launch(const RotateParams& p, cudaStream_t s) {
  constexpr int HPW = 32 / LPR;
  const int heads = p.n_heads + p.n_kv, groups = ceil_div(heads, HPW);
  const long long blocks = ((long long)p.rows + kThreads / 32 - 1) / (kThreads / 32);
  const bool large = blocks >= 2 * 148;
  // (1 + 1 heads, 30000 rows: 6.4 us against 29 with queries and keys in warps of their own; 2 + 2 heads 9.5 against 29)
  if (heads <= HPW && large) return start<T, LPR, NEIGHBOURS, kSideBySide>(p, 2, 0, 1, min(kSide, 2 * HPW / heads), s);
  // Places of a warp, by the cost of a row: about 8 for a pass and 4 for a place of it, or 5 if queries and keys share passes (their addresses take more instructions).
  // 16 + 16 heads of 64, bf16: 44 us as one kind, 52 mixed; 16 + 4: 46 mixed, 56 in two launches of one kind each; 16 + 4 of 128: 48 in two, 52 mixed.  In small calls as few places as
  // leave two blocks for each SM.
  const int most = ceil_div(groups, (int)min((long long)groups, max(1LL, 148 * 2 / blocks)));
  int mixed = 1;
  auto mixed_cost = [&](int a) { return ceil_div(groups, a) * (5 * a + 8); };
  for (int a = 2; a <= min(most, kMost<T, kMixed>); ++a) if (mixed_cost(a) <= mixed_cost(mixed)) mixed = a;
  if (p.n_heads % HPW == 0 && p.n_kv % HPW == 0) {
    const int gq = p.n_heads / HPW, gk = p.n_kv / HPW;
    int aq = 1, ak = 1, both = 1;
    for (int a = 2; a <= min(most, kMost<T, kOneKind>); ++a) {
      if (gq % a == 0) aq = a;
      if (gk % a == 0) ak = a;
      if (gq % a == 0 && gk % a == 0) both = a;
    }
    const int one = groups / both * (4 * both + 8), two = large && gk ? gq / aq * (4 * aq + 8) + gk / ak * (4 * ak + 8) : INT32_MAX;
    if (min(one, two) <= mixed_cost(mixed)) {
      if (one <= two) return start<T, LPR, NEIGHBOURS, kOneKind>(p, both, gq / both, groups / both, 1, s);
      const cudaError_t e = start<T, LPR, NEIGHBOURS, kOneKind>(p, aq, gq / aq, gq / aq, 1, s);
      return e != cudaSuccess ? e : start<T, LPR, NEIGHBOURS, kOneKind>(p, ak, 0, gk / ak, 1, s);
    }
  }
  return start<T, LPR, NEIGHBOURS, kMixed>(p, mixed, 0, ceil_div(groups, mixed), 1, s);
}
template <typename T, int LPR>
cudaError_t forward(const RotateParams& p, cudaStream_t s) {
  return p.neighbours ? forward_launch<T, LPR, true>(p, s) : forward_launch<T, LPR, false>(p, s);
}

template <typename T, int LPR, bool NEIGHBOURS, Places PLACES>
cudaError_t start_backward(const RotateParams& p, int ahead, int parts_q, int parts, int blocks, int rows_per, float* part, cudaStream_t s) {
  auto go = [&](auto* kernel, int smem) { return launch_with_smem(kernel, dim3(blocks, parts), smem, s, p, parts_q, rows_per, part); };
  if constexpr (PLACES != kSideBySide)
    if (ahead == 1) return go(rotate_backward_kernel<T, LPR, NEIGHBOURS, 1, PLACES>, Ring<T, 1, kBackStages>::BLOCK + Ring<float, 1, kBackStages>::BLOCK);
  return go(rotate_backward_kernel<T, LPR, NEIGHBOURS, 2, PLACES>, Ring<T, 2, kBackStages>::BLOCK + Ring<float, 2, kBackStages>::BLOCK);
}
// -> the blocks along the rows, whose partial sums there are
template <typename T, int LPR, bool NEIGHBOURS>
cudaError_t backward(const RotateParams& p, float* part, int* blocks, cudaStream_t s) {
  constexpr int HPW = 32 / LPR;
  const int heads = p.n_heads + p.n_kv, groups = ceil_div(heads, HPW), all = backward_blocks(p.rows);
  const bool large = all == 148 * kBlocks;
  // (100000 rows of 1 + 1 heads, fp32: 29 us against 55 with queries and keys in places of their own)
  if (heads <= HPW && large) {
    const int side = min(kSide, 2 * HPW / heads);
    *blocks = min(all, ceil_div(ceil_div(p.rows, side), kThreads / 32));
    return start_backward<T, LPR, NEIGHBOURS, kSideBySide>(p, 2, 0, 1, *blocks, side, part, s);
  }
  // two places of a lane, by the passes that they save; one in small calls.  (4 + 4 heads of 64, bf16: 52 us mixed, 65 with a pass for each kind)
  const int most = min(kBackMost, ceil_div(groups, min(groups, max(1, 148 * kBlocks / all))));
  const int mixed = most == 2 && ceil_div(groups, 2) * 16 <= groups * 12 ? 2 : 1;
  const bool whole = p.n_heads % HPW == 0 && p.n_kv % HPW == 0;
  if (whole && p.n_heads / HPW % mixed == 0 && p.n_kv / HPW % mixed == 0) {
    *blocks = min(all, max(1, 148 * kBlocks * mixed / groups));
    return start_backward<T, LPR, NEIGHBOURS, kOneKind>(p, mixed, p.n_heads / HPW / mixed, groups / mixed, *blocks, 1, part, s);
  }
  *blocks = min(all, max(1, 148 * kBlocks / ceil_div(groups, mixed)));
  return start_backward<T, LPR, NEIGHBOURS, kMixed>(p, mixed, 0, ceil_div(groups, mixed), *blocks, 1, part, s);
}
template <typename T, int LPR>
cudaError_t backward(const RotateParams& p, float* part, int* blocks, cudaStream_t s) {
  return p.neighbours ? backward<T, LPR, true>(p, part, blocks, s) : backward<T, LPR, false>(p, part, blocks, s);
}

}  // namespace

size_t rotate_backward_workspace(int heads, int hd, int rows) { return align_up((size_t)max(1, backward_blocks(rows)) * heads * hd * 4, 256); }

cudaError_t rotate_launch(int dtype, const RotateParams& p, cudaStream_t s) {
  if (dtype == RT_BF16) return p.hd == 64 ? forward<__nv_bfloat16, 8>(p, s) : forward<__nv_bfloat16, 16>(p, s);
  return p.hd == 64 ? forward<float, 8>(p, s) : forward<float, 16>(p, s);
}

cudaError_t rotate_backward_launch(int dtype, const RotateParams& p, void* workspace, cudaStream_t s) {
  const int heads = p.n_heads + p.n_kv;
  int blocks = 0;
  float* part = (p.dg_q || p.dg_k) ? (float*)workspace : nullptr;
  if (p.rows > 0) {
    cudaError_t e;
    if (dtype == RT_BF16) e = p.hd == 64 ? backward<__nv_bfloat16, 8>(p, part, &blocks, s) : backward<__nv_bfloat16, 16>(p, part, &blocks, s);
    else e = p.hd == 64 ? backward<float, 8>(p, part, &blocks, s) : backward<float, 16>(p, part, &blocks, s);
    if (e != cudaSuccess) return e;
  }
  if (!part) return cudaSuccess;
  return launch_chained(sum_parts_kernel, dim3(ceil_div(heads * p.hd, 32)), dim3(kThreads), 0, s, p.rows > 0, (const float*)part, blocks,
                        p.n_heads * p.hd, heads * p.hd, p.dg_q, p.dg_k);
}

}  // namespace rt
