// qkRMS of queries and keys for each head and the rotation by the position, in one pass, and its backward pass.
//
// Bound: HBM traffic.  head_dim / 8 neighbouring lanes hold a row of a head; each holds the two sides a[i], b[i] of four pairs of dimensions, as
// two loads of 4 elements, so the rotation needs no exchange and the norm a few shuffles.  Dimensions that are not rotated make pairs too, with an angle
// of zero.  A warp takes the heads of one row side by side and one after the other: its lanes form the row's angles once, one or two each.  All products are paired fp32
// instructions: at 6.5 TB/s an SM has 1370 issue slots for a row of 16 + 16 heads in bf16, and the pass takes 930.
// Measured on one B200, of 6.55 TB/s: 8 x 4000 rows of 16 + 16 heads of 64 with gains, bf16 50 us (81 %), fp32 90 %; gradients 111 us (92 %).  Heads of 128, whose rows carry twice the
// angles for as many bytes, 65 and 62 %; 16 query and 4 key heads 53 and 67 %.
#include "rt_paged.h"

namespace rt {
namespace {

constexpr int kThreads = 256;

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Lane c of a row holds pairs 4 c .. 4 c + 3.  Its two runs of 4 elements begin at first and second; a and b of a pair are the i-th elements of the
// two runs (halves, where rotated), or neighbours inside a run.
struct Lane { int first, second; };
template <bool NEIGHBOURS>
__device__ __forceinline__ Lane lane_of(const RotateParams& p, int c) {
  if (NEIGHBOURS || 8 * c >= p.rot) return {8 * c, 8 * c + 4};
  return {4 * c, 4 * c + p.rot / 2};
}

// a run of four elements as it lies in memory
template <typename T> struct Run;
template <> struct Run<float> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
};
template <> struct Run<__nv_bfloat16> {
  uint2 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float (&f)[4]) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
};
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) { *reinterpret_cast<uint2*>(p) = make_uint2(pack2(a, b), pack2(c, d)); }

// the two runs of a lane, and its pairs' sides: a[0] = sides a of pairs 0 and 1, a[1] of 2 and 3, b likewise
template <typename T> struct Runs {
  Run<T> x, y;
  __device__ __forceinline__ void load(const T* row, const Lane& l) { x.load(row + l.first); y.load(row + l.second); }
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

// A row's angles as a lane needs them: cos and sin of its pairs 0, 1 and 2, 3.
struct Turn {
  F2 c[2], s[2], ns[2];
  __device__ __forceinline__ Pairs forward(const Pairs& x) const {
    return {{fma(x.a[0], c[0], mul(x.b[0], ns[0])), fma(x.a[1], c[1], mul(x.b[1], ns[1]))}, {fma(x.a[0], s[0], mul(x.b[0], c[0])), fma(x.a[1], s[1], mul(x.b[1], c[1]))}};
  }
  __device__ __forceinline__ Pairs back(const Pairs& x) const {
    return {{fma(x.a[0], c[0], mul(x.b[0], s[0])), fma(x.a[1], c[1], mul(x.b[1], s[1]))}, {fma(x.a[0], ns[0], mul(x.b[0], c[0])), fma(x.a[1], ns[1], mul(x.b[1], c[1]))}};
  }
};

// Pair n's angle is formed by lane n % 32 of the warp and handed to the lanes that hold the pair through 512 bytes of shared memory of the warp's own (two loads a lane,
// where shuffles would be 8 or 16); the turns are reduced in 64 bits, so that far positions keep their angles.  All lanes of the warp call.
struct Angles { float cos[64], sin[64]; };
template <int LPR>
__device__ __forceinline__ Turn angles(const RotateParams& p, int pos, int lane, Angles& buf) {
  __syncwarp();                                                        // (what was there is read)
#pragma unroll
  for (int k = 0; k < LPR / 8; ++k) {
    float co = 1.f, si = 0.f;
    const int n = lane + 32 * k;
    if (2 * n < p.rot) {
      const double t = (double)pos * p.turns[n];
      sincospif((float)(2.0 * (t - rint(t))), &si, &co);
    }
    buf.cos[n] = co;
    buf.sin[n] = si;
  }
  __syncwarp();
  const float4 c = reinterpret_cast<const float4*>(buf.cos)[lane % LPR], s = reinterpret_cast<const float4*>(buf.sin)[lane % LPR];
  return {{f2(c.x, c.y), f2(c.z, c.w)}, {f2(s.x, s.y), f2(s.z, s.w)}, {f2(-s.x, -s.y), f2(-s.z, -s.w)}};
}

// The heads of a launch in block rows of the grid: heads_per of the queries' heads each in the first y_q of them, then heads_per of the keys' heads each.  All heads
// in one block row where there are rows enough to fill the GPU, some of them in small calls, where a warp's chain of heads would be the call's time.
struct Part { bool is_q; int first, last; };
__device__ __forceinline__ Part part_of(const RotateParams& p, int y, int heads_per, int y_q) {
  const bool is_q = y < y_q;
  const int first = (is_q ? y : y - y_q) * heads_per;
  return {is_q, first, min(is_q ? p.n_heads : p.n_kv, first + heads_per)};
}

constexpr int kBlocks = 3;      // of an SM, by registers
// AHEAD: heads of a lane in flight, and as many on their way.  WHOLE: every block row's heads fill whole batches of them (otherwise lanes without a head
// repeat the last one's, for the shuffles).
template <typename T, int LPR, bool NEIGHBOURS, int AHEAD, bool WHOLE>
__global__ void __launch_bounds__(kThreads, kBlocks) rotate_kernel(const __grid_constant__ RotateParams p, int heads_per, int y_q) {
  constexpr int HPW = 32 / LPR, HD = LPR * 8, BATCH = HPW * AHEAD;
  __shared__ __align__(16) Angles bufs[kThreads / 32];
  Angles& buf = bufs[threadIdx.x >> 5];
  const int lane = threadIdx.x & 31, hl = lane / LPR;
  const Lane l = lane_of<NEIGHBOURS>(p, lane % LPR);
  const Part part = part_of(p, blockIdx.y, heads_per, y_q);
  const int first = part.first, last = part.last;
  const T* in = (const T*)(part.is_q ? p.q : p.k);
  T* out = (T*)(part.is_q ? p.q_out : p.k_out);
  const T* g = p.norm ? (const T*)(part.is_q ? p.g_q : p.g_k) : nullptr;
  const size_t stride = part.is_q ? p.q_stride : p.k_stride, out_stride = part.is_q ? p.qo_stride : p.ko_stride;
  const unsigned warps = gridDim.x * (kThreads / 32), rows = p.rows;
  unsigned row = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (row >= rows) return;
  // the u-th head of a batch that begins at h0, from the row's start (its elements are read and written once each, so q_out may be q)
  auto at = [&](int h0, int u) { return WHOLE ? (h0 + hl) * HD + u * HPW * HD : min(h0 + hl + u * HPW, last - 1) * HD; };
  Runs<T> x[AHEAD], next[AHEAD];
  auto load = [&](Runs<T> (&to)[AHEAD], unsigned r, int h0) {
    const T* from = in + r * stride;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) to[u].load(from + at(h0, u), l);
  };
  int pos = __ldg(p.pos + row), next_pos = 0, h0 = first;
  const bool one = first + BATCH >= last;
  Runs<T> gr[AHEAD];
  if (p.norm && g && one) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) gr[u].load(g + at(first, u), l);
  }
  load(x, row, h0);
  Turn turn = angles<LPR>(p, pos, lane, buf);
  while (true) {
    const bool row_ends = h0 + BATCH >= last;
    const unsigned nr = row_ends ? row + warps : row;
    const int nh = row_ends ? first : h0 + BATCH;
    const bool more = nr < rows && nr >= row;
    if (more) {
      if (row_ends) next_pos = __ldg(p.pos + nr);
      load(next, nr, nh);
    }
    if (pos >= 0) {
      T* to = out + row * out_stride;
      float r[AHEAD];
      if (p.norm) {
        // the gains on their way, and the heads' sums side by side: a sum alone would wait for each of its shuffles
        if (g && !one) {
#pragma unroll
          for (int u = 0; u < AHEAD; ++u) gr[u].load(g + at(h0, u), l);
        }
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
        if (p.norm) y = g ? times(y, times(sides<NEIGHBOURS>(gr[u]), r[u])) : times(y, r[u]);
        y = turn.forward(y);
        if (WHOLE || h0 + hl + u * HPW < last) store_sides<NEIGHBOURS>(to + at(h0, u), l, y);
      }
    }
    if (!more) break;
    if (row_ends) {
      pos = next_pos;
      turn = angles<LPR>(p, pos, lane, buf);
    }
    row = nr;
    h0 = nh;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u] = next[u];
  }
}

// Backward: block (x, y) takes rows [x * chunk, (x + 1) * chunk) of the HPW heads that lie side by side in a warp, its warps a row each.  The gains' partial
// sums of its rows go to part[x][heads * HD], added up by sum_parts_kernel in the order of x.
template <typename T, int LPR, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, 4) rotate_backward_kernel(const __grid_constant__ RotateParams p, int chunk, float* part) {
  constexpr int HPW = 32 / LPR, HD = LPR * 8, ROWS = kThreads / 32;
  __shared__ __align__(16) float red[ROWS][HPW * HD];
  __shared__ __align__(16) Angles bufs[ROWS];
  Angles& buf = bufs[threadIdx.x >> 5];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % LPR, hl = lane / LPR;
  const Lane l = lane_of<NEIGHBOURS>(p, c);
  const int heads = p.n_heads + p.n_kv, hh = blockIdx.y * HPW + hl;
  const bool head_in = hh < heads;
  const int hc = head_in ? hh : heads - 1;
  const bool is_q = hc < p.n_heads;
  const int h = is_q ? hc : hc - p.n_heads;
  const long long stride = is_q ? p.q_stride : p.k_stride, gstride = (long long)(is_q ? p.n_heads : p.n_kv) * HD;
  const T* x0 = (const T*)(is_q ? p.q : p.k) + (size_t)h * HD;
  const float* d0 = (is_q ? p.dq_out : p.dk_out) + (size_t)h * HD;
  float* o0 = (is_q ? p.dq : p.dk) + (size_t)h * HD;
  const T* g = p.norm ? (const T*)(is_q ? p.g_q : p.g_k) : nullptr;
  const F2 zero = f2(0.f, 0.f), one = f2(1.f, 1.f);
  Pairs gv = {{one, one}, {one, one}}, dg = {{zero, zero}, {zero, zero}};
  if (g) {
    Runs<T> gr;
    gr.load(g + (size_t)h * HD, l);
    gv = sides<NEIGHBOURS>(gr);
  }
  const long long r0 = (long long)blockIdx.x * chunk, r1 = min((long long)p.rows, r0 + chunk);
  for (long long rb = r0 + warp; rb < r1; rb += ROWS) {
    // (The clamp changes no value.  Without it the compiler moves the loads behind the test of pos, and every row waits for memory twice: 120 us against 110.)
    const size_t row = (size_t)min(rb, r1 - 1);
    const int pos = __ldg(p.pos + row);
    Runs<T> x;
    Runs<float> d;
    x.load(x0 + row * stride, l);
    d.load(d0 + row * gstride, l);
    if (rb >= r1 || pos < 0) continue;
    const Turn turn = angles<LPR>(p, pos, lane, buf);
    Pairs w = turn.back(sides<NEIGHBOURS>(d));
    if (p.norm) {
      Pairs y = sides<NEIGHBOURS>(x);
      const float r = rsqrtf(row_sum<LPR>(dot(y, y)) * (1.0f / HD) + p.eps);
      y = times(y, r);
      add_to(dg, w, y);
      w = times(w, gv);
      const float mean = row_sum<LPR>(dot(w, y)) * (1.0f / HD);
      const Pairs m = {{f2(-mean, -mean), f2(-mean, -mean)}, {f2(-mean, -mean), f2(-mean, -mean)}};
      add_to(w, y, m);
      w = times(w, r);
    }
    if (head_in) store_sides<NEIGHBOURS>(o0 + (size_t)rb * gstride, l, w);
  }
  if (!part) return;
  store_sides<NEIGHBOURS>(&red[warp][hl * HD], l, dg);
  __syncthreads();
  for (int i = threadIdx.x; i < HPW * HD; i += kThreads) {
    if (blockIdx.y * HPW + i / HD >= heads) continue;
    float a = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) a += red[r][i];
    part[(size_t)blockIdx.x * heads * HD + (size_t)blockIdx.y * HPW * HD + i] = a;
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

struct Split { int chunk, parts; };
// about eight blocks for each SM, a multiple of 16 rows (two for each warp) each
int backward_most_parts(int heads, int hd) { return max(1, ceil_div(148 * 8, ceil_div(heads, 256 / hd))); }
Split backward_split(int heads, int hd, int rows) {
  const int want = backward_most_parts(heads, hd);
  const int chunk = (int)align_up((size_t)max((int)(((long long)rows + want - 1) / want), 1), 16);
  return {chunk, (int)(((long long)rows + chunk - 1) / chunk)};
}

template <typename T, int LPR, bool NEIGHBOURS>
cudaError_t forward_launch(const RotateParams& p, bool q, bool k, cudaStream_t s) {
  constexpr int HPW = 32 / LPR, MOST = sizeof(T) == 2 ? 4 : 2;
  const long long blocks = ((long long)p.rows + kThreads / 32 - 1) / (kThreads / 32);
  const int nq = q ? p.n_heads : 0, nk = k ? p.n_kv : 0, most = max(nq, nk);
  const int ways = (int)min((long long)ceil_div(most, HPW), max(1LL, 148 * 2 / blocks));       // at least two blocks for each SM if the heads allow it
  const int heads_per = ceil_div(ceil_div(most, ways), HPW) * HPW, y_q = ceil_div(nq, heads_per), parts = y_q + ceil_div(nk, heads_per);
  // as many blocks as the GPU holds at once: a warp goes on to its next row with that row's loads under way
  const dim3 grid((unsigned)min(blocks, (long long)max(1, 148 * kBlocks / parts)), parts);
  auto fits = [&](int ahead) { return heads_per % (HPW * ahead) == 0 && nq % heads_per == 0 && nk % heads_per == 0; };
  if (MOST >= 4 && fits(4)) rotate_kernel<T, LPR, NEIGHBOURS, MOST, true><<<grid, kThreads, 0, s>>>(p, heads_per, y_q);
  else if (MOST >= 3 && fits(3)) rotate_kernel<T, LPR, NEIGHBOURS, MOST - 1, true><<<grid, kThreads, 0, s>>>(p, heads_per, y_q);
  else if (fits(2)) rotate_kernel<T, LPR, NEIGHBOURS, 2, true><<<grid, kThreads, 0, s>>>(p, heads_per, y_q);
  else if (fits(1)) rotate_kernel<T, LPR, NEIGHBOURS, 1, true><<<grid, kThreads, 0, s>>>(p, heads_per, y_q);
  else rotate_kernel<T, LPR, NEIGHBOURS, 2, false><<<grid, kThreads, 0, s>>>(p, heads_per, y_q);
  return cudaGetLastError();
}
template <typename T, int LPR>
cudaError_t forward(const RotateParams& p, cudaStream_t s) {
  auto launch = p.neighbours ? forward_launch<T, LPR, true> : forward_launch<T, LPR, false>;
  // Queries and keys in one launch; in two where their heads differ in number and each fills the GPU by itself, so that each has batches that fit it and
  // neither waits for the other's longer rows (8 x 2048 rows of 16 and 4 heads: 25 us against 29).
  if (p.n_kv == p.n_heads || p.n_kv == 0 || p.rows < 148 * kBlocks * (kThreads / 32)) return launch(p, true, p.n_kv > 0, s);
  const cudaError_t e = launch(p, true, false, s);
  return e != cudaSuccess ? e : launch(p, false, true, s);
}

template <typename T, int LPR>
cudaError_t backward(const RotateParams& p, const Split& sp, float* part, cudaStream_t s) {
  const dim3 grid(sp.parts, ceil_div(p.n_heads + p.n_kv, 32 / LPR));
  if (p.neighbours) rotate_backward_kernel<T, LPR, true><<<grid, kThreads, 0, s>>>(p, sp.chunk, part);
  else rotate_backward_kernel<T, LPR, false><<<grid, kThreads, 0, s>>>(p, sp.chunk, part);
  return cudaGetLastError();
}

}  // namespace

size_t rotate_backward_workspace(int heads, int hd, int rows) {
  // (no fewer parts for more rows, so that a workspace for many rows serves fewer)
  const int most = backward_most_parts(heads, hd), parts = rows / 16 + 1;
  return align_up((size_t)(parts < most ? parts : most) * heads * hd * 4, 256);
}

cudaError_t rotate_launch(int dtype, const RotateParams& p, cudaStream_t s) {
  if (dtype == RT_BF16) return p.hd == 64 ? forward<__nv_bfloat16, 8>(p, s) : forward<__nv_bfloat16, 16>(p, s);
  return p.hd == 64 ? forward<float, 8>(p, s) : forward<float, 16>(p, s);
}

cudaError_t rotate_backward_launch(int dtype, const RotateParams& p, void* workspace, cudaStream_t s) {
  const int heads = p.n_heads + p.n_kv;
  const Split sp = backward_split(heads, p.hd, p.rows);
  float* part = (p.dg_q || p.dg_k) ? (float*)workspace : nullptr;
  if (p.rows > 0) {
    cudaError_t e;
    if (dtype == RT_BF16) e = p.hd == 64 ? backward<__nv_bfloat16, 8>(p, sp, part, s) : backward<__nv_bfloat16, 16>(p, sp, part, s);
    else e = p.hd == 64 ? backward<float, 8>(p, sp, part, s) : backward<float, 16>(p, sp, part, s);
    if (e != cudaSuccess) return e;
  }
  if (!part) return cudaSuccess;
  return launch_chained(sum_parts_kernel, dim3(ceil_div(heads * p.hd, 32)), dim3(kThreads), 0, s, p.rows > 0, (const float*)part, p.rows > 0 ? sp.parts : 0,
                        p.n_heads * p.hd, heads * p.hd, p.dg_q, p.dg_k);
}

}  // namespace rt
