// qkRMS of queries and keys for each head and the rotation by the position, in one pass, and its backward pass.
//
// Bound: HBM traffic.  head_dim / 8 neighbouring lanes hold a row of a head; each holds the two sides a[i], b[i] of four pairs of dimensions, as
// two loads of 4 elements, so the rotation needs no exchange and the norm a few shuffles.  Dimensions that are not rotated make pairs too, with an angle
// of zero.  A warp takes the heads of one row side by side and one after the other: its lanes form the row's angles once, one or two each.
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

__device__ __forceinline__ void load4(const float* p, float (&f)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&f)[4]) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  f[0] = __uint_as_float(a.x << 16); f[1] = __uint_as_float(a.x & 0xffff0000u);
  f[2] = __uint_as_float(a.y << 16); f[3] = __uint_as_float(a.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) { *reinterpret_cast<uint2*>(p) = make_uint2(pack2(a, b), pack2(c, d)); }

// the eight elements of a lane as sides of pairs: x[i] = a, x[4 + i] = b
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void load_pairs(const T* row, const Lane& l, float (&x)[8]) {
  float u[4], v[4];
  load4(row + l.first, u);
  load4(row + l.second, v);
  if (NEIGHBOURS) {
    x[0] = u[0]; x[4] = u[1]; x[1] = u[2]; x[5] = u[3]; x[2] = v[0]; x[6] = v[1]; x[3] = v[2]; x[7] = v[3];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
  }
}
template <typename T, bool NEIGHBOURS>
__device__ __forceinline__ void store_pairs(T* row, const Lane& l, const float (&x)[8]) {
  if (NEIGHBOURS) {
    store4(row + l.first, x[0], x[4], x[1], x[5]);
    store4(row + l.second, x[2], x[6], x[3], x[7]);
  } else {
    store4(row + l.first, x[0], x[1], x[2], x[3]);
    store4(row + l.second, x[4], x[5], x[6], x[7]);
  }
}

// cos and sin of this lane's four pairs.  Pair n's angle is formed by lane n % 32 of the warp; the turns are reduced in 64 bits, so that far
// positions keep their angles.  All lanes of the warp call.
template <int LPR>
__device__ __forceinline__ void angles(const RotateParams& p, int pos, int lane, float (&cs)[4], float (&sn)[4]) {
  constexpr int PER = LPR / 8;
  float co[PER], si[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    co[k] = 1.f; si[k] = 0.f;
    const int n = lane + 32 * k;
    if (2 * n < p.rot) {
      const double t = (double)pos * p.turns[n];
      sincospif((float)(2.0 * (t - rint(t))), &si[k], &co[k]);
    }
  }
  const int c = lane % LPR;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int from = (4 * c + i) & 31;
    cs[i] = __shfl_sync(0xffffffffu, co[0], from);
    sn[i] = __shfl_sync(0xffffffffu, si[0], from);
    if (PER == 2) {
      const float c1 = __shfl_sync(0xffffffffu, co[PER - 1], from), s1 = __shfl_sync(0xffffffffu, si[PER - 1], from);
      if (4 * c + i >= 32) { cs[i] = c1; sn[i] = s1; }
    }
  }
}
__device__ __forceinline__ void turn(const float (&cs)[4], const float (&sn)[4], float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[i], b = x[4 + i];
    x[i] = a * cs[i] - b * sn[i];
    x[4 + i] = a * sn[i] + b * cs[i];
  }
}

// Block row y of the grid takes the heads [y * heads_per, ...) of every row: all of them where there are rows enough to fill the GPU, some of them in
// small calls, where a warp's chain of heads would be the call's time.
constexpr int kAhead = 4;       // loads in flight
template <typename T, int LPR, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const __grid_constant__ RotateParams p, int heads_per) {
  constexpr int HPW = 32 / LPR, HD = LPR * 8;
  const int lane = threadIdx.x & 31, hl = lane / LPR;
  const Lane l = lane_of<NEIGHBOURS>(p, lane % LPR);
  const int heads = p.n_heads + p.n_kv, first = blockIdx.y * heads_per, last = min(heads, first + heads_per);
  const long long warps = (long long)gridDim.x * (kThreads / 32);
  for (long long row = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); row < p.rows; row += warps) {
    const int pos = __ldg(p.pos + row);
    if (pos < 0) continue;
    float cs[4], sn[4];
    const T *qr = (const T*)p.q + (size_t)row * p.q_stride, *kr = (const T*)p.k + (size_t)row * p.k_stride;
    T *qo = (T*)p.q_out + (size_t)row * p.qo_stride, *ko = (T*)p.k_out + (size_t)row * p.ko_stride;
    for (int h0 = first; h0 < last; h0 += HPW * kAhead) {
      float x[kAhead][8];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int h = min(h0 + u * HPW + hl, last - 1);            // (lanes without a head repeat the last one's for the shuffles)
        load_pairs<T, NEIGHBOURS>(h < p.n_heads ? qr + (size_t)h * HD : kr + (size_t)(h - p.n_heads) * HD, l, x[u]);
      }
      if (h0 == first) angles<LPR>(p, pos, lane, cs, sn);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (h0 + u * HPW >= last) break;
        const int hh = h0 + u * HPW + hl, h = min(hh, last - 1), hk = h - p.n_heads;
        if (p.norm) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += x[u][e] * x[u][e];
          const float r = rsqrtf(row_sum<LPR>(ss) * (1.0f / HD) + p.eps);
          const T* g = (const T*)(hk < 0 ? p.g_q : p.g_k);
          if (g) {
            float gv[8];
            load_pairs<T, NEIGHBOURS>(g + (size_t)(hk < 0 ? h : hk) * HD, l, gv);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] *= r * gv[e];
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] *= r;
          }
        }
        turn(cs, sn, x[u]);
        if (hh < last) store_pairs<T, NEIGHBOURS>(hk < 0 ? qo + (size_t)h * HD : ko + (size_t)hk * HD, l, x[u]);
      }
    }
  }
}

// Backward: block (x, y) takes rows [x * chunk, (x + 1) * chunk) of the HPW heads that lie side by side in a warp, its warps a row each.  The gains' partial
// sums of its rows go to part[x][heads * HD], added up by sum_parts_kernel in the order of x.
template <typename T, int LPR, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads) rotate_backward_kernel(const __grid_constant__ RotateParams p, int chunk, float* part) {
  constexpr int HPW = 32 / LPR, HD = LPR * 8, ROWS = kThreads / 32, AHEAD = 2;
  __shared__ float red[ROWS][HPW * HD];
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
  float gv[8], dg[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { gv[e] = 1.0f; dg[e] = 0.0f; }
  if (g) load_pairs<T, NEIGHBOURS>(g + (size_t)h * HD, l, gv);
  const long long r0 = (long long)blockIdx.x * chunk, r1 = min((long long)p.rows, r0 + chunk);
  for (long long rb = r0 + warp; rb < r1; rb += ROWS * AHEAD) {
    float x[AHEAD][8], d[AHEAD][8];
    int pos[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const long long row = min(rb + u * ROWS, r1 - 1);
      pos[u] = __ldg(p.pos + row);
      load_pairs<T, NEIGHBOURS>(x0 + (size_t)row * stride, l, x[u]);
      load_pairs<float, NEIGHBOURS>(d0 + (size_t)row * gstride, l, d[u]);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const long long row = rb + u * ROWS;
      if (row >= r1 || pos[u] < 0) continue;
      float cs[4], sn[4];
      angles<LPR>(p, pos[u], lane, cs, sn);
#pragma unroll
      for (int i = 0; i < 4; ++i) sn[i] = -sn[i];
      turn(cs, sn, d[u]);
      if (p.norm) {
        float ss = 0.f, du = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[u][e] * x[u][e];
        const float r = rsqrtf(row_sum<LPR>(ss) * (1.0f / HD) + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[u][e] *= r;
          dg[e] += d[u][e] * x[u][e];
          d[u][e] *= gv[e];
          du += d[u][e] * x[u][e];
        }
        const float mean = row_sum<LPR>(du) * (1.0f / HD);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[u][e] = r * (d[u][e] - x[u][e] * mean);
      }
      if (head_in) store_pairs<float, NEIGHBOURS>(o0 + (size_t)row * gstride, l, d[u]);
    }
  }
  if (!part) return;
  store_pairs<float, NEIGHBOURS>(&red[warp][hl * HD], l, dg);
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

template <typename T, int LPR>
cudaError_t forward(const RotateParams& p, cudaStream_t s) {
  constexpr int HPW = 32 / LPR;
  const long long blocks = ((long long)p.rows + kThreads / 32 - 1) / (kThreads / 32);
  const int heads = p.n_heads + p.n_kv;
  // at least two blocks for each SM if the heads allow it
  const int ways = (int)min((long long)ceil_div(heads, HPW), max(1LL, 148 * 2 / blocks));
  const int heads_per = ways == 1 ? heads : max(HPW, ceil_div(ceil_div(heads, ways), HPW) * HPW);
  const dim3 grid((unsigned)(blocks < 148 * 64 ? blocks : 148 * 64), ceil_div(heads, heads_per));
  if (p.neighbours) rotate_kernel<T, LPR, true><<<grid, kThreads, 0, s>>>(p, heads_per);
  else rotate_kernel<T, LPR, false><<<grid, kThreads, 0, s>>>(p, heads_per);
  return cudaGetLastError();
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
