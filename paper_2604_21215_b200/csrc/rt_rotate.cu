// qkRMS of queries and keys for each head and the rotation by the position, in one pass, and its backward pass.
//
// Bound: HBM traffic.  A row of a head lies on head_dim / 8 neighbouring lanes, 8 elements each, so the norm is a few shuffles, and with
// rot_dim a multiple of 16 the partners of a lane's dimensions lie on one other lane (halves) or on the lane itself (neighbours).
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

// Lane c of a row holds dimensions [8 c, 8 c + 8).  What it needs of the rotation: role 0 none, 1 first of a pair, 2 second, 3 both; the first
// of its pairs' numbers; the lane (within the row) of the partners.
struct Lane { int role, first, partner; };
__device__ __forceinline__ Lane lane_of(const RotateParams& p, int c) {
  const int half = p.rot / 2;
  if (8 * c >= p.rot) return {0, 0, c};
  if (p.neighbours) return {3, 4 * c, c};
  return 8 * c < half ? Lane{1, 8 * c, c + half / 8} : Lane{2, 8 * c - half, c - half / 8};
}

// cos and sin of the lane's angles: 8 of them (halves) or 4 (neighbours).  The turns are reduced in 64 bits, so that far positions keep theirs.
__device__ __forceinline__ void angles(const RotateParams& p, const Lane& l, int pos, float (&cs)[8], float (&sn)[8]) {
  if (!l.role) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= 4 && l.role == 3) break;
    const double t = (double)pos * p.turns[l.first + i];
    sincospif((float)(2.0 * (t - rint(t))), &sn[i], &cs[i]);
  }
}

// y: this lane's dimensions -> rotated by the angles (dir = 1) or back (dir = -1).  All lanes of the warp call.
__device__ __forceinline__ void turn(const Lane& l, int lane_base, const float (&cs)[8], const float (&sn)[8], float dir, float (&y)[8]) {
  float o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = __shfl_sync(0xffffffffu, y[i], lane_base + l.partner);
  if (l.role == 3) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = y[2 * i], b = y[2 * i + 1], s = dir * sn[i];
      y[2 * i] = a * cs[i] - b * s;
      y[2 * i + 1] = a * s + b * cs[i];
    }
  } else if (l.role) {
    const float sg = l.role == 1 ? -dir : dir;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * cs[i] + sg * o[i] * sn[i];
  }
}

// item = row * heads + head, the queries' heads first
template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const __grid_constant__ RotateParams p) {
  constexpr int RPB = kThreads / LPR, HD = LPR * 8;
  const int c = threadIdx.x % LPR, base_lane = (threadIdx.x & 31) - c;
  const Lane l = lane_of(p, c);
  const int heads = p.n_heads + p.n_kv;
  const long long items = (long long)p.rows * heads;
  for (long long base = (long long)blockIdx.x * RPB; base < items; base += (long long)gridDim.x * RPB) {
    const long long it = base + threadIdx.x / LPR;
    const bool in = it < items;
    const long long i = in ? it : items - 1;
    const int row = (int)(i / heads), hh = (int)(i % heads);
    const bool is_q = hh < p.n_heads;
    const int h = is_q ? hh : hh - p.n_heads;
    const int pos = __ldg(p.pos + row);
    const bool ok = in && pos >= 0;
    const size_t col = (size_t)h * HD + 8 * c;
    float x[8], cs[8], sn[8];
    load8((const T*)(is_q ? p.q : p.k) + (size_t)row * (is_q ? p.q_stride : p.k_stride) + col, x);
    if (p.norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
      const float r = rsqrtf(row_sum<LPR>(ss) * (1.0f / HD) + p.eps);
      const T* g = (const T*)(is_q ? p.g_q : p.g_k);
      float gv[8];
      if (g) load8(g + col, gv);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = g ? x[e] * r * gv[e] : x[e] * r;
    }
    angles(p, l, pos, cs, sn);
    turn(l, base_lane, cs, sn, 1.0f, x);
    if (ok) store8((T*)(is_q ? p.q_out : p.k_out) + (size_t)row * (is_q ? p.qo_stride : p.ko_stride) + col, x);
  }
}

// Backward: block (x, y) takes rows [x * chunk, (x + 1) * chunk) of the four heads of group y; the gains' partial sums of its rows go to
// part[x][heads * HD], added up by sum_parts_kernel in the order of x.
constexpr int kHeadsPerBlock = 4;
template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads) rotate_backward_kernel(const __grid_constant__ RotateParams p, int chunk, float* part) {
  constexpr int RPB = kThreads / LPR, HD = LPR * 8, ROWS = RPB / kHeadsPerBlock;
  __shared__ float red[RPB][HD];
  const int c = threadIdx.x % LPR, base_lane = (threadIdx.x & 31) - c, g_id = threadIdx.x / LPR;
  const Lane l = lane_of(p, c);
  const int heads = p.n_heads + p.n_kv;
  const int hh0 = blockIdx.y * kHeadsPerBlock + g_id % kHeadsPerBlock;
  const bool head_in = hh0 < heads;
  const int hh = head_in ? hh0 : heads - 1;
  const bool is_q = hh < p.n_heads;
  const int h = is_q ? hh : hh - p.n_heads;
  const size_t col = (size_t)h * HD + 8 * c;
  const T* g = p.norm ? (const T*)(is_q ? p.g_q : p.g_k) : nullptr;
  float gv[8], dg[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { gv[e] = 1.0f; dg[e] = 0.0f; }
  if (g) load8(g + col, gv);
  const long long r1 = min((long long)p.rows, (long long)(blockIdx.x + 1) * chunk);
  for (long long r0 = (long long)blockIdx.x * chunk; r0 < r1; r0 += ROWS) {
    const long long rr = r0 + g_id / kHeadsPerBlock;
    const bool in = head_in && rr < r1;
    const size_t row = (size_t)(rr < r1 ? rr : r1 - 1);
    const int pos = __ldg(p.pos + row);
    const bool ok = in && pos >= 0;
    float x[8], d[8], cs[8], sn[8];
    load8((const T*)(is_q ? p.q : p.k) + row * (is_q ? p.q_stride : p.k_stride) + col, x);
    const size_t gat = row * (size_t)(is_q ? p.n_heads : p.n_kv) * HD + col;
    load8((is_q ? p.dq_out : p.dk_out) + gat, d);
    angles(p, l, pos, cs, sn);
    turn(l, base_lane, cs, sn, -1.0f, d);
    if (p.norm) {
      float ss = 0.f, du = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
      const float r = rsqrtf(row_sum<LPR>(ss) * (1.0f / HD) + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] *= r;
        if (ok) dg[e] += d[e] * x[e];
        d[e] *= gv[e];
        du += d[e] * x[e];
      }
      const float mean = row_sum<LPR>(du) * (1.0f / HD);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = r * (d[e] - x[e] * mean);
    }
    if (ok) store8((is_q ? p.dq : p.dk) + gat, d);
  }
  if (!part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) red[g_id][8 * c + e] = dg[e];
  __syncthreads();
  for (int i = threadIdx.x; i < kHeadsPerBlock * HD; i += kThreads) {
    const int hl = i / HD, dim = i % HD;
    if (blockIdx.y * kHeadsPerBlock + hl >= heads) continue;
    float a = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) a += red[r * kHeadsPerBlock + hl][dim];
    part[((size_t)blockIdx.x * heads + blockIdx.y * kHeadsPerBlock + hl) * HD + dim] = a;
  }
}

__global__ void __launch_bounds__(kThreads) sum_parts_kernel(const float* part, int parts, int nq, int n, float* dg_q, float* dg_k) {
  __shared__ float red[8][32];
  const int i = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
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
Split backward_split(int heads, int rows) {
  // about four blocks for each SM, a multiple of 32 rows each
  const int groups = ceil_div(heads, kHeadsPerBlock);
  const int want = max(1, ceil_div(148 * 4, groups));
  int chunk = (int)(((long long)rows + want - 1) / want);
  chunk = (int)align_up((size_t)max(chunk, 1), 32);
  return {chunk, (int)(((long long)rows + chunk - 1) / chunk)};
}

}  // namespace

size_t rotate_backward_workspace(int heads, int hd, int rows) {
  return align_up((size_t)max(backward_split(heads, rows).parts, 1) * heads * hd * 4, 256);
}

cudaError_t rotate_launch(int dtype, const RotateParams& p, cudaStream_t s) {
  const int rpb = kThreads / (p.hd / 8);
  const long long blocks = ((long long)p.rows * (p.n_heads + p.n_kv) + rpb - 1) / rpb;
  const dim3 grid((unsigned)(blocks < 148 * 64 ? blocks : 148 * 64));
  if (dtype == RT_BF16) {
    if (p.hd == 64) rotate_kernel<__nv_bfloat16, 8><<<grid, kThreads, 0, s>>>(p);
    else rotate_kernel<__nv_bfloat16, 16><<<grid, kThreads, 0, s>>>(p);
  } else {
    if (p.hd == 64) rotate_kernel<float, 8><<<grid, kThreads, 0, s>>>(p);
    else rotate_kernel<float, 16><<<grid, kThreads, 0, s>>>(p);
  }
  return cudaGetLastError();
}

cudaError_t rotate_backward_launch(int dtype, const RotateParams& p, void* workspace, cudaStream_t s) {
  const int heads = p.n_heads + p.n_kv;
  const Split sp = backward_split(heads, p.rows);
  float* part = (p.dg_q || p.dg_k) ? (float*)workspace : nullptr;
  if (p.rows > 0) {
    const dim3 grid(sp.parts, ceil_div(heads, kHeadsPerBlock));
    if (dtype == RT_BF16) {
      if (p.hd == 64) rotate_backward_kernel<__nv_bfloat16, 8><<<grid, kThreads, 0, s>>>(p, sp.chunk, part);
      else rotate_backward_kernel<__nv_bfloat16, 16><<<grid, kThreads, 0, s>>>(p, sp.chunk, part);
    } else {
      if (p.hd == 64) rotate_backward_kernel<float, 8><<<grid, kThreads, 0, s>>>(p, sp.chunk, part);
      else rotate_backward_kernel<float, 16><<<grid, kThreads, 0, s>>>(p, sp.chunk, part);
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (part) sum_parts_kernel<<<ceil_div(heads * p.hd, 32), kThreads, 0, s>>>(part, p.rows > 0 ? sp.parts : 0, p.n_heads * p.hd, heads * p.hd, p.dg_q, p.dg_k);
  return cudaGetLastError();
}

}  // namespace rt
