// Attention of one new token of every sequence over its cached pairs, in pages.
//
// A block owns a sequence, a head of the cache and up to four of the query heads that share it.  Its warps take the positions 32 at a
// time; a row of keys or values lies on head_dim * size / 16 lanes, 16 bytes each, so a warp reads several positions' rows at once.  Every such
// group of lanes keeps its own running maximum, sum and output (online softmax), and they are joined at the end.
#include "rt_paged.h"

namespace rt {
namespace {

constexpr int kWarps = 8, kGroupMax = 4;

// 16 bytes of a row -> floats
__device__ __forceinline__ void unpack16(const uint4& a, float (&f)[4], float) {
  f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
}
__device__ __forceinline__ void unpack16(const uint4& a, float (&f)[8], __nv_bfloat16) { unpack8(a, f); }
__device__ __forceinline__ void unpack16(const uint4& a, float (&f)[16], __nv_fp8_e4m3) {
  const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = from_e4m3x2(w[i / 2] >> (i % 2 * 16));
    f[2 * i] = t.x; f[2 * i + 1] = t.y;
  }
}

__device__ __forceinline__ float q_at(const rt_paged_query& q, const void* p, size_t i) {
  return q.dtype == RT_BF16 ? __bfloat162float(((const __nv_bfloat16*)p)[i]) : ((const float*)p)[i];
}

template <typename CT, int HD, int G>
__global__ void __launch_bounds__(kWarps * 32) paged_attn_kernel(const __grid_constant__ PagedAttnParams p) {
  constexpr int E = 16 / sizeof(CT), LPK = HD / E, KPI = 32 / LPK;
  __shared__ float sm_o[kWarps][G][HD], sm_m[kWarps][G], sm_l[kWarps][G];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / LPK, c = lane % LPK;
  const int b = blockIdx.x / p.c.n_kv_heads, kvh = blockIdx.x % p.c.n_kv_heads;
  const int h0 = kvh * p.group + blockIdx.y * G, g_in = min(G, p.group - blockIdx.y * G);
  int n = __ldg(p.q.lens + b);
  if (n < 0) return;
  const long long room = (long long)p.c.max_pages * p.c.page_size;
  if (n > room) {
    if (threadIdx.x == 0 && p.c.status) *p.c.status = RT_ERR_INVALID_ARG;
    n = (int)room;
  }
  const int at = p.q.k_own ? n : n - 1;                            // the query's position
  float q[G][E], slope[G], m[G], l[G], o[G][E];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int h = h0 + min(g, g_in - 1);
    slope[g] = p.q.alibi_slopes ? __ldg(p.q.alibi_slopes + h) * kLog2e : 0.f;
    m[g] = -INFINITY; l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) { q[g][e] = q_at(p.q, p.q.q, (size_t)b * p.q.q_stride + (size_t)h * HD + c * E + e); o[g][e] = 0.f; }
  }
  for (int j0 = warp * KPI; j0 < n; j0 += kWarps * KPI) {
    const int j = j0 + sub;
    int page = -1;
    if (j < n) page = page_at(p.c, b, j >> p.log_page);
    const bool ok = page >= 0;
    float kf[E], vf[E], ks = 1.f, vs = 1.f;
    const size_t row = ((size_t)(ok ? page : 0) * p.c.n_kv_heads + kvh) * p.c.page_size + (size_t)(j & (p.c.page_size - 1));
    uint4 kr = make_uint4(0, 0, 0, 0), vr = kr;
    if (ok) {
      kr = __ldg((const uint4*)p.c.k + row * LPK + c);
      vr = __ldg((const uint4*)p.c.v + row * LPK + c);
      if (sizeof(CT) == 1) { ks = scale_of(__ldg(p.c.k_exp + row)); vs = scale_of(__ldg(p.c.v_exp + row)); }
    }
    unpack16(kr, kf, CT());
    unpack16(vr, vf, CT());
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float a = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) a += q[g][e] * kf[e];
#pragma unroll
      for (int w = LPK / 2; w; w >>= 1) a += __shfl_xor_sync(0xffffffffu, a, w);
      a = ok ? a * ks * p.scale_log2 - slope[g] * (float)(at - j) : -INFINITY;
      const float mn = fmaxf(m[g], a), ref = mn == -INFINITY ? 0.f : mn;
      const float w0 = exp2f(m[g] - ref), w1 = exp2f(a - ref), wv = w1 * vs;
      m[g] = mn;
      l[g] = l[g] * w0 + w1;
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = o[g][e] * w0 + (ok ? wv * vf[e] : 0.f);
    }
  }
  // the lane groups of a warp, then the warps
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int w = LPK; w < 32; w <<= 1) {
      const float mo = __shfl_xor_sync(0xffffffffu, m[g], w), lo = __shfl_xor_sync(0xffffffffu, l[g], w);
      const float mn = fmaxf(m[g], mo), ref = mn == -INFINITY ? 0.f : mn;
      const float w0 = exp2f(m[g] - ref), w1 = exp2f(mo - ref);
#pragma unroll
      for (int e = 0; e < E; ++e) o[g][e] = o[g][e] * w0 + __shfl_xor_sync(0xffffffffu, o[g][e], w) * w1;
      l[g] = l[g] * w0 + lo * w1;
      m[g] = mn;
    }
    if (sub == 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) sm_o[warp][g][c * E + e] = o[g][e];
      if (c == 0) { sm_m[warp][g] = m[g]; sm_l[warp][g] = l[g]; }
    }
  }
  __syncthreads();
  constexpr int D = HD / 32;
  for (int g = warp; g < g_in; g += kWarps) {
    const int h = h0 + g;
    float ma = -INFINITY, own = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) ma = fmaxf(ma, sm_m[w][g]);
    if (p.q.k_own) {
      float a = 0.f;
#pragma unroll
      for (int d = 0; d < D; ++d)
        a += q_at(p.q, p.q.q, (size_t)b * p.q.q_stride + (size_t)h * HD + d * 32 + lane) *
             q_at(p.q, p.q.k_own, (size_t)b * p.q.k_own_stride + (size_t)kvh * HD + d * 32 + lane);
      own = warp_sum(a) * p.scale_log2;
      ma = fmaxf(ma, own);
    }
    const float ref = ma == -INFINITY ? 0.f : ma;
    float la = 0.f, oa[D];
#pragma unroll
    for (int d = 0; d < D; ++d) oa[d] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float ww = exp2f(sm_m[w][g] - ref);
      la += sm_l[w][g] * ww;
#pragma unroll
      for (int d = 0; d < D; ++d) oa[d] += sm_o[w][g][d * 32 + lane] * ww;
    }
    if (p.q.k_own) {
      const float ww = exp2f(own - ref);
      la += ww;
#pragma unroll
      for (int d = 0; d < D; ++d) oa[d] += ww * q_at(p.q, p.q.v_own, (size_t)b * p.q.v_own_stride + (size_t)kvh * HD + d * 32 + lane);
    }
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const float y = la == 0.f ? 0.f : oa[d] / la;
      const size_t i = (size_t)b * p.q.out_stride + (size_t)h * HD + d * 32 + lane;
      if (p.q.dtype == RT_BF16) ((__nv_bfloat16*)p.q.out)[i] = __float2bfloat16_rn(y);
      else ((float*)p.q.out)[i] = y;
    }
    if (p.q.lse && lane == 0) p.q.lse[(size_t)b * p.q.n_heads + h] = la == 0.f ? -INFINITY : (ma + log2f(la)) * 0.6931471805599453f;
  }
}

template <typename CT, int HD>
cudaError_t launch(const PagedAttnParams& p, cudaStream_t s) {
  const int G = p.group >= 3 ? 4 : p.group;
  const dim3 grid((unsigned)p.c.n_seqs * (unsigned)p.c.n_kv_heads, ceil_div(p.group, G));
  if (G == 1) paged_attn_kernel<CT, HD, 1><<<grid, kWarps * 32, 0, s>>>(p);
  else if (G == 2) paged_attn_kernel<CT, HD, 2><<<grid, kWarps * 32, 0, s>>>(p);
  else paged_attn_kernel<CT, HD, 4><<<grid, kWarps * 32, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

size_t paged_attn_workspace(const rt_paged_cache*, int) { return 256; }

cudaError_t paged_attn_launch(const PagedAttnParams& p, void*, cudaStream_t s) {
  if (p.c.head_dim == 64)
    return p.c.dtype == RT_F32 ? launch<float, 64>(p, s) : p.c.dtype == RT_BF16 ? launch<__nv_bfloat16, 64>(p, s) : launch<__nv_fp8_e4m3, 64>(p, s);
  return p.c.dtype == RT_F32 ? launch<float, 128>(p, s) : p.c.dtype == RT_BF16 ? launch<__nv_bfloat16, 128>(p, s) : launch<__nv_fp8_e4m3, 128>(p, s);
}

}  // namespace rt
