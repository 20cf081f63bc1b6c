// Host-side launch interface and shared device helpers of the operators around paged caches (internal; the public ABI is
// include/rt.h): rows in and out of the pages, one-token attention, qkRMS with rotation.
#pragma once
#include <cuda_fp8.h>

#include "rt_kernels.h"

namespace rt {

struct CacheRowsParams {
  rt_paged_cache c;
  int log_page;                       // page_size = 1 << log_page
  const void *k_in, *v_in;            // write: rows of the caller
  void *k_out, *v_out;                // read
  long long k_stride, v_stride;       // elements between rows
  const int *seq, *pos;
  int rows;
};
cudaError_t cache_write_launch(int dtype, const CacheRowsParams& p, cudaStream_t s);
cudaError_t cache_read_launch(int dtype, const CacheRowsParams& p, cudaStream_t s);

struct PagedAttnParams {
  rt_paged_cache c;
  rt_paged_query q;
  int log_page, group;                // group = n_heads / n_kv_heads
  float scale_log2;
};
cudaError_t paged_attn_launch(const PagedAttnParams& p, void* workspace, cudaStream_t s);
bool paged_attn_counts(const rt_paged_cache* c, int n_heads);      // whether 32 bits count what such a call can be asked to do
size_t paged_attn_workspace(const rt_paged_cache* c, int n_heads);

constexpr int kMaxRot = 128;
struct RotateParams {
  int n_heads, n_kv, hd, norm, rot, neighbours;
  float eps;
  const void *q, *k, *g_q, *g_k;
  long long q_stride, k_stride, qo_stride, ko_stride;
  void *q_out, *k_out;
  const int* pos;
  int rows;
  const float *dq_out, *dk_out;       // backward
  float *dq, *dk, *dg_q, *dg_k;
  unsigned long long turns[kMaxRot / 2];      // turns per position, whole ones left out, in 2^-64 turns
};
cudaError_t rotate_launch(int dtype, const RotateParams& p, cudaStream_t s);
cudaError_t rotate_backward_launch(int dtype, const RotateParams& p, void* workspace, cudaStream_t s);
size_t rotate_backward_workspace(int heads, int hd, int rows);

#ifdef __CUDACC__
// ---- two fp32 numbers in a register pair: sm_100a multiplies and adds them in one instruction
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void split(F2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 add(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

// ---- eight consecutive elements <-> float ----------------------------------------------------
__device__ __forceinline__ void unpack8(const uint4& a, float (&f)[8]) {
  const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&f)[8]) { unpack8(*reinterpret_cast<const uint4*>(p), f); }
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ unsigned pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
// e4m3 codes: two in the low half of a word
__device__ __forceinline__ float2 from_e4m3x2(unsigned v) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xffffu), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// the scale 2^k of a stored exponent k + 127
__device__ __forceinline__ float scale_of(unsigned e) { return __uint_as_float(e << 23); }

// The page of position j of sequence b, or -1 with the status word set where the table names none.
__device__ __forceinline__ int page_at(const rt_paged_cache& c, int b, int page_no) {
  const int page = __ldg(c.page_table + (size_t)b * c.max_pages + page_no);
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  if (c.status) *c.status = RT_ERR_INVALID_ARG;
  return -1;
}
#endif

}  // namespace rt
