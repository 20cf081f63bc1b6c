// Rows of keys and values into the pages of a cache and out of them.
//
// Bound: HBM traffic (every row is read once and written once).  Lanes hold 8 consecutive elements (16 bytes of bf16), head_dim / 8
// lanes a row of a head, so that every access of a warp covers whole 64- or 128-byte rows on both sides.
#include "rt_paged.h"

namespace rt {
namespace {

constexpr int kThreads = 256;

// The exponent k of a row's scale 2^k: the smallest k >= -126 with amax <= 448 2^k, 448 = 1.75 * 2^8.  amax is finite.
__device__ __forceinline__ int scale_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int k = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(k, -126);
}

__device__ __forceinline__ unsigned to_e4m3x2(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// One row of a head, 8 elements a lane, into its place if `ok`.  The LPR lanes of a row are neighbours in a warp and agree on ok; all lanes
// of the warp call (shuffles).
template <int LPR>
__device__ __forceinline__ void put_row(void* pool, uint8_t* exps, int dtype, size_t row, int lane8, bool ok, float (&x)[8]) {
  const size_t at = row * (LPR * 8) + (size_t)lane8 * 8;
  if (dtype != RT_E4M3) {
    if (ok && dtype == RT_BF16) store8((__nv_bfloat16*)pool + at, x);
    else if (ok) store8((float*)pool + at, x);
    return;
  }
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (isfinite(x[i])) amax = fmaxf(amax, fabsf(x[i]));
    else x[i] = __uint_as_float(0x7fffffffu);                      // e4m3 has no infinity: stored as NaN
  }
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  const int k = scale_exponent(amax);
  const float r = __uint_as_float((unsigned)(127 - k) << 23);      // 2^-k: 127 - k is in [7, 253]
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = to_e4m3x2(x[2 * i] * r, x[2 * i + 1] * r);
  if (ok) {
    *reinterpret_cast<uint2*>((uint8_t*)pool + at) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    if (lane8 == 0) exps[row] = (uint8_t)(k + 127);
  }
}

template <int LPR>
__device__ __forceinline__ void get_row(const void* pool, const uint8_t* exps, int dtype, size_t row, int lane8, float (&x)[8]) {
  const size_t at = row * (LPR * 8) + (size_t)lane8 * 8;
  if (dtype == RT_BF16) { load8((const __nv_bfloat16*)pool + at, x); return; }
  if (dtype == RT_F32) { load8((const float*)pool + at, x); return; }
  const uint2 w = __ldg(reinterpret_cast<const uint2*>((const uint8_t*)pool + at));
  const float s = scale_of(__ldg(exps + row));
  const unsigned h[4] = {w.x, w.x >> 16, w.y, w.y >> 16};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = from_e4m3x2(h[i]);
    x[2 * i] = f.x * s; x[2 * i + 1] = f.y * s;
  }
}

// rows r, heads h and {keys, values}: item = (r * 2 + which) * n_kv + h
template <typename T, int LPR, bool WRITE>
__global__ void __launch_bounds__(kThreads) cache_rows_kernel(const CacheRowsParams p) {
  constexpr int RPB = kThreads / LPR;
  const int lane8 = threadIdx.x % LPR;
  const int n_kv = p.c.n_kv_heads;
  const long long items = (long long)p.rows * 2 * n_kv;
  for (long long it = (long long)blockIdx.x * RPB + threadIdx.x / LPR, base = (long long)blockIdx.x * RPB; base < items;
       base += (long long)gridDim.x * RPB, it += (long long)gridDim.x * RPB) {
    const bool in = it < items;
    const long long i = in ? it : items - 1;                       // (lanes beyond the end stay for the shuffles)
    const int h = (int)(i % n_kv);
    const long long rw = i / n_kv;
    const int which = (int)(rw & 1), r = (int)(rw >> 1);
    const int b = __ldg(p.seq + r), t = __ldg(p.pos + r);
    bool ok = in && t >= 0;
    int page = -1;
    if (ok) {
      if ((unsigned)b < (unsigned)p.c.n_seqs && (t >> p.log_page) < p.c.max_pages) page = page_at(p.c, b, t >> p.log_page);
      else if (p.c.status) *p.c.status = RT_ERR_INVALID_ARG;
      ok = page >= 0;
    }
    const size_t row = ((size_t)(ok ? page : 0) * n_kv + h) * p.c.page_size + (size_t)(t & (p.c.page_size - 1));
    const long long stride = which ? p.v_stride : p.k_stride;
    void* pool = which ? p.c.v : p.c.k;
    uint8_t* exps = which ? p.c.v_exp : p.c.k_exp;
    const size_t at = (size_t)r * stride + ((size_t)h * LPR + lane8) * 8;
    float x[8];
    if constexpr (WRITE) {
      load8((const T*)(which ? p.v_in : p.k_in) + at, x);
      put_row<LPR>(pool, exps, p.c.dtype, row, lane8, ok, x);
    } else if (ok) {
      get_row<LPR>(pool, exps, p.c.dtype, row, lane8, x);
      store8((T*)(which ? p.v_out : p.k_out) + at, x);
    }
  }
}

template <typename T, bool WRITE>
cudaError_t launch(const CacheRowsParams& p, cudaStream_t s) {
  const int rpb = kThreads / (p.c.head_dim / 8);
  const long long blocks = ((long long)p.rows * 2 * p.c.n_kv_heads + rpb - 1) / rpb;
  const dim3 grid((unsigned)(blocks < 148 * 64 ? blocks : 148 * 64));
  if (p.c.head_dim == 64) cache_rows_kernel<T, 8, WRITE><<<grid, kThreads, 0, s>>>(p);
  else cache_rows_kernel<T, 16, WRITE><<<grid, kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t cache_write_launch(int dtype, const CacheRowsParams& p, cudaStream_t s) {
  return dtype == RT_BF16 ? launch<__nv_bfloat16, true>(p, s) : launch<float, true>(p, s);
}
cudaError_t cache_read_launch(int dtype, const CacheRowsParams& p, cudaStream_t s) {
  return dtype == RT_BF16 ? launch<__nv_bfloat16, false>(p, s) : launch<float, false>(p, s);
}

}  // namespace rt
