// Rows of keys and values into the pages of a cache and out of them.
//
// Bound: HBM traffic (every row is read once and written once), if the instructions per byte are few: at 6.5 TB/s an SM has about two issue slots for
// every lane's 16 bytes.  So head_dim / 16 lanes hold a row of a head, 16 elements each in two runs of 8 (every access of a warp covers whole 32-byte
// sectors on both sides), the cache's type is a template argument, the largest magnitude is found on the bit patterns, two bf16 at a time, and a
// row's place is looked up once for all heads.
// Measured on one B200, of 6.55 TB/s: 16 prompts of 2020 positions, 16 heads, bf16 into e4m3 37 us (83 %); 8 of 3550 out of e4m3 as bf16 35 us (78 %); bf16 into bf16 76 %, out 86 %; a step of
// 16 rows 2.9 us (launch, row, page table, place: four trips in a row).
#include "rt_paged.h"

namespace rt {
namespace {

constexpr int kThreads = 256;

// The exponent k of a row's scale 2^k: the smallest k >= -126 with amax <= 448 2^k, 448 = 1.75 * 2^8.  u: the bits of amax, finite.
__device__ __forceinline__ int scale_exponent(unsigned u) {
  const int k = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(k, -126);
}

__device__ __forceinline__ unsigned to_e4m3x2(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// a run of 8 elements as it lies in memory
template <typename T> struct Run;
template <> struct Run<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack8(v, f); }
  __device__ __forceinline__ unsigned magnitude() const {         // bits of the largest |x| as fp32 (NaN above infinity above all numbers)
    const unsigned m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m << 16, m & 0xffff0000u);
  }
};
template <> struct Run<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ __forceinline__ void get(float (&f)[8]) const { f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w; }
  __device__ __forceinline__ unsigned magnitude() const {
    float f[8];
    get(f);
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
    return m;
  }
};

// Two runs of a row of a head into its place, if `ok`.  The LPR lanes of a row are neighbours in a warp and agree on ok; all lanes call (shuffles).
template <typename T, typename CT, int LPR>
__device__ __forceinline__ void put_row(CT* to, uint8_t* e, int c, bool ok, const Run<T> (&x)[2]) {
  float f[2][8];
  x[0].get(f[0]);
  x[1].get(f[1]);
  if constexpr (sizeof(CT) == 1) {
    unsigned u = max(x[0].magnitude(), x[1].magnitude());
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) u = max(u, __shfl_xor_sync(0xffffffffu, u, o));
    if (__any_sync(0xffffffffu, u >= 0x7f800000u)) {               // infinities and NaN: stored as NaN, and not part of the maximum
      u = 0;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (isfinite(f[r][i])) u = max(u, __float_as_uint(f[r][i]) & 0x7fffffffu);
          else f[r][i] = __uint_as_float(0x7fffffffu);
        }
#pragma unroll
      for (int o = LPR / 2; o; o >>= 1) u = max(u, __shfl_xor_sync(0xffffffffu, u, o));
    }
    const int k = scale_exponent(u);
    const float s = __uint_as_float((unsigned)(127 - k) << 23);    // 2^-k: 127 - k is in [7, 253]
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      unsigned w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = to_e4m3x2(f[r][2 * i] * s, f[r][2 * i + 1] * s);
      if (ok) *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(to) + (c + r * LPR) * 8) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
    if (ok && c == 0) *e = (uint8_t)(k + 127);
  } else if (ok) {
    store8(to + c * 8, f[0]);
    store8(to + (c + LPR) * 8, f[1]);
  }
}

template <typename CT, int LPR> struct Held {                      // two runs of a row in the cache
  Run<CT> x[2];
  __device__ __forceinline__ void load(const CT* p, const uint8_t*, int c) { x[0].load(p + c * 8); x[1].load(p + (c + LPR) * 8); }
  __device__ __forceinline__ void get(int r, float (&f)[8]) const { x[r].get(f); }
};
template <int LPR> struct Held<__nv_fp8_e4m3, LPR> {
  uint2 w[2];
  unsigned e;
  __device__ __forceinline__ void load(const __nv_fp8_e4m3* p, const uint8_t* ep, int c) {
    w[0] = __ldg(reinterpret_cast<const uint2*>(p) + c);
    w[1] = __ldg(reinterpret_cast<const uint2*>(p) + c + LPR);
    e = __ldg(ep);
  }
  __device__ __forceinline__ void get(int r, float (&f)[8]) const {
    const float s = scale_of(e);
    const unsigned h[4] = {w[r].x, w[r].x >> 16, w[r].y, w[r].y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = from_e4m3x2(h[i]);
      f[2 * i] = y.x * s; f[2 * i + 1] = y.y * s;
    }
  }
};

// A warp takes the keys or the values of rows_per consecutive rows (at most 32).  Its lanes look their places up together, one row each: the chain row ->
// page table -> place costs two trips to memory however many rows there are.  Then it goes through the rows' heads, the next loads always under way.
template <typename T, typename CT, int LPR, bool WRITE>
__global__ void __launch_bounds__(kThreads, 3) cache_rows_kernel(const __grid_constant__ CacheRowsParams p, int rows_per, unsigned magic) {
  constexpr int HPW = 32 / LPR, HD = LPR * 16;                     // heads side by side in a warp
  constexpr int AHEAD = sizeof(T) == 4 && WRITE ? 1 : 2;           // passes over the heads in flight, and as many on their way
  const int lane = threadIdx.x & 31, c = lane % LPR, hl = lane / LPR, n_kv = p.c.n_kv_heads;
  const long long w = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), r0 = (w >> 1) * rows_per;
  const bool is_v = w & 1;
  if (r0 >= p.rows) return;
  const int n = (int)min((long long)rows_per, p.rows - r0);
  CT* pool = (CT*)(is_v ? p.c.v : p.c.k);
  uint8_t* exps = is_v ? p.c.v_exp : p.c.k_exp;
  const long long stride = is_v ? p.v_stride : p.k_stride;
  const T* in = WRITE ? (const T*)(is_v ? p.v_in : p.k_in) + (size_t)r0 * stride : nullptr;
  T* out = WRITE ? nullptr : (T*)(is_v ? p.v_out : p.k_out) + (size_t)r0 * stride;
  long long place = -1;                                            // of lane i: the first head's row of position pos[r0 + i]
  if (lane < n) {
    const int b = __ldg(p.seq + r0 + lane), t = __ldg(p.pos + r0 + lane);
    if (t >= 0) {
      int page = -1;
      if ((unsigned)b < (unsigned)p.c.n_seqs && (t >> p.log_page) < p.c.max_pages) page = page_at(p.c, b, t >> p.log_page);
      else if (p.c.status) *p.c.status = RT_ERR_INVALID_ARG;
      if (page >= 0) place = (long long)page * n_kv * p.c.page_size + (t & (p.c.page_size - 1));
    }
  }
  struct Buffer { Run<T> x[WRITE ? AHEAD : 1][2]; Held<CT, LPR> y[WRITE ? 1 : AHEAD]; };
  // The rows' heads in one line, HPW side by side: head y % n_kv of row y / n_kv.  (Lanes behind the end repeat the last one for the shuffles; rows that are
  // not in use are read from place 0, which is there, and left.)
  const int total = n * n_kv;
  auto row_of = [&](int y) { return magic ? (int)__umulhi((unsigned)y, magic) : y / n_kv; };
  auto load = [&](Buffer& b, int y0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int y = min(y0 + u * HPW + hl, total - 1), i = row_of(y), h = y - i * n_kv;
      if constexpr (WRITE) {
        const T* from = in + (size_t)i * stride + h * HD;
        b.x[u][0].load(from + c * 8);
        b.x[u][1].load(from + (c + LPR) * 8);
      } else {
        const size_t row = (size_t)max(__shfl_sync(0xffffffffu, place, i), 0LL) + (size_t)h * p.c.page_size;
        b.y[u].load(pool + row * HD, exps + (sizeof(CT) == 1 ? row : 0), c);
      }
    }
  };
  Buffer now, next;
  load(now, 0);
  for (int y0 = 0; y0 < total; y0 += HPW * AHEAD) {
    if (y0 + HPW * AHEAD < total) load(next, y0 + HPW * AHEAD);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (y0 + u * HPW >= total) break;
      const int y = y0 + u * HPW + hl, yc = min(y, total - 1), i = row_of(yc), h = yc - i * n_kv;
      const long long row0 = __shfl_sync(0xffffffffu, place, i);
      const bool ok = y < total && row0 >= 0;
      if constexpr (WRITE) {
        const size_t row = (size_t)max(row0, 0LL) + (size_t)h * p.c.page_size;
        put_row<T, CT, LPR>(pool + row * HD, exps + (sizeof(CT) == 1 ? row : 0), c, ok, now.x[u]);
      } else if (ok) {
        T* to = out + (size_t)i * stride + h * HD;
        float f[8];
        now.y[u].get(0, f);
        store8(to + c * 8, f);
        now.y[u].get(1, f);
        store8(to + (c + LPR) * 8, f);
      }
    }
    now = next;
  }
}

template <typename T, typename CT, bool WRITE>
cudaError_t launch(const CacheRowsParams& p, cudaStream_t s) {
  // several rows a warp once there are more than the GPU's warps (24 an SM) take one of
  const int rows_per = (int)min(32LL, max(1LL, ((long long)p.rows * 2 + 148 * 24 - 1) / (148 * 24)));
  const long long warps = ((long long)p.rows + rows_per - 1) / rows_per * 2;
  const dim3 grid((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32)));
  // ceil(2^32 / n_kv): y / n_kv is the high word of y * magic while y * (magic * n_kv - 2^32) < 2^32, and y < 32 n_kv, that factor < n_kv
  const unsigned n_kv = (unsigned)p.c.n_kv_heads, magic = n_kv > 1 && n_kv < 8192 ? (unsigned)((0x100000000ull + n_kv - 1) / n_kv) : 0u;
  if (p.c.head_dim == 64) cache_rows_kernel<T, CT, 4, WRITE><<<grid, kThreads, 0, s>>>(p, rows_per, magic);
  else cache_rows_kernel<T, CT, 8, WRITE><<<grid, kThreads, 0, s>>>(p, rows_per, magic);
  return cudaGetLastError();
}
template <typename T, bool WRITE>
cudaError_t launch_by_cache(const CacheRowsParams& p, cudaStream_t s) {
  if (p.c.dtype == RT_E4M3) return launch<T, __nv_fp8_e4m3, WRITE>(p, s);
  return p.c.dtype == RT_BF16 ? launch<T, __nv_bfloat16, WRITE>(p, s) : launch<T, float, WRITE>(p, s);
}

}  // namespace

cudaError_t cache_write_launch(int dtype, const CacheRowsParams& p, cudaStream_t s) {
  return dtype == RT_BF16 ? launch_by_cache<__nv_bfloat16, true>(p, s) : launch_by_cache<float, true>(p, s);
}
cudaError_t cache_read_launch(int dtype, const CacheRowsParams& p, cudaStream_t s) {
  return dtype == RT_BF16 ? launch_by_cache<__nv_bfloat16, false>(p, s) : launch_by_cache<float, false>(p, s);
}

}  // namespace rt
