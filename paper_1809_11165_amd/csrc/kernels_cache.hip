// Rows into the pages of a cache, and back (see include/bbmm.h, "Cache").  A few lanes take a row, 16 bytes of the wide side each; 8-bit blocks of 32
// features are four or eight of these lanes.  Bound by memory, single rows by their launch: rows are read and written once, in whole
// pieces of 128 bytes and more.
#include "cache_dev.h"

using namespace att;

namespace {

// Largest over the lanes of a block: 4 (two-byte types) or 8 neighbours.
template <int L>
__device__ __forceinline__ float block_max(float x) {
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, true)));
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, true)));
  if constexpr (L == 8) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true)));
  return x;
}

// Where row i of entry b lies in the cache.
struct Place {
  int page, row;
  __device__ __forceinline__ Place(const CacheArgs& c, int b, int64_t at) {
    page = -1;
    if (at >= 0 && at < c.rows_most) {
      uint32_t n = over((uint32_t)at, c.page);
      row = (int)((uint32_t)at - n * c.page.d);
      page = page_of(c, b, n);
    }
  }
  __device__ __forceinline__ int64_t element(const int64_t* s, int h) const { return page * s[0] + row * s[1] + h * s[2]; }
  __device__ __forceinline__ int64_t exps(const CacheArgs& c, int h) const { return (((int64_t)page * c.HK + h) * c.page.d + row) * 4; }
};

constexpr int kRows = 4;                                   // rows of a group of lanes

template <typename T, bool E4M3, int DP>
__global__ __launch_bounds__(256) void k_cache_write(CacheArgs c, CacheMove m, int64_t n, int blocks) {
  constexpr int E = 16 / (int)sizeof(T), L = DP / E, GP = 256 / L;
  int tid = threadIdx.x, which = blockIdx.x >= (unsigned)blocks, lane = tid % L, at = lane * E;
  int64_t r0 = (int64_t)(blockIdx.x - (which ? blocks : 0)) * GP * kRows + tid / L;
  const T* src = (const T*)(which ? m.V : m.K);
  const int64_t *ss = which ? m.vs : m.ks, *ds = which ? c.vs : c.ks;
  int width = which ? c.dv : c.d, vec = which ? m.vvec : m.kvec;
  u32x4 x[kRows];
  int64_t to[kRows], ex[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    int64_t r = r0 + k * GP;
    to[k] = -1;
    if (r >= n) continue;
    uint32_t tok = over((uint32_t)r, m.by_heads), b = over(tok, m.by_rows);
    int h = (int)((uint32_t)r - tok * (uint32_t)c.HK), i = (int)(tok - b * (uint32_t)m.rows);
    if (m.n && i >= m.n[b]) continue;
    x[k] = load16<T>(src + (int64_t)b * ss[0] + (int64_t)i * ss[1] + (int64_t)h * ss[2], at, width, vec);
    Place p(c, (int)b, (int64_t)(m.start ? m.start[b] : 0) + i);
    if (p.page < 0) continue;
    to[k] = p.element(ds, h);
    if constexpr (E4M3) ex[k] = p.exps(c, h);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (to[k] < 0) continue;
    if constexpr (E4M3) {
      const T* v = reinterpret_cast<const T*>(&x[k]);
      float f[E], top = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        f[e] = (float)v[e];
        bool finite = fabsf(f[e]) < __builtin_inff();
        if (!finite) f[e] = __builtin_nanf("");
        top = fmaxf(top, finite ? fabsf(f[e]) : 0.f);
      }
      int e = block_exp(block_max<32 / E>(top));
      float down = power(-e);
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] *= down;
      if (e == (__is_same(T, _Float16) ? 8 : 120)) {       // 256 2^e is beyond T
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = f[i] > 240.f ? 240.f : f[i] < -240.f ? -240.f : f[i];
      }
      unsigned q[E / 4];
#pragma unroll
      for (int w = 0; w < E / 4; ++w) {
        int d = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * w], f[4 * w + 1], 0, false);
        q[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * w + 2], f[4 * w + 3], d, true);
      }
      uint8_t* row = (uint8_t*)(which ? c.V : c.K) + to[k] + at;
      if (at < (width + 15) / 16 * 16) {
        if constexpr (E == 8) *(uint2*)row = make_uint2(q[0], q[1]);
        else *(unsigned*)row = q[0];
      }
      if (lane % (32 / E) == 0 && at < width) (which ? c.ve : c.ke)[ex[k] + at / 32] = (uint8_t)(e + 127);
    } else {
      if (at < width) *(u32x4*)((T*)(which ? c.V : c.K) + to[k] + at) = x[k];
    }
  }
}

template <typename T, bool E4M3, int DP>
__global__ __launch_bounds__(256) void k_cache_read(CacheArgs c, CacheMove m, int64_t n, int blocks) {
  constexpr int E = 16 / (int)sizeof(T), L = DP / E, GP = 256 / L;
  int tid = threadIdx.x, which = blockIdx.x >= (unsigned)blocks, lane = tid % L, at = lane * E;
  int64_t r0 = (int64_t)(blockIdx.x - (which ? blocks : 0)) * GP * kRows + tid / L;
  T* dst = (T*)(which ? m.V : m.K);
  const int64_t* ss = which ? c.vs : c.ks;
  int width = which ? c.dv : c.d, vec = which ? m.vvec : m.kvec;
  u32x4 x[kRows];
  float scale[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    int64_t r = r0 + k * GP;
    x[k] = u32x4{0u, 0u, 0u, 0u};
    scale[k] = 1.f;
    if (r >= n || at >= width) continue;
    uint32_t tok = over((uint32_t)r, m.by_heads), b = over(tok, m.by_rows);
    int h = (int)((uint32_t)r - tok * (uint32_t)c.HK), i = (int)(tok - b * (uint32_t)m.rows);
    int64_t j = (int64_t)(m.start ? m.start[b] : 0) + i;
    if (m.n && j >= m.n[b]) continue;
    Place p(c, (int)b, j);
    if (p.page < 0) continue;
    if constexpr (E4M3) {
      const uint8_t* row = (const uint8_t*)(which ? c.V : c.K) + p.element(ss, h) + at;
      if constexpr (E == 8) {
        uint2 q = *(const uint2*)row;
        x[k][0] = q.x, x[k][1] = q.y;
      } else {
        x[k][0] = *(const unsigned*)row;
      }
      scale[k] = block_scale((which ? c.ve : c.ke)[p.exps(c, h) + at / 32], 0);
    } else {
      x[k] = *(const u32x4*)((const T*)(which ? c.V : c.K) + p.element(ss, h) + at);
    }
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    int64_t r = r0 + k * GP;
    if (r >= n || at >= width) continue;
    u32x4 y = x[k];
    if constexpr (E4M3) {
      typedef typename Wide<T>::two two;
      two* t = reinterpret_cast<two*>(&y);
#pragma unroll
      for (int w = 0; w < E / 4; ++w) {
        t[2 * w] = Wide<T>::template get<false>(x[k][w], scale[k]);
        t[2 * w + 1] = Wide<T>::template get<true>(x[k][w], scale[k]);
      }
    }
    T* row = dst + r * width;
    if (vec) {
      *(u32x4*)(row + at) = y;
    } else {
      const T* e = reinterpret_cast<const T*>(&y);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (at + i < width) row[at + i] = e[i];
    }
  }
}

template <typename T, bool E4M3>
void move_t(hipStream_t s, bool write, const CacheArgs& c, const CacheMove& m) {
  int64_t n = (int64_t)c.B * m.rows * c.HK;
  int most = c.d > c.dv ? c.d : c.dv;
  auto run = [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    int per = 256 / (DP * (int)sizeof(T) / 16) * kRows, blocks = (int)((n + per - 1) / per);
    if (write) k_cache_write<T, E4M3, DP><<<2 * blocks, 256, 0, s>>>(c, m, n, blocks);
    else k_cache_read<T, E4M3, DP><<<2 * blocks, 256, 0, s>>>(c, m, n, blocks);
  };
  if (most <= 32) run(Const<32>{});
  else if (most <= 64) run(Const<64>{});
  else run(Const<128>{});
}
template <typename T>
void move(hipStream_t s, bool write, int e4m3, const CacheArgs& c, const CacheMove& m) {
  if (e4m3) move_t<T, true>(s, write, c, m);
  else move_t<T, false>(s, write, c, m);
}
void move_any(hipStream_t s, bool write, int type, int e4m3, const CacheArgs& c, const CacheMove& m) {
  if (type == 0) move<float>(s, write, e4m3, c, m);
  else if (type == 1) move<_Float16>(s, write, e4m3, c, m);
  else move<__bf16>(s, write, e4m3, c, m);
}

}  // namespace

void launch_cache_write(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheMove& m) { move_any(s, true, type, e4m3, c, m); }
void launch_cache_read(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheMove& m) { move_any(s, false, type, e4m3, c, m); }
