// Rows into the pages of a cache, and back (see include/bbmm.h, "Cache").  A few lanes take a row, 16 bytes of the wide side each; 8-bit blocks of 32
// features are four or eight of these lanes:  e = least with max |x| / 2^e <= 448,  q = round(x / 2^e),  and back  x = q 2^e.
// Bound by memory, single rows by their launch: rows are read and written once, in whole pieces of 128 bytes and more.  4 x 2048 rows of 8 heads of
// 128 from bf16 into 8-bit pages, 51 MB: 15.1 us, 3.4 TB/s (a workgroup's rows end together, and the next one's places are looked up anew);
// 4 x 8192 read back, 204 MB: 35.3 us, 5.8 TB/s; one row of eight requests: 3.2 us, three loads in a chain and the launch.
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

// The rows of a group of lanes, kRows neighbouring (row, head) each, and where they lie in the cache.  Every step is taken for all rows before the
// next: loads in branches of their own would be waited for one by one (268 MB of bf16 rows read back and written: 128 us, so 57).  Rows that are not there
// have some place that may be read, and `there` unset.
template <int kRows>
struct Rows {
  int b[kRows], i[kRows], h[kRows], page[kRows], row[kRows];
  bool have[kRows], there[kRows];                          // a row of the call; and its place exists
  // READ: rows are those before n[b] of the sequence; else the call's rows i < n[b]
  template <bool READ>
  __device__ __forceinline__ void find(const CacheArgs& c, const CacheMove& m, int64_t r0, int64_t total) {
    int first[kRows], n[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      have[k] = r0 + k < total;
      uint32_t r = (uint32_t)min(r0 + k, total - 1), tok = over(r, m.by_heads), e = over(tok, m.by_rows);
      h[k] = (int)(r - tok * (uint32_t)c.HK), i[k] = (int)(tok - e * (uint32_t)m.rows), b[k] = (int)e;
      first[k] = 0, n[k] = INT32_MAX;
    }
    if (m.start) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) first[k] = m.start[b[k]];
    }
    if (m.n) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) n[k] = m.n[b[k]];
    }
    uint32_t index[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      int64_t at = (int64_t)first[k] + i[k];
      there[k] = have[k] && at >= 0 && at < c.rows_most && (READ ? at : (int64_t)i[k]) < n[k];
      uint32_t j = there[k] ? (uint32_t)at : 0u;
      index[k] = over(j, c.page);
      row[k] = (int)(j - index[k] * c.page.d);
      page[k] = -1;
    }
    if (c.max_pages > 0) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) page[k] = page_of(c, b[k], index[k]);
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      there[k] = there[k] && page[k] >= 0;
      page[k] = there[k] ? page[k] : 0;
    }
  }
  __device__ __forceinline__ int64_t element(const int64_t* s, int k) const { return page[k] * s[0] + row[k] * s[1] + h[k] * s[2]; }
  __device__ __forceinline__ int64_t exps(const CacheArgs& c, int k) const { return (((int64_t)page[k] * c.HK + h[k]) * c.page.d + row[k]) * 4; }
};

template <typename T, bool E4M3, int DP, int kRows>
__global__ __launch_bounds__(256) void k_cache_write(CacheArgs c, CacheMove m, int64_t n, int blocks) {
  constexpr int E = 16 / (int)sizeof(T), L = DP / E, GP = 256 / L;
  int tid = threadIdx.x, which = blockIdx.x >= (unsigned)blocks, lane = tid % L, at = lane * E;
  int64_t r0 = ((int64_t)(blockIdx.x - (which ? blocks : 0)) * GP + tid / L) * kRows;
  const T* src = (const T*)(which ? m.V : m.K);
  const int64_t *ss = which ? m.vs : m.ks, *ds = which ? c.vs : c.ks;
  int width = which ? c.dv : c.d;
  Rows<kRows> rows;
  rows.template find<false>(c, m, r0, n);
  u32x4 x[kRows];
  auto from = [&](int k) { return src + (int64_t)rows.b[k] * ss[0] + (int64_t)rows.i[k] * ss[1] + (int64_t)rows.h[k] * ss[2]; };
  if (which ? m.vvec : m.kvec) {
#pragma unroll
    for (int k = 0; k < kRows; ++k) x[k] = *(const u32x4*)(from(k) + (at < width ? at : 0));
    if (at >= width) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) x[k] = u32x4{0u, 0u, 0u, 0u};
    }
  } else {
#pragma unroll
    for (int k = 0; k < kRows; ++k) x[k] = load16<T>(from(k), at, width, 0);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
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
      if (!rows.there[k]) continue;
      uint8_t* row = (uint8_t*)(which ? c.V : c.K) + rows.element(ds, k) + at;
      if (at < (width + 15) / 16 * 16) {
        if constexpr (E == 8) *(uint2*)row = make_uint2(q[0], q[1]);
        else *(unsigned*)row = q[0];
      }
      if (lane % (32 / E) == 0 && at < width) (which ? c.ve : c.ke)[rows.exps(c, k) + at / 32] = (uint8_t)(e + 127);
    } else {
      if (rows.there[k] && at < width) *(u32x4*)((T*)(which ? c.V : c.K) + rows.element(ds, k) + at) = x[k];
    }
  }
}

template <typename T, bool E4M3, int DP, int kRows>
__global__ __launch_bounds__(256) void k_cache_read(CacheArgs c, CacheMove m, int64_t n, int blocks) {
  constexpr int E = 16 / (int)sizeof(T), L = DP / E, GP = 256 / L;
  int tid = threadIdx.x, which = blockIdx.x >= (unsigned)blocks, lane = tid % L, at = lane * E;
  int64_t r0 = ((int64_t)(blockIdx.x - (which ? blocks : 0)) * GP + tid / L) * kRows;
  T* dst = (T*)(which ? m.V : m.K);
  const int64_t* ss = which ? c.vs : c.ks;
  int width = which ? c.dv : c.d, vec = which ? m.vvec : m.kvec;
  Rows<kRows> rows;
  rows.template find<true>(c, m, r0, n);
  u32x4 x[kRows];
  float scale[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) x[k] = u32x4{0u, 0u, 0u, 0u};
  if (c.pages > 0) {
    int col = at < width ? at : 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      if constexpr (E4M3) {
        const uint8_t* row = (const uint8_t*)(which ? c.V : c.K) + rows.element(ss, k) + col;
        if constexpr (E == 8) {
          uint2 q = *(const uint2*)row;
          x[k][0] = q.x, x[k][1] = q.y;
        } else {
          x[k][0] = *(const unsigned*)row;
        }
        scale[k] = block_scale((which ? c.ve : c.ke)[rows.exps(c, k) + col / 32], 0);
      } else {
        x[k] = *(const u32x4*)((const T*)(which ? c.V : c.K) + rows.element(ss, k) + col);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
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
    if (!rows.there[k]) y = u32x4{0u, 0u, 0u, 0u};
    T* row = dst + (r0 + k) * width;
    if (!rows.have[k] || at >= width) continue;
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
  auto rows = [&](auto dp, auto r) {
    constexpr int DP = decltype(dp)::value, R = decltype(r)::value;
    int per = 256 / (DP * (int)sizeof(T) / 16) * R, blocks = (int)((n + per - 1) / per);
    if (write) k_cache_write<T, E4M3, DP, R><<<2 * blocks, 256, 0, s>>>(c, m, n, blocks);
    else k_cache_read<T, E4M3, DP, R><<<2 * blocks, 256, 0, s>>>(c, m, n, blocks);
  };
  // Eight rows a group where that still leaves a thousand workgroups; else one, whose steps take an eighth of the time (8-bit rows of 8 heads written
  // and read back, eight / one: 8 x 100 rows 10.1 / 6.1 us, 2 x 600 12.2 / 8.6, 4 x 1000 17.5 / 16.2).
  auto run = [&](auto dp) {
    constexpr int per = 256 / (decltype(dp)::value * (int)sizeof(T) / 16);
    if (n >= (int64_t)2048 * per) rows(dp, Const<8>{});
    else rows(dp, Const<1>{});
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
