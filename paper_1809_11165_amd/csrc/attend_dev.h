// Device pieces shared by the attention kernels: types, matrix fragments, LDS tiles, staging and the bias line.
//
// All matrix work is done by 32 x 32 MFMA blocks whose first operand comes from an LDS tile and whose second one stays in
// registers.  The result has its column in lane % 32 and rows 8 (r / 4) + 4 (lane / 32) + r % 4 in registers r = 0 .. 15.  The
// eight values that a second operand of the next product wants per lane may be ANY eight of its 16 summed indices, as long as the first
// operand's lane holds the same ones: so registers 8 u .. 8 u + 7 of a result are that operand as they stand (index
// 16 u + 8 (e / 4) + 4 (lane / 32) + e % 4), and scores turn into weights of the next product without leaving their lane.
#pragma once

#include "bbmm_attend.h"

namespace att {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kPad = 64;                                  // the bias line goes this far beyond the last edge
constexpr int kLine = 2 * (BBMM_ATT_FAR + kPad) + 1;

template <int V> struct Const { static constexpr int value = V; };

template <typename T> struct Frag;
template <> struct Frag<__bf16> {
  typedef bf16x8 type;
  static __device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Frag<_Float16> {
  typedef f16x8 type;
  static __device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Frag<float> {
  typedef f32x8 type;
  static __device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

// Eight registers of a result as the second operand of the next product (rounded to T once).
template <typename T>
__device__ __forceinline__ typename Frag<T>::type pack8(const f32x16& c, int u) {
  typename Frag<T>::type f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (T)c[8 * u + e];
  return f;
}

// ---- LDS tiles: rows of DP elements; the 16-byte pieces of row r stand in places c ^ swz(r).  A cycle of the LDS serves 256 bytes: 16 lanes
// of a row_frag (16 rows, one piece each), 32 lanes of a 16-bit col_frag (four rows, four neighbouring pieces) or all 64 of an fp32
// one (two rows four apart, 128 bytes each).  swz puts each of these on 16 different places of 256 bytes: no bank conflicts.  (With the pieces
// spread over 128 bytes only, a forward pass of 4096 x 10000, d = 128, spent 40 % of its LDS cycles on conflicts.)
template <typename T, int DP>
__device__ __forceinline__ int swz(int r) {
  if constexpr (sizeof(T) == 4) return (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1);
  else if constexpr (DP >= 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);      // two rows share 256 bytes
}

// First operand: element e of the lane = tile[rb + lane % 32][16 s + 8 (lane / 32) + e];  rb a multiple of 32.
template <typename T, int DP>
__device__ __forceinline__ typename Frag<T>::type row_frag(const char* tile, int rb, int s, int lane) {
  constexpr int kRow = DP * (int)sizeof(T);
  int r = lane & 31, half = lane >> 5, f = swz<T, DP>(r);
  const char* p = tile + (rb + r) * kRow;
  if constexpr (sizeof(T) == 2) {
    return *(const typename Frag<T>::type*)(p + (((2 * s + half) ^ f) << 4));
  } else {
    f32x4 lo = *(const f32x4*)(p + (((4 * s + 2 * half) ^ f) << 4));
    f32x4 hi = *(const f32x4*)(p + (((4 * s + 2 * half + 1) ^ f) << 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// First operand, transposed: element e of the lane = tile[rb + 8 (e / 4) + 4 (lane / 32) + e % 4][cb + lane % 32]; rb a multiple of
// 16, cb of 32.  Two-byte types by the transposing LDS read: 16 lanes read a block of four rows of 16 elements, eight bytes
// each (lane L: row L / 4, elements 4 (L % 4) on), and receive a column each.
template <typename T, int DP>
__device__ __forceinline__ typename Frag<T>::type col_frag(const char* tile, int rb, int cb, int lane) {
  constexpr int kRow = DP * (int)sizeof(T);
  int half = lane >> 5;
  typename Frag<T>::type f;
  if constexpr (sizeof(T) == 2) {
    int L = lane & 15, r = 4 * half + (L >> 2);
    int c = (cb >> 3) + 2 * ((lane >> 4) & 1) + ((L & 3) >> 1);
    const char* p = tile + (rb + r) * kRow + ((L & 1) << 3);
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + ((c ^ swz<T, DP>(r)) << 4)));
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * kRow + ((c ^ swz<T, DP>(r + 8)) << 4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    f = __builtin_bit_cast(typename Frag<T>::type, v);
  } else {
    int col = cb + (lane & 31);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      int r = 8 * (e >> 2) + 4 * half + (e & 3);
      f[e] = *(const float*)(tile + (rb + r) * kRow + (((col >> 2) ^ swz<T, DP>(r)) << 4) + ((col & 3) << 2));
    }
  }
  return f;
}

// Memory from `base` on with hardware bounds: reads at or behind `bytes` give zero.
// (The bound has to be in a scalar register: a lane's bound would be taken one lane after the other.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bounded(const void* base, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}
constexpr unsigned kNowhere = 0x80000000u;   // an offset behind every bound (bounds are below 2^31: wide operands only)

// 16 bytes of a row: elements [c, c + 16 / sizeof(T)) of `row`, zero from element `width` on.
template <typename T>
__device__ __forceinline__ u32x4 load16(const T* row, int c, int width, int vec) {
  constexpr int E = 16 / (int)sizeof(T);
  u32x4 v = {0u, 0u, 0u, 0u};
  if (c >= width) return v;
  if (vec) return *(const u32x4*)(row + c);
  T* e = reinterpret_cast<T*>(&v);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (c + i < width) e[i] = row[c + i];
  return v;
}

// A tile of ROWS rows on its way from memory to LDS: 256 threads, 16 bytes each per pass.  VEC: rows may be read 16 bytes at a time and a
// tile spans less than 2^31 bytes.
template <typename T, int DP, int ROWS, bool VEC>
struct Stage {
  static constexpr int E = 16 / (int)sizeof(T), CH = DP / E, RP = 256 / CH, N = ROWS / RP;
  u32x4 v[N];
  // row 0 of the tile at `base`; what is read of rows from `rows` on is within bounds, or zero, and means nothing
  __device__ __forceinline__ void load(const T* base, int64_t stride, int rows, int width, int tid) {
    int r = tid / CH, c = (tid % CH) * E;
    if constexpr (VEC) {
      unsigned pitch = (unsigned)stride * (unsigned)sizeof(T), last = (unsigned)width * (unsigned)sizeof(T);
      unsigned n = rows >= ROWS ? (unsigned)(ROWS - 1) * pitch + last : rows > 0 ? (unsigned)(rows - 1) * pitch + last : 0u;
      __amdgpu_buffer_rsrc_t mem = bounded(base, n);
      unsigned at = c < width ? (unsigned)r * pitch + (unsigned)c * (unsigned)sizeof(T) : kNowhere;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b128(mem, at + (unsigned)(i * RP) * pitch, 0, 0);
    } else {
      const T* p = base + (int64_t)r * stride;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = u32x4{0u, 0u, 0u, 0u};
        if (r + i * RP < rows) v[i] = load16<T>(p, c, width, 0);
        p += (int64_t)RP * stride;
      }
    }
  }
  // rows without a bit in `keep` are stored as zeros, whatever they held
  __device__ __forceinline__ void store(char* tile, uint64_t keep, int tid) const {
    int r = tid / CH, c = tid % CH;
    if (keep == ~0ull || (ROWS == 32 && keep == 0xffffffffull)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        int row = r + i * RP;
        *(u32x4*)(tile + row * DP * (int)sizeof(T) + ((c ^ swz<T, DP>(row)) << 4)) = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        int row = r + i * RP;
        u32x4 x = v[i];
        if (!((keep >> row) & 1)) x = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(tile + row * DP * (int)sizeof(T) + ((c ^ swz<T, DP>(row)) << 4)) = x;
      }
    }
  }
};

// Second operand kept in registers: element e = row[16 s + 8 (lane / 32) + e], zero where there is no row.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type reg_frag(const T* row, bool have, int s, int width, int vec, int lane) {
  int c = 16 * s + 8 * (lane >> 5);
  typename Frag<T>::type f;
  if constexpr (sizeof(T) == 2) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (have) v = load16<T>(row, c, width, vec);
    f = __builtin_bit_cast(typename Frag<T>::type, v);
  } else {
    u32x4 lo = {0u, 0u, 0u, 0u}, hi = lo;
    if (have) {
      lo = load16<T>(row, c, width, vec);
      hi = load16<T>(row, c + 4, width, vec);
    }
    f = __builtin_shufflevector(__builtin_bit_cast(f32x4, lo), __builtin_bit_cast(f32x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return f;
}

// ---- buckets
// The edges are read at uniform places (scalar loads), eight at a time; places behind the last edge hold the largest int.
__device__ __forceinline__ int bucket_of(const AttBuckets& bk, int r) {
  int dist = bk.two_sided ? abs(r) : max(-r, 0), n = 0;
  for (int k = 0; k < bk.n_edges; k += 8)
#pragma unroll
    for (int e = 0; e < 8; ++e) n += bk.edges[k + e] <= dist;
  return n + ((bk.two_sided && r > 0) ? bk.n_edges + 1 : 0);
}

// Sums by bucket of a workgroup of 256: diag[r + span] holds the sum of difference r, |r| <= span; `left` and `right` are sums of differences
// -far and below, far and above.  A bucket is an interval of differences on one side; eight lanes take one.
template <typename S>
__device__ __forceinline__ void bucket_sums(const AttBuckets& bk, const float* diag, int span, S left, S right, S* out, int tid) {
  int E = bk.n_edges, part = tid & 7;
  for (int n = tid >> 3; n < bk.buckets; n += 32) {
    bool ahead = n > E;                                   // two-sided, r > 0
    int c = ahead ? n - E - 1 : n;
    int near = c ? bk.edges[c - 1] : 0, beyond = c < E ? bk.edges[c] - 1 : span;
    beyond = min(beyond, span);
    int lo = ahead ? max(near, 1) : -beyond, hi = ahead ? beyond : -near;
    if (!bk.two_sided && n == 0) hi = span;
    S s = 0;
    for (int r = lo + part; r <= hi; r += 8) s += diag[r + span];
#pragma unroll
    for (int x = 1; x < 8; x *= 2) s += __shfl_xor(s, x, 64);
    if (n == E) s += left;
    if (n == (bk.two_sided ? 2 * E + 1 : 0)) s += right;
    if (part == 0) out[n] = s;
  }
}

// One wave: the sums of a head's bucket from all parts (tsum: heads x parts x buckets) in a fixed order, 64 bits.
template <typename T, typename S>
__device__ __forceinline__ void join_bucket(const S* __restrict__ tsum, int parts, int buckets, int h, int n, int lane, T* __restrict__ out) {
  double s = 0.0;
  for (int p = lane; p < parts; p += 64) s += (double)tsum[((size_t)h * parts + p) * buckets + n];
#pragma unroll
  for (int x = 1; x < 64; x *= 2) s += __shfl_xor(s, x, 64);
  if (lane == 0) out[(size_t)h * buckets + n] = (T)(float)s;
}

// Adds the 32 x 32 block s (keys in the registers, queries in the lanes) along its diagonals: line[j - i] += sum, `line` (the wave's own)
// pointing at the difference of the first key and the first query.  Halves first exchange registers so that each
// has 16 keys in a row; a sum then moves one lane per key, towards higher lanes for keys ahead (what leaves a row of 16 lanes
// lies behind), towards lower ones for keys behind.  That leaves two pieces of a diagonal in each row of 16 lanes, which rows exchange until every lane
// owns a diagonal of the block: one read and one write of LDS in a fixed order, no atomics.  (dQ pass of 8 x 12 x 512 x 640 in bf16, d = 64,
// with delta from O: 31 us; with two atomic additions per half 38, with sixteen of all lanes 106 before other steps.)
__device__ __forceinline__ float from_lane_below(float x) {   // of the row of 16, zero into the first
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x111, 0xf, 0xf, true));
}
__device__ __forceinline__ float from_lane_above(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x101, 0xf, 0xf, true));
}
__device__ __forceinline__ void add_diagonals(const f32x16& s, float* line, int lane) {
  float k[16];                                              // key 16 (lane / 32) + index
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      auto x = __builtin_amdgcn_permlane32_swap(__float_as_int(s[4 * g + e]), __float_as_int(s[4 * (g + 2) + e]), false, false);
      k[8 * g + e] = __int_as_float(x[0]);
      k[8 * g + 4 + e] = __int_as_float(x[1]);
    }
  float ahead = k[0], behind = k[15];
#pragma unroll
  for (int i = 1; i < 16; ++i) {
    ahead = from_lane_below(ahead) + k[i];
    behind = from_lane_above(behind) + k[15 - i];
  }
  behind = from_lane_above(behind);
  // Rows of 16 lanes X0 .. X3 of `ahead` and Y0 .. Y3 of `behind`; with 15 - lane % 16 added, X stand at 0, -16, 16, 0 and Y at -16, -32, 0, -16.
  typedef float pair __attribute__((ext_vector_type(2)));
  auto swap16 = [](float x, float y) {      // odd rows of x against even rows of y
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(y), false, false);
    return pair{__int_as_float(r[0]), __int_as_float(r[1])};
  };
  auto swap32 = [](float x, float y) {      // rows 2, 3 of x against rows 0, 1 of y
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(y), false, false);
    return pair{__int_as_float(r[0]), __int_as_float(r[1])};
  };
  pair t = swap16(ahead, behind);           // X0 Y0 X2 Y2,  X1 Y1 X3 Y3
  t = swap32(t[0], t[1]);                   // X0 Y0 X1 Y1,  X2 Y2 X3 Y3
  float c = t[0];
  pair d = swap16(t[1], t[1]);              // X2 X2 X3 X3,  Y2 Y2 Y3 Y3
  pair e = swap16(c, c);                    // X0 X0 X1 X1,  Y0 Y0 Y1 Y1
  pair f = swap32(d[0], e[1]);              // X2 X2 Y0 Y0,  X3 X3 Y1 Y1
  bool odd = lane & 16, up = lane & 32;
  float z = c + d[1] + (up ? f[0] : f[1]);  // rows 0: X0 + Y2 + X3,  2: X1 + Y3 + Y0
  if (odd) z = up ? c : f[0];               // rows 1: X2,  3: Y1
  float* mine = line + 15 - (lane & 15) + (odd ? (up ? -32 : 16) : up ? -16 : 0);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // another lane's write of the block before
  __builtin_amdgcn_wave_barrier();
  *mine += z;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A table entry in units of the base-2 exponent.  Finite entries stay finite: one beyond 2.3e38 in magnitude counts as that (below, the same
// weight zero beside any other score, and weights of its own where a row holds nothing else; above, all of the row's weight).
template <typename T>
__device__ __forceinline__ float bias2(T t) {
  constexpr float kMost = 3.40282347e38f;
  float x = (float)t;
  float y = x * kLog2e;
  return fabsf(x) < __builtin_inff() ? fminf(fmaxf(y, -kMost), kMost) : y;
}

// line[r + far + kPad] = bias of difference r, |r| <= far + kPad, for one head.
template <typename T>
__device__ __forceinline__ void fill_line(float* line, const AttArgs& a, int h, int tid, int threads) {
  int n = 2 * (a.bk.far + kPad) + 1;
  const T* tab = (const T*)a.table + (size_t)h * a.bk.buckets;
  for (int i = tid; i < n; i += threads) line[i] = bias2<T>(tab[bucket_of(a.bk, i - a.bk.far - kPad)]);
}

// A value that all lanes hold, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __int_as_float(uniform(__float_as_int(x))); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(((uint64_t)(unsigned)uniform((int)(x >> 32)) << 32) | (unsigned)uniform((int)x));
}
__device__ __forceinline__ int queries_of(const AttArgs& a, int b) { return a.q_len ? uniform(min(max(a.q_len[b], 0), a.nq)) : a.nq; }
__device__ __forceinline__ int keys_of(const AttArgs& a, int b) { return a.k_len ? uniform(min(max(a.k_len[b], 0), a.nk)) : a.nk; }

// Waits for all loads issued so far.  Stands before a loop whose operands were loaded ahead of it: without it the compiler's own
// counting, which meets the loop's loads and those together at the loop's head, waits for the prefetched tile in every turn.
__device__ __forceinline__ void settle() { __builtin_amdgcn_s_waitcnt(0x0f70); }

__device__ __forceinline__ int clamp_rel(int64_t r) {
  const int64_t lim = 1 << 30;
  return (int)(r < -lim ? -lim : (r > lim ? lim : r));
}

// x - y + z of a running y (or z) from 0 to 2^30 and a fixed rest r, as 32 bits: differences that leave the line of the bias stay outside.
__device__ __forceinline__ int rest_below(int64_t r) {      // r + running
  const int64_t lo = -((int64_t)1 << 30) - 4096, hi = 4096;
  return (int)(r < lo ? lo : (r > hi ? hi : r));
}
__device__ __forceinline__ int rest_above(int64_t r) {      // r - running
  const int64_t lo = -4096, hi = ((int64_t)1 << 30) + 4096;
  return (int)(r < lo ? lo : (r > hi ? hi : r));
}

// position of a batch's first query: beyond 2^40 everything is far
__device__ __forceinline__ int64_t start_of(const AttArgs& a, int b) {
  const int64_t lim = (int64_t)1 << 40;
  int64_t s = a.q_start ? uniform(a.q_start[b]) : 0;
  return s < -lim ? -lim : (s > lim ? lim : s);
}

// Scores of 32 keys against 32 queries in base-2 exponents are mul s + add after this: where all differences lie beyond the last edge on one
// side (or there is no table) s stays as the product left it, else the bias is in s already.  KEYS_DOWN: keys in the registers, queries in
// the lanes, else the other way round.  rel0: j - i - start of the first key and the first query; line: see fill_line (null: no table).
// A bias so large that it rounds scores away (a mask by values like the type's lowest) is added first all the same: rows of nothing but such
// scores then have weights of the rounded ones, as they would have from any other order of the sum.
// Returns 0 where the differences are mixed, -1 / 1 where all lie beyond the last edge on that side.
constexpr float kFoldable = 1e6f;
template <bool KEYS_DOWN>
__device__ __forceinline__ int add_bias(f32x16& s, float c2, const float* line, int far, int rel0, float left, float right, int lane,
                                        float& mul, float& add) {
  int half = lane >> 5;
  int side = !line || rel0 + 31 <= -far || rel0 - 31 >= far ? (rel0 < 0 ? -1 : 1) : 0;
  mul = 1.f;
  add = 0.f;
  if (side) {
    float cb = !line ? 0.f : uniform(side < 0 ? left : right);
    if (fabsf(cb) < kFoldable) {
      mul = c2;
      add = cb;
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], c2, cb);
    }
    return side;
  }
  const float* b = line + (KEYS_DOWN ? rel0 - (lane & 31) + 4 * half : rel0 + (lane & 31) - 4 * half) + far + kPad;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], c2, KEYS_DOWN ? b[8 * (r >> 2) + (r & 3)] : b[-(8 * (r >> 2) + (r & 3))]);
  return 0;
}

// Four consecutive features of one output row.
template <typename T>
__device__ __forceinline__ void store4(T* row, int c, int width, int vec, float x0, float x1, float x2, float x3) {
  T e[4] = {(T)x0, (T)x1, (T)x2, (T)x3};
  if (c >= width) return;
  if (vec && c + 4 <= width) {
    if constexpr (sizeof(T) == 2) *(uint2*)(row + c) = __builtin_bit_cast(uint2, e);
    else *(u32x4*)(row + c) = __builtin_bit_cast(u32x4, e);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < width) row[c + i] = e[i];
  }
}

// A column's two halves of a wave: maximum and sum.
__device__ __forceinline__ float both_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
  return __int_as_float(r[0]) + __int_as_float(r[1]);
}

// keys of a tile that take part: bit i = key j0 + i, i < 64
__device__ __forceinline__ uint64_t keep_bits(int n_left, const uint8_t* mask_row, uint8_t mask_byte) {
  uint64_t m = n_left >= 64 ? ~0ull : ((1ull << n_left) - 1);
  if (mask_row) m &= __ballot(mask_byte != 0);
  return m;
}

// Bound on exp2 arguments above the running reference: the reference is moved (and what was summed rescaled) only when a score
// exceeds it by more than this, so that most tiles leave the accumulators alone.
constexpr float kSlack = 8.f;
// fp16 weights are kept this much (log2) above one, away from that type's smallest numbers; 2^(8 + 6) is far from its largest.
template <typename T> struct Lift { static constexpr float value = 0.f; };
template <> struct Lift<_Float16> { static constexpr float value = 6.f; };

// Workgroup id -> position such that the workgroups that read the same keys (a unit: `per` neighbouring positions) run on one die, to which every
// eighth id goes, and share its L2.  Units are dealt out one by one where that comes out even, so that batches of unequal length fall on all
// dies (4 x 16 heads of 1537 .. 961 keys: the dies' work differed by 1.6); else in runs of neighbouring positions.
__device__ __forceinline__ int die_order(int id, int units, int per) {
  int die = id & 7, r = id >> 3;
  if ((units & 7) == 0) return (r / per * 8 + die) * per + r % per;
  int at = die * ((units * per + 7) / 8) + r;
  return r < (units * per + 7) / 8 ? at : units * per;
}

}  // namespace att
