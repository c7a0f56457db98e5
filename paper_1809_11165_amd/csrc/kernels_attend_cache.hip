// Attention of a sequence's new rows over its cached ones (see include/bbmm.h, "Cache"): one pass over the keys with the running reference and
// sum of the softmax, keys and values read once, straight from their pages into the registers in which the matrix instructions want them.
//
// A workgroup takes 16 (or 32) rows (query, head of the group) of one shared head and a part of the keys; its four waves take blocks of 32
// keys in turn, without barriers, and join at the end.  All products are 16 x 16 blocks: S^T = K Q^T puts a row in a lane and four keys
// 16 kb + 4 (lane / 16) + r in its registers, which are the second operand of O^T += V^T P^T as they stand.
//   keys: a lane reads 16 bytes of key 16 kb + lane % 16 at piece 4 s + lane / 16; any order of the features serves that is the queries' too.
//   values: a lane reads, of the eight keys whose weights it will meet, DP / 16 neighbouring features, 16 lanes a row.  Two-byte values then
//           change places in pairs (one byte permutation per two values); fp32 values are operands as they stand.  No LDS before the join, but for queries of 32 rows.
// 8-bit rows become T on the way, by the instruction that applies their block's power of two.
// Bound by memory with up to 16 rows a shared head (all from HBM, other data each time): 8 requests of up to 32773 keys, 8 shared heads of 128, bf16, 660 MB in 120 us,
// 5.5 TB/s (a large copy: 4.9); 16 of up to 65536 8-bit keys, 1.24 GB in 232 us, 5.3 TB/s; 64 with a window of 1024, fp16, d 64, 228 MB in 46.8 us,
// 4.9 TB/s.  With 32 rows and more by the products and the vector work beside them: 2 x 512 new rows of 32 heads on 8 over 8192 keys 304 us, 452 TFLOP/s
// (8-bit pages 305 us; fp32, 16 rows a workgroup, 1229 us, 112 TFLOP/s of 153).  Few keys: the chain length, page, keys, scores, join (77 keys 5.1 us).  3 rows
// over 10000 keys in fp32, pages of 20 rows: 27.7 us with the join, see the loop.  Up to 64 features take the width of 64, so narrower rows leave lanes idle.
#include <type_traits>

#include "cache_dev.h"

using namespace att;

namespace {

template <typename T> struct Mma;
template <> struct Mma<__bf16> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<_Float16> {
  typedef f16x8 frag;
  static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<float> {
  typedef f32x8 frag;
  static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

// Four quarters of a wave.
__device__ __forceinline__ float quarters_max(float x) {
  x = both_max(x);
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float quarters_sum(float x) {
  x = both_sum(x);
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
  return __int_as_float(r[0]) + __int_as_float(r[1]);
}

// c + a b where a, values, holds infinities or NaN: finite values are multiplied as ever; a column gets an infinity or NaN if it takes one (`took`, a bit
// a key), whatever the weight, whose parts have either sign.  b: the weights' parts.
template <typename T, int PARTS>
__device__ __forceinline__ f32x4 mma_odd(typename Mma<T>::frag a, const typename Mma<T>::frag (&b)[PARTS], unsigned took, f32x4 c) {
  const float odd[3] = {__builtin_inff(), -__builtin_inff(), __builtin_nanf("")};
  typename Mma<T>::frag x = a, ones = a;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fabsf((float)a[e]) < __builtin_inff() ? a[e] : (T)0.f, ones[e] = (took >> e) & 1 ? (T)1.f : (T)0.f;
#pragma unroll
  for (int p = 0; p < PARTS; ++p) c = Mma<T>::mma(x, b[p], c);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y = (float)a[e];
      x[e] = (k == 2 ? y != y : y == odd[k]) ? (T)1.f : (T)0.f;
    }
    f32x4 z = Mma<T>::mma(x, ones, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (z[r] != 0.f) c[r] += odd[k];
  }
  return c;
}

// fp32 numbers (no signalling NaN, whose only set bits may be cut off) as three of bf16, 8 bits each: what is left is 2^-25 of them.  Products with
// 8-bit rows, which bf16 holds exactly, then run at a fifth of the fp32 instructions' time.
__device__ __forceinline__ void in_three(const f32x8& x, bf16x8 (&p)[3]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float first = __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);   // cut off: rounding could leave the range
    float rest = fabsf(x[e]) < __builtin_inff() ? x[e] - first : 0.f;
    p[0][e] = (__bf16)first;
    p[1][e] = (__bf16)rest;
    p[2][e] = (__bf16)(rest - (float)p[1][e]);
  }
}

// cap tanh(scale x / cap) in units of the base-2 exponent, off by less than 10 u32 (2^-24) of itself however large the cap: scores that are small beside it
// are c2 x (tanh y) / y, whose last factor nears one, so a y among fp32's subnormal numbers does no harm.  NEAR: every |y| < 1/2 here.
template <bool NEAR>
__device__ __forceinline__ float capped(float x, const CacheAtt& a) {
  // |y| < 1/2: tanh y = y (1 + u P(u)), u = y^2, P of degree 3 with the least largest error, 0.3 u32
  float y = x * a.cap_in, plain = x * a.c2, u = y * y, p = fmaf(0.01725541241466999f, u, -0.05305228754878044f);
  p = fmaf(fmaf(p, u, 0.13325978815555573f), u, -0.33333149552345276f);
  float near = fmaf(plain * u, p, plain);
  if (NEAR) return near;
  // 1 - 2 / (exp 2y + 1), off by less than 5 u32: its steps are 2^-24 absolutely, and tanh 1/2 = 0.46
  float z = __builtin_amdgcn_exp2f(y * (2.f * kLog2e)), far = a.cap2 * (1.f - 2.f * __builtin_amdgcn_rcpf(z + 1.f));
  return fabsf(y) < 0.5f ? near : far;
}

constexpr int kBlock = 32;                                 // keys of a wave's turn

__device__ __forceinline__ int queries_of(const CacheAtt& a, int b) { return a.q_len ? uniform(min(max(a.q_len[b], 0), a.nq)) : a.nq; }
__device__ __forceinline__ int keys_of(const CacheArgs& c, const CacheAtt& a, int b) { return uniform((int)min((int64_t)max(a.k_len[b], 0), c.rows_most)); }

// Blocks that a sequence's rows take, and the first of them; one where there are none (somebody has to write its rows).
__device__ __forceinline__ int blocks_of(const CacheAtt& a, int qn, int kn, int* first) {
  int64_t p = (int64_t)kn - qn;
  int lo = a.window ? (int)min(max(p - a.window + 1, (int64_t)0), (int64_t)kn) : 0;
  *first = lo / kBlock;
  return max((kn + kBlock - 1) / kBlock - *first, 1);
}

// Sums over a wave without LDS: rows of 16 lanes by neighbours and mirrors, then the four rows.
template <int C, bool BOUND> __device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(0, x, C, 0xf, 0xf, BOUND); }
__device__ __forceinline__ int wave_sum(int x) {
  x += dpp<0xb1, true>(x);
  x += dpp<0x4e, true>(x);
  x += dpp<0x141, true>(x);
  x += dpp<0x140, true>(x);
  return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) + __builtin_amdgcn_readlane(x, 32) + __builtin_amdgcn_readlane(x, 48);
}
__device__ __forceinline__ int wave_before(int x, int lane) {       // of the lanes below
  int y = x;
  y += dpp<0x111, true>(y);                                // from 1, 2, 4, 8 lanes below in the row, zero before its first
  y += dpp<0x112, true>(y);
  y += dpp<0x114, true>(y);
  y += dpp<0x118, true>(y);
  int r0 = __builtin_amdgcn_readlane(y, 15), r1 = r0 + __builtin_amdgcn_readlane(y, 31), r2 = r1 + __builtin_amdgcn_readlane(y, 47);
  return y - x + (lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2);
}

// A workgroup's share: a part of a sequence's keys.  The sequences are cut into parts of about `per` blocks, per the least of nine steps that makes
// no more than `items` of them, so parts differ little however the lengths do, and none is without keys.  Every wave works this out for itself
// (up to 256 sequences, number 64 k + lane); the first of all leaves the sequences' first items for the join.
struct Share {
  int b, part, parts;
};
__device__ __forceinline__ Share share_of(const CacheArgs& c, const CacheAtt& a, int item, bool leave, int lane) {
  int n[4], sum = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    n[k] = 0;
    int b = 64 * k + lane;
    if (b >= c.B) continue;
    int s0;
    n[k] = blocks_of(a, a.q_len ? min(max(a.q_len[b], 0), a.nq) : a.nq, (int)min((int64_t)max(a.k_len[b], 0), c.rows_most), &s0);
    sum += n[k] >> 3;                                      // eighths: 256 of 2^25 blocks pass 2^31
  }
  float all = 8.f * (float)wave_sum(sum) + 8.f * (float)c.B;
  // between what would do if nothing were left over and what does in any case
  float low = fmaxf(all / (float)a.items, (float)a.least), high = fmaxf(all / (float)(a.items - c.B) * 1.0001f, low);
  int parts[4];
  for (int step = 0; step <= 8; ++step) {
    float inv = 1.f / (low + (high - low) * 0.125f * (float)step);
    sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // a part's blocks rounded up a hair: n a multiple of per makes n / per parts (a sequence of 2^25 blocks in one part and less than another's 2^-16)
      parts[k] = n[k] ? max((int)ceilf((float)n[k] * inv * 0.9999f), 1) : 0;
      sum += parts[k];
    }
    if (wave_sum(sum) <= a.items) break;
  }
  Share mine{0, 0, 0};
  int base = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (64 * k >= c.B) break;
    int at = base + wave_before(parts[k], lane), b = 64 * k + lane;
    base += wave_sum(parts[k]);
    if (leave && b < c.B) a.first[b] = at;
    uint64_t who = __ballot(item >= at && item < at + parts[k]);
    if (who) {
      int l = __ffsll((unsigned long long)who) - 1;
      mine = Share{64 * k + l, item - __builtin_amdgcn_readlane(at, l), __builtin_amdgcn_readlane(parts[k], l)};
    }
  }
  if (leave && lane == 0) a.first[c.B] = base;
  return mine;
}

// NaN if one of the four features from f on is not finite (those behind the last are whatever the rows' memory holds), else 0.
__device__ __forceinline__ float odd_of(f32x4 y, int f, int width) {
  if (f + 4 > width) {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = f + e < width ? y[e] : 0.f;
  }
  return fmaf(y[0], 0.f, fmaf(y[1], 0.f, fmaf(y[2], 0.f, y[3] * 0.f)));
}

// Waves per SIMD: what the registers admit without keeping any of the loop's in scratch.  (8-bit rows in bf16, one wave more / so: 4 requests of 40000 keys,
// 4 shared heads, d 64 31.5 / 28.3 us, d 128 45.5 / 42.4, 16 of 65536 keys, 8 shared heads of 128, 249 / 240.)  Left in scratch at two waves: 40 to 72 bytes a lane
// where page rows are no multiple of 16, of rows of 128 features in fp32 and of 32 rows of them in own type or, bf16, 8 bits; 8 bytes of 32 bf16 rows of them elsewhere.  8-bit
// pages, fp16, 64 features and 32 rows would fit three.
constexpr int waves_of(int size, bool e4m3, int dp, int nt, bool even) {
  if (nt == 2) return 2;
  if (size == 4) return dp == 64 && (even || !e4m3) ? 3 : 2;
  return dp == 64 ? (even && !e4m3 ? 4 : 3) : 2;
}

// T held as such: a key's piece is 16 bytes, a value's 16 (two-byte values of up to 64 features: 8); E4M3: the same features in a half or a quarter.
template <typename T, bool E4M3, int DP, int NT, bool EVEN>
__global__ __launch_bounds__(256, waves_of(sizeof(T), E4M3, DP, NT, EVEN)) void k_attend_cache(CacheArgs c, CacheAtt a) {
  constexpr bool kThree = sizeof(T) == 4 && E4M3;          // operands in three parts of bf16
  constexpr int PARTS = kThree ? 3 : 1;                    // of the queries, and of the weights:
  // Parts of the weights: what rounding to T leaves is a further operand, until a weight is as good as in fp32: three of bf16 hold all 24 bits, two of
  // fp16 22 and what the second's sign adds.  Outputs then fall on the wrong side of their own rounding less often than those of a plain softmax in fp32 (8
  // requests of up to 32773 keys, bf16: 0.5 of 1000 against 1.0, and 1.8 with two parts; 2 of 20000, fp16: 2.0 against 4.0).  The third part costs nothing where reads are the bound (that
  // call, two / three: 124.0 / 124.5 us; 16 of 65536 8-bit keys 235.6 / 236.7; 32 rows of 4 sequences of 40000 keys 67.3 / 67.5), else up to a sixth
  // (8-bit rows of 64 features 27.9 / 29.8; 2 x 512 new rows over 8192 keys 295 / 304, 8-bit pages 264 / 305).
  constexpr int WPARTS = kThree ? 3 : sizeof(T) == 4 ? 1 : __is_same(T, __bf16) ? 3 : 2;
  typedef std::conditional_t<kThree, __bf16, T> C;         // type of the operands
  typedef Mma<C> M;
  typedef typename M::frag frag;
  constexpr int SB = E4M3 ? 1 : (int)sizeof(T);            // bytes of a held element
  constexpr int ROWS = 16 * NT;
  constexpr int NS = DP / 32;                              // steps of eight features a lane
  constexpr int KP = DP * SB / 64;                         // 16-byte pieces of a key per lane
  constexpr int FV = DP / 16;                              // features of a value per lane
  constexpr int VW = FV * SB / 4;                          // words of a value per lane
  constexpr int kPart = ROWS * (DP + 4);
  constexpr bool kQueries = sizeof(T) == 2 && NT == 2 && DP == 128;   // queries stay in LDS: in registers, others of the loop's went to scratch
  __shared__ __align__(16) float buf[2 * kPart];
  __shared__ float wm[4][ROWS], wl[4][ROWS];
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, q4 = lane >> 4;
  // blocks of rows that read the same keys stand eight apart: on one die, whose L2 they share
  int x = blockIdx.x, of = (int)over(x >> 3, a.by_blocks), rb = (x >> 3) - of * a.blocks, unit = of * 8 + (x & 7);
  // dealt: the shared heads of an item are neighbours; else the parts of a sequence's head
  int q = (int)over(unit, a.dealt ? a.by_hk : a.by_even), seq = (int)over(q, a.by_hk);
  int hk = a.dealt ? unit - q * c.HK : q - seq * c.HK, part = a.dealt ? 0 : unit - q * a.even, item = a.dealt ? q : seq * a.even + part;
  if (item >= a.items) return;
  Share mine{seq, part, a.even};
  if (a.dealt) mine = share_of(c, a, item, x == 0 && wave == 0, lane);
  if (mine.parts == 0) return;                             // more workgroups than parts
  int b = mine.b;
  int qn = queries_of(a, b);
  int kn = keys_of(c, a, b);
  int rows = a.nq * a.G, first = rb * ROWS, i0 = first / a.G, i1 = min(min(first + ROWS, rows) - 1, qn * a.G - 1) / a.G;
  // keys that some row of these takes: [lo, hi)
  int64_t p0 = (int64_t)kn - qn + i0, p1 = (int64_t)kn - qn + i1;
  int lo = a.window ? (int)min(max(p0 - a.window + 1, (int64_t)0), (int64_t)kn) : 0;
  int hi = a.causal ? (int)max(min(p1 + 1, (int64_t)kn), (int64_t)0) : kn;
  if (first >= qn * (int64_t)a.G || c.pages == 0) hi = lo;
  int t0 = lo / kBlock, t1 = hi > lo ? (hi + kBlock - 1) / kBlock : t0;
  if (mine.parts > 1) {
    int s0, n = blocks_of(a, qn, kn, &s0);                 // of the whole sequence
    t0 = max(t0, s0 + (int)((int64_t)mine.part * n / mine.parts));
    t1 = max(min(t1, s0 + (int)((int64_t)(mine.part + 1) * n / mine.parts)), t0);
    if (t0 == t1) {                                        // nothing here: the join reads no more than this
      int r = first + tid;
      if (tid < ROWS && r < rows) a.pl[((size_t)item * a.H + hk * a.G + r % a.G) * a.nq + r / a.G] = -__builtin_inff();
      return;
    }
  }

  const char* K = (const char*)c.K + (int64_t)hk * c.ks[2] * SB;
  const char* V = (const char*)c.V + (int64_t)hk * c.vs[2] * SB;
  int64_t kpage = c.ks[0] * SB, vpage = c.vs[0] * SB, epage = (int64_t)c.HK * c.page.d * 4;
  unsigned kpitch = (unsigned)(c.ks[1] * SB), vpitch = (unsigned)(c.vs[1] * SB);
  const uint8_t *ke = E4M3 ? c.ke + (int64_t)hk * c.page.d * 4 : nullptr, *ve = E4M3 ? c.ve + (int64_t)hk * c.page.d * 4 : nullptr;
  // The table is not written while the kernel runs: read at uniform places through the scalar cache, whose loads nothing in the loop waits for (a
  // vector load there waits for all keys and values on their way: 16 requests of up to 65536 8-bit keys 360 us, so 288, before other steps).
  typedef const __attribute__((address_space(4))) int32_t* scalar_table;
  const int32_t* table = c.table + (int64_t)b * c.max_pages;

  // ---- pages of a block: EVEN (page rows a multiple of 16): two of them, in scalar registers; else one key a lane
  struct Pages { int page[2], row[2]; };
  auto find = [&](int t) {
    Pages p;
    if constexpr (EVEN) {
      uint32_t at = (uint32_t)(t * kBlock), n = over(at, c.page);
      p.row[0] = uniform((int)(at - n * c.page.d));
      p.page[0] = ((scalar_table)table)[uniform((int)n)];   // a block's first key lies before hi
      p.row[1] = p.row[0] + 16;
      p.page[1] = p.page[0];
      if (p.row[1] == (int)c.page.d) {
        p.row[1] = 0;
        p.page[1] = at + 16 < (uint32_t)hi ? ((scalar_table)table)[uniform((int)n) + 1] : -1;
      }
    } else {
      uint32_t at = (uint32_t)(t * kBlock + (lane & 31)), n = over(at, c.page);
      p.row[0] = (int)(at - n * c.page.d);
      p.page[0] = at < (uint32_t)hi ? table[n] : -1;
    }
    return p;
  };
  // keys of a block that take part, before the rows' own bounds
  auto kept = [&](int t, const Pages& p) {
    int j0 = t * kBlock;
    unsigned m = hi - j0 >= kBlock ? ~0u : (1u << (hi - j0)) - 1;
    if (lo > j0) m &= ~0u << (lo - j0);                    // lo < j0 + 32: blocks begin at lo / 32
    if constexpr (EVEN) {
      if ((unsigned)p.page[0] >= (unsigned)c.pages) m &= 0xffff0000u;
      if ((unsigned)p.page[1] >= (unsigned)c.pages) m &= 0x0000ffffu;
    } else {
      m &= (unsigned)__ballot((unsigned)p.page[0] < (unsigned)c.pages);
    }
    return m;
  };

  u32x4 kr[2][KP];
  unsigned vr[8][VW];
  unsigned kx[2];                                          // E4M3: exponents of the lane's keys,
  u32x4 vx[2];                                             // and of its values' rows
  unsigned koff = (unsigned)col * kpitch + 16u * q4, voff = (unsigned)(4 * q4) * vpitch;
  auto fetch_k = [&](const Pages& p, unsigned keep) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      unsigned gone = (~keep >> (16 * k + col)) << 31;
      if constexpr (EVEN) {
        bool there = (keep >> (16 * k)) & 0xffffu;
        int pg = there ? p.page[k] : 0, row = there ? p.row[k] : 0;
        __amdgpu_buffer_rsrc_t mem = bounded(K + pg * kpage + (int64_t)row * kpitch, there ? 15 * kpitch + (unsigned)(c.d * SB + 15) / 16 * 16 : 0u);
#pragma unroll
        for (int s = 0; s < KP; ++s)
          kr[k][s] = __builtin_amdgcn_raw_buffer_load_b128(mem, (16u * (4 * s + q4) < (unsigned)(c.d * SB) ? koff : kNowhere) | gone, 64 * s, 0);
        if constexpr (E4M3) {
          __amdgpu_buffer_rsrc_t ex = bounded(ke + pg * epage + (int64_t)row * 4, there ? 64u : 0u);
          kx[k] = __builtin_amdgcn_raw_buffer_load_b32(ex, 4 * col, 0, 0);
        }
      } else {
        int pg = __shfl(p.page[0], 16 * k + col, 64), row = __shfl(p.row[0], 16 * k + col, 64);
        if (gone) pg = row = 0;                             // some row: loads without branches are counted, and waited for, one by one
        const char* at = K + pg * kpage + (int64_t)row * kpitch;
#pragma unroll
        for (int s = 0; s < KP; ++s) {
          int o = 16 * (4 * s + q4);
          kr[k][s] = *(const u32x4*)(at + (o < c.d * SB ? o : 0));
        }
        if constexpr (E4M3) kx[k] = *(const unsigned*)(ke + pg * epage + (int64_t)row * 4);
      }
    }
  };
  auto fetch_v = [&](const Pages& p, unsigned keep) {
    unsigned o = (unsigned)(col * FV * SB);
    bool mine = o < (unsigned)(c.dv * SB);
    unsigned vlane = mine ? voff + o : kNowhere;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if constexpr (EVEN) {
        bool there = (keep >> (16 * k)) & 0xffffu;
        int pg = there ? p.page[k] : 0, row = there ? p.row[k] : 0;
        __amdgpu_buffer_rsrc_t mem = bounded(V + pg * vpage + (int64_t)row * vpitch, there ? 15 * vpitch + (unsigned)(c.dv * SB + 15) / 16 * 16 : 0u);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          unsigned gone = (~keep >> (16 * k + 4 * q4 + r)) << 31, at = vlane | gone;   // behind every bound; a branch would spoil the counting of loads
          int step = (int)(r * vpitch);
          unsigned* v = vr[4 * k + r];
          if constexpr (VW == 1) {
            v[0] = __builtin_amdgcn_raw_buffer_load_b32(mem, at, step, 0);
          } else if constexpr (VW == 2) {
            auto w = __builtin_amdgcn_raw_buffer_load_b64(mem, at, step, 0);
            v[0] = w[0], v[1] = w[1];
          } else if constexpr (VW == 4) {
            u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(mem, at, step, 0);
            v[0] = w[0], v[1] = w[1], v[2] = w[2], v[3] = w[3];
          } else {                                         // fp32, 128 features: 4 of each half
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              unsigned f = 256u * z + 16u * col;
              u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(mem, (f < 4u * c.dv ? voff + 16u * col : kNowhere) | gone, step + 256 * z, 0);
              v[4 * z] = w[0], v[4 * z + 1] = w[1], v[4 * z + 2] = w[2], v[4 * z + 3] = w[3];
            }
          }
        }
        if constexpr (E4M3) {                              // (of excluded keys: see add_values)
          __amdgpu_buffer_rsrc_t ex = bounded(ve + pg * epage + (int64_t)row * 4, there ? 64u : 0u);
          vx[k] = __builtin_amdgcn_raw_buffer_load_b128(ex, 16 * q4, 0, 0);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          int key = 16 * k + 4 * q4 + r;
          int pg = __shfl(p.page[0], key, 64), row = __shfl(p.row[0], key, 64);
          if (!((keep >> key) & 1)) pg = row = 0;
          const char* at = V + pg * vpage + (int64_t)row * vpitch;
          unsigned* v = vr[4 * k + r];
          if constexpr (VW <= 4) {
            at += mine ? o : 0u;
            if constexpr (VW == 1) v[0] = *(const unsigned*)at;
            else if constexpr (VW == 2) { uint2 w = *(const uint2*)at; v[0] = w.x, v[1] = w.y; }
            else { u32x4 w = *(const u32x4*)at; v[0] = w[0], v[1] = w[1], v[2] = w[2], v[3] = w[3]; }
          } else {
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              u32x4 w = *(const u32x4*)(at + (64 * z + 4 * col < c.dv ? 256 * z + 16 * col : 0));
              v[4 * z] = w[0], v[4 * z + 1] = w[1], v[4 * z + 2] = w[2], v[4 * z + 3] = w[3];
            }
          }
          if constexpr (E4M3) vx[k][r] = *(const unsigned*)(ve + pg * epage + (int64_t)row * 4);
        }
      }
    }
  };
  // EVEN: the bounded reads have left zeros.  Else excluded rows' values are made zeros here.
  auto clear_values = [&](unsigned keep) {
    if constexpr (!EVEN) {
      if (keep == ~0u) return;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int w = 0; w < VW; ++w) vr[e][w] = (keep >> (16 * (e >> 2) + 4 * q4 + (e & 3))) & 1 ? vr[e][w] : 0u;
    }
  };

  // Features of a lane's step s of the scores: eight from `feature(s)` on (fp32: four, twice).
  auto step_at = [&](int s) { return E4M3 ? 16 * (4 * (s >> 1) + q4) + 8 * (s & 1) : 8 * (4 * s + q4); };
  // fp32 pieces hold four features: step s has pieces 2s, 2s + 1
  frag qf[kQueries ? 1 : NT][kQueries ? 1 : NS][PARTS];
  frag* held = (frag*)buf + lane;                          // of row block n, step s: held[64 (NS n + s)]
  int rho[NT], qi[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    rho[n] = first + 16 * n + col;
    qi[n] = rho[n] / a.G;
    bool have = rho[n] < rows && qi[n] < qn;
    const T* row = (const T*)a.Q + b * a.qs[0] + (int64_t)qi[n] * a.qs[1] + (int64_t)(hk * a.G + rho[n] % a.G) * a.qs[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if constexpr (sizeof(T) == 2) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if constexpr (kQueries) {
          if (s != 0) continue;                            // each wave brings one of the four steps
          if (have) v = load16<T>(row, step_at(wave), c.d, a.qvec);
          held[64 * (NS * n + wave)] = __builtin_bit_cast(frag, v);
        } else {
          if (have) v = load16<T>(row, step_at(s), c.d, a.qvec);
          qf[n][s][0] = __builtin_bit_cast(frag, v);
        }
      } else {
        int f0 = E4M3 ? step_at(s) : 4 * (8 * s + q4), f1 = E4M3 ? f0 + 4 : 4 * (8 * s + 4 + q4);
        u32x4 v0 = {0u, 0u, 0u, 0u}, v1 = v0;
        if (have) {
          v0 = load16<T>(row, f0, c.d, a.qvec);
          v1 = load16<T>(row, f1, c.d, a.qvec);
        }
        f32x8 x = __builtin_shufflevector(__builtin_bit_cast(f32x4, v0), __builtin_bit_cast(f32x4, v1), 0, 1, 2, 3, 4, 5, 6, 7);
        if constexpr (kThree) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __builtin_canonicalizef(x[e]);
          in_three(x, qf[n][s]);
        } else qf[n][s][0] = x;
      }
    }
  }
  if constexpr (kQueries) __syncthreads();
  // Behind the last feature a piece holds whatever the row's memory does.
  bool ragged = (c.d * SB) % 16 != 0;
  unsigned blocks_there = c.d > 96 ? ~0u : (1u << (8 * ((c.d + 31) / 32))) - 1;
  auto trim = [&] {
    if constexpr (E4M3) {                                  // nothing times an exponent that nobody wrote
#pragma unroll
      for (int k = 0; k < 2; ++k) kx[k] = (kx[k] & blocks_there) | (0x7f7f7f7fu & ~blocks_there);
    }
    if (EVEN ? !ragged : c.d == DP) return;
    int last = c.d * SB / 16, left = c.d * SB - 16 * last;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int s = 0; s < KP; ++s)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          int n = min(max(left - 4 * w, 0), 4);
          if (4 * s + q4 == last) kr[k][s][w] &= n == 4 ? ~0u : (1u << (8 * n)) - 1;
          if (!EVEN && 4 * s + q4 > last) kr[k][s][w] = 0u;
        }
  };
  auto key_frag = [&](int k, int s) {
    if constexpr (!E4M3) {
      if constexpr (sizeof(T) == 2) return __builtin_bit_cast(frag, kr[k][s]);
      else return __builtin_shufflevector(__builtin_bit_cast(f32x4, kr[k][2 * s]), __builtin_bit_cast(f32x4, kr[k][2 * s + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      frag f;
      float scale = __uint_as_float(((kx[k] >> (8 * (2 * (s >> 1) + (q4 >> 1)))) & 0xffu) << 23);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        unsigned q = kr[k][s >> 1][2 * (s & 1) + w];
        auto x0 = Wide<C>::template get<false>(q, scale);
        auto x1 = Wide<C>::template get<true>(q, scale);
        f[4 * w] = x0[0], f[4 * w + 1] = x0[1], f[4 * w + 2] = x1[0], f[4 * w + 3] = x1[1];
      }
      return f;
    }
  };

  f32x4 acc[NT][FV];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int f = 0; f < FV; ++f) acc[n][f] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m[NT], l[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) m[n] = -__builtin_inff(), l[n] = 0.f;

  // Keys of the block from j0 on that the lane's row takes, of those kept.
  auto taken = [&](int n, int j0, unsigned keep) {
    int64_t p = (int64_t)kn - qn + qi[n] - j0;             // the row's place in the block
    if (a.causal) keep &= p < 0 ? 0u : p >= 31 ? ~0u : (2u << (int)p) - 1;
    if (a.window) {
      int64_t w = p - a.window + 1;                        // the first key
      keep &= w <= 0 ? ~0u : w >= 32 ? 0u : ~0u << (int)w;
    }
    return keep;
  };

  // O^T += V^T P^T; s[n][k][r]: weight of row n, key 16 k + 4 q4 + r.  fp32: eight single products make a step, of four keys each.
  auto add_values = [&](const f32x4 (*p)[2], int j0, unsigned keep, auto odd) {
    frag pf[NT][WPARTS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if constexpr (kThree) {
        in_three(__builtin_shufflevector(p[n][0], p[n][1], 0, 1, 2, 3, 4, 5, 6, 7), pf[n]);
      } else {
        f32x8 w = __builtin_shufflevector(p[n][0], p[n][1], 0, 1, 2, 3, 4, 5, 6, 7);
        pf[n][0] = __builtin_convertvector(w, frag);
        if constexpr (__is_same(T, __bf16)) {              // each pair rounded once, and taken apart
#pragma unroll
          for (int part = 1; part < WPARTS; ++part) {
            u32x4 x = __builtin_bit_cast(u32x4, pf[n][part - 1]);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] -= __uint_as_float(e & 1 ? x[e >> 1] & 0xffff0000u : x[e >> 1] << 16);
            pf[n][part] = __builtin_convertvector(w, frag);
          }
        } else if constexpr (WPARTS == 2) {
          pf[n][1] = __builtin_convertvector(w - __builtin_convertvector(pf[n][0], f32x8), frag);
        }
      }
    }
    unsigned took[NT];                                     // a bit each of the lane's eight keys
    if constexpr (decltype(odd)::value) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        unsigned mine = taken(n, j0, keep);
        took[n] = ((mine >> (4 * q4)) & 0xfu) | ((mine >> (12 + 4 * q4)) & 0xf0u);
      }
    }
    auto product = [&](frag v, int f) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if constexpr (decltype(odd)::value) {
          acc[n][f] = mma_odd<C, WPARTS>(v, pf[n], took[n], acc[n][f]);
        } else {
#pragma unroll
          for (int x = 0; x < WPARTS; ++x) acc[n][f] = M::mma(v, pf[n][x], acc[n][f]);
        }
      }
    };
    if constexpr (E4M3) {
      int shift = 8 * (col * FV / 32);
      float scale[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) scale[e] = __uint_as_float(((vx[e >> 2][e & 3] >> shift) & 0xffu) << 23);
      if (keep != ~0u) {                                   // excluded rows are zeros, whatever their exponents hold
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!((keep >> (16 * (e >> 2) + 4 * q4 + (e & 3))) & 1)) scale[e] = 1.f;
      }
#pragma unroll
      for (int w = 0; w < 2 * VW; ++w) {                   // features 2 w, 2 w + 1
        typename Wide<C>::two x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[e] = w & 1 ? Wide<C>::template get<true>(vr[e][w >> 1], scale[e]) : Wide<C>::template get<false>(vr[e][w >> 1], scale[e]);
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          u32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, x[2 * e + 1]), __builtin_bit_cast(unsigned, x[2 * e]), f ? 0x07060302u : 0x05040100u);
          frag v = __builtin_bit_cast(frag, y);
          product(v, 2 * w + f);
        }
        if (w & 1) __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int f = 0; f < FV; ++f) {
        frag v;
        if constexpr (sizeof(T) == 2) {
          u32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_perm(vr[2 * e + 1][f >> 1], vr[2 * e][f >> 1], f & 1 ? 0x07060302u : 0x05040100u);
          v = __builtin_bit_cast(frag, y);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(vr[e][f]);
        }
        product(v, f);
        if (f & 1) __builtin_amdgcn_sched_barrier(0);      // else operands of all products are made ahead, and registers run out
      }
    }
  };
  // Whether the lane's values hold an infinity or NaN.
  auto odd_values = [&] {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int w = 0; w < VW; ++w) {
        unsigned y = vr[e][w];
        if constexpr (E4M3) odd |= (((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
        else if constexpr (sizeof(T) == 4) odd |= (y & 0x7f800000u) == 0x7f800000u;
        else {
          constexpr unsigned m = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
          odd |= (y & m) == m || (y & (m << 16)) == (m << 16);
        }
      }
    return odd;
  };

  // Scores of the block in kr, and the weights that they become: s[n][k][r] of row n, key 16 k + 4 q4 + r.
  f32x4 s[NT][2];
  auto scores = [&] {
    trim();
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (kQueries) {
      int here = 0;
      asm volatile("" : "+v"(here));                       // read anew each time
#pragma unroll
      for (int z = 0; z < NS; ++z) {
        frag q[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) q[n] = held[64 * (NS * n + z) + here];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          frag f = key_frag(k, z);
#pragma unroll
          for (int n = 0; n < NT; ++n) s[n][k] = M::mma(f, q[n], s[n][k]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int z = 0; z < NS; ++z) {
          frag f = key_frag(k, z);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) s[n][k] = M::mma(f, qf[n][z][p], s[n][k]);
        }
    }
  };
  auto weights = [&](int j0, unsigned keep, auto edge) {
    // in units of the base-2 exponent
    if (a.cap2 != 0.f) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float far = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) far = fmaxf(far, fabsf(s[n][e >> 2][e & 3]));
        auto all = [&](auto near) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[n][e >> 2][e & 3] = capped<decltype(near)::value>(s[n][e >> 2][e & 3], a);
        };
        if (sizeof(T) == 4 || __any(far * a.cap_in >= 0.5f)) all(Const<0>{});   // (fp32: with two ways, others of the loop's registers went to scratch)
        else all(Const<1>{});
      }
    }
    float mul = a.cap2 != 0.f ? 1.f : a.c2;
    if (decltype(edge)::value || keep != ~0u) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        unsigned mine = decltype(edge)::value ? taken(n, j0, keep) : keep;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!((mine >> (16 * (e >> 2) + 4 * q4 + (e & 3))) & 1)) s[n][e >> 2][e & 3] = -__builtin_inff();
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float top = s[n][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, s[n][e >> 2][e & 3]);
      top *= mul;
      if (__any(top > m[n] + kSlack)) {
        top = quarters_max(top);
        bool move = top > m[n] + kSlack;
        float up = move ? __builtin_amdgcn_exp2f(m[n] - top) : 1.f;
        m[n] = move ? top : m[n];
        l[n] *= up;
#pragma unroll
        for (int f = 0; f < FV; ++f) acc[n][f] *= up;
      }
      float ref = (m[n] == -__builtin_inff() ? 0.f : m[n]) - Lift<T>::value;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float y = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 2][e & 3], mul, -ref));
        s[n][e >> 2][e & 3] = y;
        l[n] += y;
      }
    }
  };

  // Blocks of which all queries take the same keys: [a0, a1).  The next block's keys are on their way from the end of the scores on, its values from
  // the end of the products with them.
  int a0 = t0, a1 = t1;
  if (i0 != i1) {
    if (a.window) a0 = (int)min(max(p1 - a.window < 0 ? 0 : (p1 - a.window) / kBlock + 1, (int64_t)t0), (int64_t)t1);
    if (a.causal) a1 = (int)min(max(p0 < kBlock - 1 ? 0 : (p0 - (kBlock - 1)) / kBlock + 1, (int64_t)a0), (int64_t)t1);
  }
  settle();
  int t = a0 + wave;
  if (t < a1) {
    Pages here = find(t), next = t + 4 < a1 ? find(t + 4) : here;
    unsigned keep = kept(t, here);
    fetch_k(here, keep);
    __builtin_amdgcn_sched_barrier(0);                     // in the loop's order: else its first wait is for all of them
    fetch_v(here, keep);
    __builtin_amdgcn_sched_barrier(0);
    // no load under a condition: waits go by the count of the loads behind, the same on every way here
    for (; t + 4 < a1; t += 4) {
      scores();
      unsigned keep_next = kept(t + 4, next);
      Pages after = next;
      if (t + 8 < a1) after = find(t + 8);
      fetch_k(next, keep_next);
      weights(t * kBlock, keep, Const<0>{});
      clear_values(keep);
      add_values(s, t * kBlock, keep, Const<0>{});
      fetch_v(next, keep_next);
      next = after;
      keep = keep_next;
    }
    scores();
    weights(t * kBlock, keep, Const<0>{});
    clear_values(keep);
    add_values(s, t * kBlock, keep, Const<0>{});
  }
  // and the others, few: [t0, a0) and [a1, t1).  Infinities and NaN among their values are kept from rows that do not take them (an 8-bit value may
  // become infinite in fp16 as well).
  for (int u = wave; u < (a0 - t0) + (t1 - a1); u += 4) {
    int at = u < a0 - t0 ? t0 + u : a1 + u - (a0 - t0);
    Pages here = find(at);
    unsigned keep = kept(at, here);
    fetch_k(here, keep);
    fetch_v(here, keep);
    scores();
    weights(at * kBlock, keep, Const<1>{});
    clear_values(keep);
    if (__any(odd_values()) || (E4M3 && __is_same(T, _Float16))) add_values(s, at * kBlock, keep, Const<1>{});
    else add_values(s, at * kBlock, keep, Const<0>{});
  }

  // the waves' sums: each scales its own to the largest reference; two leave theirs in LDS, the other two add them, all write
  float top[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] = quarters_sum(l[n]);
    if (q4 == 0) {
      wm[wave][16 * n + col] = m[n];
      wl[wave][16 * n + col] = l[n];
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    int r = 16 * n + col;
    top[n] = fmaxf(fmaxf(wm[0][r], wm[1][r]), fmaxf(wm[2][r], wm[3][r]));
    float w = m[n] == -__builtin_inff() && l[n] == 0.f ? 0.f : __builtin_amdgcn_exp2f(m[n] - top[n]);
#pragma unroll
    for (int f = 0; f < FV; ++f) acc[n][f] *= w;
  }
  // feature of acc[.][f][r]: two bytes: FV (4 q4 + r) + f;  fp32: 64 (f / 4) + 4 (4 q4 + r) + f % 4
  auto spot = [&](int n, int f, int r) {
    int at = sizeof(T) == 2 || E4M3 ? FV * (4 * q4 + r) + f : 64 * (f >> 2) + 4 * (4 * q4 + r);
    return buf + (wave & 1) * kPart + (16 * n + col) * (DP + 4) + at;
  };
  auto each = [&](auto act) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int f = 0; f < FV; f += 4)
#pragma unroll
        for (int r = 0; r < 4; ++r) act((f32x4*)spot(n, f, r), f32x4{acc[n][f][r], acc[n][f + 1][r], acc[n][f + 2][r], acc[n][f + 3][r]});
  };
  if (wave >= 2) each([](f32x4* p, f32x4 v) { *p = v; });
  __syncthreads();
  if (wave < 2) each([](f32x4* p, f32x4 v) { *p += v; });
  __syncthreads();
  constexpr int TR = 256 / ROWS;                           // threads of a row
  int row = tid / TR, rr = first + row, i = rr / a.G, h = hk * a.G + rr % a.G;
  if (rr >= rows) return;
  float best = fmaxf(fmaxf(wm[0][row], wm[1][row]), fmaxf(wm[2][row], wm[3][row])), sum = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) sum += wm[k][row] == -__builtin_inff() && wl[k][row] == 0.f ? 0.f : __builtin_amdgcn_exp2f(wm[k][row] - best) * wl[k][row];
  bool some = sum != 0.f && i < qn;                        // NaN counts as something
  float inv = some ? 1.f / sum : 0.f;
  float lse2 = some ? (best - Lift<T>::value) + __builtin_amdgcn_logf(sum) : -__builtin_inff();
  bool whole = mine.parts == 1;
  size_t at = ((size_t)(whole ? b : item) * a.H + h) * a.nq + i;
  if (tid % TR == 0) {
    if (whole) a.lse[at] = lse2 * kLn2;
    else a.pl[at] = lse2;
  }
  if (!whole && !some) return;                             // parts without weight are not read
  const float* src = buf + row * (DP + 4);
  T* out = (T*)a.O + (((size_t)b * a.nq + i) * a.H + h) * c.dv;
  float check = 0.f;                                       // NaN if an output is not finite
  for (int f = tid % TR * 4; f < DP; f += 4 * TR) {
    f32x4 y = (*(const f32x4*)(src + f) + *(const f32x4*)(src + kPart + f)) * inv;
    if (!some) y = f32x4{0.f, 0.f, 0.f, 0.f};
    check += odd_of(y, f, c.dv);
    if (whole) store4<T>(out, f, c.dv, a.ovec, y[0], y[1], y[2], y[3]);
    else if (f < a.dv4) *(f32x4*)(a.pO + at * a.dv4 + f) = y;
  }
  if (check == 0.f || lse2 != lse2) return;
  // What is not finite is formed anew, key by key (a thread's features at once: slow, and rare).  Infinities among the values that the row takes come through: its
  // weights are positive, but a product with the weight's parts, which have either sign, or with a weight that rounds to zero is NaN.  Without one, it was
  // the sum that left fp32 before its division: with weights of the whole sum it is a mean, no larger than the values.
  constexpr int N = DP / TR;                               // features of a thread: 4 neighbours, 4 TR apart
  int64_t p = (int64_t)kn - qn + i;
  int from = max(t0 * kBlock, a.window ? (int)max(p - a.window + 1, (int64_t)0) : 0), to = (int)min((int64_t)t1 * kBlock, a.causal ? min(p + 1, (int64_t)kn) : (int64_t)kn);
  auto feature = [&](int z) { return 4 * (tid % TR + TR * (z >> 2)) + (z & 3); };
  auto value = [&](const char* row, unsigned exps, int f) {   // an element of a held row
    if constexpr (E4M3) return (float)Wide<T>::template get<false>(((const uint8_t*)row)[f], block_scale(exps, f / 32))[0];
    else return (float)((const T*)row)[f];
  };
  const T* query = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + (int64_t)h * a.qs[2];
  float odd[N], mean[N];
#pragma unroll
  for (int z = 0; z < N; ++z) odd[z] = mean[z] = 0.f;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (int j = from; j < to; ++j) {
      uint32_t n = over((uint32_t)j, c.page);
      int pg = table[n], row = j - (int)(n * c.page.d);
      if ((unsigned)pg >= (unsigned)c.pages) continue;
      unsigned vexps = 0, kexps = 0;
      if constexpr (E4M3) vexps = *(const unsigned*)(ve + pg * epage + (int64_t)row * 4), kexps = *(const unsigned*)(ke + pg * epage + (int64_t)row * 4);
      float w = 0.f;
      if (pass) {
        const char* key = K + pg * kpage + (int64_t)row * kpitch;
        float dot = 0.f;
#pragma unroll 8
        for (int x = 0; x < c.d; ++x) dot = fmaf((float)query[x], value(key, kexps, x), dot);
        w = __builtin_amdgcn_exp2f((a.cap2 != 0.f ? capped<false>(dot, a) : dot * a.c2) - lse2);
      }
#pragma unroll
      for (int z = 0; z < N; ++z) {
        if (feature(z) >= c.dv) continue;
        float y = value(V + pg * vpage + (int64_t)row * vpitch, vexps, feature(z));
        if (pass) mean[z] = fmaf(w, y, mean[z]);
        else odd[z] += fabsf(y) < __builtin_inff() ? 0.f : y;
      }
    }
    bool more = false;
#pragma unroll
    for (int z = 0; z < N; ++z) more |= feature(z) < c.dv && odd[z] == 0.f && !(fabsf((src[feature(z)] + src[kPart + feature(z)]) * inv) < __builtin_inff());
    if (!more) break;
  }
  constexpr float most = __is_same(T, __bf16) ? 0x1.fep127f : 0x1.fffffep127f;
#pragma unroll
  for (int z = 0; z < N; ++z) {
    int f = feature(z);
    if (f >= c.dv || fabsf((src[f] + src[kPart + f]) * inv) < __builtin_inff()) continue;
    float y = odd[z] != 0.f ? odd[z] : fminf(fmaxf(mean[z], -most), most);
    if (whole) out[f] = (T)y;
    else a.pO[at * a.dv4 + f] = y;
  }
}

// Parts of a row joined by their log sums (5.2 us for 8 x 32 rows of up to 12 parts, 6.3 for 16 x 32: the launch and two loads in a chain): 32 lanes a row, four features a lane, GROUPS of them that take every GROUPS-th part (and join in LDS).  What
// parts without weight hold is not used.
template <typename T, int GROUPS>
__global__ __launch_bounds__(256) void k_attend_cache_join(CacheArgs c, CacheAtt a) {
  __shared__ __align__(16) f32x4 part[8][32];
  __shared__ float tops[8], sums[8];
  int n = c.B * a.H * a.nq, row = blockIdx.x * (8 / GROUPS) + (threadIdx.x >> 5) / GROUPS;
  int lane = threadIdx.x & 31, f = 4 * lane, all = threadIdx.x >> 5, g = all % GROUPS;
  if (row >= n) return;                                    // GROUPS == 8: no workgroup is behind the last row
  int bh = (int)over(row, a.by_nq), i = row - bh * a.nq, b = (int)over(bh, a.by_heads), h = bh - b * a.H;
  int64_t first = (int64_t)b * a.even, step = (int64_t)a.H * a.nq;
  int parts = a.even;
  if (a.dealt) {
    first = a.first[b];
    parts = a.first[b + 1] - (int)first;
  }
  int64_t from = first * step + (int64_t)h * a.nq + i;
  if (parts == 1) return;                                  // written as it was
  float top = -__builtin_inff(), sum = 0.f;
  f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = g; s0 < parts; s0 += 8 * GROUPS) {
    float p[8];
    f32x4 v[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      int at = s0 + GROUPS * s, there = min(at, parts - 1); // loads without branches, behind the last part of that again
      p[s] = a.pl[from + there * step];
      v[s] = *(const f32x4*)(a.pO + (from + there * step) * a.dv4 + min(f, a.dv4 - 4));
      if (at >= parts) p[s] = -__builtin_inff();
    }
    float best = top;
#pragma unroll
    for (int s = 0; s < 8; ++s) best = fmaxf(best, p[s]);
    float up = top == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(top - best);
    sum *= up;
    y *= up;
    top = best;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (p[s] == -__builtin_inff()) continue;
      float w = __builtin_amdgcn_exp2f(p[s] - best);
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(w, v[s][e], y[e]);
    }
  }
  if constexpr (GROUPS > 1) {
    part[all][lane] = y;
    if (lane == 0) tops[all] = top, sums[all] = sum;
    __syncthreads();
    if (g) return;
    top = -__builtin_inff(), sum = 0.f;
    y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, tops[all + k]);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      if (sums[all + k] == 0.f) continue;
      float w = __builtin_amdgcn_exp2f(tops[all + k] - top);
      sum = fmaf(w, sums[all + k], sum);
      y += w * part[all + k][lane];
    }
  }
  bool some = sum != 0.f;
  float inv = some ? 1.f / sum : 0.f;
  if (lane == 0) a.lse[row] = some ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
  T* out = (T*)a.O + (((size_t)b * a.nq + i) * a.H + h) * c.dv;
  store4<T>(out, f, c.dv, a.ovec, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
  // What is not finite is formed anew: infinities of the parts come through whatever their weight, which may have rounded to zero; else the sum left fp32.
  if (odd_of(y, f, c.dv) == 0.f || sum != sum) return;
#pragma unroll 1
  for (int e = f; e < min(f + 4, c.dv); ++e) {
    float odd = 0.f, mean = 0.f;
#pragma unroll 1
    for (int s = 0; s < parts; ++s) {
      float lse2 = a.pl[from + s * step], v = a.pO[(from + s * step) * a.dv4 + e];
      if (lse2 == -__builtin_inff()) continue;
      if (fabsf(v) < __builtin_inff()) mean = fmaf(__builtin_amdgcn_exp2f(lse2 - top) * inv, v, mean);
      else odd += v;
    }
    constexpr float most = __is_same(T, __bf16) ? 0x1.fep127f : 0x1.fffffep127f;
    out[e] = (T)(odd != 0.f ? odd : fminf(fmaxf(mean, -most), most));
  }
}

template <typename T, bool E4M3, int DP, int NT>
void attend_n(hipStream_t s, const CacheArgs& c, const CacheAtt& a) {
  unsigned grid = (unsigned)(((int64_t)a.items * c.HK + 7) / 8 * 8 * a.blocks);
  if (c.page.d % 16 == 0) k_attend_cache<T, E4M3, DP, NT, true><<<grid, 256, 0, s>>>(c, a);
  else k_attend_cache<T, E4M3, DP, NT, false><<<grid, 256, 0, s>>>(c, a);
}
template <typename T, bool E4M3, int DP>
void attend_d(hipStream_t s, int type, const CacheArgs& c, const CacheAtt& a) {
  if constexpr (sizeof(T) == 2) {
    if (cache_rows(type, (int64_t)a.nq * a.G) == 32) return attend_n<T, E4M3, DP, 2>(s, c, a);
  }
  attend_n<T, E4M3, DP, 1>(s, c, a);
}
template <typename T, bool E4M3>
void attend_e(hipStream_t s, int type, const CacheArgs& c, const CacheAtt& a) {
  if (c.d <= 64 && c.dv <= 64) attend_d<T, E4M3, 64>(s, type, c, a);
  else attend_d<T, E4M3, 128>(s, type, c, a);
}
template <typename T>
void attend_t(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheAtt& a) {
  if (e4m3) attend_e<T, true>(s, type, c, a);
  else attend_e<T, false>(s, type, c, a);
}

template <typename T>
void join_t(hipStream_t s, const CacheArgs& c, const CacheAtt& a) {
  int64_t n = (int64_t)c.B * a.H * a.nq;
  if (n > 4096) k_attend_cache_join<T, 1><<<(unsigned)((n + 7) / 8), 256, 0, s>>>(c, a);
  else k_attend_cache_join<T, 8><<<(unsigned)n, 256, 0, s>>>(c, a);
}

}  // namespace

int cache_rows(int type, int64_t rows) { return type != 0 && rows > 16 ? 32 : 16; }
int cache_held(int type, int e4m3, const CacheArgs& c, int64_t rows) {
  return waves_of(type == 0 ? 4 : 2, e4m3, c.d <= 64 && c.dv <= 64 ? 64 : 128, cache_rows(type, rows) / 16, c.page.d % 16 == 0);
}

void launch_attend_cache(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheAtt& a) {
  if (type == 0) attend_t<float>(s, type, e4m3, c, a);
  else if (type == 1) attend_t<_Float16>(s, type, e4m3, c, a);
  else attend_t<__bf16>(s, type, e4m3, c, a);
}
void launch_attend_cache_join(hipStream_t s, int type, const CacheArgs& c, const CacheAtt& a) {
  if (type == 0) join_t<float>(s, c, a);
  else if (type == 1) join_t<_Float16>(s, c, a);
  else join_t<__bf16>(s, c, a);
}
