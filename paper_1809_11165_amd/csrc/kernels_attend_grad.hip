// Gradient of the attention (see kernels_attend.hip).  With p_ij = exp(s_ij - lse_i) recomputed tile by tile and delta_i = do_i.o_i,
//     dS_ij = p_ij (do_i.v_j - delta_i),
//     dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_{i, heads of the group} dS_ij q_i,  dV_j = sum_{i, heads} p_ij do_i,
//     dT[h, n] = sum of dS_ij over the pairs of bucket n.
// Two passes, each owning what it writes, so that every sum has a fixed order and nothing is added atomically in memory: k_attend_dq (a
// workgroup owns 128 queries of a head and runs over the keys; transposed scores, like the forward pass) and
// k_attend_dkv (owns 128 keys of a shared head and runs over the queries of all its heads; scores with a key in a lane).  The table's sums are
// formed by the first in two-byte types, by the second in fp32 (see there).  Seven matrix products
// where five would do with dQ added atomically.  Measured, bf16: 2 x 16 heads on 4, 2048 x 8192, d = 128: dQ 523 us and dK, dV 661 us, 788 and 832
// TFLOP/s of their own products (a large matrix product: 1200); 8 x 12 heads, 512 x 640 with lengths and a table, d = 64: 49 (33 without
// forming delta from the scores) and 35 us.  fp32, 2 x 8 heads, 500 x 1000, d = 64 with a table: 48 and 64 us; there one wave per SIMD fits
// (registers; the dK, dV pass at d = 128 keeps 180 bytes a lane in scratch), and the matrix unit is busy 54 % of either pass: the
// wave's own vector instructions and waits stand between its products.
//
// fp16: p and dS are scaled by powers of two before they are rounded, dS by |do_i| times the largest |v_j| (dQ) or the largest |do_i| |v_j| (dK) of
// the shared head (k_attend_norms): weights of long rows and small gradients would fall among that type's subnormal numbers.
#include "attend_dev.h"

using namespace att;

namespace {

template <typename T> struct PLift { static constexpr float value = 0.f; };
template <> struct PLift<_Float16> { static constexpr float value = 12.f; };

// fp16: largest |do_i| and |v_j| of a shared head (the slots of unit b HK + hk).  All lanes of a wave take part.
__device__ __forceinline__ float2 norms_of(const AttGrad& g, int unit, int lane) {
  float x = 0.f, y = 0.f;
  for (int k = lane; k < g.norm_slots; k += 64) {
    float2 z = *(const float2*)(g.norms + 2 * ((size_t)unit * g.norm_slots + k));
    x = fmaxf(x, z.x);
    y = fmaxf(y, z.y);
  }
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    x = fmaxf(x, __shfl_xor(x, k, 64));
    y = fmaxf(y, __shfl_xor(y, k, 64));
  }
  return float2{x, y};
}
// Power of two that keeps |dS| <= 2 |do| |v| below 2^15.
__device__ __forceinline__ float ds_scale(float x, float y) {
  float e = (x > 0.f && y > 0.f) ? 14.f - ceilf(__builtin_amdgcn_logf(x) + __builtin_amdgcn_logf(y)) : 0.f;
  return __builtin_amdgcn_exp2f(fminf(fmaxf(e, -100.f), 100.f));
}

// fp16: the norms of the rows that take part, 16 lanes per row; those without a finite norm are left out.  A workgroup fills one slot of a (batch,
// shared head), whose gradients so do not depend on the others in the call (a place that all rows maximise made 64 000 rows wait 200 us for each other).
__global__ __launch_bounds__(256) void k_attend_norms(AttArgs a, AttGrad g) {
  typedef _Float16 T;
  __shared__ float part[2][4];
  int tid = threadIdx.x, lane = tid & 15;
  int slot = blockIdx.x % g.norm_slots, unit = blockIdx.x / g.norm_slots, hk = unit % a.HK, b = unit / a.HK;
  int64_t rows = (int64_t)queries_of(a, b) * a.G;
  int keys = keys_of(a, b);
  auto square = [&](const T* row, int vec) {
    u32x4 x = load16<T>(row, 8 * lane, a.dv, vec);
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) q = fmaf((float)reinterpret_cast<T*>(&x)[e], (float)reinterpret_cast<T*>(&x)[e], q);
#pragma unroll
    for (int k = 1; k < 16; k *= 2) q += __shfl_xor(q, k, 16);
    return q < __builtin_inff() ? q : 0.f;
  };
  float x = 0.f, y = 0.f;
  int first = slot * 16 + (tid >> 4), step = g.norm_slots * 16;
#pragma unroll 2
  for (int64_t n = first; n < rows; n += step) {
    int h = hk * a.G + (int)(n % a.G), i = (int)(n / a.G);
    if (g.lse[((size_t)b * a.H + h) * a.nq + i] == -__builtin_inff()) continue;
    x = fmaxf(x, square((const T*)g.dO + b * g.dos[0] + (int64_t)i * g.dos[1] + h * g.dos[2], g.dovec));
  }
#pragma unroll 2
  for (int j = first; j < keys; j += step) {
    if (a.mask && !a.mask[b * a.mask_s + j]) continue;
    y = fmaxf(y, square((const T*)a.V + b * a.vs[0] + (int64_t)j * a.vs[1] + hk * a.vs[2], a.vvec));
  }
#pragma unroll
  for (int k = 16; k < 64; k *= 2) {
    x = fmaxf(x, __shfl_xor(x, k, 64));
    y = fmaxf(y, __shfl_xor(y, k, 64));
  }
  if ((tid & 63) == 0) {
    part[0][tid >> 6] = x;
    part[1][tid >> 6] = y;
  }
  __syncthreads();
  if (tid < 2) g.norms[2 * (size_t)blockIdx.x + tid] = sqrtf(fmaxf(fmaxf(part[tid][0], part[tid][1]), fmaxf(part[tid][2], part[tid][3])));
}

// Beyond this, fp32 holds lse too coarsely to recover weights from it: rounded as a logarithm to base 2, to base e and to base 2 again, it
// leaves all weights of a row off by a common factor of up to 3.3 2^-24 |lse|, which a softmax that divides by its own sum does not have.  The row's
// largest score and log2 of its sum are formed again there and kept apart.  At the bounds of two-byte types the factor is an eighth of half a step of
// the type.  fp32 divides by the sum of these weights in any case, and only keeps them from running off (rows of nothing but masks of -1e9, say).
template <typename T> struct Coarse { static constexpr float value = 65536.f; };
template <> struct Coarse<_Float16> { static constexpr float value = 256.f; };
template <> struct Coarse<__bf16> { static constexpr float value = 2048.f; };

// 64 keys a turn, as two blocks of 32 (fp32: one block a turn).  While the matrix unit forms the scores and dP of the next block, the vector unit turns this one's into dS; then
// dQ takes it up.
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, DP == 64 && sizeof(T) == 2 ? 2 : 1) void k_attend_dq(AttArgs a, AttGrad g, int nqt) {
  typedef typename Frag<T>::type frag;
  constexpr int NB = sizeof(T) == 2 ? 2 : 1, BK = 32 * NB, ND = DP / 32, NS = DP / 16, kTile = BK * DP * (int)sizeof(T);
  __shared__ __align__(16) char tile[3][2][kTile];   // K, V
  __shared__ __align__(16) float from[3][BK];        // what a key's scores start from: 0, or -infinity where it takes no part
  __shared__ float side[8];
  constexpr bool kSums = sizeof(T) == 2;             // the table's gradient is formed here
  static_assert(sizeof tile + sizeof from + sizeof side + 5 * kLine * sizeof(float) <= 160 * 1024, "the longest line fits beside the tiles");
  extern __shared__ float dyn[];                     // with a table: bias line, then (kSums) a line of diagonal sums per wave
  int id = die_order(blockIdx.x, a.B * a.HK, a.G * nqt * g.qsplit);
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
  int qt = id % nqt, sp = id / nqt % g.qsplit, bh = id / nqt / g.qsplit, h = bh % a.H, b = bh / a.H, hk = h / a.G;
  if (b >= a.B) return;
  int q0 = qt * 128 + wave * 32, i = q0 + (lane & 31);
  int qn = queries_of(a, b);
  int kn = keys_of(a, b);
  if (qt * 128 >= qn) kn = 0;
  int tiles = (kn + BK - 1) / BK, per = (tiles + g.qsplit - 1) / g.qsplit;
  int t0 = min(sp * per, tiles), t1 = min(t0 + per, tiles);
  int far = a.bk.far, span = far + kPad, nline = 2 * span + 1;
  float* line = dyn;
  float* diag = dyn + nline;

  const T* K = (const T*)a.K + b * a.ks[0] + hk * a.ks[2];
  const T* V = (const T*)a.V + b * a.vs[0] + hk * a.vs[2];
  const uint8_t* mrow = a.mask ? a.mask + b * a.mask_s : nullptr;
  constexpr uint64_t kAll = NB == 2 ? ~0ull : 0xffffffffull;
  int whole = mrow ? -1 : kn / BK;           // tiles before this one are kept as a whole
  struct Loads {
    Stage<T, DP, BK, VEC> k, v;
    uint8_t mask = 0;
  };
  Loads tl;
  auto fetch = [&](Loads& x, int t) {
    x.k.load(K + (int64_t)t * BK * a.ks[1], a.ks[1], kn - t * BK, a.d, tid);
    x.v.load(V + (int64_t)t * BK * a.vs[1], a.vs[1], kn - t * BK, a.dv, tid);
    if (mrow) x.mask = (lane < BK && t * BK + lane < kn) ? mrow[t * BK + lane] : 0;
  };
  auto put = [&](const Loads& x, int t, int at) {
    uint64_t keep = t < whole ? kAll : keep_bits(min(max(kn - t * BK, 0), BK), mrow, x.mask);
    x.k.store(tile[at][0], keep, tid);
    x.v.store(tile[at][1], keep, tid);
    if (keep != kAll && tid < BK) from[at][tid] = ((keep >> tid) & 1) ? 0.f : -__builtin_inff();
    return keep;
  };
  // All that the next loop needs first is asked for before anything is waited for (one latency instead of four): a pass over the row ahead of the
  // main one needs one tile.
  Loads t2;
  bool row_pass = g.whole_rows && (g.qsplit == 1 || g.rows_only);
  auto first_tiles = [&](bool both) {
    if (t0 < t1) {
      fetch(tl, t0);
      if (both) fetch(t2, t0 + 1);
    }
  };
  first_tiles(!row_pass);
  size_t row = ((size_t)b * a.H + h) * a.nq + i;
  float lse = i < qn ? g.lse[row] : -__builtin_inff(), delta = 0.f;
  frag q[NS], dof[NS];
  {
    const T* qr = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + h * a.qs[2];
    const T* dr = (const T*)g.dO + b * g.dos[0] + (int64_t)i * g.dos[1] + h * g.dos[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = reg_frag<T>(qr, i < qn, s, a.d, a.qvec, lane);
      dof[s] = reg_frag<T>(dr, i < qn, s, a.dv, g.dovec, lane);
    }
    const T* orow = (const T*)g.O + (((int64_t)b * a.nq + i) * a.H + h) * a.dv;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      frag o = reg_frag<T>(orow, i < qn, s, a.dv, g.ovec, lane);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)o[e], (float)dof[s][e], delta);
    }
  }
  bool some = lse != -__builtin_inff();      // something is left in the row
  bool empty = __any(!some);
  delta = some ? both_sum(delta) : 0.f;
  float lo = some ? lse * kLog2e : __builtin_inff(), hi = 0.f;   // weights are exp2((s - hi) - lo)
  bool wide = fabsf(lse) > Coarse<T>::value && fabsf(lse) < __builtin_inff();
  if (!some) {                               // whatever the row holds
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = dof[s] = frag{};
  }
  if (__any(wide) && lane == 0) side[wave] = 1.f;
  else if (lane == 0) side[wave] = 0.f;
  const float* ln = nullptr;
  if (a.table) {
    fill_line<T>(line, a, h, tid, 256);
    for (int n = tid; kSums && n < 4 * nline; n += 256) diag[n] = 0.f;
    ln = line;
  }
  // a power of two: dS is formed times it.  fp16: a row's own, from its |do_i|, so that a row of small gradients keeps its bits beside others of large ones
  // (|do| 2^-20 of the largest, weights of 1 / 2000: dQ off by 3e-2 of itself with one for all, 4e-4 so).
  float cs = 1.f, uncs = 1.f;
  if constexpr (__is_same(T, _Float16)) {
    float z = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) z = fmaf((float)dof[s][e], (float)dof[s][e], z);
    cs = ds_scale(sqrtf(both_sum(z)), norms_of(g, b * a.HK + hk, lane).y);
    uncs = 1.f / cs;
  }
  auto scores_start = [&](int at, int first) {
    f32x16 c;
    const float* x = from[at] + first + 4 * half;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      f32x4 y = *(const f32x4*)(x + 8 * n);
#pragma unroll
      for (int e = 0; e < 4; ++e) c[4 * n + e] = y[e];
    }
    return c;
  };
  f32x16 acc[ND], sc[2], pc[2];              // of a turn's two blocks: scores, dP
  sc[0] = pc[0] = f32x16{};
  uint64_t k0 = 0, k1 = 0;                   // keys of this tile and the next that take part
#pragma unroll
  for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
  float sl = 0.f, sr = 0.f, left = 0.f, right = 0.f;
  double psum = 0.0, rest = 0.0;             // fp32: sums of the row's p and dS
  int rel = rest_below(-(int64_t)q0 - start_of(a, b));
  // The row from its keys of tiles [from_, to), ahead of the pass: f(scores' products, dP, mul, add) for every block of 32.  The next tile is on its way meanwhile,
  // and the first one already where `asked`.
  auto whole_row = [&](int from_, int to, bool asked, auto f) {
    if (from_ < to && !asked) fetch(tl, from_);
    for (int t = from_, at = 0; t < to; ++t, at ^= 1) {
      uint64_t keep = put(tl, t, at);
      fetch(tl, t + 1);
      __syncthreads();
      if (ln) {
        left = uniform(line[kPad]);
        right = uniform(line[2 * far + kPad]);
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        f32x16 s = f32x16{}, dp = f32x16{};
        if (keep != kAll) s = scores_start(at, 32 * n);
#pragma unroll
        for (int k = 0; k < NS; ++k) s = Frag<T>::mma(row_frag<T, DP>(tile[at][0], 32 * n, k, lane), q[k], s);
#pragma unroll
        for (int k = 0; k < NS; ++k) dp = Frag<T>::mma(row_frag<T, DP>(tile[at][1], 32 * n, k, lane), dof[k], dp);
        float mul = a.c2, add = 0.f;
        if (ln) add_bias<true>(s, a.c2, ln, far, rel + t * BK + 32 * n, left, right, lane, mul, add);
        f(s, dp, mul, add);
      }
    }
    __syncthreads();
  };
  __syncthreads();
  bool any_wide = uniform(side[0] + side[1] + side[2] + side[3]) != 0.f;
  if (any_wide) {
    float top = -__builtin_inff(), sum = 0.f;
    whole_row(0, tiles, false, [&](const f32x16& s, const f32x16&, float mul, float add) {
      float x[16], big = top;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = fmaf(s[r], mul, add);
        big = fmaxf(big, x[r]);
      }
      float ref = big == -__builtin_inff() ? 0.f : big;
      sum *= __builtin_amdgcn_exp2f(top - ref);
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(x[r] - ref);
      top = big;
    });
    float both = both_max(top);
    sum = both_sum(top == -__builtin_inff() ? 0.f : sum * __builtin_amdgcn_exp2f(top - both));
    if (wide) hi = both, lo = __builtin_amdgcn_logf(sum);
  }
  bool coarse = __any(hi != 0.f);
  if (g.whole_rows) {
    // delta_i = sum_j p_ij dP_ij / sum_j p_ij; of a split row from the parts that a launch of this kernel with rows_only left
    float total = 0.f, sd = 0.f;
    size_t rows = (size_t)a.B * a.H * a.nq;
    if (row_pass) {
      whole_row(t0, t1, !any_wide, [&](const f32x16& s, const f32x16& dp, float mul, float add) {
        f32x16 y = s;
        if (coarse) {
#pragma unroll
          for (int r = 0; r < 16; ++r) y[r] = fmaf(s[r], mul, add) - hi;
          mul = 1.f;
          add = 0.f;
        }
        add -= lo;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float x = __builtin_amdgcn_exp2f(fmaf(y[r], mul, add));
          total += x;
          sd = fmaf(x, dp[r], sd);
        }
      });
      total = both_sum(total);
      sd = both_sum(sd);
      if (g.rows_only) {
        if (half == 0 && i < qn) *(float2*)(g.rsum + 2 * (sp * rows + row)) = float2{total, sd};
        return;
      }
    } else if (i < qn) {
      for (int k = 0; k < g.qsplit; ++k) {
        float2 x = *(const float2*)(g.rsum + 2 * (k * rows + row));
        total += x.x;
        sd += x.y;
      }
    }
    delta = some && total != 0.f ? sd / total : 0.f;
  }
  if (half == 0 && i < qn && sp == 0) g.delta[row] = delta, g.lo[row] = lo, g.hi[row] = hi;   // for the next pass
  lo -= __builtin_amdgcn_logf(cs);
  if (any_wide || row_pass) first_tiles(true);
  if (t0 < t1) {
    k0 = put(tl, t0, 0);
    k1 = put(t2, t0 + 1, 1);
  }
  settle();
  __syncthreads();
  if (ln) {
    left = uniform(line[kPad]);
    right = uniform(line[2 * far + kPad]);
  }
  if (t0 < t1) {
    if (k0 != kAll) sc[0] = scores_start(0, 0);
#pragma unroll
    for (int k = 0; k < NS; ++k) sc[0] = Frag<T>::mma(row_frag<T, DP>(tile[0][0], 0, k, lane), q[k], sc[0]);
#pragma unroll
    for (int k = 0; k < NS; ++k) pc[0] = Frag<T>::mma(row_frag<T, DP>(tile[0][1], 0, k, lane), dof[k], pc[0]);
  }
  int now = 0;
  // Block of the turn at buffer `at`; the next block: rows 32 (block ^ 1) on of buffer `on`, whose tile keeps the keys `keep`.
  auto block = [&](auto block_, int rel0, int at, int on, uint64_t keep) {
    constexpr int B = decltype(block_)::value, here = NB == 2 ? 32 * B : 0, there = NB == 2 ? 32 * (B ^ 1) : 0;   // rows in their tiles
    f32x16 &s = sc[B], &dp = pc[B], &s2 = sc[B ^ 1], &dp2 = pc[B ^ 1];
    float mul = a.c2, add = 0.f;
    int where = 1;
    if (ln) where = add_bias<true>(s, a.c2, ln, far, rel0, left, right, lane, mul, add);
    if (coarse) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], mul, add) - hi;
      mul = 1.f;
      add = 0.f;
    }
    add -= lo;
    const char *kt = tile[on][0], *vt = tile[on][1], *ko = tile[at][0];
    constexpr int A = 2 * NS, M = A + 2 * ND;
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, left_over[4] = {0.f, 0.f, 0.f, 0.f};
    auto operand = [&](int z) {
      return z < NS ? row_frag<T, DP>(kt, there, z, lane)
             : z < A ? row_frag<T, DP>(vt, there, z - NS, lane)
                     : col_frag<T, DP>(ko, here + 16 * ((z - A) / ND), 32 * ((z - A) % ND), lane);
    };
    frag f[3], ds[2];
    f[0] = operand(0);
    f[1] = operand(1);
#pragma unroll
    for (int z = 0; z < M; ++z) {
      __builtin_amdgcn_sched_barrier(0);
      if (z + 2 < M) f[(z + 2) % 3] = operand(z + 2);
      if (z == 0) {
        if (keep == kAll) s2 = Frag<T>::mma(f[0], q[0], f32x16{});
        else s2 = Frag<T>::mma(f[0], q[0], scores_start(on, there));
        dp2 = f32x16{};
      } else if (z < NS) s2 = Frag<T>::mma(f[z % 3], q[z], s2);
      else if (z < A) dp2 = Frag<T>::mma(f[z % 3], dof[z - NS], dp2);
      else acc[(z - A) % ND] = Frag<T>::mma(f[z % 3], ds[(z - A) / ND], acc[(z - A) % ND]);
      if (z < A) {
#pragma unroll
        for (int r = z * 16 / A; r < (z + 1) * 16 / A; ++r) {
          float x = __builtin_amdgcn_exp2f(fmaf(s[r], mul, add));
          // fp32: dP - delta would be rounded on dP's grid, the same way for all keys whose dP has an exponent: a delta off by that much for the row
          s[r] = kSums ? x * (dp[r] - delta) : fmaf(x, dp[r], -(x * delta));
          if constexpr (!kSums) sum[r & 3] += x, left_over[r & 3] += s[r];
          if (r == 7) ds[0] = pack8<T>(s, 0);
          if (r == 15) ds[1] = pack8<T>(s, 1);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!kSums) {
      psum += (double)((sum[0] + sum[1]) + (sum[2] + sum[3]));
      rest += (double)((left_over[0] + left_over[1]) + (left_over[2] + left_over[3]));
    }
    if (kSums && ln) {
      if (empty) {                           // an infinity in a key or value of others makes NaN of these lanes' zeros
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = some ? s[r] : 0.f;
      }
      if constexpr (__is_same(T, _Float16)) {  // rows of unlike scales meet in the table
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= uncs;
      }
      if (where == 0) {
        add_diagonals(s, diag + wave * nline + rel0 + span, lane);
      } else {
        float x = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) x += s[r];
        if (where < 0) sl += x;
        else sr += x;
      }
    }
  };
  for (int t = t0; t < t1; ++t) {
    int nxt = now == 2 ? 0 : now + 1, last = nxt == 2 ? 0 : nxt + 1;
    fetch(tl, t + 2);
    if constexpr (NB == 2) {
      block(Const<0>{}, rel + t * BK, now, now, k0);
      block(Const<1>{}, rel + t * BK + 32, now, nxt, k1);
    } else {
      block(Const<0>{}, rel + t * BK, now, nxt, k1);
      sc[0] = sc[1];
      pc[0] = pc[1];
    }
    k0 = k1;
    k1 = put(tl, t + 2, last);
    now = nxt;
    __syncthreads();
  }
  if constexpr (!kSums) {
    psum += __shfl_xor(psum, 32, 64);
    rest += __shfl_xor(rest, 32, 64);
    if (!some) psum = rest = 0.0;
    if (g.qsplit == 1) {
      double w = psum != 0.0 ? 1.0 / psum : 0.0;
      uncs = (float)w;
      if (half == 0 && i < qn) g.w[row] = uncs, g.delta[row] = (float)((double)delta + rest * w);
    } else if (half == 0 && i < a.nq) {
      *(double2*)((double*)g.rsum + 2 * ((size_t)sp * a.B * a.H * a.nq + row)) = double2{psum, rest};
    }
  }
  if (i < a.nq) {
    float f = a.scale * uncs;
    int64_t at = (((int64_t)b * a.nq + i) * a.H + h) * a.d;
    auto write = [&](auto* out, int vec) {
#pragma unroll
      for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          store4(out, 32 * n + 8 * r + 4 * half, a.d, vec, acc[n][4 * r] * f, acc[n][4 * r + 1] * f, acc[n][4 * r + 2] * f, acc[n][4 * r + 3] * f);
    };
    if (!some) {
#pragma unroll
      for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
    }
    if (g.qsplit == 1) write((T*)g.dQ + at, g.dqvec);
    else write(g.pq + sp * ((int64_t)a.B * a.nq * a.H * a.d) + at, a.d % 4 == 0);
  }
  if (kSums && ln) {                         // the loop's last barrier stands before this
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      sl += __shfl_xor(sl, x, 64);
      sr += __shfl_xor(sr, x, 64);
    }
    if (lane == 0) {
      side[wave] = sl;
      side[4 + wave] = sr;
    }
    for (int n = tid; n < nline; n += 256) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) x += diag[k * nline + n];
      line[n] = x;
    }
    __syncthreads();
    float* out = g.tsum + ((((size_t)h * a.B + b) * g.qsplit + sp) * nqt + qt) * a.bk.buckets;
    bucket_sums(a.bk, line, span, side[0] + side[1] + side[2] + side[3], side[4] + side[5] + side[6] + side[7], out, tid);
  }
}

// fp32: the dQ pass's sums of a row's p and dS in parts, and its dQ, joined: four features per thread.
__global__ __launch_bounds__(256) void k_attend_rows(AttArgs a, AttGrad g) {
  int64_t rows = (int64_t)a.B * a.H * a.nq, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int nc = (a.d + 3) / 4, c = 4 * (int)(t % nc);
  int64_t n = t / nc;
  if (n >= rows) return;
  int64_t at = (n / a.H / a.nq * a.H + n % a.H) * a.nq + n / a.H % a.nq;
  double psum = 0.0, rest = 0.0;
  float y[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < g.qsplit; ++k) {
    double2 x = *(const double2*)((const double*)g.rsum + 2 * (k * rows + at));
    psum += x.x;
    rest += x.y;
    const float* part = g.pq + (k * rows + n) * a.d + c;
    if (a.d % 4 == 0) {
      f32x4 v = *(const f32x4*)part;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < a.d) y[e] += part[e];
    }
  }
  double inv = psum != 0.0 ? 1.0 / psum : 0.0;
  float w = (float)inv;
  store4((float*)g.dQ + n * a.d, c, a.d, g.dqvec, y[0] * w, y[1] * w, y[2] * w, y[3] * w);
  if (c == 0) {
    g.w[at] = w;
    g.delta[at] = (float)((double)g.delta[at] + rest * inv);
  }
}

// 64 queries of one head a turn, the heads of the group one after the other; else like k_attend_dq.  Workgroups from `grid` on add up the table's
// gradient that the dQ pass left, a wave per entry (a launch of its own takes 4.6 us).
//
// fp32 takes p times 1 over its row's sum, and delta with the row's rest of dS, from the dQ pass, and so sums the table's gradient here, head by head.
// Weights recovered from an fp32 lse are off by up to 1e-6 a row, and a delta from the rounded o leaves a rest where dS should sum to zero, which
// stands against what is left of a bucket.  Over 30 drawn calls the errors of dQ, dK, dV and the table, in units of the formula's own steps in fp32, were
// 1.25, 1.3, 1.3 and 1.2 in the median without this and are 1.0, 1.0, 1.0 and 0.6 (training step of 2 x 8 heads, 500 x 1000: 142 / 150 us; the same
// from a pass over the row ahead of the dQ pass, as in two-byte types: 181).
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, DP == 64 && sizeof(T) == 2 ? 2 : 1) void k_attend_dkv(AttArgs a, AttGrad g, int nkt, int grid) {
  typedef typename Frag<T>::type frag;
  constexpr int NB = sizeof(T) == 2 ? 2 : 1, BQ = 32 * NB, ND = DP / 32, NS = DP / 16, kTile = BQ * DP * (int)sizeof(T);
  constexpr bool kSums = sizeof(T) == 4;              // the table's gradient is formed here
  __shared__ __align__(16) char tile[3][2][kTile];    // Q, dO
  __shared__ __align__(16) float stat[3][kSums ? 4 : 3][BQ];   // lo, delta (scaled like dS), hi, 1 / sum of p
  __shared__ double side[8];
  __shared__ int touched[4];                          // whether a wave's line holds anything
  static_assert(sizeof tile + sizeof stat + sizeof side + sizeof touched + (kSums ? 5 : 1) * kLine * sizeof(float) <= 160 * 1024, "the longest line fits beside the tiles");
  extern __shared__ float dyn[];                      // with a table: bias line, then (kSums) a line of diagonal sums per wave, turned over
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
  if ((int)blockIdx.x >= grid) {
    int n = 4 * ((int)blockIdx.x - grid) + wave;
    if (n < a.H * a.bk.buckets)
      join_bucket<T>(g.tsum, a.B * g.qsplit * ((a.nq + 127) / 128), a.bk.buckets, n / a.bk.buckets, n % a.bk.buckets, lane, (T*)g.dtable);
    return;
  }
  int id = die_order(blockIdx.x, a.B * a.HK, nkt * g.ksplit);
  int kt = id % nkt, sp = id / nkt % g.ksplit, bh = id / nkt / g.ksplit, hk = bh % a.HK, b = bh / a.HK;
  if (b >= a.B) return;
  int k0 = kt * 128 + wave * 32, j = k0 + (lane & 31);
  int qn = queries_of(a, b);
  int kn = keys_of(a, b);
  if (kt * 128 >= kn) qn = 0;
  int tiles = (qn + BQ - 1) / BQ, steps = tiles * a.G, per = (steps + g.ksplit - 1) / g.ksplit;   // a part: some tiles of some heads
  int t0 = min(sp * per, steps), t1 = min(t0 + per, steps);
  int far = a.bk.far, span = far + kPad, nline = 2 * span + 1;
  const float* ln = a.table ? dyn : nullptr;
  float* diag = dyn + nline;
  auto sums_of = [&](int head) { return (double*)g.tsum + ((((size_t)head * a.B + b) * g.ksplit + sp) * nkt + kt) * a.bk.buckets; };
  if (kSums && ln) {
    for (int n = tid; n < 4 * nline; n += 256) diag[n] = 0.f;
    // heads that this part has no tile of
    int first = t0 < t1 ? t0 / tiles : a.G, last = t0 < t1 ? (t1 - 1) / tiles : -1;
    for (int n = tid; n < a.G * a.bk.buckets; n += 256) {
      int x = n / a.bk.buckets;
      if (x < first || x > last) sums_of(hk * a.G + x)[n % a.bk.buckets] = 0.0;
    }
  }
  bool mine = j < kn;
  struct Loads {
    Stage<T, DP, BQ, VEC> q, d;
    float lo, delta, hi, w;                  // of row `lane` of the tile
  };
  Loads tl, t2;
  int h = hk * a.G + (tiles ? t0 / tiles : 0), i0 = tiles ? t0 % tiles * BQ : 0;   // head and first row of the turn's tile
  int fh = h, fi = i0;                       // and of the tile to fetch next
  auto fetch = [&](Loads& x) {
    int rows = fh < (hk + 1) * a.G ? qn - fi : 0;
    x.q.load((const T*)a.Q + b * a.qs[0] + (int64_t)fi * a.qs[1] + fh * a.qs[2], a.qs[1], rows, a.d, tid);
    x.d.load((const T*)g.dO + b * g.dos[0] + (int64_t)fi * g.dos[1] + fh * g.dos[2], g.dos[1], rows, a.dv, tid);
    size_t row = ((size_t)b * a.H + fh) * a.nq + fi + lane;
    x.lo = __builtin_inff();
    x.delta = x.hi = x.w = 0.f;
    if (lane < BQ && lane < rows) {
      x.lo = g.lo[row], x.delta = g.delta[row], x.hi = g.hi[row];
      if constexpr (kSums) x.w = g.w[row];
    }
    fi += BQ;
    if (fi >= qn) fi = 0, ++fh;
  };
  // as in k_attend_dq, ahead of the first wait
  if (t0 < t1) {
    fetch(tl);
    fetch(t2);
  }
  frag kf[NS], vf[NS];
  {
    const T* kr = (const T*)a.K + b * a.ks[0] + (int64_t)j * a.ks[1] + hk * a.ks[2];
    const T* vr = (const T*)a.V + b * a.vs[0] + (int64_t)j * a.vs[1] + hk * a.vs[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      kf[s] = reg_frag<T>(kr, mine, s, a.d, a.kvec, lane);
      vf[s] = reg_frag<T>(vr, mine, s, a.dv, a.vvec, lane);
    }
  }
  if (a.mask && mine) mine = a.mask[b * a.mask_s + j] != 0;
  if (!mine) {                               // whatever the key holds
#pragma unroll
    for (int s = 0; s < NS; ++s) kf[s] = vf[s] = frag{};
  }
  constexpr float kLift = PLift<T>::value;
  float cs = 1.f;                            // fp16: one power of two for all rows of the shared head, which add up
  if constexpr (__is_same(T, _Float16)) {
    float2 z = norms_of(g, b * a.HK + hk, lane);
    cs = uniform(ds_scale(z.x, z.y));
  }
  float unlift = 1.f / (float)(1 << (int)kLift), ck = cs * unlift;
  // Rows that take no part run along with zeros, of which a key that holds an infinity or NaN makes NaN.  Where it does (a product with zero tells such
  // keys) their blocks go the way of rows with a `hi`, where the minimum with a number makes a number of NaN; their lo is infinite, so the weight is
  // zero.  (Rows that count have a lo of NaN beside a score of NaN.  fp32: an infinite value makes NaN of their dS for the table.)
  float z = 0.f;
  if constexpr (sizeof(T) == 2) {
    f32x16 c = f32x16{};
#pragma unroll
    for (int k = 0; k < NS; ++k) c = Frag<T>::mma(frag{}, kf[k], c);
    z = c[0];
  } else {
#pragma unroll
    for (int k = 0; k < NS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) z = fmaf(kf[k][e], 0.f, fmaf(vf[k][e], 0.f, z));
  }
  bool odd = __any(z != 0.f);
  auto put = [&](const Loads& x, int at) {
    constexpr uint64_t kAll = NB == 2 ? ~0ull : 0xffffffffull;
    uint64_t keep = __ballot(x.lo != __builtin_inff()) & kAll;
    x.q.store(tile[at][0], keep, tid);
    x.d.store(tile[at][1], keep, tid);
    if (tid < BQ) {
      stat[at][0][tid] = x.lo;                 // infinite where nothing is left in the row: weights zero
      stat[at][1][tid] = x.delta * ck;
      stat[at][2][tid] = x.hi;
      if constexpr (kSums) stat[at][3][tid] = x.w;
    }
    return __any(x.hi != 0.f) || (odd && keep != kAll);
  };
  f32x16 dk[ND], dv[ND], sc[2], pc[2];       // of a turn's two blocks: scores, dP
  sc[0] = pc[0] = f32x16{};
#pragma unroll
  for (int n = 0; n < ND; ++n) dk[n] = dv[n] = f32x16{};
  float left = 0.f, right = 0.f;
  double sl = 0.0, sr = 0.0;                 // of rows beyond the last edges, whose dS sum to zero only across all keys: nothing may be lost on the way
  bool bare = __any(!mine);                  // keys that take no part
  bool near = false;                         // the wave has added to its line
  int rel = rest_above((int64_t)k0 - start_of(a, b));
  bool c0 = false, c1 = false;               // whether this tile and the next have rows with a `hi`, or zeros beside odd keys
  if (t0 < t1) {
    c0 = put(tl, 0);
    c1 = put(t2, 1);
  }
  settle();
  __syncthreads();
  if (t0 < t1) {
#pragma unroll
    for (int k = 0; k < NS; ++k) sc[0] = Frag<T>::mma(row_frag<T, DP>(tile[0][0], 0, k, lane), kf[k], sc[0]);
#pragma unroll
    for (int k = 0; k < NS; ++k) pc[0] = Frag<T>::mma(row_frag<T, DP>(tile[0][1], 0, k, lane), vf[k], pc[0]);
  }
  int now = 0;
  // Block of the turn at buffer `at` (rel0: its differences, wide: see c0); the next block: rows 32 (block ^ 1) on of buffer `on`.
  auto block = [&](auto block_, int rel0, int at, int on, bool wide) {
    constexpr int B = decltype(block_)::value, here = NB == 2 ? 32 * B : 0, there = NB == 2 ? 32 * (B ^ 1) : 0;   // rows in their tiles
    f32x16 &s = sc[B], &dp = pc[B], &s2 = sc[B ^ 1], &dp2 = pc[B ^ 1];
    float mul = a.c2, add = 0.f;
    const float* st = stat[at][0] + here + 4 * half;
    f32x4 l4[4], d4[4], w4[4];
    auto stats = [&](int n) {
      l4[n] = *(const f32x4*)(st + 8 * n);
      d4[n] = *(const f32x4*)(st + BQ + 8 * n);
      if constexpr (kSums) w4[n] = *(const f32x4*)(st + 3 * BQ + 8 * n);
    };
#pragma unroll
    for (int n = 0; n < (kSums ? 1 : 4); ++n) stats(n);   // fp32: the others as they are wanted, its products leave time and its registers no room
    int where = 1;
    if (ln) where = add_bias<false>(s, a.c2, ln, far, rel0, left, right, lane, mul, add);
    if (wide) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        f32x4 h4 = *(const f32x4*)(st + 2 * BQ + 8 * n);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * n + e] = fminf(fmaf(s[4 * n + e], mul, add) - h4[e], 3e38f);
      }
      mul = 1.f;
      add = 0.f;
    }
    add += kLift;
    const char *qt = tile[on][0], *dt = tile[on][1], *qo = tile[at][0], *od = tile[at][1];
    s2 = dp2 = f32x16{};
    constexpr int A = 2 * NS, M = A + 4 * ND;
    auto operand = [&](int z) {
      return z < NS ? row_frag<T, DP>(qt, there, z, lane)
             : z < A ? row_frag<T, DP>(dt, there, z - NS, lane)
                     : col_frag<T, DP>((z - A) / ND % 2 ? qo : od, here + 16 * ((z - A) / (2 * ND)), 32 * ((z - A) % ND), lane);
    };
    frag f[3], p[2], ds[2];
    f[0] = operand(0);
    f[1] = operand(1);
#pragma unroll
    for (int z = 0; z < M; ++z) {
      __builtin_amdgcn_sched_barrier(0);
      if (z + 2 < M) f[(z + 2) % 3] = operand(z + 2);
      constexpr int N2 = 2 * ND;
      int y = z - A;
      if (z < NS) s2 = Frag<T>::mma(f[z % 3], kf[z], s2);
      else if (z < A) dp2 = Frag<T>::mma(f[z % 3], vf[z - NS], dp2);
      else if (y / ND % 2 == 0) dv[y % ND] = Frag<T>::mma(f[z % 3], p[y / N2], dv[y % ND]);
      else dk[y % ND] = Frag<T>::mma(f[z % 3], ds[y / N2], dk[y % ND]);
      if (z < A) {
#pragma unroll
        for (int r = z * 16 / A; r < (z + 1) * 16 / A; ++r) {
          if (kSums && r % 4 == 0 && r < 12) stats(r / 4 + 1);
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, add - l4[r >> 2][r & 3]));
          if constexpr (kSums) s[r] *= w4[r >> 2][r & 3];
          dp[r] = kSums ? fmaf(s[r], dp[r], -(s[r] * d4[r >> 2][r & 3])) : s[r] * fmaf(dp[r], ck, -d4[r >> 2][r & 3]);
          if (r == 7) p[0] = pack8<T>(s, 0), ds[0] = pack8<T>(dp, 0);
          if (r == 15) p[1] = pack8<T>(s, 1), ds[1] = pack8<T>(dp, 1);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (kSums && ln) {
      if (bare) {
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = mine ? dp[r] : 0.f;
      }
      if (wide) {
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = st[8 * (r >> 2) + (r & 3)] < __builtin_inff() ? dp[r] : 0.f;
      }
      if (where == 0) {
        add_diagonals(dp, diag + wave * nline + span - rel0, lane);   // queries in the registers: the line runs the other way
        near = true;
      } else {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r & 3] += dp[r];
        (where < 0 ? sl : sr) += (double)((x[0] + x[1]) + (x[2] + x[3]));
      }
    }
  };
  // The sums of a head by bucket; a barrier stands before it and before what writes the lines next.
  auto flush = [&](int head) {
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      sl += __shfl_xor(sl, x, 64);
      sr += __shfl_xor(sr, x, 64);
    }
    if (lane == 0) {
      side[wave] = sl;
      side[4 + wave] = sr;
      touched[wave] = near;
    }
    sl = sr = 0.0;
    near = false;
    __syncthreads();
    double all_left = side[0] + side[1] + side[2] + side[3], all_right = side[4] + side[5] + side[6] + side[7], *out = sums_of(head);
    if (!uniform(touched[0] | touched[1] | touched[2] | touched[3])) {   // all beyond the last edges: the lines are zero
      int E = a.bk.n_edges;
      for (int n = tid; n < a.bk.buckets; n += 256) out[n] = (n == E ? all_left : 0.0) + (n == (a.bk.two_sided ? 2 * E + 1 : 0) ? all_right : 0.0);
      return;
    }
    for (int n = tid; n < nline; n += 256) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float* from = diag + k * nline + nline - 1 - n;
        x += *from;
        *from = 0.f;
      }
      dyn[n] = x;
    }
    __syncthreads();
    bucket_sums(a.bk, dyn, span, all_left, all_right, out, tid);
  };
  for (int t = t0; t < t1; ++t) {
    if (ln && (i0 == 0 || t == t0)) {        // another head: its bias line (nobody reads the old one any more)
      if (kSums && t > t0) {
        flush(h - 1);
        __syncthreads();
      }
      fill_line<T>(dyn, a, h, tid, 256);
      __syncthreads();
      left = uniform(ln[kPad]);
      right = uniform(ln[2 * far + kPad]);
    }
    int nxt = now == 2 ? 0 : now + 1, last = nxt == 2 ? 0 : nxt + 1;
    fetch(tl);
    if constexpr (NB == 2) {
      block(Const<0>{}, rel - i0, now, now, c0);
      block(Const<1>{}, rel - i0 - 32, now, nxt, c0);
    } else {
      block(Const<0>{}, rel - i0, now, nxt, c0);
      sc[0] = sc[1];
      pc[0] = pc[1];
    }
    c0 = c1;
    c1 = put(tl, last);
    now = nxt;
    i0 += BQ;
    if (i0 >= qn) i0 = 0, ++h;
    __syncthreads();
  }
  if (kSums && ln && t0 < t1) flush(hk * a.G + (t1 - 1) / tiles);
  if (j >= a.nk) return;
  float fk = a.scale / cs;
  int64_t at = ((int64_t)b * a.nk + j) * a.HK + hk, all = (int64_t)a.B * a.nk * a.HK;
  auto write = [&](auto* ok, int kvec, auto* ov, int vvec) {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        int c = 32 * n + 8 * r + 4 * half;
        f32x4 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = mine ? dk[n][4 * r + e] * fk : 0.f;
          y[e] = mine ? dv[n][4 * r + e] * unlift : 0.f;
        }
        store4(ok, c, a.d, kvec, x[0], x[1], x[2], x[3]);
        store4(ov, c, a.dv, vvec, y[0], y[1], y[2], y[3]);
      }
  };
  if (g.ksplit == 1) write((T*)g.dK + at * a.d, g.dkvec, (T*)g.dV + at * a.dv, g.dvvec);
  else write(g.pk + (sp * all + at) * a.d, a.d % 4 == 0, g.pv + (sp * all + at) * a.dv, a.dv % 4 == 0);
}

// Parts of a split axis added up in order, out[n] = sum over p of part[p][n], for up to three results in one launch (fp32,
// 2 x 8 heads, 500 x 1000: 6.7 us; a launch for each: 15).
struct Sums {
  const float* part[3];
  void* out[3];
  int64_t n[3];
  int parts[3];
  unsigned first[4];   // workgroups of each: [first[k], first[k + 1]); from first[3] on those that add up the table's gradient, a wave per entry
  const float* tsum;
  int tparts, heads, buckets;
  void* dtable;
};
template <typename T>
__global__ __launch_bounds__(256) void k_attend_sum(Sums z) {
  if (blockIdx.x >= z.first[3]) {
    int n = 4 * (int)(blockIdx.x - z.first[3]) + (int)(threadIdx.x >> 6);
    if (n < z.heads * z.buckets) join_bucket<T>((const double*)z.tsum, z.tparts, z.buckets, n / z.buckets, n % z.buckets, threadIdx.x & 63, (T*)z.dtable);
    return;
  }
  int k = blockIdx.x >= z.first[2] ? 2 : blockIdx.x >= z.first[1] ? 1 : 0;
  const float* part = z.part[k];
  T* out = (T*)z.out[k];
  int64_t n = z.n[k], i = ((int64_t)(blockIdx.x - z.first[k]) * 256 + threadIdx.x) * 4;
  int parts = z.parts[k];
  if (i >= n) return;
  if (n % 4 == 0) {
    f32x4 s = *(const f32x4*)(part + i);
#pragma unroll 4
    for (int p = 1; p < parts; ++p) s += *(const f32x4*)(part + p * n + i);
    store4<T>(out + i, 0, 4, (uintptr_t)out % (4 * sizeof(T)) == 0, s[0], s[1], s[2], s[3]);
  } else {
    for (int64_t j = i; j < n && j < i + 4; ++j) {
      float s = 0.f;
      for (int p = 0; p < parts; ++p) s += part[p * n + j];
      out[j] = (T)s;
    }
  }
}

template <typename T, bool VEC>
void dq_v(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  int nqt = (a.nq + 127) / 128, grid = (a.B * a.H * nqt * g.qsplit + 7) / 8 * 8;
  size_t lds = a.table ? sizeof(float) * (sizeof(T) == 2 ? 5 : 1) * (2 * (a.bk.far + kPad) + 1) : 0;
  if (a.d <= 64 && a.dv <= 64) k_attend_dq<T, 64, VEC><<<grid, 256, lds, s>>>(a, g, nqt);
  else k_attend_dq<T, 128, VEC><<<grid, 256, lds, s>>>(a, g, nqt);
}
template <typename T, bool VEC>
void dkv_v(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  int nkt = (a.nk + 127) / 128, grid = (a.B * a.HK * nkt * g.ksplit + 7) / 8 * 8;
  int more = a.table && sizeof(T) == 2 ? (a.H * a.bk.buckets + 3) / 4 : 0;
  size_t lds = a.table ? sizeof(float) * (sizeof(T) == 2 ? 1 : 5) * (2 * (a.bk.far + kPad) + 1) : 0;
  if (a.d <= 64 && a.dv <= 64) k_attend_dkv<T, 64, VEC><<<grid + more, 256, lds, s>>>(a, g, nkt, grid);
  else k_attend_dkv<T, 128, VEC><<<grid + more, 256, lds, s>>>(a, g, nkt, grid);
}
template <typename T>
void dq_t(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  auto pass = [&](const AttGrad& x) {
    if (a.kvec && a.vvec) dq_v<T, true>(s, a, x);
    else dq_v<T, false>(s, a, x);
  };
  if (g.whole_rows && g.qsplit > 1) {
    AttGrad ahead = g;
    ahead.rows_only = 1;
    pass(ahead);
  }
  pass(g);
  if (sizeof(T) == 4 && g.qsplit > 1) {
    int64_t threads = (int64_t)a.B * a.H * a.nq * ((a.d + 3) / 4);
    k_attend_rows<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a, g);
  }
}
template <typename T>
void dkv_t(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  if (a.qvec && g.dovec) dkv_v<T, true>(s, a, g);
  else dkv_v<T, false>(s, a, g);
}
template <typename T>
void sums_t(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  Sums z{};
  int k = 0;
  auto take = [&](const float* part, int parts, int64_t n, void* out) {
    if (parts < 2 || n == 0) return;
    z.part[k] = part, z.out[k] = out, z.n[k] = n, z.parts[k] = parts;
    z.first[k + 1] = z.first[k] + (unsigned)((n + 1023) / 1024);
    ++k;
  };
  int64_t rows = (int64_t)a.B * a.nq * a.H, keys = (int64_t)a.B * a.nk * a.HK;
  if (sizeof(T) == 2) take(g.pq, g.qsplit, rows * a.d, g.dQ);      // fp32: k_attend_rows
  take(g.pk, g.ksplit, keys * a.d, g.dK);
  take(g.pv, g.ksplit, keys * a.dv, g.dV);
  unsigned all = z.first[k];
  for (; k < 3; ++k) z.first[k + 1] = all;
  if (sizeof(T) == 4 && a.table && keys) {
    z.tsum = g.tsum, z.tparts = a.B * g.ksplit * ((a.nk + 127) / 128), z.heads = a.H, z.buckets = a.bk.buckets, z.dtable = g.dtable;
    all += (a.H * a.bk.buckets + 3) / 4;
  }
  if (all) k_attend_sum<T><<<all, 256, 0, s>>>(z);
}

}  // namespace

void launch_attend_norms(hipStream_t s, int type, const AttArgs& a, const AttGrad& g) {
  if (type == 1) k_attend_norms<<<(unsigned)(a.B * a.HK * g.norm_slots), 256, 0, s>>>(a, g);
}
void launch_attend_dq(hipStream_t s, int type, const AttArgs& a, const AttGrad& g) {
  if (type == 0) dq_t<float>(s, a, g);
  else if (type == 1) dq_t<_Float16>(s, a, g);
  else dq_t<__bf16>(s, a, g);
}
void launch_attend_dkv(hipStream_t s, int type, const AttArgs& a, const AttGrad& g) {
  if (type == 0) dkv_t<float>(s, a, g);
  else if (type == 1) dkv_t<_Float16>(s, a, g);
  else dkv_t<__bf16>(s, a, g);
}
void launch_attend_sums(hipStream_t s, int type, const AttArgs& a, const AttGrad& g) {
  if (type == 0) sums_t<float>(s, a, g);
  else if (type == 1) sums_t<_Float16>(s, a, g);
  else sums_t<__bf16>(s, a, g);
}
