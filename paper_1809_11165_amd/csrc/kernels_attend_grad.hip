// Gradient of the attention (see kernels_attend.hip).  With p_ij = exp(s_ij - lse_i) recomputed tile by tile and delta_i = do_i.o_i,
//     dS_ij = p_ij (do_i.v_j - delta_i),
//     dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_{i, heads of the group} dS_ij q_i,  dV_j = sum_{i, heads} p_ij do_i,
//     dT[h, n] = sum of dS_ij over the pairs of bucket n.
// Two passes, each owning what it writes, so that every sum has a fixed order and nothing is added atomically in memory: k_attend_dq (a
// workgroup owns 128 queries of a head and runs over the keys; transposed scores, like the forward pass) and
// k_attend_dkv (owns 128 keys of a shared head and runs over the queries of all its heads; scores with a key in a lane).  Seven matrix products
// where five would do with dQ added atomically.
//
// fp16: p and dS are scaled by powers of two before they are rounded, dS by the largest |do_i| |v_j| (launch_attend_delta): weights of
// long rows and small gradients would fall among that type's subnormal numbers.
#include "attend_dev.h"

using namespace att;

namespace {

template <typename T> struct PLift { static constexpr float value = 0.f; };
template <> struct PLift<_Float16> { static constexpr float value = 12.f; };

// Power of two that keeps |dS| <= 2 |do| |v| below 2^15.
template <typename T>
__device__ __forceinline__ float ds_scale(const AttGrad& g) {
  if constexpr (sizeof(T) == 2 && __is_same(T, _Float16)) {
    float x = __uint_as_float(g.norms[0]), y = __uint_as_float(g.norms[1]);
    float e = (x > 0.f && y > 0.f) ? 14.f - ceilf(__builtin_amdgcn_logf(x) + __builtin_amdgcn_logf(y)) : 0.f;
    return __builtin_amdgcn_exp2f(fminf(fmaxf(e, -100.f), 100.f));
  }
  return 1.f;
}

__global__ void k_zero_norms(unsigned* n) {
  if (threadIdx.x < 2) n[threadIdx.x] = 0;
}

// Beyond this, fp32 holds lse too coarsely to recover weights from it (a row of nothing but masks of -1e9 or of the type's lowest value).
constexpr float kCoarse = 65536.f;

// Largest score and log2 of the sum relative to it, from the row itself: 16 lanes, a key at a time.  Only for rows beyond kCoarse.
template <typename T>
__device__ void row_sums(const AttArgs& a, int b, int h, int i, int lane, float& hi, float& lo) {
  const T* q = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + h * a.qs[2];
  const T* K = (const T*)a.K + b * a.ks[0] + h / a.G * a.ks[2];
  int kn = a.k_len ? min(max(a.k_len[b], 0), a.nk) : a.nk;
  const int64_t lim = (int64_t)1 << 40;
  int64_t start = a.q_start ? min(max(a.q_start[b], -lim), lim) : 0;
  float m = -__builtin_inff(), l = 0.f;
  for (int j = 0; j < kn; ++j) {
    if (a.mask && !a.mask[b * a.mask_s + j]) continue;
    float s = 0.f;
    for (int c = lane; c < a.d; c += 16) s = fmaf((float)q[c], (float)K[(int64_t)j * a.ks[1] + c], s);
#pragma unroll
    for (int x = 1; x < 16; x *= 2) s += __shfl_xor(s, x, 16);
    float bias = a.table ? bias2<T>(((const T*)a.table)[(size_t)h * a.bk.buckets + bucket_of(a.bk, clamp_rel((int64_t)j - i - start))]) : 0.f;
    s = fmaf(s, a.c2, bias);
    if (s > m) {
      l = l * __builtin_amdgcn_exp2f(m - s) + 1.f;
      m = s;
    } else if (s != -__builtin_inff()) {
      l += __builtin_amdgcn_exp2f(s - m);
    }
  }
  hi = m;
  lo = __builtin_amdgcn_logf(l);
}

// 16 lanes per row (b, i, h): delta, hi and lo, and the largest |do_i| (finite ones) for fp16.
template <typename T>
__global__ __launch_bounds__(256) void k_attend_delta(AttArgs a, AttGrad g) {
  constexpr int E = 16 / (int)sizeof(T);
  int lane = threadIdx.x & 15;
  int64_t n = (int64_t)a.B * a.nq * a.H, row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (row >= n) return;                      // whole groups of 16 lanes
  int h = (int)(row % a.H), i = (int)(row / a.H % a.nq), b = (int)(row / a.H / a.nq);
  int qn = a.q_len ? min(max(a.q_len[b], 0), a.nq) : a.nq;
  size_t at = ((size_t)b * a.H + h) * a.nq + i;
  float s = 0.f, q = 0.f, hi = 0.f, lo = __builtin_inff();
  float lse = i < qn ? g.lse[at] : -__builtin_inff();
  if (lse != -__builtin_inff()) {
    const T* o = (const T*)g.O + row * a.dv;
    const T* d = (const T*)g.dO + b * g.dos[0] + (int64_t)i * g.dos[1] + h * g.dos[2];
    for (int c = lane * E; c < a.dv; c += 16 * E) {
      u32x4 x = load16<T>(o, c, a.dv, g.ovec), y = load16<T>(d, c, a.dv, g.dovec);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float u = (float)reinterpret_cast<T*>(&x)[e], v = (float)reinterpret_cast<T*>(&y)[e];
        s = fmaf(u, v, s);
        q = fmaf(v, v, q);
      }
    }
    lo = lse * kLog2e;
    if (fabsf(lse) > kCoarse && fabsf(lse) < __builtin_inff()) row_sums<T>(a, b, h, i, lane, hi, lo);
  }
#pragma unroll
  for (int x = 1; x < 16; x *= 2) {
    s += __shfl_xor(s, x, 16);
    q += __shfl_xor(q, x, 16);
  }
  if (lane == 0) {
    g.delta[at] = s;
    g.lo[at] = lo;
    g.hi[at] = hi;
    if (__is_same(T, _Float16) && q < __builtin_inff()) atomicMax(&g.norms[0], __float_as_uint(sqrtf(q)));   // a maximum: any order
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_attend_vnorm(AttArgs a, AttGrad g) {
  constexpr int E = 16 / (int)sizeof(T);
  int lane = threadIdx.x & 15;
  int64_t n = (int64_t)a.B * a.nk * a.HK, row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (row >= n) return;
  int h = (int)(row % a.HK), j = (int)(row / a.HK % a.nk), b = (int)(row / a.HK / a.nk);
  if ((a.k_len && j >= a.k_len[b]) || (a.mask && !a.mask[b * a.mask_s + j])) return;
  const T* v = (const T*)a.V + b * a.vs[0] + (int64_t)j * a.vs[1] + h * a.vs[2];
  float q = 0.f;
  for (int c = lane * E; c < a.dv; c += 16 * E) {
    u32x4 x = load16<T>(v, c, a.dv, a.vvec);
#pragma unroll
    for (int e = 0; e < E; ++e) q = fmaf((float)reinterpret_cast<T*>(&x)[e], (float)reinterpret_cast<T*>(&x)[e], q);
  }
#pragma unroll
  for (int x = 1; x < 16; x *= 2) q += __shfl_xor(q, x, 64);
  if (lane == 0 && q < __builtin_inff()) atomicMax(&g.norms[1], __float_as_uint(sqrtf(q)));
}

template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_attend_dq(AttArgs a, AttGrad g, int nqt) {
  typedef typename Frag<T>::type frag;
  constexpr int BK = sizeof(T) == 2 ? 64 : 32, NB = BK / 32, ND = DP / 32, NS = DP / 16, kTile = BK * DP * (int)sizeof(T);
  __shared__ __align__(16) char tile[2][2][kTile];
  extern __shared__ float dyn[];               // with a table: bias line, then eight lines of diagonal sums (wave, half)
  int id = die_order(blockIdx.x, a.B * a.HK, a.G * nqt);
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
  int qt = id % nqt, bh = id / nqt, h = bh % a.H, b = bh / a.H, hk = h / a.G;
  if (b >= a.B) return;
  int q0 = qt * 128 + wave * 32, i = q0 + (lane & 31);
  int qn = queries_of(a, b);
  int kn = keys_of(a, b);
  if (qt * 128 >= qn) kn = 0;
  int tiles = (kn + BK - 1) / BK;
  int far = a.bk.far, span = far + kPad, nline = 2 * span + 1;
  float* line = dyn;
  float* diag = dyn + nline;

  const T* K = (const T*)a.K + b * a.ks[0] + hk * a.ks[2];
  const T* V = (const T*)a.V + b * a.vs[0] + hk * a.vs[2];
  const uint8_t* mrow = a.mask ? a.mask + b * a.mask_s : nullptr;
  size_t row = ((size_t)b * a.H + h) * a.nq + i;
  float lo = __builtin_inff(), hi = 0.f, delta = 0.f;        // nothing left in the row: weights zero
  if (i < qn) lo = g.lo[row], hi = g.hi[row], delta = g.delta[row];
  bool some = lo != __builtin_inff(), coarse = __any(hi != 0.f);
  frag q[NS], dof[NS];
  {
    const T* qr = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + h * a.qs[2];
    const T* dr = (const T*)g.dO + b * g.dos[0] + (int64_t)i * g.dos[1] + h * g.dos[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = reg_frag<T>(qr, some, s, a.d, a.qvec, lane);
      dof[s] = reg_frag<T>(dr, some, s, a.dv, g.dovec, lane);
    }
  }
  const float* ln = nullptr;
  if (a.table) {
    fill_line<T>(line, a, h, tid, 256);
    for (int n = tid; n < 8 * nline; n += 256) diag[n] = 0.f;
    ln = line;
  }
  int64_t start = start_of(a, b);
  float cs = ds_scale<T>(g);

  Stage<T, DP, BK, VEC> sk, sv;
  uint64_t keep = 0;
  uint8_t mb = 0;
  auto fetch = [&](int t) {
    int j0 = t * BK, left = kn - j0;
    sk.load(K + (int64_t)j0 * a.ks[1], a.ks[1], left, a.d, tid);
    sv.load(V + (int64_t)j0 * a.vs[1], a.vs[1], left, a.dv, tid);
    if (mrow) mb = (lane < BK && lane < left) ? mrow[j0 + lane] : 0;
  };
  auto put = [&](int t) {
    keep = keep_bits(min(kn - t * BK, BK), mrow, mb);
    sk.store(tile[t & 1][0], keep, tid);
    sv.store(tile[t & 1][1], keep, tid);
  };
  f32x16 acc[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
  float sl = 0.f, sr = 0.f;
  if (tiles) {
    fetch(0);
    put(0);
  }
  settle();
  __syncthreads();
  float left = 0.f, right = 0.f;
  if (ln) {
    left = line[kPad];
    right = line[2 * far + kPad];
  }
  int rel = rest_below(-(int64_t)q0 - start);
  for (int t = 0; t < tiles; ++t) {
    const char *tk = tile[t & 1][0], *tv = tile[t & 1][1];
    uint64_t kp = keep;
    if (t + 1 < tiles) fetch(t + 1);
    if (kp) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
        for (int k = 0; k < NS; ++k) s = Frag<T>::mma(row_frag<T, DP>(tk, 32 * n, k, lane), q[k], s);
#pragma unroll
        for (int k = 0; k < NS; ++k) dp = Frag<T>::mma(row_frag<T, DP>(tv, 32 * n, k, lane), dof[k], dp);
        int rel0 = rel + t * BK + 32 * n;
        float mul, add;
        int where = add_bias<true>(s, a.c2, ln, far, rel0, left, right, lane, mul, add);
        if (coarse && mul == 1.f) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] -= hi;
        } else {
          add -= hi;
        }
        add -= lo;
        unsigned kb = (unsigned)(kp >> (32 * n));
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, add)) * (dp[r] - delta);
        if (kb != 0xffffffffu) {
          unsigned k = kb >> (4 * half);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = ((k >> (8 * (r >> 2) + (r & 3))) & 1) ? s[r] : 0.f;
        }
        if (ln) {
          if (where == 0) {
            add_diagonals(s, diag + (2 * wave + half) * nline + rel0 + span, lane);
          } else {
            float x = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) x += s[r];
            if (where < 0) sl += x;
            else sr += x;
          }
        }
        if (cs != 1.f) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= cs;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          frag p = pack8<T>(s, u);
#pragma unroll
          for (int c = 0; c < ND; ++c) acc[c] = Frag<T>::mma(col_frag<T, DP>(tk, 32 * n + 16 * u, 32 * c, lane), p, acc[c]);
        }
      }
    }
    if (t + 1 < tiles) put(t + 1);
    __syncthreads();
  }
  if (i < a.nq) {
    float f = a.scale / cs;
    T* out = (T*)g.dQ + (((int64_t)b * a.nq + i) * a.H + h) * a.d;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        store4<T>(out, 32 * n + 8 * r + 4 * half, a.d, g.dqvec, acc[n][4 * r] * f, acc[n][4 * r + 1] * f, acc[n][4 * r + 2] * f, acc[n][4 * r + 3] * f);
  }
  if (ln) {                                  // the loop's last barrier stands before this
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      sl += __shfl_xor(sl, x, 64);
      sr += __shfl_xor(sr, x, 64);
    }
    float* side = (float*)tile;
    if (lane == 0) {
      side[wave] = sl;
      side[4 + wave] = sr;
    }
    for (int n = tid; n < nline; n += 256) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += diag[k * nline + n];
      line[n] = s;
    }
    __syncthreads();
    float* out = g.tsum + ((size_t)h * a.B * nqt + (size_t)b * nqt + qt) * a.bk.buckets;
    bucket_sums(a.bk, line, span, side[0] + side[1] + side[2] + side[3], side[4] + side[5] + side[6] + side[7], out, tid);
  }
}

template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, 1) void k_attend_dkv(AttArgs a, AttGrad g, int nkt) {
  typedef typename Frag<T>::type frag;
  constexpr int BQ = sizeof(T) == 2 ? 64 : 32, NB = BQ / 32, ND = DP / 32, NS = DP / 16, kTile = BQ * DP * (int)sizeof(T);
  __shared__ __align__(16) char tile[2][2][kTile];
  __shared__ __align__(16) float stat[2][3][BQ];      // lo, delta, hi
  extern __shared__ float dyn[];                      // with a table: bias line
  int id = die_order(blockIdx.x, a.B * a.HK, nkt);
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
  int kt = id % nkt, bh = id / nkt, hk = bh % a.HK, b = bh / a.HK;
  if (b >= a.B) return;
  int k0 = kt * 128 + wave * 32, j = k0 + (lane & 31);
  int qn = queries_of(a, b);
  int kn = keys_of(a, b);
  if (kt * 128 >= kn) qn = 0;
  int tiles = (qn + BQ - 1) / BQ, steps = tiles * a.G;
  int far = a.bk.far;
  const float* ln = a.table ? dyn : nullptr;
  bool mine = j < kn && (!a.mask || a.mask[b * a.mask_s + j]);
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
  int64_t start = start_of(a, b);
  float cs = ds_scale<T>(g);

  Stage<T, DP, BQ, VEC> sq, sd;
  float lo = 0.f, delta = 0.f, hi = 0.f;     // of row `lane` of the tile
  bool coarse = false;
  auto fetch = [&](int t) {
    int h = hk * a.G + t / tiles, i0 = t % tiles * BQ, rows = qn - i0;
    sq.load((const T*)a.Q + b * a.qs[0] + (int64_t)i0 * a.qs[1] + h * a.qs[2], a.qs[1], rows, a.d, tid);
    sd.load((const T*)g.dO + b * g.dos[0] + (int64_t)i0 * g.dos[1] + h * g.dos[2], g.dos[1], rows, a.dv, tid);
    size_t row = ((size_t)b * a.H + h) * a.nq + i0 + lane;
    bool have = lane < BQ && lane < rows;
    lo = have ? g.lo[row] : __builtin_inff();
    delta = have ? g.delta[row] : 0.f;
    hi = have ? g.hi[row] : 0.f;
  };
  auto put = [&](int t) {
    uint64_t keep = __ballot(lo != __builtin_inff());
    coarse = __any(hi != 0.f);
    sq.store(tile[t & 1][0], keep, tid);
    sd.store(tile[t & 1][1], keep, tid);
    if (tid < BQ) {
      stat[t & 1][0][tid] = lo;                // infinite where nothing is left in the row: weights zero
      stat[t & 1][1][tid] = delta;
      stat[t & 1][2][tid] = hi;
    }
  };
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) dk[n] = dv[n] = f32x16{};
  float left = 0.f, right = 0.f;
  int rel = rest_above((int64_t)k0 - start);
  if (steps) {
    fetch(0);
    put(0);
  }
  settle();
  for (int t = 0; t < steps; ++t) {
    if (ln && t % tiles == 0) {              // another head: its bias line (nobody reads the old one any more)
      fill_line<T>(dyn, a, hk * a.G + t / tiles, tid, 256);
      __syncthreads();
      left = ln[kPad];
      right = ln[2 * far + kPad];
    } else if (t == 0) {
      __syncthreads();
    }
    const char *tq = tile[t & 1][0], *td = tile[t & 1][1];
    bool wide = coarse;
    if (t + 1 < steps) fetch(t + 1);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
      for (int k = 0; k < NS; ++k) s = Frag<T>::mma(row_frag<T, DP>(tq, 32 * n, k, lane), kf[k], s);
#pragma unroll
      for (int k = 0; k < NS; ++k) dp = Frag<T>::mma(row_frag<T, DP>(td, 32 * n, k, lane), vf[k], dp);
      float mul, add;
      add_bias<false>(s, a.c2, ln, far, rel - (t % tiles * BQ + 32 * n), left, right, lane, mul, add);
      if (wide) {
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 h4 = *(const f32x4*)&stat[t & 1][2][32 * n + 8 * r4 + 4 * half];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * r4 + e] = fmaf(s[4 * r4 + e], mul, add - h4[e]);
        }
        mul = 1.f;
        add = 0.f;
      }
      add += PLift<T>::value;
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 l4 = *(const f32x4*)&stat[t & 1][0][32 * n + 8 * r4 + 4 * half], d4 = *(const f32x4*)&stat[t & 1][1][32 * n + 8 * r4 + 4 * half];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float p = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + e], mul, add - l4[e]));
          s[4 * r4 + e] = p;
          dp[4 * r4 + e] = p * (dp[4 * r4 + e] - d4[e]);
          if (PLift<T>::value != 0.f) dp[4 * r4 + e] *= cs * (1.f / (float)(1 << (int)PLift<T>::value));
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        frag p = pack8<T>(s, u), ds = pack8<T>(dp, u);
#pragma unroll
        for (int c = 0; c < ND; ++c) dv[c] = Frag<T>::mma(col_frag<T, DP>(td, 32 * n + 16 * u, 32 * c, lane), p, dv[c]);
#pragma unroll
        for (int c = 0; c < ND; ++c) dk[c] = Frag<T>::mma(col_frag<T, DP>(tq, 32 * n + 16 * u, 32 * c, lane), ds, dk[c]);
      }
    }
    if (t + 1 < steps) put(t + 1);
    __syncthreads();
  }
  if (j >= a.nk) return;
  float fk = mine ? a.scale / cs : 0.f, fv = 1.f / (float)(1 << (int)PLift<T>::value);
  T* ok = (T*)g.dK + (((int64_t)b * a.nk + j) * a.HK + hk) * a.d;
  T* ov = (T*)g.dV + (((int64_t)b * a.nk + j) * a.HK + hk) * a.dv;
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int c = 32 * n + 8 * r + 4 * half;
      f32x4 x, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = mine ? dk[n][4 * r + e] * fk : 0.f;
        y[e] = mine ? dv[n][4 * r + e] * fv : 0.f;
      }
      store4<T>(ok, c, a.d, g.dkvec, x[0], x[1], x[2], x[3]);
      store4<T>(ov, c, a.dv, g.dvvec, y[0], y[1], y[2], y[3]);
    }
}

template <typename T>
void delta_t(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  int64_t n = (int64_t)a.B * a.nq * a.H, nv = (int64_t)a.B * a.nk * a.HK;
  if (__is_same(T, _Float16)) {
    k_zero_norms<<<1, 64, 0, s>>>(g.norms);
    if (nv) k_attend_vnorm<T><<<(unsigned)((nv + 15) / 16), 256, 0, s>>>(a, g);
  }
  if (n) k_attend_delta<T><<<(unsigned)((n + 15) / 16), 256, 0, s>>>(a, g);
}
template <typename T, bool VEC>
void dq_v(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  int nqt = (a.nq + 127) / 128, grid = (a.B * a.H * nqt + 7) / 8 * 8;
  size_t lds = a.table ? sizeof(float) * 9 * (2 * (a.bk.far + kPad) + 1) : 0;
  if (a.d <= 64 && a.dv <= 64) k_attend_dq<T, 64, VEC><<<grid, 256, lds, s>>>(a, g, nqt);
  else k_attend_dq<T, 128, VEC><<<grid, 256, lds, s>>>(a, g, nqt);
}
template <typename T, bool VEC>
void dkv_v(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  int nkt = (a.nk + 127) / 128, grid = (a.B * a.HK * nkt + 7) / 8 * 8;
  size_t lds = a.table ? sizeof(float) * (2 * (a.bk.far + kPad) + 1) : 0;
  if (a.d <= 64 && a.dv <= 64) k_attend_dkv<T, 64, VEC><<<grid, 256, lds, s>>>(a, g, nkt);
  else k_attend_dkv<T, 128, VEC><<<grid, 256, lds, s>>>(a, g, nkt);
}
template <typename T>
void dq_t(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  if (a.kvec && a.vvec) dq_v<T, true>(s, a, g);
  else dq_v<T, false>(s, a, g);
}
template <typename T>
void dkv_t(hipStream_t s, const AttArgs& a, const AttGrad& g) {
  if (a.qvec && g.dovec) dkv_v<T, true>(s, a, g);
  else dkv_v<T, false>(s, a, g);
}

}  // namespace

void launch_attend_delta(hipStream_t s, int type, const AttArgs& a, const AttGrad& g) {
  if (type == 0) delta_t<float>(s, a, g);
  else if (type == 1) delta_t<_Float16>(s, a, g);
  else delta_t<__bf16>(s, a, g);
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
