// Attention forward: o_i = sum_j p_ij v_j, p_i = softmax_j(scale q_i.k_j + T[h, bucket(j - i - start)]), in one pass over the keys with
// the running reference and sum of the softmax (fp32), scores never leaving the registers.
//
// k_attend: a workgroup of four waves takes 128 queries of one head, 32 per wave.  Transposed scores S^T = K Q^T put a query in
// a lane, so that maximum, sum, bias offset and rescaling are per-lane scalars and the weights are, as they stand, the
// second operand of O^T += V^T P^T (see attend_dev.h).  K and V tiles of 32 keys go through LDS, two buffers each.  In the turn of a tile its
// softmax runs on the vector unit while the matrix unit forms the scores of the tile after and adds up the values of the tile before.
// Bound by products and vector work together: 2 x 16 heads, 4096 x 10000, d = 128, bf16 with a table 707 us, 949 TFLOP/s (693 to 746 over several
// devices; a large matrix product 1200; MFMA with eight vector instructions and an exponential beside each 1370); at d = 64 a score costs the same
// exponential for half the products: 4 x 16 heads, 1000 x 1537, fp16 with a table, a mask and lengths 50 us, 410 TFLOP/s.
// k_attend_few: up to 32 rows (query, head of the group) of one shared head; the waves split the keys instead, read K straight
// into registers and V through LDS of their own, and join at the end.  Bound by reading K and V once: one query per request, 8 x 32 heads on 8,
// keys up to 32773 of 128 features, bf16 155 us with the join, 5.4 TB/s (a large copy moves 4.9, read and written); short calls by their launch (7.5 us).
// Both may split the key axis over workgroups; k_attend_join then weighs the parts.
#include "attend_dev.h"

using namespace att;

namespace {

// Scores of excluded keys at -infinity, whatever they were.  `limit`: 32 floats in LDS of this wave alone, infinity or -infinity per key; the
// minimum with it costs one instruction per score (testing bits costs three) and turns NaN into the limit.
__device__ __forceinline__ void drop_keys(f32x16& s, unsigned keep, float* limit, int lane) {
  if (keep == 0xffffffffu) return;
  if (lane < 32) limit[lane] = ((keep >> lane) & 1) ? __builtin_inff() : -__builtin_inff();
  __builtin_amdgcn_wave_barrier();
  const float* l = limit + 4 * (lane >> 5);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    f32x4 x = *(const f32x4*)(l + 8 * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) asm("v_min_f32 %0, %0, %1" : "+v"(s[4 * g + e]) : "v"(x[e]));   // fminf would first quiet both
  }
  __builtin_amdgcn_wave_barrier();
}

template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) == 4 && DP == 128 ? 1 : 2) void k_attend(AttArgs a, AttOut o, int nqt) {
  typedef typename Frag<T>::type frag;
  constexpr int BK = 32, ND = DP / 32, NS = DP / 16, kTile = BK * DP * (int)sizeof(T);
  __shared__ __align__(16) char tk[2][kTile], tv[2][kTile];
  __shared__ __align__(16) float from[2][32];   // what a key's scores start from: 0, or -infinity where it takes no part
  __shared__ float line[kLine];
  int id = die_order(blockIdx.x, a.B * a.HK, a.G * nqt * o.nsplit);
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
  int qt = id % nqt, sp = (id / nqt) % o.nsplit, bh = id / nqt / o.nsplit;
  if (bh >= a.B * a.H) return;
  int h = bh % a.H, b = bh / a.H, hk = h / a.G;
  int q0 = qt * 128 + wave * 32, i = q0 + (lane & 31);
  int qn = queries_of(a, b);
  int kn = keys_of(a, b);
  if (qt * 128 >= qn) kn = 0;
  int tiles = (kn + BK - 1) / BK, per = (tiles + o.nsplit - 1) / o.nsplit;
  int t0 = min(sp * per, tiles), t1 = min(t0 + per, tiles);

  const T* K = (const T*)a.K + b * a.ks[0] + hk * a.ks[2];
  const T* V = (const T*)a.V + b * a.vs[0] + hk * a.vs[2];
  const uint8_t* mrow = a.mask ? a.mask + b * a.mask_s : nullptr;
  int64_t start = start_of(a, b);
  int far = a.bk.far, rel = rest_below(-(int64_t)q0 - start);   // + 32 t: difference of the tile's first key and the wave's first query

  constexpr int NST = DP == 64 && sizeof(T) == 2 ? 2 : 1;   // sets of loads on their way
  Stage<T, DP, BK, VEC> sk[NST], sv[NST];
  uint8_t mb = 0;
  auto fetch_mask = [&](int t) {
    if (mrow) mb = (lane < BK && t * BK + lane < kn) ? mrow[t * BK + lane] : 0;
  };
  uint64_t k0 = 0, k1 = 0, k2 = 0;             // keys of this tile and the next two that take part
  constexpr uint64_t kAll = 0xffffffffull;
  int whole = mrow ? -1 : kn / BK;             // tiles before this one are kept as a whole
  auto keys = [&](int t) { return t < whole ? kAll : keep_bits(min(max(kn - t * BK, 0), BK), mrow, mb); };
  auto put_keys = [&](int par, uint64_t keep, const Stage<T, DP, BK, VEC>& st) {
    st.store(tk[par], keep, tid);
    if (keep != kAll && tid < BK) from[par][tid] = ((keep >> tid) & 1) ? 0.f : -__builtin_inff();
  };
  auto scores_start = [&](int par) {
    f32x16 c;
    const float* x = from[par] + 4 * half;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 y = *(const f32x4*)(x + 8 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) c[4 * g + e] = y[e];
    }
    return c;
  };
  frag q[NS], p[2];
  f32x16 acc[ND], sc[2];
  sc[0] = sc[1] = f32x16{};
#pragma unroll
  for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) p[u][e] = (T)0.f;
  float m = -__builtin_inff(), l = 0.f;     // reference and sum (this lane's half of the keys)
  float left = 0.f, right = 0.f;
  bool odd = false;                            // there are excluded keys, and some query of the wave holds an infinity or NaN
  const T* kp = K + (int64_t)t0 * BK * a.ks[1];
  const T* vp = V + (int64_t)t0 * BK * a.vs[1];
  int64_t kstep = BK * a.ks[1], vstep = BK * a.vs[1];
  const float* ln = nullptr;
  if (t0 < t1) {
    // all loads are queued before the first is waited for
    Stage<T, DP, BK, VEC> s0, s1;
    s0.load(kp, a.ks[1], kn - t0 * BK, a.d, tid);
    kp += kstep;
    s1.load(kp, a.ks[1], kn - (t0 + 1) * BK, a.d, tid);
    kp += kstep;
    fetch_mask(t0);
    uint8_t m0 = mb;
    fetch_mask(t0 + 1);
    const T* row = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + h * a.qs[2];
#pragma unroll
    for (int k = 0; k < NS; ++k) q[k] = reg_frag<T>(row, i < qn, k, a.d, a.qvec, lane);
    k1 = keys(t0 + 1);
    mb = m0;
    k0 = keys(t0);
    put_keys(0, k0, s0);
    put_keys(1, k1, s1);
    sv[0].store(tv[1], 0, tid);              // the weights of the turn before the first are zero, and so must be what they weigh
    if (NST == 2) {
      sk[0].load(kp, a.ks[1], kn - (t0 + 2) * BK, a.d, tid);
      kp += kstep;
      sv[0].load(vp, a.vs[1], kn - t0 * BK, a.dv, tid);
      vp += vstep;
    }
    if (a.table) {
      fill_line<T>(line, a, h, tid, 256);
      ln = line;
    }
    settle();
    if (whole < t1) {
      // a product with zero tells infinities and NaN apart; in fp32 the row is read again, because at d = 128 a use of the operands ahead of the
      // loop has them laid out otherwise (8 heads, 2000 x 2000: 183 us, so 177)
      float z = 0.f;
      if constexpr (sizeof(T) == 2) {
        f32x16 c = f32x16{};
#pragma unroll
        for (int k = 0; k < NS; ++k) c = Frag<T>::mma(frag{}, q[k], c);
        z = c[0];
      } else {
#pragma unroll 1
        for (int k = 0; k < NS; ++k) {
          frag x = reg_frag<T>(row, i < qn, k, a.d, a.qvec, lane);
#pragma unroll
          for (int e = 0; e < 8; ++e) z = fmaf(x[e], 0.f, z);
        }
      }
      odd = __any(z != 0.f);
    }
    __syncthreads();
    if (ln) {
      left = uniform(line[kPad]);
      right = uniform(line[2 * far + kPad]);
    }
    if (k0 != kAll) sc[0] = scores_start(0);
#pragma unroll
    for (int k = 0; k < NS; ++k) sc[0] = Frag<T>::mma(row_frag<T, DP>(tk[0], 0, k, lane), q[k], sc[0]);
    __syncthreads();
  }
  // A turn per tile.  On entry the scores' products of this tile are there, and p holds the weights of the tile before; LDS holds the keys of the
  // tile after and the values of the tile before.  Tiles up to `end` are of one kind: plain ones lie beyond the last edge on one side (or have no
  // bias); their scores are c2 s + side as they stand.  A wave with odd queries has none: excluded keys, zeros in LDS, make NaN of an infinity or NaN
  // in a query, so there their scores are set to -infinity again, whatever came out.
  int end = ln ? t0 : t1;
  bool plain = !ln && !odd;
  float side = 0.f;
  auto turn = [&](auto par_, int t) {
    constexpr int PAR = decltype(par_)::value;
    f32x16& s = sc[PAR];
    f32x16& next = sc[PAR ^ 1];
    if (t == end) {
      int r = rel + t * BK;
      end = t1;
      side = r < 0 ? left : right;
      plain = (r + 31 <= -far || r - 31 >= far) && fabsf(side) < kFoldable && !odd;
      if (r + 31 <= -far) end = min(end, t + (-far - 31 - r) / BK + 1);
      else if (r - 31 < far) end = min(end, t + (far + 30 - r) / BK + 1);
    }
    fetch_mask(t + 2);
    sk[NST == 2 ? PAR ^ 1 : 0].load(kp, a.ks[1], kn - (t + NST + 1) * BK, a.d, tid);
    sv[NST == 2 ? PAR ^ 1 : 0].load(vp, a.vs[1], kn - (t + NST - 1) * BK, a.dv, tid);
    kp += kstep;
    vp += vstep;
    float mul = a.c2, add = side;
    if (!plain) {
      add_bias<true>(s, a.c2, ln, far, rel + t * BK, left, right, lane, mul, add);
      if (odd && k0 != kAll) {
        unsigned mine = (unsigned)k0 >> (4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = (mine & (1u << (8 * (r >> 2) + (r & 3)))) ? s[r] : -__builtin_inff();
      }
    }
    // Steps kept in this order: each reads the operand of the step after next, queues one product of the tile after (scores) or before (values),
    // and does its share of this tile's softmax meanwhile.
    const char *kt = tk[PAR ^ 1], *vt = tv[PAR ^ 1];
    constexpr int M = NS + 2 * ND, E0 = M / 2 - M / 8;
    auto operand = [&](int z) { return z < NS ? row_frag<T, DP>(kt, 0, z, lane) : col_frag<T, DP>(vt, 16 * ((z - NS) / ND), 32 * ((z - NS) % ND), lane); };
    frag f[3], pn[2];
    f[0] = operand(0);
    f[1] = operand(1);
    float big = -__builtin_inff(), up = 1.f, ref = 0.f, sum = 0.f;
    bool move = false;
#pragma unroll
    for (int z = 0; z < M; ++z) {
      __builtin_amdgcn_sched_barrier(0);
      if (z + 2 < M) f[(z + 2) % 3] = operand(z + 2);
      if (z == 0) {
        if (k1 == kAll) next = Frag<T>::mma(f[0], q[0], f32x16{});
        else next = Frag<T>::mma(f[0], q[0], scores_start(PAR ^ 1));
      } else if (z < NS) next = Frag<T>::mma(f[z % 3], q[z], next);
      else acc[(z - NS) % ND] = Frag<T>::mma(f[z % 3], p[(z - NS) / ND], acc[(z - NS) % ND]);
      if (z < E0) {
#pragma unroll
        for (int r = z * 16 / E0; r < (z + 1) * 16 / E0; ++r) big = fmaxf(big, s[r]);
        if (z == E0 - 1) {
          float top = both_max(fmaf(big, mul, add));
          move = top > m + kSlack;
          up = move ? __builtin_amdgcn_exp2f(m - top) : 1.f;
          m = move ? top : m;
          ref = add - ((m == -__builtin_inff() ? 0.f : m) - Lift<T>::value);
        }
      } else {
#pragma unroll
        for (int r = (z - E0) * 16 / (M - E0); r < (z + 1 - E0) * 16 / (M - E0); ++r) {
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, ref));
          sum += s[r];
          if (r == 7) pn[0] = pack8<T>(s, 0);
          if (r == 15) pn[1] = pack8<T>(s, 1);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    p[0] = pn[0];
    p[1] = pn[1];
    asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(sum));   // the weights are wanted now, not at their use a turn later
    l = fmaf(l, up, sum);
    if (__any(move)) {
#pragma unroll
      for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] *= up;
    }
    k2 = keys(t + 2);
    put_keys(PAR, k2, sk[NST == 2 ? PAR : 0]);
    sv[NST == 2 ? PAR : 0].store(tv[PAR], k0, tid);
    k0 = k1;
    k1 = k2;
    __syncthreads();
  };
  for (int t = t0; t < t1; t += 2) {
    turn(Const<0>{}, t);
    if (t + 1 < t1) turn(Const<1>{}, t + 1);
  }
  if (t0 < t1) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < ND; ++c) acc[c] = Frag<T>::mma(col_frag<T, DP>(tv[(t1 - t0 + 1) & 1], 16 * u, 32 * c, lane), p[u], acc[c]);
  }
  l = both_sum(l);
  bool some = l != 0.f && i < qn;           // NaN counts as something
  float inv = some ? 1.f / l : 0.f;
  float lse2 = some ? (m - Lift<T>::value) + __builtin_amdgcn_logf(l) : -__builtin_inff();
  if (i >= a.nq) return;
  if (!some) {                               // zero also beside infinite values, which make NaN of weights of zero
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
  }
  size_t row = ((size_t)b * a.H + h) * a.nq + i;
  if (o.nsplit == 1) {
    if (half == 0) o.lse[row] = lse2 * kLn2;
    T* out = (T*)o.O + b * o.os[0] + (int64_t)i * o.os[1] + h * o.os[2];
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        store4<T>(out, 32 * n + 8 * r + 4 * half, a.dv, o.ovec, acc[n][4 * r] * inv, acc[n][4 * r + 1] * inv, acc[n][4 * r + 2] * inv,
                  acc[n][4 * r + 3] * inv);
  } else {
    row += (size_t)sp * a.B * a.H * a.nq;
    if (half == 0) o.pl[row] = lse2;
    float* out = o.pO + row * o.dv4;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        int c = 32 * n + 8 * r + 4 * half;
        if (c < o.dv4) *(f32x4*)(out + c) = f32x4{acc[n][4 * r] * inv, acc[n][4 * r + 1] * inv, acc[n][4 * r + 2] * inv, acc[n][4 * r + 3] * inv};
      }
  }
}

// Rows rho = 32 rb .. of shared head hk: query rho / G, head hk G + rho % G.
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_attend_few(AttArgs a, AttOut o, int nrb) {
  typedef typename Frag<T>::type frag;
  constexpr int ND = DP / 32, NS = DP / 16, E = 16 / (int)sizeof(T), CH = DP / E, NV = 32 * CH / 64;
  constexpr bool kLds = sizeof(T) == 2;      // V through LDS (four-byte elements are read as the product wants them)
  constexpr int kVt = 32 * DP * 2, kPart = 32 * (DP + 4);
  __shared__ __align__(16) char buf[kLds && 4 * kVt > 8 * kPart ? 4 * kVt : 8 * kPart];
  __shared__ float wm[4][32], wl[4][32];
  __shared__ __align__(16) float limit[4][32];
  extern __shared__ float dyn[];               // with a table: 32 rows of its entries, then the bucket of every difference (bytes)
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5, col = lane & 31;
  int x = blockIdx.x, rb = x % nrb, sp = (x / nrb) % o.nsplit, bh = x / nrb / o.nsplit, hk = bh % a.HK, b = bh / a.HK;
  int rows = a.nq * a.G, rho = rb * 32 + col, i = rho / a.G, h = hk * a.G + rho % a.G;
  int qn = queries_of(a, b);
  int kn = keys_of(a, b);
  bool mine = rho < rows && i < qn;
  int blocks = (kn + 31) / 32, per = (blocks + o.nsplit - 1) / o.nsplit;
  int t0 = min(sp * per, blocks), t1 = min(t0 + per, blocks);
  int i0 = rb * 32 / a.G;                     // first query of the rows

  const T* K = (const T*)a.K + b * a.ks[0] + hk * a.ks[2];
  const T* V = (const T*)a.V + b * a.vs[0] + hk * a.vs[2];
  const uint8_t* mrow = a.mask ? a.mask + b * a.mask_s : nullptr;
  int64_t start = start_of(a, b);
  frag q[NS], kf[NS];
  char* vt = buf + wave * kVt;
  u32x4 vr[kLds ? NV : 1];
  frag vf[kLds ? 1 : 2][kLds ? 1 : ND];      // fp32: V as the product wants it, straight from memory
  uint8_t mb = 0, mnext = 0;
  // rows of a 32-key block from memory, with bounds
  auto block = [&](const T* base, int64_t stride, int t, int width) {
    unsigned rows = (unsigned)min(kn - t * 32, 32);
    return bounded(base + (int64_t)t * 32 * stride, (rows - 1) * (unsigned)stride * (unsigned)sizeof(T) + (unsigned)width * (unsigned)sizeof(T));
  };
  auto fetch_k = [&](int t) {
    if constexpr (VEC) {
      __amdgpu_buffer_rsrc_t mem = block(K, a.ks[1], t, a.d);
      unsigned at = (unsigned)col * (unsigned)a.ks[1] * (unsigned)sizeof(T);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        int c = 16 * s + 8 * half;
        if constexpr (sizeof(T) == 2) {
          kf[s] = __builtin_bit_cast(frag, __builtin_amdgcn_raw_buffer_load_b128(mem, c < a.d ? at + 2 * c : kNowhere, 0, 0));
        } else {
          f32x4 lo = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(mem, c < a.d ? at + 4 * c : kNowhere, 0, 0));
          f32x4 hi = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(mem, c + 4 < a.d ? at + 4 * c + 16 : kNowhere, 0, 0));
          kf[s] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
      }
    } else {
      const T* row = K + (int64_t)(t * 32 + col) * a.ks[1];
#pragma unroll
      for (int s = 0; s < NS; ++s) kf[s] = reg_frag<T>(row, t * 32 + col < kn, s, a.d, 0, lane);
    }
    if (mrow) mnext = (lane < 32 && t * 32 + col < kn) ? mrow[t * 32 + col] : 0;
  };
  auto fetch_v = [&](int t) {
    if constexpr (kLds) {
      int r = lane / CH, c = (lane % CH) * E;
      if constexpr (VEC) {
        __amdgpu_buffer_rsrc_t mem = block(V, a.vs[1], t, a.dv);
        unsigned pitch = (unsigned)a.vs[1] * 2, at = c < a.dv ? (unsigned)r * pitch + 2 * c : kNowhere;
#pragma unroll
        for (int n = 0; n < NV; ++n) vr[n] = __builtin_amdgcn_raw_buffer_load_b128(mem, at + (unsigned)(n * (64 / CH)) * pitch, 0, 0);
      } else {
        const T* p = V + (int64_t)(t * 32 + r) * a.vs[1];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          vr[n] = u32x4{0u, 0u, 0u, 0u};
          if (t * 32 + r + n * (64 / CH) < kn) vr[n] = load16<T>(p, c, a.dv, 0);
          p += (int64_t)(64 / CH) * a.vs[1];
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            int r = 16 * u + 8 * (e >> 2) + 4 * half + (e & 3), c = 32 * n + col;
            if constexpr (VEC) {
              __amdgpu_buffer_rsrc_t mem = block(V, a.vs[1], t, a.dv);
              unsigned at = c < a.dv ? (unsigned)r * (unsigned)a.vs[1] * 4 + 4 * c : kNowhere;
              vf[u][n][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(mem, at, 0, 0));
            } else {
              vf[u][n][e] = t * 32 + r < kn && c < a.dv ? V[(int64_t)(t * 32 + r) * a.vs[1] + c] : (T)0.f;
            }
          }
    }
  };
  f32x16 acc[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;
  int t = t0 + wave;
  if (t < t1) {
    fetch_k(t);
    fetch_v(t);
  }
  {
    const T* row = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + h * a.qs[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = reg_frag<T>(row, mine, s, a.d, a.qvec, lane);
  }
  float left = 0.f, right = 0.f;
  int pitch = a.bk.buckets | 1;
  const float* tab = dyn + col * pitch;
  uint8_t* bline = (uint8_t*)(dyn + 32 * pitch);
  if (a.table) {
    // entries of the rows' heads, and the bucket of every difference (bytes)
    int r = rb * 32 + (tid >> 3);
    const T* src = (const T*)a.table + (size_t)(hk * a.G + r % a.G) * a.bk.buckets;
    for (int n = tid & 7; n < a.bk.buckets; n += 8) dyn[(tid >> 3) * pitch + n] = r < rows ? bias2<T>(src[n]) : 0.f;
    for (int n = tid; n < 2 * (a.bk.far + kPad) + 1; n += 256) bline[n] = (uint8_t)bucket_of(a.bk, n - a.bk.far - kPad);
    __syncthreads();
    left = tab[bline[0]];
    right = tab[bline[2 * (a.bk.far + kPad)]];
  }
  int rel = rest_below(-(int64_t)i0 - start);
  settle();
  for (; t < t1; t += 4) {
    mb = mnext;
    unsigned keep = (unsigned)keep_bits(min(kn - t * 32, 32), mrow, mb);
    if constexpr (kLds) {
      int r = lane / CH, c = lane % CH;
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        int row = r + n * (64 / CH);
        u32x4 v = vr[n];
        if (!((keep >> row) & 1)) v = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(vt + row * DP * 2 + ((c ^ swz<T, DP>(row)) << 4)) = v;
      }
    }
    f32x16 s = f32x16{};
#pragma unroll
    for (int k = 0; k < NS; ++k) s = Frag<T>::mma(kf[k], q[k], s);
    if (t + 4 < t1) {
      fetch_k(t + 4);
      if constexpr (kLds) fetch_v(t + 4);
    }
    int rel0 = rel + t * 32;                   // of the first key and the first query
    if (!a.table || rel0 + 31 <= -a.bk.far || rel0 - 31 >= a.bk.far) {
      float cb = rel0 < 0 ? left : right;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c2, cb);
    } else {
      const uint8_t* bl = bline + (rel0 - (min(i, a.nq - 1) - i0) + 4 * half + a.bk.far + kPad);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.c2, tab[bl[8 * (r >> 2) + (r & 3)]]);
    }
    drop_keys(s, keep, limit[wave], lane);
    float top = -__builtin_inff();
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
    top = both_max(top);
    bool move = top > m + kSlack;
    if (__any(move)) {
      float up = move ? __builtin_amdgcn_exp2f(m - top) : 1.f;
      m = move ? top : m;
      l *= up;
#pragma unroll
      for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] *= up;
    }
    float ref = (m == -__builtin_inff() ? 0.f : m) - Lift<T>::value;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(s[r] - ref);
      l += s[r];
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      frag p = pack8<T>(s, u);
#pragma unroll
      for (int c = 0; c < ND; ++c) {
        frag v;
        if constexpr (kLds) {
          v = col_frag<T, DP>(vt, 16 * u, 32 * c, lane);
        } else {
          v = vf[u][c];
          if (keep != 0xffffffffu) {
            unsigned k = keep >> (16 * u + 4 * half);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = ((k >> (8 * (e >> 2) + (e & 3))) & 1) ? v[e] : (T)0.f;
          }
        }
        acc[c] = Frag<T>::mma(v, p, acc[c]);
      }
    }
    if constexpr (kLds) __builtin_amdgcn_wave_barrier();
    else if (t + 4 < t1) fetch_v(t + 4);
  }
  // join the four waves: each scales its sums to the largest reference; two leave theirs in LDS, the other two add them, all write
  l = both_sum(l);
  if (half == 0) {
    wm[wave][col] = m;
    wl[wave][col] = l;
  }
  __syncthreads();
  float top = fmaxf(fmaxf(wm[0][col], wm[1][col]), fmaxf(wm[2][col], wm[3][col]));
  float w = m == -__builtin_inff() && l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top);
  float* part = (float*)buf + (wave & 1) * kPart + col * (DP + 4) + 4 * half;
  if (wave >= 2) {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(f32x4*)(part + 32 * n + 8 * r) = f32x4{acc[n][4 * r] * w, acc[n][4 * r + 1] * w, acc[n][4 * r + 2] * w, acc[n][4 * r + 3] * w};
  }
  __syncthreads();
  if (wave < 2) {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(f32x4*)(part + 32 * n + 8 * r) += f32x4{acc[n][4 * r] * w, acc[n][4 * r + 1] * w, acc[n][4 * r + 2] * w, acc[n][4 * r + 3] * w};
  }
  __syncthreads();
  // eight threads per row
  int row = tid >> 3, rr = rb * 32 + row, qi = rr / a.G, hh = hk * a.G + rr % a.G;
  if (rr >= rows) return;
  top = fmaxf(fmaxf(wm[0][row], wm[1][row]), fmaxf(wm[2][row], wm[3][row]));
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) sum += wm[k][row] == -__builtin_inff() && wl[k][row] == 0.f ? 0.f : __builtin_amdgcn_exp2f(wm[k][row] - top) * wl[k][row];
  bool some = sum != 0.f && qi < qn;
  float inv = some ? 1.f / sum : 0.f;
  float lse2 = some ? (top - Lift<T>::value) + __builtin_amdgcn_logf(sum) : -__builtin_inff();
  size_t at = ((size_t)b * a.H + hh) * a.nq + qi;
  if (o.nsplit > 1) at += (size_t)sp * a.B * a.H * a.nq;
  if ((tid & 7) == 0) {
    if (o.nsplit == 1) o.lse[at] = lse2 * kLn2;
    else o.pl[at] = lse2;
  }
  const float* src = (const float*)buf + row * (DP + 4);
  T* out = (T*)o.O + b * o.os[0] + (int64_t)qi * o.os[1] + hh * o.os[2];
  for (int c = (tid & 7) * 4; c < DP; c += 32) {
    f32x4 y = (*(const f32x4*)(src + c) + *(const f32x4*)(src + kPart + c)) * inv;
    if (!some) y = f32x4{0.f, 0.f, 0.f, 0.f};
    if (o.nsplit == 1) store4<T>(out, c, a.dv, o.ovec, y[0], y[1], y[2], y[3]);
    else if (c < o.dv4) *(f32x4*)(o.pO + at * o.dv4 + c) = y;
  }
}

// Up to kJoinFew parts: 32 lanes per row, four features per lane (8000 rows of 64 features, fp32, 4 parts: 4.9 us; a workgroup per row takes 10.6 for 3).
constexpr int kJoinFew = 8;
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join_few(AttArgs a, AttOut o) {
  int64_t n = (int64_t)a.B * a.H * a.nq, row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  int c = 4 * (threadIdx.x & 31);
  if (row >= n) return;
  float p[kJoinFew], top = -__builtin_inff(), sum = 0.f;
  f32x4 v[kJoinFew], y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kJoinFew; ++s) {
    p[s] = s < o.nsplit ? o.pl[s * n + row] : -__builtin_inff();
    v[s] = s < o.nsplit && c < o.dv4 ? *(const f32x4*)(o.pO + (s * n + row) * o.dv4 + c) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int s = 0; s < kJoinFew; ++s) top = fmaxf(top, p[s]);
#pragma unroll
  for (int s = 0; s < kJoinFew; ++s) {
    float w = p[s] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(p[s] - top);
    sum += w;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fmaf(w, v[s][e], y[e]);
  }
  bool some = sum != 0.f;
  float inv = some ? 1.f / sum : 0.f;
  if (c == 0) o.lse[row] = some ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
  int i = (int)(row % a.nq), h = (int)(row / a.nq % a.H), b = (int)(row / a.nq / a.H);
  T* out = (T*)o.O + b * o.os[0] + (int64_t)i * o.os[1] + h * o.os[2];
  store4<T>(out, c, a.dv, o.ovec, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
}

// More parts, a workgroup per row.  Eight groups of 32 lanes take every eighth part, four features per lane.
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join(AttArgs a, AttOut o) {
  __shared__ float wsum[4], wtop[4];
  __shared__ __align__(16) f32x4 part[8][32];
  int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = tid >> 5, c = 4 * (tid & 31);
  size_t n = (size_t)a.B * a.H * a.nq, row = blockIdx.x;
  float top = -__builtin_inff();
  for (int s = tid; s < o.nsplit; s += 256) top = fmaxf(top, o.pl[s * n + row]);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x, 64));
  if (lane == 0) wtop[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(wtop[0], wtop[1]), fmaxf(wtop[2], wtop[3]));
  float sum = 0.f;
  f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = g; s < o.nsplit; s += 8) {
    float p = o.pl[s * n + row];
    float w = p == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(p - top);
    sum += w;
    if (c < o.dv4) {
      f32x4 v = *(const f32x4*)(o.pO + (s * n + row) * o.dv4 + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(w, v[e], y[e]);
    }
  }
  part[g][tid & 31] = y;
  sum += __shfl_xor(sum, 32, 64);
  if (lane == 0) wsum[wave] = sum;
  __syncthreads();
  if (tid >= 32) return;
  sum = (wsum[0] + wsum[1]) + (wsum[2] + wsum[3]);
#pragma unroll
  for (int k = 1; k < 8; ++k) y += part[k][tid];
  bool some = sum != 0.f;
  float inv = some ? 1.f / sum : 0.f;
  if (tid == 0) o.lse[row] = some ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
  int i = (int)(row % a.nq), h = (int)(row / a.nq % a.H), b = (int)(row / a.nq / a.H);
  T* out = (T*)o.O + b * o.os[0] + (int64_t)i * o.os[1] + h * o.os[2];
  store4<T>(out, c, a.dv, o.ovec, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
}

template <typename T, bool VEC>
void attend_v(hipStream_t s, const AttArgs& a, const AttOut& o) {
  int nqt = (a.nq + 127) / 128, total = a.B * a.H * nqt * o.nsplit, grid = (total + 7) / 8 * 8;
  if (a.d <= 64 && a.dv <= 64) k_attend<T, 64, VEC><<<grid, 256, 0, s>>>(a, o, nqt);
  else k_attend<T, 128, VEC><<<grid, 256, 0, s>>>(a, o, nqt);
}
template <typename T, bool VEC>
void attend_few_v(hipStream_t s, const AttArgs& a, const AttOut& o) {
  int nrb = (int)(((int64_t)a.nq * a.G + 31) / 32), total = a.B * a.HK * nrb * o.nsplit;
  size_t lds = a.table ? 32 * sizeof(float) * (a.bk.buckets | 1) + 2 * (a.bk.far + kPad) + 1 : 0;
  if (a.d <= 64 && a.dv <= 64) k_attend_few<T, 64, VEC><<<total, 256, lds, s>>>(a, o, nrb);
  else k_attend_few<T, 128, VEC><<<total, 256, lds, s>>>(a, o, nrb);
}
template <typename T>
void attend_t(hipStream_t s, const AttArgs& a, const AttOut& o) {
  if (a.kvec && a.vvec) attend_v<T, true>(s, a, o);
  else attend_v<T, false>(s, a, o);
}
template <typename T>
void attend_few_t(hipStream_t s, const AttArgs& a, const AttOut& o) {
  if (a.kvec && a.vvec) attend_few_v<T, true>(s, a, o);
  else attend_few_v<T, false>(s, a, o);
}

template <typename T>
void join_t(hipStream_t s, const AttArgs& a, const AttOut& o) {
  int64_t n = (int64_t)a.B * a.H * a.nq;
  if (o.nsplit <= kJoinFew) k_attend_join_few<T><<<(unsigned)((n + 7) / 8), 256, 0, s>>>(a, o);
  else k_attend_join<T><<<(unsigned)n, 256, 0, s>>>(a, o);
}

}  // namespace

void launch_attend(hipStream_t s, int type, const AttArgs& a, const AttOut& o) {
  if (type == 0) attend_t<float>(s, a, o);
  else if (type == 1) attend_t<_Float16>(s, a, o);
  else attend_t<__bf16>(s, a, o);
}

void launch_attend_few(hipStream_t s, int type, const AttArgs& a, const AttOut& o) {
  if (type == 0) attend_few_t<float>(s, a, o);
  else if (type == 1) attend_few_t<_Float16>(s, a, o);
  else attend_few_t<__bf16>(s, a, o);
}

void launch_attend_join(hipStream_t s, int type, const AttArgs& a, const AttOut& o) {
  if (type == 0) join_t<float>(s, a, o);
  else if (type == 1) join_t<_Float16>(s, a, o);
  else join_t<__bf16>(s, a, o);
}
