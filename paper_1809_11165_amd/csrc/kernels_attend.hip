// Attention forward: o_i = sum_j p_ij v_j, p_i = softmax_j(scale q_i.k_j + T[h, bucket(j - i - start)]), in one pass over the keys with
// the running reference and sum of the softmax (fp32), scores never leaving the registers.
//
// k_attend: a workgroup of four waves takes 128 queries of one head, 32 per wave.  Transposed scores S^T = K Q^T put a query in
// a lane, so that maximum, sum, bias offset and rescaling are per-lane scalars and the weights are, as they stand, the
// second operand of O^T += V^T P^T (see attend_dev.h).  K and V tiles go through LDS, two buffers, the next tile's loads in flight
// during a tile's products.
// k_attend_few: up to 32 rows (query, head of the group) of one shared head; the waves split the keys instead, read K straight
// into registers and V through LDS of their own, and join at the end.  Bound by reading K and V once.
// Both may split the key axis over workgroups; k_attend_join then weighs the parts.
#include "attend_dev.h"

using namespace att;

namespace {

__device__ __forceinline__ void drop_keys(f32x16& s, unsigned keep, int lane) {
  if (keep == 0xffffffffu) return;
  unsigned k = keep >> (4 * (lane >> 5));
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = ((k >> (8 * (r >> 2) + (r & 3))) & 1) ? s[r] : -__builtin_inff();
}

template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(256, 2) void k_attend(AttArgs a, AttOut o, int nqt, int total, int per_die) {
  typedef typename Frag<T>::type frag;
  constexpr int BK = sizeof(T) == 2 ? 64 : 32, NB = BK / 32, ND = DP / 32, NS = DP / 16, kTile = BK * DP * (int)sizeof(T);
  __shared__ __align__(16) char tile[2][2][kTile];
  __shared__ float line[kLine];
  int id = die_order(blockIdx.x, per_die);
  if (id >= total) return;
  int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
  int qt = id % nqt, sp = (id / nqt) % o.nsplit, bh = id / nqt / o.nsplit;
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
  frag q[NS];
  {
    const T* row = (const T*)a.Q + b * a.qs[0] + (int64_t)i * a.qs[1] + h * a.qs[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = reg_frag<T>(row, i < qn, s, a.d, a.qvec, lane);
  }
  const float* ln = nullptr;
  if (a.table && t0 < t1) {
    fill_line<T>(line, a, h, tid, 256);
    ln = line;
  }
  int64_t start = start_of(a, b);

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
    sk.store(tile[t & 1][0], ~0ull, tid);             // scores of masked keys are replaced
    sv.store(tile[t & 1][1], keep, tid);
  };
  f32x16 acc[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) acc[n] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;     // reference and sum (this lane's half of the keys)
  if (t0 < t1) {
    fetch(t0);
    put(t0);
  }
  settle();
  __syncthreads();
  float left = 0.f, right = 0.f;
  if (ln) {
    left = line[kPad];
    right = line[2 * a.bk.far + kPad];
  }
  int rel = rest_below(-(int64_t)q0 - start);
  for (int t = t0; t < t1; ++t) {
    const char *tk = tile[t & 1][0], *tv = tile[t & 1][1];
    uint64_t kp = keep;
    if (t + 1 < t1) fetch(t + 1);
    if (kp) {
      f32x16 s[NB];
      float mul[NB], add[NB];
      float top = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        s[n] = f32x16{};
#pragma unroll
        for (int k = 0; k < NS; ++k) s[n] = Frag<T>::mma(row_frag<T, DP>(tk, 32 * n, k, lane), q[k], s[n]);
        add_bias<true>(s[n], a.c2, ln, a.bk.far, rel + t * BK + 32 * n, left, right, lane, mul[n], add[n]);
        drop_keys(s[n], (unsigned)(kp >> (32 * n)), lane);
        float big = -__builtin_inff();
#pragma unroll
        for (int r = 0; r < 16; ++r) big = fmaxf(big, s[n][r]);
        top = fmaxf(top, fmaf(big, mul[n], add[n]));
      }
      top = fmaxf(top, other_half(top));
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
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], mul[n], add[n] - ref));
          l += s[n][r];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          frag p = pack8<T>(s[n], u);
#pragma unroll
          for (int c = 0; c < ND; ++c) acc[c] = Frag<T>::mma(col_frag<T, DP>(tv, 32 * n + 16 * u, 32 * c, lane), p, acc[c]);
        }
      }
    }
    if (t + 1 < t1) put(t + 1);
    __syncthreads();
  }
  l += other_half(l);
  bool some = l != 0.f && i < qn;           // NaN counts as something
  float inv = some ? 1.f / l : 0.f;
  float lse2 = some ? (m - Lift<T>::value) + __builtin_amdgcn_logf(l) : -__builtin_inff();
  if (i >= a.nq) return;
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
      fetch_v(t + 4);
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
    drop_keys(s, keep, lane);
    float top = -__builtin_inff();
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
    top = fmaxf(top, other_half(top));
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
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            int r = 16 * u + 8 * (e >> 2) + 4 * half + (e & 3), cc = 32 * c + col;
            v[e] = ((keep >> r) & 1) && cc < a.dv ? V[(int64_t)(t * 32 + r) * a.vs[1] + cc] : (T)0.f;
          }
        }
        acc[c] = Frag<T>::mma(v, p, acc[c]);
      }
    }
    if constexpr (kLds) __builtin_amdgcn_wave_barrier();
  }
  // join the four waves: each scales its sums to the largest reference; two leave theirs in LDS, the other two add them, all write
  l += other_half(l);
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

// A workgroup per row: parts weighed by their sums.  Eight groups of 32 lanes take every eighth part, four features per lane.
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
  int nqt = (a.nq + 127) / 128, total = a.B * a.H * nqt * o.nsplit, per = (total + 7) / 8;
  if (a.d <= 64 && a.dv <= 64) k_attend<T, 64, VEC><<<8 * per, 256, 0, s>>>(a, o, nqt, total, per);
  else k_attend<T, 128, VEC><<<8 * per, 256, 0, s>>>(a, o, nqt, total, per);
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
  size_t n = (size_t)a.B * a.H * a.nq;
  int g = (int)n;
  if (type == 0) k_attend_join<float><<<g, 256, 0, s>>>(a, o);
  else if (type == 1) k_attend_join<_Float16><<<g, 256, 0, s>>>(a, o);
  else k_attend_join<__bf16><<<g, 256, 0, s>>>(a, o);
}
