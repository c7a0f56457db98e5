// Norm and rotation of queries and keys, and its gradient (see include/bbmm.h, "Rotation").
//
//   z = w n,  n = r x,  r = (mean x^2 + eps)^-1/2;   y = R z, R a turn of every pair by its angle
//   dz = R^T dy;  dw = sum dz n;  dx = r (w dz - n mean(w dz n))
// A few lanes take a row: each holds two pieces of it whose pairs are complete, so a turn stays in the lane and the row's sums cross
// the few lanes only.  Cosines and sines are formed once per (token, pair) of a workgroup and serve all heads.  Workgroups work on one of Q and K.
// Bound by memory: rows are read and written once (gradient: two read, one written, and the weights' sums joined).
#include "cache_dev.h"

using namespace att;

namespace {

// cos and sin of pos freq.  The angle is formed and taken modulo a turn in 64 bits: fp32 holds positions of 10^5 to 10^-2.
__device__ __forceinline__ float2 turn_of(int64_t pos, double freq) {
  constexpr double kTurns = 0.15915494309189533577;       // 1 / (2 pi)
  double t = (double)pos * freq * kTurns;
  t -= rint(t);
  float s, c;
  sincospif((float)(t + t), &s, &c);
  return make_float2(c, s);
}

// Sum (or maximum) over the LPR lanes of a row, LPR a power of two up to 16: neighbours, pairs of them, and mirrors, which meet the other half's
// result in any lane.
template <int C> __device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), C, 0xf, 0xf, true)); }
template <int LPR, typename F>
__device__ __forceinline__ float across(float x, F f) {
  if constexpr (LPR >= 2) x = f(x, dpp<0xb1>(x));          // quad_perm 1 0 3 2
  if constexpr (LPR >= 4) x = f(x, dpp<0x4e>(x));          // quad_perm 2 3 0 1
  if constexpr (LPR >= 8) x = f(x, dpp<0x141>(x));         // mirror of eight
  if constexpr (LPR >= 16) x = f(x, dpp<0x140>(x));        // mirror of sixteen
  return x;
}
template <int LPR> __device__ __forceinline__ float row_sum(float x) { return across<LPR>(x, [](float a, float b) { return a + b; }); }
template <int LPR> __device__ __forceinline__ float row_max(float x) { return across<LPR>(x, [](float a, float b) { return fmaxf(a, b); }); }

// How a row is dealt out: E elements a piece (16 bytes, or 1), slot j = lane + LPR k holds two pieces.
//   halves: j < rot / 2E holds pieces j and j + rot / 2E (turned); behind, 2j and 2j + 1;  neighbours: 2j and 2j + 1 (turned below rot).
template <typename T, int E, int LPR, int KS, bool NB>
struct Row {
  static constexpr int N = 2 * E;
  typedef T piece __attribute__((ext_vector_type(E)));
  struct Raw { piece v[2 * KS]; };
  int p0[KS], p1[KS];                                       // first elements of the two pieces
  int pair0[KS];                                            // the slot's first pair
  int d, half;
  __device__ __forceinline__ Row(const RotArgs& a, int lane) {
    d = a.d, half = a.rot >> 1;
    int h = half / E;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      int j = lane + LPR * k;
      bool split = !NB && j < h;
      p0[k] = split ? j * E : 2 * j * E;
      p1[k] = split ? (j + h) * E : (2 * j + 1) * E;
      pair0[k] = j * E;
    }
  }
  // Pieces behind the row stay as they are: zeros (see clear).
  __device__ __forceinline__ void load(Raw& r, const T* row) const {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      if (p0[k] < d) r.v[2 * k] = *(const piece*)(row + p0[k]);
      if (p1[k] < d) r.v[2 * k + 1] = *(const piece*)(row + p1[k]);
    }
  }
  __device__ __forceinline__ static void clear(Raw& r) {
#pragma unroll
    for (int k = 0; k < 2 * KS; ++k) r.v[k] = (piece)(T)0.f;
  }
  // element i < 2E of slot k
  __device__ __forceinline__ static float at(const Raw& r, int k, int i) { return (float)r.v[2 * k + i / E][i % E]; }
  __device__ __forceinline__ void weights(float* w, const T* p) const {      // ones without weights, zeros behind the row
    typedef piece some __attribute__((aligned(sizeof(T))));
#pragma unroll
    for (int k = 0; k < 2 * KS; ++k) {
      int c = k & 1 ? p1[k / 2] : p0[k / 2];
      piece v = (piece)(T)(p ? 0.f : 1.f);
      if (p && c < d) v = *(const some*)(p + c);
#pragma unroll
      for (int i = 0; i < E; ++i) w[k * E + i] = (float)v[i];
    }
  }
  __device__ __forceinline__ void store(T* row, const float* y) const {
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        int c = x ? p1[k] : p0[k];
        piece v;
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = (T)y[k * N + x * E + i];
        if (c < d) *(piece*)(row + c) = v;
      }
  }
  // Cosines and sines of the slots' pairs, from those of their token.
  __device__ __forceinline__ void angles(float2* t, const float2* trig) const {
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < E; ++i) t[k * E + i] = trig[pair0[k] + i];
  }
  // The slots' pairs turned (BACK: the other way round).  Halves are a slot's pairs or none of them.
  template <bool BACK>
  __device__ __forceinline__ void turn(float* y, const float2* t) const {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      int there = half - pair0[k];                          // pairs of the slot, if positive
      constexpr bool kInside = NB && E > 1;                 // pairs within a piece, any number of them; else a slot's pairs or none
      if (!kInside && there <= 0) continue;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        float &u = y[k * N + (kInside ? 2 * i : i)], &w = y[k * N + (kInside ? 2 * i + 1 : E + i)];
        float c = t[k * E + i].x, s = BACK ? -t[k * E + i].y : t[k * E + i].y;
        float p = u * c - w * s, q = w * c + u * s;
        u = !kInside || i < there ? p : u;
        w = !kInside || i < there ? q : w;
      }
    }
  }
};

// n = r x of a row in place, and r.  Squares that leave fp32 (or lose bits near its smallest numbers) are formed of scaled values instead.
template <int LPR, int M>
__device__ __forceinline__ float norm_row(float* x, float inv_d, float eps32, double eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < M; ++i) s = fmaf(x[i], x[i], s);
  s = row_sum<LPR>(s);
  float mean = fmaf(s, inv_d, eps32), r = __builtin_amdgcn_rsqf(mean), scale = 1.f;
  bool lost = !(s < 1e37f) || mean < 1e-27f;
  if (__any(lost)) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i) top = fmaxf(top, fabsf(x[i]));
    top = row_max<LPR>(top);
    int e = top > 0.f && top < __builtin_inff() ? ilogbf(top) : 0;
    if (eps > 0.0) e = max(e, ilogb(eps) / 2);               // beside eps smaller squares are nothing
    e = min(max(e, -126), 126);
    float down = ldexpf(1.f, -e), q = 0.f;
    if (!lost) down = 1.f;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      x[i] *= down;
      q = fmaf(x[i], x[i], q);
    }
    q = row_sum<LPR>(q);
    if (lost) {
      scale = down;
      r = 1.f / sqrtf(fmaf(q, inv_d, (float)(eps * down * down)));
    }
  }
#pragma unroll
  for (int i = 0; i < M; ++i) x[i] *= r;
  return scale * r;
}

// Row r of a workgroup's tokens: head r % heads of token r / heads.  Its place in one or two inputs, and whether it is there.
template <typename T>
struct Place {
  const T* row[2];
  int token;
  bool live;
  __device__ __forceinline__ Place(const RotArgs& a, int which, uint32_t tok0, int r, int n, const T* x0, const int64_t* s0, const T* x1, const int64_t* s1) {
    r = min(r, n - 1);
    token = (int)over(r, a.by_heads[which]);
    int head = r - token * a.heads[which];
    uint32_t tok = tok0 + token, b = over(tok, a.by_rows);
    int i = (int)(tok - b * (uint32_t)a.rows);
    live = !a.len || i < a.len[b];
    row[0] = x0 + (int64_t)b * s0[0] + (int64_t)i * s0[1] + (int64_t)head * s0[2];
    row[1] = x1 ? x1 + (int64_t)b * s1[0] + (int64_t)i * s1[1] + (int64_t)head * s1[2] : nullptr;
  }
};

__device__ __forceinline__ void fill_trig(const RotArgs& a, float2* trig, int64_t tok0, int n, int tid) {
  int half = a.rot >> 1;
  for (int i = tid; i < n * half; i += 256) {
    int t = i / half, p = i - t * half;
    trig[t * (BBMM_ATT_MAXD / 2) + p] = turn_of(a.pos[(int64_t)a.axis[p] * a.tokens + tok0 + t], a.freq[p]);
  }
}

// Rows of the workgroup's tokens, a group of LPR lanes a row at a time; the next one is on its way meanwhile (a prompt of 8192 x 40 heads of 128, bf16, one
// row in hand / so: 42.0 / 41.0 us a call).  That prompt, 168 MB: 35.3 us, 4.75 TB/s, the rate of a copy.  2 x 2309 x 32 heads of 80 in fp16, three axes,
// neighbouring pairs: 14.9 us from HBM (13.4 of data read just before), 3.2 TB/s, of which the launch and a workgroup's chain (positions, angles, rows) are 4.  One token:
// 4 us, that chain.  Halves of the turned features that are no whole 16 bytes take single elements: 8192 x 40 heads of 40, bf16, 29.7 us, floor 10.7.
template <typename T, int E, int LPR, int KS, bool NB>
__global__ __launch_bounds__(256) void k_rotate(RotArgs a) {
  typedef Row<T, E, LPR, KS, NB> Rows;
  constexpr int GP = 256 / LPR, M = Rows::N * KS;
  __shared__ float2 trig[BBMM_ROT_TOKENS * (BBMM_ATT_MAXD / 2)];
  int tid = threadIdx.x, which = blockIdx.x >= (unsigned)a.blocks[0];
  int blk = blockIdx.x - (which ? a.blocks[0] : 0), per = a.tokens_per[which], heads = a.heads[which];
  Rows rows(a, tid % LPR);
  const T* x = (const T*)a.x[which];
  T* y = (T*)a.y[which];
  float w[M];
  if (a.norm) rows.weights(w, (const T*)a.w[which]);
  struct Hand {
    typename Rows::Raw x;
    int token;
    bool live;
  } one, two;
  Rows::clear(one.x);
  Rows::clear(two.x);
  int64_t last = a.tokens * (blk + 1) / a.blocks[which];    // the workgroups' shares differ by a token at most
  for (int64_t tok0 = a.tokens * blk / a.blocks[which]; tok0 < last; tok0 += per) {
    int some = (int)min((int64_t)per, last - tok0), n = some * heads;
    auto load = [&](Hand& h, int r) {
      Place<T> at(a, which, (uint32_t)tok0, r, n, x, a.xs[which], (const T*)nullptr, nullptr);
      h.token = at.token;
      h.live = at.live;
      if (at.live) rows.load(h.x, at.row[0]);
    };
    auto work = [&](const Hand& h, int r) {
      if (r >= n) return;
      float v[M];
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < Rows::N; ++i) v[k * Rows::N + i] = h.live ? Rows::at(h.x, k, i) : 0.f;
      if (h.live) {
        float2 t[KS * E];
        rows.angles(t, trig + h.token * (BBMM_ATT_MAXD / 2));
        if (a.norm) {
          norm_row<LPR, M>(v, a.inv_d, a.eps32, a.eps);
#pragma unroll
          for (int i = 0; i < M; ++i) v[i] *= w[i];
        }
        rows.template turn<false>(v, t);
      }
      rows.store(y + ((tok0 * heads) + r) * a.d, v);
    };
    int g = tid / LPR;
    load(one, g);                                          // on its way while the angles are formed
    fill_trig(a, trig, tok0, some, tid);
    __syncthreads();
    for (int r0 = 0;; r0 += 2 * GP) {
      if (r0 + GP < n) load(two, r0 + GP + g);
      work(one, r0 + g);
      if (r0 + GP >= n) break;
      if (r0 + 2 * GP < n) load(one, r0 + 2 * GP + g);
      work(two, r0 + GP + g);
      if (r0 + 2 * GP >= n) break;
    }
    __syncthreads();
  }
}

template <typename T, int E, int LPR, int KS, bool NB>
__global__ __launch_bounds__(256) void k_rotate_grad(RotArgs a) {
  typedef Row<T, E, LPR, KS, NB> Rows;
  constexpr int GP = 256 / LPR, M = Rows::N * KS;
  __shared__ float2 trig[BBMM_ROT_TOKENS * (BBMM_ATT_MAXD / 2)];
  __shared__ float sums[4][BBMM_ATT_MAXD];
  int tid = threadIdx.x, which = blockIdx.x >= (unsigned)a.blocks[0];
  int blk = blockIdx.x - (which ? a.blocks[0] : 0), per = a.tokens_per[which], heads = a.heads[which];
  Rows rows(a, tid % LPR);
  const T *x = a.norm ? (const T*)a.x[which] : nullptr, *g = (const T*)a.g[which];
  T* dx = (T*)a.y[which];
  float w[M], dw[M];
  if (a.norm) rows.weights(w, (const T*)a.w[which]);
#pragma unroll
  for (int i = 0; i < M; ++i) dw[i] = 0.f;
  struct Hand {
    typename Rows::Raw x, g;
    int token;
    bool live;
  } one;
  Rows::clear(one.x);
  Rows::clear(one.g);
  int64_t last = a.tokens * (blk + 1) / a.blocks[which];    // the workgroups' shares differ by a token at most
  for (int64_t tok0 = a.tokens * blk / a.blocks[which]; tok0 < last; tok0 += per) {
    int some = (int)min((int64_t)per, last - tok0), n = some * heads;
    auto load = [&](Hand& h, int r) {
      Place<T> at(a, which, (uint32_t)tok0, r, n, g, a.gs[which], x, a.xs[which]);
      h.token = at.token;
      h.live = at.live;
      if (at.live) {
        rows.load(h.g, at.row[0]);
        if (a.norm) rows.load(h.x, at.row[1]);
      }
    };
    auto work = [&](const Hand& h, int r) {
      if (r >= n) return;
      float v[M];
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < Rows::N; ++i) v[k * Rows::N + i] = h.live ? Rows::at(h.g, k, i) : 0.f;
      if (h.live) {
        float2 t[KS * E];
        rows.angles(t, trig + h.token * (BBMM_ATT_MAXD / 2));
        rows.template turn<true>(v, t);
        if (a.norm) {
          float nx[M];
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < Rows::N; ++i) nx[k * Rows::N + i] = Rows::at(h.x, k, i);
          float rr = norm_row<LPR, M>(nx, a.inv_d, a.eps32, a.eps), dot = 0.f;
#pragma unroll
          for (int i = 0; i < M; ++i) {
            dw[i] = fmaf(v[i], nx[i], dw[i]);
            v[i] *= w[i];
            dot = fmaf(v[i], nx[i], dot);
          }
          dot = row_sum<LPR>(dot) * a.inv_d;
#pragma unroll
          for (int i = 0; i < M; ++i) v[i] = rr * fmaf(-nx[i], dot, v[i]);
        }
      }
      rows.store(dx + ((tok0 * heads) + r) * a.d, v);
    };
    int gr = tid / LPR;
    load(one, gr);
    fill_trig(a, trig, tok0, some, tid);
    __syncthreads();
    for (int r0 = 0;;) {
      work(one, r0 + gr);
      r0 += GP;
      if (r0 >= n) break;
      load(one, r0 + gr);
    }
    __syncthreads();
  }
  if (!a.w[which]) return;
  // the workgroup's sums: over the rows of a wave, then over the waves
  for (int i = tid; i < 4 * BBMM_ATT_MAXD; i += 256) (&sums[0][0])[i] = 0.f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int s = LPR; s < 64; s *= 2) dw[i] += __shfl_xor(dw[i], s, 64);
  if ((tid & 63) < LPR) {
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < Rows::N; ++i) {
        int c = (i < E ? rows.p0[k] : rows.p1[k]) + i % E;
        if (c < a.d) sums[tid >> 6][c] = dw[k * Rows::N + i];
      }
  }
  __syncthreads();
  T* out = (T*)a.dw[which];                                  // the only workgroup: nothing to join
  for (int c = tid; c < a.d; c += 256) {
    float sum = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    if (out) out[c] = (T)sum;
    else ((float*)a.w_part)[(size_t)blockIdx.x * a.d + c] = sum;
  }
}

// The weights' gradients from the workgroups' sums (1024 of 128, bf16: 3.9 us, the launch and one
// chain of loads; 5.7 with loads under conditions, in two rounds): 16 features a workgroup, 64 threads a feature's parts, in 64 bits and a fixed order.
template <typename T>
__global__ __launch_bounds__(1024) void k_rotate_join(RotArgs a, T* dq, T* dk, int tiles) {
  __shared__ double part[16][17];
  int which = blockIdx.x >= (unsigned)tiles, f = threadIdx.x & 15, c = (blockIdx.x - (which ? tiles : 0)) * 16 + f, p0 = threadIdx.x >> 4;
  const float* src = (const float*)a.w_part + (which ? (size_t)a.blocks[0] * a.d : 0);
  T* out = which ? dk : dq;
  if (!out) return;
  double s = 0.0;
  if (c < a.d) {
    // all that four workgroups a compute unit leave, on their way at once; places behind the last are the last, and not added
    int last = a.blocks[which] - 1;
    for (int p = p0; p <= last; p += 1024) {
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = src[(size_t)min(p + 64 * u, last) * a.d + c];
#pragma unroll
      for (int u = 0; u < 16; ++u) s += p + 64 * u <= last ? (double)v[u] : 0.0;
    }
  }
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if ((threadIdx.x & 63) < 16) part[threadIdx.x >> 6][f] = s;
  __syncthreads();
  if (threadIdx.x < 16 && c < a.d) {
#pragma unroll
    for (int p = 1; p < 16; ++p) s += part[p][f];
    out[c] = (T)(float)s;
  }
}

// 16-byte pieces: lanes of a row for features up to 32, 64, 128; else single elements, 16 lanes and four slots each.
template <typename T, typename F>
void rotate_shape(const RotArgs& a, F f) {
  constexpr int E = 16 / (int)sizeof(T);
  if (!a.vec) f(Const<1>{}, Const<16>{}, Const<4>{});
  else if (a.d <= 32) f(Const<E>{}, Const<16 / E>{}, Const<1>{});
  else if (a.d <= 64) f(Const<E>{}, Const<32 / E>{}, Const<1>{});
  else f(Const<E>{}, Const<64 / E>{}, Const<1>{});
}

template <typename T>
void rotate_t(hipStream_t s, const RotArgs& a) {
  rotate_shape<T>(a, [&](auto e, auto l, auto k) {
    constexpr int E = decltype(e)::value, L = decltype(l)::value, K = decltype(k)::value;
    if (a.neighbours) k_rotate<T, E, L, K, true><<<a.blocks[0] + a.blocks[1], 256, 0, s>>>(a);
    else k_rotate<T, E, L, K, false><<<a.blocks[0] + a.blocks[1], 256, 0, s>>>(a);
  });
}
template <typename T>
void rotate_grad_t(hipStream_t s, const RotArgs& a) {
  rotate_shape<T>(a, [&](auto e, auto l, auto k) {
    constexpr int E = decltype(e)::value, L = decltype(l)::value, K = decltype(k)::value;
    if (a.neighbours) k_rotate_grad<T, E, L, K, true><<<a.blocks[0] + a.blocks[1], 256, 0, s>>>(a);
    else k_rotate_grad<T, E, L, K, false><<<a.blocks[0] + a.blocks[1], 256, 0, s>>>(a);
  });
}
template <typename T>
void rotate_join_t(hipStream_t s, const RotArgs& a, void* dq, void* dk) {
  int tiles = (a.d + 15) / 16;
  k_rotate_join<T><<<2 * tiles, 1024, 0, s>>>(a, (T*)dq, (T*)dk, tiles);
}

}  // namespace

int rotate_rows(int type, int d, int vec) {
  int n = 0;
  RotArgs a{};
  a.d = d, a.vec = vec;
  auto f = [&](auto, auto l, auto) { n = 256 / decltype(l)::value; };
  if (type == 0) rotate_shape<float>(a, f);
  else rotate_shape<__bf16>(a, f);
  return n;
}
void launch_rotate(hipStream_t s, int type, const RotArgs& a) {
  if (type == 0) rotate_t<float>(s, a);
  else if (type == 1) rotate_t<_Float16>(s, a);
  else rotate_t<__bf16>(s, a);
}
void launch_rotate_grad(hipStream_t s, int type, const RotArgs& a) {
  if (type == 0) rotate_grad_t<float>(s, a);
  else if (type == 1) rotate_grad_t<_Float16>(s, a);
  else rotate_grad_t<__bf16>(s, a);
}
void launch_rotate_join(hipStream_t s, int type, const RotArgs& a, void* dq_weight, void* dk_weight) {
  if (type == 0) rotate_join_t<float>(s, a, dq_weight, dk_weight);
  else if (type == 1) rotate_join_t<_Float16>(s, a, dq_weight, dk_weight);
  else rotate_join_t<__bf16>(s, a, dq_weight, dk_weight);
}
