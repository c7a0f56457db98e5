// The learned bias by buckets of the position difference as a matrix, B[h][i][j] = T[h][bucket(j - i - start)], and the gradient of
// its table, dT[h][n] = sum of dB[b][h][i][j] over bucket(j - i - start) = n.  Both are bound by the matrix's bytes.  The matrix
// is constant beyond the last edge on either side and constant along diagonals between.  16 x 4096 x 8192 in bf16 is written in 183 us, 5.9 TB/s (a
// plain fill: 6.9; rows dealt out in other orders, one row per workgroup, 4 to 256 rows and non-temporal stores were none faster);
// the gradient of 4 x 16 x 1024 x 2048 in bf16 is read in 50 us, 5.4 TB/s, and its parts are joined in 5.
#include "attend_dev.h"

using namespace att;

namespace {

// A wave takes a row: 16-byte stores from the row's first aligned element on, single elements before and after.
template <typename T>
__global__ __launch_bounds__(256) void k_bucket_bias(const T* __restrict__ table, AttBuckets bk, int64_t start, int nq, int64_t nk, int rows,
                                                     T* __restrict__ out) {
  constexpr int E = 16 / (int)sizeof(T);
  __shared__ T line[kLine];
  int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.y, far = bk.far;
  for (int n = tid; n < 2 * (far + kPad) + 1; n += 256) line[n] = table[(size_t)h * bk.buckets + bucket_of(bk, n - far - kPad)];
  __syncthreads();
  T left = line[0], right = line[2 * (far + kPad)];
  u32x4 lv, rv;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    reinterpret_cast<T*>(&lv)[e] = left;
    reinterpret_cast<T*>(&rv)[e] = right;
  }
  int64_t r1 = min((int64_t)nq, (int64_t)(blockIdx.x + 1) * rows);
  for (int64_t i = (int64_t)blockIdx.x * rows + wave; i < r1; i += 4) {
    T* row = out + ((int64_t)h * nq + i) * nk;
    int rest = rest_below(-(i + start)), n = (int)nk;        // difference of column j: j + rest
    int lead = min((int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T), n);
    int body = (n - lead) / E, tail = lead + body * E;
    if (lane < lead) row[lane] = line[min(max(lane + rest, -far), far) + far + kPad];
    if (tail + lane < n) row[tail + lane] = line[min(max(tail + lane + rest, -far), far) + far + kPad];
    u32x4* to = (u32x4*)(row + lead);
    int r0 = lead + rest;
    const T* from = line + far + kPad;
    for (int c = lane; c < body; c += 64) {
      int r = r0 + c * E;
      u32x4 v = r < 0 ? lv : rv;
      if (r + E - 1 > -far && r < far) {
#pragma unroll
        for (int e = 0; e < E; ++e) reinterpret_cast<T*>(&v)[e] = from[r + e];
      }
      to[c] = v;
    }
  }
}

// A workgroup takes `rows` rows of one (batch, head).  Differences nearer than the last edge: a thread owns a diagonal, neighbours read
// neighbouring elements; further ones: 16 bytes at a time into one sum per side.  No atomics: the order is fixed.
template <typename T>
__global__ __launch_bounds__(256) void k_bucket_grad(const T* __restrict__ dB, AttBuckets bk, int64_t start, int heads, int nq, int64_t nk,
                                                     int rows, int nparts, float* __restrict__ tsum) {
  constexpr int E = 16 / (int)sizeof(T);
  __shared__ float diag[kLine];
  __shared__ float side[2][4];
  int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.y, b = blockIdx.z, far = bk.far;
  const T* mat = dB + ((int64_t)b * heads + h) * nq * nk;
  int64_t i0 = (int64_t)blockIdx.x * rows, i1 = min((int64_t)nq, i0 + rows);
  for (int n = tid; n < 2 * far - 1; n += 256) {
    int64_t r = n - (far - 1) + start;                       // j - i
    int64_t lo = max(i0, -r), hi = min(i1, nk - r);
    int count = (int)max((int64_t)0, hi - lo);
    const T* p = count ? mat + lo * nk + lo + r : mat;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};        // eight loads in flight
    for (int i = 0; i < count; i += 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += i + e < count ? (float)p[e * (nk + 1)] : 0.f;
      p += 8 * (nk + 1);
    }
    diag[n] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  }
  float sl = 0.f, sr = 0.f;
  for (int64_t i = i0 + wave; i < i1; i += 4) {
    const T* row = mat + i * nk;
    int rest = rest_below(-(i + start)), n = (int)nk;        // difference of column j: j + rest
    int lead = min((int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T), n);
    int body = (n - lead) / E, tail = lead + body * E;
    auto one = [&](int j) {
      int r = j + rest;
      if (r <= -far) sl += (float)row[j];
      else if (r >= far) sr += (float)row[j];
    };
    if (lane < lead) one(lane);
    if (tail + lane < n) one(tail + lane);
    const u32x4* at = (const u32x4*)(row + lead);
    for (int c0 = lane; c0 < body; c0 += 4 * 64) {
      u32x4 v[4];
      int r[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {                         // four loads in flight; what lies between the edges is not read
        int c = c0 + 64 * k;
        r[k] = lead + c * E + rest;
        v[k] = u32x4{0u, 0u, 0u, 0u};
        if (c < body && (r[k] <= -far || r[k] + E - 1 >= far)) v[k] = at[c];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          float x = (float)reinterpret_cast<const T*>(&v[k])[e];
          sl += r[k] + e <= -far ? x : 0.f;
          sr += r[k] + e >= far ? x : 0.f;
        }
    }
  }
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    sl += __shfl_xor(sl, x, 64);
    sr += __shfl_xor(sr, x, 64);
  }
  if (lane == 0) {
    side[0][wave] = sl;
    side[1][wave] = sr;
  }
  __syncthreads();
  float* out = tsum + ((size_t)h * nparts + (size_t)b * gridDim.x + blockIdx.x) * bk.buckets;
  bucket_sums(bk, diag, far - 1, side[0][0] + side[0][1] + side[0][2] + side[0][3], side[1][0] + side[1][1] + side[1][2] + side[1][3], out, tid);
}

// One wave per (head, bucket).
template <typename T>
__global__ __launch_bounds__(64) void k_bucket_join(const float* __restrict__ tsum, int nparts, int buckets, T* __restrict__ out) {
  join_bucket<T>(tsum, nparts, buckets, blockIdx.y, blockIdx.x, threadIdx.x, out);
}

}  // namespace

void launch_bucket_bias(hipStream_t s, int type, const void* table, const AttBuckets& bk, int64_t start, int heads, int nq, int64_t nk, int rows,
                        void* out) {
  dim3 g((nq + rows - 1) / rows, heads);
  if (type == 0) k_bucket_bias<float><<<g, 256, 0, s>>>((const float*)table, bk, start, nq, nk, rows, (float*)out);
  else if (type == 1) k_bucket_bias<_Float16><<<g, 256, 0, s>>>((const _Float16*)table, bk, start, nq, nk, rows, (_Float16*)out);
  else k_bucket_bias<__bf16><<<g, 256, 0, s>>>((const __bf16*)table, bk, start, nq, nk, rows, (__bf16*)out);
}

void launch_bucket_grad(hipStream_t s, int type, const void* dB, const AttBuckets& bk, int64_t start, int batch, int heads, int nq, int64_t nk,
                        int rows, float* tsum) {
  int parts = (nq + rows - 1) / rows;
  dim3 g(parts, heads, batch);
  if (type == 0) k_bucket_grad<float><<<g, 256, 0, s>>>((const float*)dB, bk, start, heads, nq, nk, rows, parts * batch, tsum);
  else if (type == 1) k_bucket_grad<_Float16><<<g, 256, 0, s>>>((const _Float16*)dB, bk, start, heads, nq, nk, rows, parts * batch, tsum);
  else k_bucket_grad<__bf16><<<g, 256, 0, s>>>((const __bf16*)dB, bk, start, heads, nq, nk, rows, parts * batch, tsum);
}

void launch_bucket_join(hipStream_t s, int type, const float* tsum, int nparts, int heads, int buckets, void* out) {
  dim3 g(buckets, heads);
  if (type == 0) k_bucket_join<float><<<g, 64, 0, s>>>(tsum, nparts, buckets, (float*)out);
  else if (type == 1) k_bucket_join<_Float16><<<g, 64, 0, s>>>(tsum, nparts, buckets, (_Float16*)out);
  else k_bucket_join<__bf16><<<g, 64, 0, s>>>(tsum, nparts, buckets, (__bf16*)out);
}
