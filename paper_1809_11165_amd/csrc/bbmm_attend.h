// Declarations of the attention and bucketed-bias kernels, shared with the host orchestrator.  Not part of the public
// ABI (see include/bbmm.h, "Attention").
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#define BBMM_ATT_MAXD 128      // features of Q, K and of V
#define BBMM_ATT_MAXEDGES 63   // edges of the buckets
#define BBMM_ATT_FAR 1024      // largest edge
#define BBMM_ATT_NORM_SLOTS 512   // workgroups that look for the norms of a call, or one per (batch, shared head)

// The buckets of a difference r = j - i - start (edges ascending; further than the last one, everything on a side shares a bucket).
struct AttBuckets {
  int n_edges, two_sided;
  int far;       // the last edge (1 without edges: then only the sign tells buckets apart)
  int buckets;
  int edges[BBMM_ATT_MAXEDGES + 1];   // behind the last one: the largest int
};

struct AttArgs {
  const void *Q, *K, *V;
  int64_t qs[3], ks[3], vs[3];   // strides of batch, row, head in elements
  const int32_t *q_len, *k_len;  // per batch, may be null
  const uint8_t* mask;           // batch x nk, may be null
  int64_t mask_s;
  const void* table;             // H x buckets, may be null
  const int64_t* q_start;        // per batch, may be null
  int B, H, HK, G, nq, nk, d, dv;
  float scale, c2;               // c2 = scale log2(e)
  int qvec, kvec, vvec;          // rows may be read 16 bytes at a time
  AttBuckets bk;
};

struct AttOut {
  void* O;
  int64_t os[3];
  int ovec;                      // rows may be written four elements at a time
  float* lse;                    // B x H x nq, natural logarithm
  float *pO, *pl;                // parts of a split key axis: nsplit x B x H x nq (x dv4) and their log2 sums
  int nsplit, dv4;
};

struct AttGrad {
  const void *O, *dO;            // O dense
  int64_t dos[3];
  int ovec, dovec, dqvec, dkvec, dvvec;
  const float* lse;
  void *dQ, *dK, *dV, *dtable;   // dense
  // B x H x nq, left by the dQ pass for the next: do_i.o_i, and the row's log2 of the sum as hi + lo (p = exp2((s - hi) - lo); nothing left: lo infinite)
  // fp32: w = 1 / sum of these p, and delta with the row's rest of dS, sum p (do_i.v_j - do_i.o_i) w
  float *delta, *lo, *hi, *w;
  float* tsum;                   // sums of dS by bucket per workgroup: H x (B qsplit ceil(nq / 128)) x buckets; fp32 H x (B ksplit ceil(nk / 128)) x buckets doubles
  float* norms;                  // fp16: largest |do_i| and |v_j| of each (batch, shared head), a pair per slot: B x HK x norm_slots
  int norm_slots;
  int whole_rows;                // the dQ pass forms delta from the row itself
  int rows_only;                 // a launch of the dQ kernel for just that, where the keys are split: into rsum
  float* rsum;                   // qsplit x B x H x nq pairs: sum of p, sum of p dP (fp32: sum of dS, both doubles)
  int qsplit, ksplit;            // parts that the keys of the dQ pass, and the queries of the dK, dV pass, are split into
  float *pq, *pk, *pv;           // their results: parts x the size of dQ, dK, dV
};

// type: 0 fp32, 1 fp16, 2 bf16
void launch_attend(hipStream_t s, int type, const AttArgs& a, const AttOut& o);        // 128 queries of one head per workgroup
void launch_attend_few(hipStream_t s, int type, const AttArgs& a, const AttOut& o);    // rows (i, g) of a shared head packed
void launch_attend_join(hipStream_t s, int type, const AttArgs& a, const AttOut& o);   // joins the parts
void launch_attend_norms(hipStream_t s, int type, const AttArgs& a, const AttGrad& g);
void launch_attend_dq(hipStream_t s, int type, const AttArgs& a, const AttGrad& g);
void launch_attend_dkv(hipStream_t s, int type, const AttArgs& a, const AttGrad& g);
void launch_attend_sums(hipStream_t s, int type, const AttArgs& a, const AttGrad& g);   // adds up what the two passes left in parts (fp32: and the table's gradient)

// The bias as a matrix (heads x nq x nk, `rows` rows per workgroup), and the sums of a matrix's gradient (batch x heads x nq x nk) by bucket:
// tsum holds heads x (batch ceil(nq / rows)) x buckets floats, which launch_bucket_join adds up.
void launch_bucket_bias(hipStream_t s, int type, const void* table, const AttBuckets& bk, int64_t start, int heads, int nq, int64_t nk, int rows,
                        void* out);
void launch_bucket_grad(hipStream_t s, int type, const void* dB, const AttBuckets& bk, int64_t start, int batch, int heads, int nq, int64_t nk,
                        int rows, float* tsum);
void launch_bucket_join(hipStream_t s, int type, const float* tsum, int nparts, int heads, int buckets, void* out);
