// Declarations of the rotation, cache and cached-attention kernels, shared with the host orchestrator.  Not part of the public ABI (see
// include/bbmm.h, "Rotation" and "Cache").
#pragma once

#include "bbmm_attend.h"
#include "bbmm_div.h"

#define BBMM_ROT_AXES 4
#define BBMM_ROT_TOKENS 8      // tokens of a workgroup, at most

struct RotArgs {
  const void *x[2], *g[2];       // Q and K, and the gradients of their outputs
  void *y[2], *w_part;           // dense outputs (the gradients of Q and K); w_part: parts x d floats, those of K behind those of Q
  int64_t xs[2][3], gs[2][3];
  const void* w[2];
  void* dw[2];                   // the weights' gradients, where one workgroup each sums them
  int heads[2];
  int tokens_per[2], blocks[2];  // tokens of a workgroup, workgroups
  Div by_heads[2], by_rows;
  const int64_t* pos;
  const double* freq;
  const int32_t* len;
  int64_t tokens;                // batch x rows
  int rows, d, rot, norm, neighbours;
  double eps;                    // as the caller has it: beside tiny rows a subnormal one counts
  float eps32, inv_d;
  int vec;                       // all rows may be read and written 16 bytes at a time, and pairs are pieces or lie within one
  uint8_t axis[BBMM_ATT_MAXD / 2];
};
void launch_rotate(hipStream_t s, int type, const RotArgs& a);
void launch_rotate_grad(hipStream_t s, int type, const RotArgs& a);                    // and what each workgroup has of the weights' gradients
void launch_rotate_join(hipStream_t s, int type, const RotArgs& a, void* dq_weight, void* dk_weight);
// Rows that a workgroup has in hand at a time.
int rotate_rows(int type, int d, int vec);

struct CacheArgs {
  void *K, *V;
  int64_t ks[3], vs[3];          // strides of page, row, head in elements
  uint8_t *ke, *ve;              // E4M3: exponent bytes, dense
  const int32_t* table;
  int pages, max_pages, B, HK, d, dv;
  Div page;                      // rows of a page
  int64_t rows_most;             // max_pages x rows of a page
};
struct CacheMove {
  const void *K, *V;             // write: sources.  Read: dense outputs (cast)
  int64_t ks[3], vs[3];
  int kvec, vvec;
  const int32_t *start, *n;      // write: rows of each entry; read: rows of each sequence
  int rows;
  Div by_rows, by_heads;
};
// type: of the rows outside (0 fp32, 1 fp16, 2 bf16); e4m3: the cache holds that
void launch_cache_write(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheMove& m);
void launch_cache_read(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheMove& m);

struct CacheAtt {
  const void* Q;
  int64_t qs[3];
  const int32_t *q_len, *k_len;
  int H, G, nq, qvec, causal, window;
  float c2;                      // scale log2(e)
  float cap2, cap_in;            // cap log2(e), scale / cap (0: none)
  void* O;                       // dense
  float* lse;
  float *pO, *pl;                // parts: items x H x nq (x dv4), and their log2 sums
  int* first;                    // each sequence's first item, and one behind the last: B + 1
  int items, even, dealt;        // parts of all sequences; `even` of each, or (dealt) as the lengths want it, `items` in all at most
  int least;                     // blocks of 32 keys in a part, at least (dealt)
  int dv4, ovec, blocks;         // blocks of rows per shared head
  Div by_blocks, by_hk, by_even, by_nq, by_heads;
};
int cache_rows(int type, int64_t rows);     // rows (query, head of the group) of a workgroup, where there are so many
int cache_held(int type, int e4m3, const CacheArgs& c, int64_t rows);   // workgroups that a compute unit holds
void launch_attend_cache(hipStream_t s, int type, int e4m3, const CacheArgs& c, const CacheAtt& a);
void launch_attend_cache_join(hipStream_t s, int type, const CacheArgs& c, const CacheAtt& a);
