// The dense path of several rollouts (fastar_block_tables, fastar_kv8_append, fastar_kv8_attention, fastar_packed_attention): what its kernels
// share, and the index arithmetic that runs on the host too.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/fastar.h"

namespace fastar {

// Attention of packed queries.  Either keys and values are packed like the queries (k, v), or they are codes in pages (kc, vc).
struct DenseArgs {
  const void* q;                   // [H][T][D]
  void* out;
  int64_t q_hs, q_ts;              // elements
  int T, B, H, KV, G;              // G = H / KV query heads share a key head
  const int32_t* cu;               // [B + 1]
  int frame;                       // a query sees the keys up to the end of its frame of so many tokens; 0: all of its sequence
  int max_new, max_len;
  int32_t* status;                 // may be null
  const void *k, *v;               // [KV][T][D]
  int64_t kv_hs, kv_ts;
  const uint8_t *kc, *vc;          // [pages][KV][PT][D]
  const float *ks, *vs;            // [pages][KV]
  const int32_t* table;            // [B][W]
  const int32_t* lens;             // [B]
  int W, pages, PT;
  int few_rows;                    // sequences of at most so many rows (tokens x G) belong to the kernel for few rows, the others to the one for many
  // many rows: keys in parts of `chunk`, whose results are joined by a kernel of their own (parts > 1)
  int chunk, parts;
  float* part_o;                   // [parts][T][H][D]
  float2* part_ml;                 // [parts][T][H]  reference (binary orders) and sum
  // few rows: items are cut where a CTA's share of all tiles ends (dense_few.cu)
  int few_ctas, few_tile, few_row_tiles;       // rows of an item, most items of a sequence and key head
  int cta_share;                   // CTAs of an item, a cluster, which takes all of it; 0: items are cut as above
  float* few_o;                    // [2 few_ctas][few_tile][D]
  float2* few_ml;                  // [2 few_ctas][few_tile]
  int2* few_pieces;                // [T][H]  place of the row's first piece, and the last CTA that has one (-1: the row is not cut)
};

// A sequence: tokens [t0, t0 + n) of the packed axis, at positions [len - n, len) of its keys.
constexpr int kFewKeys = 128;      // keys of a unit of the kernel for few rows
struct DenseSeq {
  int t0, n, len;
};

// What the host's arrays may say of a sequence and what not.  0: there is nothing to do (n = 0, or len < 0: the tables refused the request), 1: fine,
// -1: out of range, nothing is done.
inline __host__ __device__ int check_seq(DenseSeq& s, int t0, int t1, int len, int T, int max_new, int max_len) {
  s = DenseSeq{t0, 0, 0};
  if (t0 < 0 || t1 < t0 || t1 > T || t1 - t0 > max_new) return -1;
  if (t1 == t0 || len < 0) return 0;
  if (len < t1 - t0 || len > max_len) return -1;
  s.n = t1 - t0;
  s.len = len;
  return 1;
}
// The keys that the token at position `pos` of a sequence of `len` sees: [0, end).
inline __host__ __device__ int visible_end(int pos, int len, int frame) {
  if (frame == 0) return len;
  const int64_t end = (static_cast<int64_t>(pos / frame) + 1) * frame;
  return end < len ? static_cast<int>(end) : len;
}
inline __host__ __device__ int pages_of(int tokens, int page_tokens) { return tokens / page_tokens + (tokens % page_tokens != 0 ? 1 : 0); }

// The scale of values up to amax: the least power of two with amax / scale <= 448, as an exponent; 448 = 0.875 x 2^9.
constexpr int kMinScaleExp = -126;
inline __host__ __device__ int scale_exp_of(uint32_t amax_bits) {       // bits of a finite fp32 >= 0
  const int e = static_cast<int>(amax_bits >> 23), m = static_cast<int>(amax_bits & 0x7FFFFFu);
  if (e == 0) return kMinScaleExp;                                      // below 2^-126: fits with the least scale
  const int s = e - 126 - 9 + (m > 0x600000 ? 1 : 0);                   // amax = (1 + m / 2^23) / 2 x 2^(e - 126)
  return s < kMinScaleExp ? kMinScaleExp : s;
}

#ifdef __CUDACC__
__device__ __forceinline__ int seq_of(const DenseArgs& a, int b, DenseSeq& s) {
  const int t0 = a.cu[b], t1 = a.cu[b + 1];
  return check_seq(s, t0, t1, a.lens ? a.lens[b] : t1 - t0, a.T, a.max_new, a.max_len);
}
// A page that the table names; one that does not exist is reported, and read as page 0.
__device__ __forceinline__ int page_of(const DenseArgs& a, int b, int i) {
  const int p = a.table[static_cast<int64_t>(b) * a.W + i];
  if (p >= 0 && p < a.pages) return p;
  if (a.status) atomicCAS(a.status, 0, FASTAR_ERR_BOUNDS);
  return 0;
}
#endif

int launch_block_tables(const int32_t* held, const int32_t* add, int B, int PT, const int32_t* free_pages, int n_free, const int32_t* first, int32_t* table, int W,
                        int32_t* cu, int32_t* lens, int64_t* slots, int max_add, int32_t* first_out, int32_t* status, cudaStream_t st);
struct AppendArgs {
  const void *k, *v;               // [KV][T][D]
  int64_t hs, ts;
  int T, B, KV, D, PT, W, pages;
  uint8_t *kc, *vc;
  float *ks, *vs;
  const int32_t *table, *lens, *cu;
  int32_t* status;
};
int launch_kv8_append(const AppendArgs& a, bool fp16, cudaStream_t st);
int launch_dense_many(const DenseArgs& a, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int D, bool fp16, cudaStream_t st);
int few_tile_of(int64_t rows, int D);
int few_ctas_an_sm(int rows, int D);
int launch_dense_few(const DenseArgs& a, int D, bool fp16, cudaStream_t st);
int launch_dense_join(const DenseArgs& a, int D, bool fp16, cudaStream_t st);

}  // namespace fastar
