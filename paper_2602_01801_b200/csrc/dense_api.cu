// C entries of the dense path (include/fastar.h): argument checks and the choice of kernels.  No device memory is allocated here.
#include <cudaTypedefs.h>

#include <cstring>
#include <mutex>
#include <tuple>
#include <type_traits>
#include <utility>

#include "common.h"
#include "dense.h"

namespace fastar {

// First error of the dense path's kernels on a device; zero when the library is loaded.
static __device__ int32_t g_dense_status;

namespace {
std::mutex g_dense_mu;
int32_t* g_dense_word[64] = {};
PFN_cuTensorMapEncodeTiled_v12000 g_dense_encode = nullptr;

int dense_device(int32_t** status) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return FASTAR_ERR_CUDA;
  if (dev < 0 || dev >= 64) return FASTAR_ERR_INVALID_ARG;
  std::lock_guard<std::mutex> lock(g_dense_mu);
  if (!g_dense_word[dev]) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return FASTAR_ERR_CUDA;
    if (major != 10) return FASTAR_ERR_NOT_SM100;
    if (!g_dense_encode) {
      void* fn = nullptr;
      cudaDriverEntryPointQueryResult q;
      if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || !fn || q != cudaDriverEntryPointSuccess) return FASTAR_ERR_CUDA;
      g_dense_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_dense_status) != cudaSuccess || !p) return FASTAR_ERR_CUDA;
    g_dense_word[dev] = static_cast<int32_t*>(p);
  }
  *status = g_dense_word[dev];
  return FASTAR_OK;
}

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
struct Span {                      // bytes of an array
  const void* p;
  int64_t bytes;
};
bool apart(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x <= y ? y - x >= static_cast<uint64_t>(a.bytes) : x - y >= static_cast<uint64_t>(b.bytes);
}
// Rows of `heads` heads: 16-byte pieces, not overlapping (a stride over one head or one token is not used)
bool rows_ok(const void* p, int64_t hs, int64_t ts, int heads, int tokens, int d) {
  return p && aligned(p, 16) && (tokens == 1 || (ts >= d && ts % 8 == 0)) && (heads == 1 || (hs >= d && hs % 8 == 0));
}
int shape_ok(int H, int KV, int D, int dtype) {
  if (KV < 1 || H < KV || H % KV != 0) return FASTAR_ERR_INVALID_ARG;
  if (dtype != FASTAR_BF16 && dtype != FASTAR_FP16) return FASTAR_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  if (H > 65535) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  return FASTAR_OK;
}
// Rows and positions are counted in 32 bits.
constexpr int64_t kMostRows = int64_t{1} << 30;
bool too_long(int total, int max_len, int H) { return static_cast<int64_t>(total) * H > kMostRows || max_len > kMostRows; }
constexpr int kMostSeqs = 1 << 20;
// ... and shares of all tiles in 64: sequences x key heads x tiles x CTAs
bool too_many(int seqs, int max_len, int KV) { return seqs > kMostSeqs || static_cast<int64_t>(seqs) * KV * (max_len / kFewKeys + 1) > (int64_t{1} << 50); }
// Tiles of 128 tokens x 64 columns of a packed tensor [heads][T][d].
int encode_packed(CUtensorMap* m, const void* ptr, int d, int64_t tokens, int heads, int64_t ts, int64_t hs, bool fp16) {
  if (tokens == 1) ts = d;                                         // (a stride over one token or one head is not used)
  if (heads == 1) hs = ts;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(tokens), static_cast<cuuint64_t>(heads)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ts) * 2, static_cast<cuuint64_t>(hs) * 2};
  const cuuint32_t box[3] = {64, 128, 1}, estr[3] = {1, 1, 1};
  return g_dense_encode(m, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? FASTAR_OK
             : FASTAR_ERR_CUDA;
}

// How attention over the cache is launched: which kernels, on how many CTAs, the parts of the kernel for many rows (of a multiple of 128 keys), and the workspace.
struct AttendPlan {
  int few_rows, few_ctas, few_tile, few_row_tiles, cta_share;      // 0: the kernel for few rows is not launched; its items are cut
  bool many, join;
  int chunk, parts;
  size_t few_o, few_ml, few_pieces, part_o, part_ml, bytes;        // offsets
};
// Up to so many rows (tokens x query heads of a key head) a sequence has the kernel for few rows; it reads and converts every code once for 16 of them at d = 128, for 32 at
// 64, the one for many once for 256.  32 sequences of 8 192 keys, 12 heads, d = 128, us there / here: 20 rows 256 / 477, 32 rows 267 / 447, 33-48 rows 403 / 469,
// 64 rows 546 / 457, 96 rows 823 / 439; d = 64: 32 rows 148 / 345, 64 rows 274 / 356, 96 rows 397 / 346.  One sequence of 32 768 keys, d = 128: 24 rows 44 / 60, 40 rows 59 / 60,
// 64 rows 74 / 62.  (Floors by bytes: 122 and 61 us for the 32 sequences, 15 for the one.)
constexpr int kFewRows = 32;
constexpr int kSms = 148;
AttendPlan attend_plan(int B, int T, int max_new, int max_len, int H, int KV, int D) {
  AttendPlan p{};
  const int64_t G = H / KV, rows = static_cast<int64_t>(max_new) * G, len = max_len, tiles = (len + 127) / 128;
  p.many = rows > kFewRows;
  const bool equal = static_cast<int64_t>(B) * max_new <= T;       // the sequences may all be that long; if they are not, the kernel for many rows serves them too
  p.chunk = static_cast<int>(tiles * 128);
  p.parts = 1;
  if (!p.many || !equal) {
    // as many CTAs as the SMs hold, or one for every 128 keys where there are fewer of those
    p.few_rows = kFewRows;
    p.few_tile = few_tile_of(rows, D);
    p.few_row_tiles = static_cast<int>(((rows < kFewRows ? rows : kFewRows) + p.few_tile - 1) / p.few_tile);
    const int64_t items = static_cast<int64_t>(B) * KV * p.few_row_tiles, units = items * tiles, most = few_ctas_an_sm(p.few_tile, D) * kSms;
    p.few_ctas = static_cast<int>(units < most ? units : most);
    p.join = tiles > 1;
    // A cluster an item, where none has more than four tiles a CTA and all are on the SMs at once.  One token, us with clusters / cut items: 4 096 keys (four tiles a CTA),
    // one sequence of 12 heads 12.6 / 10.9, four 17.4 / 17.9; 8 192 keys 18.8 / 14.8 and 27.6 / 26.8.  Up to 2 048 keys cut items have the join's launch on top of 7.6-12.5.
    int share = 8;
    while (share > 1 && share > tiles) share /= 2;
    if (items * share <= most && tiles <= 4 * share) {
      p.cta_share = share;
      p.few_ctas = static_cast<int>(items * share);
      p.join = false;
    }
  }
  if (p.many) {
    // One CTA an SM: the parts that take the fewest rounds x (key tiles + 3, what a CTA takes to begin and end), with three more for the join
    const int64_t ctas = ((static_cast<int64_t>(T) * G + 255) / 256) * KV;
    int64_t best = INT64_MAX, parts = 1;
    for (int64_t k = 1; k <= 64 && k * 4 <= tiles + 3; ++k) {
      const int64_t cost = (ctas * k + kSms - 1) / kSms * ((tiles + k - 1) / k + 3) + (k > 1 ? 3 : 0);
      if (cost < best) { best = cost; parts = k; }
      if (ctas * k > 8 * kSms) break;
    }
    p.chunk = static_cast<int>((tiles + parts - 1) / parts * 128);
    p.parts = static_cast<int>((len + p.chunk - 1) / p.chunk);
    p.join |= p.parts > 1;
  }
  auto take = [&](size_t bytes) {
    const size_t at = p.bytes;
    p.bytes += (bytes + 15) / 16 * 16;
    return at;
  };
  p.bytes = 16;
  if (p.few_ctas > 0 && p.cta_share == 0) {
    p.few_o = take(static_cast<size_t>(2 * p.few_ctas) * p.few_tile * D * 4);
    p.few_ml = take(static_cast<size_t>(2 * p.few_ctas) * p.few_tile * 8);
    p.few_pieces = take(static_cast<size_t>(T) * H * 8);
  }
  if (p.parts > 1) {
    p.part_o = take(static_cast<size_t>(p.parts) * T * H * D * 4);
    p.part_ml = take(static_cast<size_t>(p.parts) * T * H * 8);
  }
  return p;
}
}  // namespace
}  // namespace fastar

using namespace fastar;

extern "C" int fastar_block_tables(const int32_t* held, const int32_t* add, int32_t num_seqs, int32_t page_tokens, const int32_t* free_pages,
                                   int32_t num_free, const int32_t* first, int32_t* table, int32_t table_width, int32_t* cu, int32_t* lens,
                                   int64_t* slots, int32_t max_add, int32_t* first_out, void* stream) {
  if (!held || !add || (!free_pages && num_free != 0) || !first || !table || !cu || !lens || !first_out || (!slots && max_add > 0)) return FASTAR_ERR_INVALID_ARG;
  if (num_seqs < 1 || num_free < 0 || table_width < 1 || max_add < 0) return FASTAR_ERR_INVALID_ARG;
  if ((page_tokens != 64 && page_tokens != 128) || num_seqs > kMostSeqs || max_add > kMostRows) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(held, 4) || !aligned(add, 4) || !aligned(free_pages, 4) || !aligned(first, 4) || !aligned(table, 4) || !aligned(cu, 4) || !aligned(lens, 4) ||
      !aligned(slots, 8) || !aligned(first_out, 4))
    return FASTAR_ERR_INVALID_ARG;
  // every CTA reads all requests, and one writes the outputs
  const int64_t n = num_seqs;
  const Span out[5] = {{table, 4 * n * table_width}, {cu, 4 * (n + 1)}, {lens, 4 * n}, {first_out, 4}, {slots, 8 * static_cast<int64_t>(max_add)}};
  const Span in[4] = {{held, 4 * n}, {add, 4 * n}, {free_pages, 4 * static_cast<int64_t>(num_free)}, {first, 4}};
  for (int o = 0; o < 5; ++o) {
    if (out[o].bytes == 0) continue;
    for (const Span& x : in)
      if (x.bytes > 0 && !apart(out[o], x)) return FASTAR_ERR_INVALID_ARG;
    for (int x = 0; x < o; ++x)
      if (!apart(out[o], out[x])) return FASTAR_ERR_INVALID_ARG;
  }
  int32_t* status = nullptr;
  const int r = dense_device(&status);
  if (r != FASTAR_OK) return r;
  return launch_block_tables(held, add, num_seqs, page_tokens, free_pages, num_free, first, table, table_width, cu, lens, slots, max_add, first_out, status,
                             static_cast<cudaStream_t>(stream));
}

extern "C" int fastar_kv8_append(const void* k_new, const void* v_new, int64_t head_stride, int64_t token_stride, uint8_t* k_codes, uint8_t* v_codes,
                                 float* k_scale, float* v_scale, int32_t num_pages, int32_t page_tokens, const int32_t* table, int32_t table_width,
                                 const int32_t* lens, const int32_t* cu, int32_t num_seqs, int32_t total_tokens, int32_t num_kv_heads, int32_t head_dim,
                                 int32_t dtype, void* stream) {
  int r = shape_ok(num_kv_heads, num_kv_heads, head_dim, dtype);
  if (r != FASTAR_OK) return r;
  if (num_seqs < 1 || total_tokens < 0 || num_pages < 1 || table_width < 1 || !table || !lens || !cu) return FASTAR_ERR_INVALID_ARG;
  if (page_tokens != 64 && page_tokens != 128) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  if (!k_codes || !v_codes || !k_scale || !v_scale || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scale, 4) || !aligned(v_scale, 4))
    return FASTAR_ERR_INVALID_ARG;
  if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(cu, 4)) return FASTAR_ERR_INVALID_ARG;
  if (total_tokens == 0) return FASTAR_OK;
  if (!rows_ok(k_new, head_stride, token_stride, num_kv_heads, total_tokens, head_dim) || !rows_ok(v_new, head_stride, token_stride, num_kv_heads, total_tokens, head_dim))
    return FASTAR_ERR_INVALID_ARG;
  if (too_long(total_tokens, 1, num_kv_heads) || too_many(num_seqs, 1, num_kv_heads)) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  AppendArgs a{};
  a.k = k_new; a.v = v_new; a.hs = head_stride; a.ts = token_stride;
  a.T = total_tokens; a.B = num_seqs; a.KV = num_kv_heads; a.D = head_dim; a.PT = page_tokens; a.W = table_width; a.pages = num_pages;
  a.kc = k_codes; a.vc = v_codes; a.ks = k_scale; a.vs = v_scale;
  a.table = table; a.lens = lens; a.cu = cu;
  r = dense_device(&a.status);
  if (r != FASTAR_OK) return r;
  return launch_kv8_append(a, dtype == FASTAR_FP16, static_cast<cudaStream_t>(stream));
}

extern "C" size_t fastar_kv8_attention_workspace_bytes(int32_t num_seqs, int32_t total_tokens, int32_t max_new, int32_t max_len, int32_t num_heads,
                                                       int32_t num_kv_heads, int32_t head_dim) {
  if (shape_ok(num_heads, num_kv_heads, head_dim, FASTAR_BF16) != FASTAR_OK || num_seqs < 1 || total_tokens < 0 || max_new < 1 || max_len < max_new ||
      too_long(total_tokens, max_len, num_heads) || too_many(num_seqs, max_len, num_kv_heads))
    return 0;
  return attend_plan(num_seqs, total_tokens, max_new, max_len, num_heads, num_kv_heads, head_dim).bytes;
}

extern "C" int fastar_kv8_attention(const void* q, void* out, int64_t head_stride, int64_t token_stride, const uint8_t* k_codes, const uint8_t* v_codes,
                                    const float* k_scale, const float* v_scale, int32_t num_pages, int32_t page_tokens, const int32_t* table,
                                    int32_t table_width, const int32_t* lens, const int32_t* cu, int32_t num_seqs, int32_t total_tokens, int32_t max_new,
                                    int32_t max_len, int32_t num_heads, int32_t num_kv_heads, int32_t head_dim, int32_t dtype, int32_t frame_len,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  int r = shape_ok(num_heads, num_kv_heads, head_dim, dtype);
  if (r != FASTAR_OK) return r;
  if (num_seqs < 1 || total_tokens < 0 || max_new < 1 || max_len < max_new || frame_len < 0 || num_pages < 1 || table_width < 1) return FASTAR_ERR_INVALID_ARG;
  if (page_tokens != 64 && page_tokens != 128) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  if (max_len > static_cast<int64_t>(table_width) * page_tokens) return FASTAR_ERR_INVALID_ARG;
  if (too_long(total_tokens, max_len, num_heads) || too_many(num_seqs, max_len, num_kv_heads)) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  if (!table || !lens || !cu || !aligned(table, 4) || !aligned(lens, 4) || !aligned(cu, 4)) return FASTAR_ERR_INVALID_ARG;
  if (!k_codes || !v_codes || !k_scale || !v_scale || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scale, 4) || !aligned(v_scale, 4))
    return FASTAR_ERR_INVALID_ARG;
  const AttendPlan p = attend_plan(num_seqs, total_tokens, max_new, max_len, num_heads, num_kv_heads, head_dim);
  if (p.bytes > 16 && (!workspace || !aligned(workspace, 16) || workspace_bytes < p.bytes)) return FASTAR_ERR_WORKSPACE;
  if (total_tokens == 0) return FASTAR_OK;
  if (!rows_ok(q, head_stride, token_stride, num_heads, total_tokens, head_dim) || !rows_ok(out, head_stride, token_stride, num_heads, total_tokens, head_dim) || q == out)
    return FASTAR_ERR_INVALID_ARG;
  DenseArgs a{};
  a.q = q; a.out = out; a.q_hs = head_stride; a.q_ts = token_stride;
  a.T = total_tokens; a.B = num_seqs; a.H = num_heads; a.KV = num_kv_heads; a.G = num_heads / num_kv_heads;
  a.cu = cu; a.frame = frame_len; a.max_new = max_new; a.max_len = max_len;
  a.kc = k_codes; a.vc = v_codes; a.ks = k_scale; a.vs = v_scale; a.table = table; a.lens = lens;
  a.W = table_width; a.pages = num_pages; a.PT = page_tokens;
  uint8_t* w = static_cast<uint8_t*>(workspace);
  a.few_rows = p.few_rows; a.few_ctas = p.few_ctas; a.few_tile = p.few_tile; a.few_row_tiles = p.few_row_tiles; a.cta_share = p.cta_share;
  a.few_o = reinterpret_cast<float*>(w + p.few_o); a.few_ml = reinterpret_cast<float2*>(w + p.few_ml); a.few_pieces = reinterpret_cast<int2*>(w + p.few_pieces);
  a.parts = p.parts; a.chunk = p.chunk;
  a.part_o = reinterpret_cast<float*>(w + p.part_o); a.part_ml = reinterpret_cast<float2*>(w + p.part_ml);
  r = dense_device(&a.status);
  if (r != FASTAR_OK) return r;
  const bool fp16 = dtype == FASTAR_FP16;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.few_ctas > 0) r = launch_dense_few(a, head_dim, fp16, st);
  if (r == FASTAR_OK && p.many) r = launch_dense_many(a, CUtensorMap{}, CUtensorMap{}, head_dim, fp16, st);
  if (r == FASTAR_OK && p.join) r = launch_dense_join(a, head_dim, fp16, st);
  return r;
}

extern "C" int fastar_packed_attention(const void* q, const void* k, const void* v, void* out, int64_t head_stride, int64_t token_stride,
                                       int64_t kv_head_stride, int64_t kv_token_stride, const int32_t* cu, int32_t num_seqs, int32_t total_tokens,
                                       int32_t max_tokens, int32_t num_heads, int32_t num_kv_heads, int32_t head_dim, int32_t dtype, int32_t frame_len,
                                       void* stream) {
  int r = shape_ok(num_heads, num_kv_heads, head_dim, dtype);
  if (r != FASTAR_OK) return r;
  if (num_seqs < 1 || total_tokens < 0 || max_tokens < 1 || frame_len < 0 || !cu || !aligned(cu, 4)) return FASTAR_ERR_INVALID_ARG;
  if (too_long(total_tokens, max_tokens, num_heads) || too_many(num_seqs, 1, num_kv_heads)) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  if (total_tokens == 0) return FASTAR_OK;
  if (!rows_ok(q, head_stride, token_stride, num_heads, total_tokens, head_dim) || !rows_ok(out, head_stride, token_stride, num_heads, total_tokens, head_dim) || q == out)
    return FASTAR_ERR_INVALID_ARG;
  if (!rows_ok(k, kv_head_stride, kv_token_stride, num_kv_heads, total_tokens, head_dim) || !rows_ok(v, kv_head_stride, kv_token_stride, num_kv_heads, total_tokens, head_dim) ||
      k == out || v == out)
    return FASTAR_ERR_INVALID_ARG;
  DenseArgs a{};
  a.q = q; a.out = out; a.q_hs = head_stride; a.q_ts = token_stride;
  a.T = total_tokens; a.B = num_seqs; a.H = num_heads; a.KV = num_kv_heads; a.G = num_heads / num_kv_heads;
  a.cu = cu; a.frame = frame_len; a.max_new = max_tokens; a.max_len = max_tokens;
  a.k = k; a.v = v; a.kv_hs = kv_head_stride; a.kv_ts = kv_token_stride;
  a.parts = 1; a.chunk = max_tokens;
  r = dense_device(&a.status);
  if (r != FASTAR_OK) return r;
  const bool fp16 = dtype == FASTAR_FP16;
  CUtensorMap tm_k, tm_v;
  r = encode_packed(&tm_k, k, head_dim, total_tokens, num_kv_heads, kv_token_stride, kv_head_stride, fp16);
  if (r == FASTAR_OK) r = encode_packed(&tm_v, v, head_dim, total_tokens, num_kv_heads, kv_token_stride, kv_head_stride, fp16);
  if (r != FASTAR_OK) return r;
  return launch_dense_many(a, tm_k, tm_v, head_dim, fp16, static_cast<cudaStream_t>(stream));
}

namespace {
template <class A>
A from_word(int64_t w, bool& ok) {
  if constexpr (std::is_pointer<A>::value) {
    return reinterpret_cast<A>(static_cast<uintptr_t>(w));
  } else {
    const A a = static_cast<A>(w);
    if (static_cast<int64_t>(a) != w) ok = false;
    return a;
  }
}
template <class... A, size_t... I>
int call_with(int (*f)(A...), const int64_t* w, std::index_sequence<I...>) {
  bool ok = true;
  const std::tuple<A...> args{from_word<A>(w[I], ok)...};
  return ok ? f(std::get<I>(args)...) : FASTAR_ERR_INVALID_ARG;
}
template <class... A>
int call_with(int (*f)(A...), const void* args, int32_t count) {
  if (!args || count != static_cast<int32_t>(sizeof...(A))) return FASTAR_ERR_INVALID_ARG;
  int64_t w[sizeof...(A)];
  std::memcpy(w, args, sizeof(w));
  return call_with(f, w, std::make_index_sequence<sizeof...(A)>());
}
}  // namespace

extern "C" int fastar_dense_call(int32_t call, const void* args, int32_t count) {
  switch (call) {
    case FASTAR_DENSE_TABLES: return call_with(fastar_block_tables, args, count);
    case FASTAR_DENSE_APPEND: return call_with(fastar_kv8_append, args, count);
    case FASTAR_DENSE_ATTENTION: return call_with(fastar_kv8_attention, args, count);
    case FASTAR_DENSE_PACKED: return call_with(fastar_packed_attention, args, count);
    default: return FASTAR_ERR_INVALID_ARG;
  }
}

extern "C" int fastar_dense_last_status(void* stream) {
  int32_t* word = nullptr;
  const int r = dense_device(&word);
  if (r != FASTAR_OK) return r;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t status = 0;
  if (cudaMemcpyAsync(&status, word, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess) return FASTAR_ERR_CUDA;
  if (cudaMemsetAsync(word, 0, 4, st) != cudaSuccess) return FASTAR_ERR_CUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return FASTAR_ERR_CUDA;
  return status;
}
