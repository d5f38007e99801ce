// Page tables of many requests, and the way of new rows into the 8-bit pages.
#include "common.h"
#include "dense.h"
#include "dense_rows.cuh"

namespace fastar {

// Sums over the threads before this one, for two numbers at once; `all` gets the sums over the block.  `red`: 2 x 33 words of shared memory.
__device__ __forceinline__ void block_scan2(int64_t& x, int64_t& y, int64_t& all_x, int64_t& all_y, int64_t* red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int64_t x0 = x, y0 = y;
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, x, w), v = __shfl_up_sync(0xffffffffu, y, w);
    if (lane >= w) { x += u; y += v; }
  }
  if (lane == 31) { red[warp] = x; red[33 + warp] = y; }
  __syncthreads();
  if (warp == 0) {
    int64_t u = lane < warps ? red[lane] : 0, v = lane < warps ? red[33 + lane] : 0;
    const int64_t u0 = u, v0 = v;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const int64_t p = __shfl_up_sync(0xffffffffu, u, w), q = __shfl_up_sync(0xffffffffu, v, w);
      if (lane >= w) { u += p; v += q; }
    }
    red[lane] = u - u0;
    red[33 + lane] = v - v0;
    if (lane == 31) { red[32] = u; red[65] = v; }
  }
  __syncthreads();
  x += red[warp] - x0;
  y += red[33 + warp] - y0;
  all_x = red[32];
  all_y = red[65];
}

// ---- tables ------------------------------------------------------------------------------------------------------------------------------
// need_b = pages(held + add) - pages(held); the requests' needs and tokens are summed up in order, and request b gets the free pages from its
// predecessors' sum on.  Every CTA sums up all requests by itself (1024 a step, 8 bytes each, out of L2 but for the first), so that none waits for
// another, and writes its share of the tokens' slots and of the new table entries, for which it looks up the request by bisection.  What bounds it
// is the chain of three loads, two sums and ten steps of bisection.  Slots and requests are counted in 32 bits: 2^30 of the former at most, so that a grid's
// step behind the last is one too.
constexpr int kTableThreads = 1024;

struct TableReq {
  int32_t cu, upto, held, need;          // tokens and needs before it; need < 0: refused
};

__global__ void __launch_bounds__(kTableThreads)
block_tables_kernel(const int32_t* held, const int32_t* add, int B, int PT, const int32_t* free_pages, int n_free, const int32_t* first, int32_t* table, int W, int32_t* __restrict__ cu, int32_t* __restrict__ lens, int64_t* __restrict__ slots,
                    int max_add, int32_t* __restrict__ first_out, int32_t* status) {
  __shared__ TableReq req[kTableThreads + 1];
  __shared__ int64_t red[66];
  __shared__ int granted_s;
  chain_wait();
  chain_next();
  const int f0 = *first;
  const bool list_ok = f0 >= 0 && f0 <= n_free;
  const int avail = list_ok ? n_free - f0 : 0;
  bool bad = !list_ok, full = false;
  int64_t tokens = 0, needs = 0;         // of the requests before
  if (threadIdx.x == 0) granted_s = 0;
  for (int b0 = 0; b0 < B; b0 += kTableThreads) {
    const int b = b0 + threadIdx.x, nb = min(kTableThreads, B - b0);
    int h = 0, n = 0;
    if (b < B) {
      h = held[b];
      n = add[b];
    }
    const bool odd = h < 0 || n < 0 || static_cast<int64_t>(h) + n > INT32_MAX;
    h = max(h, 0);
    n = max(n, 0);
    const int had = pages_of(h, PT), now = odd ? had : pages_of(h + n, PT);
    const bool fits = !odd && now <= W;
    int64_t c = n, u = fits ? now - had : 0, all_c, all_u;
    const int need = static_cast<int>(u);
    block_scan2(c, u, all_c, all_u, red);
    c += tokens;
    u += needs;
    const bool room = c + n <= max_add, ok = fits && room && (need == 0 || u + need <= avail);
    bad |= odd || !room;
    full |= b < B && !odd && room && !ok;
    const int ci = static_cast<int>(c < max_add ? c : max_add), ui = static_cast<int>(u < INT32_MAX ? u : INT32_MAX);
    if (threadIdx.x < nb) {
      req[threadIdx.x] = TableReq{ci, ui, h, ok ? need : -1};
      if (ok && need > 0) atomicMax(&granted_s, ui + need);
      if (blockIdx.x == 0) {
        cu[b] = ci;
        lens[b] = ok ? h + n : -1;
      }
    }
    tokens += all_c;
    needs += all_u;
    const int end = static_cast<int>(tokens < max_add ? tokens : max_add);
    if (threadIdx.x == 0) {
      req[nb] = TableReq{end, 0, 0, -1};
      if (blockIdx.x == 0 && b0 + nb == B) cu[B] = end;
    }
    __syncthreads();
    // the slots of this step's tokens
    const int t_lo = req[0].cu;
    for (int t = t_lo + blockIdx.x * kTableThreads + threadIdx.x; t < end; t += gridDim.x * kTableThreads) {
      int lo = 0, hi = nb;               // req[lo].cu <= t < req[hi].cu
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (req[mid].cu <= t) lo = mid;
        else hi = mid;
      }
      const TableReq r = req[lo];
      int64_t slot = -1;
      if (r.need >= 0) {
        const int pos = r.held + (t - r.cu), i = pos / PT, before = pages_of(r.held, PT);
        const int page = i < before ? table[static_cast<int64_t>(b0 + lo) * W + i] : free_pages[f0 + r.upto + i - before];
        if (page >= 0) slot = static_cast<int64_t>(page) * PT + pos % PT;
      }
      slots[t] = slot;
    }
    // its new table entries: a warp a request (few entries each, or a prompt's many)
    for (int i = blockIdx.x * (kTableThreads / 32) + (threadIdx.x >> 5); i < nb; i += gridDim.x * (kTableThreads / 32)) {
      const TableReq r = req[i];
      for (int p = threadIdx.x & 31; p < r.need; p += 32) table[static_cast<int64_t>(b0 + i) * W + pages_of(r.held, PT) + p] = free_pages[f0 + r.upto + p];
    }
    __syncthreads();
  }
  const int total = static_cast<int>(tokens < max_add ? tokens : max_add);
  for (int t = total + blockIdx.x * kTableThreads + threadIdx.x; t < max_add; t += gridDim.x * kTableThreads) slots[t] = -1;
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) *first_out = list_ok ? f0 + granted_s : f0;
    if (status) {
      if (bad) record_status(status, kErrBounds);
      else if (full) record_status(status, kErrCapacity);
    }
  }
}

int launch_block_tables(const int32_t* held, const int32_t* add, int B, int PT, const int32_t* free_pages, int n_free, const int32_t* first, int32_t* table, int W,
                        int32_t* cu, int32_t* lens, int64_t* slots, int max_add, int32_t* first_out, int32_t* status, cudaStream_t st) {
  const int64_t ctas = (static_cast<int64_t>(max_add) + kTableThreads - 1) / kTableThreads;
  const int grid = ctas < 1 ? 1 : ctas > 148 ? 148 : static_cast<int>(ctas);
  return launch_chained(block_tables_kernel, grid, kTableThreads, 0, st, held, add, B, PT, free_pages, n_free, first, table, W, cu, lens, slots, max_add, first_out,
                        status) == cudaSuccess
             ? FASTAR_OK
             : FASTAR_ERR_CUDA;
}

// ---- append ------------------------------------------------------------------------------------------------------------------------------
// codes = e4m3(x / s), s = 2^ceil(log2(amax / 448)) of the page's rows: with a power of two both the division and the product code x s are exact, and a
// page whose scale grows is recoded exactly but for codes that fall below e4m3's least normal number.  A CTA takes the rows that go to one page of a
// head, keys or values: they stay in registers (32 a thread) between the search for their largest value and the coding, so that every element is read once.
// Where sequences bring a few tokens each, the way to the page is what takes time, and a warp does that for a head's keys or values.
// The largest magnitude is looked for in pairs of 16-bit patterns, and only where that finds something that is not finite once more without it.
// (B200: 4 680 tokens of 12 heads of 128 10.5 us, 4.1 TB/s of its bytes, 37 440 tokens 59 us, 5.8 TB/s; with a look at every element apart 12.0 and 78.  128 threads
// with 64 registers of rows each 3 % slower, 512 with 16 a quarter.  One token each of 512 sequences, 8 heads: a CTA each 67 us, a warp each 9.5.)
constexpr int kAppendWarps = 8;                                    // of a CTA that has a warp for every head and tensor
template <int D>
constexpr int kAppendThreads = 2 * D;

__device__ __forceinline__ uint32_t e4m3x4(float x0, float x1, float x2, float x3) {
  uint32_t r;
  asm("{.reg .b16 l, h; cvt.rn.satfinite.e4m3x2.f32 l, %2, %1; cvt.rn.satfinite.e4m3x2.f32 h, %4, %3; mov.b32 %0, {l, h};}" : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
  return r;
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }      // -126 <= e <= 127
// Neither a number nor infinite values have a code of their own: both become the code that is no number.
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) <= 3.4028235e38f ? x : __int_as_float(0x7FC00000); }

// The larger magnitude of both halves, as 16-bit patterns (they are in the order of the values; above those of the finite ones lie infinity and what is no number).
__device__ __forceinline__ uint32_t larger2(uint32_t most, uint32_t pair) { return __vmaxu2(most, pair & 0x7FFF7FFFu); }
template <class T>
constexpr uint32_t kInfinite = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
// The same without what is not finite
template <class T>
__device__ __forceinline__ uint32_t larger2_finite(uint32_t most, uint32_t pair) {
  const uint32_t lo = pair & 0x7FFFu, hi = (pair >> 16) & 0x7FFFu;
  return __vmaxu2(most, (lo < kInfinite<T> ? lo : 0u) | (hi < kInfinite<T> ? hi << 16 : 0u));
}
template <class T>
__device__ __forceinline__ uint32_t bits_of_pattern(uint32_t pattern) {  // of the value in fp32
  return __float_as_uint(widen2<T>(pattern).x);
}
// 16 elements as codes.  ALL: all are finite.
template <class T, bool ALL>
__device__ __forceinline__ uint4 code16(const uint4& x0, const uint4& x1, float inv) {
  uint4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint4& x = h ? x1 : x0;
      float2 a = widen2<T>((&x.x)[2 * w]), b = widen2<T>((&x.x)[2 * w + 1]);
      a.x *= inv; a.y *= inv; b.x *= inv; b.y *= inv;
      (&o.x)[2 * h + w] = ALL ? e4m3x4(a.x, a.y, b.x, b.y) : e4m3x4(finite_or_nan(a.x), finite_or_nan(a.y), finite_or_nan(b.x), finite_or_nan(b.y));
    }
  return o;
}
// The page's other rows, from row `r0` on by `step`, at a scale larger by 1 / f
template <int D>
__device__ __forceinline__ void recode(uint8_t* page, int r0, int step, int page_rows, int row0, int rows, int c, float f) {
  for (int r = r0; r < page_rows; r += step) {
    if (r >= row0 && r < row0 + rows) continue;
    uint4* at = reinterpret_cast<uint4*>(page + r * D + c * 16);
    uint4 v = *at;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t& u = (&v.x)[w];
      const float2 a = widen2<__half>(e4m3x2_to_half2(u & 0xFFFFu)), b = widen2<__half>(e4m3x2_to_half2(u >> 16));
      u = e4m3x4(a.x * f, a.y * f, b.x * f, b.y * f);
    }
    *at = v;
  }
}

struct AppendRun {                       // rows of the call that go to rows [row0, row0 + rows) of a page, which starts anew with the first
  int64_t at, src;                       // page and head, first element
  int rows, row0;
};
template <class T, int D>
__device__ __forceinline__ void append_rows(const AppendArgs& a, const AppendRun& w, bool v, uint32_t* red) {
  constexpr int THREADS = kAppendThreads<D>, TPR = D / 16, RPP = THREADS / TPR, MAXP = 128 / RPP;      // threads a row, rows a pass
  const T* src = static_cast<const T*>(v ? a.v : a.k) + w.src;
  uint8_t* page = (v ? a.vc : a.kc) + w.at * a.PT * D;
  float* scale = (v ? a.vs : a.ks) + w.at;
  const int c = threadIdx.x % TPR, r0 = threadIdx.x / TPR;
  uint4 x[MAXP][2];
#pragma unroll
  for (int p = 0; p < MAXP; ++p) {
    const int r = p * RPP + r0;
    x[p][0] = x[p][1] = make_uint4(0u, 0u, 0u, 0u);
    if (r < w.rows) {
      const uint4* at = reinterpret_cast<const uint4*>(src + r * a.ts + c * 16);
      x[p][0] = __ldcg(at);
      x[p][1] = __ldcg(at + 1);
    }
  }
  const float was = w.row0 == 0 ? 0.f : *scale;
  auto all_threads = [&](auto larger) {
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < MAXP; ++p)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = larger(m, (&x[p][e >> 2].x)[e & 3]);
    m = __reduce_max_sync(0xffffffffu, max(m & 0xFFFFu, m >> 16));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) m = max(m, red[i]);
    return m;
  };
  uint32_t most = all_threads(larger2);
  const bool all = most < kInfinite<T>;
  if (!all) {
    __syncthreads();
    most = all_threads(larger2_finite<T>);
  }
  const float to = fmaxf(exp2i(scale_exp_of(bits_of_pattern<T>(most))), was), inv = 1.f / to;        // a power of two (2^126 at most)
#pragma unroll
  for (int p = 0; p < MAXP; ++p) {
    const int r = p * RPP + r0;
    if (r >= w.rows) break;
    *reinterpret_cast<uint4*>(page + (w.row0 + r) * D + c * 16) = all ? code16<T, true>(x[p][0], x[p][1], inv) : code16<T, false>(x[p][0], x[p][1], inv);
  }
  if (w.row0 > 0 && was < to) recode<D>(page, r0, RPP, a.PT, w.row0, w.rows, c, was * inv);
  // (every thread has read the scale before the barrier)
  if (threadIdx.x == 0 && was != to) *scale = to;
}
// The same by a warp, for any number of rows; those beyond the first pass are read twice.
template <class T, int D>
__device__ __forceinline__ void append_rows_warp(const AppendArgs& a, const AppendRun& w, bool v) {
  constexpr int TPR = D / 16, RPP = 32 / TPR;
  const T* src = static_cast<const T*>(v ? a.v : a.k) + w.src;
  uint8_t* page = (v ? a.vc : a.kc) + w.at * a.PT * D;
  float* scale = (v ? a.vs : a.ks) + w.at;
  const int lane = threadIdx.x & 31, c = lane % TPR, r0 = lane / TPR;
  const float was = w.row0 == 0 ? 0.f : *scale;
  uint32_t most = 0;
  uint4 x0 = make_uint4(0u, 0u, 0u, 0u), x1 = x0;
  auto read = [&](int r) {
    const uint4* at = reinterpret_cast<const uint4*>(src + r * a.ts + c * 16);
    x0 = __ldcg(at);
    x1 = __ldcg(at + 1);
  };
  for (int r = r0 + (w.rows - 1 - r0) / RPP * RPP; r >= r0 && r0 < w.rows; r -= RPP) {      // the first pass last, to stay in registers
    read(r);
#pragma unroll
    for (int e = 0; e < 8; ++e) most = larger2_finite<T>(most, (&(e < 4 ? x0 : x1).x)[e & 3]);
  }
  most = __reduce_max_sync(0xffffffffu, max(most & 0xFFFFu, most >> 16));
  const float to = fmaxf(exp2i(scale_exp_of(bits_of_pattern<T>(most))), was), inv = 1.f / to;
  for (int r = r0; r < w.rows; r += RPP) {
    if (r != r0) read(r);
    *reinterpret_cast<uint4*>(page + (w.row0 + r) * D + c * 16) = code16<T, false>(x0, x1, inv);
  }
  if (w.row0 > 0 && was < to) recode<D>(page, r0, RPP, a.PT, w.row0, w.rows, c, was * inv);
  if (lane == 0 && was != to) *scale = to;                         // (all lanes have read it: they met in the maximum)
}

// WARP: a warp for every head's keys and values, blockIdx.y counts eights of them; else a CTA for blockIdx.y's head, blockIdx.z its keys or values.
template <class T, int D, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kAppendWarps : kAppendThreads<D>) kv8_append_kernel(const AppendArgs a) {
  __shared__ int64_t red[66];
  __shared__ int found[2];
  __shared__ uint32_t most[kAppendThreads<D> / 32];
  chain_wait();
  chain_next();
  // the item-th touched page of the call
  int64_t before = 0;
  const int64_t item = blockIdx.x;
  if (threadIdx.x == 0) found[0] = -1;
  __syncthreads();
  for (int b0 = 0; b0 < a.B && before <= item; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    int64_t n = 0, none = 0, all, all_none;
    int mine = 0;
    if (b < a.B) {
      DenseSeq s;
      const int r = check_seq(s, a.cu[b], a.cu[b + 1], a.lens[b], a.T, a.T, a.W * static_cast<int64_t>(a.PT) > INT32_MAX ? INT32_MAX : a.W * a.PT);
      if (r < 0 && a.status) record_status(a.status, kErrBounds);
      if (r > 0) mine = pages_of(s.len, a.PT) - (s.len - s.n) / a.PT;
    }
    n = mine;
    block_scan2(n, none, all, all_none, red);
    n += before;
    if (mine > 0 && item >= n && item < n + mine) {
      found[0] = b;
      found[1] = static_cast<int>(item - n);
    }
    before += all;
    __syncthreads();
  }
  const int b = found[0];
  if (b < 0) return;
  const int t0 = a.cu[b], n = a.cu[b + 1] - t0, len = a.lens[b], past = len - n, i = past / a.PT + found[1];
  const int page = a.table[static_cast<int64_t>(b) * a.W + i];
  if (page < 0 || page >= a.pages) {
    if (threadIdx.x == 0 && a.status) record_status(a.status, kErrBounds);
    return;
  }
  const int job = blockIdx.y * kAppendWarps + (threadIdx.x >> 5), kvh = WARP ? job >> 1 : blockIdx.y;
  if (kvh >= a.KV) return;                                         // (a warp of its own)
  const int lo = max(past, i * a.PT);
  AppendRun w;
  w.row0 = lo - i * a.PT;
  w.rows = min(len - i * a.PT, a.PT) - w.row0;
  w.at = static_cast<int64_t>(page) * a.KV + kvh;
  w.src = kvh * a.hs + (t0 + lo - past) * a.ts;
  if constexpr (WARP) append_rows_warp<T, D>(a, w, (job & 1) != 0);
  else append_rows<T, D>(a, w, blockIdx.z != 0, most);
}

template <class T, int D>
static int launch_append_t(const AppendArgs& a, cudaStream_t st) {
  // n tokens lie in no more pages than n, nor than (n - 2) / PT + 2
  const int64_t most = static_cast<int64_t>(a.T) / a.PT + 2 * static_cast<int64_t>(a.B), items = most < a.T ? most : a.T;
  // A warp a head and tensor up to eight tokens a sequence.  us as warps / as CTAs (in replayed graphs, d = 128): 32 sequences of 8 heads, 1 token 3.1 / 4.3, 8 tokens 3.7 / 5.3, 16 4.9 / 5.5,
  // 32 7.4 / 7.1; 512 sequences, 1 token 9.6 / 46.7, 8 14.9 / 80, 16 20 / 85, 64 55 / 131; 4 sequences of 12 heads, 8 3.6 / 3.0, 16 4.9 / 3.1, 64 8.0 / 3.4: beyond eight
  // it depends on how many CTAs there are.
  const bool warp = a.T <= static_cast<int64_t>(a.B) * 8;
  const dim3 grid(static_cast<unsigned>(items), warp ? (2 * a.KV + kAppendWarps - 1) / kAppendWarps : a.KV, warp ? 1 : 2);
  return launch_chained(warp ? kv8_append_kernel<T, D, true> : kv8_append_kernel<T, D, false>, grid, warp ? 32 * kAppendWarps : kAppendThreads<D>, 0, st, a) == cudaSuccess
             ? FASTAR_OK
             : FASTAR_ERR_CUDA;
}
int launch_kv8_append(const AppendArgs& a, bool fp16, cudaStream_t st) {
  if (fp16) return a.D == 128 ? launch_append_t<__half, 128>(a, st) : launch_append_t<__half, 64>(a, st);
  return a.D == 128 ? launch_append_t<__nv_bfloat16, 128>(a, st) : launch_append_t<__nv_bfloat16, 64>(a, st);
}

}  // namespace fastar
