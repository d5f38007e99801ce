// Attention over the 8-bit cache for sequences with few rows (new tokens x query heads of a key head), one token above all, and the join of parts.
//
//   x_rj = q_r . (c_j s_page) / sqrt(d),   p = exp2(x - m),   o_r = sum_j p_rj (w_j u_page) / sum_j p_rj     (codes c, w; scales s, u)
//
// Every code is read once and used for a few rows only, so memory bounds it: 2 d bytes a key and head.  A CTA takes a part of the keys of one (sequence, key
// head, 16 rows); its four warps take tiles of 32 keys in turn, each with a ring and a soft-max of its own, so that nobody waits for anybody until the end, where
// the four are added up in shared memory.  Rows whose keys are cut into parts go through memory and are joined by a kernel of their own (join_kernel).
//   - The products are m16n8k16 with fp16 operands: e4m3 values are fp16 values, and one instruction converts two.  Queries are divided by a power of two so that
//     the row's largest is in [1, 2): fp16 then holds them to 2^-25 of it, better than their own type.  Probabilities are at most 1.
//   - The order of the d products of a logit is free, so a thread takes 32 neighbouring codes of a key (two 16-byte reads) as its part of eight k-steps.
//   - Values come through ldmatrix.trans as pairs of neighbouring columns; even and odd columns are separate n-tiles, so one byte permutation makes both operands.
//   - A page's value scale is a unit of the accumulators: they are multiplied by a power of two where it changes from page to page, exactly.  The unit is kept
//     within 2^60 of the largest seen, so that a page of zeros (scale 2^-126) does not take the sums out of range.
//   - The row sums add up the probabilities as rounded.
#include "common.h"
#include "dense.h"
#include "dense_rows.cuh"

namespace fastar {

constexpr int kFewThreads = 128, kFewTile = 32, kFewStages = 3;

template <int D>
struct FewSmem {
  static constexpr int tile = kFewTile * D;                        // bytes of a tile of keys, or of values
  static constexpr int stage = 2 * tile;
  static constexpr int scales = 4 * kFewStages * stage;            // [4][stages][2] floats behind the rings
  static constexpr int total = scales + 4 * kFewStages * 8;
  static constexpr int pitch = D + 4;                              // floats of a row in the join of the warps
  static constexpr int stat = 4 * 16 * pitch * 4;                  // [4][16] (m, l) behind the rows
  static_assert(stat + 4 * 16 * 8 <= scales, "the join takes the rings' place");
};

// Where a 16-byte piece of a row lies: eight rows' same piece, and a row pair's neighbouring ones, fall into different banks.
template <int D>
__device__ __forceinline__ uint32_t few_at(int row, int piece) {
  return D == 128 ? row * 128 + ((piece ^ (row & 7)) << 4) : row * 64 + ((piece ^ ((row >> 1) & 3)) << 4);
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&v)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at));
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ uint32_t f16x2_of(float lo, float hi) { return narrow2<__half>(lo, hi); }
// Bytes that are e4m3's NaN code become 0; `any` tells whether there were some.
__device__ __forceinline__ uint32_t without_nan_codes(uint32_t v, bool& any) {
  const uint32_t nan = __vcmpeq4(v & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
  any |= nan != 0;
  return v & ~nan;
}

template <class T, int D>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const DenseArgs a, int row_tiles) {
  using SM = FewSmem<D>;
  constexpr int KS = D / 16;                                       // k-steps of a logit, and 16-column blocks of the values
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  const int warp = warp_index(), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int b = blockIdx.x / row_tiles, rt = blockIdx.x % row_tiles, part = blockIdx.y, kvh = blockIdx.z;
  chain_wait();
  DenseSeq s;
  const int found = seq_of(a, b, s);
  if (found < 0 && threadIdx.x == 0 && a.status) record_status(a.status, kErrBounds);
  if (found <= 0) return;
  const int rows = s.n * a.G;
  if (rows > a.few_rows || rt * 16 >= rows) return;
  const bool whole = a.parts == 1 || s.len <= a.chunk;
  if (whole ? part > 0 : static_cast<int64_t>(part) * a.chunk >= s.len) return;
  const int past = s.len - s.n, r_last = min(rows, rt * 16 + 16) - 1;
  const int see_all = visible_end(past + rt * 16 / a.G, s.len, a.frame), see_any = visible_end(past + r_last / a.G, s.len, a.frame);
  const int k0 = whole ? 0 : part * a.chunk, k1 = whole ? see_any : min(see_any, k0 + a.chunk);

  // this thread's rows: their end, their queries as fp16 operands and what those were divided by
  int end[2];
  float factor[2];
  uint32_t qf[KS][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = rt * 16 + g + 8 * h;
    const bool live = r < rows;
    const int i = live ? r / a.G : 0, head = kvh * a.G + (live ? r % a.G : 0);
    end[h] = live ? visible_end(past + i, s.len, a.frame) : 0;
    const T* src = static_cast<const T*>(a.q) + head * a.q_hs + (s.t0 + i) * a.q_ts + c * (D / 4);
    uint4 v[D / 32];
    uint32_t most = 0;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      v[w] = live ? *reinterpret_cast<const uint4*>(src + 8 * w) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = widen2<T>((&v[w].x)[e]);
        most = max(most, max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu));
      }
    }
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    int e = static_cast<int>(most >> 23) - 127;
    e = most == 0 || e == 128 ? 0 : max(-126, min(126, e));        // (a row that is not finite stays as it is)
    const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    factor[h] = __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * (rsqrtf(static_cast<float>(D)) * 1.4426950408889634f);
#pragma unroll
    for (int w = 0; w < D / 32; ++w)
#pragma unroll
      for (int e2 = 0; e2 < 4; ++e2) {
        const float2 f = widen2<T>((&v[w].x)[e2]);
        qf[2 * w + (e2 >> 1)][h + 2 * (e2 & 1)] = f16x2_of(f.x * down, f.y * down);
      }
  }

  const uint32_t ring = sbase + warp * kFewStages * SM::stage, scale_s = sbase + SM::scales + warp * kFewStages * 8;
  // pages of the sequence, 32 at a time, one a lane
  const int n_pages = pages_of(s.len, a.PT);
  int window = -64, window_page = 0;
  const int tiles = k1 > k0 ? (k1 - k0 + kFewTile - 1) / kFewTile : 0;
  auto ask = [&](int t) {                                          // tile t goes into its stage; an empty group past the end
    if (t < tiles) {
      const int key0 = k0 + t * kFewTile, p = key0 / a.PT;
      if (p - window >= 32 || window < 0) {
        window = p;
        window_page = p + lane < n_pages ? page_of(a, b, p + lane) : 0;
      }
      const int64_t at = static_cast<int64_t>(__shfl_sync(0xffffffffu, window_page, p - window)) * a.KV + kvh;
      const int64_t off = (at * a.PT + key0 % a.PT) * D;
      const int st = (t / 4) % kFewStages;
      const uint32_t dst = ring + st * SM::stage;
      constexpr int PPR = D / 16, RPI = 32 / PPR;                  // pieces a row, rows an instruction
      const int piece = lane % PPR;
#pragma unroll
      for (int i = 0; i < kFewTile / RPI; ++i) {
        const int row = i * RPI + lane / PPR;
        const bool there = key0 + row < k1;
        const int64_t from = off + (there ? row * D + piece * 16 : 0);
        cp_async16(dst + few_at<D>(row, piece), a.kc + from, there);
        cp_async16(dst + SM::tile + few_at<D>(row, piece), a.vc + from, there);
      }
      if (lane < 2) cp_async4(scale_s + st * 8 + lane * 4, (lane ? a.vs : a.ks) + at);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[KS][2][4];
#pragma unroll
  for (int k = 0; k < KS; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[k][0][e] = o[k][1][e] = 0.f;
  float unit = 1.17549435e-38f, most_unit = 0.f;
  bool spoilt = false;
#pragma unroll
  for (int i = 0; i < kFewStages - 1; ++i) ask(warp + 4 * i);
  for (int t = warp; t < tiles; t += 4) {
    ask(t + 4 * (kFewStages - 1));
    asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 1) : "memory");
    __syncwarp();
    const int st = (t / 4) % kFewStages;
    const uint32_t ks_s = ring + st * SM::stage, vs_s = ks_s + SM::tile;
    float k_scale, v_scale;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(k_scale), "=f"(v_scale) : "r"(scale_s + st * 8));
    // logits
    float x[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
      uint32_t w[D / 16];
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint4 v = lds128(ks_s + few_at<D>(n * 8 + g, c * (D / 64) + i));
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) mma_f16(x[n], qf[k], e4m3x2_to_half2(w[k] & 0xFFFFu), e4m3x2_to_half2(w[k] >> 16));
    }
    const int key0 = k0 + t * kFewTile;
    const bool masked = key0 + kFewTile > see_all;
    const float f0 = factor[0] * k_scale, f1 = factor[1] * k_scale;
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float& v = x[n][e];
        v *= e < 2 ? f0 : f1;
        if (masked && key0 + n * 8 + 2 * c + (e & 1) >= end[e >> 1]) v = -INFINITY;
        mx[e >> 1] = fmaxf(mx[e >> 1], v);
      }
    // the accumulators' unit
    most_unit = fmaxf(most_unit, v_scale);
    const float to = fmaxf(fmaxf(v_scale, most_unit * 8.67361738e-19f), 1.17549435e-38f), p_factor = v_scale / to;
    float alpha[2], ref[2];
    const float change = unit / to;
    unit = to;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
      const float top = fmaxf(m[h], mx[h]);
      alpha[h] = m[h] == -INFINITY ? 0.f : fast_exp2(m[h] - top);
      m[h] = top;
      ref[h] = top == -INFINITY ? 0.f : top;
      l[h] *= alpha[h];
      alpha[h] *= change;
    }
    if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[k][0][e] *= alpha[e >> 1];
          o[k][1][e] *= alpha[e >> 1];
        }
    }
    uint32_t p[2][4];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = fast_exp2(x[n][2 * h] - ref[h]), p1 = fast_exp2(x[n][2 * h + 1] - ref[h]);
        uint32_t v = f16x2_of(p0, p1);
        const float2 r = __half22float2(*reinterpret_cast<__half2*>(&v));
        l[h] += r.x + r.y;
        if (p_factor != 1.f) v = f16x2_of(r.x * p_factor, r.y * p_factor);
        p[n >> 1][h + 2 * (n & 1)] = v;
      }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint32_t v[4];
      ldmatrix4_trans(v, vs_s + few_at<D>(lane, k));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (masked) v[i] = without_nan_codes(v[i], spoilt);
        v[i] = __byte_perm(v[i], 0u, 0x3120);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        mma_f16(o[k][0], p[h], e4m3x2_to_half2(v[2 * h] & 0xFFFFu), e4m3x2_to_half2(v[2 * h + 1] & 0xFFFFu));
        mma_f16(o[k][1], p[h], e4m3x2_to_half2(v[2 * h] >> 16), e4m3x2_to_half2(v[2 * h + 1] >> 16));
      }
    }
    __syncwarp();                                                  // the stage may be filled again
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  if (__syncthreads_or(spoilt ? 1 : 0)) {
    // values that are no numbers where some row does not see them: straight from the definition
    for (int r = rt * 16 + warp; r <= r_last; r += 4) dense_row_whole<T, D, true>(a, b, s.t0 + r / a.G, kvh * a.G + r % a.G, s, part);
    return;
  }
  // the warps' rows, with their units
  float* join = reinterpret_cast<float*>(smem);
  float2* stat = reinterpret_cast<float2*>(smem + SM::stat);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int row = warp * 16 + g + 8 * h;
#pragma unroll
    for (int k = 0; k < KS; ++k)
      *reinterpret_cast<float4*>(join + row * SM::pitch + 16 * k + 4 * c) =
          make_float4(o[k][0][2 * h] * unit, o[k][1][2 * h] * unit, o[k][0][2 * h + 1] * unit, o[k][1][2 * h + 1] * unit);
    if (c == 0) stat[row] = make_float2(m[h], l[h]);
  }
  __syncthreads();
  const int row = threadIdx.x >> 3, r = rt * 16 + row;
  if (r >= rows) return;
  float top = -INFINITY, sum = 0.f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[w * 16 + row].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 ml = stat[w * 16 + row];
    f[w] = ml.x == -INFINITY && ml.y == 0.f ? 0.f : fast_exp2(ml.x - top);
    sum = fmaf(ml.y, f[w], sum);
  }
  const int t = s.t0 + r / a.G, head = kvh * a.G + r % a.G;
  const int64_t part_row = (static_cast<int64_t>(part) * a.T + t) * a.H + head;
  const float inv = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
  T* out = static_cast<T*>(a.out) + head * a.q_hs + t * a.q_ts;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int col = 32 * i + 4 * (threadIdx.x & 7);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(join + (w * 16 + row) * SM::pitch + col);
      v.x = fmaf(x.x, f[w], v.x);
      v.y = fmaf(x.y, f[w], v.y);
      v.z = fmaf(x.z, f[w], v.z);
      v.w = fmaf(x.w, f[w], v.w);
    }
    if (whole) *reinterpret_cast<uint2*>(out + col) = make_uint2(narrow2<T>(v.x * inv, v.y * inv), narrow2<T>(v.z * inv, v.w * inv));
    else *reinterpret_cast<float4*>(a.part_o + part_row * D + col) = v;
  }
  if (!whole && (threadIdx.x & 7) == 0) a.part_ml[part_row] = make_float2(top, sum);
}

// The sequence of token t, or -1: the last b with cu[b] <= t, by a search with 32 probes a step.
__device__ __forceinline__ int seq_of_token(const DenseArgs& a, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = a.B;                                             // among [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, i = lo + lane * step;
    const uint32_t below = __ballot_sync(0xffffffffu, lane * step < n && a.cu[i] <= t);
    const int last = below ? 31 - __clz(below) : 0;
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}

// Rows whose keys lie in more than one part: o = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p, a warp a row, in the order of the parts.
template <class T, int D>
__global__ void __launch_bounds__(128) join_kernel(const DenseArgs a) {
  chain_wait();
  const int lane = threadIdx.x & 31;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + warp_index();
  if (row >= static_cast<int64_t>(a.T) * a.H) return;
  const int t = static_cast<int>(row / a.H), head = static_cast<int>(row % a.H), b = seq_of_token(a, t);
  DenseSeq s;
  if (seq_of(a, b, s) <= 0 || t < s.t0 || t >= s.t0 + s.n || s.len <= a.chunk) return;
  const int parts = (s.len - 1) / a.chunk + 1;
  const int64_t step = static_cast<int64_t>(a.T) * a.H;
  float top = -INFINITY;
  for (int p = lane; p < parts; p += 32) top = fmaxf(top, __ldcg(a.part_ml + row + p * step).x);
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
  float sum = 0.f, o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const float2 ml = __ldcg(a.part_ml + row + p * step);
    const float* src = a.part_o + (row + p * step) * D + lane * (D / 32);
    float x[D / 32];
    if constexpr (D == 128) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(src));
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
      const float2 v = __ldcg(reinterpret_cast<const float2*>(src));
      x[0] = v.x; x[1] = v.y;
    }
    // (a part that the row sees nothing of has no rows in memory)
    const bool none = ml.x == -INFINITY && ml.y == 0.f;
    const float f = none ? 0.f : fast_exp2(ml.x - top);
    sum = none ? sum : fmaf(ml.y, f, sum);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = none ? o[i] : fmaf(x[i], f, o[i]);
  }
  store_cols<T, D>(static_cast<T*>(a.out) + head * a.q_hs + t * a.q_ts, lane, o, sum == 0.f ? 0.f : 1.f / sum);
}

int launch_dense_few(const DenseArgs& a, int D, bool fp16, cudaStream_t st) {
  const int64_t most = static_cast<int64_t>(a.max_new) * a.G, rows = most < a.few_rows ? most : a.few_rows;
  const int row_tiles = static_cast<int>((rows + 15) / 16);
  void (*kern)(DenseArgs, int) = fp16 ? (D == 128 ? few_kernel<__half, 128> : few_kernel<__half, 64>) : (D == 128 ? few_kernel<__nv_bfloat16, 128> : few_kernel<__nv_bfloat16, 64>);
  const int smem = D == 128 ? FewSmem<128>::total : FewSmem<64>::total;
  const int r = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
  if (r != FASTAR_OK) return r;
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.B) * row_tiles), a.parts, a.KV);
  return launch_chained(kern, grid, kFewThreads, smem, st, a, row_tiles) == cudaSuccess ? FASTAR_OK : FASTAR_ERR_CUDA;
}

int launch_dense_join(const DenseArgs& a, int D, bool fp16, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(a.T) * a.H + 3) / 4));
  void (*kern)(DenseArgs) = fp16 ? (D == 128 ? join_kernel<__half, 128> : join_kernel<__half, 64>) : (D == 128 ? join_kernel<__nv_bfloat16, 128> : join_kernel<__nv_bfloat16, 64>);
  return launch_chained(kern, grid, 128, 0, st, a) == cudaSuccess ? FASTAR_OK : FASTAR_ERR_CUDA;
}

}  // namespace fastar
