// One row of dense attention on the FMA units, by a warp, straight from the definition: every key that the row sees, in order, and no other is
// touched.  The kernels on the tensor cores fall back to it where values that a row does not see are not finite (0 x inf would reach it).
#pragma once
#include <type_traits>

#include "dense.h"
#include "ptx.cuh"

namespace fastar {

template <class T>
__device__ __forceinline__ float2 widen2(uint32_t v) {
  if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<__half2*>(&v));
  else return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
template <class T>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    return pack_bf16x2(lo, hi);
  }
}
// Two e4m3 codes as fp16 values (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t r;
  asm("{.reg .b16 c; cvt.u16.u32 c, %1; cvt.rn.f16x2.e4m3x2 %0, c;}" : "=r"(r) : "r"(two));
  return r;
}
// The four codes of a word.
__device__ __forceinline__ void e4m3x4_to_half2(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}" : "=r"(lo), "=r"(hi) : "r"(four));
}
// Both halves of an fp16 pair to a sum each, as they are.
__device__ __forceinline__ void add_f16x2(float2& s, uint32_t b) {
  asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; add.f32.f16 %0, l, %0; add.f32.f16 %1, h, %1;}" : "+f"(s.x), "+f"(s.y) : "r"(b));
}

// fp16 probabilities are taken relative to a reference that lies so many binary orders below the largest logit it was taken from.  The reference is raised when a logit
// exceeds it by kHalfLift + 8, so they are 2^15 at most, and those of keys down to 2^-21 of the row's largest at least (2^-29 at best) keep all their bits: relative to the
// largest itself it would be 2^-14, and thousands of keys at 2^-20 beside one that has no value of its own were off by up to 3 %.
constexpr float kHalfLift = 7.f;

// What a logit is multiplied by: the power of two that its query row was divided by, 1 / sqrt(d), and the scale of its key's page.  The product of queries below 2^-20 and
// a page of zero keys (scale 2^-126) would round to 0, and that of large ones overflow: kept positive and finite, -inf stays what it is where a key is not seen, and a
// logit of 0 too.  Logits that the lower end scales are below 2^-100 either way.
__device__ __forceinline__ float logit_factor(float row, float page) { return fminf(fmaxf(row * page, 1.17549435e-38f), 3.4028235e38f); }

// D / 32 neighbouring columns of a row a lane.
template <class T, int D>
__device__ __forceinline__ void load_cols(const T* row, int lane, float (&x)[D / 32]) {
  if constexpr (D == 128) {
    const uint2 v = *reinterpret_cast<const uint2*>(row + lane * 4);
    const float2 a = widen2<T>(v.x), b = widen2<T>(v.y);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  } else {
    const float2 a = widen2<T>(*reinterpret_cast<const uint32_t*>(row + lane * 2));
    x[0] = a.x; x[1] = a.y;
  }
}
template <int D>
__device__ __forceinline__ void load_codes(const uint8_t* row, float scale, int lane, float (&x)[D / 32]) {
  uint32_t v;
  if constexpr (D == 128) v = *reinterpret_cast<const uint32_t*>(row + lane * 4);
  else v = *reinterpret_cast<const uint16_t*>(row + lane * 2);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const float2 f = widen2<__half>(e4m3x2_to_half2(v >> (16 * i)));
    x[2 * i] = f.x * scale;
    x[2 * i + 1] = f.y * scale;
  }
}

// Keys [k0, k1) for query head `head`, token t of the packed axis; m (binary orders), l and this lane's columns of sum p v.
template <class T, int D, bool PAGED>
__device__ __forceinline__ void dense_row(const DenseArgs& a, int b, int t, int head, const DenseSeq& s, int k0, int k1, float& m, float& l, float (&o)[D / 32]) {
  const int lane = threadIdx.x & 31, kvh = head / a.G;
  float q[D / 32];
  load_cols<T, D>(static_cast<const T*>(a.q) + head * a.q_hs + t * a.q_ts, lane, q);
  const float scale = rsqrtf(static_cast<float>(D)) * 1.4426950408889634f;
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
  for (int j = k0; j < k1; ++j) {
    float k[D / 32], v[D / 32];
    if (PAGED) {
      const int page = page_of(a, b, j / a.PT);
      const int64_t at = static_cast<int64_t>(page) * a.KV + kvh, row = (at * a.PT + j % a.PT) * D;
      load_codes<D>(a.kc + row, a.ks[at], lane, k);
      load_codes<D>(a.vc + row, a.vs[at], lane, v);
    } else {
      const int64_t row = kvh * a.kv_hs + (s.t0 + j) * a.kv_ts;
      load_cols<T, D>(static_cast<const T*>(a.k) + row, lane, k);
      load_cols<T, D>(static_cast<const T*>(a.v) + row, lane, v);
    }
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) x = fmaf(q[i], k[i], x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
    x *= scale;
    const float top = fmaxf(m, x), f = m == -INFINITY ? 0.f : fast_exp2(m - top), p = x == -INFINITY ? 0.f : fast_exp2(x - top);
    l = fmaf(l, f, p);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = fmaf(o[i], f, p * v[i]);
    m = top;
  }
}

// The row's end: into `out`, or as a part of it.  inv = 0: only logits of -inf were seen, the row is zeros whatever o holds (0 x NaN).
__device__ __forceinline__ float times(float o, float inv) { return inv == 0.f ? 0.f : o * inv; }
template <class T, int D>
__device__ __forceinline__ void store_cols(T* row, int lane, const float (&o)[D / 32], float inv) {
  if constexpr (D == 128)
    *reinterpret_cast<uint2*>(row + lane * 4) = make_uint2(narrow2<T>(times(o[0], inv), times(o[1], inv)), narrow2<T>(times(o[2], inv), times(o[3], inv)));
  else *reinterpret_cast<uint32_t*>(row + lane * 2) = narrow2<T>(times(o[0], inv), times(o[1], inv));
}
// (`whole`: all that the row sees is in [k0, k1), and it goes into `out`; otherwise a part of it, to part_o and part_ml.)
template <class T, int D, bool PAGED>
__device__ __forceinline__ void dense_row_to(const DenseArgs& a, int b, int t, int head, const DenseSeq& s, int k0, int k1, bool whole, float* part_o, float2* part_ml) {
  const int lane = threadIdx.x & 31, end = visible_end(s.len - s.n + (t - s.t0), s.len, a.frame);
  float m, l, o[D / 32];
  dense_row<T, D, PAGED>(a, b, t, head, s, k0, min(end, k1), m, l, o);
  if (whole) {
    // (a sum of NaN has to reach the row)
    store_cols<T, D>(static_cast<T*>(a.out) + head * a.q_hs + t * a.q_ts, lane, o, l == 0.f ? 0.f : 1.f / l);
  } else {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) part_o[lane * (D / 32) + i] = o[i];
    if (lane == 0) *part_ml = make_float2(m, l);
  }
}

}  // namespace fastar
