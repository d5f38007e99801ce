// Attention over the 8-bit cache for sequences with few rows (new tokens x query heads of a key head), one token above all, and the join of parts.
//
//   x_jr = (c_j s_page) . q_r / sqrt(d),   p = exp2(x - m),   o_r = sum_j p_jr (w_j u_page) / sum_j p_jr     (codes c, w; scales s, u)
//
// Every code is read once and used for a few rows only, so memory bounds it: 2 d bytes a key and head.  The four warps of a CTA take tiles of keys in turn, each with
// a ring and a soft-max of its own, so that nobody waits for anybody until the end of a piece, where the four are added up in shared memory.
//   - Keys are the products' rows (m16n8k16: 16 keys x 8 query rows), so one token's few rows fill an instruction, and 8, 16 or 32 rows share a key's conversion.
//   - fp16 operands: e4m3 values are fp16 values, and one instruction converts two.  Queries are divided by a power of two so that the row's largest is in [1, 2):
//     fp16 then holds them to 2^-25 of it, better than their own type.  Probabilities are 2^15 at most (kHalfLift).
//   - The order of the d products of a logit is free, so a thread takes 32 neighbouring codes of a key (two 16-byte reads) as its part of eight k-steps.
//   - Values come through ldmatrix.trans as pairs of neighbouring columns; even and odd columns are rows 0-7 and 8-15 of the product's first operand, so one byte
//     permutation makes two operands.  Probabilities turn by movmatrix.
//   - A page's value scale is a unit of the accumulators: they are multiplied by a power of two where it changes from page to page, exactly.  The unit is kept
//     within 2^60 of the largest seen, so that a page of zeros (scale 2^-126) does not take the sums out of range.
//   - The row sums add up the probabilities as rounded.
// Measured (B200, us): one token each of eight sequences of 65 536 keys, 40 query and 8 key heads 174-191 (6.2 TB/s of codes cool, 5.6 at the power limit), with rows as the products'
// first operand, 16 of them, and a CTA for every 4 096 keys 282; of 32 sequences of 1 to 16 384 keys 66-68 (4.8 TB/s) after 134; of 512 sequences of up to 1 000 keys 89-102.
// Two CTAs an SM with tiles of 32 keys: 67, 121 for the last two.
#include "common.h"
#include "dense.h"
#include "dense_rows.cuh"

namespace fastar {

constexpr int kFewThreads = 128;
constexpr float kFewRaise = kHalfLift + 8.f;                       // the reference is raised when a logit exceeds it by so many binary orders, to kHalfLift below it
constexpr float kLeastScale = 1.17549435e-38f, kUnitSpan = 8.67361738e-19f;      // 2^-126, 2^-60

// NR: groups of 8 rows; TILE keys of a warp's tile, in STAGES stages
template <int D, int NR>
struct FewConf {
  // Tiles of 16 keys leave room for four CTAs an SM where there are 8 rows; with more rows they do not, and 32 keys a tile are better
  static constexpr int TILE = NR == 1 ? 16 : 32, STAGES = 2, CTAS = NR == 1 ? 4 : 2;
  static constexpr int tile = TILE * D;                            // bytes of a tile of keys, or of values
  static constexpr int stage = 2 * tile;
  static constexpr int scales = 4 * STAGES * stage;                // [4][stages][2] floats behind the rings
  static constexpr int pitch = D + 4;                              // floats of a row in the join of the warps
  static constexpr int join = scales + 4 * STAGES * 8;
  static constexpr int stat = join + 4 * 8 * NR * pitch * 4;       // [4][8 NR] (m, l) behind the rows
  static constexpr int sums = stat + 4 * 8 * NR * 8;               // [8 NR] of the CTA, its rows where the first warp's were
  static constexpr int total = sums + 8 * NR * 8;
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
__device__ __forceinline__ uint32_t turn8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
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

// The units (128 keys of a key head, few_tile rows) of a sequence, sequences after one another, in a sequence key heads, in these row tiles.  CTA c of n takes the units
// [U c / n, U (c + 1) / n): all have the same share, whatever the lengths are, and a CTA has two cut items at most, its first and its last.
struct FewSeq {
  DenseSeq s;
  int tiles, row_tiles;                                            // of 128 keys, of few_tile rows
  int64_t units;
};
__device__ __forceinline__ int64_t few_seq(const DenseArgs& a, int b, FewSeq& f) {
  const int r = seq_of(a, b, f.s);
  if (r < 0 && a.status) record_status(a.status, kErrBounds);
  const int rows = f.s.n * a.G;
  f.row_tiles = rows <= a.few_rows ? (rows + a.few_tile - 1) / a.few_tile : 0;
  f.tiles = f.s.len / kFewKeys + (f.s.len % kFewKeys != 0 ? 1 : 0);
  return f.units = static_cast<int64_t>(f.tiles) * f.row_tiles * a.KV;
}
// A CTA's way through its pieces.
struct FewWalk {
  int b;
  FewSeq f;
  int64_t base, x, x_end;                                          // units before the sequence; the next piece's first; the CTA's end
  // the piece: key head, row tile, tiles [tile0, tile1) of the item, keys [k0, k1) of which some row sees all
  int kvh, rt, tile0, tile1, k0, k1;
  __device__ __forceinline__ bool next(const DenseArgs& a) {
    if (x >= x_end) return false;
    if (x - base == f.units) {                                     // the next sequence that has some
      base += f.units;
      while (few_seq(a, ++b, f) == 0) {}
    }
    const int64_t at = x - base;
    const int item = f.units <= INT32_MAX ? static_cast<int>(at) / f.tiles : static_cast<int>(at / f.tiles);
    tile0 = static_cast<int>(at - static_cast<int64_t>(item) * f.tiles);
    kvh = f.row_tiles == 1 ? item : item / f.row_tiles;
    rt = item - kvh * f.row_tiles;
    tile1 = static_cast<int>(min(static_cast<int64_t>(f.tiles), tile0 + x_end - x));
    x += tile1 - tile0;
    k0 = tile0 * kFewKeys;
    const int last = min(f.s.n * a.G, (rt + 1) * a.few_tile) - 1;
    k1 = min(visible_end(f.s.len - f.s.n + last / a.G, f.s.len, a.frame), tile1 == f.tiles ? f.s.len : tile1 * kFewKeys);
    return true;
  }
};
__device__ __forceinline__ int64_t few_first(int64_t units, int c, int n) { return units * c / n; }
__device__ __forceinline__ int few_cta_of(int64_t units, int64_t x, int n) { return static_cast<int>(((x + 1) * n - 1) / units); }

// Clusters: where all items' shares fit the SMs at once, `cta_share` CTAs (1, 2, 4 or 8, a cluster) take equal parts of an item's keys and add them up out of each
// other's shared memory, which spares the way through memory, the join's launch, and the sum over all sequences.  (SMALL)
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t at_rank(uint32_t shared, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(shared), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 ld_rank4(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float2 ld_rank2(uint32_t at) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

template <class T, int D, int NR, bool SMALL>
__global__ void __launch_bounds__(kFewThreads, FewConf<D, NR>::CTAS) few_kernel(const DenseArgs a) {
  using SM = FewConf<D, NR>;
  constexpr int TILE = SM::TILE, STAGES = SM::STAGES, MT = TILE / 16, R = 8 * NR;
  constexpr int KS = D / 16;                                       // k-steps of a logit, and 16-column blocks of the values
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t found_s[3];                                   // all units, those before the sequence that this CTA begins in, that sequence
  const uint32_t sbase = smem_u32(smem);
  const int warp = warp_index(), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  chain_wait();
  chain_next();
  FewWalk walk, asked;
  int64_t units = 0;
  int ctas = 0;
  if constexpr (SMALL) {
    const int share = a.cta_share, id = blockIdx.x / share, rank = blockIdx.x % share, of_seq = a.KV * a.few_row_tiles;
    walk.b = id / of_seq;
    few_seq(a, walk.b, walk.f);
    walk.kvh = (id % of_seq) / a.few_row_tiles;
    walk.rt = id % a.few_row_tiles;
    if (walk.rt >= walk.f.row_tiles || walk.f.tiles == 0) return;  // (the whole cluster)
    const int64_t item = (static_cast<int64_t>(walk.kvh) * walk.f.row_tiles + walk.rt) * walk.f.tiles;
    walk.base = 0;
    walk.x = item + static_cast<int64_t>(walk.f.tiles) * rank / share;
    walk.x_end = item + static_cast<int64_t>(walk.f.tiles) * (rank + 1) / share;
  } else {
    if (a.B <= 32) {                                               // every warp by itself, a sequence a lane
      FewSeq f;
      const int64_t mine = lane < a.B ? few_seq(a, lane, f) : 0;
      int64_t upto = mine;
#pragma unroll
      for (int w = 1; w < 32; w <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, upto, w);
        if (lane >= w) upto += u;
      }
      units = __shfl_sync(0xffffffffu, upto, 31);
      ctas = units < gridDim.x ? static_cast<int>(units) : gridDim.x;
      if (static_cast<int>(blockIdx.x) >= ctas) return;
      walk.x = few_first(units, blockIdx.x, ctas);
      walk.b = __ffs(__ballot_sync(0xffffffffu, walk.x < upto)) - 1;
      walk.base = __shfl_sync(0xffffffffu, upto - mine, walk.b);
    } else {
      int64_t* red = reinterpret_cast<int64_t*>(smem);
      FewSeq f;
      auto scan = [&](int b, int64_t& mine, int64_t& step) {         // units before sequence b of this step's, b's and the step's
        mine = b < a.B ? few_seq(a, b, f) : 0;
        int64_t x = mine;
#pragma unroll
        for (int w = 1; w < 32; w <<= 1) {
          const int64_t u = __shfl_up_sync(0xffffffffu, x, w);
          if (lane >= w) x += u;
        }
        __syncthreads();
        if (lane == 31) red[warp] = x;
        __syncthreads();
        int64_t off = 0;
        step = 0;
#pragma unroll
        for (int w = 0; w < kFewThreads / 32; ++w) {
          if (w < warp) off += red[w];
          step += red[w];
        }
        return off + x - mine;
      };
      int64_t mine, step, before = scan(threadIdx.x, mine, step), all = step;
      for (int b0 = kFewThreads; b0 < a.B; b0 += kFewThreads) {
        int64_t unused;
        scan(b0 + threadIdx.x, unused, step);
        all += step;
      }
      const int n = all < gridDim.x ? static_cast<int>(all) : gridDim.x;
      if (static_cast<int>(blockIdx.x) >= n) return;
      const int64_t first = few_first(all, blockIdx.x, n);
      int64_t base = 0;
      for (int b0 = 0;; b0 += kFewThreads) {                         // (the first step's sums are at hand)
        if (b0 > 0 || a.B > kFewThreads) before = scan(b0 + threadIdx.x, mine, step);
        else step = all;
        if (mine > 0 && first >= base + before && first < base + before + mine) {
          found_s[0] = all;
          found_s[1] = base + before;
          found_s[2] = b0 + threadIdx.x;
        }
        base += step;
        if (base > first) break;
      }
      __syncthreads();
      units = found_s[0];
      ctas = units < gridDim.x ? static_cast<int>(units) : gridDim.x;
      walk.b = static_cast<int>(found_s[2]);
      walk.base = found_s[1];
      walk.x = few_first(units, blockIdx.x, ctas);
    }
    walk.x_end = few_first(units, blockIdx.x + 1, ctas);
    few_seq(a, walk.b, walk.f);
  }
  asked = walk;

  // ---- copies: a warp's tiles of all pieces, one after the other
  const uint32_t ring = sbase + warp * STAGES * SM::stage, scale_s = sbase + SM::scales + warp * STAGES * 8;
  constexpr int PPR = D / 16, RPI = 32 / PPR, COPIES = TILE / RPI;             // 16-byte pieces a row, rows an instruction, instructions a tile
  const int my_row = lane / PPR, my_piece = lane % PPR;
  uint32_t ask_st = 0;
  int key0_ask = 0, window = 0, window_page = 0;                   // pages of the sequence, 32 at a time, one a lane
  asked.k1 = 0;
  bool more = true;
  auto ask = [&]() {                                               // the next tile goes into its stage; an empty group past the end
    while (more && key0_ask >= asked.k1) {
      more = asked.next(a);
      key0_ask = asked.k0 + warp * TILE;
      window = -64;
    }
    if (more) {
      const int p = key0_ask / a.PT;
      if (p - window >= 32) {
        window = p;
        window_page = p + lane < pages_of(asked.f.s.len, a.PT) ? page_of(a, asked.b, p + lane) : 0;
      }
      const int64_t at = static_cast<int64_t>(__shfl_sync(0xffffffffu, window_page, p - window)) * a.KV + asked.kvh;
      const int64_t off = (at * a.PT + key0_ask % a.PT) * D;
      const uint32_t dst = ring + ask_st * SM::stage;
      const int rows_there = asked.k1 - key0_ask;
      if (rows_there >= TILE) {
        const uint8_t *k_src = a.kc + off + lane * 16, *v_src = a.vc + off + lane * 16;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
          const uint32_t to = dst + i * 512 + few_at<D>(my_row + (i & 1) * RPI, my_piece) - (i & 1) * 512;
          cp_async16(to, k_src + i * 512);
          cp_async16(to + SM::tile, v_src + i * 512);
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < COPIES; ++i) {
          const int row = i * RPI + my_row;
          const bool there = row < rows_there;
          const int64_t from = off + (there ? row * D + my_piece * 16 : 0);
          cp_async16(dst + few_at<D>(row, my_piece), a.kc + from, there);
          cp_async16(dst + SM::tile + few_at<D>(row, my_piece), a.vc + from, there);
        }
      }
      if (lane < 2) cp_async4(scale_s + ask_st * 8 + lane * 4, (lane ? a.vs : a.ks) + at);
      key0_ask += 4 * TILE;
      ask_st = ask_st + 1 == STAGES ? 0 : ask_st + 1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) ask();
  uint32_t st = 0;

  if (SMALL && walk.x == walk.x_end)                               // more CTAs than tiles: nothing to add to the cluster's sums
    for (int r = threadIdx.x; r < R; r += kFewThreads) *reinterpret_cast<float2*>(smem + SM::sums + r * 8) = make_float2(-INFINITY, 0.f);
  for (bool first_piece = true; walk.next(a); first_piece = false) {
    const DenseSeq s = walk.f.s;
    const int b = walk.b, kvh = walk.kvh, k0 = walk.k0, k1 = walk.k1;
    const bool whole = SMALL ? a.cta_share == 1 : walk.tile0 == 0 && walk.tile1 == walk.f.tiles;
    const int place = (2 * blockIdx.x + (first_piece ? 0 : 1)) * R;            // where a cut item's piece goes
    const int row0 = walk.rt * R, rows = min(s.n * a.G - row0, R), past = s.len - s.n;      // this piece's first row, and how many it has
    const int see_all = visible_end(past + row0 / a.G, s.len, a.frame);
    if (!SMALL && walk.tile0 == 0 && static_cast<int>(threadIdx.x) < rows) {
      const int r = row0 + threadIdx.x, last = whole ? -1 : few_cta_of(units, walk.x - walk.tile1 + walk.f.tiles - 1, ctas);      // the CTA that has the item's last unit
      a.few_pieces[static_cast<int64_t>(s.t0 + r / a.G) * a.H + kvh * a.G + r % a.G] = make_int2(place / R, last);
    }

    // queries: row g of every group, this thread's D / 4 columns, as fp16 operands; what they were divided by goes to those who have the row's logits
    uint32_t qf[NR][KS][2];
    float factor[NR][2];
    int end[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const bool live = n * 8 + g < rows;
      const int r = live ? row0 + n * 8 + g : 0, i = r / a.G, head = kvh * a.G + r - i * a.G;
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
      e = most == 0 ? 0 : e == 128 ? 113 : max(-126, min(126, e));        // (a row that is not finite: its finite numbers stay so, 2^15 at most)
      const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
      const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * (rsqrtf(static_cast<float>(D)) * 1.4426950408889634f);
#pragma unroll
      for (int w = 0; w < D / 32; ++w)
#pragma unroll
        for (int e2 = 0; e2 < 4; ++e2) {
          const float2 f = widen2<T>((&v[w].x)[e2]);
          qf[n][2 * w + (e2 >> 1)][e2 & 1] = f16x2_of(f.x * down, f.y * down);
        }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        factor[n][h] = __shfl_sync(0xffffffffu, up, (2 * c + h) * 4);
        const int r2 = n * 8 + 2 * c + h;
        end[n][h] = r2 < rows ? visible_end(past + (row0 + r2) / a.G, s.len, a.frame) : 0;
      }
    }

    float m[NR][2], o[KS][NR][4];
    float2 l[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n] = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][n][e] = 0.f;
    }
    float unit = kLeastScale, most_unit = 0.f;
    bool spoilt = false;
    auto tile = [&](int key0, auto way) {
      constexpr bool MASKED = decltype(way)::value;
      const uint32_t ks_s = ring + st * SM::stage, vs_s = ks_s + SM::tile;
      float k_scale, v_scale;
      asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(k_scale), "=f"(v_scale) : "r"(scale_s + st * 8));
      // logits: x[mt][n][e] is key mt 16 + g + 8 (e / 2), row n 8 + 2 c + e % 2
      float x[MT][NR][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int n = 0; n < NR; ++n) x[mt][n][0] = x[mt][n][1] = x[mt][n][2] = x[mt][n][3] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          const uint4 v0 = lds128(ks_s + few_at<D>(mt * 16 + g, c * (D / 64) + i)), v1 = lds128(ks_s + few_at<D>(mt * 16 + g + 8, c * (D / 64) + i));
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t k[4];
            e4m3x4_to_half2((&v0.x)[w], k[0], k[2]);
            e4m3x4_to_half2((&v1.x)[w], k[1], k[3]);
#pragma unroll
            for (int n = 0; n < NR; ++n) mma_f16(x[mt][n], k, qf[n][4 * i + w][0], qf[n][4 * i + w][1]);
          }
        }
      }
      if (MASKED) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key0 + mt * 16 + g + 8 * (e >> 1) >= end[n][e & 1]) x[mt][n][e] = -INFINITY;
      }
      // the reference is raised for all rows of the warp at once; the accumulators follow it, and their unit
      most_unit = fmaxf(most_unit, v_scale);
      const float to = fmaxf(fmaxf(v_scale, most_unit * kUnitSpan), kLeastScale);
      float mx[NR][2];
      bool change = to != unit;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v = fmaxf(x[0][n][h], x[0][n][2 + h]);
#pragma unroll
          for (int mt = 1; mt < MT; ++mt) v = fmax3(v, x[mt][n][h], x[mt][n][2 + h]);
          mx[n][h] = v * logit_factor(factor[n][h], k_scale);
          change |= mx[n][h] > m[n][h] + kFewRaise;
        }
      if (__any_sync(0xffffffffu, change)) {
        const float ratio = unit / to;
        unit = to;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float alpha[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mx[n][h] = fmaxf(mx[n][h], __shfl_xor_sync(0xffffffffu, mx[n][h], w));
            const float top = fmaxf(m[n][h], mx[n][h] - kHalfLift);
            alpha[h] = m[n][h] == -INFINITY ? 0.f : fast_exp2(m[n][h] - top);
            m[n][h] = top;
          }
          l[n].x *= alpha[0];
          l[n].y *= alpha[1];
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][n][e] *= alpha[e & 1] * ratio;
        }
      }
      const float p_factor = v_scale / unit;
      uint32_t p[MT][NR][2];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float2 f = make_float2(logit_factor(factor[n][0], k_scale), logit_factor(factor[n][1], k_scale));
        const float2 ref = make_float2(m[n][0] == -INFINITY ? 0.f : -m[n][0], m[n][1] == -INFINITY ? 0.f : -m[n][1]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 u = ffma2(make_float2(x[mt][n][2 * h], x[mt][n][2 * h + 1]), f, ref);
            uint32_t v = f16x2_of(fast_exp2(u.x), fast_exp2(u.y));
            add_f16x2(l[n], v);
            if (p_factor != 1.f) {                                 // (a page whose scale is below 2^-60 of the largest)
              const float2 r = __half22float2(*reinterpret_cast<__half2*>(&v));
              v = f16x2_of(r.x * p_factor, r.y * p_factor);
            }
            p[mt][n][h] = turn8x8(v);
          }
      }
      // o[k][n][e] is column 16 k + 2 g + e / 2, row n 8 + 2 c + e % 2
#pragma unroll
      for (int k = 0; k < KS; k += 2 / MT) {
        uint32_t v[4];
        // four 8 x 8 blocks: 32 keys of one block of columns, or 16 keys of two
        ldmatrix4_trans(v, vs_s + (MT == 2 ? few_at<D>(lane, k) : few_at<D>(lane & 15, k + (lane >> 4))));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t u = v[2 * i + h];
            if (MASKED) u = without_nan_codes(u, spoilt);
            e4m3x4_to_half2(__byte_perm(u, 0u, 0x3120), w[2 * h], w[2 * h + 1]);
          }
          const int kk = MT == 2 ? k : k + i, mt = MT == 2 ? i : 0;
#pragma unroll
          for (int n = 0; n < NR; ++n) mma_f16(o[kk][n], w, p[mt][n][0], p[mt][n][1]);
        }
      }
      st = st + 1 == STAGES ? 0 : st + 1;
    };
    for (int key0 = k0 + warp * TILE; key0 < k1; key0 += 4 * TILE) {
      ask();
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      __syncwarp();
      if (key0 + TILE <= see_all) tile(key0, std::false_type{});
      else tile(key0, std::true_type{});
      __syncwarp();                                                // the stage may be filled again
    }

    float* join = reinterpret_cast<float*>(smem + SM::join);
    float2 *stat = reinterpret_cast<float2*>(smem + SM::stat), *sums = reinterpret_cast<float2*>(smem + SM::sums);
    if (__syncthreads_or(spoilt ? 1 : 0)) {
      // values that are no numbers where some row does not see them: straight from the definition
      for (int r = warp; r < rows; r += 4)
        dense_row_to<T, D, true>(a, b, s.t0 + (row0 + r) / a.G, kvh * a.G + (row0 + r) % a.G, s, k0, k1, whole,
                                 SMALL ? join + r * SM::pitch : a.few_o + static_cast<int64_t>(place + r) * D, SMALL ? sums + r : a.few_ml + place + r);
      if (SMALL && !whole) break;
      continue;
    }
    // the warps' rows, with their units
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) {
        l[n].x += __shfl_xor_sync(0xffffffffu, l[n].x, w);
        l[n].y += __shfl_xor_sync(0xffffffffu, l[n].y, w);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = warp * R + n * 8 + 2 * c + h;
#pragma unroll
        for (int k = 0; k < KS; ++k) *reinterpret_cast<float2*>(join + row * SM::pitch + 16 * k + 2 * g) = make_float2(o[k][n][h] * unit, o[k][n][2 + h] * unit);
        if (g == 0) stat[row] = make_float2(m[n][h], h ? l[n].y : l[n].x);
      }
    }
    __syncthreads();
    constexpr int TPW = kFewThreads / R;                           // threads a row
    const int r = threadIdx.x / TPW;
    if (r < rows) {
      float top = -INFINITY, sum = 0.f, f[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[w * R + r].x);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 ml = stat[w * R + r];
        f[w] = ml.x == -INFINITY && ml.y == 0.f ? 0.f : fast_exp2(ml.x - top);
        sum = fmaf(ml.y, f[w], sum);
      }
      const int t = s.t0 + (row0 + r) / a.G, head = kvh * a.G + (row0 + r) % a.G;
      const float inv = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
      T* out = static_cast<T*>(a.out) + head * a.q_hs + t * a.q_ts;
#pragma unroll
      for (int i = 0; i < D / (4 * TPW); ++i) {
        const int col = 4 * TPW * i + 4 * (threadIdx.x % TPW);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float4 x4 = *reinterpret_cast<const float4*>(join + (w * R + r) * SM::pitch + col);
          v.x = fmaf(x4.x, f[w], v.x);
          v.y = fmaf(x4.y, f[w], v.y);
          v.z = fmaf(x4.z, f[w], v.z);
          v.w = fmaf(x4.w, f[w], v.w);
        }
        if (whole) *reinterpret_cast<uint2*>(out + col) = make_uint2(narrow2<T>(times(v.x, inv), times(v.y, inv)), narrow2<T>(times(v.z, inv), times(v.w, inv)));
        else if (SMALL) *reinterpret_cast<float4*>(join + r * SM::pitch + col) = v;        // (this thread has read what was there)
        else *reinterpret_cast<float4*>(a.few_o + static_cast<int64_t>(place + r) * D + col) = v;
      }
      if (!whole && threadIdx.x % TPW == 0) (SMALL ? sums[r] : a.few_ml[place + r]) = make_float2(top, sum);
    }
    if (SMALL) break;
  }
  if constexpr (SMALL) {
    if (a.cta_share == 1) return;
    // every CTA has a share of the columns of all rows: the parts' sums over the cluster, in the order of the keys
    cluster_sync();
    const DenseSeq s = walk.f.s;
    const int row0 = walk.rt * R, rows = min(s.n * a.G - row0, R), share = a.cta_share, cols = D / share, rank = blockIdx.x % share;
    for (int i = threadIdx.x; i < rows * (cols / 4); i += kFewThreads) {
      const int r = i / (cols / 4), col = rank * cols + i % (cols / 4) * 4;
      float top = -INFINITY, sum = 0.f;
      float2 ml[8];
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        ml[p] = p < share ? ld_rank2(at_rank(sbase + SM::sums + r * 8, p)) : make_float2(-INFINITY, 0.f);
        top = fmaxf(top, ml[p].x);
      }
      float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        if (ml[p].x == -INFINITY && ml[p].y == 0.f) continue;      // nothing of it is seen, or there is none
        const float f = fast_exp2(ml[p].x - top);
        const float4 v = ld_rank4(at_rank(sbase + SM::join + (r * SM::pitch + col) * 4, p));
        sum = fmaf(ml[p].y, f, sum);
        o4.x = fmaf(v.x, f, o4.x);
        o4.y = fmaf(v.y, f, o4.y);
        o4.z = fmaf(v.z, f, o4.z);
        o4.w = fmaf(v.w, f, o4.w);
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int t = s.t0 + (row0 + r) / a.G, head = walk.kvh * a.G + (row0 + r) % a.G;
      *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + head * a.q_hs + t * a.q_ts + col) = make_uint2(narrow2<T>(o4.x * inv, o4.y * inv), narrow2<T>(o4.z * inv, o4.w * inv));
    }
    cluster_sync();                                                // nobody leaves while its shared memory is read
  }
}

// The sequence of token t where cu is in order: the last b with cu[b] <= t, by a search with 32 probes a step.
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

// Whether token t is one of a sequence that is served, and of which.  Where the search does not find it (a token of no sequence, or an entry of cu that is out of order
// and leads it astray), all sequences are looked at.
__device__ __forceinline__ bool owner_of_token(const DenseArgs& a, int t, int& b, DenseSeq& s) {
  b = seq_of_token(a, t);
  const int r = seq_of(a, b, s);
  if (r > 0 && t >= s.t0 && t < s.t0 + s.n) return true;
  if (r == 0 && t >= a.cu[b] && t < a.cu[b + 1]) return false;     // (refused)
  for (int b0 = 0; b0 < a.B; b0 += 32) {
    b = b0 + (threadIdx.x & 31);
    const uint32_t has = __ballot_sync(0xffffffffu, b < a.B && seq_of(a, b, s) > 0 && t >= s.t0 && t < s.t0 + s.n);
    if (has) {
      b = b0 + __ffs(has) - 1;
      seq_of(a, b, s);
      return true;
    }
  }
  return false;
}

// Rows whose keys were cut: o = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p over the pieces p.  WARPS warps a row take its pieces in turn, four at a time, and are
// added up in order: eight where there are few rows, each of which may lie in hundreds of pieces, one where there are many.
constexpr int kJoinThreads = 256;

template <class T, int D, int WARPS>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const DenseArgs a) {
  __shared__ float o_s[WARPS][D];
  __shared__ float2 ml_s[WARPS];
  const int lane = threadIdx.x & 31, warp = WARPS == 1 ? 0 : warp_index();
  const int64_t row = WARPS == 1 ? static_cast<int64_t>(blockIdx.x) * (kJoinThreads / 32) + warp_index() : blockIdx.x;
  if (row >= static_cast<int64_t>(a.T) * a.H) return;              // (a whole CTA, or a warp of its own)
  chain_wait();                                                    // for cu and lens too: only this makes what was written before visible here
  const int t = static_cast<int>(row / a.H), head = static_cast<int>(row - static_cast<int64_t>(t) * a.H);
  int b;
  DenseSeq s;
  if (!owner_of_token(a, t, b, s)) return;
  const bool few = s.n * a.G <= a.few_rows;
  int parts, first = 0, row_of_few = 0;
  if (few) {
    if (a.cta_share > 0) return;                                   // clusters leave nothing to join
    const int2 p = __ldcg(a.few_pieces + row);
    if (p.y < 0) return;
    first = p.x;
    parts = p.y - p.x / 2 + 1;
    row_of_few = ((t - s.t0) * a.G + head % a.G) % a.few_tile;
  } else {
    if (a.parts == 1 || s.len <= a.chunk) return;
    parts = (s.len - 1) / a.chunk + 1;
  }
  auto place = [&](int p) {                                        // row of few_o, or of part_o
    return few ? static_cast<int64_t>(p == 0 ? first : 2 * (first / 2 + p)) * a.few_tile + row_of_few : row + p * (static_cast<int64_t>(a.T) * a.H);
  };
  const float* from = few ? a.few_o : a.part_o;
  const float2* stat = few ? a.few_ml : a.part_ml;
  float m = -INFINITY, l = 0.f, o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
  for (int p0 = warp; p0 < parts; p0 += 4 * WARPS) {
    float2 ml[4];
    float x[4][D / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + i * WARPS;
      ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) x[i][e] = 0.f;
      if (p < parts) {
        const int64_t at = place(p);
        ml[i] = __ldcg(stat + at);
        const float* src = from + at * D + lane * (D / 32);
        if constexpr (D == 128) {
          const float4 v = __ldcg(reinterpret_cast<const float4*>(src));
          x[i][0] = v.x; x[i][1] = v.y; x[i][2] = v.z; x[i][3] = v.w;
        } else {
          const float2 v = __ldcg(reinterpret_cast<const float2*>(src));
          x[i][0] = v.x; x[i][1] = v.y;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (ml[i].x == -INFINITY && ml[i].y == 0.f) continue;        // nothing of it is seen (and its row may not be in memory)
      const float top = fmaxf(m, ml[i].x), f = m == -INFINITY && l == 0.f ? 0.f : fast_exp2(m - top), w = fast_exp2(ml[i].x - top);
      m = top;
      l = l * f + ml[i].y * w;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = o[e] * f + x[i][e] * w;
    }
  }
  if constexpr (WARPS > 1) {
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o_s[warp][lane * (D / 32) + e] = o[e];
    if (lane == 0) ml_s[warp] = make_float2(m, l);
    __syncthreads();
    if (warp != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, ml_s[w].x);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 ml = ml_s[w];
      if (ml.x == -INFINITY && ml.y == 0.f) continue;
      const float f = fast_exp2(ml.x - top);
      l = fmaf(ml.y, f, l);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = fmaf(o_s[w][lane * (D / 32) + e], f, o[e]);
    }
  }
  store_cols<T, D>(static_cast<T*>(a.out) + head * a.q_hs + t * a.q_ts, lane, o, l == 0.f ? 0.f : 1.f / l);
}

// Rows of an item where a sequence has so many at most.  32 rows of 128 columns do not fit the registers; two items of 16 read the keys twice, the second time
// out of L2 (32 sequences of 24 tokens, 12 heads, 8 192 keys on average: 544 us as one item, with 700 bytes a thread spilled, 404 as two; of 8 192 keys each 262).
// 32 rows of 64 columns fit but for some 100 bytes a thread, and take 143 us there, 16 rows 102.
int few_tile_of(int64_t rows, int D) { return rows <= 8 ? 8 : rows <= 16 || D == 128 ? 16 : 32; }

template <class T, int D>
static int launch_few_t(const DenseArgs& a, cudaStream_t st) {
  auto go = [&](auto rows) {
    constexpr int NR = decltype(rows)::value;
    void (*kern)(DenseArgs) = a.cta_share > 0 ? few_kernel<T, D, NR, true> : few_kernel<T, D, NR, false>;
    const int r = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), FewConf<D, NR>::total);
    if (r != FASTAR_OK) return r;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = a.cta_share;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = a.few_ctas;
    cfg.blockDim = kFewThreads;
    cfg.dynamicSmemBytes = FewConf<D, NR>::total;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = a.cta_share > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a) == cudaSuccess ? FASTAR_OK : FASTAR_ERR_CUDA;
  };
  if constexpr (D == 64) {
    if (a.few_tile == 32) return go(std::integral_constant<int, 4>{});
  }
  return a.few_tile == 8 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 2>{});
}
int few_ctas_an_sm(int tile, int D) {
  return tile == 8 ? (D == 128 ? FewConf<128, 1>::CTAS : FewConf<64, 1>::CTAS) : tile == 16 ? (D == 128 ? FewConf<128, 2>::CTAS : FewConf<64, 2>::CTAS) : FewConf<64, 4>::CTAS;
}

int launch_dense_few(const DenseArgs& a, int D, bool fp16, cudaStream_t st) {
  if (fp16) return D == 128 ? launch_few_t<__half, 128>(a, st) : launch_few_t<__half, 64>(a, st);
  return D == 128 ? launch_few_t<__nv_bfloat16, 128>(a, st) : launch_few_t<__nv_bfloat16, 64>(a, st);
}

template <class T, int D>
static int launch_join_t(const DenseArgs& a, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(a.T) * a.H;
  if (rows > INT32_MAX) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  const bool few = rows < 4096;                                    // eight warps a row are as many as the SMs hold at once then
  const unsigned grid = static_cast<unsigned>(few ? rows : (rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32));
  return launch_chained(few ? join_kernel<T, D, 8> : join_kernel<T, D, 1>, grid, kJoinThreads, 0, st, a) == cudaSuccess ? FASTAR_OK : FASTAR_ERR_CUDA;
}
int launch_dense_join(const DenseArgs& a, int D, bool fp16, cudaStream_t st) {
  if (fp16) return D == 128 ? launch_join_t<__half, 128>(a, st) : launch_join_t<__half, 64>(a, st);
  return D == 128 ? launch_join_t<__nv_bfloat16, 128>(a, st) : launch_join_t<__nv_bfloat16, 64>(a, st);
}

}  // namespace fastar
