// Dense attention for sequences with many rows: packed prompts over their own keys (TMA), and chunks over the 8-bit cache (codes converted on the way).
//
// The rows of a key head are (token, query head) pairs, token-major, so that G query heads that share keys share their tiles, and a causal limit moves by one
// token every G rows.  A CTA takes 256 of them as two query tiles of 128 (TMEM lanes) and walks the key tiles of 128, in parts of kSub keys:
//   S_t  = Q_t K_j^T              tcgen05.mma, shared memory x shared memory -> TMEM
//   P_t  = exp2(S_t f - m)        a thread a row
//   O_t += P_t V_j                tcgen05.mma, TMEM x shared memory
// TMEM holds two S of 128 columns and two O of d.  At d = 128 that is all of it: P takes the place of its S, and a tile goes in two halves of 64 keys, so that the
// products of one half run while the other is in its exponentials.  At d = 64 P lies beside, and Q K^T of the next tile follows as soon as the logits are in registers.
// The reference of the exponentials is raised only when a logit exceeds the maximum it was taken from by 8 binary orders (O is rescaled then, by the warps that own its
// rows); it is that maximum where probabilities are bf16, and kHalfLift below it where they are fp16.  Sums add up the probabilities as rounded.  Some of the
// exponentials go to the FMA units.
// 8-bit cache: four warps read codes, two tiles ahead in registers, convert them to fp16 (exact) and put them where TMA would have put them.  Queries are fp16
// too, their row divided by a power of two; a page's key scale goes into the factor of the logits, value scales are taken relative to the largest of the
// CTA's keys (a power of two, so nothing is rounded within 2^15 of it, and a value by 2^-14 of its page's largest at most within 2^18; beyond that, and where there are NaN
// codes in a tile that some row does not see as a whole, the rows are worked out from the definition).
// What a row does not see must not reach it: V rows behind the last visible key are zeroed, and values that are not finite in a tile that some row does not see as
// a whole are taken out, and all rows of the CTA are worked out from the definition afterwards (dense_rows.cuh).
// What bounds it: at d = 128 the card's power limit (990 W, 1.7 GHz of 1.965) with the tensor pipe 0.51 of the cycles packed and exponentials 0.42; over codes their conversion
// (5 000 cycles a tile for 3 525 packed; tensor pipe 0.40, exponentials 0.36); where items have few tiles their start and end.  At d = 64 the soft-max warps' chain of load,
// maximum, exponentials, store.
// Measured (B200, us): 16 384 tokens, 8 query and 2 key heads 472 cool, 515-547 at the limit (1.03 PFLOP/s); one warp issuing for both tiles, whole tiles of 128, 520-540; the same at
// d = 64 369, whole tiles with P over S 445.  Three times 4 680 tokens, 12 heads, by frames 292-327, at d = 64 231.  1 560 queries over 29 640 8-bit keys, 12 heads 364-380, at d = 64 287:
// with the codes one tile ahead and NaN and scale work in every tile 614, whole tiles 455, queries by one warpgroup row by row and outputs by thread 396.  What an item costs
// beside its tiles: some 5 000 cycles, 14 500 with queries and outputs that way (25 000 over codes).  The way from the definition (below): 64 ms for the 1 560 queries.
// Warp roles: 0-3 and 4-7 soft-max of the two tiles (and their queries and outputs), 8-11 the codes' way in (or the look at V), 12 and 13 MMAs of the two tiles, 14 K, 15 V (TMA).
#include <cudaTypedefs.h>

#include "common.h"
#include "dense.h"
#include "dense_rows.cuh"

namespace fastar {

constexpr int kManyThreads = 512, kMoveWarp = 8, kMmaWarp = 12, kKWarp = 14, kVWarp = 15;
constexpr int kRowsCta = 256, kKeys = 128;
// The keys of a Q K^T and soft-max, and the registers a thread, dealt anew by role from 512 x 128 at launch: soft-max 256, movers 128, the rest 128 threads.
template <int D>
struct ManyRoles {
  static constexpr int kSub = D == 128 ? 64 : 128;
  static constexpr int kSoftmax = D == 128 ? 152 : 184, kMove = D == 128 ? 144 : 96, kRest = D == 128 ? 64 : 48;
  static_assert(2 * kSoftmax + kMove + kRest <= 4 * 128, "what rises takes what falls gives");
};
template <int N>
__device__ __forceinline__ void set_regs() {
  if constexpr (N > 128) setmaxnreg_inc<N>();
  else if constexpr (N < 128) setmaxnreg_dec<N>();
}
constexpr float kLeastShare = 3.8146973e-6f;                        // 2^-18: fp16 ends at 2^-24, a half of whose step is 2^-14.8 of the least such page's largest value
constexpr float kRaise = 8.f;
// Pairs of every 16 whose exponentials the FMA units work out: the converting warps want their issue slots.  Packed, 16 384 tokens, d = 128, 2 / 3 / 4 / 5: 538 / 530 / 518 /
// 527 us, d = 64 369 / 369 / 370 / 379; a frame over 8-bit keys 390 / 396 / 400 with 2 / 3 / 4 and 413 with 6.
template <bool PAGED>
constexpr int kPoly = PAGED ? 2 : 4;

template <int D>
struct ManySmem {
  static constexpr int q_tile = (D / 64) * 128 * 128;              // bytes of a query tile, and of a K or V tile
  static constexpr int SK = D == 128 ? 3 : 4, SV = D == 128 ? 2 : 4;
  static constexpr int k_off = 2 * q_tile, v_off = k_off + SK * q_tile, bar_off = v_off + SV * q_tile;
  static constexpr int scale_off = bar_off + 512;                  // [8][2] key scales of a tile's two halves
  static constexpr int misc_off = scale_off + 64;
  static constexpr int total = misc_off + 64;
  static_assert(total <= 227 * 1024, "shared memory");
};

struct ManyItem {
  int b, kvh, part, row0, rows;                                    // rows of the sequence, first of the CTA
  int past, k0;
  int nt[2], whole_from[2];                                        // key tiles of the query tiles; from which tile on some row does not see all of it
  int see;                                                         // end of the keys that any row sees
};

__host__ __device__ constexpr uint32_t make_idesc_f16(int m, int n, int b_mn_major) {
  return (1u << 4) | (static_cast<uint32_t>(b_mn_major) << 16) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
__device__ __forceinline__ void sts128(uint32_t at, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Place of a 16-byte piece of a row in a tile of 128 rows (128-byte swizzle, 64 columns of 16 bits a chunk).
__device__ __forceinline__ uint32_t tile_at16(int row, int piece) { return (piece >> 3) * 16384 + row * 128 + (((piece & 7) ^ (row & 7)) << 4); }

template <class T, int D, bool PAGED>
__global__ void __launch_bounds__(kManyThreads, 1)
many_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const DenseArgs a) {
  using SM = ManySmem<D>;
  using M = typename std::conditional<PAGED, __half, T>::type;     // the products' type
  constexpr bool kHalf = std::is_same<M, __half>::value;
  constexpr float kLift = kHalf ? kHalfLift : 0.f;
  constexpr bool kOver = D == 128;                                 // P lies over S: there is no more room in tensor memory
  constexpr int kSub = ManyRoles<D>::kSub, NS = kKeys / kSub;      // parts of a key tile
  constexpr int SK = SM::SK, SV = SM::SV;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  if (sbase & 1023u) {
    if (threadIdx.x == 0 && a.status) record_status(a.status, FASTAR_ERR_CUDA);
    return;
  }
  const uint32_t bar = sbase + SM::bar_off;
  const uint32_t bar_q = bar, bar_k_full = bar + 8, bar_k_empty = bar_k_full + 8 * SK, bar_v_full = bar_k_empty + 8 * SK, bar_v_empty = bar_v_full + 8 * SV;
  const uint32_t bar_v_clean = bar_v_empty + 8 * SV, bar_v_asked = bar_v_clean + 8 * SV;
  // [query tile][half of the keys] each: logits; they are in registers; probabilities; P V
  const uint32_t bar_s = bar_v_asked + 8 * SV, bar_ld = bar_s + 32, bar_p = bar_ld + 32, bar_pv = bar_p + 32, bar_drain = bar_pv + 32;
  constexpr int kRoleBars = 1 + 2 * SK + 4 * SV, kNumBars = kRoleBars + 18;
  static_assert(kNumBars * 8 <= 512, "barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SM::misc_off);
  volatile int* spoilt_s = abort_flag + 1;
  volatile int* done_flag = abort_flag + 2;                        // stays 0
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + SM::misc_off + 12);
  volatile float* unit_s = reinterpret_cast<volatile float*>(smem + SM::misc_off + 16);        // [4] by mover warp
  volatile int* item_s = reinterpret_cast<volatile int*>(smem + SM::misc_off + 32);           // sequence, tile of it, and its DenseSeq
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x < kNumBars) {
    const int i = threadIdx.x, role = i - kRoleBars;
    // q; k_full, k_empty; v_full, v_empty, v_clean, v_asked; s, ld, p, pv, drain
    const int count = i == 0 ? kMoveWarp : i < 1 + SK ? (PAGED ? 4 : 1) : i < 1 + 2 * SK ? 2 : i < 1 + 2 * SK + SV ? (PAGED ? 4 : 1) : i < 1 + 2 * SK + 2 * SV ? 2
                      : i < 1 + 2 * SK + 3 * SV ? 4 : role < 0 ? 1 : role < 4 ? 2 : role < 12 ? 4 : 1;
    mbar_init(bar + 8 * i, count);
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  if (!PAGED && warp == kKWarp && lane == 0) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (threadIdx.x == 0) {
    item_s[0] = -1;
    *abort_flag = *spoilt_s = *done_flag = 0;
  }
  tc_fence_before();
  chain_wait();

  // ---- the item: tiles of the sequences in order, a sequence's last (longest) first
  ManyItem it;
  DenseSeq s{0, 0, 0};
  int item_tile = 0;
  auto tiles_of = [&](int b, DenseSeq& found) {
    const int r = seq_of(a, b, found);
    if (r < 0 && a.status) record_status(a.status, kErrBounds);
    const int rows = found.n * a.G;
    return r > 0 && rows > a.few_rows ? (rows + kRowsCta - 1) / kRowsCta : 0;
  };
  if (a.B <= 32) {                                                 // every warp by itself, a sequence a lane
    const int tile = blockIdx.x / a.KV, mine = lane < a.B ? tiles_of(lane, s) : 0;
    int64_t upto = mine;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, upto, w);
      if (lane >= w) upto += u;
    }
    const unsigned has = __ballot_sync(0xffffffffu, tile < upto);  // the first of these lanes' sequence, if any
    const int b = has ? __ffs(has) - 1 : 0;
    it.b = has ? b : -1;
    item_tile = static_cast<int>(__shfl_sync(0xffffffffu, upto, b)) - 1 - tile;
    s = DenseSeq{__shfl_sync(0xffffffffu, s.t0, b), __shfl_sync(0xffffffffu, s.n, b), __shfl_sync(0xffffffffu, s.len, b)};
    __syncthreads();
  } else {
    int* red = reinterpret_cast<int*>(smem);                       // 17 words
    const int tile = blockIdx.x / a.KV;
    int64_t before = 0;
    for (int b0 = 0; b0 < a.B && before <= tile; b0 += kManyThreads) {
      const int b = b0 + threadIdx.x;
      const int mine = b < a.B ? tiles_of(b, s) : 0;
      int x = mine;
#pragma unroll
      for (int w = 1; w < 32; w <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, x, w);
        if (lane >= w) x += u;
      }
      if (lane == 31) red[warp] = x;
      __syncthreads();
      int off = 0, all = 0;
#pragma unroll
      for (int w = 0; w < kManyThreads / 32; ++w) {
        if (w < warp) off += red[w];
        all += red[w];
      }
      const int64_t first = before + off + x - mine;
      if (mine > 0 && tile >= first && tile < first + mine) {
        item_s[0] = b;
        item_s[1] = mine - 1 - static_cast<int>(tile - first);
        item_s[2] = s.t0;
        item_s[3] = s.n;
        item_s[4] = s.len;
      }
      before += all;
      __syncthreads();
    }
    it.b = item_s[0];
    item_tile = item_s[1];
    s = DenseSeq{item_s[2], item_s[3], item_s[4]};
  }
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  chain_next();
  it.kvh = blockIdx.x % a.KV;
  it.part = blockIdx.y;
  const bool whole = !PAGED || a.parts == 1 || s.len <= a.chunk;     // (packed: the keys are never cut)
  if (it.b < 0 || (whole ? it.part > 0 : static_cast<int64_t>(it.part) * a.chunk >= s.len)) {        // nothing to do
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
    return;
  }
  it.rows = s.n * a.G;
  it.row0 = item_tile * kRowsCta;
  it.past = s.len - s.n;
  it.k0 = whole ? 0 : it.part * a.chunk;
  it.see = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r0 = it.row0 + 128 * t, r1 = min(it.rows, r0 + 128) - 1;
    int any = r0 < it.rows ? visible_end(it.past + r1 / a.G, s.len, a.frame) : 0;
    if (!whole) any = min(any, it.k0 + a.chunk);
    const int all = r0 < it.rows ? visible_end(it.past + r0 / a.G, s.len, a.frame) : 0;
    it.nt[t] = any > it.k0 ? (any - it.k0 + kKeys - 1) / kKeys : 0;
    it.whole_from[t] = all > it.k0 ? (all - it.k0) / kKeys : 0;
    it.see = max(it.see, any);
  }
  const int nt = max(it.nt[0], it.nt[1]);
  const int clean_from = it.nt[1] > 0 ? (it.nt[0] > 0 ? min(it.whole_from[0], it.whole_from[1]) : it.whole_from[1]) : it.whole_from[0];


  if (warp >= kMmaWarp) {
    set_regs<ManyRoles<D>::kRest>();
    if (warp < kKWarp) {
      // ================================================================ MMAs of query tile t
      const int t = warp - kMmaWarp, n = it.nt[t];
      const uint32_t lead = elect_lane();
      constexpr uint32_t id_s = kHalf ? make_idesc_f16(128, kSub, 0) : make_idesc_bf16(128, kSub, 0);
      constexpr uint32_t id_o = kHalf ? make_idesc_f16(128, D, 1) : make_idesc_bf16(128, D, 1);
      const uint64_t qd = make_smem_desc(sbase + t * SM::q_tile, 16, 1024), kd = make_smem_desc(sbase + SM::k_off, 16, 1024);
      const uint64_t vd = make_smem_desc(sbase + SM::v_off, 16384, 1024);
      const uint32_t s_t = tmem + t * 128, o_t = tmem + 256 + t * D;
      bool ok = nt == 0 || mbar_wait_warp<kIssueWaitHintNs>(bar_q, 0, abort_flag, a.status);
      auto scores = [&](int j, int h) {                            // of the h-th kSub keys of tile j
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = ((k >> 2) * 16384 + (k & 3) * 32) >> 4;
          umma_ss(s_t + 64 * h, qd + off, kd + (((j % SK) * SM::q_tile + h * 8192) >> 4) + off, id_s, k != 0, lead);
        }
        umma_commit(bar_s + 16 * t + 8 * h, lead);
        if (lead) mbar_arrive(bar_s + 16 * t + 8 * h);             // what this warp has seen arrive (key scales) is there for those who wait
      };
      auto values = [&](int j, int h) {
        const uint32_t p = kOver ? s_t + 64 * h : tmem + 384 + t * 64;
#pragma unroll
        for (int k = 0; k < kSub / 16; ++k) umma_ts(o_t, p + k * 8, vd + (((j % SV) * SM::q_tile + (4 * h + k) * 2048) >> 4), id_o, (j | h | k) != 0, lead);
        umma_commit(bar_pv + 16 * t + 8 * h, lead);
      };
      auto leave = [&](uint32_t empty, bool used) {                // a stage that has been waited for
        if (used) umma_commit(empty, lead);
        else if (lead) mbar_arrive(empty);
      };
      auto have_k = [&](int j) {
        const bool there = mbar_wait_warp<kIssueWaitHintNs>(bar_k_full + 8 * (j % SK), (j / SK) & 1, abort_flag, a.status);
        tc_fence_after();
        return there;
      };
      if (ok && nt > 0) {
        ok = have_k(0);
        if (ok) {
          if (n > 0) {
            for (int h = 0; h < NS; ++h) scores(0, h);
          }
          leave(bar_k_empty, n > 0);
        }
      }
      for (int j = 0; j < nt && ok; ++j) {
        const bool mine = j < n, next = j + 1 < n;
        for (int h = 0; h < NS && ok; ++h) {
          auto next_scores = [&]() {                               // Q K^T of the same keys of the next tile
            if (j + 1 >= nt) return;
            if (h == 0) ok = ok && have_k(j + 1);
            if (next && !kOver) ok = ok && mbar_wait_warp(bar_ld + 16 * t + 8 * h, j & 1, abort_flag, a.status);
            if (!ok) return;
            if (!kOver) tc_fence_after();
            if (next) scores(j + 1, h);
            if (h == NS - 1) leave(bar_k_empty + 8 * ((j + 1) % SK), next);
          };
          if (!kOver) next_scores();                               // beside the exponentials of this one
          if (h == 0) {
            ok = ok && mbar_wait_warp<kIssueWaitHintNs>(bar_v_full + 8 * (j % SV), (j / SV) & 1, abort_flag, a.status);
            if (!PAGED && j >= clean_from) ok = ok && mbar_wait_warp(bar_v_clean + 8 * (j % SV), ((j - clean_from) / SV) & 1, abort_flag, a.status);
          }
          if (mine) ok = ok && mbar_wait_warp(bar_p + 16 * t + 8 * h, j & 1, abort_flag, a.status);
          if (!ok) break;
          tc_fence_after();
          if (mine) values(j, h);
          if (kOver) next_scores();
        }
        if (ok) leave(bar_v_empty + 8 * (j % SV), mine);
      }
      umma_commit(bar_drain + 8 * t, lead);                        // nothing is in flight when tensor memory goes back
      mbar_wait_warp(bar_drain + 8 * t, 0, done_flag, a.status);
    } else if (!PAGED && (warp == kKWarp || warp == kVWarp)) {
      // ================================================================ K or V tiles by TMA
      const bool is_k = warp == kKWarp;
      const int stages = is_k ? SK : SV;
      const uint32_t full = is_k ? bar_k_full : bar_v_full, empty = is_k ? bar_k_empty : bar_v_empty, ring = sbase + (is_k ? SM::k_off : SM::v_off);
      const CUtensorMap* tm = is_k ? &tm_k : &tm_v;
      int copied = 0;
      for (int j = 0; j < nt; ++j) {
        const int st = j % stages;
        if (j >= stages && !mbar_wait_warp<kIssueWaitHintNs>(empty + 8 * st, (j / stages - 1) & 1, abort_flag, a.status)) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(full + 8 * st, SM::q_tile);
          for (int kc = 0; kc < D / 64; ++kc) tma_load_3d(ring + st * SM::q_tile + kc * 16384, tm, full + 8 * st, kc * 64, s.t0 + it.k0 + j * kKeys, it.kvh);
          if (!is_k && j >= clean_from) mbar_arrive(bar_v_asked + 8 * st);
        }
        ++copied;
      }
      for (int j = max(0, copied - stages); j < copied; ++j) mbar_wait_warp(full + 8 * (j % stages), (j / stages) & 1, done_flag, a.status);      // all copies have landed
    }
  } else if (warp >= kMoveWarp) {
    set_regs<ManyRoles<D>::kMove>();
    const int tid = threadIdx.x - kMoveWarp * 32;
    bool spoilt = false;
    if constexpr (!PAGED) {
      // ================================================================ V of tiles that some row does not see as a whole
      for (int j = clean_from; j < nt; ++j) {
        const int st = j % SV;
        // (a parity tells two phases apart: the copy before this one into the stage is through once this one has been asked for)
        if (!mbar_wait_warp<kIssueWaitHintNs>(bar_v_asked + 8 * st, ((j - clean_from) / SV) & 1, abort_flag, a.status)) break;
        if (!mbar_wait_warp<kIssueWaitHintNs>(bar_v_full + 8 * st, (j / SV) & 1, abort_flag, a.status)) break;
        const uint32_t tile = sbase + SM::v_off + st * SM::q_tile;
        const bool gone = it.k0 + j * kKeys + tid >= it.see;
        constexpr uint32_t kExp = kHalf ? 0x7C00u : 0x7F80u;
#pragma unroll 4
        for (int p = 0; p < D / 8; ++p) {
          const uint32_t at = tile + tile_at16(tid, p);
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          bool change = gone;
          if (!gone) {
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t& u = (&v.x)[w];
              if ((u & kExp) == kExp) { u &= 0xFFFF0000u; change = spoilt = true; }
              if ((u & (kExp << 16)) == kExp << 16) { u &= 0xFFFFu; change = spoilt = true; }
            }
          }
          if (change) sts128(at, v);
        }
        fence_proxy_async_smem();
        mbar_arrive_warp(bar_v_clean + 8 * st);
      }
    } else {
      // ================================================================ codes -> fp16 tiles
      const int n_pages = pages_of(s.len, a.PT), p_first = it.k0 / a.PT, p_end = it.see > it.k0 ? (it.see - 1) / a.PT + 1 : p_first;
      // the largest value scale of the keys, in which the values are taken
      float most = 1.17549435e-38f;
      for (int p = p_first + tid; p < p_end; p += 128) most = fmaxf(most, a.vs[static_cast<int64_t>(page_of(a, it.b, p)) * a.KV + it.kvh]);
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, w));
      if (lane == 0) unit_s[warp - kMoveWarp] = most;
      named_barrier_sync(1, 128);
      most = fmaxf(fmaxf(unit_s[0], unit_s[1]), fmaxf(unit_s[2], unit_s[3]));
      // Units of work: K(0), then K(j + 1) and V(j) in turn.  While one is converted the codes of the next are on their way, and those of the one after it are asked
      // for piece by piece, where its own have been used.
      constexpr int TPR = D / 16, RPP = 128 / TPR, PASSES = 128 / RPP;           // threads a row, rows a pass
      const int c = tid % TPR, r0 = tid / TPR;
      int window = -64, window_page = 0;
      __half2 nan_seen = __float2half2_rn(0.f);
      const int units = 2 * nt + 1;                                // (K(nt) is none)
      struct Unit {
        bool there, is_v, full;
        int j, left;                                               // its tile; rows of it that are seen
        const uint8_t *at0, *at1;                                  // this thread's codes in the first and the second 64 rows
        float2 scale;
      };
      auto find = [&](int u) {
        Unit w;
        w.is_v = u > 0 && (u & 1) == 0;
        w.j = u == 0 ? 0 : w.is_v ? u / 2 - 1 : (u + 1) / 2;
        w.there = u < units && w.j < nt;
        w.scale = make_float2(0.f, 0.f);
        w.at0 = w.at1 = nullptr;
        w.left = 0;
        if (w.there) {
          const int key0 = it.k0 + w.j * kKeys;
          w.left = it.see - key0;
          const int p0 = key0 / a.PT, p1 = a.PT == 64 && w.left > 64 ? p0 + 1 : p0;
          if (p1 - window >= 32 || window < 0 || p0 < window) {
            window = p0;
            window_page = p0 + lane < n_pages ? page_of(a, it.b, p0 + lane) : 0;
          }
          const int64_t at0 = static_cast<int64_t>(__shfl_sync(0xffffffffu, window_page, p0 - window)) * a.KV + it.kvh;
          const int64_t at1 = static_cast<int64_t>(__shfl_sync(0xffffffffu, window_page, p1 - window)) * a.KV + it.kvh;
          const uint8_t* codes = w.is_v ? a.vc : a.kc;
          const float* scales = w.is_v ? a.vs : a.ks;
          w.scale = make_float2(scales[at0], scales[at1]);
          w.at0 = codes + at0 * a.PT * D + tid * 16;
          w.at1 = a.PT == 64 ? codes + at1 * a.PT * D + tid * 16 - 64 * D : w.at0;
        }
        return w;
      };
      auto ask = [&](const Unit& w, int p) {                       // RPP rows x D codes are 2048 bytes
        const uint8_t* at = (p < PASSES / 2 ? w.at0 : w.at1) + p * 2048;
        return w.there && p * RPP + r0 < w.left ? __ldcg(reinterpret_cast<const uint4*>(at)) : make_uint4(0u, 0u, 0u, 0u);
      };
      auto convert = [&](const Unit& w, uint4 (&raw)[PASSES], const Unit& next) {
        if (!w.there) return true;                                 // (K(nt) only: behind it there is V(nt - 1), which has been asked for)
        const int st = w.is_v ? w.j % SV : w.j % SK, n = w.is_v ? SV : SK;
        const uint32_t full = (w.is_v ? bar_v_full : bar_k_full) + 8 * st, empty = (w.is_v ? bar_v_empty : bar_k_empty) + 8 * st;
        if (w.j >= n && !mbar_wait_warp<kIssueWaitHintNs>(empty, (w.j / n - 1) & 1, abort_flag, a.status)) return false;
        const uint32_t tile = sbase + (w.is_v ? SM::v_off : SM::k_off) + st * SM::q_tile;
        const float f0 = w.is_v ? w.scale.x / most : 1.f, f1 = w.is_v ? w.scale.y / most : 1.f;
        // (2^-126 is the scale of a page of zeros)
        if ((f0 < kLeastShare && w.scale.x > 1.17549435e-38f) || (f1 < kLeastShare && w.scale.y > 1.17549435e-38f)) spoilt = true;
        const __half2 h0 = __float2half2_rn(f0), h1 = __float2half2_rn(f1);
        const int first = D == 128 ? c >> 2 : 0;                   // which of its two pieces a thread stores first: eight lanes, eight banks
        auto pass = [&](int p, auto look) {
          uint32_t o[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) e4m3x4_to_half2((&raw[p].x)[e], o[2 * e], o[2 * e + 1]);
          raw[p] = ask(next, p);
          if (decltype(look)::value) {
            const __half2 f = p < PASSES / 2 ? h0 : h1;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              __half2& h = *reinterpret_cast<__half2*>(&o[e]);
              nan_seen = __hmax2_nan(nan_seen, h);
              h = __hmul2(h, f);
            }
          }
          const int row = p * RPP + r0;
          const uint4 lo = make_uint4(o[0], o[1], o[2], o[3]), hi = make_uint4(o[4], o[5], o[6], o[7]);
          sts128(tile + tile_at16(row, 2 * c + first), first ? hi : lo);
          sts128(tile + tile_at16(row, 2 * c + 1 - first), first ? lo : hi);
        };
        // Most tiles are seen by all rows, so that NaN codes go where they have to, and most pages have the largest scale
        if (w.j < clean_from && f0 == 1.f && f1 == 1.f) {
#pragma unroll
          for (int p = 0; p < PASSES; ++p) pass(p, std::false_type{});
        } else {
#pragma unroll
          for (int p = 0; p < PASSES; ++p) pass(p, std::true_type{});
        }
        if (!w.is_v && tid == 0)
          asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(sbase + SM::scale_off + (w.j & 7) * 8), "f"(w.scale.x), "f"(w.scale.y) : "memory");
        fence_proxy_async_smem();
        mbar_arrive_warp(full);
        return true;
      };
      if (nt > 0) {
        uint4 ra[PASSES], rb[PASSES];
        Unit ua = find(0), ub = find(1);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) ra[p] = ask(ua, p);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) rb[p] = ask(ub, p);
        for (int u = 0; u < units; u += 2) {
          const Unit na = find(u + 2);
          if (!convert(ua, ra, na)) break;
          ua = na;
          const Unit nb = find(u + 3);
          if (!convert(ub, rb, nb)) break;
          ub = nb;
        }
      }
      spoilt |= __hisnan(__low2half(nan_seen)) || __hisnan(__high2half(nan_seen));
    }
    if (spoilt) *spoilt_s = 1;
  } else {
    // ================================================================== soft-max of query tile t, a thread a row
    set_regs<ManyRoles<D>::kSoftmax>();
    const int t = warp >> 2, n = it.nt[t];
    constexpr int PPR = D / 8, RPI = 32 / PPR;                     // 16-byte pieces a row, rows that a warp reads or writes at once
    struct Row {
      int r, i, head;                                              // row of the sequence, its token and query head
      bool live;
    };
    // (asked for before and after the loop, so that it does not live through it)
    auto row_of = [&](int at) {
      asm volatile("" : "+r"(at));
      Row w;
      w.r = it.row0 + at;
      w.live = w.r < it.rows;
      w.i = w.live ? w.r / a.G : 0;
      w.head = it.kvh * a.G + (w.live ? w.r - w.i * a.G : 0);
      return w;
    };
    const uint32_t lane_t = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_t = lane_t + t * 128, o_t = lane_t + 256 + t * D;
    float factor = rsqrtf(static_cast<float>(D)) * 1.4426950408889634f;
    int end;                                                       // of the keys that this thread's row sees, from the part's first on
    // ---- this warp's 32 queries, PPR lanes a row
    {
      const Row w = row_of(threadIdx.x);
      const bool live = w.live;
      end = live ? visible_end(it.past + w.i, s.len, a.frame) - it.k0 : 0;
      const int my_row = lane / PPR, piece = lane % PPR;
      const T* mine = static_cast<const T*>(a.q) + w.head * a.q_hs + (s.t0 + w.i) * a.q_ts;
      const uint32_t tile = sbase + t * SM::q_tile;
      const unsigned lives = __ballot_sync(0xffffffffu, live);
      auto from = [&](int r2) { return reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), r2)) + piece * 8; };
      if constexpr (!PAGED) {
#pragma unroll 4
        for (int p = 0; p < PPR; ++p) {
          const int r2 = p * RPI + my_row;
          cp_async16(tile + tile_at16((warp & 3) * 32 + r2, piece), from(r2), (lives >> r2) & 1);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
      } else {
        const float scale = factor;
#pragma unroll 1
        for (int p0 = 0; p0 < PPR; p0 += 4) {
          uint4 v[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const int r2 = (p0 + p) * RPI + my_row;
            const T* src = from(r2);
            v[p] = (lives >> r2) & 1 ? __ldcg(reinterpret_cast<const uint4*>(src)) : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = widen2<T>((&v[p].x)[e]);
              most = max(most, max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu));
            }
#pragma unroll
            for (int w = 1; w < PPR; w <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, w));
            int e = static_cast<int>(most >> 23) - 127;
            e = most == 0 ? 0 : e == 128 ? 113 : max(-126, min(126, e));        // (a row that is not finite: its finite numbers stay so, 2^15 at most)
            const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23), up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * scale;
            // what the row was divided by goes to the thread that has it
            const float theirs = __shfl_sync(0xffffffffu, up, lane % RPI * PPR);
            if (lane / RPI == p0 + p) factor = theirs;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float2 f = widen2<T>((&v[p].x)[w]);
              (&v[p].x)[w] = narrow2<__half>(f.x * down, f.y * down);
            }
            sts128(tile + tile_at16((warp & 3) * 32 + (p0 + p) * RPI + my_row, piece), v[p]);
          }
        }
      }
      fence_proxy_async_smem();
      mbar_arrive_warp(bar_q);
    }
    float m = -INFINITY;
    float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    bool ok = true;
    for (int i2 = 0; i2 < NS * n; ++i2) {                          // the h-th kSub keys of tile j
      const int j = i2 / NS, h = i2 % NS;
      const uint32_t at = 16 * t + 8 * h;
      ok = ok && mbar_wait_warp(bar_s + at, j & 1, abort_flag, a.status);
      if (!ok) break;
      tc_fence_after();
      uint32_t x[kSub / 32][32];
#pragma unroll
      for (int q = 0; q < kSub / 32; ++q) tmem_ld32(s_t + kSub * h + 32 * q, x[q]);
      float f[2] = {factor, factor};                               // of the first and the second 64 keys of those
      if (PAGED) {
        float2 ks;
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(ks.x), "=f"(ks.y) : "r"(sbase + SM::scale_off + (j & 7) * 8));
        f[0] = logit_factor(factor, a.PT == 64 && NS == 2 && h == 1 ? ks.y : ks.x);
        f[1] = logit_factor(factor, a.PT == 64 ? ks.y : ks.x);
      }
      tmem_wait_ld();
      if (!kOver) {
        tc_fence_before();
        mbar_arrive_warp(bar_ld + at);
      }
      if (j >= it.whole_from[t]) {
        const int valid = end - i2 * kSub;
#pragma unroll
        for (int q = 0; q < kSub / 32; ++q)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (q * 32 + e >= valid) x[q][e] = 0xFF800000u;
      }
      float top;
#pragma unroll
      for (int h2 = 0; h2 < kSub / 64; ++h2) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t* y = &x[2 * h2 + (q >> 1)][16 * (q & 1)];
          v[q] = fmax3_nan(__uint_as_float(y[0]), __uint_as_float(y[1]), __uint_as_float(y[2]));
#pragma unroll
          for (int e = 3; e < 15; e += 2) v[q] = fmax3_nan(v[q], __uint_as_float(y[e]), __uint_as_float(y[e + 1]));
        }
        v[0] = fmax3_nan(v[0], __uint_as_float(x[2 * h2][15]), __uint_as_float(x[2 * h2][31]));
        v[1] = fmax3_nan(v[1], __uint_as_float(x[2 * h2 + 1][15]), __uint_as_float(x[2 * h2 + 1][31]));
        const float w = fmax3_nan(fmax3_nan(v[0], v[1], v[2]), v[3], v[3]) * f[h2];
        top = h2 ? fmax3_nan(top, w, w) : w;
      }
      // P V of the same keys of the tile before is over: P lies where its probabilities were
      if (!kOver && j > 0) {
        ok = mbar_wait_warp(bar_pv + at, (j - 1) & 1, abort_flag, a.status);
        if (!ok) break;
        tc_fence_after();
      }
      const bool raise = !(top <= m + (kRaise + kLift));           // (at first m is -inf; a logit that is no number makes m, and with it all, none)
      if (__any_sync(0xffffffffu, raise)) {
        const float to = raise ? top - kLift : m, alpha = to == m ? 1.f : m == -INFINITY ? 0.f : fast_exp2(m - to);
        m = to;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          l[q].x *= alpha;
          l[q].y *= alpha;
        }
        if (i2 > 0) {                                              // O follows, once the keys before have been added to it
          ok = mbar_wait_warp(bar_pv + 16 * t + 8 * ((i2 - 1) % NS), ((i2 - 1) / NS) & 1, abort_flag, a.status);
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int q = 0; q < D / 16; ++q) {
            uint32_t y[16];
            tmem_ld16(o_t + q * 16, y);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * alpha);
            tmem_st16(o_t + q * 16, y);
          }
        }
      }
      const float ref = fabsf(m) < INFINITY ? -m : m == -INFINITY ? 0.f : __int_as_float(0x7FC00000);
      const float2 rr = make_float2(ref, ref);
#pragma unroll
      for (int h2 = 0; h2 < kSub / 64; ++h2) {
        const float2 ff = make_float2(f[h2], f[h2]);
        uint32_t p[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const uint32_t* y = &x[2 * h2 + (e >> 4)][2 * (e & 15)];
          const float2 u = ffma2(make_float2(__uint_as_float(y[0]), __uint_as_float(y[1])), ff, rr);
          const float2 pr = e % 16 < kPoly<PAGED> ? poly_exp2(u) : make_float2(fast_exp2(u.x), fast_exp2(u.y));
          p[e] = narrow2<M>(pr.x, pr.y);
          if (kHalf) add_f16x2(l[e & 1], p[e]);
          else add_bf16x2(l[e & 1], p[e]);
        }
        tmem_st32(kOver ? s_t + 64 * h : lane_t + 384 + t * 64 + 32 * h2, p);
      }
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive_warp(bar_p + at);
    }
    // ---- the row's end
    if (ok && n > 0) ok = mbar_wait_warp(bar_pv + 16 * t + 8 * (NS - 1), (n - 1) & 1, abort_flag, a.status);      // (in order: the other half is over too)
    tc_fence_after();
    const float sum = (l[0].x + l[0].y) + (l[1].x + l[1].y);
    float unit = 1.f;
    if (PAGED && n > 0) unit = fmaxf(fmaxf(unit_s[0], unit_s[1]), fmaxf(unit_s[2], unit_s[3]));
    const Row w = row_of(threadIdx.x);
    const bool live = w.live;
    const int tok = s.t0 + w.i, row = threadIdx.x;
    const int64_t part_row = (static_cast<int64_t>(it.part) * a.T + tok) * a.H + w.head;
    const float inv = whole ? (sum == 0.f ? 0.f : unit / sum) : unit;
    T* out = static_cast<T*>(a.out) + w.head * a.q_hs + tok * a.q_ts;
    // At d = 128 rows go through the place of the warp's queries, D 16-bit columns (half as many 32-bit ones) at a time, so that a store writes whole rows (30 prompts of
    // 300 tokens 66.9 -> 64.6 us).  At 64, where a row is 128 bytes, the same costs the loop above more than it saves here (16 384 tokens 369 -> 397 us).
    if (D == 64 && ok && n > 0) {
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t v[32];
        tmem_ld32(o_t + c0, v);
        tmem_wait_ld();
        if (!live) continue;
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = sum == 0.f ? 0u : __float_as_uint(__uint_as_float(v[e]) * inv);
        if (whole) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint4 o;
#pragma unroll
            for (int w = 0; w < 4; ++w) (&o.x)[w] = narrow2<T>(__uint_as_float(v[8 * e + 2 * w]), __uint_as_float(v[8 * e + 2 * w + 1]));
            *reinterpret_cast<uint4*>(out + c0 + 8 * e) = o;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) *reinterpret_cast<uint4*>(a.part_o + part_row * D + c0 + 4 * e) = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        }
      }
    }
    if (D == 128 && ok && n > 0) {
      const uint32_t tile = sbase + t * SM::q_tile;
      const int my_row = lane / PPR, piece = lane % PPR;
      const unsigned lives = __ballot_sync(0xffffffffu, live);
      uint8_t* mine = whole ? reinterpret_cast<uint8_t*>(out) : reinterpret_cast<uint8_t*>(a.part_o + part_row * D);
#pragma unroll 1
      for (int half = 0; half < (whole ? 1 : 2); ++half) {
#pragma unroll 1
        for (int c0 = 0; c0 < (whole ? D : D / 2); c0 += 32) {
          uint32_t v[32];
          tmem_ld32(o_t + half * (D / 2) + c0, v);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = sum == 0.f ? 0u : __float_as_uint(__uint_as_float(v[e]) * inv);
          if (whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint4 o;
#pragma unroll
              for (int w = 0; w < 4; ++w) (&o.x)[w] = narrow2<T>(__uint_as_float(v[8 * e + 2 * w]), __uint_as_float(v[8 * e + 2 * w + 1]));
              sts128(tile + tile_at16(row & 127, c0 / 8 + e), o);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) sts128(tile + tile_at16(row & 127, c0 / 4 + e), make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]));
          }
        }
        __syncwarp();
#pragma unroll 4
        for (int p = 0; p < PPR; ++p) {
          const int r2 = p * RPI + my_row;
          uint8_t* to = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), r2)) + half * (D * 2) + piece * 16;
          uint4 o;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(o.x), "=r"(o.y), "=r"(o.z), "=r"(o.w) : "r"(tile + tile_at16((warp & 3) * 32 + r2, piece)));
          if ((lives >> r2) & 1) *reinterpret_cast<uint4*>(to) = o;
        }
        __syncwarp();
      }
    }
    if (ok && !whole && live) a.part_ml[part_row] = make_float2(m, sum);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (*spoilt_s && warp < kMoveWarp) {
    const int last = min(it.rows, it.row0 + kRowsCta);
    for (int r = it.row0 + warp; r < last; r += kMoveWarp) {
      const int tok = s.t0 + r / a.G, head = it.kvh * a.G + r % a.G;
      const int64_t part_row = (static_cast<int64_t>(it.part) * a.T + tok) * a.H + head;
      dense_row_to<T, D, PAGED>(a, it.b, tok, head, s, it.k0, whole ? s.len : it.k0 + a.chunk, whole, a.part_o + part_row * D, a.part_ml + part_row);
    }
  }
}

int launch_dense_many(const DenseArgs& a, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int D, bool fp16, cudaStream_t st) {
  // the sequences' last tiles are less than one each
  const int64_t tiles = static_cast<int64_t>(a.T) * a.G / kRowsCta + (a.B < a.T ? a.B : a.T), ctas = tiles * a.KV;
  if (ctas > INT32_MAX || a.parts > 65535) return FASTAR_ERR_UNSUPPORTED_SHAPE;
  using Kern = void (*)(CUtensorMap, CUtensorMap, DenseArgs);
  Kern kern;
  if (a.kc) kern = fp16 ? (D == 128 ? many_kernel<__half, 128, true> : many_kernel<__half, 64, true>)
                        : (D == 128 ? many_kernel<__nv_bfloat16, 128, true> : many_kernel<__nv_bfloat16, 64, true>);
  else kern = fp16 ? (D == 128 ? many_kernel<__half, 128, false> : many_kernel<__half, 64, false>)
                   : (D == 128 ? many_kernel<__nv_bfloat16, 128, false> : many_kernel<__nv_bfloat16, 64, false>);
  const int smem = D == 128 ? ManySmem<128>::total : ManySmem<64>::total;
  const int r = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
  if (r != FASTAR_OK) return r;
  return launch_chained(kern, dim3(static_cast<unsigned>(ctas), a.parts), kManyThreads, smem, st, tm_k, tm_v, a) == cudaSuccess ? FASTAR_OK : FASTAR_ERR_CUDA;
}

}  // namespace fastar
