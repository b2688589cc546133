// Backward pass of attention for gfx950: dq, dk and dv, the probabilities recomputed.
//
//   P = exp(S - lse), S = scale Q K^T     dS = P (dO V^T - delta), delta_i = dO_i . O_i
//   dV = P^T dO      dK = scale dS^T Q    dQ = scale dS K
//
// Two kernels share the work: one owns keys and streams queries (dK, dV: four products), one
// owns queries and streams keys (dQ: three products, and a fourth for its accuracy, see there).
// One kernel for all would need five products instead of eight, but would have to add every
// workgroup's part of dQ in memory: 64 KiB of fp32 atomics for each 21 MFLOP, in an order that
// changes from run to run.  Two kernels' sums are always in the same order.
//
// The dense kernels run their products at the rate of a large library product, so what bounds them is
// the power that products and LDS reads draw (1 KiB of operand per MFMA, 3/4 in the dq kernel, where
// two products share an operand: 4 % faster than reading it for each; the other operand stays in
// registers).  Instruction order is fixed by fences: operands are read two MFMAs ahead, exponentials
// run under the dP products, dS under the dV products (P K in the dq kernel).
// N = 32760, 10 heads: 18.1-18.3 ms, 750-759 TFLOP/s of the five products the mathematics needs and
// 1200-1215 of the eight computed; a large library product reached 1209-1223 on the same card.
// The dk, dv kernel's loops hold more waits than they need: its own rows, loaded before the loop, count
// as pending at every entry, so a block's first products wait for the next tile's loads; and without
// a bias its tile offset is spilled and read back before each tile's loads.  Its waves wait on 32 % of
// their cycles, those of the dq kernel on 19 %.

#include "attn_bwd_launch.h"
#include "attn_tiles.h"

#include <type_traits>

namespace dsattn {
namespace {

constexpr int kMaxTiles = 4096;   // 64-row tiles that a visit list can hold

// ---- visit lists -------------------------------------------------------------------------

// What a workgroup visits, in order: tiles of the streamed axis that have an open pair, and for
// each of them keep bit 4 b + x: 32-row half b of the tile and own 32-row block x (that of
// wave x) have one.
struct VisitList {
  uint16_t tile[kMaxTiles];
  uint8_t bits[kMaxTiles];
  int count;
};

// Whether the 32 x 32 block of query block qb and key block kb has an open pair.
__device__ __forceinline__ bool block_open(const BwdParams& p, int bh, int qb, int kb) {
  if (32 * qb >= p.n_q || 32 * kb >= p.n_k) return false;
  const int u = 32 * qb / p.tile_q, d = 32 * kb / p.tile_k;
  return p.mask[((size_t)bh * p.n_units + u) * p.n_dec + d] == 0;
}

// Fill the list: own 32-row blocks own0 .. own0 + 3, streamed tiles 0 .. n_tiles - 1.
// Q_OWN: the own blocks are query blocks, the tiles key tiles.
template <bool Q_OWN>
__device__ __forceinline__ void build_list(VisitList& list, const BwdParams& p, int bh, int own0,
                                           int n_tiles) {
  const int tid = threadIdx.x, lane = tid & 63;
  // eight threads a tile note its bits in place, four tiles at a time for their loads' sake, then
  // the first wave closes the gaps in order
  constexpr int kStep = kThreads / 8;
  for (int t0 = tid >> 3; t0 < n_tiles; t0 += 4 * kStep) {
    bool open[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = t0 + u * kStep, j = tid & 7, b = 2 * t + (j >> 2), x = own0 + (j & 3);
      open[u] = t < n_tiles && (Q_OWN ? block_open(p, bh, x, b) : block_open(p, bh, b, x));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = t0 + u * kStep;
      const uint32_t bits = (uint32_t)(__ballot(open[u]) >> (lane & 56)) & 0xffu;
      if ((tid & 7) == 0 && t < n_tiles) list.bits[t] = (uint8_t)bits;
    }
  }
  __syncthreads();
  if (tid < 64) {
    int n = 0;
    for (int t0 = 0; t0 < n_tiles; t0 += 64) {
      const int t = t0 + lane;
      const uint32_t bits = t < n_tiles ? list.bits[t] : 0u;
      const uint64_t have = __ballot(bits != 0);
      const int at = n + __popcll(have & ((1ull << lane) - 1ull));
      if (bits != 0) {   // at <= t, and the whole wave has read its 64 tiles
        list.tile[at] = (uint16_t)t;
        list.bits[at] = (uint8_t)bits;
      }
      n += __popcll(have);
    }
    if (lane == 0) list.count = n;
  }
  __syncthreads();
}

// ---- position bias -----------------------------------------------------------------------

// What a wave's two 32 x 32 blocks of a tile lie in, by ascending distance: run[j] as a word of
// runs, but with the position counted from the tile's smallest distance, and the value at the
// block's first query and key.  A block's 63 distances begin in word m (m + 1 for the second) of
// the tile's words and end at most two words on; what lies in them beyond the block may make it
// count as less even than it is, which costs time only.  start: distance index of word 0 (at or
// below the tile's smallest); flat[b] is read from value[step b].
struct TileRuns {
  int run[2];
  float flat[2];
  __device__ __forceinline__ void read(const int32_t (&runs)[64], int m, int start, const float* value,
                                       int step) {
    int x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_readfirstlane(runs[m + j]);
    const float f = value[0];
    flat[0] = flat[1] =
        __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, f)));
    run[0] = run[1] = x[0];
    if (x[0] == x[1] && x[0] == x[2] && x[0] == x[3] && !is_step(x[0])) return;   // nearly always
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int steps = 0, cut = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int y = x[j + i], at = 32 * (m + j + i) + start;
        if (y == kRunMixed) steps = 2;
        if (is_step(y)) {
          steps += 1;
          cut = at + run_pos(y);
        }
        if (i < 2 && run_last(y) != run_first(x[j + i + 1])) {
          steps += 1;
          cut = at + 32;
        }
      }
      run[j] = steps == 0   ? x[j]
               : steps == 1 ? run_step(run_first(x[j]), run_last(x[j + 2]), max(cut, 0))
                            : (int)kRunMixed;
      flat[j] = __builtin_bit_cast(
          float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, value[step * j])));
    }
  }
};

// Whether a run is one bucket (or closed) throughout.
__device__ __forceinline__ bool is_flat(int run) { return run != kRunMixed && !is_step(run); }

// Sum over a wave, in every lane.  (Data-parallel moves within the vector unit: the shuffles'
// way through LDS takes ten times as long.)
__device__ __forceinline__ float wave_sum(float x) {
  auto add = [&](auto ctrl, auto rows) {
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x),
                                                               decltype(ctrl)::value,
                                                               decltype(rows)::value, 0xf, false));
  };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr 1
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast 31
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// ---- dk, dv ------------------------------------------------------------------------------

// What a workgroup's LDS holds besides tiles.
struct NoList {};
struct DkvBias {
  alignas(16) float win[2][kWindow];       // bias / scale
  alignas(16) int32_t bucket[2][kWindow];
  int32_t runs[2][64];
  float bins[kWaves][kMaxBuckets];         // sums over buckets
  float closed[32];                        // -inf, read by lanes whose key does not exist
  int ends[2];   // of the open runs, see open_tiles
};
struct DqBias {
  alignas(16) float win[2][kWindow];
  f32x4 sums[kThreads];   // see flush_sums
  int32_t runs[2][64];
  int ends[2];   // of the open runs, see open_tiles
};
template <int MODE, typename BIAS>
struct SideOf {
  typedef VisitList type;
};
template <typename BIAS>
struct SideOf<kBwdDense, BIAS> {
  typedef NoList type;
};
template <typename BIAS>
struct SideOf<kBwdBias, BIAS> {
  typedef BIAS type;
};

template <int MODE>
struct DkvSmem {
  alignas(16) uint16_t q[2][kTileElems];
  alignas(16) uint16_t g[2][kTileElems];   // dO
  alignas(16) float nl[2][kTile];
  alignas(16) float nd[2][kTile];
  typename SideOf<MODE, DkvBias>::type side;
};

// The bias of a 32 x 32 block: the run it lies in, its value there, and where the single values
// of a mixed block begin.
struct BlockBias {
  int run;
  float flat;
  const float* win;   // of the block's smallest distance
  int first;          // the same, counted from the tile's
};

__device__ __forceinline__ void lds_add(float* p, float x) {
  __hip_atomic_fetch_add(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// Sums of a 32 x 32 block over its diagonals: lane l gets that of the block's l-th smallest
// column - row distance.  Row after row is added to what came before, moved on by one lane, so
// that row i ends 31 - i lanes on.  (32 additions that read their neighbour's lane.  Adding up in
// LDS took 16 atomics of a wave, some 200 cycles each.)
__device__ __forceinline__ float diagonal_sums(const f32x16& s) {
  float x = 0.f;
  const auto add = [&](uint32_t row) {   // 0x138: a lane reads the one below, the first reads 0
    x = __builtin_bit_cast(float, row) +
        __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x138,
                                                              0xf, 0xf, true));
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t upper[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      // rows of 32 lanes each in 64: 8 i + t, then 8 i + 4 + t
      const float y = s[4 * i + t];   // (a bit cast of the element itself takes the vector's first)
      const auto sw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, y), 0u, false,
                                                       false);
      add(sw[0]);
      upper[t] = sw[1];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) add(upper[t]);
  }
  return x;
}

// Register v's row, 8 (v / 4) + v % 4, counted back from the last one's.
__device__ __forceinline__ constexpr int back(int v) { return 27 - 8 * (v >> 2) - (v & 3); }

// A workgroup owns 128 keys, a wave 32 of them, and streams the queries in tiles of 64.  Per 32
// queries: S = Q K^T and dP = dO V^T with keys as columns, so that
// P and dS are B operands of dV^T += dO^T P and dK^T += Q^T dS.
template <int MODE>
__device__ __forceinline__ void dkv_block(DkvSmem<MODE>& sm, int buf, int b, uint32_t row_at,
                                          uint32_t col_at, const bf16x8 (&kf)[8],
                                          const bf16x8 (&vf)[8], f32x16 (&dk)[4],
                                          f32x16 (&dv)[4], float c, int lane, int w, bool there,
                                          const BlockBias& bias, float& all, float& below) {
  const uint32_t q_at = lds_addr(sm.q), g_at = lds_addr(sm.g);
  const uint32_t block = (uint32_t)(buf * kTileElems * 2 + b * 32 * kRowBytes);
  const int g = lane >> 5;
  f32x16 s = f32x16{}, dp, nd;
  if constexpr (MODE == kBwdBias) {
    if (!is_flat(bias.run)) {
      const int l = lane_now();
      const float* win = there ? bias.win + 4 + (l & 31) - 4 * (l >> 5) : sm.side.closed;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = win[back(v)];
      asm volatile("" : "+v"(s));   // put in order here, not where both ways meet
    } else {
      const float flat = there ? bias.flat : neg_inf();
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = flat;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(&sm.nd[buf][32 * b + 8 * i + 4 * g]);
#pragma unroll
    for (int t = 0; t < 4; ++t) nd[4 * i + t] = x[t];
  }
  // -lse of registers 4 i .. 4 i + 3, read shortly before their exponentials
  f32x4 nl[4];
  auto rows = [&](int i) {
    nl[i] = *reinterpret_cast<const f32x4*>(&sm.nl[buf][32 * b + 8 * i + 4 * g]);
  };
  // A operands in the order of their products: S, dP, dV, dK (eight each)
  auto operand = [&](int i) {
    if (i < 16) return row_operand(row_at, block, i < 8 ? q_at : g_at, i & 7);
    return col_operand(col_at, block, i < 24 ? g_at : q_at, (i & 7) >> 2, i & 3);
  };
  bf16x8 pf[2], df[2];
  auto prob = [&](int v) {
    s[v] = exp2_fast(fmaf(s[v], c, nl[v >> 2][v & 3]));
    pf[v >> 3][v & 7] = (__bf16)s[v];
  };
  auto grad = [&](int v) {
    const float x = s[v] * dp[v];
    df[v >> 3][v & 7] = (__bf16)x;
    if constexpr (MODE == kBwdBias) s[v] = x;
  };
  constexpr int RK = 3;
  bf16x8 a[RK];
#pragma unroll
  for (int i = 0; i < RK - 1; ++i) a[i] = operand(i);
  sched_fence();
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (i + RK - 1 < 32) a[(i + RK - 1) % RK] = operand(i + RK - 1);
    const bf16x8& x = a[i % RK];
    if (i < 8)
      s = mfma(x, kf[i], s);
    else if (i < 16)
      dp = mfma(x, vf[i - 8], i == 8 ? nd : dp);
    else if (i < 24)
      dv[i & 3] = mfma(x, pf[(i & 7) >> 2], dv[i & 3]);
    else
      dk[i & 3] = mfma(x, df[(i & 7) >> 2], dk[i & 3]);
    // 3/4 of the exponentials under the dP products, the rest under the first dV products
    // (which do not read them yet), dS under the dV products
    if (i == 7 || i == 8 || i == 11 || i == 14) rows(i < 9 ? i - 7 : i / 3 - 1);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (i >= 9 && i < 15) prob((i - 9) * 2 + e);
      if (i >= 16 && i < 20 && e < 1) prob(i - 4);
      if (i >= 16 && i < 24) grad((i - 16) * 2 + e);
    }
    // dS in 32 bits, now in s: its sum under the dK products
    if constexpr (MODE == kBwdBias) {
      if (i == 24) all = s[0] + s[1];
      if (i > 24) all += s[2 * (i - 24)] + s[2 * (i - 24) + 1];
    }
    sched_fence();
  }
  __builtin_amdgcn_s_setprio(0);
  // of a mixed block its sums by distance instead, of one with a step the parts above and below it
  if constexpr (MODE == kBwdBias) {
    if (is_step(bias.run)) {
      // (not one of them as a difference: where a part's dS are zeros, so is its sum)
      const int l = lane_now(), cut = run_pos(bias.run) - bias.first - 4 - (l & 31) + 4 * (l >> 5);
      all = below = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        below += back(v) < cut ? s[v] : 0.f;
        all += back(v) < cut ? 0.f : s[v];
      }
    } else if (bias.run == kRunMixed) {
      all = diagonal_sums(s);
    }
  }
}

// Sum over block elements of one bucket that is not in the bins yet: blocks come by descending
// distance, so most have the bucket of the one before.  A lane's part is a sum of block sums of 16,
// the bins take sums of at most 64 blocks: errors grow with the root of each count.
struct FarSum {
  int run = kRunClosed;
  float x = 0.f;
  __device__ __forceinline__ static void put(float* bins, int run, float x) {
    const float total = wave_sum(x);
    if (lane_now() == 0 && run >= 0) lds_add(&bins[run], total);
  }
  __device__ __forceinline__ void flush(float* bins) {
    put(bins, run, x);
    run = kRunClosed;
    x = 0.f;
  }
  // One block's sum, or its sums above and below its step.
  __device__ __forceinline__ void add(float* bins, int block, float all, float below) {
    if (block != run) {   // seldom
      const int high = run_last(block);
      if (high != run) {
        flush(bins);
        run = high;
      }
      if (is_step(block)) put(bins, run_first(block), below);
    }
    x += all;
  }
};

// Add a mixed block's sums by distance, x, to their buckets.  A bucket that many of the distances
// share is summed up first: atomics on one address wait for each other.
__device__ __forceinline__ void add_by_distance(float x, const int32_t* bucket, float* bins,
                                                int n_buckets) {
  const int lane = lane_now();
  int at = bucket[lane];
  if (lane == 63 || (uint32_t)at >= (uint32_t)n_buckets) at = kRunClosed;
  // the ends of the range are where wide buckets are
#pragma unroll
  for (int end = 0; end < 2; ++end) {
    const int wide = __builtin_amdgcn_readlane(at, end == 0 ? 0 : 62);
    if (wide >= 0 && __popcll(__ballot(at == wide)) >= 8) {
      const float total = wave_sum(at == wide ? x : 0.f);
      if (lane == 0) lds_add(&bins[wide], total);
      if (at == wide) at = kRunClosed;
    }
  }
  if (at >= 0) lds_add(&bins[at], x);
}

template <int MODE>
__global__ __launch_bounds__(kThreads, 2) void bwd_dkv_kernel(BwdParams p) {
  __shared__ DkvSmem<MODE> sm;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = blockIdx.x;
  const Place at = place_of(p.dkv_split, MODE == kBwdBias, p.dkv_split.unit(x), p.bh,
                            (p.n_k + 127) / 128, false);
  const int bh = at.bh, key0 = at.group * 128;
  const int n_tiles = (p.n_q + kTile - 1) / kTile;
  const size_t qoff = (size_t)bh * p.n_q * kD, koff = (size_t)bh * p.n_k * kD;
  const auto qrs = row_buffer(p.q + qoff, p.n_q), grs = row_buffer(p.dout + qoff, p.n_q);
  const auto lrs = word_buffer(p.neg_lse2 + (size_t)bh * p.n_rows, p.n_rows);
  const auto drs = word_buffer(p.neg_delta + (size_t)bh * p.n_rows, p.n_rows);
  const uint32_t row_at = row_lane(r, g), col_at = col_lane(lane);
  const auto first_distance = [&](int t) { return key0 - (t * kTile + 63) + p.n_q - 1; };
  const auto wrs = word_buffer(p.bias.by_dist + (size_t)(MODE == kBwdBias ? bh % p.H : 0) * p.bias.dist_stride, p.bias.n_dist);
  const auto brs = word_buffer(p.bias.bucket, p.bias.n_dist), rrs = word_buffer(p.bias.runs, p.bias.n_runs);

  const uint32_t off = tile_lane_offset(w, lane);
  auto fetch = [&](int buf, int t) {
    const int l = MODE == kBwdBias ? lane_now() : lane;
    const uint32_t at = MODE == kBwdBias ? tile_lane_offset(w, l) : off;
    load_tile(sm.q[buf], qrs, at, t * kTile, w);
    load_tile(sm.g[buf], grs, at, t * kTile, w);
    if (w == 0) load_words(sm.nl[buf], lrs, t * kTile, l);
    if (w == 1) load_words(sm.nd[buf], drs, t * kTile, l);
    if constexpr (MODE == kBwdBias) {
      const int e = first_distance(t);
      if (w < 3) load_words(sm.side.win[buf] + 64 * w, wrs, e + 64 * w, l);
      if (w > 0) load_words(sm.side.bucket[buf] + 64 * (w - 1), brs, e + 64 * (w - 1), l);
      if (w == 3) load_words(sm.side.runs[buf], rrs, e >> 5, l);
    }
  };

  bf16x8 kf[8], vf[8];
  int key = key0 + w * 32 + r;
  load_row(kf, p.k + koff, key, key < p.n_k, g);
  load_row(vf, p.v + koff, key, key < p.n_k, g);

  int count = n_tiles, first = 0;
  if constexpr (MODE == kBwdMask) {
    build_list<false>(sm.side, p, bh, key0 / 32, n_tiles);
    count = sm.side.count;
  }
  if constexpr (MODE == kBwdBias) {
    const TileRange open = open_tiles<-1>(sm.side.ends, p.bias.runs, p.bias.n_runs, n_tiles,
                                          first_distance(0));
    first = open.first;
    count = max(0, open.last - first + 1);
    for (int i = tid; i < kWaves * kMaxBuckets; i += kThreads) sm.side.bins[0][i] = 0.f;
    if (tid < 32) sm.side.closed[tid] = neg_inf();
    __syncthreads();
  }
  int skip, end;
  p.dkv_split.share(x, count, skip, end);
  first += skip;
  count = end - skip;
  auto tile_at = [&](int i) {
    if constexpr (MODE == kBwdMask)
      return (int)__builtin_amdgcn_readfirstlane(sm.side.tile[first + i]);
    else
      return first + i;
  };

  if (count > 0) fetch(0, tile_at(0));
  f32x16 dk[4], dv[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) dk[db] = dv[db] = f32x16{};

  // one loop over the 32-row halves: with a loop over tiles around one over their halves the
  // compiler moves all accumulators between the loops
  const bool own = key0 + 32 * w < p.n_k;   // this wave has a key
  const bool there = key < p.n_k;
  uint32_t bits = 0xffu;
  TileRuns tile{};
  FarSum far;
  for (int i = 0; i < 2 * count; ++i) {
    const int buf = i >> 1 & 1, b = i & 1;
    if (b == 0) {
      tiles_ready();
      if (i + 2 < 2 * count) fetch(buf ^ 1, tile_at((i >> 1) + 1));
      if constexpr (MODE == kBwdMask) bits = __builtin_amdgcn_readfirstlane(sm.side.bits[first + (i >> 1)]);
      if constexpr (MODE == kBwdBias)
        tile.read(sm.side.runs[buf], w, -(first_distance(tile_at(i >> 1)) & 31),
                  &sm.side.win[buf][32 * w + 63], -32);
    }
    bool visit = own;
    if constexpr (MODE == kBwdMask) visit = bits >> (4 * b + w) & 1u;
    BlockBias bias{};
    if constexpr (MODE == kBwdBias) {
      bias.run = b == 0 ? tile.run[1] : tile.run[0];
      bias.flat = b == 0 ? tile.flat[0] : tile.flat[1];
      bias.first = 32 * w + 32 - 32 * b;
      bias.win = &sm.side.win[buf][bias.first];
      visit = own && bias.run != kRunClosed;
    }
    float all = 0.f, below = 0.f;
    if (visit)
      dkv_block<MODE>(sm, buf, b, row_at, col_at, kf, vf, dk, dv, p.c, lane, w, there, bias,
                      all, below);
    if constexpr (MODE == kBwdBias) {
      if (visit && bias.run == kRunMixed)
        add_by_distance(all, &sm.side.bucket[buf][bias.first], sm.side.bins[w], p.bias.n_buckets);
      else if (visit)
        far.add(sm.side.bins[w], bias.run, all, below);
      if ((i & 63) == 63) far.flush(sm.side.bins[w]);
    }
  }
  const int l = lane_now(), half = l >> 5;
  key = key0 + w * 32 + (l & 31);
  if (x < p.dkv_split.full) {
    if (key < p.n_k) {
      store_row(p.dv + koff, key, dv, 1.f, half);
      store_row(p.dk + koff, key, dk, p.scale, half);
    }
  } else if (own) {
    const size_t slot = x - p.dkv_split.full;
    const int rows = part_rows(p.n_k);
    store_part(p.part_a + slot * rows * kD, dk, rows, w, l);
    store_part(p.part_b + slot * rows * kD, dv, rows, w, l);
  }
  if constexpr (MODE == kBwdBias) {
    far.flush(sm.side.bins[w]);
    __syncthreads();
    float* part = p.dtable_part + (size_t)x * p.bias.n_buckets;
    for (int i = tid; i < p.bias.n_buckets; i += kThreads)
      part[i] = (sm.side.bins[0][i] + sm.side.bins[1][i]) + (sm.side.bins[2][i] + sm.side.bins[3][i]);
  }
}

// ---- dq ----------------------------------------------------------------------------------

template <int MODE>
struct DqSmem {
  alignas(16) uint16_t k[2][kTileElems];
  alignas(16) uint16_t v[2][kTileElems];
  typename SideOf<MODE, DqBias>::type side;
};

// A workgroup owns 128 queries, a wave 32 of them, and streams the keys in tiles of 64.  Per 32
// keys: S^T = K Q^T and dP^T = V dO^T with queries as columns, then dQ^T += K^T dS^T.
//
// delta: dO . O is off by the rounding of o, which matters where one key has most of a row, dS being
// a small difference there.  So dQ is taken with delta' = dO . O and put right at the end, and the dk,
// dv kernel gets delta' + (sum of P (dP - delta')), exact to 32 bits.  (Both kernels begin dP with
// -delta or nearly that: the matrix unit's rounding leans one way along a sum, the same way then.)
//
// A row's dS sum up to zero, so what the rounded P (dP - delta') that went into the products sum up
// to, r, is their error; taking it back as r P,
//   dQ = scale (sum of bf16(P (dP - delta')) k - r sum of P k),
// removes that of delta' and most of the rounding's, which is largest where P is.  The fourth
// product, sum of P k, is the price: some 2 of 18 ms at N = 32760 and 10 heads, for dq off by
// 2.1e-3 of its norm instead of 4.5e-3 (1.7e-3 is the rounding of the result).
//
// With a bias the correction of delta' is divided by the sum of P, which the LSE's rounding leaves
// some 1e-7 off one, so that a row's dS sum up to zero in the table's gradient, too, whose far
// buckets add up very many.
struct RowSums {
  float ds = 0.f;        // of P (dP - delta')
  float rounded = 0.f;   // of the same, rounded
  float p = 0.f;         // of P (kBwdBias)
};

// a + b into a, what that rounds off into rest.
__device__ __forceinline__ void add_exactly(float& a, float& rest, float b) {
  const float x = a + b, y = x - a;
  rest += (a - (x - y)) + (b - y);
  a = x;
}

// With a bias, the sums of 8 tiles at a time go to a lane's sums in LDS: {ds, its rest, p, its rest}.
__device__ __forceinline__ void flush_sums(f32x4& lane_sums, RowSums& sums) {
  const f32x4 x = lane_sums;
  float ds = x[0], ds_rest = x[1], p = x[2], p_rest = x[3];
  add_exactly(ds, ds_rest, sums.ds);
  add_exactly(p, p_rest, sums.p);
  lane_sums = f32x4{ds, ds_rest, p, p_rest};
  sums.ds = sums.p = 0.f;
}

template <int MODE, bool TAIL>
__device__ __forceinline__ void dq_block(DqSmem<MODE>& sm, int buf, int b, uint32_t row_at, uint32_t col_at,
                                         const bf16x8 (&qf)[8], const bf16x8 (&gf)[8],
                                         f32x16 (&dq)[4], f32x16 (&pk)[4], float nl, float nd,
                                         float c, int left, int run, float flat,
                                         const float* win, RowSums& sums) {
  const uint32_t k_at = lds_addr(sm.k), v_at = lds_addr(sm.v);
  const uint32_t block = (uint32_t)(buf * kTileElems * 2 + b * 32 * kRowBytes);
  f32x16 s = f32x16{}, dp;
  if constexpr (MODE == kBwdBias) {
    if (!is_flat(run)) {
      const int l = lane_now();
      const float* at = win + 4 * (l >> 5) - (l & 31);
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = at[27 - back(v)];
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = flat;
    }
  }
  if constexpr (TAIL) {   // keys past the end
    const int l = lane_now(), limit = left - 4 * (l >> 5);
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (27 - back(v) >= limit) s[v] = neg_inf();
  }
  here(nd);   // (the 16 copies of it are made here, not kept in registers around the loop)
#pragma unroll
  for (int v = 0; v < 16; ++v) dp[v] = nd;
  bf16x8 pf[2], df[2];
  // A operands: eight of S, eight of dP, and eight that P K and dQ share, read once: those of the
  // first 16 keys stay for both, those of the others serve two products in a row
  auto operand = [&](int i) {
    if (i < 16) return row_operand(row_at, block, i < 8 ? k_at : v_at, i & 7);
    return col_operand(col_at, block, k_at, (i & 7) >> 2, i & 3);
  };
  auto prob = [&](int v) {
    s[v] = exp2_fast(fmaf(s[v], c, nl));
    pf[v >> 3][v & 7] = (__bf16)s[v];
  };
  auto grad = [&](int v) {
    const float x = s[v] * dp[v];
    sums.ds += x;
    if constexpr (MODE == kBwdBias) sums.p += s[v];
    df[v >> 3][v & 7] = (__bf16)x;
  };
  bf16x8 a[3], first[4], rest[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) a[i] = operand(i);
  sched_fence();
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    // each is read two products ahead
    if (i < 14) a[(i + 2) % 3] = operand(i + 2);
    if (i >= 14 && i < 18) first[i - 14] = operand(i + 2);
    if (i >= 22 && i < 30 && i % 2 == 0) rest[(i - 22) / 2 % 2] = operand(20 + (i - 22) / 2);
    if (i < 8) {
      s = mfma(a[i % 3], qf[i], s);
    } else if (i < 16) {
      dp = mfma(a[i % 3], gf[i - 8], dp);
    } else if (i < 20) {
      pk[i - 16] = mfma(first[i - 16], pf[0], pk[i - 16]);
    } else if (i < 24) {
      dq[i - 20] = mfma(first[i - 20], df[0], dq[i - 20]);
    } else {
      const int db = (i - 24) / 2;
      f32x16& to = i % 2 == 0 ? pk[db] : dq[db];
      to = mfma(rest[db % 2], i % 2 == 0 ? pf[1] : df[1], to);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {   // as in dkv_block
      if (i >= 9 && i < 15) prob((i - 9) * 2 + e);
      if (i >= 16 && i < 20 && e < 1) prob(i - 4);
      if (i >= 16 && i < 24) grad((i - 16) * 2 + e);
    }
    if (i >= 24) {
      const bf16x8& d = df[(i - 24) >> 2];
      const int j = 2 * (i & 3);
      sums.rounded = __builtin_amdgcn_fdot2_f32_bf16(
          bf16x2{d[j], d[j + 1]}, bf16x2{(__bf16)1.f, (__bf16)1.f}, sums.rounded, false);
    }
    sched_fence();
  }
  __builtin_amdgcn_s_setprio(0);
}

template <int MODE>
__global__ __launch_bounds__(kThreads, 2) void bwd_dq_kernel(BwdParams p) {
  __shared__ DqSmem<MODE> sm;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = blockIdx.x;
  const Place at = place_of(p.dq_split, MODE == kBwdBias, p.dq_split.unit(x), p.bh,
                            (p.n_q + 127) / 128, true);
  const int bh = at.bh, q0 = at.group * 128;
  const int n_tiles = (p.n_k + kTile - 1) / kTile;
  const size_t qoff = (size_t)bh * p.n_q * kD, koff = (size_t)bh * p.n_k * kD;
  const auto krs = row_buffer(p.k + koff, p.n_k), vrs = row_buffer(p.v + koff, p.n_k);
  const uint32_t row_at = row_lane(r, g), col_at = col_lane(lane);
  const auto first_distance = [&](int t) { return t * kTile - (q0 + 127) + p.n_q - 1; };
  const auto wrs = word_buffer(p.bias.by_dist + (size_t)(MODE == kBwdBias ? bh % p.H : 0) * p.bias.dist_stride, p.bias.n_dist);
  const auto rrs = word_buffer(p.bias.runs, p.bias.n_runs);
  const uint32_t off = tile_lane_offset(w, lane);
  auto fetch = [&](int buf, int t) {
    const int l = MODE == kBwdBias ? lane_now() : lane;
    const uint32_t at = MODE == kBwdBias ? tile_lane_offset(w, l) : off;
    load_tile(sm.k[buf], krs, at, t * kTile, w);
    load_tile(sm.v[buf], vrs, at, t * kTile, w);
    if constexpr (MODE == kBwdBias) {
      const int e = first_distance(t);
      if (w < 3) load_words(sm.side.win[buf] + 64 * w, wrs, e + 64 * w, l);
      if (w == 3) load_words(sm.side.runs[buf], rrs, e >> 5, l);
    }
  };
  bf16x8 qf[8], gf[8], of[8];
  int row = q0 + w * 32 + r;
  load_row(qf, p.q + qoff, row, row < p.n_q, g);
  load_row(gf, p.dout + qoff, row, row < p.n_q, g);
  load_row(of, p.o + qoff, row, row < p.n_q, g);
  const float lse = row < p.n_q ? p.lse[(size_t)bh * p.n_q + row] : neg_inf();

  int count = n_tiles, first = 0;
  if constexpr (MODE == kBwdMask) {
    build_list<true>(sm.side, p, bh, q0 / 32, n_tiles);
    count = sm.side.count;
  }
  if constexpr (MODE == kBwdBias) {
    const TileRange open = open_tiles<1>(sm.side.ends, p.bias.runs, p.bias.n_runs, n_tiles,
                                         first_distance(0));
    first = open.first;
    count = max(0, open.last - first + 1);
  }
  int skip, end;
  p.dq_split.share(x, count, skip, end);
  first += skip;
  count = end - skip;
  auto tile_at = [&](int i) {
    if constexpr (MODE == kBwdMask)
      return (int)__builtin_amdgcn_readfirstlane(sm.side.tile[first + i]);
    else
      return first + i;
  };
  if (count > 0) fetch(0, tile_at(0));
  f32x16 dq[4], pk[4];
  // -lse * log2 e and -(dO . O); for the dk, dv kernel padded rows are rows that saw no key
  float nl = neg_inf(), nd = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) nd = fmaf(-(float)of[i][j], (float)gf[i][j], nd);
  nd = half_sum(nd);
  if (lse == neg_inf())
    nd = 0.f;   // whatever o and dO hold where there is no key
  else
    nl = -lse * 1.4426950408889634f;   // (of a NaN the row's probabilities are NaN, too)
  if (p.dq_split.part(x) == 0 && row < p.n_rows && g == 0) {
    p.neg_lse2[(size_t)bh * p.n_rows + row] = nl;
    p.neg_delta[(size_t)bh * p.n_rows + row] = nd;   // for the join, and where there is no such row
  }
#pragma unroll
  for (int db = 0; db < 4; ++db) dq[db] = pk[db] = f32x16{};
  const bool own = q0 + 32 * w < p.n_q;   // this wave has a query
  uint32_t bits = 0xffu;
  TileRuns tile{};
  RowSums sums;
  if constexpr (MODE == kBwdBias) sm.side.sums[tid] = f32x4{};   // read by this lane alone
  // Visits i0 .. i1 of the 32-key halves.  A ragged last tile has a copy of the block to itself:
  // masking its keys under a branch in every block took 12 registers, and spilled.
  auto visit_blocks = [&](auto tail, int i0, int i1) {
    for (int i = i0; i < i1; ++i) {
      const int buf = i >> 1 & 1, b = i & 1;
      if (b == 0) {
        tiles_ready();
        if (i + 2 < 2 * count) fetch(buf ^ 1, tile_at((i >> 1) + 1));
        if constexpr (MODE == kBwdMask) bits = __builtin_amdgcn_readfirstlane(sm.side.bits[first + (i >> 1)]);
        if constexpr (MODE == kBwdBias)
          tile.read(sm.side.runs[buf], 3 - w, 0, &sm.side.win[buf][127 - 32 * w], 32);
      }
      bool visit = own;
      const float* win = nullptr;
      if constexpr (MODE == kBwdMask) visit = bits >> (4 * b + w) & 1u;
      const int run = b == 0 ? tile.run[0] : tile.run[1];
      if constexpr (MODE == kBwdBias) {
        visit = own && run != kRunClosed;
        win = &sm.side.win[buf][32 * b - 32 * w + 127];
      }
      if (visit)
        dq_block<MODE, decltype(tail)::value>(sm, buf, b, row_at, col_at, qf, gf, dq, pk, nl, nd, p.c,
                                              p.n_k - (n_tiles - 1) * kTile - 32 * b,
                                              run, b == 0 ? tile.flat[0] : tile.flat[1], win, sums);
      if constexpr (MODE == kBwdBias) {
        if ((i & 15) == 15) flush_sums(sm.side.sums[64 * w + lane_now()], sums);
      }
    }
  };
  const bool ragged = count > 0 && p.n_k % kTile != 0 && tile_at(count - 1) == n_tiles - 1;
  visit_blocks(std::false_type{}, 0, ragged ? 2 * count - 2 : 2 * count);
  if (ragged) visit_blocks(std::true_type{}, 2 * count - 2, 2 * count);
  if constexpr (MODE == kBwdBias) {
    f32x4& mine = sm.side.sums[64 * w + lane_now()];
    flush_sums(mine, sums);
    sums.ds = mine[0] + mine[1];
    sums.p = mine[2] + mine[3];
  }
  const float ds = half_sum(sums.ds), rounded = half_sum(sums.rounded), total = half_sum(sums.p);
  const int l = lane_now(), half = l >> 5;
  row = q0 + w * 32 + (l & 31);
  if (x >= p.dq_split.full) {
    if (own) {
      const size_t slot = x - p.dq_split.full;
      const int rows = part_rows(p.n_q);
      store_part(p.part_a + slot * rows * kD, dq, rows, w, l);
      store_part(p.part_b + slot * rows * kD, pk, rows, w, l);
      float* part = p.part_sums + slot * kPartSums + (row - q0);
      if (half == 0) {
        part[0] = ds;
        part[128] = rounded;
        if (MODE == kBwdBias) part[256] = total;
      }
    }
    return;
  }
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) dq[db][v] = fmaf(-rounded, pk[db][v], dq[db][v]);
  if (row < p.n_q) {
    store_row(p.dq + qoff, row, dq, p.scale, half);
    if (half == 0)
      p.neg_delta[(size_t)bh * p.n_rows + row] = nd - (MODE == kBwdBias && total > 0.f ? ds / total : ds);
  }
}

// ---- joins -------------------------------------------------------------------------------

// Sum of a shared unit's parts in their order, four columns of one row.
__device__ __forceinline__ f32x4 sum_parts(const float* part, const WorkSplit& split, int rows,
                                           const PartPlace& me) {
  f32x4 x = f32x4{};
#pragma unroll 8   // loads in flight; they come first, the sums keep their order
  for (int j = 0; j < split.parts; ++j)
    x += *reinterpret_cast<const f32x4*>(
        part + (size_t)(me.slot0 + j * split.shared()) * rows * kD + me.offset);
  return x;
}

// dq and delta, as at the end of bwd_dq_kernel.
__global__ __launch_bounds__(256) void bwd_join_dq_kernel(BwdParams p, bool bias) {
  const int rows = part_rows(p.n_q);
  const PartPlace me = part_place(blockIdx.x * 256 + threadIdx.x, rows);
  if (me.slot0 >= p.dq_split.shared()) return;
  const Place at = place_of(p.dq_split, bias, p.dq_split.full + me.slot0, p.bh, (p.n_q + 127) / 128, true);
  const int row = at.group * 128 + me.row;
  if (row >= p.n_q) return;
  float ds = 0.f, rounded = 0.f, total = 0.f;
#pragma unroll 8
  for (int j = 0; j < p.dq_split.parts; ++j) {
    const float* part = p.part_sums + (size_t)(me.slot0 + j * p.dq_split.shared()) * kPartSums + me.row;
    ds += part[0];
    rounded += part[128];
    if (bias) total += part[256];
  }
  f32x4 x = sum_parts(p.part_a, p.dq_split, rows, me);
  const f32x4 y = sum_parts(p.part_b, p.dq_split, rows, me);
#pragma unroll
  for (int t = 0; t < 4; ++t) x[t] = fmaf(-rounded, y[t], x[t]);
  store_cols(p.dq + ((size_t)at.bh * p.n_q + row) * kD + me.col, x, p.scale);
  if (me.col == 0)   // the row's only thread that reads -delta' and writes -delta
    p.neg_delta[(size_t)at.bh * p.n_rows + row] -= bias && total > 0.f ? ds / total : ds;
}

__global__ __launch_bounds__(256) void bwd_join_dkv_kernel(BwdParams p, bool bias) {
  const int rows = part_rows(p.n_k);
  const PartPlace me = part_place(blockIdx.x * 256 + threadIdx.x, rows);
  if (me.slot0 >= p.dkv_split.shared()) return;
  const Place at = place_of(p.dkv_split, bias, p.dkv_split.full + me.slot0, p.bh, (p.n_k + 127) / 128, false);
  const int row = at.group * 128 + me.row;
  if (row >= p.n_k) return;
  const size_t out = ((size_t)at.bh * p.n_k + row) * kD + me.col;
  store_cols(p.dk + out, sum_parts(p.part_a, p.dkv_split, rows, me), p.scale);
  store_cols(p.dv + out, sum_parts(p.part_b, p.dkv_split, rows, me), 1.f);
}

// ---- the bias by distance, and the table's gradient -----------------------------------------

// by_dist[h][e] and, from the workgroups of the first head, runs[e / 32].
__global__ __launch_bounds__(256) void bias_prepare_kernel(BiasParams b, int H, float scale) {
  const int e = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y;
  const bool there = e < b.n_dist;
  int at = there ? b.bucket[e] : -1;
  if ((uint32_t)at >= (uint32_t)b.n_buckets) at = kRunClosed;
  if (there) {
    const float x = at < 0 ? neg_inf() : b.table[(size_t)at * H + h];
    b.by_dist[(size_t)h * b.dist_stride + e] = x < kClosedBelow ? neg_inf() : x / scale;
  }
  if (h == 0) {
    // the runs of this half wave: where neighbours differ
    const int lane = threadIdx.x & 63, half = lane & 32;
    const int before = __shfl_up(at, 1);
    const uint32_t change = (uint32_t)(__ballot(there && (lane & 31) != 0 && at != before) >> half);
    const int pos = __popc(change) == 1 ? __ffs(change) - 1 : 0;
    const int last = __shfl(at, half + pos);
    if ((lane & 31) == 0 && there)
      b.runs[e >> 5] = change == 0 ? at : pos != 0 ? run_step(at, last, pos) : (int)kRunMixed;
  }
}

// dtable[i][h]: the parts of all workgroups of the head, in 64 bits and a fixed order.  Lane i of
// every wave takes bucket i, the 16 waves share the units.
__global__ __launch_bounds__(1024) void bias_dtable_kernel(BwdParams p, int B, int groups) {
  __shared__ double sum[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, h = blockIdx.y;
  const int i = blockIdx.x * 64 + lane, n = p.bias.n_buckets;
  const WorkSplit& split = p.dkv_split;
  double x = 0.0;
  if (i < n)
    for (int j = w; j < B * groups; j += 16) {
      const int group = j / B, head = j % B * p.H + h;
      const int unit = split.order == kGroupByGroup ? group * p.bh + head : head * groups + group;
      const int parts = unit < split.full ? 1 : split.parts;
      for (int k = 0; k < parts; ++k)
        x += p.dtable_part[(size_t)(split.workgroup(unit) + k * split.shared()) * n + i];
    }
  sum[w][lane] = x;
  __syncthreads();
  if (w == 0 && i < n) {
    for (int j = 1; j < 16; ++j) x += sum[j][lane];
    p.dtable[(size_t)i * p.H + h] = (float)x;
  }
}

// (Without queries, keys or batches, which only a bias call passes on, the rest still runs.)
template <int MODE>
hipError_t launch_mode(const BwdParams& p, hipStream_t stream) {
  constexpr bool bias = MODE == kBwdBias;
  const dim3 block(kThreads);
  auto joined = [](const WorkSplit& s, int n) { return dim3((s.shared() * part_rows(n) + 7) / 8); };
  if (bias) {
    const hipError_t e = launch_bias_prepare(p.bias, p.H, p.scale, stream);
    if (e != hipSuccess) return e;
  }
  if (p.bh > 0 && p.n_q > 0) {
    hipLaunchKernelGGL((bwd_dq_kernel<MODE>), dim3(p.dq_split.grid()), block, 0, stream, p);
    if (p.dq_split.shared() > 0)
      hipLaunchKernelGGL(bwd_join_dq_kernel, joined(p.dq_split, p.n_q), dim3(256), 0, stream, p, bias);
  }
  if (p.bh > 0 && p.n_k > 0) {
    hipLaunchKernelGGL((bwd_dkv_kernel<MODE>), dim3(p.dkv_split.grid()), block, 0, stream, p);
    if (p.dkv_split.shared() > 0)
      hipLaunchKernelGGL(bwd_join_dkv_kernel, joined(p.dkv_split, p.n_k), dim3(256), 0, stream, p, bias);
  }
  if (bias)
    hipLaunchKernelGGL(bias_dtable_kernel, dim3((p.bias.n_buckets + 63) / 64, p.H), dim3(1024), 0,
                       stream, p, p.bh / p.H, (p.n_k + 127) / 128);
  return hipGetLastError();
}

}  // namespace

int bwd_padded_rows(int n_q) { return (n_q + kTile - 1) / kTile * kTile; }

// A part's 128 KiB of sums are written and read in about 0.04 us; a tile takes 3.5 us.
WorkSplit bwd_split(int mode, int bh, int n_own, int n_streamed) {
  const long long units = (long long)bh * ((n_own + 127) / 128);
  return make_split(units, (n_streamed + kTile - 1) / kTile, 0.012 * part_rows(n_own) / 128,
                    unit_order(mode == kBwdBias, mode == kBwdMask, bh, units));
}

hipError_t launch_bias_prepare(const BiasParams& b, int H, float scale, hipStream_t stream) {
  if (b.n_dist == 0) return hipSuccess;
  hipLaunchKernelGGL(bias_prepare_kernel, dim3((b.n_dist + 255) / 256, H), dim3(256), 0, stream, b,
                     H, scale);
  return hipGetLastError();
}

hipError_t launch_attn_bwd(int mode, const BwdParams& p, hipStream_t stream) {
  switch (mode) {
    case kBwdDense: return launch_mode<kBwdDense>(p, stream);
    case kBwdMask: return launch_mode<kBwdMask>(p, stream);
    case kBwdBias: return launch_mode<kBwdBias>(p, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace dsattn
