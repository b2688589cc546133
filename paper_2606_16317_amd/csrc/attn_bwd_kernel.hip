// Backward pass of attention for gfx950: dq, dk and dv, the probabilities recomputed.
//
//   P = exp(S - lse), S = scale Q K^T     dS = P (dO V^T - delta), delta_i = dO_i . O_i
//   dV = P^T dO      dK = scale dS^T Q    dQ = scale dS K
//
// Two kernels share the work: one owns keys and streams queries (dK, dV: four products), one
// owns queries and streams keys (dQ: three products).  One kernel for all would need five
// products instead of seven, but would have to add every workgroup's part of dQ in memory:
// 64 KiB of fp32 atomics for each 21 MFLOP, in an order that changes from run to run.  Seven
// products at the rate of the forward pass cost less than five with those, and their sums are
// always in the same order.
//
// Both are bound by MFMA and, equally, by LDS reads (1 KiB of operand per MFMA, the other
// operand stays in registers).  Instruction order is fixed by fences: operands are read two
// MFMAs ahead, exponentials run under the dP products, dS under the dV products.
// N = 32760, 10 heads: 16.1 ms, 852 TFLOP/s of the five products the mathematics needs and
// 1193 of the seven computed; a large library product reaches 1215 on the same card.

#include "attn_bwd_launch.h"
#include "attn_tiles.h"

namespace dsattn {
namespace {

constexpr int kMaxTiles = 4096;   // 64-row tiles that a visit list can hold

// ---- per-row quantities ----------------------------------------------------------------

// One row per 16 lanes: -lse * log2 e and -(dO . O), padded rows as rows that saw no key.
__global__ __launch_bounds__(256) void bwd_rows_kernel(BwdParams p) {
  const int row = blockIdx.x * 16 + (threadIdx.x >> 4);
  const int bh = blockIdx.y;
  const int part = threadIdx.x & 15;
  if (row >= p.n_rows) return;
  float dot = 0.f, nl = neg_inf();
  if (row < p.n_q) {
    const size_t at = ((size_t)bh * p.n_q + row) * kD + part * 8;
    const bf16x8 a = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p.o + at));
    const bf16x8 b = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p.dout + at));
#pragma unroll
    for (int i = 0; i < 8; ++i) dot = fmaf((float)a[i], (float)b[i], dot);
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) dot += __shfl_xor(dot, m);
    const float l = p.lse[(size_t)bh * p.n_q + row];
    if (l > neg_inf()) nl = -l * 1.4426950408889634f;
  }
  if (part == 0) {
    p.neg_lse2[(size_t)bh * p.n_rows + row] = nl;
    p.neg_delta[(size_t)bh * p.n_rows + row] = -dot;
  }
}

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
template <int MODE>
__device__ __forceinline__ bool block_open(const BwdParams& p, int bh, int qb, int kb) {
  if (32 * qb >= p.n_q || 32 * kb >= p.n_k) return false;
  const int u = 32 * qb / p.tile_q, d = 32 * kb / p.tile_k;
  return p.mask[((size_t)bh * p.n_units + u) * p.n_dec + d] == 0;
}

// Fill the list: own 32-row blocks own0 .. own0 + 3, streamed tiles 0 .. n_tiles - 1.
// Q_OWN: the own blocks are query blocks, the tiles key tiles.
template <int MODE, bool Q_OWN>
__device__ __forceinline__ void build_list(VisitList& list, const BwdParams& p, int bh, int own0,
                                           int n_tiles) {
  const int tid = threadIdx.x, lane = tid & 63;
  // every thread notes its tiles' bits in place, then the first wave closes the gaps in order
  for (int t = tid; t < n_tiles; t += kThreads) {
    uint32_t bits = 0;
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
      const int b = 2 * t + (j >> 2), x = own0 + (j & 3);
      if (Q_OWN ? block_open<MODE>(p, bh, x, b) : block_open<MODE>(p, bh, b, x)) bits |= 1u << j;
    }
    list.bits[t] = (uint8_t)bits;
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

// ---- dk, dv ------------------------------------------------------------------------------

struct NoList {};
template <int MODE>
struct ListOf {
  typedef VisitList type;
};
template <>
struct ListOf<kBwdDense> {
  typedef NoList type;
};

template <int MODE>
struct DkvSmem {
  alignas(16) uint16_t q[2][kTileElems];
  alignas(16) uint16_t g[2][kTileElems];   // dO
  alignas(16) float nl[2][kTile];
  alignas(16) float nd[2][kTile];
  typename ListOf<MODE>::type list;
};

// A workgroup owns 128 keys, a wave 32 of them, and streams the queries in tiles of 64.  Per 32
// queries: S = Q K^T and dP = dO V^T with keys as columns, so that
// P and dS are B operands of dV^T += dO^T P and dK^T += Q^T dS.
template <int MODE>
__device__ __forceinline__ void dkv_block(const DkvSmem<MODE>& sm, int buf, int b, uint32_t row_at,
                                          uint32_t col_at, const bf16x8 (&kf)[8],
                                          const bf16x8 (&vf)[8], f32x16 (&dk)[4],
                                          f32x16 (&dv)[4], float c, int g) {
  constexpr int kG = 2 * kTileElems * 2;   // bytes from the q tiles to the dO tiles
  const uint32_t block = (uint32_t)(buf * kTileElems * 2 + b * 32 * kRowBytes);
  row_at += block;
  col_at += block;
  here(row_at);
  here(col_at);
  f32x16 s, dp, nd;
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
    if (i < 16) return row_operand(row_at, i < 8 ? 0 : kG, i & 7);
    return col_operand(col_at, i < 24 ? kG : 0, (i & 7) >> 2, i & 3);
  };
  bf16x8 pf[2], df[2];
  auto prob = [&](int v) {
    s[v] = exp2_fast(fmaf(s[v], c, nl[v >> 2][v & 3]));
    pf[v >> 3][v & 7] = (__bf16)s[v];
  };
  auto grad = [&](int v) { df[v >> 3][v & 7] = (__bf16)(s[v] * dp[v]); };
  constexpr int RK = 3;
  bf16x8 a[RK];
#pragma unroll
  for (int i = 0; i < RK - 1; ++i) a[i] = operand(i);
  sched_fence();
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (i + RK - 1 < 32) a[(i + RK - 1) % RK] = operand(i + RK - 1);
    const bf16x8& x = a[i % RK];
    if (i < 8)
      s = mfma(x, kf[i], i == 0 ? f32x16{} : s);
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
    sched_fence();
  }
}

template <int MODE>
__global__ __launch_bounds__(kThreads, 2) void bwd_dkv_kernel(BwdParams p) {
  __shared__ DkvSmem<MODE> sm;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y;
  const int key0 = blockIdx.x * 128;
  const int n_tiles = (p.n_q + kTile - 1) / kTile;
  const size_t qoff = (size_t)bh * p.n_q * kD, koff = (size_t)bh * p.n_k * kD;
  const auto qrs = row_buffer(p.q + qoff, p.n_q), grs = row_buffer(p.dout + qoff, p.n_q);
  const auto lrs = word_buffer(p.neg_lse2 + (size_t)bh * p.n_rows, p.n_rows);
  const auto drs = word_buffer(p.neg_delta + (size_t)bh * p.n_rows, p.n_rows);
  const uint32_t off = tile_lane_offset(w, lane);
  const uint32_t row_at = lds_addr(sm.q) + row_lane(r, g), col_at = lds_addr(sm.q) + col_lane(lane);

  auto fetch = [&](int buf, int t) {
    load_tile(sm.q[buf], qrs, off, t * kTile, w);
    load_tile(sm.g[buf], grs, off, t * kTile, w);
    if (w == 0) load_words(sm.nl[buf], lrs, t * kTile, lane);
    if (w == 1) load_words(sm.nd[buf], drs, t * kTile, lane);
  };

  int count = n_tiles;
  if constexpr (MODE != kBwdDense) {
    build_list<MODE, false>(sm.list, p, bh, key0 / 32, n_tiles);
    count = sm.list.count;
  }
  auto tile_at = [&](int i) {
    if constexpr (MODE == kBwdDense)
      return i;
    else
      return (int)__builtin_amdgcn_readfirstlane(sm.list.tile[i]);
  };

  if (count > 0) fetch(0, tile_at(0));
  bf16x8 kf[8], vf[8];
  f32x16 dk[4], dv[4];
  const int key = key0 + w * 32 + r;
  load_row(kf, p.k + koff, key, key < p.n_k, g);
  load_row(vf, p.v + koff, key, key < p.n_k, g);
#pragma unroll
  for (int db = 0; db < 4; ++db) dk[db] = dv[db] = f32x16{};

  // one loop over the 32-row halves: with a loop over tiles around one over their halves the
  // compiler moves all accumulators between the loops
  uint32_t bits = 0xffffu;
  for (int i = 0; i < 2 * count; ++i) {
    const int buf = i >> 1 & 1, b = i & 1;
    if (b == 0) {
      tiles_ready();
      if (i + 2 < 2 * count) fetch(buf ^ 1, tile_at((i >> 1) + 1));
      if constexpr (MODE != kBwdDense) bits = __builtin_amdgcn_readfirstlane(sm.list.bits[i >> 1]);
    }
    const uint32_t keep = bits >> (4 * b + w) & 1u;
    if (MODE == kBwdDense || keep != 0)
      dkv_block<MODE>(sm, buf, b, row_at, col_at, kf, vf, dk, dv, p.c, g);
  }
  if (key < p.n_k) {
    store_row(p.dv + koff, key, dv, 1.f, g);
    store_row(p.dk + koff, key, dk, p.scale, g);
  }
}

// ---- dq ----------------------------------------------------------------------------------

template <int MODE>
struct DqSmem {
  alignas(16) uint16_t k[2][kTileElems];
  alignas(16) uint16_t v[2][kTileElems];
  typename ListOf<MODE>::type list;
};

// A workgroup owns 128 queries, a wave 32 of them, and streams the keys in tiles of 64.  Per 32
// keys: S^T = K Q^T and dP^T = V dO^T with queries as columns, then
// dQ^T += K^T dS^T.
__device__ __forceinline__ void dq_block(int buf, int b, uint32_t row_at, uint32_t col_at,
                                         const bf16x8 (&qf)[8], const bf16x8 (&gf)[8],
                                         f32x16 (&dq)[4], float nl, float nd, float c, int lim) {
  constexpr int kV = 2 * kTileElems * 2;   // bytes from the k tiles to the v tiles
  const uint32_t block = (uint32_t)(buf * kTileElems * 2 + b * 32 * kRowBytes);
  row_at += block;
  col_at += block;
  here(row_at);
  here(col_at);
  f32x16 s, dp;
  bf16x8 df[2];
  // A operands in the order of their products: S, dP, dQ (eight each)
  auto operand = [&](int i) {
    if (i < 16) return row_operand(row_at, i < 8 ? 0 : kV, i & 7);
    return col_operand(col_at, 0, (i & 7) >> 2, i & 3);
  };
  auto prob = [&](int v) { s[v] = exp2_fast(fmaf(s[v], c, nl)); };
  auto grad = [&](int v) {
    float x = s[v] * (dp[v] + nd);
    // keys past the end: their rows are zeros, but exp2(-lse) may be infinite
    if (8 * (v >> 2) + (v & 3) >= lim) x = 0.f;
    df[v >> 3][v & 7] = (__bf16)x;
  };
  constexpr int RK = 3;
  bf16x8 a[RK];
#pragma unroll
  for (int i = 0; i < RK - 1; ++i) a[i] = operand(i);
  sched_fence();
#pragma unroll
  for (int i = 0; i < 24; ++i) {
    if (i + RK - 1 < 24) a[(i + RK - 1) % RK] = operand(i + RK - 1);
    const bf16x8& x = a[i % RK];
    if (i < 8)
      s = mfma(x, qf[i], i == 0 ? f32x16{} : s);
    else if (i < 16)
      dp = mfma(x, gf[i - 8], i == 8 ? f32x16{} : dp);
    else
      dq[i & 3] = mfma(x, df[(i & 7) >> 2], dq[i & 3]);
    if (i >= 9 && i < 16) {
      prob(2 * (i - 9));
      prob(2 * (i - 9) + 1);
    }
    if (i == 15) {
      prob(14);
      prob(15);
#pragma unroll
      for (int v = 0; v < 8; ++v) grad(v);
    }
    if (i >= 16 && i < 20) {
      grad(8 + 2 * (i - 16));
      grad(9 + 2 * (i - 16));
    }
    sched_fence();
  }
}

template <int MODE>
__global__ __launch_bounds__(kThreads, 2) void bwd_dq_kernel(BwdParams p) {
  __shared__ DqSmem<MODE> sm;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y;
  const int q0 = blockIdx.x * 128;
  const int n_tiles = (p.n_k + kTile - 1) / kTile;
  const size_t qoff = (size_t)bh * p.n_q * kD, koff = (size_t)bh * p.n_k * kD;
  const auto krs = row_buffer(p.k + koff, p.n_k), vrs = row_buffer(p.v + koff, p.n_k);
  const uint32_t off = tile_lane_offset(w, lane);
  const uint32_t row_at = lds_addr(sm.k) + row_lane(r, g), col_at = lds_addr(sm.k) + col_lane(lane);
  auto fetch = [&](int buf, int t) {
    load_tile(sm.k[buf], krs, off, t * kTile, w);
    load_tile(sm.v[buf], vrs, off, t * kTile, w);
  };
  int count = n_tiles;
  if constexpr (MODE != kBwdDense) {
    build_list<MODE, true>(sm.list, p, bh, q0 / 32, n_tiles);
    count = sm.list.count;
  }
  auto tile_at = [&](int i) {
    if constexpr (MODE == kBwdDense)
      return i;
    else
      return (int)__builtin_amdgcn_readfirstlane(sm.list.tile[i]);
  };
  if (count > 0) fetch(0, tile_at(0));
  bf16x8 qf[8], gf[8];
  f32x16 dq[4];
  const int row = q0 + w * 32 + r;
  load_row(qf, p.q + qoff, row, row < p.n_q, g);
  load_row(gf, p.dout + qoff, row, row < p.n_q, g);
  const size_t at = (size_t)bh * p.n_rows + row;
  const float nl = row < p.n_q ? p.neg_lse2[at] : neg_inf();
  const float nd = row < p.n_q ? p.neg_delta[at] : 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) dq[db] = f32x16{};
  uint32_t bits = 0xffu;
  int t = 0;
  for (int i = 0; i < 2 * count; ++i) {
    const int buf = i >> 1 & 1, b = i & 1;
    if (b == 0) {
      t = tile_at(i >> 1);
      tiles_ready();
      if (i + 2 < 2 * count) fetch(buf ^ 1, tile_at((i >> 1) + 1));
      if constexpr (MODE != kBwdDense) bits = __builtin_amdgcn_readfirstlane(sm.list.bits[i >> 1]);
    }
    const uint32_t keep = bits >> (4 * b + w) & 1u;
    if (MODE == kBwdDense || keep != 0)
      dq_block(buf, b, row_at, col_at, qf, gf, dq, nl, nd, p.c, p.n_k - t * kTile - 32 * b - 4 * g);
  }
  if (row < p.n_q) store_row(p.dq + qoff, row, dq, p.scale, g);
}

template <int MODE>
hipError_t launch_mode(const BwdParams& p, int bh, hipStream_t stream) {
  hipLaunchKernelGGL(bwd_rows_kernel, dim3((p.n_rows + 15) / 16, bh), dim3(256), 0, stream, p);
  hipLaunchKernelGGL((bwd_dq_kernel<MODE>), dim3((p.n_q + 127) / 128, bh), dim3(kThreads), 0,
                     stream, p);
  hipLaunchKernelGGL((bwd_dkv_kernel<MODE>), dim3((p.n_k + 127) / 128, bh), dim3(kThreads), 0,
                     stream, p);
  return hipGetLastError();
}

}  // namespace

int bwd_padded_rows(int n_q) { return (n_q + kTile - 1) / kTile * kTile; }
int bwd_key_groups(int n_k) { return (n_k + 127) / 128; }

hipError_t launch_attn_bwd(int mode, const BwdParams& p, int bh, hipStream_t stream) {
  switch (mode) {
    case kBwdDense: return launch_mode<kBwdDense>(p, bh, stream);
    case kBwdMask: return launch_mode<kBwdMask>(p, bh, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace dsattn
