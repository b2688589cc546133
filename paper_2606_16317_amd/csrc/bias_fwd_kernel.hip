// Attention with a learned position bias by buckets, forward pass, for gfx950:
//
//   S_ij = scale q_i . k_j + T[bucket(j - i)][h]      O = softmax(S) V      lse = log sum exp S
//
// A workgroup owns 128 queries of one head, a wave 32 of them, and streams keys in tiles of 64
// with a running maximum and sum.  S_{j+1} is computed during step j, under the exponentials of
// tile j; its row maximum under the P V products.  The bias is laid out by distance beforehand
// (one value per head and distance).  A 32 x 32 block whose distances share a bucket, as nearly
// all do when buckets widen with the distance, adds that one number to the row's reference
// maximum; only mixed blocks read single values, as the first accumulator of S.
//
// 24 heads of 27280 rows: 8.64-8.67 ms, 1050 TFLOP/s, where the dense kernel takes 8.25.  The loop waits
// for its own prefetch: the query rows, loaded before it, count as pending at every entry, so each
// step's first products wait for the loads just issued.  Waves wait on 28 % of their cycles (21 % in
// the dense kernel), the matrix pipes are busy on 57 % (70 %); the core clock, 1.57 GHz against 1.55,
// makes up for little of it.

#include "attn_tiles.h"
#include "bias_fwd_launch.h"

#include <type_traits>

namespace dsattn {
namespace {

constexpr float kRescaleSlack = 8.0f;    // log2 units

struct FwdSmem {
  alignas(16) uint16_t k[2][kTileElems];
  alignas(16) uint16_t v[2][kTileElems];
  alignas(16) float win[2][kWindow];
  int32_t runs[2][64];
  int ends[2];
};

__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A query row's softmax so far, in log2 units, and the tile at hand.
struct RowState {
  float m_ref;    // reference maximum, -inf before the first open key
  float l_half;   // this lane's share of the row sum, relative to m_ref
};

// What a tile's two 32-key blocks add to S c: nothing where single values started S.
struct TileBias {
  float flat[2];
};

// First product of a block's S: onto the single values of a mixed block, or onto zero.
__device__ __forceinline__ f32x16 first_product(const bf16x8& a, const bf16x8& q, bool mixed,
                                                const float* win) {
  if (mixed) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = win[8 * (v >> 2) + (v & 3)];
    return mfma(a, q, s);
  }
  return mfma(a, q, f32x16{});
}

__device__ __forceinline__ float block_max(const f32x16& s) {
  float m = s[0];
#pragma unroll
  for (int v = 1; v < 16; ++v) m = maximum(m, s[v]);
  return m;
}

// Maximum over the two lanes of a row.
__device__ __forceinline__ float row_join(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const auto sw = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return maximum(__builtin_bit_cast(float, (uint32_t)sw[0]), __builtin_bit_cast(float, (uint32_t)sw[1]));
}

// LSE (natural) of a row from its reference maximum (log2) and sum; the sum is 0 where it saw no key,
// NaN where a logit was.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l != 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : neg_inf();
}

__device__ __forceinline__ void mask_keys(f32x16 (&s)[2], int lim) {
  here(lim);   // (or the compiler selects in every tile instead of branching in the last)
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (32 * b + 8 * (v >> 2) + (v & 3) >= lim) s[b][v] = neg_inf();
}

__global__ __launch_bounds__(kThreads, 2) void bias_fwd_kernel(BiasFwdParams p) {
  __shared__ FwdSmem sm;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = blockIdx.x;
  const Place at = place_of(p.split, true, p.split.unit(x), p.bh, (p.n_q + 127) / 128, true);
  const int bh = at.bh, q0 = at.group * 128;
  const size_t qoff = (size_t)bh * p.n_q * kD, koff = (size_t)bh * p.k_rows * kD;
  const auto krs = row_buffer(p.k + koff, p.n_k), vrs = row_buffer(p.v + koff, p.n_k);
  const auto wrs = word_buffer(p.bias.by_dist + (size_t)(bh % p.H) * p.bias.dist_stride, p.bias.n_dist);
  const auto rrs = word_buffer(p.bias.runs, p.bias.n_runs);
  const uint32_t off = tile_lane_offset(w, lane);
  const uint32_t row_at = lds_addr(sm.k) + row_lane(r, g), col_at = lds_addr(sm.v) + col_lane(lane);
  const auto first_distance = [&](int t) { return t * kTile - (q0 + 127) + p.n_q - 1; };

  const int row = q0 + 32 * w + r;
  const bool own = q0 + 32 * w < p.n_q;   // this wave has a query
  bf16x8 qf[8];
  load_row(qf, p.q + qoff, row, row < p.n_q, g);

  // tiles with an open run of distances, and of those this workgroup's share
  const TileRange open = open_tiles<1>(sm.ends, p.bias.runs, p.bias.n_runs,
                                       (p.n_k + kTile - 1) / kTile, first_distance(0));
  int t0 = open.first, t1 = open.last + 1;   // none open: t1 = 0 <= t0
  if (t0 < t1) {
    int first, last;
    p.split.share(x, t1 - t0, first, last);
    t1 = t0 + last;
    t0 += first;
  }

  auto fetch_k = [&](int buf, int t) {
    load_tile(sm.k[buf], krs, off, t * kTile, w);
    const int e = first_distance(t);
    if (w < 3) load_words(sm.win[buf] + 64 * w, wrs, e + 64 * w, lane);
    if (w == 3) load_words(sm.runs[buf], rrs, e >> 5, lane);
  };
  auto fetch_v = [&](int buf, int t) { load_tile(sm.v[buf], vrs, off, t * kTile, w); };

  f32x16 o[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) o[db] = f32x16{};
  RowState rs{neg_inf(), 0.f};

  if (t0 < t1) {
    fetch_k(0, t0);
    fetch_v(0, t0);
    if (t0 + 1 < t1) fetch_k(1, t0 + 1);
    tiles_ready();

    // The bias of tile t in buffer buf: which blocks are mixed, and what the others add.
    auto tile_bias = [&](int buf, TileBias& tb, bool (&mixed)[2]) {
      int run[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) run[j] = __builtin_amdgcn_readfirstlane(sm.runs[buf][3 - w + j]);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        mixed[b] = !(run[b] == run[b + 1] && run[b] == run[b + 2]) || run[b] == kRunMixed || is_step(run[b]);
        tb.flat[b] = mixed[b] ? 0.f : sm.win[buf][32 * b - 32 * w + 127] * p.c;
      }
    };
    auto win_at = [&](int buf, int b) { return &sm.win[buf][32 * b + 4 * g - 32 * w - r + 127]; };

    f32x16 s[2];
    TileBias tb, tb_next{};
    bool mixed[2];
    float m_hat = neg_inf();
    if (own) {
      tile_bias(0, tb, mixed);
      uint32_t at = row_at;
      here(at);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const bf16x8 a = row_operand(at, InLane{}, b * kBlockBytes, i);
          s[b] = i == 0 ? first_product(a, qf[0], mixed[b], win_at(0, b)) : mfma(a, qf[i], s[b]);
        }
      const int lim = p.n_k - t0 * kTile - 4 * g;
      if (p.n_k - t0 * kTile < kTile) mask_keys(s, lim);
      m_hat = row_join(maximum(fmaf(block_max(s[0]), p.c, tb.flat[0]),
                               fmaf(block_max(s[1]), p.c, tb.flat[1])));
    }

    // Tile t, in buffer BUF: s holds its S, sn receives the next one's.
    auto step = [&](auto BUF, int t, f32x16 (&s)[2], f32x16 (&sn)[2]) {
      constexpr int buf = decltype(BUF)::value;
      tiles_ready();
      if (t + 2 < t1) fetch_k(buf, t + 2);
      if (t + 1 < t1) fetch_v(buf ^ 1, t + 1);
      if (!own) return;

      if (__ballot(m_hat > rs.m_ref + kRescaleSlack) != 0) {
        const bool need = m_hat > rs.m_ref + kRescaleSlack;
        const float alpha = need ? exp2_fast(rs.m_ref - m_hat) : 1.f;
        rs.m_ref = need ? m_hat : rs.m_ref;
        rs.l_half *= alpha;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
      }
      const float base = rs.m_ref == neg_inf() ? 0.f : -rs.m_ref;
      const float add[2] = {base + tb.flat[0], base + tb.flat[1]};

      // past the last tile these read what an earlier one left, and the results go unused
      tile_bias(buf ^ 1, tb_next, mixed);
      uint32_t ka = row_at + (uint32_t)((buf ^ 1) * kTileElems * 2);
      uint32_t va = col_at + (uint32_t)(buf * kTileElems * 2);
      here(ka);
      here(va);
      // operands in the order of their products: 16 of S (key blocks alternating), 16 of P V
      auto operand = [&](int i) {
        if (i < 16) return row_operand(ka, InLane{}, (i & 1) * kBlockBytes, i >> 1);
        return col_operand(va, InLane{}, ((i - 16) >> 3) * kBlockBytes, ((i - 16) >> 2) & 1, i & 3);
      };
      float xs[32];
      bf16x8 pf[4];
      auto prob = [&](int e) {
        const int b = e >> 4, v = e & 15;
        const float x = exp2_fast(fmaf(s[b][v], p.c, add[b]));
        xs[e] = x;
        pf[e >> 3][e & 7] = (__bf16)x;
      };
      constexpr int RK = 3;
      bf16x8 a[RK];
#pragma unroll
      for (int i = 0; i < RK - 1; ++i) a[i] = operand(i);
      sched_fence();
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        if (i + RK - 1 < 32) a[(i + RK - 1) % RK] = operand(i + RK - 1);
        const bf16x8& x = a[i % RK];
        if (i < 2)
          sn[i] = first_product(x, qf[0], mixed[i], win_at(buf ^ 1, i));
        else if (i < 16)
          sn[i & 1] = mfma(x, qf[i >> 1], sn[i & 1]);
        else
          o[i & 3] = mfma(x, pf[(i - 16) >> 2], o[i & 3]);
        // two exponentials under each of the first eight products, one under the next sixteen
        if (i < 8) {
          prob(2 * i);
          prob(2 * i + 1);
        } else if (i < 24) {
          prob(i + 8);
        }
        sched_fence();
      }
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) sum += xs[e];
      rs.l_half += sum;
      const int left = p.n_k - (t + 1) * kTile;
      if (left < kTile) mask_keys(sn, left - 4 * g);   // the last tile is next, and not full
      m_hat = row_join(maximum(fmaf(block_max(sn[0]), p.c, tb_next.flat[0]),
                               fmaf(block_max(sn[1]), p.c, tb_next.flat[1])));
      tb = tb_next;
    };
    f32x16 s1[2];   // alternating with s: no copies
    for (int t = t0; t < t1; t += 2) {
      step(std::integral_constant<int, 0>{}, t, s, s1);
      if (t + 1 < t1) step(std::integral_constant<int, 1>{}, t + 1, s1, s);
    }
  }

  const float l = half_sum(rs.l_half);
  if (x >= p.split.full) {
    if (!own) return;
    const size_t slot = x - p.split.full, local = row - q0;
    const int rows = part_rows(p.n_q);
    store_part(p.part_o + slot * rows * kD, o, rows, w, lane);
    if (g == 0) {
      p.part_ml[2 * (128 * slot + local)] = rs.m_ref;
      p.part_ml[2 * (128 * slot + local) + 1] = l;
    }
  } else if (row < p.n_q) {
    store_row(p.o + qoff, row, o, l > 0.f ? 1.f / l : 0.f, g);
    if (g == 0 && p.lse != nullptr)
      p.lse[(size_t)bh * p.n_q + row] = row_lse(rs.m_ref, l);
  }
}

// Join the parts of a row, four columns a thread.
__global__ __launch_bounds__(256) void bias_join_kernel(BiasFwdParams p) {
  const int rows = part_rows(p.n_q);
  const PartPlace me = part_place(blockIdx.x * 256 + threadIdx.x, rows);
  if (me.slot0 >= p.split.shared()) return;
  const Place at = place_of(p.split, true, p.split.full + me.slot0, p.bh, (p.n_q + 127) / 128, true);
  const int row = at.group * 128 + me.row;
  if (row >= p.n_q) return;
  const auto slot = [&](int i) { return (size_t)(me.slot0 + i * p.split.shared()); };
  const auto ml = [&](int i) { return p.part_ml + 2 * (128 * slot(i) + me.row); };
  float m = neg_inf();
#pragma unroll 8
  for (int i = 0; i < p.split.parts; ++i) m = fmaxf(m, ml(i)[0]);
  // (a part without an open key has the reference -inf and zeros, one of NaN alone the same and NaN,
  // which the factor 0 leaves)
  const float ref = m == neg_inf() ? 0.f : m;
  float l = 0.f;
  f32x4 x = f32x4{};
#pragma unroll 4
  for (int i = 0; i < p.split.parts; ++i) {
    const float f = exp2_fast(ml(i)[0] - ref);
    l = fmaf(f, ml(i)[1], l);
    const f32x4 z = *reinterpret_cast<const f32x4*>(p.part_o + slot(i) * rows * kD + me.offset);
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = fmaf(f, z[t], x[t]);
  }
  store_cols(p.o + ((size_t)at.bh * p.n_q + row) * kD + me.col, x, l > 0.f ? 1.f / l : 0.f);
  if (me.col == 0 && p.lse != nullptr)
    p.lse[(size_t)at.bh * p.n_q + row] = row_lse(ref, l);
}

}  // namespace

// A part's 64 KiB are written and read in about 0.02 us; a tile takes 2 us.
WorkSplit bias_fwd_split(int bh, int n_q, int n_k) {
  const long long units = (long long)bh * ((n_q + 127) / 128);
  return make_split(units, (n_k + kTile - 1) / kTile, 0.010 * part_rows(n_q) / 128,
                    unit_order(true, false, bh, units));
}

hipError_t launch_bias_fwd(const BiasFwdParams& p, hipStream_t stream) {
  const hipError_t e = launch_bias_prepare(p.bias, p.H, p.scale, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(bias_fwd_kernel, dim3(p.split.grid()), dim3(kThreads), 0, stream, p);
  if (p.split.shared() > 0)
    hipLaunchKernelGGL(bias_join_kernel, dim3((p.split.shared() * part_rows(p.n_q) + 7) / 8), dim3(256),
                       0, stream, p);
  return hipGetLastError();
}

}  // namespace dsattn
