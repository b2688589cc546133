// Internal interface between the C-ABI entry points and the kernels of the backward pass.
#ifndef DSATTN_ATTN_BWD_LAUNCH_H
#define DSATTN_ATTN_BWD_LAUNCH_H

#include "attn_split.h"

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace dsattn {

enum { kBwdDense = 0, kBwdMask = 1, kBwdBias = 2 };

// Learned position bias: what the caller gives, and what launch_bias_prepare makes of it.
struct BiasParams {
  const float* table;      // [n_buckets][H]
  const int32_t* bucket;   // [n_dist]: bucket of distance e - (n_q - 1), outside [0, n_buckets): closed
  int n_buckets;
  int n_dist;              // bias_distances
  float* by_dist;          // workspace [H][dist_stride]: bias / scale by distance, -inf: closed
  int32_t* runs;           // workspace [n_runs]: what 32 distances hold, see below
  int dist_stride;         // floats, a multiple of 32
  int n_runs;              // ceil(n_dist / 32)
};

// Distances that a problem has: none without a query, a key or a batch.  Then nothing reads the table
// or the buckets, so these are needed, checked, and laid out, only where there are distances.
inline int bias_distances(int bh, int n_q, int n_k) {
  return bh > 0 && n_q > 0 && n_k > 0 ? n_q + n_k - 1 : 0;
}

// A word of runs: the bucket of 32 distances that share one (kRunClosed: all closed), kRunMixed,
// or run_step where the first `pos` of them share one and the rest another.
enum { kRunClosed = -1, kRunMixed = -2, kRunStep = 1 << 30 };
constexpr int run_step(int first, int last, int pos) {
  return kRunStep | pos << 20 | (first + 1) << 10 | (last + 1);
}
constexpr bool is_step(int run) { return run >= kRunStep; }
constexpr int run_first(int run) { return is_step(run) ? (run >> 10 & 1023) - 1 : run; }
constexpr int run_last(int run) { return is_step(run) ? (run & 1023) - 1 : run; }
constexpr int run_pos(int run) { return run >> 20 & 1023; }
// Biases below this close their pairs.  Next to any other key exp of them is zero; in a row of
// nothing else they would be open, but with logits and an LSE of that size in 32 bits, one step of
// which (2^-9 here) goes into the recomputed probabilities as a factor.
constexpr float kClosedBelow = -30000.f;
constexpr int kMaxBuckets = 512;   // what the backward pass keeps of them in LDS

// Fill by_dist and runs (no launch without distances).
hipError_t launch_bias_prepare(const BiasParams& b, int H, float scale, hipStream_t stream);

constexpr int kPartSums = 3 * 128;

struct BwdParams {
  const uint16_t* q;       // bf16 [BH][n_q][128]
  const uint16_t* k;       // bf16 [BH][n_k][128]
  const uint16_t* v;
  const uint16_t* o;
  const uint16_t* dout;
  const float* lse;        // [BH][n_q], natural logarithm, -inf: the row saw no key
  uint16_t* dq;
  uint16_t* dk;
  uint16_t* dv;
  int bh, H, n_q, n_k;     // bh: batches times heads
  float c;                 // scale * log2(e)
  float scale;
  // workspace, rows padded to n_rows (a multiple of 64)
  float* neg_lse2;         // [BH][n_rows]: -lse * log2(e); -inf for rows that saw no key or do not exist
  float* neg_delta;        // [BH][n_rows]: -delta
  int n_rows;
  // units of the dq and of the dk, dv kernel, and the partial results of units that are shared
  WorkSplit dq_split, dkv_split;
  float* part_a;           // [slots][part_rows(n)][128]: sums of dS K, later of dS^T Q
  float* part_b;           // of P K, later of P^T dO
  float* part_sums;        // [slots][kPartSums]: the sums of a row's RowSums
  // kBwdMask
  const uint8_t* mask;     // [BH][n_units][n_dec], nonzero: skipped
  int tile_q, tile_k;
  int n_units, n_dec;
  // kBwdBias
  BiasParams bias;
  float* dtable;           // [n_buckets][H]
  float* dtable_part;      // workspace [dkv_split.grid()][n_buckets]
};

// Rows of a head's padded per-row workspace.
int bwd_padded_rows(int n_q);

// The launches' units.
WorkSplit bwd_split(int mode, int bh, int n_own, int n_streamed);

hipError_t launch_attn_bwd(int mode, const BwdParams& p, hipStream_t stream);

}  // namespace dsattn

#endif
