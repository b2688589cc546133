// Internal interface between the C-ABI entry points and the forward kernels with a position bias.
#ifndef DSATTN_BIAS_FWD_LAUNCH_H
#define DSATTN_BIAS_FWD_LAUNCH_H

#include "attn_bwd_launch.h"

namespace dsattn {

struct BiasFwdParams {
  const uint16_t* q;       // bf16 [BH][n_q][128]
  const uint16_t* k;       // bf16 [BH][k_rows][128], n_k <= k_rows of them keys
  const uint16_t* v;
  uint16_t* o;
  float* lse;              // [BH][n_q] or null
  int H, n_q, n_k, k_rows;
  float c;                 // scale * log2(e)
  float scale;
  BiasParams bias;
  int bh;                  // batches times heads
  WorkSplit split;
  float* part_o;           // workspace [slots][part_rows(n_q)][128]
  float* part_ml;          // workspace [slots][128][2]: reference maximum (log2) and row sum
};

// The launch's units.
WorkSplit bias_fwd_split(int bh, int n_q, int n_k);

hipError_t launch_bias_fwd(const BiasFwdParams& p, hipStream_t stream);

}  // namespace dsattn

#endif
