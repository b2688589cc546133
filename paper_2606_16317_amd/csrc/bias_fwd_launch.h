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
  int splits;              // workgroups that share the keys of a query tile
  float* part_o;           // workspace [splits][BH][n_q][128], or null for one split
  float* part_ml;          // workspace [splits][BH][n_q][2]: reference maximum (log2) and row sum
};

// Parts that a problem's keys are split into.
int bias_fwd_splits(int bh, int n_q, int n_k);

hipError_t launch_bias_fwd(const BiasFwdParams& p, int bh, hipStream_t stream);

}  // namespace dsattn

#endif
