// Arguments and launchers of the feed-forward block (cardan_ffn.hip) and of
// the distillation loss (cardan_distill.hip), shared with the C ABI.
#ifndef CARDAN_FFN_H
#define CARDAN_FFN_H

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cardan_ffn_plan.h"

namespace cardan {

// One call of the feed-forward block. Rows n of group e are off[e] <= n <
// off[e + 1] (off == nullptr: one group of all N rows).
struct FfnArgs {
  int32_t N, E, H, I;
  int32_t relu2;                 // up-only squared-ReLU experts (Wg unused)
  const int32_t* off;            // [E + 1] or nullptr
  const uint16_t *x, *dy;        // [N][H]
  const uint16_t *Wg, *Wu, *Wd;  // [E][H][I], [E][H][I], [E][I][H]
  float *g, *u;                  // [N][I] projections kept for the backward pass, or nullptr
  uint16_t* h;                   // [N][I] hidden activations
  uint16_t *dg, *du;             // [N][I] gradients of the projections (workspace)
  uint16_t *y, *dx;              // [N][H]
  uint16_t *dWg, *dWu, *dWd;     // as the weights
  float* part;                   // partial sums of split products (ffn_partial_bytes)
};

// One call of the distillation loss over the rows of [N][ld] logits.
struct DistillArgs {
  int32_t N, V, K;
  int32_t f32;                   // logits are float32 (else bf16)
  int64_t ld, dld;               // row strides of logits and gradient, in elements
  const void* logits;
  const float* teacher;          // [N][K]
  const int32_t* ids;            // [N][K]; outside [0, V): no entry
  const int32_t* labels;         // [N] or nullptr; outside [0, V): no label
  const float* weight;           // [N] or nullptr (1)
  float temperature, ce_weight;
  float* loss;                   // [N][2]
  void* dlogits;                 // [N][dld] or nullptr
};

hipError_t launch_distill(const DistillArgs&, hipStream_t);
hipError_t launch_ffn_forward(const FfnArgs&, hipStream_t);
hipError_t launch_ffn_backward(const FfnArgs&, hipStream_t);

}  // namespace cardan

#endif  // CARDAN_FFN_H
