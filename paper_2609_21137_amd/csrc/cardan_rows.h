// Arguments and launchers of the routing of many rows, of rows to their
// experts and back (cardan_route.hip, cardan_rows.hip) and of the AdamW step
// (cardan_adamw.hip), shared with the C ABI.
#ifndef CARDAN_ROWS_H
#define CARDAN_ROWS_H

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cardan_ffn_plan.h"


namespace cardan {

enum LogitType { LOGIT_BF16 = 0, LOGIT_F32 = 1, LOGIT_F64 = 2 };

// The blocks of rows that count their experts' selections before the rows'
// places are known: this many at most, so that their sums stay short, unless a
// block had more rows than 16 bits count (a row chooses an expert once).
constexpr int kRouteBlocks = 256, kBlockRows = 1 << 15;
__host__ __device__ inline int count_row(int E) { return (E + 7) / 8 * 8; }
// Rows of one call that a single workgroup routes and places by itself: two
// passes of its threads (2.5 us each; a second launch takes 6).
inline int route_small(int E) { return E <= 128 ? 64 : E <= 256 ? 32 : 8; }

// One call of the routing of N rows (the backward pass reads idx and dweight).
struct RouteArgs {
  int32_t N, E, k;
  int32_t sigmoid, renorm;
  int32_t groups, top_groups, best, each;  // each = E / groups experts a group
  int32_t by_score;                        // float64 scores are needed: a bias, or groups by their best two
  int32_t type;                            // LogitType
  int32_t wide;                            // rows and strides allow 16-byte accesses
  float scale;
  int64_t ld, dld;                         // row strides in elements
  const void* logits;
  const float* bias;                       // [E] or nullptr
  int32_t* idx;                            // [N][k], -1: no expert
  float* weight;                           // [N][k]
  int32_t* place;                          // [N][k] or nullptr, -1: none
  int32_t* offsets;                        // [E + 1] with place
  uint16_t* count;                         // [blocks][count_row(E)] (workspace)
  int32_t block_rows, blocks;
  Divisor by_each;                         // division by `each`
  int32_t group_lanes, group_split, row_lds, slots;
  const float* dweight;                    // [N][k]
  void* dlogits;                           // [N][dld]
};

// Rows of N tokens and their k copies in an array of M rows grouped by expert.
struct RowsArgs {
  int32_t N, k, H, M;
  int32_t f32;               // y or dy is float32 (else bf16)
  int32_t wide;              // every row starts on 16 bytes and H % 8 == 0
  const int32_t* place;      // [N][k]; outside [0, M): none
  const float* weight;       // [N][k] or nullptr (1)
  const uint16_t *x, *ye;    // [N][H], [M][H]
  const void* dy;            // [N][H]
  uint16_t *xe, *dye;        // [M][H]
  void* y;                   // [N][H]
  float* dweight;            // [N][k] or nullptr
};

constexpr int kAdamwBlock = 256;  // values that share a scale
constexpr int kAdamwWork = 2048;  // values of a workgroup
constexpr int64_t kAdamwMost = (int64_t)1 << 34;  // values of a launch: its threads are counted in 32 bits
constexpr int kAdamwTensors = 40; // tensors of one launch (their table is a kernel argument)

struct AdamwTensor {
  void* p;
  const void* g;
  void *m, *v;
  float *ms, *vs;
  uint16_t* copy;
  int64_t n;
};

struct AdamwArgs {
  AdamwTensor t[kAdamwTensors];
  int32_t first[kAdamwTensors + 1];  // first workgroup of every tensor
  int32_t count;
  int32_t step;
  double beta1, beta2, lr, decay;    // for a step or a rate on the device
  float b1, a1, b2, a2, eps;         // beta and 1 - beta
  float lr_decay, lr_c1, inv_c2;     // lr decay, lr / (1 - beta1^t), 1 / (1 - beta2^t)
  const float* lr_device;
  const int32_t* step_device;
  const float* grad_scale;
};

hipError_t launch_route(const RouteArgs&, hipStream_t);
hipError_t launch_route_backward(const RouteArgs&, hipStream_t);
hipError_t launch_dispatch(const RowsArgs&, hipStream_t);
hipError_t launch_combine(const RowsArgs&, hipStream_t);
hipError_t launch_combine_backward(const RowsArgs&, hipStream_t);
hipError_t launch_adamw(const AdamwArgs&, bool param_bf16, bool grad_bf16, bool state8, hipStream_t);

}  // namespace cardan

#endif  // CARDAN_ROWS_H
