// Internal interface of the router's gradient (route_grad.cu, route_grad_tc.cu).
#pragma once
#include "gmm.cuh"

namespace capmoe {

// What the gradient of the logits is made from; fields as in capmoe_route_backward.
struct ScoreGrad {
  const float *scores, *dweight, *dscores;
  const int32_t *topk_idx, *slot_row, *token_group;
  int64_t N, rows, dscores_ld;
  int E, k, slots, D;
};

// Adds dweight of token t's kept rows to its row of dS (shared memory; E words, set to dscores before), the lanes lane,
// lane + lanes .. of the slots.  A token has one row of an expert: each word has one addition, whatever the order of the lanes.
__device__ __forceinline__ void add_kept(const ScoreGrad& a, int64_t t, int lane, int lanes, float* row) {
  for (int s = lane; s < a.slots; s += lanes) {
    const int32_t r = a.slot_row[t * a.slots + s];
    if (r >= 0 && r < a.rows) {
      const int e = s < a.k ? a.topk_idx[t * a.k + s] : home_group(t, a.N, a.D, a.token_group) * (a.E / a.D) + (s - a.k);
      if ((unsigned)e < (unsigned)a.E) atomicAdd(&row[e], a.dweight[r]);
    }
  }
}

// dx = dl W_r and the parts of dW_r = dl^T x over `ranges` ranges of tokens on tcgen05: bf16, d a multiple of 8, E <= 128.
// pair [N, 2 Eq]: dl as two bf16 numbers, Eq a multiple of 8 >= E; parts [ranges][E][d].  The kernel before it on the stream
// wrote `pair` and let its successor start only after its own wait for what came before.
inline bool route_grad_tc_supported(int d, int E, int dtype) { return dtype == CAPMOE_BF16 && d % 8 == 0 && E > 16 && E <= 128; }
int route_grad_tc_ranges(int64_t N, int d, int E);
int route_grad_tc(const void* pair, const void* x, const void* w, int64_t N, int d, int E, int Eq, int ranges, void* dx, float* parts,
                  int32_t* dev_status, cudaStream_t st);

}  // namespace capmoe
