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

// Adds dweight of the kept rows of tokens t0 .. t0 + n - 1 to their rows of dS (shared memory, `ld` words apart, set to dscores
// before), the (token, slot) pairs spread over threads `me` of `of`, so that the lookups of many tokens are in flight together.
// A token has one row of an expert: each word has one addition, whatever the order.
__device__ __forceinline__ void add_kept(const ScoreGrad& a, int64_t t0, int n, int me, int of, float* ds, int ld) {
  const int pairs = n * a.slots, m = a.D > 0 ? a.E / a.D : 0;
  for (int i = me; i < pairs; i += of) {
    const int32_t r = a.slot_row[t0 * a.slots + i];
    const int tok = i / a.slots, s = i - tok * a.slots;
    const int64_t t = t0 + tok;
    if (r >= 0 && r < a.rows) {
      const int e = s < a.k ? a.topk_idx[t * a.k + s] : home_group(t, a.N, a.D, a.token_group) * m + (s - a.k);
      if ((unsigned)e < (unsigned)a.E) atomicAdd(&ds[tok * ld + e], a.dweight[r]);
    }
  }
}

// Ranges of whole stages of 64 tokens, none of them empty: one wave of CTAs, 128 tokens each at least, or as many waves as keep a range
// within `most` tokens.
inline int route_ranges(int64_t N, int64_t slices, int64_t most) {
  const int64_t units = ceil_div(N, 64), wave = sm_count() / slices > 1 ? sm_count() / slices : 1;
  int64_t r = wave * ceil_div(N, wave * most);
  if (r > ceil_div(units, 2)) r = ceil_div(units, 2);
  return (int)ceil_div(units, ceil_div(units, r));
}

// dx = dl W_r and the parts of dW_r = dl^T x over `ranges` ranges of tokens on tcgen05.
// split [N, ROUTE_PARTS Eq]: dl as bf16 numbers, Eq a multiple of 8 >= E; parts [ranges][E][d].  The kernel before it on the
// stream wrote `split` and let its successor start only after its own wait for what came before.
// With one range dW_r is final: it goes to `parts`, or as bf16 to dw16, and dbias is made too, from dl [N, E].
struct RouteOut {
  float* parts;
  __nv_bfloat16* dw16;                       // else NULL, as the other two
  const float* dl;
  float* dbias;
};
// Sums of the columns of dl [n, E], threads `me` of `of`.
__device__ __forceinline__ void sum_bias(const RouteOut& o, int64_t n, int E, int me, int of) {
  for (int e = me; e < E; e += of) {
    float s = 0.f;
#pragma unroll 16
    for (int64_t t = 0; t < n; ++t) s += o.dl[t * E + e];
    o.dbias[e] = s;
  }
}
constexpr int ROUTE_PARTS = 3;
//   bf16, d a multiple of 8
inline bool route_grad_tc_supported(int d, int dtype) { return dtype == CAPMOE_BF16 && d % 8 == 0; }
int route_grad_tc_ranges(int64_t N, int d, int E);
int route_grad_tc(const void* split, const void* x, const void* w, int64_t N, int d, int E, int Eq, int ranges, void* dx, const RouteOut& out,
                  int32_t* dev_status, cudaStream_t st);
//   any
int route_grad_any_ranges(int64_t N, int d, int E, int dtype);
int route_grad_any(const void* split, const void* x, const void* w, int64_t N, int d, int E, int Eq, int ranges, int dtype, void* dx,
                   const RouteOut& out, int32_t* dev_status, cudaStream_t st);

}  // namespace capmoe
