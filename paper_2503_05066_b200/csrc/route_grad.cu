// Gradient of the router: from the gradients of the kept pairs' scores (and, with dscores, of all scores) to those of
// logits, tokens, router weights and bias.  S is the softmax over the E experts that the route stage left.
//   dS[t,e] = sum of dweight[r] over the slots of t that keep a row r of e  (+ dscores[t,e])
//   dl[t,e] = S[t,e] (dS[t,e] - sum_f S[t,f] dS[t,f])
//   dx = dl W_r,   dW_r = dl^T x,   dbias = sum_t dl
// The two products run as grouped products of one expert (dx) and of ranges of tokens (dW_r, added in their order here).
// bf16: dl is fp32, and one rounding to bf16 could cost it 2^-8; it goes in as two bf16 numbers, its rounding and the
// rounding of what that leaves out (2^-16 of dl is lost at most), side by side as 2E columns, against W_r twice.
#include "gmm.cuh"
#include "rowvec.cuh"

namespace capmoe {
namespace {

constexpr int RG_WARPS = 8;
constexpr int RG_BLOCKS = 8;                 // blocks per SM at most (walks the tokens, so that dbias has few parts)

struct LogitArgs {
  const float *scores, *dweight, *dscores;
  const int32_t *topk_idx, *slot_row, *token_group;
  int64_t N, rows, dscores_ld;
  int E, k, slots, D;
  float *dlogits, *dbias_part;
  __nv_bfloat16* pair;                       // bf16: [N, 2 Ep], else NULL
  int Ep;
  const __nv_bfloat16* w;                    // bf16: W_r [E, d] and its copy with itself [2 Ep, d]
  __nv_bfloat16* w2;
  int d;
  int32_t* offsets;                          // [0, N], then `ranges` + 1 bounds of the ranges of tokens
  int ranges, range;
};

// One warp a token, lane + 32 i an expert.
template <int EPL>
__global__ void __launch_bounds__(RG_WARPS * 32) k_route_logit_grad(const LogitArgs a) {
  allow_next_kernel();
  wait_for_previous_kernel();
  __shared__ float ds[RG_WARPS][EPL * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.E;
  const int64_t tid = (int64_t)blockIdx.x * (RG_WARPS * 32) + threadIdx.x, threads = (int64_t)gridDim.x * (RG_WARPS * 32);
  if (tid < 2) a.offsets[tid] = tid ? (int32_t)a.N : 0;
  if (tid <= a.ranges) a.offsets[2 + tid] = (int32_t)min(a.N, tid * (int64_t)a.range);
  if (a.w2) {
    const int64_t half = (int64_t)a.Ep * a.d;
    for (int64_t i = tid; i < 2 * half; i += threads) {
      const int64_t j = i < half ? i : i - half;
      a.w2[i] = j < (int64_t)E * a.d ? a.w[j] : __float2bfloat16_rn(0.f);
    }
  }
  float bias[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) bias[i] = 0.f;
  for (int64_t t = (int64_t)blockIdx.x * RG_WARPS + warp; t < a.N; t += (int64_t)gridDim.x * RG_WARPS) {
    float* row = ds[warp];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane + 32 * i;
      row[e] = a.dscores && e < E ? a.dscores[t * a.dscores_ld + e] : 0.f;
    }
    __syncwarp();
    for (int s = lane; s < a.slots; s += 32) {
      const int32_t r = a.slot_row[t * a.slots + s];
      if (r >= 0 && r < a.rows) {
        const int e = s < a.k ? a.topk_idx[t * a.k + s] : home_group(t, a.N, a.D, a.token_group) * (E / a.D) + (s - a.k);
        if ((unsigned)e < (unsigned)E) atomicAdd(&row[e], a.dweight[r]);       // (one addition: a token has one row of an expert)
      }
    }
    __syncwarp();
    float s[EPL], g[EPL], dot = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane + 32 * i;
      s[i] = e < E ? a.scores[t * E + e] : 0.f;
      g[i] = row[e];
      dot = fmaf(s[i], g[i], dot);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane + 32 * i;
      const float dl = s[i] * (g[i] - dot);
      if (e < E) {
        a.dlogits[t * E + e] = dl;
        bias[i] += dl;
      }
      if (a.pair && e < a.Ep) {
        const __nv_bfloat16 hi = __float2bfloat16_rn(dl);
        a.pair[t * 2 * a.Ep + e] = hi;
        a.pair[t * 2 * a.Ep + a.Ep + e] = __float2bfloat16_rn(dl - __bfloat162float(hi));
      }
    }
    __syncwarp();                            // row is rewritten by the next token
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) ds[warp][lane + 32 * i] = bias[i];
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += RG_WARPS * 32) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < RG_WARPS; ++i) sum += ds[i][e];
    a.dbias_part[(int64_t)blockIdx.x * E + e] = sum;
  }
}

// dw [E, d] from parts [ranges][copies * Ep][d] (copies = 2: both halves of dl), in a fixed order.
template <typename TO>
__global__ void __launch_bounds__(256) k_join_dw(const float* __restrict__ part, int ranges, int copies, int E, int Ep, int d, TO* __restrict__ dw) {
  allow_next_kernel();
  wait_for_previous_kernel();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)E * d) return;
  const int64_t half = (int64_t)Ep * d;
  float s = 0.f;
#pragma unroll 4
  for (int p = 0; p < ranges * copies; ++p) s += part[p * half + i];
  dw[i] = from_float<TO>(s);
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

// Ranges of tokens whose dW_r are summed apart: enough for the tiles of 256 x 256 to fill the pairs of SMs, 512 tokens each at least.
int ranges_of(int64_t N, int d, int n) {
  const int64_t tiles = ceil_div(d, 256) * ceil_div(n, 256), want = (sm_count() / 2) / tiles, most = N / 512;
  int64_t r = want < most ? want : most;
  return (int)(r < 1 ? 1 : r > 64 ? 64 : r);
}
struct RouteWs {
  int copies, Ep, ranges, blocks;
  size_t offsets, bias, pair, w2, parts, dw, dw_bytes, total;
};
RouteWs route_ws(int64_t N, int d, int E, int dtype) {
  RouteWs w;
  w.copies = dtype == CAPMOE_BF16 ? 2 : 1;
  w.Ep = dtype == CAPMOE_BF16 ? (E + 3) / 4 * 4 : E;         // rows of `pair` in whole 16-byte vectors
  w.ranges = ranges_of(N, d, w.copies * w.Ep);
  const int64_t want = ceil_div(N, RG_WARPS), most = (int64_t)sm_count() * RG_BLOCKS;
  w.blocks = (int)(want < most ? want : most);
  if (w.blocks < 1) w.blocks = 1;
  w.offsets = 0;
  w.bias = up256((size_t)(w.ranges + 3) * 4);
  w.pair = w.bias + up256((size_t)w.blocks * E * 4);
  w.w2 = w.pair + (w.copies == 2 ? up256((size_t)N * 2 * w.Ep * 2) : 0);
  w.parts = w.w2 + (w.copies == 2 ? up256((size_t)2 * w.Ep * d * 2) : 0);
  w.dw = w.parts + (w.copies * w.ranges > 1 ? up256((size_t)w.ranges * w.copies * w.Ep * d * 4) : 0);
  w.dw_bytes = 0;
  capmoe_grouped_mm_dw_workspace_bytes(w.ranges, &w.dw_bytes);
  w.total = w.dw + up256(w.dw_bytes) + 256;                  // 256: to align all of it
  return w;
}

int check_route(int64_t N, int d, int E, int dtype) {
  if (N < 0 || d < 1 || E < 1) return CAPMOE_EINVAL;
  if ((dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) || E > 256 || N > GMM_MAX_ROWS || ceil_div(d, 64) > 65535) return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}
template <class... P>
bool usable(P... p) {
  return ((p != nullptr && aligned16(p)) && ...);
}

}  // namespace
}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_route_backward_workspace_bytes(int64_t N, int d, int E, int dtype, size_t* bytes) {
  const int rc = check_route(N, d, E, dtype);
  if (!bytes) return CAPMOE_EINVAL;
  if (rc == CAPMOE_OK) *bytes = route_ws(N, d, E, dtype).total;
  return rc;
}

extern "C" int capmoe_route_backward(const void* x, const void* w_router, const float* scores, const int32_t* topk_idx, const int32_t* slot_row,
                                     const float* dweight, int64_t N, int d, int E, int k, int slots, int D, const int32_t* token_group,
                                     const float* dscores, int64_t dscores_ld, int dtype, int out_dtype, int64_t A_max, float* dlogits, void* dx,
                                     void* dw, float* dbias, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  int rc = check_route(N, d, E, dtype);
  if (rc != CAPMOE_OK) return rc;
  if (k < 1 || k > E || D < 0 || A_max < 0) return CAPMOE_EINVAL;
  if (D > 0 ? E % D != 0 || slots != k + E / D : slots != k) return CAPMOE_EINVAL;
  if (dscores_ld != 0 && dscores_ld < E) return CAPMOE_EINVAL;
  if (k > 32 || A_max >= ((int64_t)1 << 31)) return CAPMOE_EUNSUPPORTED;
  if (out_dtype != CAPMOE_F32 && (out_dtype != CAPMOE_BF16 || dtype != CAPMOE_BF16)) return CAPMOE_EUNSUPPORTED;
  if (!usable(dw) || !dbias) return CAPMOE_EINVAL;
  cudaStream_t st = as_stream(stream);
  if (N == 0) {
    rc = note_cuda(cudaMemsetAsync(dw, 0, (size_t)E * d * elt_size(out_dtype), st));
    return rc != CAPMOE_OK ? rc : note_cuda(cudaMemsetAsync(dbias, 0, (size_t)E * 4, st));
  }
  if (!usable(x, w_router, dlogits, dx, ws) || !scores || !topk_idx || !slot_row || (A_max > 0 && !dweight)) return CAPMOE_EINVAL;
  const RouteWs w = route_ws(N, d, E, dtype);
  if (ws_bytes < w.total) return CAPMOE_EWORKSPACE;
  uint8_t* b = (uint8_t*)up256((size_t)ws);
  const bool bf16 = dtype == CAPMOE_BF16;
  const int n = w.copies * w.Ep;
  LogitArgs a = {};
  a.scores = scores; a.dweight = dweight; a.dscores = dscores;
  a.topk_idx = topk_idx; a.slot_row = slot_row; a.token_group = token_group;
  a.N = N; a.rows = A_max; a.dscores_ld = dscores_ld;
  a.E = E; a.k = k; a.slots = slots; a.D = D;
  a.dlogits = dlogits; a.dbias_part = (float*)(b + w.bias);
  a.offsets = (int32_t*)(b + w.offsets); a.ranges = w.ranges; a.range = (int)ceil_div(N, w.ranges);
  a.Ep = w.Ep; a.d = d;
  if (bf16) {
    a.pair = (__nv_bfloat16*)(b + w.pair);
    a.w = (const __nv_bfloat16*)w_router;
    a.w2 = (__nv_bfloat16*)(b + w.w2);
  }
  auto kernel = E <= 32 ? k_route_logit_grad<1> : E <= 64 ? k_route_logit_grad<2> : E <= 128 ? k_route_logit_grad<4> : k_route_logit_grad<8>;
  rc = note_cuda(launch_chained(kernel, (unsigned)w.blocks, RG_WARPS * 32, 0, st, a));
  count_launch(1);
  if (rc != CAPMOE_OK) return rc;
  const void* dl = bf16 ? (const void*)a.pair : dlogits;
  const void* wr = bf16 ? (const void*)a.w2 : w_router;
  if ((rc = capmoe_grouped_mm_dx(dl, a.offsets, wr, 1, d, n, dtype, dx, N, dev_status, stream)) != CAPMOE_OK) return rc;
  const bool joined = w.copies * w.ranges > 1;
  float* parts = joined ? (float*)(b + w.parts) : (float*)dw;
  rc = capmoe_grouped_mm_dw(dl, x, a.offsets + 2, w.ranges, d, n, dtype, CAPMOE_F32, parts, N, b + w.dw, w.dw_bytes, dev_status, stream);
  if (rc != CAPMOE_OK) return rc;
  if (joined) {
    const int64_t blocks = ceil_div((int64_t)E * d, 256);
    rc = note_cuda(out_dtype == CAPMOE_F32
                       ? launch_chained(k_join_dw<float>, (unsigned)blocks, 256, 0, st, (const float*)parts, w.ranges, w.copies, E, w.Ep, d, (float*)dw)
                       : launch_chained(k_join_dw<__nv_bfloat16>, (unsigned)blocks, 256, 0, st, (const float*)parts, w.ranges, w.copies, E, w.Ep, d,
                                        (__nv_bfloat16*)dw));
    count_launch(1);
    if (rc != CAPMOE_OK) return rc;
  }
  return sum_parts(a.dbias_part, w.blocks, E, CAPMOE_F32, dbias, st);
}
