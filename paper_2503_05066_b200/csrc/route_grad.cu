// Gradient of the router: from the gradients of the kept pairs' scores (and, with dscores, of all scores) to those of
// logits, tokens, router weights and bias.  S is the softmax over the E experts that the route stage left.
//   dS[t,e] = sum of dweight[r] over the slots of t that keep a row r of e  (+ dscores[t,e])
//   dl[t,e] = S[t,e] (dS[t,e] - sum_f S[t,f] dS[t,f])
//   dx = dl W_r,   dW_r = dl^T x,   dbias = sum_t dl
// Three forms of the products, all with fp32 accumulation and parts of dW_r and dbias over ranges of tokens that one last kernel
// adds in their order:
//   fp32, up to eight experts             k_route_grad_few: everything in one kernel on plain FMAs, W_r and dW_r in registers
//   bf16, rows of whole 16-byte vectors   k_route_logit_grad, then both products in one pass over x (route_grad_tc.cu)
//   others                                the same with x read and laid out by warps (route_grad_any.cu)
// Tensor cores take dl, which is fp32, as three bf16 numbers whose sum it is: the top 16 bits of an fp32 number are a bf16 number, so are
// those of the rest, and what that leaves has 8 bits.
#include "route_grad.cuh"

namespace capmoe {
namespace {

constexpr int RG_WARPS = 8;
constexpr int RG_BLOCKS = 4;                 // blocks per SM at most (walks the tokens, so that dbias has few parts)

struct LogitArgs {
  ScoreGrad s;
  float *dlogits, *dbias_part;               // dbias_part may be NULL
  __nv_bfloat16* split;                      // [N, ROUTE_PARTS Eq]
  int Eq;
};

// A warp takes four tokens at a time (their lookups in flight together), lane + 32 i an expert of each.
constexpr int RG_TOK = 4;
template <int EPL>
__global__ void __launch_bounds__(RG_WARPS * 32) k_route_logit_grad(const LogitArgs a) {
  wait_for_previous_kernel();
  allow_next_kernel();                       // in this order: an early successor reads what came before (gmm.cuh)
  __shared__ float ds[RG_WARPS][RG_TOK][EPL * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.s.E;
  float bias[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) bias[i] = 0.f;
  for (int64_t t0 = ((int64_t)blockIdx.x * RG_WARPS + warp) * RG_TOK; t0 < a.s.N; t0 += (int64_t)gridDim.x * RG_WARPS * RG_TOK) {
    const int n = (int)min((int64_t)RG_TOK, a.s.N - t0);
    float s[RG_TOK][EPL];
#pragma unroll
    for (int j = 0; j < RG_TOK; ++j)
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const int e = lane + 32 * i;
        const bool in = j < n && e < E;
        s[j][i] = in ? a.s.scores[(t0 + j) * E + e] : 0.f;
        ds[warp][j][e] = in && a.s.dscores ? a.s.dscores[(t0 + j) * a.s.dscores_ld + e] : 0.f;
      }
    __syncwarp();
    add_kept(a.s, t0, n, lane, 32, ds[warp][0], EPL * 32);
    __syncwarp();
    float dot[RG_TOK];
#pragma unroll
    for (int j = 0; j < RG_TOK; ++j) {
      dot[j] = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) dot[j] = fmaf(s[j][i], ds[warp][j][lane + 32 * i], dot[j]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int j = 0; j < RG_TOK; ++j) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], o);
#pragma unroll
    for (int j = 0; j < RG_TOK; ++j) {
      if (j >= n) break;
      const int64_t t = t0 + j;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const int e = lane + 32 * i;
        const float dl = e < E ? s[j][i] * (ds[warp][j][e] - dot[j]) : 0.f;
        bias[i] += dl;
        if (e < E) a.dlogits[t * E + e] = dl;
        if (e < a.Eq) {
          __nv_bfloat16* p = a.split + t * ROUTE_PARTS * a.Eq + e;
          float rest = dl;
#pragma unroll
          for (int q = 0; q < ROUTE_PARTS; ++q) {
            const uint32_t top = __float_as_uint(rest) & 0xffff0000u;
            p[q * a.Eq] = __ushort_as_bfloat16((unsigned short)(top >> 16));
            rest = rest == __uint_as_float(top) ? 0.f : rest - __uint_as_float(top);         // (an infinity: zeros, not inf - inf)
          }
        }
      }
    }
    __syncwarp();                            // the rows are rewritten for the next tokens
  }
  if (!a.dbias_part) return;
#pragma unroll
  for (int i = 0; i < EPL; ++i) ds[warp][0][lane + 32 * i] = bias[i];
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += RG_WARPS * 32) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < RG_WARPS; ++i) sum += ds[i][0][e];
    a.dbias_part[(int64_t)blockIdx.x * E + e] = sum;
  }
}

// ---------------------------------------------------------------- fp32, up to eight experts: plain FMAs
// A thread owns four columns: their W_r and dW_r stay in its registers, x goes by once.  A block is `tx` threads across the columns
// by `ty` tokens at a time; it walks a range of tokens in chunks, whose dl it makes first in shared memory.  4 E FMAs an element of
// x and dx: bound by HBM as long as enough loads are in flight (eight tokens a thread): 16,384 tokens of 4096 columns, eight
// experts 108 us (169 on tensor cores, where three parts of everything pass through shared memory; with 16 experts, and half as
// many columns a thread, this took 165).
constexpr int FEW_N = 256;                   // threads
constexpr int FEW_TOK = 64;                  // tokens of a chunk
constexpr int FEW_E = 8;
constexpr int FEW_V = 4;                     // columns of a thread

// A thread's columns, `step` apart (1 with VEC, which takes them in one access); without VEC columns that do not exist repeat the first.
template <bool VEC> struct Few {
  float v[FEW_V];
  __device__ __forceinline__ void load(const float* p, int step, int left) {
    if constexpr (VEC) {
      const float4 w = *reinterpret_cast<const float4*>(p);
      v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
#pragma unroll
      for (int j = 0; j < FEW_V; ++j) v[j] = p[j * step < left ? j * step : 0];
    }
  }
  __device__ __forceinline__ void store(float* p, int step, int left) const {
    if constexpr (VEC) {
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int j = 0; j < FEW_V; ++j)
        if (j * step < left) p[j * step] = v[j];
    }
  }
};

struct FewArgs {
  ScoreGrad s;
  const float *x, *w;
  int d, tx, per;                            // per: tokens of a range
  float* dx;
  float *dlogits, *parts, *dbias_part;       // parts [ranges][E][d], dbias_part [ranges][E]
};

template <bool VEC>
__global__ void __launch_bounds__(FEW_N, 2) k_route_grad_few(const FewArgs a) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int U = 8;                       // tokens in flight
  constexpr int BY = FEW_N / FEW_E, EACH = FEW_TOK / BY;                // tokens whose dl is made at a time, and of a thread
  __shared__ __align__(16) float dl[FEW_TOK][FEW_E];
  __shared__ float sum[FEW_N][FEW_V];
  const int E = a.s.E, d = a.d, tx = a.tx, ty = FEW_N / tx, cx = threadIdx.x & (tx - 1), cy = threadIdx.x / tx;
  const int step = VEC ? 1 : tx, c = (int)blockIdx.x * tx * FEW_V + (VEC ? cx * FEW_V : cx), left = d - c;
  const bool cols = left > 0;
  const int range = blockIdx.y;
  const int64_t first = (int64_t)range * a.per, last = min(a.s.N, first + a.per);
  const int e = threadIdx.x & (FEW_E - 1), i0 = threadIdx.x / FEW_E;
  float dw[FEW_E][FEW_V], bias = 0.f;
  Few<VEC> w[FEW_E];
#pragma unroll
  for (int f = 0; f < FEW_E; ++f) {
#pragma unroll
    for (int j = 0; j < FEW_V; ++j) w[f].v[j] = dw[f][j] = 0.f;
    if (f < E && cols) w[f].load(a.w + (int64_t)f * d + c, step, left);
  }
  for (int64_t t0 = first; t0 < last; t0 += FEW_TOK) {
    const int n = (int)min((int64_t)FEW_TOK, last - t0);
    float s[EACH];
    __syncthreads();                         // the last chunk's dl has been read
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = i0 + k * BY;
      const bool mine = i < n && e < E;
      s[k] = mine ? a.s.scores[(t0 + i) * E + e] : 0.f;
      dl[i][e] = mine && a.s.dscores ? a.s.dscores[(t0 + i) * a.s.dscores_ld + e] : 0.f;
    }
    __syncthreads();
    add_kept(a.s, t0, n, threadIdx.x, FEW_N, &dl[0][0], FEW_E);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = i0 + k * BY;
      const float g = dl[i][e];
      float dot = s[k] * g;
#pragma unroll
      for (int o = FEW_E / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      const bool mine = i < n && e < E;
      const float v = mine ? s[k] * (g - dot) : 0.f;
      dl[i][e] = v;
      bias += v;
      if (mine && blockIdx.x == 0) a.dlogits[(t0 + i) * E + e] = v;
    }
    __syncthreads();
    if (cols) {
      for (int i1 = cy; i1 < n; i1 += ty * U) {
        Few<VEC> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load(a.x + (t0 + min(i1 + u * ty, n - 1)) * d + c, step, left);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i1 + u * ty;
          if (i >= n) break;
          Few<VEC> y;
#pragma unroll
          for (int j = 0; j < FEW_V; ++j) y.v[j] = 0.f;
#pragma unroll
          for (int f = 0; f < FEW_E; f += 4) {
            const float4 q = *reinterpret_cast<const float4*>(&dl[i][f]);
            const float l[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
              for (int j = 0; j < FEW_V; ++j) {
                y.v[j] = fmaf(l[m], w[f + m].v[j], y.v[j]);
                dw[f + m][j] = fmaf(l[m], x[u].v[j], dw[f + m][j]);
              }
          }
          y.store(a.dx + (t0 + i) * d + c, step, left);
        }
      }
    }
  }
  // the ty shares of dW_r in their order, then a part
  float* part = a.parts + (int64_t)range * E * d;
#pragma unroll
  for (int f = 0; f < FEW_E; ++f) {
    if (ty > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < FEW_V; ++j) sum[threadIdx.x][j] = dw[f][j];
      __syncthreads();
      if (cy == 0)
        for (int k = 1; k < ty; ++k)
#pragma unroll
          for (int j = 0; j < FEW_V; ++j) dw[f][j] += sum[cx + k * tx][j];
    }
    if (cy == 0 && f < E && cols) {
#pragma unroll
      for (int j = 0; j < FEW_V; ++j)
        if (j * step < left) part[(int64_t)f * d + c + j * step] = dw[f][j];
    }
  }
  if (blockIdx.x == 0) {
    __syncthreads();
    sum[threadIdx.x][0] = bias;
    __syncthreads();
    if (threadIdx.x < E) {
      float b = 0.f;
      for (int k = threadIdx.x; k < FEW_N; k += FEW_E) b += sum[k][0];
      a.dbias_part[(int64_t)range * E + threadIdx.x] = b;
    }
  }
}

// dW_r [E, d] from parts [ranges][E][d] and, in the blocks behind, dbias [E] from parts [bias_parts][E], all in a fixed order.
constexpr int JOIN_N = 256, JOIN_E = 8;      // threads; experts of a block for dbias
constexpr int JOIN_G = 8;                    // threads that share an output's parts (every JOIN_G-th each, their loads in flight together)
template <typename TO, int VW>
__global__ void __launch_bounds__(JOIN_N) k_join_route(const float* __restrict__ part, int parts, int64_t size, int dw_blocks,
                                                       TO* __restrict__ dw, const float* __restrict__ bias_part, int bias_parts, int E,
                                                       float* __restrict__ dbias) {
  allow_next_kernel();
  wait_for_previous_kernel();
  if ((int)blockIdx.x < dw_blocks) {
    __shared__ float share[JOIN_N][VW];
    constexpr int COLS = JOIN_N / JOIN_G;
    const int col = threadIdx.x & (COLS - 1), g = threadIdx.x / COLS;
    const int64_t i = ((int64_t)blockIdx.x * COLS + col) * VW;
    float s[VW];
#pragma unroll
    for (int j = 0; j < VW; ++j) s[j] = 0.f;
    if (i < size)
#pragma unroll 4
      for (int p = g; p < parts; p += JOIN_G) {
        if constexpr (VW == 4) {
          const float4 v = __ldcs(reinterpret_cast<const float4*>(part + p * size + i));
          s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
        } else {
          s[0] += part[p * size + i];
        }
      }
#pragma unroll
    for (int j = 0; j < VW; ++j) share[threadIdx.x][j] = s[j];
    __syncthreads();
    if (g == 0 && i < size) {
#pragma unroll
      for (int k = 1; k < JOIN_G; ++k)
#pragma unroll
        for (int j = 0; j < VW; ++j) s[j] += share[k * COLS + col][j];
#pragma unroll
      for (int j = 0; j < VW; ++j) dw[i + j] = from_float<TO>(s[j]);
    }
    return;
  }
  __shared__ float sum[JOIN_N];
  const int e = (int)(blockIdx.x - dw_blocks) * JOIN_E + (threadIdx.x & (JOIN_E - 1)), r = threadIdx.x / JOIN_E;
  float s = 0.f;
  if (e < E)
#pragma unroll 8
    for (int p = r; p < bias_parts; p += JOIN_N / JOIN_E) s += bias_part[(int64_t)p * E + e];
  sum[threadIdx.x] = s;
  __syncthreads();
  if (r == 0 && e < E) {
#pragma unroll 8
    for (int k = 1; k < JOIN_N / JOIN_E; ++k) s += sum[k * JOIN_E + threadIdx.x];
    dbias[e] = s;
  }
}

template <typename TO>
int join_run(const float* part, int parts, int64_t size, void* dw, const float* bias_part, int bias_parts, int E, float* dbias,
             cudaStream_t st) {
  const bool wide = size % 4 == 0;
  const int64_t dw_blocks = ceil_div(size, (int64_t)(JOIN_N / JOIN_G) * (wide ? 4 : 1)), blocks = dw_blocks + ceil_div(E, JOIN_E);
  if (blocks > 0x7fffffff) return CAPMOE_EUNSUPPORTED;
  auto k = wide ? k_join_route<TO, 4> : k_join_route<TO, 1>;
  const int rc = note_cuda(launch_chained(k, (unsigned)blocks, JOIN_N, 0, st, part, parts, size, (int)dw_blocks, (TO*)dw, bias_part, bias_parts, E,
                                          dbias));
  count_launch(1);
  return rc;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

enum Form { FEW, TC, ANY };
struct RouteWs {
  Form form;
  int Eq, ranges, blocks;                    // blocks of the logits' kernel (FEW: ranges)
  size_t bias, split, parts, total;
};
int few_tx(int d) {
  int tx = 32;
  while (tx < FEW_N && tx * FEW_V < d) tx *= 2;
  return tx;
}
RouteWs route_ws(int64_t N, int d, int E, int dtype) {
  RouteWs w = {};
  w.form = route_grad_tc_supported(d, dtype) ? TC : dtype == CAPMOE_F32 && E <= FEW_E ? FEW : ANY;
  w.Eq = (E + 7) / 8 * 8;                    // rows of `split` in whole 16-byte vectors
  const int64_t sms = sm_count();
  if (w.form == FEW) {
    // two blocks per SM; 32 tokens each at least, or a part of dW_r would be as long as its tokens
    const int64_t across = ceil_div(d, few_tx(d) * FEW_V), want = 2 * sms / across, most = ceil_div(N, 32);
    int64_t r = want < most ? want : most;
    if (r < 1) r = 1;
    if (r > 65535) r = 65535;
    w.ranges = (int)ceil_div(N, ceil_div(N, r));
  } else {
    w.ranges = w.form == TC ? route_grad_tc_ranges(N, d, E) : route_grad_any_ranges(N, d, E, dtype);
  }
  const int64_t want = ceil_div(N, RG_WARPS * RG_TOK), most = sms * RG_BLOCKS;
  w.blocks = w.form == FEW ? w.ranges : (int)(want < most ? want : most);
  if (w.ranges < 1) w.ranges = 1;
  if (w.blocks < 1) w.blocks = 1;
  w.split = up256((size_t)w.blocks * E * 4);
  w.parts = w.split + (w.form == FEW ? 0 : up256((size_t)N * ROUTE_PARTS * w.Eq * 2));
  w.total = w.parts + up256((size_t)w.ranges * E * d * 4) + 256;         // 256: to align all of it
  return w;
}

int few_run(const ScoreGrad& s, const void* x, const void* w, int d, int ranges, float* dlogits, void* dx, float* parts, float* bias, cudaStream_t st) {
  const FewArgs a{s, (const float*)x, (const float*)w, d, few_tx(d), (int)ceil_div(s.N, ranges), (float*)dx, dlogits, parts, bias};
  const int rc = note_cuda(launch_chained(d % FEW_V == 0 ? k_route_grad_few<true> : k_route_grad_few<false>,
                                          dim3((unsigned)ceil_div(d, a.tx * FEW_V), (unsigned)ranges), FEW_N, 0, st, a));
  count_launch(1);
  return rc;
}

int check_route(int64_t N, int d, int E, int dtype) {
  if (N < 0 || d < 1 || E < 1) return CAPMOE_EINVAL;
  if ((dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) || E > 256 || N > GMM_MAX_ROWS || ceil_div(d, 64) > 65535) return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}

}  // namespace
}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_route_backward_workspace_bytes(int64_t N, int d, int E, int dtype, size_t* bytes) {
  const int rc = check_route(N, d, E, dtype);
  if (!bytes) return CAPMOE_EINVAL;
  if (rc == CAPMOE_OK) *bytes = N ? route_ws(N, d, E, dtype).total : 0;
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
  const ScoreGrad sg{scores, dweight, dscores, topk_idx, slot_row, token_group, N, A_max, dscores_ld, E, k, slots, D};
  // nothing to join: a launch less for up to 128 tokens (32 of FEW; dbias is then the sum of one thread an expert: not of many tokens)
  const bool single = w.ranges == 1 && (w.form == FEW || N <= 256);
  const bool whole = single && out_dtype == CAPMOE_F32;
  float *parts = whole ? (float*)dw : (float*)(b + w.parts), *bias = single ? dbias : (float*)(b + w.bias);
  if (w.form == FEW) {
    rc = few_run(sg, x, w_router, d, w.ranges, dlogits, dx, parts, bias, st);
  } else {
    LogitArgs a = {};
    a.s = sg;
    a.dlogits = dlogits; a.dbias_part = single ? nullptr : bias;
    a.split = (__nv_bfloat16*)(b + w.split);
    a.Eq = w.Eq;
    auto kernel = E <= 32 ? k_route_logit_grad<1> : E <= 64 ? k_route_logit_grad<2> : E <= 128 ? k_route_logit_grad<4> : k_route_logit_grad<8>;
    rc = note_cuda(launch_chained(kernel, (unsigned)w.blocks, RG_WARPS * 32, 0, st, a));
    count_launch(1);
    if (rc != CAPMOE_OK) return rc;
    const RouteOut out{parts, single && !whole ? (__nv_bfloat16*)dw : nullptr, dlogits, single ? dbias : nullptr};
    rc = w.form == TC ? route_grad_tc(a.split, x, w_router, N, d, E, w.Eq, w.ranges, dx, out, dev_status, st)
                      : route_grad_any(a.split, x, w_router, N, d, E, w.Eq, w.ranges, dtype, dx, out, dev_status, st);
  }
  if (rc != CAPMOE_OK || single) return rc;
  const int64_t size = (int64_t)E * d;
  return out_dtype == CAPMOE_F32 ? join_run<float>(parts, w.ranges, size, dw, bias, w.blocks, E, dbias, st)
                                 : join_run<__nv_bfloat16>(parts, w.ranges, size, dw, bias, w.blocks, E, dbias, st);
}
