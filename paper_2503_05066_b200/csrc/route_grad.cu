// Gradient of the router: from the gradients of the kept pairs' scores (and, with dscores, of all scores) to those of
// logits, tokens, router weights and bias.  S is the softmax over the E experts that the route stage left.
//   dS[t,e] = sum of dweight[r] over the slots of t that keep a row r of e  (+ dscores[t,e])
//   dl[t,e] = S[t,e] (dS[t,e] - sum_f S[t,f] dS[t,f])
//   dx = dl W_r,   dW_r = dl^T x,   dbias = sum_t dl
// Three forms of the products, all with fp32 accumulation and parts of dW_r and dbias over ranges of tokens that one last kernel
// adds in their order:
//   bf16, rows of whole 16-byte vectors   k_route_logit_grad, then both products in one pass over x (route_grad_tc.cu)
//   others, E <= 32   k_route_grad_few: everything in one kernel on plain FMAs, W_r and dW_r in registers
//   others            k_route_logit_grad, then the grouped products (gmm.cuh) of one expert (dx) and of ranges of tokens (dW_r)
// bf16 products on tensor cores: dl is fp32, and one rounding to bf16 could cost it 2^-8; it goes in as two bf16 numbers, its
// rounding and the rounding of what that leaves out (2^-16 of dl is lost at most).
#include "route_grad.cuh"
#include "rowvec.cuh"

namespace capmoe {
namespace {

constexpr int RG_WARPS = 8;
constexpr int RG_BLOCKS = 4;                 // blocks per SM at most (walks the tokens, so that dbias has few parts)

struct LogitArgs {
  ScoreGrad s;
  float *dlogits, *dbias_part;
  __nv_bfloat16* pair;                       // bf16: [N, 2 Eq], else NULL
  int Eq;
  const __nv_bfloat16* w;                    // for the grouped product: W_r [E, d] and its copy with itself [2 Eq, d], else NULL
  __nv_bfloat16* w2;
  int d;
  int32_t* offsets;                          // for the grouped products: [0, N], then `ranges` + 1 bounds of tokens, else NULL
  int ranges, range;
};

// A warp takes four tokens at a time (their lookups in flight together), lane + 32 i an expert of each.
constexpr int RG_TOK = 4;
template <int EPL>
__global__ void __launch_bounds__(RG_WARPS * 32) k_route_logit_grad(const LogitArgs a) {
  wait_for_previous_kernel();
  allow_next_kernel();                       // in this order: an early successor reads what came before (gmm.cuh)
  __shared__ float ds[RG_WARPS][RG_TOK][EPL * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.s.E;
  const int64_t tid = (int64_t)blockIdx.x * (RG_WARPS * 32) + threadIdx.x, threads = (int64_t)gridDim.x * (RG_WARPS * 32);
  if (a.offsets) {
    if (tid < 2) a.offsets[tid] = tid ? (int32_t)a.s.N : 0;
    if (tid <= a.ranges) a.offsets[2 + tid] = (int32_t)min(a.s.N, tid * (int64_t)a.range);
  }
  if (a.w2) {
    const int64_t half = (int64_t)a.Eq * a.d, have = (int64_t)E * a.d;       // (Eq is a multiple of 8: both in whole vectors)
    const bool vec = have % 8 == 0;
    for (int64_t i = tid * 8; i < half; i += threads * 8) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (vec) {
        if (i < have) v = *reinterpret_cast<const uint4*>(a.w + i);
      } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = i + j < have ? __bfloat162float(a.w[i + j]) : 0.f;
        v = Vec16<__nv_bfloat16>::store(f);
      }
      *reinterpret_cast<uint4*>(a.w2 + i) = v;
      *reinterpret_cast<uint4*>(a.w2 + half + i) = v;
    }
  }
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
        if (a.pair && e < a.Eq) {
          const __nv_bfloat16 hi = __float2bfloat16_rn(dl);
          a.pair[t * 2 * a.Eq + e] = hi;
          a.pair[t * 2 * a.Eq + a.Eq + e] = __float2bfloat16_rn(dl - __bfloat162float(hi));
        }
      }
    }
    __syncwarp();                            // the rows are rewritten for the next tokens
  }
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

// ---------------------------------------------------------------- up to 32 experts, plain FMAs
// A thread owns V columns: their W_r and dW_r (EM >= E experts each, 128 registers at most) stay in its registers, x goes by once.  A
// block is `tx` threads across the columns by `ty` tokens at a time; it walks a range of tokens in chunks, whose dl it makes first
// in shared memory.  4 E FMAs an element of x and dx: bound by HBM up to 8 experts or so as long as enough loads are in flight (U
// tokens a thread), by the FMAs beyond.
constexpr int FEW_N = 256;                   // threads
constexpr int FEW_TOK = 64;                  // tokens of a chunk
constexpr int FEW_MAX_E = 32;
template <int EM> constexpr int few_v = EM <= 16 ? 4 : 2;

template <int BYTES> struct Word;
template <> struct Word<16> { using type = uint4; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<4> { using type = uint32_t; };
// V columns as they are stored, `step` apart (1 with VEC, which takes them in one access); without VEC columns that do not exist
// repeat the first.
template <typename T, bool VEC, int V> struct Few {
  using W = typename Word<V * (int)sizeof(T)>::type;
  T v[V];
  __device__ __forceinline__ void load(const T* p, int step, int left) {
    if constexpr (VEC) {
      const W w = *reinterpret_cast<const W*>(p);
      memcpy(v, &w, sizeof(W));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = p[j * step < left ? j * step : 0];
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = to_float(v[j]);
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = from_float<T>(f[j]);
  }
  __device__ __forceinline__ void store(T* p, int step, int left) const {
    if constexpr (VEC) {
      W w;
      memcpy(&w, v, sizeof(W));
      *reinterpret_cast<W*>(p) = w;
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j * step < left) p[j * step] = v[j];
    }
  }
};

template <typename T>
struct FewArgs {
  ScoreGrad s;
  const T *x, *w;
  int d, tx, per;                            // per: tokens of a range
  T* dx;
  float *dlogits, *parts, *dbias_part;       // parts [ranges][E][d], dbias_part [ranges][E]
};

template <typename T, bool VEC, int EM>
__global__ void __launch_bounds__(FEW_N, EM == 8 ? 2 : 1) k_route_grad_few(const FewArgs<T> a) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int V = few_v<EM>;
  constexpr int U = 8;                       // tokens in flight
  constexpr int P = 4 / V;                   // sums of dx that run side by side: four chains of FMAs whatever V
  constexpr int G = EM < 32 ? EM : 32, EPL = EM / G;                    // lanes of a token's dl, experts of a lane
  constexpr int BY = FEW_N / G, EACH = FEW_TOK / BY;                    // tokens at a time, and of a thread
  __shared__ __align__(16) float dl[FEW_TOK][EM];
  __shared__ float sum[FEW_N][V > EPL ? V : EPL];
  const int E = a.s.E, d = a.d, tx = a.tx, ty = FEW_N / tx, cx = threadIdx.x & (tx - 1), cy = threadIdx.x / tx;
  const int step = VEC ? 1 : tx, c = (int)blockIdx.x * tx * V + (VEC ? cx * V : cx), left = d - c;
  const bool cols = left > 0;
  const int range = blockIdx.y;
  const int64_t first = (int64_t)range * a.per, last = min(a.s.N, first + a.per);
  const int e0 = threadIdx.x & (G - 1), i0 = threadIdx.x / G;
  float w[EM][V], dw[EM][V], bias[EPL];
#pragma unroll
  for (int m = 0; m < EPL; ++m) bias[m] = 0.f;
#pragma unroll
  for (int e = 0; e < EM; ++e) {
#pragma unroll
    for (int j = 0; j < V; ++j) w[e][j] = dw[e][j] = 0.f;
    if (e < E && cols) {
      Few<T, VEC, V> q;
      q.load(a.w + (int64_t)e * d + c, step, left);
      q.get(w[e]);
    }
  }
  for (int64_t t0 = first; t0 < last; t0 += FEW_TOK) {
    const int n = (int)min((int64_t)FEW_TOK, last - t0);
    float s[EACH][EPL];
    __syncthreads();                         // the last chunk's dl has been read
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int m = 0; m < EPL; ++m) {
        const int i = i0 + k * BY, e = e0 + m * G;
        const bool mine = i < n && e < E;
        s[k][m] = mine ? a.s.scores[(t0 + i) * E + e] : 0.f;
        dl[i][e] = mine && a.s.dscores ? a.s.dscores[(t0 + i) * a.s.dscores_ld + e] : 0.f;
      }
    __syncthreads();
    add_kept(a.s, t0, n, threadIdx.x, FEW_N, &dl[0][0], EM);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = i0 + k * BY;
      float g[EPL], dot = 0.f;
#pragma unroll
      for (int m = 0; m < EPL; ++m) {
        g[m] = dl[i][e0 + m * G];
        dot = fmaf(s[k][m], g[m], dot);
      }
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
#pragma unroll
      for (int m = 0; m < EPL; ++m) {
        const int e = e0 + m * G;
        const bool mine = i < n && e < E;
        const float v = mine ? s[k][m] * (g[m] - dot) : 0.f;
        dl[i][e] = v;
        bias[m] += v;
        if (mine && blockIdx.x == 0) a.dlogits[(t0 + i) * E + e] = v;
      }
    }
    __syncthreads();
    auto fetch = [&](Few<T, VEC, V>& x, int i) { x.load(a.x + (t0 + min(i, n - 1)) * d + c, step, left); };
    auto work = [&](int i, const Few<T, VEC, V>& x) {
      float f[V], y[P][V];
      x.get(f);
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) y[p][j] = 0.f;
#pragma unroll
      for (int e4 = 0; e4 < EM; e4 += 4) {
        const float4 q = *reinterpret_cast<const float4*>(&dl[i][e4]);
        const float l[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            y[m % P][j] = fmaf(l[m], w[e4 + m][j], y[m % P][j]);
            dw[e4 + m][j] = fmaf(l[m], f[j], dw[e4 + m][j]);
          }
      }
#pragma unroll
      for (int p = 1; p < P; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) y[0][j] += y[p][j];
      Few<T, VEC, V> out;
      out.set(y[0]);
      out.store(a.dx + (t0 + i) * d + c, step, left);
    };
    if (cols) {
      if constexpr (EM <= 16) {
        for (int i1 = cy; i1 < n; i1 += ty * U) {
          Few<T, VEC, V> x[U];
#pragma unroll
          for (int u = 0; u < U; ++u) fetch(x[u], i1 + u * ty);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (i1 + u * ty >= n) break;
            work(i1 + u * ty, x[u]);
          }
        }
      } else {                               // a token is hundreds of instructions: eight of them side by side would miss the instruction cache
        Few<T, VEC, V> x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) fetch(x[u], cy + u * ty);
#pragma unroll 1
        for (int i = cy; i < n; i += ty) {
          const Few<T, VEC, V> now = x[0];
          x[0] = x[1]; x[1] = x[2]; x[2] = x[3];
          fetch(x[3], i + 4 * ty);
          work(i, now);
        }
      }
    }
  }
  // the ty shares of dW_r in their order, then a part
  float* part = a.parts + (int64_t)range * E * d;
#pragma unroll
  for (int e = 0; e < EM; ++e) {
    if (ty > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) sum[threadIdx.x][j] = dw[e][j];
      __syncthreads();
      if (cy == 0)
        for (int k = 1; k < ty; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) dw[e][j] += sum[cx + k * tx][j];
    }
    if (cy == 0 && e < E && cols) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j * step < left) part[(int64_t)e * d + c + j * step] = dw[e][j];
    }
  }
  if (blockIdx.x == 0) {
    __syncthreads();
#pragma unroll
    for (int m = 0; m < EPL; ++m) sum[threadIdx.x][m] = bias[m];
    __syncthreads();
    if (threadIdx.x < E) {
      float b = 0.f;
      for (int k = threadIdx.x & (G - 1); k < FEW_N; k += G) b += sum[k][threadIdx.x / G];
      a.dbias_part[(int64_t)range * E + threadIdx.x] = b;
    }
  }
}

// dW_r [E, d] from parts [ranges][copies][rows][d] (copies = 2: both halves of dl) and, in the blocks behind, dbias [E] from parts
// [bias_parts][E], all in a fixed order.
constexpr int JOIN_N = 256, JOIN_E = 8;      // threads; experts of a block for dbias
constexpr int JOIN_G = 8;                    // threads that share an output's parts (every JOIN_G-th each, their loads in flight together)
template <typename TO, int VW>
__global__ void __launch_bounds__(JOIN_N) k_join_route(const float* __restrict__ part, int parts, int64_t each, int64_t size, int dw_blocks,
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
          const float4 v = __ldcs(reinterpret_cast<const float4*>(part + p * each + i));
          s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
        } else {
          s[0] += part[p * each + i];
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
int join_run(const float* part, int parts, int64_t each, int64_t size, void* dw, const float* bias_part, int bias_parts, int E, float* dbias,
             cudaStream_t st) {
  const bool wide = each % 4 == 0 && size % 4 == 0;
  const int64_t dw_blocks = parts ? ceil_div(size, (int64_t)(JOIN_N / JOIN_G) * (wide ? 4 : 1)) : 0, blocks = dw_blocks + ceil_div(E, JOIN_E);
  if (blocks > 0x7fffffff) return CAPMOE_EUNSUPPORTED;
  auto k = wide ? k_join_route<TO, 4> : k_join_route<TO, 1>;
  const int rc = note_cuda(launch_chained(k, (unsigned)blocks, JOIN_N, 0, st, part, parts, each, size, (int)dw_blocks, (TO*)dw, bias_part, bias_parts, E,
                                          dbias));
  count_launch(1);
  return rc;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

enum Form { FEW, TC, GENERAL };
struct RouteWs {
  Form form;
  int copies, Eq, ranges, blocks;            // general form, tensor cores: blocks of the logits' kernel
  size_t offsets, bias, pair, w2, parts, dw, dw_bytes, total;
};
int few_columns(int E) { return E <= 16 ? few_v<16> : few_v<32>; }                               // of a thread
int few_tx(int d, int E) {
  int tx = 32;
  while (tx < FEW_N && tx * few_columns(E) < d) tx *= 2;
  return tx;
}
RouteWs route_ws(int64_t N, int d, int E, int dtype) {
  RouteWs w = {};
  const bool bf16 = dtype == CAPMOE_BF16;
  w.form = route_grad_tc_supported(d, dtype) ? TC : E <= FEW_MAX_E ? FEW : GENERAL;
  w.copies = w.form != FEW && bf16 ? 2 : 1;
  w.Eq = w.copies == 2 ? (E + 7) / 8 * 8 : E;                // rows of `pair` in whole 16-byte vectors
  const int64_t sms = sm_count();
  if (w.form == FEW) {
    // two blocks per SM; 32 tokens each at least, or a part of dW_r would be as long as its tokens
    const int64_t across = ceil_div(d, few_tx(d, E) * few_columns(E)), want = 2 * sms / across, most = ceil_div(N, 32);
    int64_t r = want < most ? want : most;
    if (r < 1) r = 1;
    if (r > 65535) r = 65535;
    w.ranges = (int)ceil_div(N, ceil_div(N, r));
  } else if (w.form == TC) {
    w.ranges = route_grad_tc_ranges(N, d, E);
  } else {
    // plain FMAs: tiles of 32 x 64 for four blocks per SM, 128 tokens each at least (fp32, 64 experts: 4096 tokens of 1024 columns
    // 55.7 us, 58.0 with twice the ranges; 21,900 tokens of 96 columns 43, 50 with 512 tokens each at least)
    const int64_t want = sms * 4 / (ceil_div(d, 64) * ceil_div(w.copies * w.Eq, 32)), most = N / 128;
    const int64_t r = want < most ? want : most;
    w.ranges = (int)(r < 1 ? 1 : r > 64 ? 64 : r);
  }
  const int64_t want = ceil_div(N, RG_WARPS * RG_TOK), most = sms * RG_BLOCKS;
  w.blocks = w.form == FEW ? w.ranges : (int)(want < most ? want : most);
  if (w.ranges < 1) w.ranges = 1;
  if (w.blocks < 1) w.blocks = 1;
  w.bias = w.form == GENERAL ? up256((size_t)(w.ranges + 3) * 4) : 0;
  w.pair = w.bias + up256((size_t)w.blocks * E * 4);
  w.w2 = w.pair + (w.copies == 2 ? up256((size_t)N * 2 * w.Eq * 2) : 0);
  w.parts = w.w2 + (w.form == GENERAL && bf16 ? up256((size_t)2 * w.Eq * d * 2) : 0);
  const size_t rows = w.form == GENERAL ? (size_t)w.copies * w.Eq : (size_t)E;
  w.dw = w.parts + up256((size_t)w.ranges * rows * d * 4);
  if (w.form == GENERAL) capmoe_grouped_mm_dw_workspace_bytes(w.ranges, &w.dw_bytes);
  w.total = w.dw + up256(w.dw_bytes) + 256;                  // 256: to align all of it
  return w;
}

template <typename T>
int few_run(const ScoreGrad& s, const void* x, const void* w, int d, const RouteWs& ws, uint8_t* b, float* dlogits, void* dx, cudaStream_t st) {
  const FewArgs<T> a{s, (const T*)x, (const T*)w, d, few_tx(d, s.E), (int)ceil_div(s.N, ws.ranges), (T*)dx, dlogits, (float*)(b + ws.parts), (float*)(b + ws.bias)};
  const int V = few_columns(s.E);
  const bool vec = d % V == 0;
  auto k = s.E <= 8    ? (vec ? k_route_grad_few<T, true, 8> : k_route_grad_few<T, false, 8>)
           : s.E <= 16 ? (vec ? k_route_grad_few<T, true, 16> : k_route_grad_few<T, false, 16>)
                       : (vec ? k_route_grad_few<T, true, 32> : k_route_grad_few<T, false, 32>);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ceil_div(d, a.tx * V), (unsigned)ws.ranges);
  cfg.blockDim = dim3(FEW_N);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const int rc = note_cuda(cudaLaunchKernelEx(&cfg, k, a));
  count_launch(1);
  return rc;
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
  const bool bf16 = dtype == CAPMOE_BF16;
  const ScoreGrad sg{scores, dweight, dscores, topk_idx, slot_row, token_group, N, A_max, dscores_ld, E, k, slots, D};
  float *parts = (float*)(b + w.parts), *bias = (float*)(b + w.bias);
  if (w.form == FEW) {
    rc = bf16 ? few_run<__nv_bfloat16>(sg, x, w_router, d, w, b, dlogits, dx, st) : few_run<float>(sg, x, w_router, d, w, b, dlogits, dx, st);
  } else {
    LogitArgs a = {};
    a.s = sg;
    a.dlogits = dlogits; a.dbias_part = bias;
    a.pair = bf16 ? (__nv_bfloat16*)(b + w.pair) : nullptr;
    a.Eq = w.Eq; a.d = d;
    if (w.form == GENERAL) {
      a.offsets = (int32_t*)b; a.ranges = w.ranges; a.range = (int)ceil_div(N, w.ranges);
      if (bf16) { a.w = (const __nv_bfloat16*)w_router; a.w2 = (__nv_bfloat16*)(b + w.w2); }
    }
    auto kernel = E <= 32 ? k_route_logit_grad<1> : E <= 64 ? k_route_logit_grad<2> : E <= 128 ? k_route_logit_grad<4> : k_route_logit_grad<8>;
    rc = note_cuda(launch_chained(kernel, (unsigned)w.blocks, RG_WARPS * 32, 0, st, a));
    count_launch(1);
    if (rc != CAPMOE_OK) return rc;
    if (w.form == TC) {
      rc = route_grad_tc(a.pair, x, w_router, N, d, E, w.Eq, w.ranges, dx, parts, dev_status, st);
    } else {
      const int n = w.copies * w.Eq;
      const void *dl = bf16 ? (const void*)a.pair : dlogits, *wr = bf16 ? (const void*)a.w2 : w_router;
      rc = capmoe_grouped_mm_dx(dl, a.offsets, wr, 1, d, n, dtype, dx, N, dev_status, stream);
      if (rc == CAPMOE_OK)
        rc = capmoe_grouped_mm_dw(dl, x, a.offsets + 2, w.ranges, d, n, dtype, CAPMOE_F32, parts, N, b + w.dw, w.dw_bytes, dev_status, stream);
    }
  }
  if (rc != CAPMOE_OK) return rc;
  // (the grouped product's parts hold a range's two halves one behind the other, of Eq rows each)
  const int copies = w.form == GENERAL ? w.copies : 1;
  const int64_t each = (int64_t)(w.form == GENERAL ? w.Eq : E) * d, size = (int64_t)E * d;
  return out_dtype == CAPMOE_F32 ? join_run<float>(parts, w.ranges * copies, each, size, dw, bias, w.blocks, E, dbias, st)
                                 : join_run<__nv_bfloat16>(parts, w.ranges * copies, each, size, dw, bias, w.blocks, E, dbias, st);
}
