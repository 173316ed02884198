// 8-bit form of the grouped products: e4m3 values with one power-of-two scale per 128 columns of an
// activation row, or per 128 x 128 block of a weight matrix.
//   scale 2^e, e the smallest with max|block| <= 448 * 2^e;  q = e4m3(v * 2^-e), round to nearest even
// The product with a power of two is exact, so a value has one rounding, its own to e4m3 (at most 2^-4 of
// it), and the codes do not depend on how a division rounds.  A block that holds a NaN or an infinity
// becomes NaN as a whole.
// This file: the two quantisers, the host side, and the plain-FMA kernels for sizes the tensor-core
// kernels do not take.
#include "gmm_simt.cuh"

namespace capmoe {
namespace {

using G8 = Geo<ST, 8>;                     // block of the fallback product
constexpr int QN = 256;                    // threads of the quantisers
constexpr int Q_MAX = 0x7fffffff - 1023;   // columns, rows of a weight: 32 bits after rounding up to eight blocks of 128

// Eight consecutive elements of a row, kept as they are stored until they are used (half the registers of fp32 for bf16,
// so more loads in flight): 16-byte loads with VEC, else the first `left` one by one.
template <typename T, bool VEC>
struct Eight {
  uint32_t w[sizeof(T) * 2];
  __device__ __forceinline__ void load(const T* p, int left) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4*>(p) + i);
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
      }
    } else {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? to_float(p[i]) : 0.f;
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) * 2; ++i)
        w[i] = sizeof(T) == 4 ? __float_as_uint(v[i]) : (__float_as_uint(v[2 * i % 8]) >> 16) | (__float_as_uint(v[(2 * i + 1) % 8]) & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; ++i) w[i] = 0u;
  }
  // bit pattern of the largest magnitude: of non-negative floats the larger has the larger pattern; NaN is above all
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(w);
      const __nv_bfloat162 m2 = __hmax2_nan(__hmax2_nan(__habs2(h[0]), __habs2(h[1])), __hmax2_nan(__habs2(h[2]), __habs2(h[3])));
      const uint32_t m = *reinterpret_cast<const uint32_t*>(&m2);
      return max(m << 16, m & 0xffff0000u);
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
      return m;
    }
  }
  // codes of elements 2i (low byte) and 2i + 1 under scale code `code` (a power of two: exact in bf16 as in fp32, but for
  // results below 2^-126, which become zero codes either way)
  __device__ __forceinline__ uint32_t codes(int i, uint32_t code) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t f = (254u - code) << 7, f2 = f | f << 16;
      const __nv_bfloat162 p = __hmul2(reinterpret_cast<const __nv_bfloat162*>(w)[i], *reinterpret_cast<const __nv_bfloat162*>(&f2));
      const uint32_t q = *reinterpret_cast<const uint32_t*>(&p);
      return to_e4m3x2(__uint_as_float(q << 16), __uint_as_float(q & 0xffff0000u));
    } else {
      const float f = inv_scale(code);
      return to_e4m3x2(__uint_as_float(w[2 * i]) * f, __uint_as_float(w[2 * i + 1]) * f);
    }
  }
};

template <typename T, bool VEC>
__device__ __forceinline__ void store8(uint8_t* p, int left, const Eight<T, VEC>& v, uint32_t code) {
  uint32_t lo = 0x7f7f7f7fu, hi = 0x7f7f7f7fu;
  if (code != (uint32_t)Q_NAN_SCALE) {
    lo = v.codes(0, code) | (v.codes(1, code) << 16);
    hi = v.codes(2, code) | (v.codes(3, code) << 16);
  }
  if constexpr (VEC) {
    *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = (uint8_t)((i < 4 ? lo >> (8 * i) : hi >> (8 * (i - 4))) & 0xffu);
  }
}

// Rows: half a warp per block of 128 columns, a warp per QROW_U pairs of blocks, all of them in flight.  Bound by HBM (3
// bytes per bf16 element; 42,700 of 98,000 allocated rows of 2048: 46 us, 0.87 of the copy bandwidth) and, close behind,
// by instructions: bf16 is searched and scaled two at a time.  The grid is about two blocks to each one that is resident and
// walks the rows that exist (a block per unit of allocated rows took 56 us there, a grid that is just resident 50).
constexpr int QROW_U = 4;
template <typename T, bool VEC>
__global__ void __launch_bounds__(QN)
k_quantize_rows(const T* __restrict__ x, const int32_t* __restrict__ n_rows, int rows, int d, uint32_t per_row, uint8_t* __restrict__ q,
                uint8_t* __restrict__ scale, int64_t scale_ld) {
  wait_for_previous_kernel();
  allow_next_kernel();                       // in this order: an early successor reads what came before (gmm.cuh)
  const int lane = threadIdx.x & 31, sub = lane & 15;
  const int nb = (d + QBLOCK - 1) / QBLOCK;
  if (n_rows) rows = min(rows, *n_rows);
  for (uint32_t unit = blockIdx.x * (QN / 32) + (threadIdx.x >> 5);; unit += gridDim.x * (QN / 32)) {
    const uint32_t row = unit / per_row;
    if ((int64_t)row >= rows) return;
    const int64_t r = row;
    const int b0 = (int)(unit - row * per_row) * 2 * QROW_U + (lane >> 4);
    Eight<T, VEC> v[QROW_U];
#pragma unroll
    for (int u = 0; u < QROW_U; ++u) {
      const int c = (b0 + 2 * u) * QBLOCK + sub * 8;
      if (c < d) v[u].load(x + r * d + c, d - c);
      else v[u].clear();
    }
#pragma unroll
    for (int u = 0; u < QROW_U; ++u) {
      const int b = b0 + 2 * u, c = b * QBLOCK + sub * 8;
      uint32_t m = v[u].top();
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const uint32_t code = scale_code(m);
      if (c < d) store8(q + r * d + c, d - c, v[u], code);
      if (sub == 0 && b < nb) scale[r * scale_ld + b] = (uint8_t)code;
    }
  }
}

// Weights: one CTA per 128 x 128 block, the whole block in registers (eight passes of 16 rows).  Bound by HBM.
template <typename T, bool VEC>
__global__ void __launch_bounds__(QN, sizeof(T) == 2 ? 3 : 2)
k_quantize_weights(const T* __restrict__ w, int n, int d, uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
  allow_next_kernel();
  wait_for_previous_kernel();
  __shared__ uint32_t part[QN / 32];
  const int db = (d + QBLOCK - 1) / QBLOCK, nb = (n + QBLOCK - 1) / QBLOCK;
  const int64_t blk = blockIdx.x;
  const int jb = (int)(blk % db), ib = (int)(blk / db % nb);
  const int64_t e = blk / db / nb;
  const int c = jb * QBLOCK + (threadIdx.x & 15) * 8, r0 = ib * QBLOCK + (threadIdx.x >> 4);
  const int64_t base = e * n * d;
  Eight<T, VEC> v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < n && c < d) v[i].load(w + base + (int64_t)r * d + c, d - c);
    else v[i].clear();
  }
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, v[i].top());
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QN / 32; ++i) m = max(m, part[i]);
  const uint32_t code = scale_code(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < n && c < d) store8(q + base + (int64_t)r * d + c, d - c, v[i], code);
  }
  if (threadIdx.x == 0) scale[blk] = (uint8_t)code;
}

// y = x W^T from codes; SWIGLU: silu(x W_g^T) * (x W_u^T)
template <typename TO, bool SWIGLU>
__global__ void __launch_bounds__(G8::SN)
k_mm_fp8(const uint8_t* __restrict__ xq, const uint8_t* __restrict__ xs, const uint8_t* __restrict__ w0,
         const uint8_t* __restrict__ s0, const uint8_t* __restrict__ w1, const uint8_t* __restrict__ s1, TO* __restrict__ out,
         Segments sg, int K, int Nout) {
  wait_for_previous_kernel();
  SimtTile<G8>& sm = simt_tile<G8>();
  RowTile t;
  if (!find_row_tile<G8>(sg, blockIdx.x, t)) return;
  const int col0 = blockIdx.y * ST, kb = (K + QBLOCK - 1) / QBLOCK, nb = (Nout + QBLOCK - 1) / QBLOCK;
  const Coded<1> la{xq + (int64_t)t.row0 * K, xs + (int64_t)t.row0 * kb, K, kb};
  const int64_t wo = ((int64_t)t.e * Nout + col0) * K, so = ((int64_t)t.e * nb + col0 / QBLOCK) * kb;
  constexpr int R = G8::R;
  float acc[R][4], up[R][4];
  clear_acc(acc);
  // (a 64-column tile lies inside one block of 128 weight rows: one row of scales serves it)
  tile_product<G8>(la, Coded<QBLOCK>{w0 + wo, s0 + so, K, kb}, t.rows, Nout - col0, K, sm, acc);
  if (SWIGLU) {
    clear_acc(up);
    tile_product<G8>(la, Coded<QBLOCK>{w1 + wo, s1 + so, K, kb}, t.rows, Nout - col0, K, sm, up);
  }
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = out_row<G8>(i), c = col0 + out_col<G8>(j);
      float v = acc[i][j];
      if (SWIGLU) v = v / (1.0f + expf(-v)) * up[i][j];
      if (r < t.rows && c < Nout) out[(int64_t)(t.row0 + r) * Nout + c] = from_float<TO>(v);
    }
}

template <typename T>
int quantize_rows_run(const void* x, const int32_t* n_rows, int64_t rows, int d, void* q, void* scale, int64_t scale_ld, cudaStream_t st) {
  const uint32_t per_row = (uint32_t)ceil_div(ceil_div(d, QBLOCK), 2 * QROW_U);
  if (rows * per_row >= (int64_t)1 << 31) return CAPMOE_EUNSUPPORTED;
  const int64_t want = ceil_div(rows * per_row, QN / 32), most = (int64_t)sm_count() * 16;
  const unsigned grid = (unsigned)(want < most ? want : most);
  // 16-byte loads of eight columns need rows that start on 16 bytes; the codes' rows then start on 8
  const int rc = note_cuda(d % 8 == 0 ? launch_chained(k_quantize_rows<T, true>, grid, QN, 0, st, (const T*)x, n_rows, (int)rows, d,
                                                       per_row, (uint8_t*)q, (uint8_t*)scale, scale_ld)
                                      : launch_chained(k_quantize_rows<T, false>, grid, QN, 0, st, (const T*)x, n_rows, (int)rows, d,
                                                       per_row, (uint8_t*)q, (uint8_t*)scale, scale_ld));
  count_launch(1);
  return rc;
}

template <typename T>
int quantize_weights_run(const void* w, int E, int n, int d, void* q, void* scale, cudaStream_t st) {
  const int64_t grid = (int64_t)E * ceil_div(n, QBLOCK) * ceil_div(d, QBLOCK);
  if (grid >= ((int64_t)1 << 31)) return CAPMOE_EUNSUPPORTED;
  const int rc = note_cuda(d % 8 == 0 ? launch_chained(k_quantize_weights<T, true>, (unsigned)grid, QN, 0, st, (const T*)w, n, d,
                                                       (uint8_t*)q, (uint8_t*)scale)
                                      : launch_chained(k_quantize_weights<T, false>, (unsigned)grid, QN, 0, st, (const T*)w, n, d,
                                                       (uint8_t*)q, (uint8_t*)scale));
  count_launch(1);
  return rc;
}

template <class... KArgs, class... Args>
int launch_tiles(void (*kernel)(KArgs...), const Segments& sg, int cols, cudaStream_t st, Args... args) {
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SimtTile<G8>));
  if (err != cudaSuccess) return note_cuda(err);
  cudaLaunchConfig_t cfg = {};
  cfg.dynamicSmemBytes = sizeof(SimtTile<G8>);
  cfg.gridDim = dim3((unsigned)(ceil_div(sg.rows, ST) + sg.E), (unsigned)ceil_div(cols, ST));
  cfg.blockDim = dim3(G8::SN);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const int rc = note_cuda(cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...));
  count_launch(1);
  return rc;
}

int check_shape(const int32_t* offsets, int E, int d, int n, int64_t rows) {
  if (E < 1 || d < 1 || n < 1 || rows < 0 || !offsets) return CAPMOE_EINVAL;
  if (E > GMM_MAX_E || rows > GMM_MAX_ROWS || ceil_div(d, ST) > 65535 || ceil_div(n, ST) > 65535)
    return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}
template <class... P>
bool usable(P... p) {
  return ((p != nullptr && aligned16(p)) && ...);
}

// Workspace of the 8-bit FFN: codes and scales of x and of the hidden rows, and (sizes without a
// tensor-core kernel) the hidden rows in fp32.  Rows of scales start on 16 bytes (one load for 16 of them: with packed rows
// of 11 the down product of 43,000 rows took 100 us more), except where the fallback product reads them.
struct FfnWs { size_t xq, xs, hq, hs, h, total; int64_t xs_ld, hs_ld; };
FfnWs ffn_ws(int64_t A_max, int d, int F) {
  auto up = [](size_t b) { return (b + 255) / 256 * 256; };
  const size_t A = (size_t)A_max;
  FfnWs w;
  const int64_t pad = gmm8_supported(d, F) ? 16 : 1;
  w.xs_ld = ceil_div(ceil_div(d, QBLOCK), pad) * pad;
  w.hs_ld = ceil_div(ceil_div(F, QBLOCK), pad) * pad;
  w.xq = 0;
  w.xs = w.xq + up(A * d);
  w.hq = w.xs + up(A * w.xs_ld);
  w.hs = w.hq + up(A * F);
  w.h = w.hs + up(A * w.hs_ld);
  w.total = w.h + (gmm8_supported(d, F) ? 0 : up(A * F * 4)) + 256;
  return w;
}

}  // namespace
}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_quantize_rows(const void* x, const int32_t* n_rows, int64_t rows, int d, int dtype, void* q, void* scale,
                                    void* stream) {
  if (rows < 0 || d < 1) return CAPMOE_EINVAL;
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  if (rows >= ((int64_t)1 << 31) || d > Q_MAX) return CAPMOE_EUNSUPPORTED;
  if (rows == 0) return CAPMOE_OK;
  if (!usable(x, q) || !scale) return CAPMOE_EINVAL;
  if (dtype == CAPMOE_F32) return quantize_rows_run<float>(x, n_rows, rows, d, q, scale, ceil_div(d, QBLOCK), as_stream(stream));
  return quantize_rows_run<__nv_bfloat16>(x, n_rows, rows, d, q, scale, ceil_div(d, QBLOCK), as_stream(stream));
}

extern "C" int capmoe_quantize_weights(const void* w, int E, int n, int d, int dtype, void* q, void* scale, void* stream) {
  if (E < 1 || n < 1 || d < 1) return CAPMOE_EINVAL;
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  if (n > Q_MAX || d > Q_MAX) return CAPMOE_EUNSUPPORTED;
  if (!usable(w, q) || !scale) return CAPMOE_EINVAL;
  if (dtype == CAPMOE_F32) return quantize_weights_run<float>(w, E, n, d, q, scale, as_stream(stream));
  return quantize_weights_run<__nv_bfloat16>(w, E, n, d, q, scale, as_stream(stream));
}

extern "C" int capmoe_grouped_mm_fp8(const void* x_q, const void* x_scale, const int32_t* expert_offsets, const void* w_q,
                                     const void* w_scale, int E, int d, int n, void* y, int64_t rows, int32_t* dev_status,
                                     void* stream) {
  int rc = check_shape(expert_offsets, E, d, n, rows);
  if (rc != CAPMOE_OK || rows == 0) return rc;
  if (!usable(x_q, w_q, y) || !x_scale || !w_scale) return CAPMOE_EINVAL;
  const Segments sg{expert_offsets, E, (int)rows};
  if (gmm8_supported(d, n)) {
    int32_t* counters = counters_of(sg, dev_status);
    if ((rc = begin_counters(counters, 1, as_stream(stream))) != CAPMOE_OK) return rc;
    return gmm8((const uint8_t*)x_q, (const uint8_t*)x_scale, ceil_div(d, QBLOCK), sg, (const uint8_t*)w_q, (const uint8_t*)w_scale, d, n, y,
                dev_status, counter_at(counters, 0), false, as_stream(stream));
  }
  const uint8_t* none = nullptr;
  return launch_tiles(k_mm_fp8<__nv_bfloat16, false>, sg, n, as_stream(stream), (const uint8_t*)x_q, (const uint8_t*)x_scale,
                      (const uint8_t*)w_q, (const uint8_t*)w_scale, none, none, (__nv_bfloat16*)y, sg, d, n);
}

extern "C" int capmoe_ffn_fp8_workspace_bytes(int64_t A_max, int d, int F, size_t* bytes) {
  if (!bytes || A_max < 0 || d < 1 || F < 1) return CAPMOE_EINVAL;
  *bytes = ffn_ws(A_max, d, F).total;
  return CAPMOE_OK;
}

extern "C" int capmoe_grouped_ffn_fp8(const void* x_perm, const int32_t* expert_offsets, int E, int d, int F, const void* wg_q,
                                      const void* wg_scale, const void* wu_q, const void* wu_scale, const void* wd_q,
                                      const void* wd_scale, void* y_perm, int64_t A_max, void* ws, size_t ws_bytes,
                                      int32_t* dev_status, void* stream) {
  int rc = check_shape(expert_offsets, E, d, F, A_max);
  if (rc != CAPMOE_OK || A_max == 0) return rc;
  if (!usable(x_perm, wg_q, wu_q, wd_q, y_perm, ws) || !wg_scale || !wu_scale || !wd_scale) return CAPMOE_EINVAL;
  const FfnWs w = ffn_ws(A_max, d, F);
  if (ws_bytes < w.total) return CAPMOE_EWORKSPACE;
  const Segments sg{expert_offsets, E, (int)A_max};
  cudaStream_t st = as_stream(stream);
  uint8_t* b = (uint8_t*)ws;
  const bool tc = gmm8_supported(d, F);
  int32_t* counters = counters_of(sg, dev_status);
  if (tc && (rc = begin_counters(counters, 2, st)) != CAPMOE_OK) return rc;
  rc = quantize_rows_run<__nv_bfloat16>(x_perm, expert_offsets + E, A_max, d, b + w.xq, b + w.xs, w.xs_ld, st);
  if (rc != CAPMOE_OK) return rc;
  if (tc) {
    rc = gmm8_swiglu(b + w.xq, b + w.xs, w.xs_ld, sg, (const uint8_t*)wg_q, (const uint8_t*)wg_scale, (const uint8_t*)wu_q,
                        (const uint8_t*)wu_scale, d, F, b + w.hq, b + w.hs, w.hs_ld, dev_status, counter_at(counters, 0), true, st);
    if (rc != CAPMOE_OK) return rc;
    return gmm8(b + w.hq, b + w.hs, w.hs_ld, sg, (const uint8_t*)wd_q, (const uint8_t*)wd_scale, F, d, y_perm, dev_status,
                counter_at(counters, 1), true, st);
  }
  float* h = (float*)(b + w.h);
  rc = launch_tiles(k_mm_fp8<float, true>, sg, F, st, b + w.xq, b + w.xs, (const uint8_t*)wg_q, (const uint8_t*)wg_scale,
                    (const uint8_t*)wu_q, (const uint8_t*)wu_scale, h, sg, d, F);
  if (rc != CAPMOE_OK) return rc;
  rc = quantize_rows_run<float>(h, expert_offsets + E, A_max, F, b + w.hq, b + w.hs, w.hs_ld, st);
  if (rc != CAPMOE_OK) return rc;
  const uint8_t* none = nullptr;
  return launch_tiles(k_mm_fp8<__nv_bfloat16, false>, sg, d, st, b + w.hq, b + w.hs, (const uint8_t*)wd_q,
                      (const uint8_t*)wd_scale, none, none, (__nv_bfloat16*)y_perm, sg, F, d);
}
