// Rows sorted by expert in 8 bits, and the gradients of the permutation and of the gate-weighted sum:
//   permute8      x_q[r] = q[t], scales with it, for the rows r = slot_row[t, s]
//   combine_grad  dy_perm[r] = w[r] dy[t],  dw[r] = dy[t] . y_perm[r]
//   permute_grad  dx[t] = sum_s dx_perm[slot_row[t, s]] + add0[t] + add1[t]
// Pure data movement, bound by HBM.  A token's row is read once for all its slots; every sum has a fixed order and fp32 terms.
#include "gmm.cuh"
#include "rowvec.cuh"

namespace capmoe {
namespace {

constexpr int TG_WARPS = 8;                  // warps of a block
constexpr int VPL = 4;                       // 16-byte vectors a lane holds of a row: chunks of 2 KB a warp
constexpr int CHUNK_VECS = 32 * VPL;
constexpr int MAX_SLOTS = 288;               // k + m <= 32 + 256

// A slot's row, or -1: also where it lies outside the buffers.
__device__ __forceinline__ int32_t slot_at(const int32_t* sr, int s, int slots, int64_t rows) {
  const int32_t r = s < slots ? sr[s] : -1;
  return r < rows ? r : -1;
}

__global__ void __launch_bounds__(TG_WARPS * 32)
k_permute8(const uint4* __restrict__ q, const uint8_t* __restrict__ scale, int64_t N, int row_vecs, int chunks, int nb, int E, int k,
           int slots, int D, int64_t rows, const float* __restrict__ scores, const int32_t* __restrict__ topk_idx,
           const int32_t* __restrict__ token_group, const int32_t* __restrict__ slot_row, uint4* __restrict__ q_perm,
           uint8_t* __restrict__ scale_perm, int32_t* __restrict__ perm_token, float* __restrict__ perm_weight) {
  allow_next_kernel();
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * TG_WARPS + (threadIdx.x >> 5);
  const int64_t t = unit / chunks;
  const int chunk = (int)(unit - t * chunks);
  if (t >= N) return;
  const int32_t* sr = slot_row + t * slots;
  const int v0 = chunk * CHUNK_VECS + lane;
  uint4 val[VPL];
  bool loaded = false;
  for (int s0 = 0; s0 < slots; s0 += 32) {
    const int32_t mine = slot_at(sr, s0 + lane, slots, rows);
    if (chunk == 0 && mine >= 0) {
      const int s = s0 + lane, m = D > 0 ? E / D : 0;
      const int e = s < k ? topk_idx[t * k + s] : home_group(t, N, D, token_group) * m + (s - k);
      perm_token[mine] = (int32_t)t;
      perm_weight[mine] = scores[t * E + e];
    }
    unsigned rem = __ballot_sync(0xffffffffu, mine >= 0);
    if (!rem) continue;
    if (!loaded) {                           // a token nobody keeps is never read
#pragma unroll
      for (int u = 0; u < VPL; ++u) val[u] = v0 + u * 32 < row_vecs ? __ldcs(q + t * row_vecs + v0 + u * 32) : make_uint4(0u, 0u, 0u, 0u);
      loaded = true;
    }
    while (rem) {
      const int b = __ffs(rem) - 1;
      rem &= rem - 1;
      const int64_t r = __shfl_sync(0xffffffffu, mine, b);
      uint4* dst = q_perm + r * row_vecs + v0;
#pragma unroll
      for (int u = 0; u < VPL; ++u)
        if (v0 + u * 32 < row_vecs) dst[u * 32] = val[u];
      if (chunk == 0)
        for (int i = lane; i < nb; i += 32) scale_perm[r * nb + i] = scale[t * nb + i];
    }
  }
}

// `wpt` warps to a token, each with every wpt-th chunk of its row: the chunk of dy stays in registers while the kept rows'
// chunks go by, two at a time.  Lane s of a group of 32 slots keeps slot s's share of the dot product.
template <typename T>
__global__ void __launch_bounds__(TG_WARPS * 32)
k_combine_grad(const uint4* __restrict__ dy, const uint4* __restrict__ y_perm, const int32_t* __restrict__ slot_row,
               const float* __restrict__ perm_weight, int64_t N, int row_vecs, int chunks, int slots, int64_t rows, int wpt,
               uint4* __restrict__ dy_perm, float* __restrict__ dweight) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int NV = Vec16<T>::n;
  __shared__ float part[TG_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp & (wpt - 1);
  const int64_t t = (int64_t)blockIdx.x * (TG_WARPS / wpt) + warp / wpt;
  const bool live = t < N;
  const int32_t* sr = slot_row + t * slots;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  for (int s0 = 0; s0 < slots; s0 += 32) {
    const int32_t mine = live ? slot_at(sr, s0 + lane, slots, rows) : -1;
    const float wmine = mine >= 0 ? perm_weight[mine] : 0.f;
    const unsigned kept = __ballot_sync(0xffffffffu, mine >= 0);
    float dot = 0.f;
    for (int chunk = sub; kept && chunk < chunks; chunk += wpt) {
      const int v0 = chunk * CHUNK_VECS + lane;
      float g[VPL][NV];
#pragma unroll
      for (int u = 0; u < VPL; ++u) Vec16<T>::load(v0 + u * 32 < row_vecs ? dy[t * row_vecs + v0 + u * 32] : zero, g[u]);
      unsigned rem = kept;
      while (rem) {
        const int b0 = __ffs(rem) - 1;
        rem &= rem - 1;
        const bool two = rem != 0;
        const int b1 = two ? __ffs(rem) - 1 : b0;
        rem &= rem - 1;                      // no-op when rem is already 0
        const int64_t r0 = __shfl_sync(0xffffffffu, mine, b0), r1 = __shfl_sync(0xffffffffu, mine, b1);
        const float w0 = __shfl_sync(0xffffffffu, wmine, b0), w1 = __shfl_sync(0xffffffffu, wmine, b1);
        uint4 raw0[VPL], raw1[VPL];
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
          const bool in = v0 + u * 32 < row_vecs;
          raw0[u] = in ? __ldcs(y_perm + r0 * row_vecs + v0 + u * 32) : zero;
          raw1[u] = in && two ? __ldcs(y_perm + r1 * row_vecs + v0 + u * 32) : zero;
        }
        float d0 = 0.f, d1 = 0.f;
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
          float f[NV];
          Vec16<T>::load(raw0[u], f);
#pragma unroll
          for (int i = 0; i < NV; ++i) d0 = fmaf(g[u][i], f[i], d0);
          Vec16<T>::load(raw1[u], f);
#pragma unroll
          for (int i = 0; i < NV; ++i) d1 = fmaf(g[u][i], f[i], d1);
          if (v0 + u * 32 < row_vecs) {
#pragma unroll
            for (int i = 0; i < NV; ++i) f[i] = w0 * g[u][i];
            dy_perm[r0 * row_vecs + v0 + u * 32] = Vec16<T>::store(f);
            if (two) {
#pragma unroll
              for (int i = 0; i < NV; ++i) f[i] = w1 * g[u][i];
              dy_perm[r1 * row_vecs + v0 + u * 32] = Vec16<T>::store(f);
            }
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          d0 += __shfl_xor_sync(0xffffffffu, d0, o);
          d1 += __shfl_xor_sync(0xffffffffu, d1, o);
        }
        if (lane == b0) dot += d0;
        if (two && lane == b1) dot += d1;
      }
    }
    if (wpt > 1) {                           // the warps' shares in their order
      __syncthreads();
      part[warp][lane] = dot;
      __syncthreads();
      dot = 0.f;
      for (int i = 0; i < wpt; ++i) dot += part[warp - sub + i][lane];
    }
    if (sub == 0 && mine >= 0) dweight[mine] = dot;
  }
}

// Work unit = (token, 2 KB chunk of its row), one warp each; two kept rows in flight.
template <typename T>
__global__ void __launch_bounds__(TG_WARPS * 32, 4)
k_permute_grad(const uint4* __restrict__ dx_perm, const int32_t* __restrict__ slot_row, int64_t N, int row_vecs, int chunks, int slots,
               int64_t rows, const uint4* add0, const uint4* add1, uint4* dx /* may be add0 or add1 */) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int NV = Vec16<T>::n;
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * TG_WARPS + (threadIdx.x >> 5);
  const int64_t t = unit / chunks;
  const int chunk = (int)(unit - t * chunks);
  if (t >= N) return;
  const int32_t* sr = slot_row + t * slots;
  const int v0 = chunk * CHUNK_VECS + lane;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  float acc[VPL][NV];
#pragma unroll
  for (int u = 0; u < VPL; ++u) {
    const bool in = v0 + u * 32 < row_vecs;
    Vec16<T>::load(add0 && in ? __ldcs(add0 + t * row_vecs + v0 + u * 32) : zero, acc[u]);
    if (add1) {
      float f[NV];
      Vec16<T>::load(in ? __ldcs(add1 + t * row_vecs + v0 + u * 32) : zero, f);
#pragma unroll
      for (int i = 0; i < NV; ++i) acc[u][i] += f[i];
    }
  }
  for (int s0 = 0; s0 < slots; s0 += 32) {
    const int32_t mine = slot_at(sr, s0 + lane, slots, rows);
    unsigned rem = __ballot_sync(0xffffffffu, mine >= 0);
    while (rem) {
      const int b0 = __ffs(rem) - 1;
      rem &= rem - 1;
      const bool two = rem != 0;
      const int b1 = two ? __ffs(rem) - 1 : b0;
      rem &= rem - 1;
      const int64_t r0 = __shfl_sync(0xffffffffu, mine, b0), r1 = __shfl_sync(0xffffffffu, mine, b1);
      uint4 raw0[VPL], raw1[VPL];
#pragma unroll
      for (int u = 0; u < VPL; ++u) {
        const bool in = v0 + u * 32 < row_vecs;
        raw0[u] = in ? __ldcs(dx_perm + r0 * row_vecs + v0 + u * 32) : zero;
        raw1[u] = in && two ? __ldcs(dx_perm + r1 * row_vecs + v0 + u * 32) : zero;
      }
#pragma unroll
      for (int u = 0; u < VPL; ++u) {
        float f[NV];
        Vec16<T>::load(raw0[u], f);
#pragma unroll
        for (int i = 0; i < NV; ++i) acc[u][i] += f[i];
        if (two) {
          Vec16<T>::load(raw1[u], f);
#pragma unroll
          for (int i = 0; i < NV; ++i) acc[u][i] += f[i];
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < VPL; ++u)
    if (v0 + u * 32 < row_vecs) dx[t * row_vecs + v0 + u * 32] = Vec16<T>::store(acc[u]);
}

int check_rows(int64_t N, int d, int slots, int64_t rows, size_t elt) {
  if (N < 0 || d < 1 || slots < 1 || rows < 0) return CAPMOE_EINVAL;
  if (slots > MAX_SLOTS || ((size_t)d * elt) % 16 != 0 || rows >= ((int64_t)1 << 31) || N >= ((int64_t)1 << 31)) return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}
template <class... P>
bool usable(P... p) {
  return ((p != nullptr && aligned16(p)) && ...);
}
int chunks_of(int row_vecs) { return (row_vecs + CHUNK_VECS - 1) / CHUNK_VECS; }

}  // namespace
}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_permute_fp8(const void* x_q, const void* x_scale, int64_t N, int d, int E, int k, int slots, int D, int64_t A_max,
                                  const float* scores, const int32_t* topk_idx, const int32_t* token_group, const int32_t* slot_row,
                                  void* q_perm, void* scale_perm, int32_t* perm_token, float* perm_weight, void* stream) {
  if (E < 1 || k < 1 || k > E || D < 0 || slots < k) return CAPMOE_EINVAL;
  if (D > 0 ? E % D != 0 || slots != k + E / D : slots != k) return CAPMOE_EINVAL;
  const int rc = check_rows(N, d, slots, A_max, 1);
  if (rc != CAPMOE_OK) return rc;
  if (N == 0) return CAPMOE_OK;
  if (!usable(x_q, q_perm) || !x_scale || !scale_perm || !scores || !topk_idx || !slot_row || !perm_token || !perm_weight) return CAPMOE_EINVAL;
  const int row_vecs = d / 16, chunks = chunks_of(row_vecs);
  const int64_t blocks = ceil_div(N * chunks, TG_WARPS);
  if (blocks > 0x7fffffff) return CAPMOE_EUNSUPPORTED;
  const int status = note_cuda(launch_chained(k_permute8, (unsigned)blocks, TG_WARPS * 32, 0, as_stream(stream), (const uint4*)x_q,
                                              (const uint8_t*)x_scale, N, row_vecs, chunks, (int)ceil_div(d, QBLOCK), E, k, slots, D, A_max,
                                              scores, topk_idx, token_group, slot_row, (uint4*)q_perm, (uint8_t*)scale_perm, perm_token,
                                              perm_weight));
  count_launch(1);
  return status;
}

extern "C" int capmoe_combine_backward(const void* dy, const void* y_perm, const int32_t* slot_row, const float* perm_weight, int64_t N, int d,
                                       int slots, int dtype, int64_t A_max, void* dy_perm, float* dweight, void* stream) {
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  const int rc = check_rows(N, d, slots, A_max, elt_size(dtype));
  if (rc != CAPMOE_OK) return rc;
  if (N == 0 || A_max == 0) return CAPMOE_OK;
  if (!usable(dy, y_perm, dy_perm) || !slot_row || !perm_weight || !dweight) return CAPMOE_EINVAL;
  const int row_vecs = (int)((size_t)d * elt_size(dtype) / 16), chunks = chunks_of(row_vecs);
  int wpt = 1;                               // more warps to a token while the tokens leave warps of the device without one
  while (wpt < TG_WARPS && wpt < chunks && N * wpt < (int64_t)sm_count() * 32) wpt *= 2;
  const int64_t blocks = ceil_div(N, TG_WARPS / wpt);
  if (blocks > 0x7fffffff) return CAPMOE_EUNSUPPORTED;
  auto k = dtype == CAPMOE_F32 ? k_combine_grad<float> : k_combine_grad<__nv_bfloat16>;
  const int status = note_cuda(launch_chained(k, (unsigned)blocks, TG_WARPS * 32, 0, as_stream(stream), (const uint4*)dy, (const uint4*)y_perm,
                                              slot_row, perm_weight, N, row_vecs, chunks, slots, A_max, wpt, (uint4*)dy_perm, dweight));
  count_launch(1);
  return status;
}

extern "C" int capmoe_permute_backward(const void* dx_perm, const int32_t* slot_row, int64_t N, int d, int slots, int dtype, int64_t A_max,
                                       const void* add0, const void* add1, void* dx, void* stream) {
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  const int rc = check_rows(N, d, slots, A_max, elt_size(dtype));
  if (rc != CAPMOE_OK) return rc;
  if (N == 0) return CAPMOE_OK;
  if (!usable(dx) || !slot_row || (A_max > 0 && !dx_perm) || !aligned16(dx_perm) || !aligned16(add0) || !aligned16(add1)) return CAPMOE_EINVAL;
  const int row_vecs = (int)((size_t)d * elt_size(dtype) / 16), chunks = chunks_of(row_vecs);
  const int64_t blocks = ceil_div(N * chunks, TG_WARPS);
  if (blocks > 0x7fffffff) return CAPMOE_EUNSUPPORTED;
  auto k = dtype == CAPMOE_F32 ? k_permute_grad<float> : k_permute_grad<__nv_bfloat16>;
  const int status = note_cuda(launch_chained(k, (unsigned)blocks, TG_WARPS * 32, 0, as_stream(stream), (const uint4*)dx_perm, slot_row, N, row_vecs,
                                              chunks, slots, A_max, (const uint4*)add0, (const uint4*)add1, (uint4*)dx));
  count_launch(1);
  return status;
}
