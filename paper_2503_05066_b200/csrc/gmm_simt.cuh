// Plain-FMA tile product shared by the grouped products' fp32, odd-size and 8-bit fallback kernels:
// C[TM, 64] += A[TM, K] B[64, K]^T with fp32 accumulation, operands read through small loader types that
// hide storage type, major order and block scales.  256 threads, each a TM/16 x 4 micro-tile.  fp32 operands are
// fetched element by element with cp.async into a ring of four k-steps (rows need no alignment, and the copies
// transpose on the way); other types go through registers, one k-step ahead.
// The fp32 layers this serves have a few hundred tiles at most, one or two per SM, so latency, not FMA rate, is what
// these kernels fight: deep prefetch, and TM = 32 where 64-row tiles would leave SMs without one.
#pragma once
#include "gmm.cuh"

namespace capmoe {
namespace {

constexpr int ST = 64;        // tile columns (and rows, or half of them)
constexpr int SK = 16;        // k-step
constexpr int SN = 256;       // threads
constexpr int SROW = ST + 4;  // row of a staged operand: 16-byte aligned, shifted by four banks
constexpr int SDEPTH = 4;     // k-steps in the ring

// element (i, k) of an operand stored with k contiguous (KMAJ) or i contiguous
template <typename T, bool KMAJ>
struct Dense {
  static constexpr bool k_fast = KMAJ, direct = sizeof(T) == 4;
  const T* p;
  int64_t ld;
  __device__ __forceinline__ const T* ptr(int i, int k) const { return KMAJ ? p + (int64_t)i * ld + k : p + (int64_t)k * ld + i; }
  __device__ __forceinline__ float at(int i, int k) const { return to_float(*ptr(i, k)); }
};
// e4m3 with one scale per TALL rows x 128 columns
template <int TALL>
struct Coded {
  static constexpr bool k_fast = true, direct = false;
  const uint8_t* q;
  const uint8_t* s;
  int64_t ld, sld;
  __device__ __forceinline__ float at(int i, int k) const {
    uint32_t h2;
    const uint16_t c = q[(int64_t)i * ld + k];
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(c));
    float v;
    asm("cvt.f32.f16 %0, %1;" : "=f"(v) : "h"((uint16_t)(h2 & 0xffffu)));
    return v * scale_value(s[(int64_t)(i / TALL) * sld + k / QBLOCK]);
  }
};

template <int TM> struct alignas(16) SimtTile { float a[SDEPTH][SK][TM + 4], b[SDEPTH][SK][SROW]; };

__device__ __forceinline__ void copy4(float* dst, const float* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
               "r"(there ? 4 : 0)
               : "memory");
}

template <int TM, class LA, class LB>
__device__ __forceinline__ void tile_product(const LA& la, const LB& lb, int rows, int cols, int K, SimtTile<TM>& sm,
                                             float (&acc)[TM / 16][4]) {
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  constexpr int NA = TM * SK / SN, NB = ST * SK / SN;
  constexpr bool ring = LA::direct && LB::direct;
  if (K <= 0) return;
  const int steps = (K + SK - 1) / SK;
  auto a_k = [&](int x) { return LA::k_fast ? x % SK : x / TM; };
  auto a_i = [&](int x) { return LA::k_fast ? x / SK : x % TM; };
  auto b_k = [&](int x) { return LB::k_fast ? x % SK : x / ST; };
  auto b_i = [&](int x) { return LB::k_fast ? x / SK : x % ST; };
  auto multiply = [&](int buf) {
#pragma unroll
    for (int kk = 0; kk < SK; ++kk) {
      float av[TM / 16];
      if constexpr (TM == 64) {
        const float4 a = *reinterpret_cast<const float4*>(&sm.a[buf][kk][ty * 4]);
        av[0] = a.x; av[1] = a.y; av[2] = a.z; av[3] = a.w;
      } else {
        const float2 a = *reinterpret_cast<const float2*>(&sm.a[buf][kk][ty * 2]);
        av[0] = a.x; av[1] = a.y;
      }
      const float4 b = *reinterpret_cast<const float4*>(&sm.b[buf][kk][tx * 4]);
      const float bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < TM / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
    }
  };
  __syncthreads();                                  // an earlier product may still read the buffers
  if constexpr (ring) {
    auto issue = [&](int step) {
      if (step < steps) {
        const int k0 = step * SK, buf = step % SDEPTH;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
          const int x = tid + i * SN, k = a_k(x), r = a_i(x);
          const bool there = r < rows && k0 + k < K;
          copy4(&sm.a[buf][k][r], there ? la.ptr(r, k0 + k) : la.p, there);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int x = tid + i * SN, k = b_k(x), c = b_i(x);
          const bool there = c < cols && k0 + k < K;
          copy4(&sm.b[buf][k][c], there ? lb.ptr(c, k0 + k) : lb.p, there);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < SDEPTH - 1; ++s) issue(s);
    for (int step = 0; step < steps; ++step) {
      asm volatile("cp.async.wait_group %0;" ::"n"(SDEPTH - 2) : "memory");
      __syncthreads();                              // this step is in; the buffer of the step before it has been read
      issue(step + SDEPTH - 1);
      multiply(step % SDEPTH);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  } else {
    float ra[NA], rb[NB];
    auto fetch = [&](int k0) {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int x = tid + i * SN;
        ra[i] = (a_i(x) < rows && k0 + a_k(x) < K) ? la.at(a_i(x), k0 + a_k(x)) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int x = tid + i * SN;
        rb[i] = (b_i(x) < cols && k0 + b_k(x) < K) ? lb.at(b_i(x), k0 + b_k(x)) : 0.f;
      }
    };
    auto put = [&](int buf) {
#pragma unroll
      for (int i = 0; i < NA; ++i) sm.a[buf][a_k(tid + i * SN)][a_i(tid + i * SN)] = ra[i];
#pragma unroll
      for (int i = 0; i < NB; ++i) sm.b[buf][b_k(tid + i * SN)][b_i(tid + i * SN)] = rb[i];
    };
    fetch(0);
    put(0);
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
      if (step + 1 < steps) fetch((step + 1) * SK);
      multiply(step & 1);
      if (step + 1 < steps) put((step + 1) & 1);    // last read two steps ago, before the previous barrier
      __syncthreads();
    }
  }
}

template <int R>
__device__ __forceinline__ void clear_acc(float (&acc)[R][4]) {
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
}

// The row tile that block `slot` of a launch works on: segments in order, ceil(rows / TM) tiles each.
// Returns false when the slot lies behind the last tile.  All threads call it.
struct RowTile { int e, row0, rows; };
template <int TM>
__device__ __forceinline__ bool find_row_tile(const Segments& sg, int slot, RowTile& t) {
  __shared__ int warp_sum[SN / 32], found[3];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int begin = 0, n = 0;
  if (tid < sg.E) { begin = seg_at(sg, tid); n = max(0, seg_at(sg, tid + 1) - begin); }
  const int mine = (n + TM - 1) / TM;
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
  if (tid == 0) found[0] = -1;
  if (lane == 31) warp_sum[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; ++w) upto += warp_sum[w];
  if (slot < upto && slot >= upto - mine) {
    const int b = (slot - (upto - mine)) * TM;
    found[0] = tid; found[1] = begin + b; found[2] = min(TM, n - b);
  }
  __syncthreads();
  t.e = found[0]; t.row0 = found[1]; t.rows = found[2];
  return t.e >= 0;
}

}  // namespace
}  // namespace capmoe
