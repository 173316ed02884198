// Plain-FMA tile product shared by the grouped products' fp32, odd-size and 8-bit fallback kernels:
// C[64, 64] += A[64, K] B[64, K]^T with fp32 accumulation, operands read through small loader types that
// hide storage type, major order and block scales.  256 threads, each a 4 x 4 micro-tile; the next
// k-step's elements are fetched into registers while the current one is multiplied.
#pragma once
#include "gmm.cuh"

namespace capmoe {
namespace {

constexpr int ST = 64;        // tile rows and columns
constexpr int SK = 16;        // k-step
constexpr int SN = 256;       // threads
constexpr int SROW = ST + 4;  // row of a staged operand: 16-byte aligned, shifted by four banks

// element (i, k) of an operand stored with k contiguous (KMAJ) or i contiguous
template <typename T, bool KMAJ>
struct Dense {
  static constexpr bool k_fast = KMAJ;
  const T* p;
  int64_t ld;
  __device__ __forceinline__ float at(int i, int k) const {
    return to_float(KMAJ ? p[(int64_t)i * ld + k] : p[(int64_t)k * ld + i]);
  }
};
// e4m3 with one scale per TALL rows x 128 columns
template <int TALL>
struct Coded {
  static constexpr bool k_fast = true;
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

struct alignas(16) SimtTile { float a[2][SK][SROW], b[2][SK][SROW]; };

template <class LA, class LB>
__device__ __forceinline__ void tile_product(const LA& la, const LB& lb, int rows, int cols, int K, SimtTile& sm,
                                             float (&acc)[4][4]) {
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  float ra[4], rb[4];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = tid + i * SN;
      const int ak = LA::k_fast ? x % SK : x / ST, ai = LA::k_fast ? x / SK : x % ST;
      const int bk = LB::k_fast ? x % SK : x / ST, bi = LB::k_fast ? x / SK : x % ST;
      ra[i] = (ai < rows && k0 + ak < K) ? la.at(ai, k0 + ak) : 0.f;
      rb[i] = (bi < cols && k0 + bk < K) ? lb.at(bi, k0 + bk) : 0.f;
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = tid + i * SN;
      sm.a[buf][LA::k_fast ? x % SK : x / ST][LA::k_fast ? x / SK : x % ST] = ra[i];
      sm.b[buf][LB::k_fast ? x % SK : x / ST][LB::k_fast ? x / SK : x % ST] = rb[i];
    }
  };
  if (K <= 0) return;
  __syncthreads();                                  // an earlier product may still read the buffers
  fetch(0);
  put(0);
  __syncthreads();
  int buf = 0;
  for (int k0 = 0; k0 < K; k0 += SK) {
    const bool more = k0 + SK < K;
    if (more) fetch(k0 + SK);
#pragma unroll
    for (int kk = 0; kk < SK; ++kk) {
      const float4 a = *reinterpret_cast<const float4*>(&sm.a[buf][kk][ty * 4]);
      const float4 b = *reinterpret_cast<const float4*>(&sm.b[buf][kk][tx * 4]);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
    }
    if (more) put(buf ^ 1);                         // last read two k-steps ago, before the previous barrier
    __syncthreads();
    buf ^= 1;
  }
}

__device__ __forceinline__ void clear_acc(float (&acc)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
}

// The row tile that block `slot` of a launch works on: segments in order, ceil(rows / 64) tiles each.
// Returns false when the slot lies behind the last tile.  All threads call it.
struct RowTile { int e, row0, rows; };
__device__ __forceinline__ bool find_row_tile(const Segments& sg, int slot, RowTile& t) {
  __shared__ int warp_sum[SN / 32], found[3];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int begin = 0, n = 0;
  if (tid < sg.E) { begin = seg_at(sg, tid); n = max(0, seg_at(sg, tid + 1) - begin); }
  const int mine = (n + ST - 1) / ST;
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
  if (tid == 0) found[0] = -1;
  if (lane == 31) warp_sum[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; ++w) upto += warp_sum[w];
  if (slot < upto && slot >= upto - mine) {
    const int b = (slot - (upto - mine)) * ST;
    found[0] = tid; found[1] = begin + b; found[2] = min(ST, n - b);
  }
  __syncthreads();
  t.e = found[0]; t.row0 = found[1]; t.rows = found[2];
  return t.e >= 0;
}

}  // namespace
}  // namespace capmoe
