// Plain-FMA tile product shared by the grouped products' fp32, odd-size and 8-bit fallback kernels:
// C[TM, TN] += A[TM, K] B[TN, K]^T with fp32 accumulation, operands read through small loader types that
// hide storage type, major order and block scales.
// 64-column tiles: a block is G groups of 64 threads; a k-step is KG G long and each group multiplies its KG of it over the
// whole tile, a thread with a TM/8 x 8 micro-tile (rows and columns 8 apart); the partial tiles are added in shared memory
// at the end, in a fixed order.  Many tiles: 128 x 128 by one group of 256 threads with 8 x 8 micro-tiles, four times the
// FMAs between two barriers (0.52 of the FMA rate at 16,305 rows, 1000 x 1024; 0.42 with 64 x 64).
// What bounds the small ones is latency: a k-step of two resident blocks takes about 2000 cycles, 1024 of them
// FMA issue, in a call that lasts 8 of those and 6000 cycles around them.  Micro-tiles of 8 x 8 for 32-row tiles too (a
// warp per group, a third fewer shared-memory reads) changed nothing or cost up to 8 %, packed pairs of FMAs 30 %.
// The fp32 layers this serves have a few hundred tiles at most.  G = 4, two blocks to an SM, hides one block's latency
// behind the other; when the tiles do not outnumber the SMs, G = 8 gives a tile a whole SM: of 124 blocks that could
// share an SM the hardware puts two on some and none on others.  (1034 rows, 7 experts, 250 x 515 weights: y 13.2 us
// with G = 4, 17 with 8; dx, 124 tiles, 28 and 16.7; with 64-row tiles 25 and 31.)
// An operand is staged as it lies in memory: [index][k] when k is contiguous, [k][index] otherwise.  fp32 operands come
// in by cp.async, two or three k-steps ahead, in 16-byte pieces when their rows start on 16 bytes, else in 4-byte ones;
// other types go through registers, one k-step ahead.  TM = 32 where 64-row tiles would leave SMs without one.
#pragma once
#include <cooperative_groups.h>
#include "gmm.cuh"

namespace capmoe {
namespace {

constexpr int ST = 64;        // columns of the smaller tiles
// Geometry of a block: TM tile rows, G thread groups
template <int TM_, int G_, int TN_ = ST>
struct Geo {
  static constexpr int TM = TM_, TN = TN_, G = G_;
  static constexpr int TG = TN == ST ? 64 : 256;    // threads of a group
  static constexpr int KG = G == 1 ? 16 : TM == 64 ? 4 : 8;   // a group's part of a k-step (eight spill the large micro-tile)
  static constexpr int SK = KG * G;                 // k-step
  static constexpr int SN = TG * G;                 // threads
  static constexpr int BLOCKS = 512 / SN;           // resident blocks that registers are kept for
  static constexpr int DEPTH = TM == 32 ? 3 : 4;    // k-steps in the ring
  // a thread's micro-tile: MR rows, RS apart, by 8 columns, CS apart
  static constexpr int RS = TN == ST ? 8 : 16, MR = TM / RS, CS = RS;
  // result elements of a thread: R x C; with one group its micro-tile, else its share of the joined tile
  static constexpr int C = G == 1 ? 8 : 4, R = TM * TN / SN / C;
  // floats of one k-step of an operand of W rows (columns): [W][SK + 4] or [SK][W + 4]; both row pitches are odd multiples
  // of 16 bytes
  static constexpr int staged(int W) { return W * (SK + 4) > SK * (W + 4) ? W * (SK + 4) : SK * (W + 4); }
};

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

template <class GE> struct alignas(16) SimtTile { float a[GE::DEPTH][GE::staged(GE::TM)], b[GE::DEPTH][GE::staged(GE::TN)]; };

__device__ __forceinline__ void copy16(uint32_t dst, const float* src, int valid) {    // valid: bytes that exist, the rest is zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const float* src, int valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
}

// A thread's share of staging an fp32 operand of W rows (columns), n of which exist: one address is worked out once and
// advances by a k-step, the other copies of a step lie at equal distances from it (worked out per copy, the addresses cost
// twice the FMAs' instructions; one held for each copy, the registers spill).
template <class GE, int W, class L>
struct Stager {
  static constexpr int SK = GE::SK, SN = GE::SN;
  static constexpr int N4 = W * SK / SN;           // 4-byte copies per thread and step
  static constexpr int N16 = (N4 + 3) / 4;         // 16-byte copies (of the first threads only if N4 < 4)
  static constexpr int V = SK / 4;                 // 16-byte pieces of a k-step of one row, k contiguous
  static constexpr int E16 = L::k_fast ? SN / V : SN / (W / 4), E4 = L::k_fast ? SN / SK : SN / W;   // rows (k) between two copies
  const float *src, *base;                         // this thread's first copy of the step in hand; some valid address
  int64_t between, step_len;
  uint32_t dst0, size;                             // size: per copy, 4-byte form a bit, 16-byte form the bytes inside (8 bits)
  int left;                                        // reduction steps from this thread's first k on
  bool vec, idle;
  __device__ __forceinline__ Stager(const L& l, int n, int K, const float* ring) : base(l.p) {
    const int tid = threadIdx.x;
    vec = l.ld % 4 == 0 && ((uintptr_t)l.p & 15u) == 0;
    step_len = L::k_fast ? SK : SK * l.ld;
    size = 0;
    idle = vec && tid >= W * SK / 4;
    const int i0 = vec ? (L::k_fast ? tid / V : tid % (W / 4) * 4) : (L::k_fast ? tid / SK : tid % W);
    const int k = vec ? (L::k_fast ? tid % V * 4 : tid / (W / 4)) : (L::k_fast ? tid % SK : tid / W);
    dst0 = (uint32_t)__cvta_generic_to_shared(ring) + 4u * (uint32_t)(L::k_fast ? i0 * (SK + 4) + k : k * (W + 4) + i0);
    src = l.ptr(i0, k);                            // (used only where the element exists)
    left = K - k;
    between = (vec ? E16 : E4) * l.ld;
    if (vec) {
#pragma unroll
      for (int e = 0; e < N16; ++e) {
        const int i = L::k_fast ? i0 + e * E16 : i0;
        const int in = idle ? 0 : L::k_fast ? (i < n ? 4 : 0) : n - i;
        size |= (in <= 0 ? 0u : in >= 4 ? 16u : 4u * (uint32_t)in) << (8 * e);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N4; ++e) size |= (uint32_t)((L::k_fast ? i0 + e * E4 : i0) < n) << e;
    }
  }
  // copies the step in hand into the ring's buffer at byte offset `off` and moves on
  __device__ __forceinline__ void step(uint32_t off) {
    const float* p = src;
    if (vec) {
      if (!idle) {
#pragma unroll
        for (int e = 0; e < N16; ++e) {
          const uint32_t bytes = (size >> (8 * e)) & 255u;
          const int l = left - (L::k_fast ? 0 : e * E16);
          const uint32_t valid = L::k_fast ? (l <= 0 ? 0u : min(bytes, 4u * (uint32_t)min(l, 4))) : l > 0 ? bytes : 0u;
          copy16(dst0 + off + 4u * (uint32_t)(L::k_fast ? e * E16 * (SK + 4) : e * E16 * (W + 4)), valid ? p : base, (int)valid);
          p += between;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < N4; ++e) {
        const bool in = ((size >> e) & 1u) && left > (L::k_fast ? 0 : e * E4);
        copy4(dst0 + off + 4u * (uint32_t)(L::k_fast ? e * E4 * (SK + 4) : e * E4 * (W + 4)), in ? p : base, in ? 4 : 0);
        p += between;
      }
    }
    left -= SK;
    src += step_len;
  }
};

// Result element (i, j) of a thread, i < R, j < 4: row and column in the tile (a store's lanes write runs of 64 bytes; four
// columns side by side in a thread, each stored by itself as rows of odd length want it, take four times the requests)
template <class GE> __device__ __forceinline__ int micro_row(int tid) {       // first row (column) of a thread's micro-tile
  return GE::TN == ST ? (tid >> 3) & 7 : (tid >> 6) * 4 + ((tid >> 3) & 3);
}
template <class GE> __device__ __forceinline__ int micro_col(int tid) { return GE::TN == ST ? tid & 7 : ((tid >> 5) & 1) * 8 + (tid & 7); }
template <class GE> __device__ __forceinline__ int out_row(int i) {
  return GE::G == 1 ? micro_row<GE>((int)threadIdx.x) + GE::RS * i : (int)(threadIdx.x >> 4) + (GE::SN / 16) * i;
}
template <class GE> __device__ __forceinline__ int out_col(int j) {
  return GE::G == 1 ? micro_col<GE>((int)threadIdx.x) + GE::CS * j : (int)(threadIdx.x & 15) + 16 * j;
}
constexpr int CROW = ST + 8;                        // row of a partial tile

// acc += A B^T over the tile; result elements at out_row / out_col
template <class GE, class LA, class LB>
__device__ __forceinline__ void tile_product(const LA& la, const LB& lb, int rows, int cols, int K, SimtTile<GE>& sm,
                                             float (&acc)[GE::R][GE::C]) {
  constexpr int TM = GE::TM, TN = GE::TN, SK = GE::SK, SN = GE::SN, SDEPTH = GE::DEPTH;
  const int tid = threadIdx.x, tx = micro_col<GE>(tid), ty = micro_row<GE>(tid), group = tid / GE::TG;
  constexpr int R = GE::MR, RS = GE::RS, CS = GE::CS;
  constexpr bool ring = LA::direct && LB::direct;
  static_assert(GE::G == 1 || sizeof(SimtTile<GE>) >= 2 * TM * CROW * sizeof(float), "two partial tiles fit the staging buffers");
  if (K <= 0) return;
  const int steps = (K + SK - 1) / SK;
  float part[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) part[i][j] = GE::G == 1 ? acc[i % GE::R][j % GE::C] : 0.f;
  auto multiply = [&](int buf) {
    const float *A = sm.a[buf], *B = sm.b[buf];
#pragma unroll
    for (int k0 = group * GE::KG; k0 < group * GE::KG + GE::KG; k0 += 4) {
      float a[R][4];
      if constexpr (LA::k_fast) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float4 f = *reinterpret_cast<const float4*>(A + (ty + RS * i) * (SK + 4) + k0);
          a[i][0] = f.x; a[i][1] = f.y; a[i][2] = f.z; a[i][3] = f.w;
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int i = 0; i < R; ++i) a[i][kk] = A[(k0 + kk) * (TM + 4) + ty + RS * i];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float b[4];
        if constexpr (LB::k_fast) {
          const float4 f = *reinterpret_cast<const float4*>(B + (tx + CS * j) * (SK + 4) + k0);
          b[0] = f.x; b[1] = f.y; b[2] = f.z; b[3] = f.w;
        } else {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) b[kk] = B[(k0 + kk) * (TN + 4) + tx + CS * j];
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int i = 0; i < R; ++i) part[i][j] = fmaf(a[i][kk], b[kk], part[i][j]);
      }
    }
  };
  __syncthreads();                                  // an earlier product may still read the buffers
  if constexpr (ring) {
    Stager<GE, TM, LA> sa(la, rows, K, sm.a[0]);
    Stager<GE, TN, LB> sb(lb, cols, K, sm.b[0]);
    uint32_t buf = 0;                               // ring buffer of the next step to copy
    int left = steps;                               // steps not yet copied
    auto issue = [&]() {
      if (left > 0) {
        sa.step(buf * (uint32_t)sizeof(sm.a[0]));
        sb.step(buf * (uint32_t)sizeof(sm.b[0]));
        --left;
        buf = buf + 1 == SDEPTH ? 0 : buf + 1;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < SDEPTH - 1; ++s) issue();
    for (int step = 0; step < steps; ++step) {
      asm volatile("cp.async.wait_group %0;" ::"n"(SDEPTH - 2) : "memory");
      __syncthreads();                              // this step is in; the buffer of the step before it has been read
      issue();
      multiply(step % SDEPTH);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  } else {
    constexpr int NA = TM * SK / SN, NB = TN * SK / SN;
    float ra[NA], rb[NB];
    auto a_k = [&](int x) { return LA::k_fast ? x % SK : x / TM; };
    auto a_i = [&](int x) { return LA::k_fast ? x / SK : x % TM; };
    auto b_k = [&](int x) { return LB::k_fast ? x % SK : x / TN; };
    auto b_i = [&](int x) { return LB::k_fast ? x / SK : x % TN; };
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
      for (int i = 0; i < NA; ++i) {
        const int x = tid + i * SN;
        sm.a[buf][LA::k_fast ? a_i(x) * (SK + 4) + a_k(x) : a_k(x) * (TM + 4) + a_i(x)] = ra[i];
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int x = tid + i * SN;
        sm.b[buf][LB::k_fast ? b_i(x) * (SK + 4) + b_k(x) : b_k(x) * (TN + 4) + b_i(x)] = rb[i];
      }
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
  if constexpr (GE::G == 1) {
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = part[i][j];
    return;
  }
  // the even and the odd groups, one after the other from the last to the first, in the staging buffers, then both sums
  __syncthreads();
  float* C = &sm.a[0][0] + (group & 1) * TM * CROW;
#pragma unroll
  for (int turn = SN / 128 - 1; turn >= 0; --turn) {
    if ((group >> 1) == turn) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float& c = C[(ty + 8 * i) * CROW + tx + 8 * j];
          c = turn == SN / 128 - 1 ? part[i][j] : c + part[i][j];
        }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < GE::R; ++i) {
    const float* c0 = &sm.a[0][0] + out_row<GE>(i) * CROW;
#pragma unroll
    for (int j = 0; j < GE::C; ++j) acc[i][j] += c0[out_col<GE>(j)] + c0[TM * CROW + out_col<GE>(j)];
  }
}

// A reduction split over the blocks of a cluster (gridDim.z of them): this block's share of K, in whole 16-byte pieces.  With
// 18 tiles and sums of 787 terms an FFN's gradients take 66 us, 102 unsplit; joining costs about 2 us of a launch.
struct Share { int k0, len; };
__device__ __forceinline__ Share share_of(int K) {
  const int each = ((K + (int)gridDim.z - 1) / (int)gridDim.z + 3) & ~3, k0 = (int)blockIdx.z * each;
  return {k0, min(each, K - k0)};                   // (may be negative: nothing)
}
// Joins the blocks' partial results through distributed shared memory, in the blocks' order: each block sums its part of the tile's rows from all of them.
// False for a thread whose rows another block stores.  All threads of the cluster call it.
template <class GE, int N>
__device__ __forceinline__ bool join_shares(SimtTile<GE>& sm, float (&acc)[N][GE::R][GE::C]) {
  const int S = (int)gridDim.z;
  if (GE::R > 1 || S == 1) return true;             // only the smallest geometry is split
  static_assert(GE::R > 1 || sizeof(SimtTile<GE>) >= N * GE::TM * ST * sizeof(float), "the partial results fit the staging buffers");
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const int row = out_row<GE>(0);
  float* C = &sm.a[0][0] + row * ST;
  __syncthreads();                                  // the last product's partial tiles have been read
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) C[n * GE::TM * ST + out_col<GE>(j)] = acc[n][0][j];
  cluster.sync();
  const bool mine = row * S / GE::TM == (int)blockIdx.z;
  if (mine) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      for (int z = 0; z < S; ++z) {
        const float* p = cluster.map_shared_rank(C + n * GE::TM * ST, z);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += p[out_col<GE>(j)];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[n][0][j] = s[j];
    }
  }
  cluster.sync();                                   // nobody reads this block's memory any more
  return mine;
}

template <int R, int C>
__device__ __forceinline__ void clear_acc(float (&acc)[R][C]) {
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < C; ++j) acc[i][j] = 0.f;
}

template <class GE>
__device__ __forceinline__ SimtTile<GE>& simt_tile() {
  extern __shared__ __align__(16) uint8_t simt_smem[];
  return *reinterpret_cast<SimtTile<GE>*>(simt_smem);
}

// The row tile that block `slot` of a launch works on: segments in order, ceil(rows / TM) tiles each.
// Returns false when the slot lies behind the last tile.  All threads call it.
struct RowTile { int e, row0, rows; };
template <class GE>
__device__ __forceinline__ bool find_row_tile(const Segments& sg, int slot, RowTile& t) {
  constexpr int TM = GE::TM;
  __shared__ int warp_sum[GE::SN / 32], found[3];
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
