// Root-mean-square norm of the rows in front of an expert layer, with the residual's addition and the 8-bit codes that the
// expert products read, and its gradients.
//   h = x + residual (rounded to the storage type: what the residual stream keeps)
//   rstd = (sum_c h_c^2 / d + eps)^(-1/2),  y = h rstd w,  codes of the rounded y as capmoe_quantize_rows makes them
//   dx = rstd (g - n (sum_c g_c n_c) / d) + dh with g = dy w and n = h rstd,  dw = sum over the rows of dy n
// All of it in fp32; what is stored has one rounding (h, y, dx) or none before the last (rstd, dw).
#include "gmm.cuh"
#include "rowvec.cuh"

namespace capmoe {
namespace {

constexpr int NW = 8;                        // warps of a block, `wpr` of them to a row (a row of 16 warps is a block of its own)
constexpr int NT_MAX = 512;
constexpr int NORM_MAX_D = 16384;

// A thread's NV columns of a vector's place u are NV / W accesses of W neighbouring columns: with W = NV (rows that start on 16 bytes)
// one; else four bytes (or, bf16 rows that do not start on four, one column) at a time, and the lanes of a warp take turns, so that
// their accesses lie side by side.  Either way a warp has the same 32 NV columns, whole blocks of 128 of them.  (16,384 bf16 rows with
// residual: 2048 columns 41 us, 2046 46, 2047 62, and 76 for both of the latter with accesses of one column converted on the way; the
// gradient with dh 46, 52, 94, and 91.)
template <int W, int NV>
__device__ __forceinline__ int column(int u, int tpr, int t) {           // the first
  return W == NV ? (u * tpr + t) * NV : (u * tpr + (t & ~31)) * NV + (t & 31) * W;
}
template <int W, int NV>
__device__ __forceinline__ constexpr int other(int i) {                  // from there to the i-th
  return W == NV ? i : i / W * 32 * W + i % W;
}
template <int BYTES> struct Access;
template <> struct Access<4> { using type = uint32_t; };
template <> struct Access<2> { using type = uint16_t; };
// The columns from p on, as they are stored; `left`: columns from there to the end of the row.
template <typename T, int W>
__device__ __forceinline__ uint4 get_cells(const T* p, int left) {
  constexpr int NV = Vec16<T>::n;
  if constexpr (W == NV) {
    return __ldcs(reinterpret_cast<const uint4*>(p));
  } else {
    using A = typename Access<W * (int)sizeof(T)>::type;
    union { uint4 v; A a[NV / W]; } x;
#pragma unroll
    for (int i = 0; i < NV / W; ++i) x.a[i] = i * 32 * W < left ? *reinterpret_cast<const A*>(p + i * 32 * W) : A(0);
    return x.v;
  }
}
template <typename T, int W>
__device__ __forceinline__ void put_cells(T* p, int left, const uint4& v) {
  constexpr int NV = Vec16<T>::n;
  if constexpr (W == NV) {
    *reinterpret_cast<uint4*>(p) = v;
  } else {
    using A = typename Access<W * (int)sizeof(T)>::type;
    union { uint4 v; A a[NV / W]; } x;
    x.v = v;
#pragma unroll
    for (int i = 0; i < NV / W; ++i)
      if (i * 32 * W < left) *reinterpret_cast<A*>(p + i * 32 * W) = x.a[i];
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Sum over the wpr warps of a row (a power of two), the same bits in all of them.  `red`: a word per warp of the block.
__device__ __forceinline__ float row_sum(float v, int wpr, float* red) {
  v = warp_sum(v);
  if (wpr > 1) {
    const int warp = threadIdx.x >> 5, first = warp & ~(wpr - 1);
    if ((threadIdx.x & 31) == 0) red[warp] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < wpr; ++i) v += red[first + i];
  }
  return v;
}

__device__ __forceinline__ uint32_t two_codes(float a, float b, uint32_t code) {
  const float inv = inv_scale(code);
  return code == (uint32_t)Q_NAN_SCALE ? 0x7f7fu : to_e4m3x2(a * inv, b * inv);
}
// Codes of a thread's columns under the scales of their blocks of 128, which are made here.
template <typename T, int W>
__device__ __forceinline__ void put_codes(const uint4& v, int c, int d, uint8_t* q, uint8_t* scale) {
  // a block: all NV columns of LANES lanes, or, lanes taking turns, PER columns of all lanes
  constexpr int NV = Vec16<T>::n, LANES = W == NV ? QBLOCK / NV : 32, PER = W == NV ? NV : QBLOCK / 32;
  float f[NV];
  Vec16<T>::load(v, f);
#pragma unroll
  for (int b = 0; b < NV; b += PER) {
    uint32_t m = 0;                          // of non-negative floats the larger has the larger pattern; NaN is above all
#pragma unroll
    for (int i = 0; i < PER; ++i) m = max(m, __float_as_uint(f[b + i]) & 0x7fffffffu);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const uint32_t code = scale_code(m);
    const int at = c + other<W, NV>(b);      // first of the thread's columns in the block
    if (at >= d) continue;
#pragma unroll
    for (int i = 0; i < PER; i += 4) {
      const uint32_t w = two_codes(f[b + i], f[b + i + 1], code) | two_codes(f[b + i + 2], f[b + i + 3], code) << 16;
      if constexpr (W == NV) {
        *reinterpret_cast<uint32_t*>(q + at + i) = w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + other<W, NV>(i + j) < d) q[at + other<W, NV>(i + j)] = (uint8_t)(w >> (8 * j));
      }
    }
    if ((threadIdx.x & (LANES - 1)) == 0) scale[at / QBLOCK] = (uint8_t)code;
  }
}

template <typename T>
struct NormArgs {
  const T *x, *res, *w;
  int64_t N;
  int d, wpr;
  float eps;
  T *h, *y;
  float* rstd;
  uint8_t *q, *scale;
};

// A row stays in the registers of its warps between the two uses, VPT vectors a thread: one pass over HBM, which bounds it
// (16,384 rows of 2048 bf16 columns with residual and codes: 47.8 us, 0.97 of the copy bandwidth).  Few vectors a thread and many
// warps mix reads and writes: with eight vectors a thread, a warp to a row, the same took 59.9 us, with one 51.2.
template <typename T, int W, int VPT>
__global__ void __launch_bounds__(NT_MAX) k_rms_norm(const NormArgs<T> a) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int NV = Vec16<T>::n;
  __shared__ float red[NT_MAX / 32];
  const int tpr = a.wpr * 32, t = threadIdx.x & (tpr - 1), d = a.d;
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / tpr) + threadIdx.x / tpr;
  const bool live = row < a.N;
  const int64_t at = row * d;
  uint4 v[VPT];
#pragma unroll
  for (int u = 0; u < VPT; ++u) {
    const int c = column<W, NV>(u, tpr, t);
    v[u] = live && c < d ? get_cells<T, W>(a.x + at + c, d - c) : make_uint4(0u, 0u, 0u, 0u);
  }
  if (a.res) {
    uint4 r[VPT];
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const int c = column<W, NV>(u, tpr, t);
      r[u] = live && c < d ? get_cells<T, W>(a.res + at + c, d - c) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const int c = column<W, NV>(u, tpr, t);
      float f[NV], g[NV];
      Vec16<T>::load(v[u], f);
      Vec16<T>::load(r[u], g);
#pragma unroll
      for (int i = 0; i < NV; ++i) f[i] += g[i];
      v[u] = Vec16<T>::store(f);
      if (live && c < d) put_cells<T, W>(a.h + at + c, d - c, v[u]);
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < VPT; ++u) {
    float f[NV];
    Vec16<T>::load(v[u], f);
#pragma unroll
    for (int i = 0; i < NV; ++i) sum = fmaf(f[i], f[i], sum);
  }
  const float ms = row_sum(sum, a.wpr, red) / (float)d + a.eps;
  float rstd = rsqrtf(ms);
  const float left = fmaf(-ms * rstd, rstd, 1.f);            // one Newton step: what rsqrtf leaves would be the largest error of an fp32 y
  if (fabsf(left) < 0.5f) rstd = fmaf(0.5f * rstd, left, rstd);   // (not from an infinity or a zero)
  if (!live) return;                         // whole warps; nothing below crosses a warp
  if (a.rstd && t == 0) a.rstd[row] = rstd;
  const int nb = (d + QBLOCK - 1) / QBLOCK;
#pragma unroll
  for (int u = 0; u < VPT; ++u) {
    const int c = column<W, NV>(u, tpr, t);
    float f[NV], g[NV];
    Vec16<T>::load(v[u], f);
    Vec16<T>::load(c < d ? (W == NV ? __ldg(reinterpret_cast<const uint4*>(a.w + c)) : get_cells<T, W>(a.w + c, d - c)) : make_uint4(0u, 0u, 0u, 0u), g);
#pragma unroll
    for (int i = 0; i < NV; ++i) f[i] = f[i] * rstd * g[i];
    const uint4 y = Vec16<T>::store(f);
    if (c < d) put_cells<T, W>(a.y + at + c, d - c, y);
    if (a.q) put_codes<T, W>(y, c, d, a.q + at, a.scale + row * nb);
  }
}

template <typename T>
struct GradArgs {
  const T *dy, *h, *w;
  const float* rstd;
  const T* dh;
  int64_t N;
  int d, wpr;
  T* dx;
  float* part;                               // [blocks][d]
  __nv_bfloat16* dw16;                       // one block: dw itself, as bf16; else NULL
};

__device__ __forceinline__ uint4 together(const uint32_t* a) { return make_uint4(a[0], a[1], a[2], a[3]); }
__device__ __forceinline__ uint4 together(const uint16_t* a) {
  return make_uint4(a[0] | (uint32_t)a[1] << 16, a[2] | (uint32_t)a[3] << 16, a[4] | (uint32_t)a[5] << 16, a[6] | (uint32_t)a[7] << 16);
}

// Per-thread ring of the rows to come: every thread copies the 16-byte vectors that it will use itself into its own places of
// shared memory, so nothing but its own copies has to be waited for.
__device__ __forceinline__ uint4 get_shared(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// A group of wpr warps walks its rows, DEPTH - 1 of them in flight ahead of the one it works on; a thread's columns are the same
// in all of them: dw is summed in registers, over a block's groups in shared memory, and written once per block for k_sum_parts to
// join, all in a fixed order.  (A part per group: 12,247 rows of 192 bf16 columns 14.2 us,
// like this 11.9.)  So few rows that a block walks four at most have the block to themselves, and no parts.  Bound by HBM
// (16,384 rows of 4096 bf16 columns with dh: 83.6 us with the sum of the parts, 0.98 of the copy bandwidth; 108 with each row's loads
// waited for, 88 with the next row's in registers); narrower rows also by the row's sum, a barrier a row (16,384 of 2048 without
// dh: 40 us, 0.76).
template <typename T, int W, int VPT, int DEPTH>
__global__ void __launch_bounds__(NT_MAX) k_rms_norm_grad(const GradArgs<T> a) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int NV = Vec16<T>::n;
  constexpr bool ASYNC = W == NV;
  __shared__ float red[2][NT_MAX / 32];
  extern __shared__ uint4 ring[];            // [PLACES][dy, h, dh][VPT][threads]
  const int tpr = a.wpr * 32, t = threadIdx.x & (tpr - 1), d = a.d;
  const int64_t group = (int64_t)blockIdx.x * (blockDim.x / tpr) + threadIdx.x / tpr, groups = (int64_t)gridDim.x * (blockDim.x / tpr);
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring + threadIdx.x), step = blockDim.x * 16u;
  uint4 w[VPT];
  float dw[VPT][NV];
#pragma unroll
  for (int u = 0; u < VPT; ++u) {
    const int c = column<W, NV>(u, tpr, t);
    w[u] = c < d ? get_cells<T, W>(a.w + c, d - c) : zero;
#pragma unroll
    for (int i = 0; i < NV; ++i) dw[u][i] = 0.f;
  }
  // Rows of whole vectors: asynchronous copies, DEPTH - 1 rows ahead.  Others: the next row's columns wait in registers while this
  // row is worked on, and take its place afterwards (asynchronous copies of four bytes: 8192 rows of 2049 fp32 columns 79 -> 152 us).
  constexpr int PLACES = ASYNC ? DEPTH : 1;
  using A = typename Access<ASYNC ? 4 : W * (int)sizeof(T)>::type;
  A raw[ASYNC ? 1 : 3][ASYNC ? 1 : VPT][ASYNC ? 1 : NV / W];
  const T* const from3[3] = {a.dy, a.h, a.dh};
  auto fetch = [&](int64_t row, int slot) {
#pragma unroll
    for (int m = 0; m < 3; ++m)
#pragma unroll
      for (int u = 0; u < VPT; ++u) {
        const int c = column<W, NV>(u, tpr, t);
        const bool in = row < a.N && from3[m];
        const T* p = in ? from3[m] + row * d : a.w;
        const uint32_t to = mine + (uint32_t)((slot * 3 + m) * VPT + u) * step;
        if constexpr (W == NV) {
          copy16(to, p + (c < d ? c : 0), in && c < d);
        } else {
#pragma unroll
          for (int i = 0; i < NV / W; ++i) raw[m][u][i] = *reinterpret_cast<const A*>(p + (c + i * 32 * W < d ? c + i * 32 * W : 0));
        }
      }
    if constexpr (ASYNC) copies_commit();
  };
  auto place = [&](int64_t row, int slot) {  // what fetch left in registers, zeros where there is nothing
    if constexpr (!ASYNC) {
#pragma unroll
      for (int m = 0; m < 3; ++m)
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
          const int c = column<W, NV>(u, tpr, t);
          A cells[NV / W];
#pragma unroll
          for (int i = 0; i < NV / W; ++i) cells[i] = row < a.N && from3[m] && c + i * 32 * W < d ? raw[m][u][i] : A(0);
          ring[(size_t)((slot * 3 + m) * VPT + u) * blockDim.x + threadIdx.x] = together(cells);
        }
    }
  };
  constexpr int AHEAD = ASYNC ? DEPTH - 1 : 1;
#pragma unroll
  for (int s = 0; s < AHEAD; ++s) fetch(group + s * groups, s);
  place(group, 0);
  float rstd = group < a.N ? a.rstd[group] : 0.f;
  int it = 0, slot = 0;
  for (int64_t row0 = 0; row0 < a.N; row0 += groups, it ^= 1) {      // the same count in all warps of the block
    const int64_t row = row0 + group;
    const bool live = row < a.N;
    fetch(row + AHEAD * groups, slot == 0 ? PLACES - 1 : slot - 1);
    const float rstd1 = row + groups < a.N ? a.rstd[row + groups] : 0.f;
    if constexpr (ASYNC) copies_wait<AHEAD>();
    const uint32_t from = mine + (uint32_t)(slot * 3 * VPT) * step;
    uint4 dy[VPT], h[VPT];
    float dot = 0.f;
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      dy[u] = get_shared(from + (uint32_t)u * step);
      h[u] = get_shared(from + (uint32_t)(VPT + u) * step);
      float p[NV], q[NV], g[NV];
      Vec16<T>::load(dy[u], p);
      Vec16<T>::load(h[u], q);
      Vec16<T>::load(w[u], g);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float n = q[i] * rstd;
        dot = fmaf(p[i] * g[i], n, dot);
        dw[u][i] = fmaf(p[i], n, dw[u][i]);
      }
    }
    const float mean = row_sum(dot, a.wpr, red[it]) / (float)d;
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const int c = column<W, NV>(u, tpr, t);
      float p[NV], q[NV], g[NV], e[NV];
      Vec16<T>::load(dy[u], p);
      Vec16<T>::load(h[u], q);
      Vec16<T>::load(w[u], g);
      Vec16<T>::load(get_shared(from + (uint32_t)(2 * VPT + u) * step), e);
#pragma unroll
      for (int i = 0; i < NV; ++i) p[i] = fmaf(rstd, fmaf(-q[i] * rstd, mean, p[i] * g[i]), e[i]);      // (rstd^2 alone may pass fp32)
      if (live && c < d) put_cells<T, W>(a.dx + row * d + c, d - c, Vec16<T>::store(p));
    }
    rstd = rstd1;
    if (++slot == PLACES) slot = 0;
    place(row + groups, slot);
  }
  float* to = a.part + (int64_t)blockIdx.x * d;                // the block's part, of its groups' sums in their order
  const bool staged = tpr < (int)blockDim.x || a.dw16 || (reinterpret_cast<uintptr_t>(a.part) & 15);
  if (staged) {
    if constexpr (ASYNC) copies_wait<0>();
    __syncthreads();                         // the ring is free
    to = reinterpret_cast<float*>(ring) + (threadIdx.x / tpr) * d;
  }
#pragma unroll
  for (int u = 0; u < VPT; ++u) {
    const int c = column<W, NV>(u, tpr, t);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (W == NV && i % 4 == 0 && c < d) *reinterpret_cast<float4*>(to + c + i) = make_float4(dw[u][i], dw[u][i + 1], dw[u][i + 2], dw[u][i + 3]);
      if (W < NV && c + other<W, NV>(i) < d) to[c + other<W, NV>(i)] = dw[u][i];
    }
  }
  if (staged) {
    __syncthreads();
    const float* sums = reinterpret_cast<const float*>(ring);
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
      float v = sums[c];
      for (int g = 1; g < (int)blockDim.x / tpr; ++g) v += sums[g * d + c];
      if (a.dw16) a.dw16[c] = __float2bfloat16_rn(v);
      else a.part[(int64_t)blockIdx.x * d + c] = v;
    }
  }
}

// out[c] = sum over g of part[g][c]: a block per SUM_COLS columns (a half line), SUM_ROWS threads to a column, then their
// sums in order.  (A block per 32 columns leaves most SMs without one.)
constexpr int SUM_COLS = 16, SUM_ROWS = 32;
template <typename TO>
__global__ void __launch_bounds__(SUM_COLS * SUM_ROWS) k_sum_parts(const float* __restrict__ part, int64_t parts, int d, TO* __restrict__ out) {
  allow_next_kernel();
  wait_for_previous_kernel();
  __shared__ float sum[SUM_ROWS][SUM_COLS];
  const int i = threadIdx.x & (SUM_COLS - 1), c = blockIdx.x * SUM_COLS + i, r = threadIdx.x / SUM_COLS;
  float s = 0.f;
  if (c < d)
#pragma unroll 8
    for (int64_t g = r; g < parts; g += SUM_ROWS) s += part[g * d + c];
  sum[r][i] = s;
  __syncthreads();
  if (r == 0 && c < d) {
#pragma unroll 8
    for (int j = 1; j < SUM_ROWS; ++j) s += sum[j][i];
    out[c] = from_float<TO>(s);
  }
}

constexpr int NORM_VPT = 2;                  // vectors a thread that a row's warps are chosen for, with many rows
constexpr int GRAD_VPT = 2;                  // the same of the gradient, whose threads also hold dw and w
constexpr int GRAD_BLOCKS = 2;               // blocks per SM at most
constexpr int GRAD_DEPTH1 = 3, GRAD_DEPTH2 = 4;   // rows in the ring with one and two vectors a thread
// Warps to a row: as few as hold it in `vpt` vectors a thread, more while the rows leave warps of the device without one; 16
// where eight would have to hold more than `most` vectors a thread.
int warps_per_row(int64_t N, int vecs, int vpt, int most) {
  int wpr = 1;
  while (wpr < NW && vecs > 32 * wpr && (vecs > 32 * wpr * vpt || N * wpr < (int64_t)sm_count() * NW)) wpr *= 2;
  return vecs > 32 * NW * most ? 2 * NW : wpr;
}
int norm_warps(int64_t N, int vecs) { return warps_per_row(N, vecs, NORM_VPT, 8); }
int rows_per_block(int wpr) { return wpr < NW ? NW / wpr : 1; }
constexpr int ALONE = 4;                     // rows that a group of the gradient's only block walks at most (of rows that eight warps hold)
int grad_warps(int64_t N, int vecs) {
  const int few = warps_per_row((int64_t)1 << 40, vecs, GRAD_VPT, 2);
  return few <= NW && N <= ALONE * rows_per_block(few) ? few : warps_per_row(N, vecs, GRAD_VPT, 2);
}
unsigned threads_of(int wpr) { return 32u * (unsigned)(wpr < NW ? NW : wpr); }
int vecs_of(int d, int dtype) { return (int)ceil_div((int64_t)d * (int64_t)elt_size(dtype), 16); }
int grad_blocks(int64_t N, int wpr) {
  const int64_t want = ceil_div(N, rows_per_block(wpr)), most = (int64_t)sm_count() * GRAD_BLOCKS;
  return wpr <= NW && want <= ALONE ? 1 : (int)(want < most ? want : most);
}

template <typename T, int W>
int norm_run(const NormArgs<T>& a, cudaStream_t st) {
  const int vpt = (int)ceil_div(ceil_div(a.d, Vec16<T>::n), 32 * a.wpr);
  const int64_t blocks = ceil_div(a.N, rows_per_block(a.wpr));
  if (blocks > 0x7fffffff) return CAPMOE_EUNSUPPORTED;
  auto k = vpt <= 1 ? k_rms_norm<T, W, 1> : vpt <= 2 ? k_rms_norm<T, W, 2> : vpt <= 4 ? k_rms_norm<T, W, 4> : k_rms_norm<T, W, 8>;
  const int rc = note_cuda(launch_chained(k, (unsigned)blocks, threads_of(a.wpr), 0, st, a));
  count_launch(1);
  return rc;
}
template <typename T>
int norm(const void* x, const void* res, const void* w, int64_t N, int d, float eps, void* h, void* y, float* rstd, void* q, void* scale,
         int dtype, cudaStream_t st) {
  const NormArgs<T> a{(const T*)x, (const T*)res, (const T*)w, N, d, norm_warps(N, vecs_of(d, dtype)), eps, (T*)h, (T*)y, rstd,
                      (uint8_t*)q, (uint8_t*)scale};
  constexpr int NV = Vec16<T>::n, W = 4 / sizeof(T);
  return d % NV == 0 ? norm_run<T, NV>(a, st) : d % W == 0 ? norm_run<T, W>(a, st) : norm_run<T, 1>(a, st);
}

template <typename T, int W>
int grad_run(const GradArgs<T>& a, cudaStream_t st) {
  const int vpt = (int)ceil_div(ceil_div(a.d, Vec16<T>::n), 32 * a.wpr);
  const int room = vpt <= 1 ? 1 : vpt <= 2 ? 2 : vpt <= 4 ? 4 : 8;
  const int depth = W < Vec16<T>::n ? 1 : room == 1 ? GRAD_DEPTH1 : room == 2 ? GRAD_DEPTH2 : 8 / room;
  auto k = room == 1 ? k_rms_norm_grad<T, W, 1, GRAD_DEPTH1> : room == 2 ? k_rms_norm_grad<T, W, 2, GRAD_DEPTH2>
           : room == 4 ? k_rms_norm_grad<T, W, 4, 2> : k_rms_norm_grad<T, W, 8, 1>;
  const size_t smem = (size_t)depth * 3 * (size_t)room * threads_of(a.wpr) * 16;
  const cudaError_t err = allow_smem(k, smem);
  if (err != cudaSuccess) return note_cuda(err);
  const int rc = note_cuda(launch_chained(k, (unsigned)grad_blocks(a.N, a.wpr), threads_of(a.wpr), smem, st, a));
  count_launch(1);
  return rc;
}
template <typename T>
int norm_grad(const void* dy, const void* h, const void* w, const float* rstd, const void* dh, int64_t N, int d, int dtype, int out_dtype,
              void* dx, void* dw, float* part, cudaStream_t st) {
  GradArgs<T> a{(const T*)dy, (const T*)h, (const T*)w, rstd, (const T*)dh, N, d, grad_warps(N, vecs_of(d, dtype)), (T*)dx, part, nullptr};
  const int blocks = grad_blocks(N, a.wpr);
  if (blocks == 1 && out_dtype == CAPMOE_F32) a.part = (float*)dw;
  if (blocks == 1 && out_dtype == CAPMOE_BF16) a.dw16 = (__nv_bfloat16*)dw;
  constexpr int NV = Vec16<T>::n, W = 4 / sizeof(T);
  const int rc = d % NV == 0 ? grad_run<T, NV>(a, st) : d % W == 0 ? grad_run<T, W>(a, st) : grad_run<T, 1>(a, st);
  if (rc != CAPMOE_OK || blocks == 1) return rc;
  return sum_parts(part, blocks, d, out_dtype, dw, st);
}

int check_norm(int64_t N, int d, int dtype) {
  if (N < 0 || d < 1) return CAPMOE_EINVAL;
  if ((dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) || d > NORM_MAX_D) return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}

}  // namespace

int sum_parts(const float* part, int64_t parts, int d, int out_dtype, void* out, cudaStream_t st) {
  const unsigned grid = (unsigned)ceil_div(d, SUM_COLS), block = SUM_COLS * SUM_ROWS;
  const int rc = note_cuda(out_dtype == CAPMOE_F32 ? launch_chained(k_sum_parts<float>, grid, block, 0, st, part, parts, d, (float*)out)
                                                   : launch_chained(k_sum_parts<__nv_bfloat16>, grid, block, 0, st, part, parts, d, (__nv_bfloat16*)out));
  count_launch(1);
  return rc;
}

}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_rms_norm(const void* x, const void* residual, const void* w, int64_t N, int d, int dtype, float eps, void* h, void* y,
                               float* rstd, void* q, void* scale, void* stream) {
  const int rc = check_norm(N, d, dtype);
  if (rc != CAPMOE_OK) return rc;
  if (!(eps >= 0.f)) return CAPMOE_EINVAL;
  if (N == 0) return CAPMOE_OK;
  if (!usable(x, w, y) || !aligned16(residual) || !aligned16(h) || !aligned16(q)) return CAPMOE_EINVAL;
  if (!residual != !h || !q != !scale) return CAPMOE_EINVAL;
  if (dtype == CAPMOE_F32) return norm<float>(x, residual, w, N, d, eps, h, y, rstd, q, scale, dtype, as_stream(stream));
  return norm<__nv_bfloat16>(x, residual, w, N, d, eps, h, y, rstd, q, scale, dtype, as_stream(stream));
}

extern "C" int capmoe_rms_norm_backward_workspace_bytes(int64_t N, int d, int dtype, size_t* bytes) {
  const int rc = check_norm(N, d, dtype);
  if (!bytes) return CAPMOE_EINVAL;
  if (rc != CAPMOE_OK) return rc;
  const int wpr = grad_warps(N, vecs_of(d, dtype));
  *bytes = N ? (size_t)grad_blocks(N, wpr) * (size_t)d * sizeof(float) : 0;
  return CAPMOE_OK;
}

extern "C" int capmoe_rms_norm_backward(const void* dy, const void* h, const void* w, const float* rstd, const void* dh, int64_t N, int d,
                                        int dtype, int out_dtype, void* dx, void* dw, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = capmoe_rms_norm_backward_workspace_bytes(N, d, dtype, &need);
  if (rc != CAPMOE_OK) return rc;
  if (out_dtype != CAPMOE_F32 && (out_dtype != CAPMOE_BF16 || dtype != CAPMOE_BF16)) return CAPMOE_EUNSUPPORTED;
  if (!dw) return CAPMOE_EINVAL;
  if (N == 0) return note_cuda(cudaMemsetAsync(dw, 0, (size_t)d * elt_size(out_dtype), as_stream(stream)));
  if (!usable(dy, h, w, dx, ws) || !rstd || !aligned16(dh)) return CAPMOE_EINVAL;
  if (ws_bytes < need) return CAPMOE_EWORKSPACE;
  if (dtype == CAPMOE_F32) return norm_grad<float>(dy, h, w, rstd, dh, N, d, dtype, out_dtype, dx, dw, (float*)ws, as_stream(stream));
  return norm_grad<__nv_bfloat16>(dy, h, w, rstd, dh, N, d, dtype, out_dtype, dx, dw, (float*)ws, as_stream(stream));
}
