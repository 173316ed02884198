// Rows sorted by expert in 8 bits, and the gradients of the permutation and of the gate-weighted sum:
//   permute8      x_q[r] = q[t], scales with it, for the rows r = slot_row[t, s]
//   combine_grad  dy_perm[r] = w[r] dy[t],  dw[r] = dy[t] . y_perm[r]
//   permute_grad  dx[t] = sum_s dx_perm[slot_row[t, s]] + add0[t] + add1[t]
// Pure data movement, bound by HBM.  A token's row is read once for all its slots; every sum has a fixed order and fp32 terms.
#include "gmm.cuh"
#include "mbarrier.cuh"
#include "rowvec.cuh"

namespace capmoe {
namespace {

// What a kernel like these needs is bytes in flight, and what it has is a chain of look-ups (slot list, row) per token: warps that
// wait for each in turn reached 0.75 to 0.8 of the copy bandwidth with four vectors a lane and less with fewer.  So every warp
// runs a pipeline of its own: it walks tokens, looks up the next token's slots while it works on this one, and copies the chunks
// of the rows that it will need asynchronously into a ring of stages in shared memory, DEPTH - 1 of them ahead of the one it uses.
// A lane copies the vectors that it will read itself; only a stage's few words of description cross lanes.
constexpr int PV = 2;                        // 16-byte vectors a lane holds of a row: chunks of 1 KB
constexpr int CHUNK = 32 * PV;               // vectors of a chunk
constexpr int MAX_SLOTS = 288;               // k + m <= 32 + 256
constexpr int ROWS = 4;                      // row chunks of a stage

// The row of a token's slot, or -1: also where there is no such token or slot, or the row lies outside the buffers.
__device__ __forceinline__ int32_t slot_at(const int32_t* slot_row, int64_t t, int64_t N, int s, int slots, int64_t rows) {
  const int32_t r = t < N && s < slots ? slot_row[t * slots + s] : -1;
  return r < rows ? r : -1;
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// What a stage holds: `n` row chunks (below zero: there are no further stages), vectors from `v0` on; `first` and `last` of the sums
// that they belong to; the rows, and their weights.
struct Stage {
  int n, v0, first, last;
  int32_t row[ROWS];
  float w[ROWS];
};
template <int CHUNKS, int DEPTH>             // chunks of a stage
struct alignas(16) Ring {
  uint4 data[DEPTH][CHUNKS][CHUNK];
  Stage stage[DEPTH];
};
template <class R>
__device__ __forceinline__ void fetch_chunk(R& ring, int s, int c, const uint4* row, int v0, int row_vecs) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int u = 0; u < PV; ++u)
    if (v0 + u * 32 + lane < row_vecs) copy16((uint32_t)__cvta_generic_to_shared(&ring.data[s][c][u * 32 + lane]), row + v0 + u * 32 + lane);
}

// n bytes, `width` (16, 8, 4 or 1) at a time, which divides n and both addresses
__device__ __forceinline__ void copy_bytes(uint8_t* to, const uint8_t* from, int n, int width) {
  if (width == 16) for (int j = 0; j < n; j += 16) *reinterpret_cast<uint4*>(to + j) = *reinterpret_cast<const uint4*>(from + j);
  else if (width == 8) for (int j = 0; j < n; j += 8) *reinterpret_cast<uint2*>(to + j) = *reinterpret_cast<const uint2*>(from + j);
  else if (width == 4) for (int j = 0; j < n; j += 4) *reinterpret_cast<uint32_t*>(to + j) = *reinterpret_cast<const uint32_t*>(from + j);
  else for (int j = 0; j < n; ++j) to[j] = from[j];
}

// The rows of codes never pass through registers: a warp is a block, a lane has a token, fetches its row (a piece of it, 16 KB at
// most) with one bulk copy into shared memory and sends it out with one bulk copy per kept row.  While the rows are on their way
// the lanes share the tokens' (token, slot) pairs: token, weight and scales of every kept row.
// Four tokens to a block (eight of short rows), as many as 18 KB hold: with larger blocks the warp that waits for its last row keeps
// the others' places (32,700 rows of 2048: 19.8 us, 22.7 with eight tokens, 29.5 with 18, 38.8 with 32, 22.6 with one).
constexpr int P8_PIECE = 16384, P8_BYTES = 18 * 1024;          // bytes of a piece, of a block's pieces
__global__ void __launch_bounds__(32)
k_permute8(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale, int64_t N, int d, int piece, int per, int nb, int width, int E, int k,
           int slots, int D, int64_t rows, const float* __restrict__ scores, const int32_t* __restrict__ topk_idx,
           const int32_t* __restrict__ token_group, const int32_t* __restrict__ slot_row, uint8_t* __restrict__ q_perm,
           uint8_t* __restrict__ scale_perm, int32_t* __restrict__ perm_token, float* __restrict__ perm_weight, int32_t* __restrict__ dev_status) {
  allow_next_kernel();
  extern __shared__ __align__(128) uint8_t buf[];              // [per][piece]
  __shared__ uint64_t bars[32];
  __shared__ int abort_flag;
  const int lane = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int n = (int)min((int64_t)per, N - t0);
  const int c0 = (int)blockIdx.y * piece, bytes = min(piece, d - c0);
  const uint32_t bar = smem_u32(&bars[lane]), mine = smem_u32(buf) + (uint32_t)(lane * piece);
  mbar_init(bar, 1);
  if (lane == 0) abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  wait_for_previous_kernel();
  const int32_t* sr = slot_row + (t0 + lane) * slots;
  bool any = false;
  if (lane < n) {
#pragma unroll 8
    for (int s = 0; s < slots; ++s) {        // (all look-ups at once: no early end)
      const int32_t r = sr[s];
      any |= (r >= 0) & (r < rows);
    }
  }
  if (any) {                                 // a token nobody keeps is never read
    mbar_expect_tx(bar, (uint32_t)bytes);
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(mine), "l"(q + (t0 + lane) * d + c0), "r"((uint32_t)bytes), "r"(bar) : "memory");
  }
  if (c0 == 0) {
    const int m = D > 0 ? E / D : 0;
    for (int i = lane; i < n * slots; i += 32) {
      const int32_t r = slot_row[t0 * slots + i];
      if (r < 0 || r >= rows) continue;
      const int tok = i / slots, s = i - tok * slots;
      const int64_t t = t0 + tok;
      const int e = s < k ? topk_idx[t * k + s] : home_group(t, N, D, token_group) * m + (s - k);
      perm_token[r] = (int32_t)t;
      perm_weight[r] = (unsigned)e < (unsigned)E ? scores[t * E + e] : 0.f;
      copy_bytes(scale_perm + (int64_t)r * nb, scale + t * nb, nb, width);
    }
  }
  if (any) {
    if (mbar_wait(bar, 0u, &abort_flag)) {
      for (int s = 0; s < slots; ++s) {
        const int32_t r = sr[s];
        if (r >= 0 && r < rows)
          asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                       ::"l"(q_perm + (int64_t)r * d + c0), "r"(mine), "r"((uint32_t)bytes) : "memory");
      }
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");          // they have landed before the block ends
    } else if (dev_status) {
      atomicExch(dev_status, (int)CAPMOE_ETIMEOUT);
    }
  }
  __syncwarp();
  if (abort_flag) {                          // a wait ran out: copies may still be on their way to this shared memory (10 ms)
    const long long t1 = clock64();
    while (clock64() - t1 < 20000000LL) {}
  }
}

// A stage: a chunk of dy and the same chunk of up to ROWS kept rows.  A lane's share of their dot products stays in its registers
// over all chunks of the row, so the lanes meet once a row.
// Blocks are as short as they can be, a token to a warp: kept rows differ from token to token, and longer walks left SMs waiting for
// each other (58,700 rows of 2048 columns: 89 us, two tokens to a warp 92, four 95, eight 113, one block per SM 110).
// SPLIT, for fewer than two tokens per SM: a block of eight warps to a token, each with its share of the row's chunks; their dots
// meet at the end (64 tokens of 7168 columns, top-8: 7.5 us, 28 without; 200 of 4096, top-4: 6.7 and 9.4; 512: 15.7 and 11.8).
constexpr int CG_WARPS = 2, CG_DEPTH = 3, CG_SPLIT = 8, SPLIT_BELOW = 2;
using RingC = Ring<ROWS + 1, CG_DEPTH>;
template <typename T, bool SPLIT>
__global__ void __launch_bounds__((SPLIT ? CG_SPLIT : CG_WARPS) * 32)
k_combine_grad(const uint4* __restrict__ dy, const uint4* __restrict__ y_perm, const int32_t* __restrict__ slot_row,
               const float* __restrict__ perm_weight, int64_t N, int row_vecs, int slots, int64_t rows,
               uint4* __restrict__ dy_perm, float* __restrict__ dweight) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int NV = Vec16<T>::n;
  extern __shared__ uint4 smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  RingC& ring = reinterpret_cast<RingC*>(smem)[warp];
  __shared__ float part[SPLIT ? MAX_SLOTS : 1][CG_SPLIT];
  __shared__ int32_t part_row[SPLIT ? MAX_SLOTS : 1];
  const int64_t t = SPLIT ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * CG_WARPS + warp;
  const int share = SPLIT ? (row_vecs + CHUNK * CG_SPLIT - 1) / (CHUNK * CG_SPLIT) * CHUNK : row_vecs;
  const int begin = SPLIT ? min(row_vecs, warp * share) : 0, end = min(row_vecs, begin + share);
  int32_t mine = slot_at(slot_row, t, N, lane, slots, rows);
  int s0 = 0, v0 = begin;
  unsigned rem = __ballot_sync(0xffffffffu, mine >= 0);
  auto step = [&](int s) {                   // describes and fetches the next stage: rows four at a time, all chunks of them
    while (!rem && s0 + 32 < slots) {
      s0 += 32;
      mine = slot_at(slot_row, t, N, s0 + lane, slots, rows);
      rem = __ballot_sync(0xffffffffu, mine >= 0);
    }
    Stage& st = ring.stage[s];
    int n = -1;
    if (rem && begin < end) {
      fetch_chunk(ring, s, ROWS, dy + t * row_vecs, v0, end);
      unsigned left = rem;
#pragma unroll
      for (n = 0; n < ROWS; ++n) {
        if (!left) break;
        const int32_t r = __shfl_sync(0xffffffffu, mine, __ffs(left) - 1);
        left &= left - 1;
        fetch_chunk(ring, s, n, y_perm + (int64_t)r * row_vecs, v0, end);
        if (lane == n) {
          st.row[n] = r;
          copy4((uint32_t)__cvta_generic_to_shared(&st.w[n]), perm_weight + r);
        }
      }
      if (lane == 0) { st.v0 = v0; st.first = v0 == begin; st.last = v0 + CHUNK >= end; }
      v0 += CHUNK;
      if (v0 >= end) { v0 = begin; rem = left; }
    }
    if (lane == 0) st.n = n;
    copies_commit();
  };
#pragma unroll 1
  for (int s = 0; s < CG_DEPTH - 1; ++s) step(s);
  float dot[ROWS] = {0.f, 0.f, 0.f, 0.f};
  int done = 0;                              // rows
  for (int s = 0;;) {
    step(s == 0 ? CG_DEPTH - 1 : s - 1);
    copies_wait<CG_DEPTH - 1>();
    __syncwarp();
    const Stage& st = ring.stage[s];
    const int n = st.n;
    if (n < 0) break;
    if (st.first) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) dot[i] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < PV; ++u) {
      const int v = st.v0 + u * 32 + lane;
      if (v < end) {
        float g[NV];
        Vec16<T>::load(ring.data[s][ROWS][u * 32 + lane], g);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          if (i >= n) break;
          float f[NV];
          Vec16<T>::load(ring.data[s][i][u * 32 + lane], f);
          const float w = st.w[i];
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            dot[i] = fmaf(g[j], f[j], dot[i]);
            f[j] = w * g[j];
          }
          dy_perm[(int64_t)st.row[i] * row_vecs + v] = Vec16<T>::store(f);
        }
      }
    }
    if (st.last) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        if (i >= n) break;
        float d = dot[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
        if (lane == 0) {
          if constexpr (SPLIT) {
            part[done + i][warp] = d;
            if (warp == 0) part_row[done + i] = st.row[i];
          } else {
            dweight[st.row[i]] = d;
          }
        }
      }
      done += n;
    }
    __syncwarp();                            // the stage's description is rewritten next
    if (++s == CG_DEPTH) s = 0;
  }
  if constexpr (SPLIT) {                     // all warps with a share have seen the same rows in the same order; warp 0 has one
    __syncthreads();
    if (warp == 0) {
      const int with = min(CG_SPLIT, (row_vecs + share - 1) / share);
      for (int i = lane; i < done; i += 32) {
        float d = 0.f;
        for (int w = 0; w < with; ++w) d += part[i][w];
        dweight[part_row[i]] = d;
      }
    }
  }
}

// Work unit = (token, 1 KB chunk of its row), one warp each, up to ROWS rows of it at once in registers; warps walk the units.
constexpr int PG_WARPS = 8, PG_BLOCKS = 4;   // of a block, blocks per SM
template <typename T>
__device__ __forceinline__ void add_vec(float* acc, const uint4& v) {
  float f[Vec16<T>::n];
  Vec16<T>::load(v, f);
#pragma unroll
  for (int i = 0; i < Vec16<T>::n; ++i) acc[i] += f[i];
}
template <typename T>
__global__ void __launch_bounds__(PG_WARPS * 32, PG_BLOCKS)
k_permute_grad(const uint4* __restrict__ dx_perm, const int32_t* __restrict__ slot_row, int64_t N, int row_vecs, int chunks, int slots,
               int64_t rows, const uint4* add0, const uint4* add1, uint4* dx /* may be add0 or add1 */) {
  allow_next_kernel();
  wait_for_previous_kernel();
  constexpr int NV = Vec16<T>::n;
  const int lane = threadIdx.x & 31;
  const int64_t units = N * chunks, step = (int64_t)gridDim.x * PG_WARPS;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  int64_t unit = (int64_t)blockIdx.x * PG_WARPS + (threadIdx.x >> 5), t = unit / chunks;
  int32_t mine = slot_at(slot_row, t, N, lane, slots, rows);
  for (; unit < units; unit += step) {
    const int v0 = (int)(unit - t * chunks) * CHUNK + lane;
    const int64_t t_next = (unit + step) / chunks;
    const int32_t next = slot_at(slot_row, t_next, N, lane, slots, rows);
    float acc[PV][NV];
#pragma unroll
    for (int u = 0; u < PV; ++u) {
      const bool in = v0 + u * 32 < row_vecs;
      Vec16<T>::load(add0 && in ? __ldcs(add0 + t * row_vecs + v0 + u * 32) : zero, acc[u]);
      if (add1) add_vec<T>(acc[u], in ? __ldcs(add1 + t * row_vecs + v0 + u * 32) : zero);
    }
    for (int s0 = 0; s0 < slots; s0 += 32) {
      if (s0 > 0) mine = slot_at(slot_row, t, N, s0 + lane, slots, rows);
      for (unsigned rem = __ballot_sync(0xffffffffu, mine >= 0); rem;) {
        uint4 raw[ROWS][PV];
        int n = 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          const int64_t r = __shfl_sync(0xffffffffu, mine, rem ? __ffs(rem) - 1 : 0);
          n += rem != 0;
#pragma unroll
          for (int u = 0; u < PV; ++u) raw[i][u] = rem && v0 + u * 32 < row_vecs ? __ldcs(dx_perm + r * row_vecs + v0 + u * 32) : zero;
          rem &= rem - 1;                    // no-op when rem is already 0
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          if (i >= n) break;
#pragma unroll
          for (int u = 0; u < PV; ++u) add_vec<T>(acc[u], raw[i][u]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < PV; ++u)
      if (v0 + u * 32 < row_vecs) dx[t * row_vecs + v0 + u * 32] = Vec16<T>::store(acc[u]);
    mine = next;
    t = t_next;
  }
}

static_assert(CG_SPLIT * sizeof(RingC) + sizeof(float) * MAX_SLOTS * (CG_SPLIT + 1) <= 227 * 1024, "shared memory of a thread block");

template <class... KArgs, class... Args>
int launch_wide(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t st, Args... args) {
  const cudaError_t err = allow_smem(kernel, smem);
  if (err != cudaSuccess) return note_cuda(err);
  const int rc = note_cuda(launch_chained(kernel, grid, block, smem, st, args...));
  count_launch(1);
  return rc;
}
template <typename T>
int combine_grad(const void* dy, const void* y_perm, const int32_t* slot_row, const float* perm_weight, int64_t N, int row_vecs, int slots, int64_t rows,
                 void* dy_perm, float* dweight, cudaStream_t st) {
  const bool split = row_vecs > 2 * CHUNK && N < SPLIT_BELOW * (int64_t)sm_count();
  auto k = split ? k_combine_grad<T, true> : k_combine_grad<T, false>;
  const int warps = split ? CG_SPLIT : CG_WARPS;
  return launch_wide(k, dim3((unsigned)(split ? N : ceil_div(N, CG_WARPS))), 32u * (unsigned)warps, warps * sizeof(RingC), st, (const uint4*)dy,
                     (const uint4*)y_perm, slot_row, perm_weight, N, row_vecs, slots, rows, (uint4*)dy_perm, dweight);
}

int check_rows(int64_t N, int d, int slots, int64_t rows, size_t elt) {
  if (N < 0 || d < 1 || slots < 1 || rows < 0) return CAPMOE_EINVAL;
  if (slots > MAX_SLOTS || ((size_t)d * elt) % 16 != 0 || rows >= ((int64_t)1 << 31) || N >= ((int64_t)1 << 31)) return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}

}  // namespace
}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_permute_fp8(const void* x_q, const void* x_scale, int64_t N, int d, int E, int k, int slots, int D, int64_t A_max,
                                  const float* scores, const int32_t* topk_idx, const int32_t* token_group, const int32_t* slot_row,
                                  void* q_perm, void* scale_perm, int32_t* perm_token, float* perm_weight, int32_t* dev_status, void* stream) {
  if (E < 1 || k < 1 || k > E || D < 0 || slots < k) return CAPMOE_EINVAL;
  if (D > 0 ? E % D != 0 || slots != k + E / D : slots != k) return CAPMOE_EINVAL;
  const int rc = check_rows(N, d, slots, A_max, 1);
  if (rc != CAPMOE_OK) return rc;
  if (N == 0 || A_max == 0) return CAPMOE_OK;
  if (!usable(x_q, q_perm) || !x_scale || !scale_perm || !scores || !topk_idx || !slot_row || !perm_token || !perm_weight) return CAPMOE_EINVAL;
  const int nb = (int)ceil_div(d, QBLOCK);
  const uintptr_t all = (uintptr_t)nb | (uintptr_t)x_scale | (uintptr_t)scale_perm;
  const int width = all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : 1;
  const int piece = d < P8_PIECE ? d : P8_PIECE;
  int64_t per = d <= 512 ? 8 : P8_BYTES / piece < 4 ? P8_BYTES / piece : 4;
  const int64_t even = ceil_div(N, (int64_t)sm_count() * 12);  // (few tokens: spread over the SMs)
  per = per < even ? per : even;
  return launch_wide(k_permute8, dim3((unsigned)ceil_div(N, per), (unsigned)ceil_div(d, piece)), 32, (size_t)per * piece, as_stream(stream),
                     (const uint8_t*)x_q, (const uint8_t*)x_scale, N, d, piece, (int)per, nb, width, E, k, slots, D, A_max, scores, topk_idx,
                     token_group, slot_row, (uint8_t*)q_perm, (uint8_t*)scale_perm, perm_token, perm_weight, dev_status);
}

extern "C" int capmoe_combine_backward(const void* dy, const void* y_perm, const int32_t* slot_row, const float* perm_weight, int64_t N, int d,
                                       int slots, int dtype, int64_t A_max, void* dy_perm, float* dweight, void* stream) {
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  const int rc = check_rows(N, d, slots, A_max, elt_size(dtype));
  if (rc != CAPMOE_OK) return rc;
  if (N == 0 || A_max == 0) return CAPMOE_OK;
  if (!usable(dy, y_perm, dy_perm) || !slot_row || !perm_weight || !dweight) return CAPMOE_EINVAL;
  const int row_vecs = (int)((size_t)d * elt_size(dtype) / 16);
  if (dtype == CAPMOE_F32) return combine_grad<float>(dy, y_perm, slot_row, perm_weight, N, row_vecs, slots, A_max, dy_perm, dweight, as_stream(stream));
  return combine_grad<__nv_bfloat16>(dy, y_perm, slot_row, perm_weight, N, row_vecs, slots, A_max, dy_perm, dweight, as_stream(stream));
}

extern "C" int capmoe_permute_backward(const void* dx_perm, const int32_t* slot_row, int64_t N, int d, int slots, int dtype, int64_t A_max,
                                       const void* add0, const void* add1, void* dx, void* stream) {
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  const int rc = check_rows(N, d, slots, A_max, elt_size(dtype));
  if (rc != CAPMOE_OK) return rc;
  if (N == 0) return CAPMOE_OK;
  if (!usable(dx) || !slot_row || (A_max > 0 && !dx_perm) || !aligned16(dx_perm) || !aligned16(add0) || !aligned16(add1)) return CAPMOE_EINVAL;
  const int row_vecs = (int)((size_t)d * elt_size(dtype) / 16), chunks = (int)ceil_div(row_vecs, CHUNK);
  const int64_t want = ceil_div(N * chunks, PG_WARPS), most = (int64_t)sm_count() * PG_BLOCKS;
  const int status = note_cuda(launch_chained(dtype == CAPMOE_F32 ? k_permute_grad<float> : k_permute_grad<__nv_bfloat16>,
                                              (unsigned)(want < most ? want : most), PG_WARPS * 32, 0, as_stream(stream), (const uint4*)dx_perm,
                                              slot_row, N, row_vecs, chunks, slots, A_max, (const uint4*)add0, (const uint4*)add1, (uint4*)dx));
  count_launch(1);
  return status;
}
