// Additions to tc_common.cuh for the grouped products: MN-major operands, the wide and the transposing epilogue, the tile
// ring with its scheduler, and what the block-scaled 8-bit MMAs need.
#pragma once
#include "tc_common.cuh"

namespace capmoe {
namespace {

// Shared-memory descriptor of an MN-major operand: boxes of 64 output indices (one 128-byte swizzle row) by 64
// reduction steps, 8 KB apart along the output index (leading byte offset), 8 reduction steps 1 KB apart (stride
// byte offset).
__device__ __forceinline__ uint64_t umma_desc_mn(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3ffffu) >> 4);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// kind::f16 on a CTA pair: D = fp32, A = B = bf16, M = 256, N = n; transpose bits for MN-major operands
__device__ __forceinline__ uint32_t pair_idesc(int n, bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)((2 * BM) >> 4) << 24);
}

// A wide piece of an output: 32 rows of 128 bytes (64 bf16 or 32 fp32 columns), lane r holding row r as 32 words.  With all
// 32 rows inside the segment it goes out as one TMA box (128-byte swizzle) from a 4 KB buffer of the warp, else row by
// row.  `bytes_left`: of the output row from this piece on, a multiple of 16.  Against 64-byte pieces this halves the
// proxy fences and store instructions, which cost about 400 cycles a piece and bound short reductions.
constexpr int WIDE_BYTES = 32 * 128;
__device__ __forceinline__ void put_wide(const uint32_t* w, bool full_rows, bool row_ok, uint8_t* stg, const CUtensorMap* map_out,
                                         int col, int row0_of_warp, void* orow_c, int bytes_left) {
  const int lane = threadIdx.x & 31;
  if (full_rows) {
    if (lane == 0) bulk_wait_read_all();                       // the previous piece has left the buffer
    __syncwarp();
    const uint32_t base = smem_u32(stg) + (uint32_t)lane * 128u;
#pragma unroll
    for (int v = 0; v < 8; ++v)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (uint32_t)((v ^ (lane & 7)) * 16)), "r"(w[4 * v]),
                   "r"(w[4 * v + 1]), "r"(w[4 * v + 2]), "r"(w[4 * v + 3])
                   : "memory");
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(map_out, col, row0_of_warp, smem_u32(stg));
      bulk_commit();
    }
  } else if (row_ok) {
#pragma unroll
    for (int v = 0; v < 8; ++v)
      if (v * 16 + 16 <= bytes_left)
        reinterpret_cast<uint4*>(orow_c)[v] = make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
  }
}

// ---- transposing epilogue: accumulator lanes are output columns, accumulator columns are output rows (tokens)
// 16 lanes x 32 columns of the accumulator as 8 x 8 fragments: of columns 8j .. 8j+7, thread t gets lane t/4, columns
// 8j + 2(t%4) and the next (r[4j], r[4j+1]), and the same of lane t/4 + 8 (r[4j+2], r[4j+3]).
__device__ __forceinline__ void tmem_ld_frag(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// A warp's buffer: 32 tokens x 64 bytes (32 columns of 16 bits), 16-byte chunks swizzled.  Four 8 x 8 fragments of 16-bit
// values, lanes 0..31 of tokens 8j .. 8j+7, written transposed.
__device__ __forceinline__ void put_frag(uint32_t stg, int j, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const int lane = threadIdx.x & 31;
  const uint32_t row = (uint32_t)(8 * j + (lane & 7)), chunk = (uint32_t)(lane >> 3);
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
               ::"r"(stg + row * 64u + ((chunk ^ ((row >> 1) & 3u)) << 4)), "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}
__device__ __forceinline__ uint4 get_chunk(uint32_t stg, uint32_t row, uint32_t chunk) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(stg + row * 64u + ((chunk ^ ((row >> 1) & 3u)) << 4))
               : "memory");
  return v;
}
// The buffer's first n tokens to global memory, four lanes per token (whole 64-byte runs); `out`: first token, first of the
// warp's columns; `cols`: columns that exist from there on (a multiple of 8; may be zero or negative).
__device__ __forceinline__ void flush_tokens(uint32_t stg, __nv_bfloat16* out, int64_t ld, int n, int cols) {
  const int lane = threadIdx.x & 31, chunk = lane & 3;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 8 * i + (lane >> 2);
    const uint4 v = get_chunk(stg, (uint32_t)row, (uint32_t)chunk);
    if (row < n && chunk * 8 < cols) *reinterpret_cast<uint4*>(out + (int64_t)row * ld + chunk * 8) = v;
  }
  __syncwarp();
}
// The same for 8-bit values, one in the low byte of each 16: two lanes per token, 16 columns each.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x6420); }
__device__ __forceinline__ void flush_tokens_u8(uint32_t stg, uint8_t* out, int64_t ld, int n, int cols) {
  const int lane = threadIdx.x & 31, part = lane & 1;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 16 * i + (lane >> 1);
    const uint4 a = get_chunk(stg, (uint32_t)row, (uint32_t)(2 * part)), b = get_chunk(stg, (uint32_t)row, (uint32_t)(2 * part + 1));
    if (row < n && part * 16 < cols)
      *reinterpret_cast<uint4*>(out + (int64_t)row * ld + part * 16) =
          make_uint4(low_bytes(a.x, a.y), low_bytes(a.z, a.w), low_bytes(b.x, b.y), low_bytes(b.z, b.w));
  }
  __syncwarp();
}

__device__ __forceinline__ void tma2_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}

// Output matrix [rows, cols] (elements of 4 or 2 bytes) in boxes of 32 rows x 128 bytes, 128-byte swizzle
bool make_wide_map(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, int elt) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {cols, rows};
  cuuint64_t strides[1] = {cols * (uint64_t)elt};
  cuuint32_t box[2] = {(cuuint32_t)(128 / elt), 32};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, elt == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// MN-major operand: bf16 [rows, cols] or [batch, rows, cols], the reduction along the rows.  When the columns are whole
// blocks of 64 the map splits them, (64, rows, cols / 64 [, batch]), and one box brings 128 columns by 64 rows in the order
// the MMA descriptor wants; otherwise boxes of 64 columns.  mn_wide tells which.
bool mn_wide(int64_t cols) { return cols % 64 == 0; }
bool make_mn_map(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint64_t batch) {
  if (!mn_wide((int64_t)cols)) return make_map(m, base, cols, rows, batch, BK);
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {64, rows, cols / 64, batch};
  cuuint64_t strides[3] = {cols * 2, 128, cols * rows * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)BK, 2, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, batch > 0 ? 4 : 3, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 128 columns from c on (a multiple of 64) by 64 reduction steps from k on
__device__ __forceinline__ void load_mn(uint32_t dst, const CUtensorMap* m, bool wide, int c, int k, uint32_t bar) {
  if (wide) {
    tma2_load_3d(dst, m, 0, k, c >> 6, bar);
  } else {
    tma2_load_2d(dst, m, c, k, bar);
    tma2_load_2d(dst + 8192u, m, c + 64, k, bar);
  }
}
__device__ __forceinline__ void load_mn(uint32_t dst, const CUtensorMap* m, bool wide, int c, int k, int e, uint32_t bar) {
  if (wide) {
    tma2_load_4d(dst, m, 0, k, c >> 6, e, bar);
  } else {
    tma2_load_3d(dst, m, c, k, e, bar);
    tma2_load_3d(dst + 8192u, m, c + 64, k, e, bar);
  }
}

// ---------------------------------------------------------------- tile ring
// One thread of its own warp (the scheduler) picks a CTA's tiles, works out where they lie and hands each on as a record of
// eight ints through a ring in shared memory; the other roles only read records.  The first tile of a pair is its
// index; with a counter the further ones are claimed from it by the leader's scheduler, which passes them to the
// peer's through a two-deep mailbox.  Decoding a tile and claiming the next takes about 1300 cycles; inside the TMA
// thread that was a quarter of a weight-gradient tile's time.
// Four records: one each for epilogue, MMAs and loads, and one ahead.
constexpr int TR = 4;
constexpr int TR_BYTES = TR * 32;
struct TileRing {
  uint32_t bar0;                     // barriers: full[TR], empty[TR], xfull[2], xempty[2] (leader's used), then two ints
  uint32_t rec0;                     // records
  uint32_t rank;
  volatile int* abort_flag;
  long long limit = WAIT_LIMIT_CYCLES;   // of a wait, which may last as long as a tile
  __device__ __forceinline__ uint32_t full(int j) const { return bar0 + 8u * (uint32_t)(j & (TR - 1)); }
  __device__ __forceinline__ uint32_t empty(int j) const { return bar0 + 8u * (uint32_t)(TR + (j & (TR - 1))); }
  __device__ __forceinline__ uint32_t xfull(int q) const { return bar0 + 8u * (uint32_t)(2 * TR + (q & 1)); }
  __device__ __forceinline__ uint32_t xempty(int q) const { return bar0 + 8u * (uint32_t)(2 * TR + 2 + (q & 1)); }
  __device__ __forceinline__ uint32_t xval(int q) const { return bar0 + 8u * (uint32_t)(2 * TR + 4) + 4u * (uint32_t)(q & 1); }
  __device__ __forceinline__ void init(int readers) const {
    for (int i = 0; i < TR; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), (uint32_t)readers); }
    for (int q = 0; q < 2; ++q) { mbar_init(xfull(q), 1); mbar_init(xempty(q), 1); }
  }
  // Record j for one thread or one whole warp; false when there is no further tile or a wait ran out.
  __device__ __forceinline__ bool get(int j, bool whole_warp, int4& a, int4& b) const {
    bool ok = mbar_wait(full(j), ((uint32_t)j / TR) & 1u, abort_flag, limit);
    if (whole_warp) ok = __all_sync(0xffffffffu, ok);
    if (!ok) return false;
    const uint32_t r = rec0 + 32u * (uint32_t)(j & (TR - 1));
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w) : "r"(r) : "memory");
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(r + 16u) : "memory");
    if (whole_warp) __syncwarp();
    if (!whole_warp || (threadIdx.x & 31) == 0) mbar_arrive(empty(j));
    return a.x >= 0;
  }
  __device__ __forceinline__ bool put(int j, const int4& a, const int4& b) const {
    if (!mbar_wait(empty(j), (((uint32_t)j / TR) & 1u) ^ 1u, abort_flag, limit)) return false;
    const uint32_t r = rec0 + 32u * (uint32_t)(j & (TR - 1));
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(r), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(r + 16u), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
    mbar_arrive(full(j));
    return true;
  }
  // The scheduler thread of either CTA.  decode(tile, a, b) fills the record of a tile below tile_hi; a.x >= 0.
  template <class Decode>
  __device__ __forceinline__ void run(int pair, int npairs, int tile_hi, int32_t* counter, const Decode& decode) const {
    int claim = 0;
    const bool leader = rank == 0;
    if (counter && leader && pair < tile_hi) claim = atomicAdd(counter, 1);
    for (int j = 0;; ++j) {
      int tile = pair + j * npairs;
      if (counter && j > 0) {
        const int q = j - 1;
        const uint32_t use = (uint32_t)q >> 1;
        if (leader) {
          tile = npairs + claim;
          if (tile < tile_hi) claim = atomicAdd(counter, 1);
          if (!mbar_wait_cluster(xempty(q), (use & 1u) ^ 1u, abort_flag, limit)) return;
          const uint32_t pfull = peer_addr(xfull(q));
          asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(pfull), "r"(4u) : "memory");
          asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];"
                       ::"r"(peer_addr(xval(q))), "r"((uint32_t)tile), "r"(pfull)
                       : "memory");
        } else {
          if (!mbar_wait_cluster(xfull(q), use & 1u, abort_flag, limit)) return;
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tile) : "r"(xval(q)) : "memory");
          give_back_slot(xempty(q));
        }
      }
      int4 a = make_int4(-1, 0, 0, 0), b = make_int4(0, 0, 0, 0);
      const bool any = tile < tile_hi;
      if (any) decode(tile, a, b);
      if (!put(j, a, b) || !any) return;
    }
  }
};
constexpr int RING_BAR = 36;              // first of the ring's barriers in a kernel's barrier block

}  // namespace
}  // namespace capmoe

// ---------------------------------------------------------------- 8-bit, block-scaled products
namespace capmoe {
namespace {

// A k-block is 128 bytes of codes = one block of 128 columns, so one scale per operand row and k-block.  The MMA
// (kind::mxf8f6f4, scale_vec::1X) takes 32 columns at a time and one scale byte per row, picked by the descriptor
// out of the 32-bit word that tensor memory holds for the row: a word carries the scales of four k-blocks (a "scale
// group"), and the four MMAs of a k-block name the same byte.  128 rows of scales are 32 lanes x 4 columns (row r in
// lane r % 32, column r / 32), copied by tcgen05.cp from 512 bytes of shared memory with row r's word at
// (r % 32) * 16 + (r / 32) * 4, and repeated for the four lane quarters.
// Shared memory holds them in slots of four groups (16 k-blocks, one 16-byte load per row): the hand-over from the warp
// that stages them to the MMA thread, a fence and a release across the pair, takes about 1300 cycles, more than a
// group of a decode step lasts (one group per slot: 41 us for a decode step's product, 8-bit, of 166 MB of weights).
// Tensor memory holds four groups; a barrier per group says when its MMAs are done.
constexpr int SF_RING = 2;                  // slots
constexpr int SF_GROUPS = 4;                // groups per slot, and in tensor memory
constexpr int SF_CHUNK = 512;               // bytes of shared memory for 128 rows
constexpr int SF_COLS = 16;                 // tensor-memory columns per group (12 used)
constexpr int SF_TMEM = 448;                // first column of the scales
constexpr int F8_THREADS = TC_THREADS + 64; // two more warps: scales and scheduler

__device__ __forceinline__ uint32_t f8_idesc(int n) {     // D = fp32, A = B = e4m3, K-major, ue8m0 scales, M = 256
  return (1u << 23) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)((2 * BM) >> 4) << 24);
}
__device__ __forceinline__ uint32_t f8_scale_byte(int kb) { return ((uint32_t)(kb & 3) << 4) | ((uint32_t)(kb & 3) << 29); }

__device__ __forceinline__ void umma2_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// 32 rows of 16 bytes (no swizzle, 8-row groups 128 bytes apart) to four columns of every lane quarter, in both CTAs
// from their own shared memory
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3ffffu) >> 4);
  d |= (uint64_t)1 << 16;
  d |= (uint64_t)(128 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
}
// arrives on this CTA's barrier once the MMAs and copies issued so far are done
__device__ __forceinline__ void umma2_commit_own(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Scale bytes k .. k + 15 of a row of nb (four scale groups): one 16-byte load where rows start on 16 bytes, else the
// aligned words that hold a byte of the row, shifted into place.  Bytes behind the row are whatever lies there: no k-block
// asks for them.
__device__ __forceinline__ bool scales_aligned(int64_t ld, const void* p) { return (((uintptr_t)ld | (uintptr_t)p) & 15u) == 0; }
__device__ __forceinline__ uint4 scale_words(const uint8_t* row, int k, int nb, bool aligned) {
  if (aligned) return *reinterpret_cast<const uint4*>(row + k);
  const uintptr_t at = (uintptr_t)(row + k), end = (uintptr_t)(row + nb);
  const uint32_t* w = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3);
  const uint32_t shift = (uint32_t)(at & 3u) * 8u;
  uint32_t v[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) v[i] = (uintptr_t)(w + i) < end ? w[i] : 0u;
  return make_uint4(__funnelshift_r(v[0], v[1], shift), __funnelshift_r(v[1], v[2], shift), __funnelshift_r(v[2], v[3], shift),
                    __funnelshift_r(v[3], v[4], shift));
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ void put_words(uint32_t saddr, int lane, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(saddr + (uint32_t)lane * 16u), "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}

// 8-bit tensor [rows, cols] or [batch, rows, cols] in boxes of 128 columns x box_rows
bool make_map_u8(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint64_t batch, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {cols, rows, batch};
  cuuint64_t strides[2] = {cols, cols * rows};
  cuuint32_t box[3] = {128, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, batch > 0 ? 3 : 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 8-bit matrix as 32-row x 64-column boxes with the 64-byte swizzle (stores)
bool make_store_map_u8(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {cols, rows};
  cuuint64_t strides[1] = {cols};
  cuuint32_t box[2] = {64, 32};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace capmoe
