// Additions to tc_common.cuh for the grouped products: MN-major operand descriptors, fp32 store boxes.
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

// store_piece for the second and third piece of a chunk: the wait for this warp's earlier stores, made by the
// first piece, covers their staging buffers too.
__device__ __forceinline__ void store_piece2(const uint32_t* packed, bool full_rows, bool row_ok, uint8_t* stg,
                                             const CUtensorMap* map_out, int col, int row0_of_warp, __nv_bfloat16* orow_c,
                                             int cols_left) {
  const int lane = threadIdx.x & 31;
  if (full_rows) {
    const uint32_t base = smem_u32(stg) + (uint32_t)lane * 64u;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (uint32_t)((v ^ ((lane >> 1) & 3)) * 16)),
                   "r"(packed[4 * v]), "r"(packed[4 * v + 1]), "r"(packed[4 * v + 2]), "r"(packed[4 * v + 3])
                   : "memory");
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(map_out, col, row0_of_warp, smem_u32(stg));
      bulk_commit();
    }
  } else if (row_ok) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (v * 8 + 8 <= cols_left)
        *reinterpret_cast<uint4*>(orow_c + v * 8) =
            make_uint4(packed[4 * v], packed[4 * v + 1], packed[4 * v + 2], packed[4 * v + 3]);
  }
}

// fp32 matrix [rows, cols] as 32-row x 16-column boxes (64-byte rows, as the bf16 boxes of 32 columns)
bool make_store_map_f32(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {cols, rows};
  cuuint64_t strides[1] = {cols * 4};
  cuuint32_t box[2] = {16, 32};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

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
constexpr int SF_RING = 3;                  // scale groups in flight
constexpr int SF_CHUNK = 512;               // bytes of shared memory for 128 rows
constexpr int SF_COLS = 16;                 // tensor-memory columns per group (12 used)
constexpr int SF_TMEM = 448;                // first column of the scales
constexpr int F8_THREADS = TC_THREADS + 32; // one more warp: it stages the scales
constexpr int TQ_READERS_F8 = TQ_READERS_PAIR + 2;

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
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_acquire_cluster() { asm volatile("fence.acq_rel.cluster;" ::: "memory"); }

// Four scale bytes s[0..3] of a row of nb scales from position k on; those behind the row count as 2^0 (their codes are
// zeros that TMA filled in).
__device__ __forceinline__ uint32_t scale_word(const uint8_t* row, int k, int nb, bool words) {
  if (words) return *reinterpret_cast<const uint32_t*>(row + k);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) w |= (k + i < nb ? (uint32_t)row[k + i] : 127u) << (8 * i);
  return w;
}
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
