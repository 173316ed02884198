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
