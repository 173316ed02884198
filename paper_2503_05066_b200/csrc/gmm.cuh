// Internal interface of the grouped products (grouped_mm.cu and the tensor-core files behind it).
#pragma once
#include "common.cuh"

namespace capmoe {

constexpr int GMM_MAX_E = 256;               // segments per call (the kernels keep their bounds in shared memory)
constexpr int QBLOCK = 128;                  // columns (and, for weights, rows) that share one scale
constexpr int Q_NAN_SCALE = 255;             // scale code of a block that holds a NaN or an infinity

// Rows [seg[e], seg[e+1]) of expert e, clamped to the rows that were allocated.
struct Segments { const int32_t* offsets; int E; int rows; };

__device__ __forceinline__ int seg_at(const Segments& s, int e) {
  const int v = s.offsets[e];
  return v < 0 ? 0 : v > s.rows ? s.rows : v;
}

// Scale code of a block whose largest magnitude has these fp32 bits: 127 + e with the smallest e such
// that 448 * 2^e is not below it (448 = 1.75 * 2^8 is the largest e4m3 value), at least 2^-127; an
// all-zero block has e = 0, and one with a NaN or an infinity the code of a NaN.
__device__ __forceinline__ uint32_t scale_code(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return Q_NAN_SCALE;
  if (amax_bits == 0u) return 127u;
  const int c = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)(c < 0 ? 0 : c);
}
// 2^-e of a scale code below 255 (a normal number: codes go up to 247), and 2^e.
__device__ __forceinline__ float inv_scale(uint32_t code) { return __uint_as_float((254u - code) << 23); }
__device__ __forceinline__ float scale_value(uint32_t code) {
  if (code == (uint32_t)Q_NAN_SCALE) return __uint_as_float(0x7fffffffu);
  return code ? __uint_as_float(code << 23) : __uint_as_float(0x00400000u);
}
// Two floats to two e4m3 codes (a in the low byte), round to nearest even; |a|, |b| <= 448 after scaling.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}

// Whether a call runs the short-segment kernels (gmm_short.cu): average segment below `limit` rows, unless
// capmoe_debug_ffn_variant forces one form.
inline bool use_short(const Segments& sg, int64_t limit) {
  const int v = ffn_variant();
  if (v == FFN_SHORT) return true;
  if (v == FFN_PAIR) return false;
  return (int64_t)sg.rows < limit * sg.E;
}

// Tensor-core kernels (gmm_tc.cu): bf16 with rows of whole 16-byte vectors.  All matrices 16-byte aligned, map_ws
// 128-byte aligned with gmm_tc_map_bytes(E, lists) bytes (dw: 2 lists, ffn_grad: 5).
bool gmm_tc_supported(int E, int d, int n, int dtype);
size_t gmm_tc_map_bytes(int E, int lists);
int gmm_tc_fwd(const void* x, const Segments& sg, const void* w, int d, int n, void* y, int32_t* dev_status, cudaStream_t st);
int gmm_tc_dx(const void* dy, const Segments& sg, const void* w, int d, int n, void* dx, int32_t* dev_status, cudaStream_t st);
int gmm_tc_dw(const void* dy, const void* x, const Segments& sg, int d, int n, bool out_f32, void* dw, void* map_ws,
              int32_t* dev_status, cudaStream_t st);
int gmm_tc_ffn_grad(const void* x, const void* dy, const Segments& sg, int d, int F, const void* wg, const void* wu,
                    const void* wd, void* dx, void* dwg, void* dwu, void* dwd, void* map_ws, void* hidden, int32_t* dev_status,
                    cudaStream_t st);

// The same products with the weights on the M side (gmm_short.cu).  `sched`: a zeroed tile counter or NULL.
int gmm_short_fwd(const void* x, const Segments& sg, const void* w, int d, int n, void* y, int32_t* dev_status, int32_t* sched,
                  cudaStream_t st);
int gmm_short_dx(const void* dy, const Segments& sg, const void* w, int d, int n, void* dx, int32_t* dev_status, int32_t* sched,
                 cudaStream_t st);
int gmm_short_hidden(const void* x, const void* dy, const Segments& sg, int d, int F, const void* wg, const void* wu,
                     const void* wd, void* dg, void* du, void* h, int32_t* dev_status, int32_t* sched, cudaStream_t st);
int gmm_short_dx2(const void* dg, const void* du, const Segments& sg, int d, int F, const void* wg, const void* wu, void* dx,
                  int32_t* dev_status, int32_t* sched, cudaStream_t st);
int gmm8_short(const uint8_t* xq, const uint8_t* xs, const Segments& sg, const uint8_t* wq, const uint8_t* ws, int d, int n,
               void* y, int32_t* dev_status, int32_t* sched, cudaStream_t st);
int gmm8_short_swiglu(const uint8_t* xq, const uint8_t* xs, const Segments& sg, const uint8_t* wg, const uint8_t* wgs,
                      const uint8_t* wu, const uint8_t* wus, int d, int F, uint8_t* hq, uint8_t* hs, int32_t* dev_status,
                      int32_t* sched, cudaStream_t st);

// Block-scaled 8-bit kernels (gmm_fp8_tc.cu): d and n (F) multiples of 16.  `sched`: a zeroed tile counter or NULL.
bool gmm8_tc_supported(int d, int n);
int gmm8_tc(const uint8_t* xq, const uint8_t* xs, const Segments& sg, const uint8_t* wq, const uint8_t* ws, int d, int n, void* y,
            int32_t* dev_status, int32_t* sched, cudaStream_t st);
int gmm8_tc_swiglu(const uint8_t* xq, const uint8_t* xs, const Segments& sg, const uint8_t* wg, const uint8_t* wgs,
                   const uint8_t* wu, const uint8_t* wus, int d, int F, uint8_t* hq, uint8_t* hs, int32_t* dev_status,
                   int32_t* sched, cudaStream_t st);

}  // namespace capmoe
