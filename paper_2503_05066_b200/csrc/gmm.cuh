// Internal interface of the grouped products (grouped_mm.cu and the tensor-core files behind it).
#pragma once
#include "common.cuh"

namespace capmoe {

constexpr int GMM_MAX_E = 256;               // segments per call (the kernels keep their bounds in shared memory)
// Row counts are rounded up to whole tiles (256 rows) and row numbers run up to a tile past the last row, in 32 bits.
constexpr int64_t GMM_MAX_ROWS = ((int64_t)1 << 31) - 512;
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

// Whether the 8-bit gate/up product takes its tokens on the N side (gmm_rows.cu): average segment below `limit` rows,
// unless capmoe_debug_ffn_variant forces one form.
inline bool use_short(const Segments& sg, int64_t limit) {
  const int v = ffn_variant();
  if (v == FFN_SHORT) return true;
  if (v == FFN_PAIR) return false;
  return (int64_t)sg.rows < limit * sg.E;
}

// Tensor-core kernels.  All matrices 16-byte aligned, `sched` a zeroed tile counter or NULL.
// bf16 (gmm_rows.cu, gmm_dw.cu): rows of whole 16-byte vectors; dw's E * n (E * d) rows are 32-bit coordinates.  map_ws is
// 128-byte aligned with gmm_dw_map_bytes(E, lists) bytes (gmm_dw: 2 lists, gmm_dw_ffn_maps: 5).  gmm_dw clears its counter itself.
inline bool gmm_supported(int E, int d, int n, int dtype) {
  const int64_t lim = (int64_t)1 << 31;
  return dtype == CAPMOE_BF16 && d % 8 == 0 && n % 8 == 0 && (int64_t)E * n < lim && (int64_t)E * d < lim;
}
// `early`: the caller vouches that offsets, weights and the cleared counter were final before any kernel of this call that
// may still run began its work: the call's first kernel lets its successor start only after its own wait for what came
// before (wait_for_previous_kernel, then allow_next_kernel), the ones between may be early themselves.  The kernel then
// fetches its first weights while the previous one, which makes the token rows, still runs (8-bit FFN of a decode step,
// 310 rows of 60 experts, with tile counters: 96 us, 102 without).
int gmm_fwd(const void* x, const Segments& sg, const void* w, int d, int n, void* y, int32_t* dev_status, int32_t* sched,
            bool early, cudaStream_t st);
int gmm_dx(const void* dy, const Segments& sg, const void* w, int d, int n, void* dx, int32_t* dev_status, int32_t* sched,
           bool early, cudaStream_t st);
int gmm_hidden(const void* x, const void* dy, const Segments& sg, int d, int F, const void* wg, const void* wu, const void* wd,
               void* dg, void* du, void* h, int32_t* dev_status, int32_t* sched, bool early, cudaStream_t st);
int gmm_dx2(const void* dg, const void* du, const Segments& sg, int d, int F, const void* wg, const void* wu, void* dx,
            int32_t* dev_status, int32_t* sched, bool early, cudaStream_t st);
size_t gmm_dw_map_bytes(int E, int lists);
// into how many parts the reductions of `products` gradients are split when `parts` (16-byte aligned) has room for them
int gmm_dw_split(int64_t rows, int E, int d, int n, int products);
size_t gmm_dw_parts_bytes(int E, int d, int n, int products, int split);
int gmm_dw(const void* dy, const void* x, const Segments& sg, int d, int n, bool out_f32, void* dw, void* map_ws, float* parts,
           int split, int32_t* dev_status, int32_t* sched, cudaStream_t st);
// the FFN's three weight gradients: the maps first (they need the addresses only, so they can be made ahead)
int gmm_dw_ffn_maps(const void* dg, const void* du, const void* dy, const void* x, const void* h, const Segments& sg, int d, int F,
                    void* map_ws, cudaStream_t st);
int gmm_dw_ffn(const Segments& sg, int d, int F, void* dwg, void* dwu, void* dwd, const void* map_ws, float* parts, int split,
               int32_t* dev_status, int32_t* sched, cudaStream_t st);
// 8-bit (gmm_rows.cu, gmm_swiglu8.cu): d and n (F) multiples of 16; xs_ld, hs_ld: bytes from one row's scales to the next's
inline bool gmm8_supported(int d, int n) { return d % 16 == 0 && n % 16 == 0; }
int gmm8(const uint8_t* xq, const uint8_t* xs, int64_t xs_ld, const Segments& sg, const uint8_t* wq, const uint8_t* ws, int d, int n, void* y,
         int32_t* dev_status, int32_t* sched, bool early, cudaStream_t st);
int gmm8_swiglu(const uint8_t* xq, const uint8_t* xs, int64_t xs_ld, const Segments& sg, const uint8_t* wg, const uint8_t* wgs,
                const uint8_t* wu, const uint8_t* wus, int d, int F, uint8_t* hq, uint8_t* hs, int64_t hs_ld, int32_t* dev_status,
                int32_t* sched, bool early, cudaStream_t st);
// Whether gmm8_swiglu's kernel lets its successor start only after its own wait for what came before: its short form does.
bool gmm8_swiglu_waits_first(const Segments& sg);
int gmm8_swiglu_short(const uint8_t* xq, const uint8_t* xs, int64_t xs_ld, const Segments& sg, const uint8_t* wg, const uint8_t* wgs,
                      const uint8_t* wu, const uint8_t* wus, int d, int F, uint8_t* hq, uint8_t* hs, int64_t hs_ld, int32_t* dev_status,
                      int32_t* sched, bool early, cudaStream_t st);

// Tile counters in the caller's status block, one per launch of a call: cleared by begin_counters, slot i by counter_at.
// Row products of up to 64 allocated rows per expert do without: every tile streams the same weight bytes, so fixed lists
// are as even, and the launch that clears the counter costs 3 us (8-bit product of a decode step, 310 rows of 60 experts:
// 33.7 us without, 36.8 with).
inline int32_t* counter_at(int32_t* dev_status, int i) { return dev_status ? dev_status + 1 + i : nullptr; }
inline int begin_counters(int32_t* dev_status, int n, cudaStream_t st) {
  return dev_status ? clear_words(dev_status + 1, n, nullptr, 0, st) : CAPMOE_OK;
}
inline int32_t* counters_of(const Segments& sg, int32_t* dev_status) {
  return (int64_t)sg.rows > (int64_t)64 * sg.E ? dev_status : nullptr;
}

}  // namespace capmoe
