// The two products of the router's gradient on tcgen05 for fp32, and for bf16 rows that TMA cannot address:
//   dx[t] = sum_e dl[t,e] W_r[e],   dW_r[e] = sum_t dl[t,e] x[t]
// As in route_grad_tc.cu one pass over x serves both: a CTA owns 128 columns and a range of tokens, W_r's columns stay in shared
// memory, dl comes in tiles of 64 experts by TMA, dW_r^T stays in tensor memory until the range ends.  But x and W_r are read by
// eight warps of their own, element by element or in pairs, neighbouring columns on neighbouring lanes, and laid out for the MMAs
// on the way (rows of 128 bytes, their 16-byte pieces swapped by the row's last three bits).
// fp32 goes in exactly, as three bf16 numbers whose sum it is (route_grad.cu).  Of the nine products of two such sums all but the last
// (2^-30 of the product at most) are added up in fp32, the smallest first (with the six largest, which leave out up to 2^-21, 3 % less
// time).  Three numbers of W_r, x and dl fill the shared memory with 64 experts; more come in passes of 64, the later ones adding to dx.
// The MMAs cut their sums off where fp32 ends.  With up to 64 experts the largest products have an accumulator of dW_r^T to
// themselves, and both are added up in registers every 256 tokens (the error of fp32's dW_r over 4096 tokens a CTA is 3 10^-7 of it like
// this, 3 10^-5 with one accumulator to the end; the time is the same).  bf16 tokens of more experts have one accumulator, registers
// for no more, and ranges of ROUTE_CHAIN tokens at most.
// fp32, 16,384 tokens of 4096 columns, 64 experts: 179 us (plain FMAs 556), bound by the loading warps (two parts of three go
// through subtractions) and by shared memory, which the MMAs read at its full rate; bf16, 16,384 of 2047, 32 experts: 57 us, bound by
// instructions (two loads of two bytes for a word).  Left out: two stages of x ahead in registers (17 % slower, spilled).
#include "gmm_tc.cuh"
#include "route_grad.cuh"

namespace capmoe {
namespace {

constexpr int LOAD_WARPS = 8;
constexpr int ANY_THREADS = TC_THREADS + LOAD_WARPS * 32;
constexpr int DC = 128;                      // columns of a CTA
constexpr int BOX = 64 * 128;                // 64 rows of 64 columns
constexpr int TILE = 2 * BOX;                // 64 rows of 128 columns of x or W_r; 128 tokens of 64 experts of dl

template <typename T, int KB>                // KB: tiles of 64 experts, at most: 1, or of bf16 also 2 or 4
struct RA {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int P = F32 ? 3 : 1;                        // bf16 numbers of an element of x and W_r
  static constexpr int W_BYTES = KB * P * TILE, DL_BYTES = ROUTE_PARTS * TILE, X_BYTES = P * TILE;
  static constexpr int RING = F32 ? 1 : 2;                     // tiles of dl
  static constexpr int NST = F32 || KB == 4 ? 2 : 4;           // stages of x, 64 tokens each
  static constexpr int STG_BYTES = 32 * 33 * 4;                // an epilogue warp's 32 x 32 sums of dx
  static constexpr int DL_OFF = W_BYTES, X_OFF = DL_OFF + RING * DL_BYTES, STG_OFF = X_OFF + NST * X_BYTES;
  static constexpr int TAIL = STG_OFF + EPI_WARPS * STG_BYTES;
  static constexpr int SMEM = TAIL + 1024 + 256;
  static constexpr bool FLUSH = KB == 1;                       // accumulators of dW_r^T: two, of the large products and the others; else one
  static constexpr int GROUP = FLUSH ? 2 : 1 << 30;            // blocks that a set of two takes, two sets in turn
  static constexpr int DW_COLS = FLUSH ? 4 * 64 : KB * 64;     // tensor-memory columns of dW_r^T, then SLOTS x 128 for dx
  static constexpr int SLOTS = 2;
  static_assert(SMEM <= 227 * 1024, "shared memory of a thread block");
  static_assert(DW_COLS + SLOTS * 128 <= 512, "tensor memory");
};
// The products of part i of one factor with part j of the other, the smallest first; w: part of W_r or x, l: part of dl.  (The MMAs cut
// their sums off where fp32 ends: sums should be large late, and not often.)
template <typename T> struct Pairs;
template <> struct Pairs<float> {
  static constexpr int n = 8;
  __device__ static constexpr int l(int i) { constexpr int v[n] = {1, 2, 0, 1, 2, 0, 1, 0}; return v[i]; }
  __device__ static constexpr int w(int i) { constexpr int v[n] = {2, 1, 2, 1, 0, 1, 0, 0}; return v[i]; }
};
template <> struct Pairs<__nv_bfloat16> {
  static constexpr int n = ROUTE_PARTS;
  __device__ static constexpr int l(int i) { return n - 1 - i; }
  __device__ static constexpr int w(int) { return 0; }
};

struct RAMaps { CUtensorMap dl[ROUTE_PARTS]; };
template <typename T>
struct RAArgs {
  const T *x, *w;
  int64_t N;
  int d, E, e0, n, slices, per;              // experts e0 .. e0 + n - 1 of E; per: tokens of a range, a multiple of 64
  T* dx;                                     // is added to from the second pass on
  RouteOut out;
  int32_t* dev_status;
};

// 64 rows of a matrix as the loading warps take them: warp i has 64 of the 128 columns (i & 1) of every fourth row, a lane two
// columns.  PAIR: rows of whole pairs.
template <typename T, bool PAIR>
struct Rows {
  T v[16][2];
  // p: the lane's first column (or any that exists) of row 0; k: the warp's first row; left: rows that exist; next: from a column that
  // does to the one behind it, if that exists, else 0
  __device__ __forceinline__ void fetch(const T* p, int64_t d, int k, int left, int next) {
    const T* q = p + k * d;
    const int64_t step = 4 * d;
#pragma unroll
    for (int i = 0; i < 16; ++i, q += step) {
      const T* at = k + 4 * i < left ? q : p;
      if constexpr (PAIR && sizeof(T) == 4) {
        const float2 f = *reinterpret_cast<const float2*>(at);
        v[i][0] = f.x;
        v[i][1] = f.y;
      } else if constexpr (PAIR) {
        const __nv_bfloat162 f = *reinterpret_cast<const __nv_bfloat162*>(at);
        v[i][0] = f.x;
        v[i][1] = f.y;
      } else {
        v[i][0] = at[0];
        v[i][1] = at[next];
      }
    }
  }
  // `to`: the first of the parts' tiles.  Zeros for rows that do not exist and, by their masks, columns.
  __device__ __forceinline__ void put(uint8_t* to, int k, int left, int half, uint32_t mask0, uint32_t mask1) const {
    const int lane = threadIdx.x & 31;
    to += half * BOX + k * 128;              // row k + 4 i: its last three bits are those of k, the third flipped for odd i
    const int at0 = (lane * 4) ^ (k << 4), at1 = at0 ^ (4 << 4);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      uint8_t* at = to + i * 512 + (i & 1 ? at1 : at0);
      const bool in = k + 4 * i < left;
      if constexpr (sizeof(T) == 4) {
        uint32_t a = __float_as_uint(v[i][0]) & mask0, b = __float_as_uint(v[i][1]) & mask1;
        if (!in) a = b = 0u;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          *reinterpret_cast<uint32_t*>(at + p * TILE) = __byte_perm(a, b, 0x7632);
          const uint32_t ta = a & 0xffff0000u, tb = b & 0xffff0000u;           // (an infinity: zeros, not inf - inf)
          a = a == ta ? 0u : __float_as_uint(__uint_as_float(a) - __uint_as_float(ta));
          b = b == tb ? 0u : __float_as_uint(__uint_as_float(b) - __uint_as_float(tb));
        }
      } else {
        const uint32_t w = (__bfloat16_as_ushort(v[i][0]) & mask0) | (__bfloat16_as_ushort(v[i][1]) & mask1) << 16;
        *reinterpret_cast<uint32_t*>(at) = in ? w : 0u;
      }
    }
  }
};

// Columns of dx, lane r holding row r: `cols` of them of the first `rows` rows go to `out`, whose rows are `ld` apart.  stg: 32 x 33
// words of the warp.
// fp32: 32 columns, with `add` onto what is there (sectors of eight columns straight from registers: 173 -> 181 us for 16,384
// tokens, 64 experts, 4096 columns).
__device__ __forceinline__ void put_sums(const uint32_t* g, uint32_t* stg, float* out, int ld, int rows, int cols, bool add) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 32; ++i) stg[lane * 33 + i] = g[i];
  __syncwarp();
  if (lane < cols) {
    float* to = out + lane;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += 8, to += 8 * (int64_t)ld) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = add && r0 + j < rows ? to[j * (int64_t)ld] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += __uint_as_float(stg[(r0 + j) * 33 + lane]);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (r0 + j < rows) to[j * (int64_t)ld] = v[j];
    }
  }
}
// bf16: a row of 64 columns, which the warp has packed into stg, in words that lie on four bytes, the element in front of them and
// behind them by itself.
__device__ __forceinline__ void put_packed(const uint32_t* stg, __nv_bfloat16* out, int ld, int rows, int cols) {
  const int lane = threadIdx.x & 31;
  const int odd0 = (int)((reinterpret_cast<uintptr_t>(out) >> 1) & 1), odd1 = odd0 ^ (ld & 1);       // rows that start between words
  const int col0 = 2 * lane - odd0, col1 = 2 * lane - odd1;
  const bool in0 = col0 >= 0 && col0 + 1 < cols, in1 = col1 >= 0 && col1 + 1 < cols;
  const uint32_t pick0 = odd0 ? 0x5432u : 0x7654u, pick1 = odd1 ? 0x5432u : 0x7654u;
  const int64_t step = 2 * (int64_t)ld;
  __nv_bfloat16 *p0 = out + col0, *p1 = out + ld + col1;
  const uint32_t* from = stg + lane;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += 8) {       // (eight rows' words first: the compiler keeps stores and loads that might overlap in order)
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __byte_perm(from[(r0 + j) * 33 - (lane > 0)], from[(r0 + j) * 33], j & 1 ? pick1 : pick0);
#pragma unroll
    for (int j = 0; j < 8; j += 2, p0 += step, p1 += step) {
      if (in0 && r0 + j < rows) *reinterpret_cast<uint32_t*>(p0) = w[j];
      if (in1 && r0 + j + 1 < rows) *reinterpret_cast<uint32_t*>(p1) = w[j + 1];
    }
  }
  if (lane < rows) {
    const int odd = lane & 1 ? odd1 : odd0;
    __nv_bfloat16* p = out + (int64_t)lane * ld;
    if (odd) p[0] = __ushort_as_bfloat16((unsigned short)(stg[lane * 33] & 0xffffu));
    if ((cols & 1) != odd) p[cols - 1] = __ushort_as_bfloat16((unsigned short)(stg[lane * 33 + (cols - 1) / 2] >> (cols & 1 ? 0 : 16)));
  }
}

template <typename T, int KB, bool PAIR>
__global__ void __launch_bounds__(ANY_THREADS, 1) k_route_grad_any(const __grid_constant__ RAMaps mp, const __grid_constant__ RAArgs<T> ar) {
  using S = RA<T, KB>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (tiles - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + S::TAIL);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 24);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto xfull = [&](int s) { return bar0 + 8u * (uint32_t)s; };                 // stages of x
  auto xempty = [&](int s) { return bar0 + 8u * (uint32_t)(4 + s); };
  auto dfull = [&](int r) { return bar0 + 8u * (uint32_t)(8 + r); };           // tiles of dl
  auto dempty = [&](int r) { return bar0 + 8u * (uint32_t)(10 + r); };
  auto sfull = [&](int s) { return bar0 + 8u * (uint32_t)(12 + s); };          // dx accumulators
  auto sempty = [&](int s) { return bar0 + 8u * (uint32_t)(14 + s); };
  const uint32_t wfull = bar0 + 8u * 16u;                                      // W_r has arrived
  auto gfull = [&](int g) { return bar0 + 8u * (uint32_t)(17 + g); };          // accumulators of dW_r
  auto gempty = [&](int g) { return bar0 + 8u * (uint32_t)(19 + g); };

  if (tid == 0) {
    for (int s = 0; s < S::NST; ++s) { mbar_init(xfull(s), LOAD_WARPS); mbar_init(xempty(s), 1); }
    for (int r = 0; r < S::RING; ++r) { mbar_init(dfull(r), 1); mbar_init(dempty(r), 1); }
    for (int s = 0; s < S::SLOTS; ++s) { mbar_init(sfull(s), 1); mbar_init(sempty(s), EPI_WARPS); }
    mbar_init(wfull, LOAD_WARPS);
    for (int g = 0; g < 2; ++g) { mbar_init(gfull(g), 1); mbar_init(gempty(g), EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  allow_next_kernel();
  const uint32_t tmem_base = *tmem_slot;

  const int slice = (int)(blockIdx.x % (unsigned)ar.slices), range = (int)(blockIdx.x / (unsigned)ar.slices);
  const int c0 = slice * DC;
  const int64_t first = (int64_t)range * ar.per, last = min(ar.N, first + ar.per);      // first < last
  const int blocks = (int)((last - first + 127) >> 7);
  const int halves = (int)((last - first + 63) >> 6);                                   // stages of x
  const int kbs = (ar.n + 63) >> 6;                                                     // tiles of a block
  constexpr uint32_t W = 0, DL = S::DL_OFF, X = S::X_OFF;

  if (warp >= 2 + EPI_WARPS) {
    // ------------------------------------------------------------ x and W_r: from before the kernel that makes dl
    const int lw = warp - 2 - EPI_WARPS, half = lw & 1, k = lw >> 1, c = c0 + half * 64 + lane * 2;
    const uint32_t mask0 = c < ar.d ? ~0u : 0u, mask1 = c + 1 < ar.d ? ~0u : 0u;
    const int at = c < ar.d ? c : 0, next = c + 1 < ar.d ? 1 : 0;
    const int64_t d = ar.d;
    Rows<T, PAIR> rows;
    for (int kb = 0; kb < kbs; ++kb) {
      const int e = ar.e0 + kb * 64, left = ar.E - e;
      rows.fetch(ar.w + e * d + at, d, k, left, next);
      rows.put(gen + W + kb * S::P * TILE, k, left, half, mask0, mask1);
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(wfull);
    int s = 0, left = (int)(last - first);
    uint32_t ph = 0;
    const T* x = ar.x + first * d + at;
    rows.fetch(x, d, k, left, next);
#pragma unroll 1
    for (int h = 0; h < halves; ++h) {
      if (!mbar_wait(xempty(s), ph ^ 1u, abort_flag)) break;
      rows.put(gen + X + s * S::X_BYTES, k, left, half, mask0, mask1);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(xfull(s));
      if (++s == S::NST) { s = 0; ph ^= 1u; }
      left -= 64;
      if (left <= 0) break;
      x += 64 * d;
      rows.fetch(x, d, k, left, next);
    }
  } else if (warp == 0) {
    // ------------------------------------------------------------ dl by TMA
    if (elect_one()) {
      wait_for_previous_kernel();
      int r = 0;
      uint32_t rph = 0;
      bool ok = true;
      for (int b = 0; ok && b < blocks; ++b)
        for (int kb = 0; ok && kb < kbs; ++kb) {
          ok = mbar_wait(dempty(r), rph ^ 1u, abort_flag);
          if (!ok) break;
          mbar_expect_tx(dfull(r), (uint32_t)S::DL_BYTES);
#pragma unroll
          for (int q = 0; q < ROUTE_PARTS; ++q)
            tma_load_2d(tiles + DL + (uint32_t)(r * S::DL_BYTES + q * TILE), &mp.dl[q], ar.e0 + kb * 64, (int)first + b * 128, dfull(r));
          if (++r == S::RING) { r = 0; rph ^= 1u; }
        }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (elect_one()) {
      const uint32_t id_x = one_idesc(128, false, true);
      int s = 0, sl = 0, r = 0;
      uint32_t ph = 0, slp = 0, rph = 0;
      bool ok = mbar_wait(wfull, 0u, abort_flag);
      for (int b = 0; ok && b < blocks; ++b) {
        const int here = min(2, halves - 2 * b);                  // stages of x in this block
        const int in = b % S::GROUP, set = b / S::GROUP & 1;      // (without FLUSH one group)
        if (S::FLUSH && in == 0 && !mbar_wait(gempty(set), (uint32_t)(b / S::GROUP >> 1 & 1) ^ 1u, abort_flag)) { ok = false; break; }
        for (int kb = 0; ok && kb < kbs; ++kb) {
          const uint32_t dl = tiles + DL + (uint32_t)(r * S::DL_BYTES);
          const int steps = min(4, (ar.n - kb * 64 + 15) >> 4);   // of 16 experts
          if (!mbar_wait(dfull(r), rph, abort_flag)) { ok = false; break; }
          if (kb == 0 && !mbar_wait(sempty(sl), slp ^ 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + (uint32_t)(S::DW_COLS + sl * 128);
#pragma unroll
          for (int p = 0; p < Pairs<T>::n; ++p) {
            const uint64_t a = umma_desc(dl + (uint32_t)(Pairs<T>::l(p) * TILE));
            const uint64_t w = umma_desc_mn(tiles + W + (uint32_t)((kb * S::P + Pairs<T>::w(p)) * TILE));
            for (int ks = 0; ks < steps; ++ks) umma(acc, a + 2 * ks, w + 128 * ks, id_x, (kb | ks | p) != 0 ? 1u : 0u);
          }
          if (kb == kbs - 1) {
            umma_commit(sfull(sl));
            if (++sl == S::SLOTS) { sl = 0; slp ^= 1u; }
          }
          const uint32_t id_w = one_idesc(steps * 16, true, true);
          int xs = s;
          uint32_t xph = ph;
          for (int i = 0; ok && i < here; ++i) {                  // dW_r^T, 64 tokens at a time
            if (!mbar_wait(xfull(xs), xph, abort_flag)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int p = 0; p < Pairs<T>::n; ++p) {
              const uint64_t a = umma_desc_mn(tiles + X + (uint32_t)(xs * S::X_BYTES + Pairs<T>::w(p) * TILE));
              const uint64_t l = umma_desc_mn(dl + (uint32_t)(Pairs<T>::l(p) * TILE + i * BOX));
#pragma unroll
              for (int ks = 0; ks < 4; ++ks) {
                const bool large = S::FLUSH && p == Pairs<T>::n - 1;
                umma(tmem_base + (uint32_t)(S::FLUSH ? set * 128 + (large ? 64 : 0) : kb * 64), a + 128 * ks, l + 128 * ks, id_w,
                     (in | i | ks | (large ? 0 : p)) != 0 ? 1u : 0u);
              }
            }
            if (kb == kbs - 1) umma_commit(xempty(xs));
            if (++xs == S::NST) { xs = 0; xph ^= 1u; }
          }
          if (kb == kbs - 1) { s = xs; ph = xph; }
          if (ok) umma_commit(dempty(r));
          if (++r == S::RING) { r = 0; rph ^= 1u; }
        }
        if (ok && (in == S::GROUP - 1 || b == blocks - 1)) umma_commit(gfull(set));
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue: two warps per quarter of the lanes
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    uint32_t* stg = reinterpret_cast<uint32_t*>(gen + S::STG_OFF + (warp - 2) * S::STG_BYTES);
    int sl = 0;
    uint32_t slp = 0;
    bool ok = true;
    float sum[S::FLUSH ? 32 : 1];
#pragma unroll
    for (int i = 0; i < (S::FLUSH ? 32 : 1); ++i) sum[i] = 0.f;
    if (ar.e0) wait_for_previous_kernel();                        // it made the dx that this one adds to
    if (ar.out.dbias && slice == 0) {
      wait_for_previous_kernel();
      sum_bias(ar.out, ar.N, ar.E, tid - 64, EPI_WARPS * 32);
    }
    for (int b = 0; ok && b < blocks; ++b) {
      const int64_t row = first + (int64_t)b * 128 + quarter * 32;
      const int rows = (int)max((int64_t)0, min((int64_t)32, last - row));
      ok = mbar_wait(sfull(sl), slp, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + lanes + (uint32_t)(S::DW_COLS + sl * 128 + half * 64);
      const int col0 = c0 + half * 64, cols = min(64, ar.d - col0);
      T* out = ar.dx + row * ar.d + col0;
      auto drained = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sempty(sl));
      };
      if constexpr (!S::F32) __syncwarp();                        // the last block's columns have left the staging buffer
#pragma unroll 1
      for (int p = 0; p < 2; ++p) {                               // 32 columns at a time: `sum` holds registers
        uint32_t g[32];
        tmem_ld32(taddr + (uint32_t)(p * 32), g);
        tmem_ld_wait();
        if (p) drained();
        if constexpr (S::F32) {
          put_sums(g, stg, out + p * 32, ar.d, rows, cols - p * 32, ar.e0 != 0);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) stg[lane * 33 + p * 16 + i] = pack_bf16(__uint_as_float(g[2 * i]), __uint_as_float(g[2 * i + 1]));
        }
      }
      if constexpr (!S::F32) {
        __syncwarp();
        if (cols > 0) put_packed(stg, out, ar.d, rows, cols);
      }
      if (++sl == S::SLOTS) { sl = 0; slp ^= 1u; }
      if constexpr (S::FLUSH) {
        const int set = b / S::GROUP & 1;
        if (b % S::GROUP == S::GROUP - 1 || b == blocks - 1) {    // experts half * 32 on, of this lane's column
          ok = mbar_wait(gfull(set), (uint32_t)(b / S::GROUP >> 1 & 1), abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          uint32_t g[32];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            tmem_ld32(tmem_base + lanes + (uint32_t)((set * 2 + q) * 64 + half * 32), g);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[i] += __uint_as_float(g[i]);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(gempty(set));
        }
      }
    }
    const int64_t part = ((int64_t)range * ar.E + ar.e0) * ar.d;
    const int col = c0 + quarter * 32 + lane;
    if constexpr (S::FLUSH) {
      if (ok && col < ar.d)
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (half * 32 + i < ar.n) {
            const int64_t at = part + (int64_t)(half * 32 + i) * ar.d + col;
            if (ar.out.dw16) ar.out.dw16[at] = __float2bfloat16_rn(sum[i]);
            else ar.out.parts[at] = sum[i];
          }
    } else if (ok) {
      ok = mbar_wait(gfull(0), 0u, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {                                                   // lane: a column; 16 experts at a time, the halves in turn
        tc_fence_after();
#pragma unroll 1
        for (int e = half * 16; e < ar.n; e += 32) {
          uint32_t g[16];
          tmem_ld16(tmem_base + lanes + (uint32_t)e, g);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (e + i < ar.n && col < ar.d) {
              const int64_t at = part + (int64_t)(e + i) * ar.d + col;
              if (ar.out.dw16) ar.out.dw16[at] = __float2bfloat16_rn(__uint_as_float(g[i]));
              else ar.out.parts[at] = __uint_as_float(g[i]);
            }
        }
        tc_fence_before();
      }
    }
  }

  // ------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {                // a wait ran out: copies may still be on their way to this shared memory (10 ms)
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000LL) {}
    __syncthreads();
  }
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
  if (tid == 0 && *abort_flag && ar.dev_status) atomicExch(ar.dev_status, (int)CAPMOE_ETIMEOUT);
}

template <typename T, int KB>
int run(const void* split, const void* x, const void* w, int64_t N, int d, int E, int Eq, int ranges, void* dx, const RouteOut& out, int32_t* dev_status,
        cudaStream_t st) {
  using S = RA<T, KB>;
  RAMaps mp = {};
  for (int q = 0; q < ROUTE_PARTS; ++q)
    if (!make_part_map(&mp.dl[q], split, q, ROUTE_PARTS, (uint64_t)Eq, (uint64_t)N)) return note_cuda(cudaErrorInvalidValue);
  auto k = d % 2 == 0 ? k_route_grad_any<T, KB, true> : k_route_grad_any<T, KB, false>;
  const cudaError_t err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
  if (err != cudaSuccess) return note_cuda(err);
  RAArgs<T> ar = {};
  ar.x = (const T*)x; ar.w = (const T*)w; ar.N = N; ar.d = d; ar.E = E;
  ar.slices = (int)ceil_div(d, DC);
  ar.per = (int)(ceil_div(ceil_div(N, 64), ranges) * 64);
  ar.dx = (T*)dx; ar.out = out; ar.dev_status = dev_status;
  for (int e0 = 0; e0 < E; e0 += KB * 64) {
    ar.e0 = e0;
    ar.n = E - e0 < KB * 64 ? E - e0 : KB * 64;
    const int rc = note_cuda(launch_chained(k, (unsigned)(ar.slices * ranges), ANY_THREADS, S::SMEM, st, mp, ar));
    count_launch(1);
    if (rc != CAPMOE_OK) return rc;
    ar.out.dbias = nullptr;                    // the first pass makes it
  }
  return CAPMOE_OK;
}

}  // namespace

// The longest sum of bf16 tokens with more than 64 experts that one accumulator takes (64 groups of 16 tokens, three MMAs each:
// dW_r is off by 4 10^-6 of it, 2.8 10^-5 after 8192 tokens).
constexpr int64_t ROUTE_CHAIN = 1024;
int route_grad_any_ranges(int64_t N, int d, int E, int dtype) {
  return route_ranges(N, ceil_div(d, DC), dtype == CAPMOE_F32 || E <= 64 ? N : ROUTE_CHAIN);
}

int route_grad_any(const void* split, const void* x, const void* w, int64_t N, int d, int E, int Eq, int ranges, int dtype, void* dx,
                   const RouteOut& out, int32_t* dev_status, cudaStream_t st) {
  if (dtype == CAPMOE_F32) return run<float, 1>(split, x, w, N, d, E, Eq, ranges, dx, out, dev_status, st);
  auto of = E <= 64 ? run<__nv_bfloat16, 1> : E <= 128 ? run<__nv_bfloat16, 2> : run<__nv_bfloat16, 4>;
  return of(split, x, w, N, d, E, Eq, ranges, dx, out, dev_status, st);
}

}  // namespace capmoe
