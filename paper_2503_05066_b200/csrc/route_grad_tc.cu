// The two products of the router's gradient on tcgen05, in one pass over x:
//   dx[t] = sum_e dl[t,e] W_r[e],   dW_r[e] = sum_t dl[t,e] x[t]
// dl comes as three bf16 numbers per element whose sum it is (route_grad.cu), each multiplied on its own into the same fp32
// accumulators, the smallest first.
// A CTA owns DC columns of x, W_r and dx and a range of tokens, which it walks in blocks of 128.  W_r's columns stay in shared
// memory.  dl of a block comes in tiles of 64 experts (128 x 64, three parts, 48 KB): a tile is the A operand of dx = dl W_r
// (tokens are the M side, 128 columns the N side) and, read along the other axis from the same bytes, the B operand of
// dW_r^T = x^T dl (128 columns are the M side, experts the N side); x comes in stages of 64 tokens and stays for all tiles of its
// block.  The MMAs cut their sums off where fp32 ends, so dW_r^T stays in tensor memory for GROUP blocks only; the epilogue adds the
// groups up in registers, and the range's sum leaves as a part, fp32, that route_grad.cu adds up in order.  dx passes through two
// accumulators of 128 columns, so that its epilogue overlaps the MMAs.
// What bounds it: up to 64 experts HBM, x is read and dx written once; beyond, dl's way from L2, which every slice of columns reads
// again (256 experts, 2048 columns: 400 MB), and the MMAs.  16,384 tokens of 2048 columns, with the other two launches: 64 experts
// 41.5 us (37.6 without the MMAs), 128 experts 67 to 74 (54), 256 experts 125 (93).  dl as two numbers, which lose 2^-18 of it, and one
// accumulator for a range, which loses up to 2 10^-5 of dW_r: 41.8, 51, 93.
#include "gmm_tc.cuh"
#include "route_grad.cuh"

namespace capmoe {
namespace {

template <int KB, int DC_>                   // tiles of 64 experts, at most: 1, 2 or 4; columns of a CTA: 128, or with one tile also 256
struct RG {
  static constexpr int DC = DC_;
  static constexpr int BOX = 64 * 64 * 2;                      // 64 columns by 64 rows, bf16
  static constexpr int W_BYTES = KB * (DC / 64) * BOX;
  static constexpr int DL_PART = 2 * BOX, DL_BYTES = ROUTE_PARTS * DL_PART;      // a tile: 128 tokens by 64 experts
  static constexpr int RING = 2;                               // tiles of dl
  static constexpr int X_BYTES = (DC / 64) * BOX;
  static constexpr int NST = DC == 256 ? 2 : KB == 4 ? 3 : 4;  // stages of x
  static constexpr bool WIDE = KB < 4;                         // dx leaves in pieces of 64 columns, else 32 (half the staging)
  static constexpr int STG_BYTES = WIDE ? WIDE_BYTES : STG_WARP_BYTES;
  static constexpr int DL_OFF = W_BYTES, X_OFF = DL_OFF + RING * DL_BYTES, STG_OFF = X_OFF + NST * X_BYTES;
  static constexpr int TAIL = STG_OFF + EPI_WARPS * STG_BYTES;
  static constexpr int SMEM = TAIL + 1024 + 256;
  static constexpr int CHUNKS = DC / 128;
  static constexpr int SETS = KB < 4 ? 2 : 1, SET_COLS = CHUNKS * KB * 64;       // accumulators of dW_r^T, filled in turn
  static constexpr int GROUP = 2;                              // blocks that a set takes
  static constexpr int DW_COLS = SETS * SET_COLS;              // tensor-memory columns of them, then SLOTS x 128 for dx
  static constexpr int SLOTS = 2;
  static constexpr int SUMS = CHUNKS * KB * 2;                 // of 16 experts each, that a thread of the epilogue holds
  static_assert(SMEM <= 227 * 1024, "shared memory of a thread block");
  static_assert(DW_COLS + SLOTS * 128 <= 512, "tensor memory");
};

struct RGMaps { CUtensorMap dl[ROUTE_PARTS], x, w, o; };
struct RGArgs {
  int64_t N;
  int d, E, slices, per;                     // per: tokens of a range, a multiple of 64
  __nv_bfloat16* dx;
  RouteOut out;
  int32_t* dev_status;
};

template <int KB, int DC>
__global__ void __launch_bounds__(TC_THREADS, 1) k_route_grad(const __grid_constant__ RGMaps mp, const __grid_constant__ RGArgs ar) {
  using S = RG<KB, DC>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (tiles - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + S::TAIL);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 25);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto xfull = [&](int s) { return bar0 + 8u * (uint32_t)s; };                 // stages of x
  auto xempty = [&](int s) { return bar0 + 8u * (uint32_t)(4 + s); };
  auto dfull = [&](int r) { return bar0 + 8u * (uint32_t)(8 + r); };           // tiles of dl
  auto dempty = [&](int r) { return bar0 + 8u * (uint32_t)(11 + r); };
  auto sfull = [&](int s) { return bar0 + 8u * (uint32_t)(14 + s); };          // dx accumulators
  auto sempty = [&](int s) { return bar0 + 8u * (uint32_t)(17 + s); };
  const uint32_t wfull = bar0 + 8u * 20u;                                      // W_r has arrived
  auto gfull = [&](int g) { return bar0 + 8u * (uint32_t)(21 + g); };          // accumulators of dW_r^T
  auto gempty = [&](int g) { return bar0 + 8u * (uint32_t)(23 + g); };

  if (tid == 0) {
    for (int s = 0; s < S::NST; ++s) { mbar_init(xfull(s), 1); mbar_init(xempty(s), 1); }
    for (int r = 0; r < S::RING; ++r) { mbar_init(dfull(r), 1); mbar_init(dempty(r), 1); }
    for (int s = 0; s < S::SLOTS; ++s) { mbar_init(sfull(s), 1); mbar_init(sempty(s), EPI_WARPS); }
    mbar_init(wfull, 1);
    for (int g = 0; g < S::SETS; ++g) { mbar_init(gfull(g), 1); mbar_init(gempty(g), EPI_WARPS); }
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
  const int c0 = slice * S::DC;
  const int64_t first = (int64_t)range * ar.per, last = min(ar.N, first + ar.per);      // first < last
  const int blocks = (int)((last - first + 127) >> 7);
  const int halves = (int)((last - first + 63) >> 6);                                   // stages of x
  const int kbs = (ar.E + 63) >> 6;                                                     // tiles of a block
  constexpr uint32_t W = 0, DL = S::DL_OFF, X = S::X_OFF;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (elect_one()) {
      // W_r and x come from before the kernel that makes dl: they are fetched while it still runs
      mbar_expect_tx(wfull, (uint32_t)(kbs * (S::DC / 64) * S::BOX));
      for (int kb = 0; kb < kbs; ++kb)
#pragma unroll
        for (int i = 0; i < S::DC / 64; ++i)
          tma_load_2d(tiles + W + (uint32_t)((kb * (S::DC / 64) + i) * S::BOX), &mp.w, c0 + i * 64, kb * 64, wfull);
      int s = 0, h = 0;
      uint32_t ph = 0;
      bool ok = true;
      auto load_x = [&]() {                                      // stage h of x
        if (!mbar_wait(xempty(s), ph ^ 1u, abort_flag)) return false;
        mbar_expect_tx(xfull(s), (uint32_t)S::X_BYTES);
#pragma unroll
        for (int i = 0; i < S::DC / 64; ++i)
          tma_load_2d(tiles + X + (uint32_t)(s * S::X_BYTES + i * S::BOX), &mp.x, c0 + i * 64, (int)first + h * 64, xfull(s));
        ++h;
        if (++s == S::NST) { s = 0; ph ^= 1u; }
        return true;
      };
      const int ahead = min(halves, S::NST);
      while (ok && h < ahead) ok = load_x();
      wait_for_previous_kernel();
      int r = 0;
      uint32_t rph = 0;
      for (int b = 0; ok && b < blocks; ++b)
        for (int kb = 0; ok && kb < kbs; ++kb) {
          if (!mbar_wait(dempty(r), rph ^ 1u, abort_flag)) { ok = false; break; }
          mbar_expect_tx(dfull(r), (uint32_t)S::DL_BYTES);
          const uint32_t to = tiles + DL + (uint32_t)(r * S::DL_BYTES);
#pragma unroll
          for (int p = 0; p < ROUTE_PARTS; ++p)
            tma_load_2d(to + (uint32_t)(p * S::DL_PART), &mp.dl[p], kb * 64, (int)first + b * 128, dfull(r));
          if (++r == S::RING) { r = 0; rph ^= 1u; }
          while (ok && h < min(halves, 2 * b + 2)) ok = load_x();    // (the first tile's MMAs are the first to need them)
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
        const int in = b % S::GROUP, use = b / S::GROUP, set = use % S::SETS;
        for (int kb = 0; ok && kb < kbs; ++kb) {
          const uint32_t dl = tiles + DL + (uint32_t)(r * S::DL_BYTES);
          const int steps = min(4, (ar.E - kb * 64 + 15) >> 4);   // of 16 experts
          if (!mbar_wait(dfull(r), rph, abort_flag)) { ok = false; break; }
          for (int u = 0; ok && u < S::CHUNKS; ++u) {             // dx, 128 columns at a time (kbs == 1 where there are two)
            if (kb == 0 && !mbar_wait(sempty(sl), slp ^ 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t acc = tmem_base + (uint32_t)(S::DW_COLS + sl * 128);
            const uint64_t wd = umma_desc_mn(tiles + W + (uint32_t)((kb * (S::DC / 64) + u * 2) * S::BOX));
#pragma unroll
            for (int p = ROUTE_PARTS - 1; p >= 0; --p)
              for (int ks = 0; ks < steps; ++ks)
                umma(acc, umma_desc(dl + (uint32_t)(p * S::DL_PART)) + 2 * ks, wd + 128 * ks, id_x, (kb | ks) != 0 || p < ROUTE_PARTS - 1 ? 1u : 0u);
            if (kb == kbs - 1) {
              umma_commit(sfull(sl));
              if (++sl == S::SLOTS) { sl = 0; slp ^= 1u; }
            }
          }
          if (ok && kb == 0 && in == 0) ok = mbar_wait(gempty(set), (uint32_t)(use / S::SETS & 1) ^ 1u, abort_flag);
          const uint32_t id_w = one_idesc(steps * 16, true, true);
          int xs = s;
          uint32_t xph = ph;
          for (int i = 0; ok && i < here; ++i) {                  // dW_r^T, 64 tokens at a time
            if (!mbar_wait(xfull(xs), xph, abort_flag)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < S::CHUNKS; ++c) {
              const uint64_t xd = umma_desc_mn(tiles + X + (uint32_t)(xs * S::X_BYTES + c * 2 * S::BOX));
#pragma unroll
              for (int p = ROUTE_PARTS - 1; p >= 0; --p)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                  umma(tmem_base + (uint32_t)(set * S::SET_COLS + (c * KB + kb) * 64), xd + 128 * ks,
                       umma_desc_mn(dl + (uint32_t)(p * S::DL_PART + i * S::BOX)) + 128 * ks, id_w,
                       (in | i | ks) != 0 || p < ROUTE_PARTS - 1 ? 1u : 0u);
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
    uint8_t* stg = gen + S::STG_OFF + (warp - 2) * S::STG_BYTES;
    int sl = 0;
    uint32_t slp = 0;
    bool ok = true;
    float sum[S::SUMS][16];                                       // lane: a column of each chunk; 16 experts at a time, the halves in turn
#pragma unroll
    for (int j = 0; j < S::SUMS; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[j][i] = 0.f;
    auto expert = [&](int j) { return half * 16 + j % (KB * 2) * 32; };
    if (ar.out.dbias && slice == 0) {
      wait_for_previous_kernel();
      sum_bias(ar.out, ar.N, ar.E, tid - 64, EPI_WARPS * 32);
    }
    for (int b = 0; ok && b < blocks; ++b) {
      const int64_t row = first + (int64_t)b * 128 + quarter * 32;
      const bool full_rows = row + 32 <= last, row_ok = row + lane < last;
      for (int u = 0; u < S::CHUNKS; ++u) {
        ok = mbar_wait(sfull(sl), slp, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t taddr = tmem_base + lanes + (uint32_t)(S::DW_COLS + sl * 128 + half * 64);
        const int col = c0 + u * 128 + half * 64;
        __nv_bfloat16* out = ar.dx + (row + lane) * ar.d + col;
        auto drained = [&]() {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(sempty(sl));
        };
        if constexpr (S::WIDE) {
          uint32_t g[64], w[32];
          tmem_ld32(taddr, g);
          tmem_ld32(taddr + 32u, g + 32);
          tmem_ld_wait();
          drained();
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = pack_bf16(__uint_as_float(g[2 * i]), __uint_as_float(g[2 * i + 1]));
          if (col < ar.d) put_wide(w, full_rows, row_ok, stg, &mp.o, col, (int)row, out, (ar.d - col) * 2);
        } else {                                                  // 32 columns at a time: the sums hold registers
#pragma unroll 1
          for (int p = 0; p < 2; ++p) {
            uint32_t g[32], w[16];
            tmem_ld32(taddr + (uint32_t)(p * 32), g);
            tmem_ld_wait();
            if (p) drained();
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(g[2 * i]), __uint_as_float(g[2 * i + 1]));
            if (col + p * 32 < ar.d) store_piece(w, full_rows, row_ok, stg, &mp.o, col + p * 32, (int)row, out + p * 32, ar.d - col - p * 32);
          }
        }
        if (++sl == S::SLOTS) { sl = 0; slp ^= 1u; }
      }
      if (ok && (b % S::GROUP == S::GROUP - 1 || b == blocks - 1)) {
        const int use = b / S::GROUP, set = use % S::SETS;
        ok = mbar_wait(gfull(set), (uint32_t)(use / S::SETS & 1), abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < S::SUMS; ++j)
          if (expert(j) < ar.E) {
            uint32_t g[16];
            tmem_ld16(tmem_base + lanes + (uint32_t)(set * S::SET_COLS + j / (KB * 2) * KB * 64 + expert(j)), g);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[j][i] += __uint_as_float(g[i]);
          }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(gempty(set));
      }
    }
    if (ok) {
      const int64_t part = (int64_t)range * ar.E * ar.d;
#pragma unroll
      for (int j = 0; j < S::SUMS; ++j) {
        const int col = c0 + j / (KB * 2) * 128 + quarter * 32 + lane;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (expert(j) + i < ar.E && col < ar.d) {
            const int64_t at = part + (int64_t)(expert(j) + i) * ar.d + col;
            if (ar.out.dw16) ar.out.dw16[at] = __float2bfloat16_rn(sum[j][i]);
            else ar.out.parts[at] = sum[j][i];
          }
      }
    }
    if (lane == 0) bulk_wait_all();                               // this lane's stores have landed before the CTA ends
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

// Columns of a CTA: with up to 64 experts 256, unless 128 give as many CTAs, which then have twice as many stages of x (16,384 tokens,
// 64 experts, 2048 columns, 144 CTAs either way: 41.7 us, 45.8 with 256; 7168 columns: 112 CTAs 117 us, 140 of 256 columns 108).
int columns_of(int64_t N, int d, int E) {
  auto ctas = [&](int dc) { return ceil_div(d, dc) * route_ranges(N, ceil_div(d, dc), N); };
  return E > 64 || ctas(128) >= ctas(256) ? 128 : 256;
}

template <int KB, int DC>
int run(const RGMaps& mp, const RGArgs& ar, int ranges, cudaStream_t st) {
  using S = RG<KB, DC>;
  const cudaError_t err = cudaFuncSetAttribute(k_route_grad<KB, DC>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
  if (err != cudaSuccess) return note_cuda(err);
  const int rc = note_cuda(launch_chained(k_route_grad<KB, DC>, (unsigned)(ar.slices * ranges), TC_THREADS, S::SMEM, st, mp, ar));
  count_launch(1);
  return rc;
}

}  // namespace

int route_grad_tc_ranges(int64_t N, int d, int E) { return route_ranges(N, ceil_div(d, columns_of(N, d, E)), N); }

int route_grad_tc(const void* split, const void* x, const void* w, int64_t N, int d, int E, int Eq, int ranges, void* dx, const RouteOut& out,
                  int32_t* dev_status, cudaStream_t st) {
  RGMaps mp = {};
  for (int p = 0; p < ROUTE_PARTS; ++p)
    if (!make_part_map(&mp.dl[p], split, p, ROUTE_PARTS, (uint64_t)Eq, (uint64_t)N)) return note_cuda(cudaErrorInvalidValue);
  if (!make_map(&mp.x, x, (uint64_t)d, (uint64_t)N, 0, 64) || !make_map(&mp.w, w, (uint64_t)d, (uint64_t)E, 0, 64) ||
      !(E <= 128 ? make_wide_map(&mp.o, dx, (uint64_t)d, (uint64_t)N, 2) : make_store_map(&mp.o, dx, (uint64_t)d, (uint64_t)N)))
    return note_cuda(cudaErrorInvalidValue);
  RGArgs ar = {};
  ar.N = N; ar.d = d; ar.E = E;
  const int dc = columns_of(N, d, E);
  ar.slices = (int)ceil_div(d, dc);
  ar.per = (int)(ceil_div(ceil_div(N, 64), ranges) * 64);
  ar.dx = (__nv_bfloat16*)dx; ar.out = out; ar.dev_status = dev_status;
  auto of = dc == 256 ? run<1, 256> : E <= 64 ? run<1, 128> : E <= 128 ? run<2, 128> : run<4, 128>;
  return of(mp, ar, ranges, st);
}

}  // namespace capmoe
