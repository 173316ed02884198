// Gate and up products of the 8-bit FFN on tcgen05's block-scaled MMA (kind::mxf8f6f4): e4m3 codes, power-of-two scales
// per 128 columns of a row and per 128 x 128 block of a weight, applied by the tensor cores, fp32 accumulation.
//   h[r] = silu(W_g[e] x[r]) * (W_u[e] x[r]), quantised: codes and scales
// Persistent kernel over CTA pairs, tiles of 256 tokens by 128 hidden columns, the structure of k_gmm_dw (gmm_dw.cu) with
// one more warp that stages scale words (see gmm_tc.cuh).  A tile puts 128 gate and 128 up columns of the same hidden
// columns side by side, which is one block of 128 hidden columns per row: its largest magnitude meets between the two
// threads that share a row, and the hidden row leaves the kernel as codes, never as fp32.
// Tensor memory: two accumulators of 256 columns and four groups of scales do not fit 512 columns, so the
// accumulators overlap by 64 columns ([0,256) and [192,448)).  The next tile's MMAs wait for the warps that read those 64
// columns, which, like the others, hold a tile's hidden values in registers before they let go of any of its columns; they
// do not wait for the other half of the warps, nor for anyone's quantising and storing.  (With the tokens on the N side, as
// in gmm_rows.cu, gate and up would fill the 448 columns at 224 tokens, and an epilogue could not overlap the next tile.)
// silu: __expf and __fdividef, as in gmm_rows.cu.
// What bounds it: the tensor pipe; the scale copies take about 10 % of it.
#include "gmm.cuh"
#include "gmm_tc.cuh"

namespace capmoe {
namespace {

// Allocated rows per expert on average below which gmm_rows.cu takes over (60 experts, 2048 x 1408, whole FFN: 144 us
// against 155 at 136 rows, 205 against 207 at 273, 387 against 342 at 546).
constexpr int64_t SHORT_LIMIT = 300;

constexpr int NST8 = 6;
constexpr int STAGE8 = 2 * A_BYTES;                       // 128 rows of A, 128 rows of B: 32 KB
constexpr int STG8_OFF = NST8 * STAGE8;
constexpr int SF_OFF = STG8_OFF + EPI_WARPS * STG_WARP_BYTES;
constexpr int SF_GROUP = 3 * SF_CHUNK;                    // A rows, B rows 0..127, B rows 128..255
constexpr int SF_SLOT = SF_GROUPS * SF_GROUP;
constexpr int TAIL8 = SF_OFF + SF_RING * SF_SLOT;
constexpr int SMEM8 = TAIL8 + 1024 + 512 + 3 * (GMM_MAX_E + 1) * 4 + 16 + 2 * 2 * 128 * 4 + TR_BYTES;
static_assert(SMEM8 <= 227 * 1024, "shared memory of a thread block");
constexpr int ACC_STEP = 192;                             // columns between the two accumulators

struct F8Args {
  Segments sg;
  int K, Nout;
  const uint8_t *xs, *s0, *s1;      // scales of the rows, of W_g and of W_u
  uint8_t *out, *out_scale;         // codes and scales of h
  int64_t xs_ld, os_ld;             // bytes between rows of xs and of out_scale
  int32_t* dev_status;
  int32_t* sched;
};
struct F8Maps { CUtensorMap a, b0, b1, o; };

__global__ void __launch_bounds__(F8_THREADS, 1) k_gmm_swiglu8(const __grid_constant__ F8Maps mp, const __grid_constant__ F8Args ar) {
  constexpr int N_TILE = 128, BM2 = 2 * BM;
  allow_next_kernel();
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (tiles - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + TAIL8);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 52);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* offs = reinterpret_cast<int*>(gen + TAIL8 + 512);
  int* ends = offs + (GMM_MAX_E + 1);
  int* tile_start = ends + (GMM_MAX_E + 1);
  uint32_t* row_max = reinterpret_cast<uint32_t*>(tile_start + (GMM_MAX_E + 1) + 1);   // (16-byte aligned) [2 tiles][2 halves][128 rows]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank();
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };                 // 0..5
  auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(8 + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (uint32_t)(16 + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (uint32_t)(18 + b); };
  auto shared_bar = [&](int b) { return bar0 + 8u * (uint32_t)(20 + b); };        // the overlap columns have been read
  auto sfull_bar = [&](int r) { return bar0 + 8u * (uint32_t)(24 + r); };
  auto sempty_bar = [&](int r) { return bar0 + 8u * (uint32_t)(26 + r); };
  auto gfree_bar = [&](int g) { return bar0 + 8u * (uint32_t)(28 + g); };
  const TileRing ring{bar0 + 8u * RING_BAR, smem_u32(row_max + 512), rank, abort_flag};

  if (tid == 0) {
    for (int s = 0; s < NST8; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), 2 * EPI_WARPS * 32);
      mbar_init(shared_bar(b), EPI_WARPS * 32);                 // one half of the warps of each CTA
    }
    for (int r = 0; r < SF_RING; ++r) { mbar_init(sfull_bar(r), 2); mbar_init(sempty_bar(r), 1); }
    for (int g = 0; g < SF_GROUPS; ++g) mbar_init(gfree_bar(g), 1);
    ring.init(2 + (rank == 0 ? 1 : 0) + EPI_WARPS);             // TMA thread, scales, MMA thread, epilogue warps
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  wait_for_previous_kernel();
  const int E = ar.sg.E;
  for (int i = tid; i < E; i += F8_THREADS) { offs[i] = seg_at(ar.sg, i); ends[i] = max(offs[i], seg_at(ar.sg, i + 1)); }
  __syncthreads();
  if (warp == 0) {
    const int n_blocks = (ar.Nout + N_TILE - 1) / N_TILE;
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int e = e0 + lane;
      const int mine = e < E ? ((ends[e] - offs[e] + BM2 - 1) / BM2) * n_blocks : 0;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
      if (e < E) tile_start[e] = carry + upto - mine;
      carry += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) tile_start[E] = carry;
  }
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int tile_hi = tile_start[E];
  auto get_tile = [&](int j, bool whole_warp, Tile& t) -> bool {
    int4 a, b;
    if (!ring.get(j, whole_warp, a, b)) return false;
    t.e = a.x; t.row0 = a.y; t.rows = a.z; t.n0 = a.w;
    return true;
  };
  const int num_kb = (ar.K + QBLOCK - 1) / QBLOCK;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (both CTAs)
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 0;
      Tile t;
      bool ok = true;
      for (int j = 0; ok; ++j) {
        if (!get_tile(j, false, t)) break;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t bar = full_bar(s) & PEER_MASK;
          if (rank == 0) mbar_expect_tx(full_bar(s), 2 * STAGE8);
          const uint32_t a_dst = tiles + (uint32_t)s * STAGE8;
          tma2_load_2d(a_dst, &mp.a, kb * QBLOCK, t.row0 + (int)rank * BM, bar);
          tma2_load_3d(a_dst + A_BYTES, rank == 0 ? &mp.b0 : &mp.b1, kb * QBLOCK, t.n0, t.e, bar);
          if (++s == NST8) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (leader CTA only)
    if (rank == 0 && elect_one()) {
      int s = 0, r = 0, g = 0;
      uint32_t it = 0, ph = 0, rph = 0, gph = 0;
      const uint32_t idesc0 = f8_idesc(256);
      const uint64_t a0 = umma_desc(tiles), b0 = umma_desc(tiles + A_BYTES);
      uint64_t off = 0;
      Tile t;
      bool ok = true;
      for (int j = 0; ok; ++j, ++it) {
        if (!get_tile(j, false, t)) break;
        const uint32_t b = it & 1u, use = it >> 1;
        // this accumulator has been converted, and the one before it has been read where the two overlap
        if (!mbar_wait(tempty_bar(b), (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        if (it > 0 && !mbar_wait(shared_bar(b ^ 1u), ((it - 1) >> 1) & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem_base + b * (uint32_t)ACC_STEP;
        uint32_t sf = 0;
        for (int kb = 0; kb < num_kb; ++kb) {
          if ((kb & 15) == 0 && !mbar_wait_cluster(sfull_bar(r), rph, abort_flag)) { ok = false; break; }
          if ((kb & 3) == 0) {
            if (!mbar_wait(gfree_bar(g), gph ^ 1u, abort_flag)) { ok = false; break; }   // its last MMAs are done
            tc_fence_after();
            sf = tmem_base + (uint32_t)(SF_TMEM + g * SF_COLS);
            const uint32_t src = tiles + SF_OFF + (uint32_t)(r * SF_SLOT + ((kb >> 2) & 3) * SF_GROUP);
            copy_scales(sf + 8u, src);                          // A rows
            copy_scales(sf, src + SF_CHUNK);                    // B rows 0..127
            copy_scales(sf + 4u, src + 2 * SF_CHUNK);           // B rows 128..255
          }
          if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t idesc = idesc0 | f8_scale_byte(kb);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma2_f8(d, a0 + off + 2 * k, b0 + off + 2 * k, idesc, sf + 8u, sf, (kb | k) != 0 ? 1u : 0u);
          umma2_commit_both(empty_bar(s));
          const bool last = kb == num_kb - 1;
          if ((kb & 3) == 3 || last) {
            umma2_commit_own(gfree_bar(g));
            if (++g == SF_GROUPS) { g = 0; gph ^= 1u; }
          }
          if ((kb & 15) == 15 || last) {
            umma2_commit_both(sempty_bar(r));
            if (++r == SF_RING) { r = 0; rph ^= 1u; }
          }
          off += (uint64_t)(STAGE8 >> 4);
          if (++s == NST8) { s = 0; ph ^= 1u; off = 0; }
        }
        if (ok) umma2_commit_both(tfull_bar(b));
      }
    }
  } else if (warp == 2 + EPI_WARPS) {
    // ------------------------------------------------------------ scales (both CTAs)
    int r = 0;
    uint32_t rph = 0;
    Tile t;
    bool ok = true;
    const int nb = num_kb, wb = (ar.Nout + QBLOCK - 1) / QBLOCK;
    const bool xa = scales_aligned(ar.xs_ld, ar.xs), ga = scales_aligned(nb, ar.s0), ua = scales_aligned(nb, ar.s1);
    for (int j = 0; ok; ++j) {
      if (!get_tile(j, true, t)) break;
      const uint8_t* rows[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = min(t.row0 + (int)rank * BM + lane + 32 * i, ar.sg.rows - 1);   // rows past the tile: any scale
        rows[i] = ar.xs + (int64_t)row * ar.xs_ld;
      }
      const int blk = t.n0 / QBLOCK;
      const uint8_t* w0 = ar.s0 + ((int64_t)t.e * wb + blk) * nb;
      const uint8_t* w1 = ar.s1 + ((int64_t)t.e * wb + blk) * nb;
      for (int k = 0; ok && k < nb; k += 16) {
        uint4 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = scale_words(rows[i], k, nb, xa);
        const uint4 b = scale_words(w0, k, nb, ga), c = scale_words(w1, k, nb, ua);
        bool free_slot = mbar_wait(sempty_bar(r), rph ^ 1u, abort_flag);
        free_slot = __all_sync(0xffffffffu, free_slot);
        if (!free_slot) { ok = false; break; }
#pragma unroll
        for (int g = 0; g < SF_GROUPS; ++g) {
          const uint32_t dst = tiles + SF_OFF + (uint32_t)(r * SF_SLOT + g * SF_GROUP);
          const uint32_t bw = word_of(b, g), cw = word_of(c, g);
          put_words(dst, lane, word_of(a[0], g), word_of(a[1], g), word_of(a[2], g), word_of(a[3], g));
          put_words(dst + SF_CHUNK, lane, bw, bw, bw, bw);
          put_words(dst + 2 * SF_CHUNK, lane, cw, cw, cw, cw);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive_release_cluster(sfull_bar(r) & PEER_MASK);
        if (++r == SF_RING) { r = 0; rph ^= 1u; }
      }
    }
  } else if (warp == 3 + EPI_WARPS) {
    // ------------------------------------------------------------ scheduler (both CTAs)
    if (elect_one()) {
      int cursor = 0;
      ring.run(pair, npairs, tile_hi, ar.sched, [&](int tile, int4& a, int4&) {
        Tile q;
        locate_tile(tile, cursor, tile_start, offs, ends, E, N_TILE, BM2, q);
        a = make_int4(q.e, q.row0, q.rows, q.n0);
      });
    }
  } else {
    // ------------------------------------------------------------ epilogue (both CTAs, own 128 rows)
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint32_t it = 0;
    Tile t;
    uint8_t* stg = gen + STG8_OFF + (warp - 2) * STG_WARP_BYTES;
    for (int j = 0;; ++j, ++it) {
      if (!get_tile(j, true, t)) break;
      const uint32_t b = it & 1u, use = it >> 1;
      bool ready = mbar_wait(tfull_bar(b), use & 1u, abort_flag);
      ready = __all_sync(0xffffffffu, ready);
      ready = group_all(1 + quarter, 64, ready);   // the two threads of a row stop together
      if (!ready) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + b * (uint32_t)ACC_STEP;
      const int warp_row0 = (int)rank * BM + quarter * 32;
      const bool full_rows = warp_row0 + 32 <= t.rows, row_ok = warp_row0 + lane < t.rows;
      const int row = t.row0 + warp_row0;
      // the overlap is the last 64 columns of accumulator 0 and the first 64 of accumulator 1
      const bool mine_shared = half == (b == 0 ? 1 : 0);
      // hidden columns half * 64 .. + 63 of the tile: gate there, up 128 columns further on
      float h[64];
      uint32_t top = 0;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        uint32_t g[32], u[32];
        tmem_ld32(taddr + (uint32_t)(half * 64 + 32 * v), g);
        tmem_ld32(taddr + (uint32_t)(128 + half * 64 + 32 * v), u);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float gv = __uint_as_float(g[i]);
          h[32 * v + i] = __fdividef(gv, 1.0f + __expf(-gv)) * __uint_as_float(u[i]);
          top = max(top, __float_as_uint(h[32 * v + i]) & 0x7fffffffu);
        }
      }
      tc_fence_before();
      if (mine_shared) mbar_arrive_cluster(shared_bar(b) & PEER_MASK);
      mbar_arrive_cluster(tempty_bar(b) & PEER_MASK);
      uint32_t* rm = row_max + b * 256 + quarter * 32 + lane;
      rm[half * 128] = top;
      group_sync(1 + quarter, 64);
      top = max(top, rm[(half ^ 1) * 128]);
      const uint32_t code = scale_code(top);
      uint32_t packed[16];
      if (code == (uint32_t)Q_NAN_SCALE) {
#pragma unroll
        for (int i = 0; i < 16; ++i) packed[i] = 0x7f7f7f7fu;
      } else {
        const float f = inv_scale(code);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          packed[i] = to_e4m3x2(h[4 * i] * f, h[4 * i + 1] * f) | (to_e4m3x2(h[4 * i + 2] * f, h[4 * i + 3] * f) << 16);
      }
      const int c = t.n0 + half * 64;
      if (half == 0 && row_ok)
        ar.out_scale[(int64_t)(row + lane) * ar.os_ld + t.n0 / QBLOCK] = (uint8_t)code;
      if (c < ar.Nout)                                        // 64 codes are the 64 bytes of a piece's row
        store_piece(packed, full_rows, row_ok, stg, &mp.o, c, row,
                    reinterpret_cast<__nv_bfloat16*>(ar.out + (int64_t)(row + lane) * ar.Nout + c),
                    (ar.Nout - c) / 2);
    }
    if (lane == 0) bulk_wait_all();
  }

  // ------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
  if (tid == 0 && *abort_flag && ar.dev_status) atomicExch(ar.dev_status, (int)CAPMOE_ETIMEOUT);
}

int launch(const F8Maps& mp, const F8Args& ar, cudaStream_t st) {
  const int pairs = sm_count() / 2;
  if (pairs < 1) return CAPMOE_EUNSUPPORTED;
  cudaError_t err = cudaFuncSetAttribute(k_gmm_swiglu8, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM8);
  if (err != cudaSuccess) return note_cuda(err);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(F8_THREADS);
  cfg.dynamicSmemBytes = SMEM8;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  err = cudaLaunchKernelEx(&cfg, k_gmm_swiglu8, mp, ar);
  count_launch(1);
  return note_cuda(err);
}

}  // namespace

bool gmm8_swiglu_waits_first(const Segments& sg) { return use_short(sg, SHORT_LIMIT); }

int gmm8_swiglu(const uint8_t* xq, const uint8_t* xs, int64_t xs_ld, const Segments& sg, const uint8_t* wg, const uint8_t* wgs,
                   const uint8_t* wu, const uint8_t* wus, int d, int F, uint8_t* hq, uint8_t* hs, int64_t hs_ld, int32_t* dev_status,
                   int32_t* sched, bool early, cudaStream_t st) {
  if (use_short(sg, SHORT_LIMIT))
    return gmm8_swiglu_short(xq, xs, xs_ld, sg, wg, wgs, wu, wus, d, F, hq, hs, hs_ld, dev_status, sched, early, st);
  F8Maps mp = {};
  F8Args ar = {};
  if (!make_map_u8(&mp.a, xq, d, sg.rows, 0, BM) || !make_map_u8(&mp.b0, wg, d, F, sg.E, 128) ||
      !make_map_u8(&mp.b1, wu, d, F, sg.E, 128) || !make_store_map_u8(&mp.o, hq, F, sg.rows))
    return note_cuda(cudaErrorInvalidValue);
  ar.sg = sg; ar.K = d; ar.Nout = F; ar.xs = xs; ar.xs_ld = xs_ld; ar.s0 = wgs; ar.s1 = wus; ar.out = hq;
  ar.out_scale = hs; ar.os_ld = hs_ld;
  ar.dev_status = dev_status; ar.sched = sched;
  return launch(mp, ar, st);
}

}  // namespace capmoe
