// Grouped products over expert rows on tcgen05, in bf16 and in 8 bits (kind::mxf8f6f4, see gmm_tc.cuh): persistent,
// warp-specialised kernels over CTA pairs (cta_group::2), TMA-fed operand rings, fp32 accumulators in tensor memory.  The
// WEIGHTS are the M side (256 weight rows per pair, 128 per CTA), the tokens the N side, which the MMA takes in steps of
// 16, so an expert with a few rows pays for 16 of them and one with a few hundred for at most 15 more than it has; a
// segment longer than a tile is cut into equal token blocks.  (With the tokens on the M side, 256 to a tile, the same
// products were 2 % faster at best, at 2000 rows per expert and more, and up to half as fast below 300.)
//   T_FWD   y^T  = W[e] x^T             T_DX  dx^T = W[e]^T dy^T         T_DX2  dx^T = W_g[e]^T dg^T + W_u[e]^T du^T
//   T_HID   dg, du, h of the SwiGLU FFN's backward pass: g, u and dh of a tile side by side in tensor memory, the
//           elementwise part in the epilogue, so that g, u and dh are never rounded or written; dg, du and h are rounded
//           to bf16, because the MMAs that read them multiply bf16: a quarter of the FFN gradients' error (0.23 % of their
//           norm, 0.17 % with those three exact), and half the bytes of fp32 copies
//   T_F8    8-bit T_FWD                 T_F8SW  8-bit gate/up with SwiGLU, hidden rows quantised
// Weights whose output index is contiguous (W^T) are MN-major operands, loaded as they lie (make_mn_map).
// One token's row of an output is one column of an accumulator.  The epilogue reads 8 x 8 fragments, which stmatrix
// writes transposed to shared memory, so that whole 64-byte runs of a token's row leave the warp.  (Two-byte stores
// straight from the accumulator's columns took 15,000 cycles for a 128-token tile of T_HID, half as long as its MMAs.)
// silu is computed with __expf and __fdividef: a few units of 2^-23 while |g| is below 10, about 100 at -87, and 0 for g
// below -87 (the exact value is under 2^-118 there); the result is then rounded to 8 bits of mantissa or fewer.
// In T_F8SW a CTA's 128 weight rows are exactly one block of 128 hidden columns, whose maximum is taken per token over
// the lanes (shuffles) and the four warps (shared memory).
// A stage holds the weights of one k-block and `tb` token rows per CTA; `tb` follows the average segment so that short
// segments leave the ring to the weights, which is what a decode step has to stream.  What bounds it: HBM for few rows
// per expert (a decode step's 332 MB of bf16 weights: 55 us, 0.92 of the copy bandwidth), else the tensor pipe and the L2
// traffic of the weights, once per token block.
// Tensor memory: accumulators of `tt` columns, two sets of them when they fit, so that an epilogue overlaps the next
// tile's MMAs.
#include "gmm.cuh"
#include "gmm_tc.cuh"

namespace capmoe {
namespace {

enum Kind { T_FWD = 0, T_DX, T_DX2, T_HID, T_F8, T_F8SW };

template <int KIND>
struct ShapeT {
  static constexpr bool FP8 = KIND == T_F8 || KIND == T_F8SW;
  static constexpr int NACC = KIND == T_HID ? 3 : KIND == T_F8SW ? 2 : 1;     // accumulators = weight tiles per stage
  static constexpr int NX = KIND == T_HID ? 2 : 1;                             // token tiles per stage
  static constexpr int KE = FP8 ? 128 : 64;                                    // reduction steps per k-block: 128 bytes
  static constexpr int EW = 8;                                                 // epilogue warps
  static constexpr int THREADS = 64 + EW * 32 + 32 + (FP8 ? 32 : 0);           // roles, scheduler, scales
  static constexpr int READERS = 1 + EW + (FP8 ? 1 : 0);                       // of the tile ring, and the leader's MMA thread
  static constexpr int COLS = FP8 ? SF_TMEM : 512;                             // tensor-memory columns for accumulators
  static constexpr int SF_GROUP = 4 * SF_CHUNK;                                // tokens 0..127, 128..255, weights, second weights
  static constexpr int SF_SLOT = SF_GROUPS * SF_GROUP;
  static constexpr int RING = (FP8 ? 186 : 204) * 1024;
  static constexpr int STG_OFF = RING;                                         // 2 KB per epilogue warp
  static constexpr int SF_OFF = RING + EW * STG_WARP_BYTES;
  static constexpr int TAIL = SF_OFF + (FP8 ? SF_RING * SF_SLOT : 0);
  static constexpr int RED = KIND == T_F8SW ? 2 * 2 * 4 * 32 * 4 : 0;
  static constexpr int SMEM = TAIL + 1024 + 512 + 3 * (GMM_MAX_E + 1) * 4 + 16 + RED + TR_BYTES;
  static_assert(SMEM <= 227 * 1024, "shared memory of a thread block");
};
constexpr int MAX_NST = 12;

struct TMaps { CUtensorMap x0, x1, w0, w1, w2; };
struct TArgs {
  Segments sg;
  int K, Nout;
  int early;                        // offsets and weights are final before the previous kernel ends (gmm.cuh)
  int wide;                         // MN-major weights: one box per k-block
  int tb, tt, bufs, nst;            // token rows per CTA and stage, tokens per tile, accumulator sets, stages
  void* out[3];
  const uint8_t *xs, *s0, *s1;      // 8-bit: scales of the rows, of W (W_g) and of W_u
  uint8_t* out_scale;
  int64_t xs_ld, os_ld;             // bytes between rows of xs and of out_scale
  int32_t* dev_status;
  int32_t* sched;
};

struct STile { int e, row0, rows, nt, w0; };   // segment, first token row, tokens, MMA N, first weight row

template <int KIND>
__global__ void __launch_bounds__(ShapeT<KIND>::THREADS, 1)
k_gmm_rows(const __grid_constant__ TMaps mp, const __grid_constant__ TArgs ar) {
  using S = ShapeT<KIND>;
  constexpr bool FP8 = S::FP8, W_MN = KIND == T_DX || KIND == T_DX2;
  constexpr int EW = S::EW, NACC = S::NACC;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (tiles - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + S::TAIL);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 52);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* offs = reinterpret_cast<int*>(gen + S::TAIL + 512);
  int* ends = offs + (GMM_MAX_E + 1);
  int* tile_start = ends + (GMM_MAX_E + 1);
  uint32_t* red = reinterpret_cast<uint32_t*>(tile_start + (GMM_MAX_E + 1) + 1);       // (16-byte aligned) T_F8SW: [2][2 warp groups][4][32]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank();
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };                 // MAX_NST each
  auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(MAX_NST + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (uint32_t)(24 + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (uint32_t)(26 + b); };
  auto sfull_bar = [&](int r) { return bar0 + 8u * (uint32_t)(28 + r); };
  auto sempty_bar = [&](int r) { return bar0 + 8u * (uint32_t)(30 + r); };
  auto gfree_bar = [&](int g) { return bar0 + 8u * (uint32_t)(32 + g); };
  const TileRing ring{bar0 + 8u * RING_BAR, smem_u32(red) + S::RED, rank, abort_flag};
  const int nst = ar.nst, tt = ar.tt, bufs = ar.bufs;
  const uint32_t x_bytes = (uint32_t)ar.tb * 128u;
  const uint32_t stage = (uint32_t)(NACC * A_BYTES) + (uint32_t)S::NX * x_bytes;

  if (tid == 0) {
    for (int s = 0; s < nst; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * EW * 32); }
    for (int r = 0; r < SF_RING; ++r) { mbar_init(sfull_bar(r), 2); mbar_init(sempty_bar(r), 1); }
    for (int g = 0; g < SF_GROUPS; ++g) mbar_init(gfree_bar(g), 1);
    ring.init(S::READERS + (rank == 0 ? 1 : 0));
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (!ar.early) wait_for_previous_kernel();
  allow_next_kernel();
  const int E = ar.sg.E;
  for (int i = tid; i < E; i += S::THREADS) { offs[i] = seg_at(ar.sg, i); ends[i] = max(offs[i], seg_at(ar.sg, i + 1)); }
  __syncthreads();
  const int w_blocks = (ar.Nout + 255) >> 8;
  if (warp == 0) {
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int e = e0 + lane;
      const int mine = e < E ? (ends[e] - offs[e] + tt - 1) / tt * w_blocks : 0;
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
  auto get_tile = [&](int j, bool whole_warp, STile& t) -> bool {
    int4 a, b;
    if (!ring.get(j, whole_warp, a, b)) return false;
    t.e = a.x; t.row0 = a.y; t.rows = a.z; t.nt = a.w; t.w0 = b.x;
    return true;
  };
  const int kbs = (ar.K + S::KE - 1) / S::KE;
  const int num_kb = kbs * (KIND == T_DX2 ? 2 : 1);

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (both CTAs)
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 0;
      STile t;
      bool ok = true;
      // In an early start the first ring's weights are fetched while the previous kernel, which makes the token rows, still
      // runs; their token rows follow when it has ended.
      int fetched = 0;
      bool waited = !ar.early;
      auto load_weights = [&](int kb, int w, int e, uint32_t w_dst, uint32_t bar) {
        if (rank == 0) mbar_expect_tx(bar, 2u * stage);           // (the leader's own address)
        if constexpr (KIND == T_FWD || KIND == T_F8) {
          tma2_load_3d(w_dst, &mp.w0, kb * S::KE, w, e, bar);
        } else if constexpr (KIND == T_F8SW || KIND == T_HID) {
          tma2_load_3d(w_dst, &mp.w0, kb * S::KE, w, e, bar);
          tma2_load_3d(w_dst + A_BYTES, &mp.w1, kb * S::KE, w, e, bar);
          if (KIND == T_HID) load_mn(w_dst + 2 * A_BYTES, &mp.w2, ar.wide, w, kb * S::KE, e, bar);
        } else {
          const bool second = KIND == T_DX2 && kb >= kbs;
          load_mn(w_dst, second ? &mp.w1 : &mp.w0, ar.wide, w, (second ? kb - kbs : kb) * S::KE, e, bar);
        }
      };
      auto load_tokens = [&](int kb, int x, uint32_t x_dst, uint32_t bar) {
        const bool second = KIND == T_DX2 && kb >= kbs;
        tma2_load_2d(x_dst, second ? &mp.x1 : &mp.x0, (second ? kb - kbs : kb) * S::KE, x, bar);
        if (KIND == T_HID) tma2_load_2d(x_dst + x_bytes, &mp.x1, kb * S::KE, x, bar);
      };
      for (int j = 0; ok; ++j) {
        if (!get_tile(j, false, t)) break;
        const int w = t.w0 + (int)rank * BM;                     // this CTA's 128 weight rows
        const int x = t.row0 + (int)rank * (t.nt >> 1);          // and its half of the tokens
        if (!waited) {                                           // first tile of an early start
          fetched = min(nst, num_kb);
          for (int kb = 0; kb < fetched; ++kb) load_weights(kb, w, t.e, tiles + (uint32_t)kb * stage, full_bar(kb) & PEER_MASK);
          wait_for_previous_kernel();
          waited = true;
        }
        for (int kb = 0; kb < num_kb; ++kb) {
          const uint32_t bar = full_bar(s) & PEER_MASK;
          const uint32_t w_dst = tiles + (uint32_t)s * stage;
          if (fetched > 0) {
            --fetched;
          } else {
            if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag)) { ok = false; break; }
            load_weights(kb, w, t.e, w_dst, bar);
          }
          load_tokens(kb, x, w_dst + (uint32_t)(NACC * A_BYTES), bar);
          if (++s == nst) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (leader CTA only)
    if (rank == 0 && elect_one()) {
      int s = 0, r = 0, b = 0, g = 0;
      uint32_t ph = 0, rph = 0, bph = 0, gph = 0;
      const uint64_t w0 = W_MN ? umma_desc_mn(tiles) : umma_desc(tiles);
      const uint64_t x0 = umma_desc(tiles + (uint32_t)(NACC * A_BYTES));
      const uint64_t w2 = umma_desc_mn(tiles + 2 * A_BYTES);
      const uint64_t x_step = (uint64_t)(x_bytes >> 4), stage_step = (uint64_t)(stage >> 4);
      uint64_t off = 0;
      STile t;
      bool ok = true;
      for (int j = 0; ok; ++j) {
        if (!get_tile(j, false, t)) break;
        const uint32_t idesc = FP8 ? f8_idesc(t.nt) : pair_idesc(t.nt, W_MN, false), idesc2 = pair_idesc(t.nt, true, false);
        if (!mbar_wait(tempty_bar(b), bph ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)(b * NACC * tt);
        uint32_t sf = 0;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (FP8 && (kb & 15) == 0 && !mbar_wait_cluster(sfull_bar(r), rph, abort_flag)) { ok = false; break; }
          if (FP8 && (kb & 3) == 0) {
            if (!mbar_wait(gfree_bar(g), gph ^ 1u, abort_flag)) { ok = false; break; }   // its last MMAs are done
            tc_fence_after();
            sf = tmem_base + (uint32_t)(SF_TMEM + g * SF_COLS);
            const uint32_t src = tiles + (uint32_t)(S::SF_OFF + r * S::SF_SLOT + ((kb >> 2) & 3) * S::SF_GROUP);
            copy_scales(sf, src);
            if (t.nt > 128) copy_scales(sf + 4u, src + SF_CHUNK);
            copy_scales(sf + 8u, src + 2 * SF_CHUNK);
            if (KIND == T_F8SW) copy_scales(sf + 12u, src + 3 * SF_CHUNK);
          }
          if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t acc = (kb | k) != 0 ? 1u : 0u;
            const uint64_t xd = x0 + off + 2 * k;
            if constexpr (FP8) {
              const uint32_t id = idesc | f8_scale_byte(kb);
              umma2_f8(d, w0 + off + 2 * k, xd, id, sf + 8u, sf, acc);
              if (KIND == T_F8SW)
                umma2_f8(d + (uint32_t)tt, w0 + off + (uint64_t)((A_BYTES >> 4) + 2 * k), xd, id, sf + 12u, sf, acc);
            } else {
              umma2(d, w0 + off + (W_MN ? 128 : 2) * k, xd, idesc, acc);
              if (KIND == T_HID) {
                umma2(d + (uint32_t)tt, w0 + off + (uint64_t)((A_BYTES >> 4) + 2 * k), xd, idesc, acc);
                umma2(d + (uint32_t)(2 * tt), w2 + off + 128 * k, xd + x_step, idesc2, acc);
              }
            }
          }
          umma2_commit_both(empty_bar(s));
          const bool last = kb == num_kb - 1;
          if (FP8 && ((kb & 3) == 3 || last)) {
            umma2_commit_own(gfree_bar(g));
            if (++g == SF_GROUPS) { g = 0; gph ^= 1u; }
          }
          if (FP8 && ((kb & 15) == 15 || last)) {
            umma2_commit_both(sempty_bar(r));
            if (++r == SF_RING) { r = 0; rph ^= 1u; }
          }
          off += stage_step;
          if (++s == nst) { s = 0; ph ^= 1u; off = 0; }
        }
        if (ok) umma2_commit_both(tfull_bar(b));
        if (++b == bufs) { b = 0; bph ^= 1u; }
      }
    }
  } else if (warp == 2 + EW) {
    // ------------------------------------------------------------ scheduler (both CTAs)
    // Tiles of a segment: token block fastest (pairs side by side share a weight tile through L2), then weight block.
    if (elect_one()) {
      int cursor = 0;
      ring.run(pair, npairs, tile_hi, ar.sched, [&](int tile, int4& a, int4& b) {
        while (tile >= tile_start[cursor + 1]) ++cursor;
        const int local = tile - tile_start[cursor], cnt = ends[cursor] - offs[cursor];
        const int ntb = (cnt + tt - 1) / tt;
        const int per = (cnt / ntb + (cnt % ntb != 0) + 15) & ~15;       // equal token blocks of whole MMA steps (cnt + ntb may pass 2^31)
        const int wb = local / ntb, r0 = (local - wb * ntb) * per;
        const int rows = min(per, cnt - r0);                             // at least one: (ntb - 1) * per < cnt
        a = make_int4(cursor, offs[cursor] + r0, rows, (rows + 15) & ~15);
        b = make_int4(wb * 256, 0, 0, 0);
      });
    }
  } else if (FP8 && warp == 3 + EW) {
    // ------------------------------------------------------------ scales (both CTAs)
    if (ar.early) wait_for_previous_kernel();
    int r = 0;
    uint32_t rph = 0;
    STile t;
    bool ok = true;
    const int nb = kbs, wb = (ar.Nout + QBLOCK - 1) / QBLOCK;
    const bool xa = scales_aligned(ar.xs_ld, ar.xs), ga = scales_aligned(nb, ar.s0), ua = scales_aligned(nb, ar.s1);
    for (int j = 0; ok; ++j) {
      if (!get_tile(j, true, t)) break;
      const int64_t blk = (int64_t)t.e * wb + min(t.w0 / QBLOCK + (int)rank, wb - 1);
      for (int k = 0; ok && k < nb; k += 16) {
        uint4 a[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          a[i] = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
          if (32 * i < t.nt)                                    // the same for the whole warp
            a[i] = scale_words(ar.xs + (int64_t)min(t.row0 + lane + 32 * i, ar.sg.rows - 1) * ar.xs_ld, k, nb, xa);
        }
        const uint4 g4 = scale_words(ar.s0 + blk * nb, k, nb, ga);
        const uint4 u4 = KIND == T_F8SW ? scale_words(ar.s1 + blk * nb, k, nb, ua) : g4;
        bool free_slot = mbar_wait(sempty_bar(r), rph ^ 1u, abort_flag);
        free_slot = __all_sync(0xffffffffu, free_slot);
        if (!free_slot) { ok = false; break; }
#pragma unroll
        for (int g = 0; g < SF_GROUPS; ++g) {
          const uint32_t dst = tiles + (uint32_t)(S::SF_OFF + r * S::SF_SLOT + g * S::SF_GROUP);
          const uint32_t gw = word_of(g4, g), uw = word_of(u4, g);
          put_words(dst, lane, word_of(a[0], g), word_of(a[1], g), word_of(a[2], g), word_of(a[3], g));
          if (t.nt > 128) put_words(dst + SF_CHUNK, lane, word_of(a[4], g), word_of(a[5], g), word_of(a[6], g), word_of(a[7], g));
          put_words(dst + 2 * SF_CHUNK, lane, gw, gw, gw, gw);
          if (KIND == T_F8SW) put_words(dst + 3 * SF_CHUNK, lane, uw, uw, uw, uw);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive_release_cluster(sfull_bar(r) & PEER_MASK);
        if (++r == SF_RING) { r = 0; rph ^= 1u; }
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue (both CTAs, own 128 weight rows)
    if (ar.early) wait_for_previous_kernel();
    const int quarter = warp & 3, sub = (warp - 2) >> 2;         // lane quarter; this warp's share of the token chunks
    int b = 0;
    uint32_t bph = 0, flip = 0;
    STile t;
    const uint32_t stg = tiles + (uint32_t)(S::STG_OFF + (warp - 2) * STG_WARP_BYTES);
    for (int j = 0;; ++j) {
      if (!get_tile(j, true, t)) break;
      bool ready = mbar_wait(tfull_bar(b), bph, abort_flag);
      ready = __all_sync(0xffffffffu, ready);
      if (KIND == T_F8SW) ready = group_all(1 + sub, 128, ready);    // the four warps of a token chunk stop together
      if (!ready) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * NACC * tt);
      const int col0 = t.w0 + (int)rank * BM;                    // first output column of this CTA
      // the accumulators go back to the MMA thread as soon as this warp has read its last columns
      bool held = true;
      auto release = [&]() {
        tc_fence_before();
        mbar_arrive_cluster(tempty_bar(b) & PEER_MASK);          // the leader waits for both CTAs' epilogues
        held = false;
      };
      const int wcol = col0 + quarter * 32, cols = ar.Nout - wcol;   // this warp's 32, and how many exist from there on
      if (col0 < ar.Nout) {                                      // (all of a CTA's warps agree)
#pragma unroll 1
        for (int c = sub * 32; c < t.nt; c += EW * 8) {          // 32 tokens at a time
          const int n = t.rows - c;                              // tokens that exist from here on (may be negative)
          const int64_t o = (int64_t)(t.row0 + c) * ar.Nout + wcol;
          const uint32_t ta = taddr + (uint32_t)c;
          const bool last = c + EW * 8 >= t.nt;
          if constexpr (KIND == T_HID) {
            uint32_t pg[2][8], pu[2][8], ph[2][8];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {                     // 16 lanes at a time
              uint32_t g[16], u[16], h[16];
              tmem_ld_frag(ta + ((uint32_t)(16 * hf) << 16), g);
              tmem_ld_frag(ta + ((uint32_t)(16 * hf) << 16) + (uint32_t)tt, u);
              tmem_ld_frag(ta + ((uint32_t)(16 * hf) << 16) + (uint32_t)(2 * tt), h);
              tmem_ld_wait();
              if (last && hf == 1) release();
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float dg[2], du[2], hh[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                  const float gv = __uint_as_float(g[2 * i + q]), uv = __uint_as_float(u[2 * i + q]), dv = __uint_as_float(h[2 * i + q]);
                  const float p = __fdividef(1.0f, 1.0f + __expf(-gv));
                  const float a = gv * p;
                  dg[q] = dv * uv * (p + a * (1.0f - p));
                  du[q] = dv * a;
                  hh[q] = a * uv;
                }
                pg[hf][i] = pack_bf16(dg[0], dg[1]);
                pu[hf][i] = pack_bf16(du[0], du[1]);
                ph[hf][i] = pack_bf16(hh[0], hh[1]);
              }
            }
            auto put = [&](const uint32_t (&p)[2][8], void* out) {
#pragma unroll
              for (int i = 0; i < 4; ++i) put_frag(stg, i, p[0][2 * i], p[0][2 * i + 1], p[1][2 * i], p[1][2 * i + 1]);
              flush_tokens(stg, (__nv_bfloat16*)out + o, ar.Nout, n, cols);
            };
            put(pg, ar.out[0]);
            put(pu, ar.out[1]);
            put(ph, ar.out[2]);
          } else if constexpr (KIND == T_F8SW) {
            uint32_t h[2][16];
            uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};          // largest magnitude of tokens 8j + 2(lane % 4) and the next
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              uint32_t u[16];
              tmem_ld_frag(ta + ((uint32_t)(16 * hf) << 16), h[hf]);
              tmem_ld_frag(ta + ((uint32_t)(16 * hf) << 16) + (uint32_t)tt, u);
              tmem_ld_wait();
              if (last && hf == 1) release();
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float gv = __uint_as_float(h[hf][i]);
                h[hf][i] = __float_as_uint(__fdividef(gv, 1.0f + __expf(-gv)) * __uint_as_float(u[i]));
                uint32_t& m = top[(i >> 2) * 2 + (i & 1)];
                m = max(m, h[hf][i] & 0x7fffffffu);
              }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], x));
            uint32_t* rd = red + ((flip * 2 + (uint32_t)sub) * 4) * 32;
            if (lane < 4) {
#pragma unroll
              for (int i = 0; i < 8; ++i) rd[quarter * 32 + (i >> 1) * 8 + 2 * lane + (i & 1)] = top[i];
            }
            group_sync(1 + sub, 128);
            flip ^= 1u;                                          // the next chunk writes the other copy
            if (quarter == 0 && lane < n)
              ar.out_scale[(int64_t)(t.row0 + c + lane) * ar.os_ld + col0 / QBLOCK] =
                  (uint8_t)scale_code(max(max(rd[lane], rd[32 + lane]), max(rd[64 + lane], rd[96 + lane])));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float f[2];
              bool bad[2];
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const int at = 8 * i + 2 * (lane & 3) + q;
                const uint32_t code = scale_code(max(max(rd[at], rd[32 + at]), max(rd[64 + at], rd[96 + at])));
                bad[q] = code == (uint32_t)Q_NAN_SCALE;
                f[q] = bad[q] ? 0.f : inv_scale(code);
              }
              uint32_t p[4];                                     // lanes 0-7, 8-15, 16-23, 24-31
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t* v = &h[k >> 1][4 * i + 2 * (k & 1)];
                const uint32_t q2 = to_e4m3x2(__uint_as_float(v[0]) * f[0], __uint_as_float(v[1]) * f[1]);
                p[k] = (bad[0] ? 0x7fu : q2 & 0xffu) | (bad[1] ? 0x7f0000u : (q2 & 0xff00u) << 8);
              }
              put_frag(stg, i, p[0], p[1], p[2], p[3]);
            }
            flush_tokens_u8(stg, (uint8_t*)ar.out[0] + o, ar.Nout, n, cols);
          } else {
            uint32_t g[2][16];
            tmem_ld_frag(ta, g[0]);
            tmem_ld_frag(ta + (16u << 16), g[1]);
            tmem_ld_wait();
            if (last) release();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t p[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t* v = &g[k >> 1][4 * i + 2 * (k & 1)];
                p[k] = pack_bf16(__uint_as_float(v[0]), __uint_as_float(v[1]));
              }
              put_frag(stg, i, p[0], p[1], p[2], p[3]);
            }
            flush_tokens(stg, (__nv_bfloat16*)ar.out[0] + o, ar.Nout, n, cols);
          }
        }
      }
      if (held) release();
      if (++b == bufs) { b = 0; bph ^= 1u; }
    }
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

// Token rows per CTA and stage for segments of `avg` rows on average: twice the average fits a tile of two CTAs, in
// steps of 16 rows, at least 16 and at most what `tt_max` columns allow.
int token_rows(int64_t avg, int tt_max) {
  int64_t tb = (avg + 15) / 16 * 16;
  if (tb < 16) tb = 16;
  if (tb > tt_max / 2) tb = tt_max / 2;
  return (int)tb;
}

// Sets the tile geometry of a launch; tt_max as for token_rows.
template <int KIND>
void geometry(TArgs& ar, int tt_max) {
  using S = ShapeT<KIND>;
  ar.tb = token_rows(ar.sg.rows / ar.sg.E, tt_max);
  ar.tt = 2 * ar.tb;
  ar.bufs = 2 * S::NACC * ar.tt <= S::COLS ? 2 : 1;
  const int stage = S::NACC * A_BYTES + S::NX * ar.tb * 128;
  ar.nst = S::RING / stage < MAX_NST ? S::RING / stage : MAX_NST;
}

template <int KIND>
int launch(const TMaps& mp, TArgs& ar, bool early, cudaStream_t st) {
  ar.early = early;
  using S = ShapeT<KIND>;
  const int pairs = sm_count() / 2;
  if (pairs < 1) return CAPMOE_EUNSUPPORTED;
  cudaError_t err = cudaFuncSetAttribute(k_gmm_rows<KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
  if (err != cudaSuccess) return note_cuda(err);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(S::THREADS);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  err = cudaLaunchKernelEx(&cfg, k_gmm_rows<KIND>, mp, ar);
  count_launch(1);
  return note_cuda(err);
}

bool map2(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, uint32_t box_rows) {
  return make_map(m, p, (uint64_t)cols, (uint64_t)rows, 0, box_rows);
}
bool map3(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t batch, uint32_t box_rows) {
  return make_map(m, p, (uint64_t)cols, (uint64_t)rows, (uint64_t)batch, box_rows);
}

}  // namespace

int gmm_fwd(const void* x, const Segments& sg, const void* w, int d, int n, void* y, int32_t* dev_status, int32_t* sched,
                  bool early, cudaStream_t st) {
  TMaps mp = {};
  TArgs ar = {};
  ar.sg = sg; ar.K = d; ar.Nout = n; ar.out[0] = y; ar.dev_status = dev_status; ar.sched = sched;
  geometry<T_FWD>(ar, 256);
  if (!map2(&mp.x0, x, d, sg.rows, (uint32_t)ar.tb) || !map3(&mp.w0, w, d, n, sg.E, BM)) return note_cuda(cudaErrorInvalidValue);
  return launch<T_FWD>(mp, ar, early, st);
}

int gmm_dx(const void* dy, const Segments& sg, const void* w, int d, int n, void* dx, int32_t* dev_status, int32_t* sched,
                 bool early, cudaStream_t st) {
  TMaps mp = {};
  TArgs ar = {};
  ar.sg = sg; ar.K = n; ar.Nout = d; ar.out[0] = dx; ar.dev_status = dev_status; ar.sched = sched;
  geometry<T_DX>(ar, 256);
  if (!map2(&mp.x0, dy, n, sg.rows, (uint32_t)ar.tb) || !make_mn_map(&mp.w0, w, d, n, sg.E)) return note_cuda(cudaErrorInvalidValue);
  ar.wide = mn_wide(d);
  return launch<T_DX>(mp, ar, early, st);
}

int gmm_hidden(const void* x, const void* dy, const Segments& sg, int d, int F, const void* wg, const void* wu,
                     const void* wd, void* dg, void* du, void* h, int32_t* dev_status, int32_t* sched, bool early, cudaStream_t st) {
  TMaps mp = {};
  TArgs ar = {};
  ar.sg = sg; ar.K = d; ar.Nout = F; ar.out[0] = dg; ar.out[1] = du; ar.out[2] = h; ar.dev_status = dev_status; ar.sched = sched;
  geometry<T_HID>(ar, 160);
  if (!map2(&mp.x0, x, d, sg.rows, (uint32_t)ar.tb) || !map2(&mp.x1, dy, d, sg.rows, (uint32_t)ar.tb) ||
      !map3(&mp.w0, wg, d, F, sg.E, BM) || !map3(&mp.w1, wu, d, F, sg.E, BM) || !make_mn_map(&mp.w2, wd, F, d, sg.E))
    return note_cuda(cudaErrorInvalidValue);
  ar.wide = mn_wide(F);
  return launch<T_HID>(mp, ar, early, st);
}

int gmm_dx2(const void* dg, const void* du, const Segments& sg, int d, int F, const void* wg, const void* wu, void* dx,
                  int32_t* dev_status, int32_t* sched, bool early, cudaStream_t st) {
  TMaps mp = {};
  TArgs ar = {};
  ar.sg = sg; ar.K = F; ar.Nout = d; ar.out[0] = dx; ar.dev_status = dev_status; ar.sched = sched;
  geometry<T_DX2>(ar, 256);
  if (!map2(&mp.x0, dg, F, sg.rows, (uint32_t)ar.tb) || !map2(&mp.x1, du, F, sg.rows, (uint32_t)ar.tb) ||
      !make_mn_map(&mp.w0, wg, d, F, sg.E) || !make_mn_map(&mp.w1, wu, d, F, sg.E))
    return note_cuda(cudaErrorInvalidValue);
  ar.wide = mn_wide(d);
  return launch<T_DX2>(mp, ar, early, st);
}

int gmm8(const uint8_t* xq, const uint8_t* xs, int64_t xs_ld, const Segments& sg, const uint8_t* wq, const uint8_t* ws, int d, int n,
               void* y, int32_t* dev_status, int32_t* sched, bool early, cudaStream_t st) {
  TMaps mp = {};
  TArgs ar = {};
  ar.sg = sg; ar.K = d; ar.Nout = n; ar.out[0] = y; ar.xs = xs; ar.xs_ld = xs_ld; ar.s0 = ws; ar.dev_status = dev_status; ar.sched = sched;
  geometry<T_F8>(ar, 224);
  if (!make_map_u8(&mp.x0, xq, d, sg.rows, 0, (uint32_t)ar.tb) || !make_map_u8(&mp.w0, wq, d, n, sg.E, BM))
    return note_cuda(cudaErrorInvalidValue);
  return launch<T_F8>(mp, ar, early, st);
}

int gmm8_swiglu_short(const uint8_t* xq, const uint8_t* xs, int64_t xs_ld, const Segments& sg, const uint8_t* wg, const uint8_t* wgs,
                      const uint8_t* wu, const uint8_t* wus, int d, int F, uint8_t* hq, uint8_t* hs, int64_t hs_ld, int32_t* dev_status,
                      int32_t* sched, bool early, cudaStream_t st) {
  TMaps mp = {};
  TArgs ar = {};
  ar.sg = sg; ar.K = d; ar.Nout = F; ar.out[0] = hq; ar.out_scale = hs; ar.os_ld = hs_ld; ar.xs = xs; ar.xs_ld = xs_ld; ar.s0 = wgs; ar.s1 = wus;
  ar.dev_status = dev_status; ar.sched = sched;
  geometry<T_F8SW>(ar, 224);
  if (!make_map_u8(&mp.x0, xq, d, sg.rows, 0, (uint32_t)ar.tb) || !make_map_u8(&mp.w0, wg, d, F, sg.E, BM) ||
      !make_map_u8(&mp.w1, wu, d, F, sg.E, BM))
    return note_cuda(cudaErrorInvalidValue);
  return launch<T_F8SW>(mp, ar, early, st);
}

}  // namespace capmoe
