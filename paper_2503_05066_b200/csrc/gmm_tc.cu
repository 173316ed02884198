// Grouped products and their gradients in bf16 on tcgen05: persistent, warp-specialised kernels over CTA
// pairs (cta_group::2), TMA-fed operand rings, fp32 accumulators in tensor memory.
//   FWD   y[r]   = W[e] x[r]                 A = x rows, K contiguous;  B = W[e], K contiguous
//   DX    dx[r]  = W[e]^T dy[r]              A = dy rows;               B = W[e] with the output columns contiguous
//   DX2   dx[r]  = W_g[e]^T dg[r] + W_u[e]^T du[r]     DX over both weights, one accumulator
//   DW    dW[e]  = sum_r dy[r] x[r]^T        reduction over the rows: both operands have their non-reduced
//                                            index contiguous; up to three products in one launch
//   HID   dg, du, h of the SwiGLU FFN's backward pass: g, u and dh of a tile side by side in tensor memory,
//         the elementwise part in the epilogue, so that g, u and dh are never rounded or written
// An operand whose output index is contiguous is "MN-major": TMA brings it in as boxes of 64 output indices (one
// 128-byte swizzle row) by 64 reduction steps, 8 KB each, and the MMA descriptor says so; nothing is transposed
// in memory.  DW's reduction runs over the ragged rows of an expert: its tensor maps are copies, one per expert,
// whose row count ends where the expert's rows end (made on the device by k_segment_maps, since the host does not
// know the offsets), so TMA fills the rows behind with zeros and no other expert's row, NaN or not, enters the sum.
// A tile is 256 x 256 (HID: 256 rows x 128 hidden columns, three accumulators); each CTA of the pair loads its 128 A
// rows and half of B, and the pair's leader issues the MMAs.  Roles, tile queue and bounded waits as in ffn_tc.cu.
// What bounds them: the tensor pipe, for every shape whose experts hold a few hundred rows.
#include "gmm.cuh"
#include "gmm_tc.cuh"

namespace capmoe {
namespace {

constexpr int64_t SHORT_LIMIT = 1024;        // rows per expert on average below which gmm_short.cu takes over

enum Kind { FWD = 0, DX = 1, DX2 = 2, DW = 3, HID = 4 };

struct GmmMaps { CUtensorMap a0, a1, b0, b1, b2, o0, o1, o2; };
struct GmmArgs {
  Segments sg;
  int K, Nout;                 // reduction length and output columns (DW: unused)
  void* out[3];                // o0..o2 as plain pointers, for pieces that do not fill a box
  int count, M[3], N[3];       // DW: products, their sizes
  int ia[3], ib[3];            // DW: which of the per-expert map lists holds A and B
  int wide_a, wide_b;          // MN-major operands: one box per k-block (DW: a bit per product)
  const CUtensorMap* maps;     // DW: [lists][E]
  int32_t* dev_status;
  int32_t* sched;
};

// DW's tensor maps: list l, expert e = the base map of matrix l with its row count set to the end of e's rows.
constexpr int MAP_LISTS = 5;
struct BaseMaps { CUtensorMap m[MAP_LISTS]; };
__global__ void __launch_bounds__(GMM_MAX_E) k_segment_maps(const __grid_constant__ BaseMaps base, Segments sg, CUtensorMap* maps) {
  allow_next_kernel();
  wait_for_previous_kernel();
  const int e = threadIdx.x, l = blockIdx.x;
  if (e >= sg.E) return;
  CUtensorMap* to = maps + (size_t)l * sg.E + e;
  const uint4* src = reinterpret_cast<const uint4*>(&base.m[l]);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(CUtensorMap) / 16); ++i) reinterpret_cast<uint4*>(to)[i] = src[i];
  const int end = max(seg_at(sg, e + 1), 1);                // a dimension is at least 1; an empty expert's map is not used
  asm volatile("tensormap.replace.tile.global_dim.global.b1024.b32 [%0], 1, %1;" ::"l"(__cvta_generic_to_global(to)), "r"(end)
               : "memory");
  asm volatile("fence.proxy.tensormap::generic.release.gpu;" ::: "memory");
}

template <int KIND>
struct Shape {
  static constexpr int A_TILES = KIND == HID ? 2 : 1;
  static constexpr int B_BYTES_CTA = KIND == HID ? 3 * 64 * BK * 2 : 128 * BK * 2;
  static constexpr int STAGE = A_TILES * A_BYTES + B_BYTES_CTA;      // 32 KB / 56 KB
  static constexpr int NST = KIND == HID ? 3 : 5;
  static constexpr int STG = KIND == HID ? 3 * STG_WARP_BYTES : WIDE_BYTES;   // staging per epilogue warp
  static constexpr int N_TILE = KIND == HID ? 128 : 256;
  static constexpr int STG_OFF = NST * STAGE;
  static constexpr int TAIL = STG_OFF + EPI_WARPS * STG;
  static constexpr int SMEM = TAIL + 1024 + 512 + 3 * (GMM_MAX_E + 1) * 4 + 16 + TR_BYTES;
  static constexpr int BUFS = KIND == HID ? 1 : 2;                   // accumulators of 256 columns, or three of 128
};
static_assert(Shape<HID>::SMEM <= 227 * 1024 && Shape<FWD>::SMEM <= 227 * 1024, "shared memory of a thread block");

// rows: valid rows of the tile from row0 (DW: of the output); k0: first row of the expert
struct GTile { int e, row0, rows, n0, p, num_kb, k0; };

constexpr int GMM_THREADS = TC_THREADS + 32;             // one more warp: the scheduler

template <int KIND, typename TO>
__global__ void __launch_bounds__(GMM_THREADS, 1) k_gmm2(const __grid_constant__ GmmMaps mp, const __grid_constant__ GmmArgs ar) {
  using S = Shape<KIND>;
  constexpr int NST = S::NST, N_TILE = S::N_TILE, BM2 = 2 * BM;
  constexpr bool A_MN = KIND == DW, B_MN = KIND == DX || KIND == DX2 || KIND == DW;
  allow_next_kernel();
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

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank();                      // 0 = leader (issues the MMAs)
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(MAX_STAGES + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (uint32_t)(2 * MAX_STAGES + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (uint32_t)(2 * MAX_STAGES + 2 + b); };
  const TileRing ring{bar0 + 8u * RING_BAR, smem_u32(tile_start + (GMM_MAX_E + 1) + 1) /* 3 * 257 + 1 ints: 16-byte aligned */,
                      rank, abort_flag};

  // set-up that touches no global memory comes before the wait for the previous kernel
  if (tid == 0) {
    for (int s = 0; s < NST; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < S::BUFS; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * EPI_WARPS * 32); }
    ring.init(1 + (rank == 0 ? 1 : 0) + EPI_WARPS);             // TMA thread, MMA thread, epilogue warps
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
  for (int i = tid; i < E; i += GMM_THREADS) { offs[i] = seg_at(ar.sg, i); ends[i] = max(offs[i], seg_at(ar.sg, i + 1)); }
  __syncthreads();
  int per_e = 0;                                                // DW: tiles of one expert
  if (KIND == DW)
    for (int p = 0; p < ar.count; ++p) per_e += ((ar.M[p] + 255) >> 8) * ((ar.N[p] + 255) >> 8);
  if (KIND != DW && warp == 0) {                                // tile_start: exclusive prefix, 32 experts at a time
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
  cluster_sync_all();             // the peer's barriers are initialised and its tensor memory allocated
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int tile_hi = KIND == DW ? E * per_e : tile_start[E];
  auto get_tile = [&](int j, bool whole_warp, GTile& t) -> bool {
    int4 a, b;
    if (!ring.get(j, whole_warp, a, b)) return false;
    t.e = a.x; t.row0 = a.y; t.rows = a.z; t.n0 = a.w;
    t.p = b.x; t.num_kb = b.y; t.k0 = b.z;
    return true;
  };

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (both CTAs)
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 0;
      GTile t;
      bool ok = true;
      int mapped = -1;                                          // DW: expert whose maps were last acquired
      for (int j = 0; ok; ++j) {
        if (!get_tile(j, false, t)) break;
        const CUtensorMap *ma = &mp.a0, *mb = &mp.b0;
        if (KIND == DW) {
          ma = ar.maps + (size_t)ar.ia[t.p] * E + t.e;
          mb = ar.maps + (size_t)ar.ib[t.p] * E + t.e;
          if (mapped != t.e * 4 + t.p) {
            asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(ma) : "memory");
            asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(mb) : "memory");
            mapped = t.e * 4 + t.p;
          }
        }
        const int half_kb = KIND == DX2 ? t.num_kb / 2 : t.num_kb;
        for (int kb = 0; kb < t.num_kb; ++kb) {
          if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t bar = full_bar(s) & PEER_MASK;         // the leader's barrier counts both CTAs' bytes
          if (rank == 0) mbar_expect_tx(full_bar(s), 2 * S::STAGE);
          const uint32_t a_dst = tiles + (uint32_t)s * S::STAGE;
          const uint32_t b_dst = a_dst + S::A_TILES * A_BYTES;
          const int m0 = t.row0 + (int)rank * BM;
          if constexpr (KIND == FWD) {
            tma2_load_2d(a_dst, ma, kb * BK, m0, bar);
            tma2_load_3d(b_dst, mb, kb * BK, t.n0 + (int)rank * 128, t.e, bar);
          } else if constexpr (KIND == DX || KIND == DX2) {
            const bool second = KIND == DX2 && kb >= half_kb;
            const int k = (second ? kb - half_kb : kb) * BK, n = t.n0 + (int)rank * 128;
            tma2_load_2d(a_dst, second ? &mp.a1 : ma, k, m0, bar);
            load_mn(b_dst, second ? &mp.b1 : mb, ar.wide_b, n, k, t.e, bar);
          } else if constexpr (KIND == DW) {
            const int r = t.k0 + kb * BK, n = t.n0 + (int)rank * 128;
            load_mn(a_dst, ma, (ar.wide_a >> t.p) & 1, m0, r, bar);
            load_mn(b_dst, mb, (ar.wide_b >> t.p) & 1, n, r, bar);
          } else {
            const int n = t.n0 + (int)rank * 64;
            tma2_load_2d(a_dst, &mp.a0, kb * BK, m0, bar);
            tma2_load_2d(a_dst + A_BYTES, &mp.a1, kb * BK, m0, bar);
            tma2_load_3d(b_dst, &mp.b0, kb * BK, n, t.e, bar);
            tma2_load_3d(b_dst + 8192u, &mp.b1, kb * BK, n, t.e, bar);
            tma2_load_3d(b_dst + 16384u, &mp.b2, n, kb * BK, t.e, bar);
          }
          if (++s == NST) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (leader CTA only)
    if (rank == 0 && elect_one()) {
      int s = 0;
      uint32_t it = 0, ph = 0;
      const uint32_t i0 = pair_idesc(256, A_MN, B_MN), i1 = pair_idesc(128, false, true);
      const uint64_t a0 = A_MN ? umma_desc_mn(tiles) : umma_desc(tiles);
      const uint64_t b0 = B_MN ? umma_desc_mn(tiles + S::A_TILES * A_BYTES) : umma_desc(tiles + S::A_TILES * A_BYTES);
      const uint64_t a1 = umma_desc(tiles + A_BYTES);                                   // HID: dy
      const uint64_t b1 = umma_desc_mn(tiles + S::A_TILES * A_BYTES + 16384u);          // HID: W_d
      constexpr uint64_t KA = A_MN ? 128 : 2, KB = B_MN ? 128 : 2;   // 16 reduction steps: 16 rows of 128 bytes, or 32 bytes
      uint64_t off = 0;
      GTile t;
      bool ok = true;
      for (int j = 0; ok; ++j, ++it) {
        if (!get_tile(j, false, t)) break;
        const uint32_t b = S::BUFS == 2 ? it & 1u : 0u, use = S::BUFS == 2 ? it >> 1 : it;
        if (!mbar_wait(tempty_bar(b), (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem_base + b * 256u;
        for (int kb = 0; kb < t.num_kb; ++kb) {
          if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k) {
            const uint32_t acc = (kb | k) != 0 ? 1u : 0u;
            umma2(d, a0 + off + KA * k, b0 + off + KB * k, i0, acc);
            if (KIND == HID) umma2(d + 256u, a1 + off + 2 * k, b1 + off + 128 * k, i1, acc);
          }
          umma2_commit_both(empty_bar(s));                      // both CTAs may refill this stage
          off += (uint64_t)(S::STAGE >> 4);
          if (++s == NST) { s = 0; ph ^= 1u; off = 0; }
        }
        if (ok) umma2_commit_both(tfull_bar(b));
      }
    }
  } else if (warp == 2 + EPI_WARPS) {
    // ------------------------------------------------------------ scheduler (both CTAs)
    if (elect_one()) {
      int cursor = 0;
      ring.run(pair, npairs, tile_hi, ar.sched, [&](int tile, int4& a, int4& b) {
        if (KIND == DW) {
          const int e = tile / per_e;
          int local = tile - e * per_e, p = 0, nmb = (ar.M[0] + 255) >> 8;
          while (p + 1 < ar.count) {
            const int here = nmb * ((ar.N[p] + 255) >> 8);
            if (local < here) break;
            local -= here;
            nmb = (ar.M[++p] + 255) >> 8;
          }
          const int nb = local / nmb, m0 = (local - nb * nmb) * BM2;
          a = make_int4(e, m0, min(BM2, ar.M[p] - m0), nb * 256);
          b = make_int4(p, (ends[e] - offs[e] + BK - 1) / BK, offs[e], 0);
        } else {
          Tile q;
          locate_tile(tile, cursor, tile_start, offs, ends, E, N_TILE, BM2, q);
          a = make_int4(q.e, q.row0, q.rows, q.n0);
          b = make_int4(0, (ar.K + BK - 1) / BK * (KIND == DX2 ? 2 : 1), 0, 0);
        }
      });
    }
  } else {
    // ------------------------------------------------------------ epilogue (both CTAs, own 128 rows)
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint32_t it = 0;
    GTile t;
    uint8_t* stg = gen + S::STG_OFF + (warp - 2) * S::STG;
    for (int j = 0;; ++j, ++it) {
      if (!get_tile(j, true, t)) break;
      const uint32_t b = S::BUFS == 2 ? it & 1u : 0u, use = S::BUFS == 2 ? it >> 1 : it;
      bool ready = mbar_wait(tfull_bar(b), use & 1u, abort_flag);
      ready = __all_sync(0xffffffffu, ready);
      if (!ready) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + b * 256u;
      const int warp_row0 = (int)rank * BM + quarter * 32;      // first of this warp's 32 rows in the pair's tile
      const bool full_rows = warp_row0 + 32 <= t.rows, row_ok = warp_row0 + lane < t.rows;
      const bool empty_sum = KIND == DW && t.num_kb == 0;       // an expert without rows: zeros
      const int Nout = KIND == DW ? ar.N[t.p] : ar.Nout;
      const int64_t row = (KIND == DW ? (int64_t)t.e * ar.M[t.p] : 0) + t.row0 + warp_row0;
      const CUtensorMap* mo = KIND != DW || t.p == 0 ? &mp.o0 : t.p == 1 ? &mp.o1 : &mp.o2;
      TO* orow = reinterpret_cast<TO*>(ar.out[KIND == DW ? t.p : 0]) + (row + lane) * Nout + t.n0;
      if constexpr (KIND == HID) {
        // hidden column c of the tile: g in accumulator column (c / 64) * 128 + c % 64, u 64 further on, dh in 256 + c
#pragma unroll 1
        for (int c = half * 64; c < half * 64 + 64; c += 32) {
          if (t.n0 + c >= Nout) break;
          uint32_t g[32], u[32], h[32];
          tmem_ld32(taddr + (uint32_t)(half * 128 + (c & 63)), g);
          tmem_ld32(taddr + (uint32_t)(half * 128 + 64 + (c & 63)), u);
          tmem_ld32(taddr + 256u + (uint32_t)c, h);
          tmem_ld_wait();
          uint32_t pg[16], pu[16], phd[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
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
            pg[i] = pack_bf16(dg[0], dg[1]);
            pu[i] = pack_bf16(du[0], du[1]);
            phd[i] = pack_bf16(hh[0], hh[1]);
          }
          const int64_t o = (row + lane) * Nout + t.n0 + c;
          const int left = Nout - (t.n0 + c);
          put_piece(pg, true, full_rows, row_ok, stg, &mp.o0, t.n0 + c, (int)row, (__nv_bfloat16*)ar.out[0] + o, left);
          put_piece(pu, false, full_rows, row_ok, stg + STG_WARP_BYTES, &mp.o1, t.n0 + c, (int)row, (__nv_bfloat16*)ar.out[1] + o, left);
          put_piece(phd, false, full_rows, row_ok, stg + 2 * STG_WARP_BYTES, &mp.o2, t.n0 + c, (int)row,
                       (__nv_bfloat16*)ar.out[2] + o, left);
        }
      } else {
        constexpr int PC = 128 / (int)sizeof(TO);               // columns of a piece
#pragma unroll 1
        for (int c = half * 128; c < half * 128 + 128; c += PC) {
          if (t.n0 + c >= Nout) break;
          uint32_t g[PC], w[32];
          if (empty_sum) {
#pragma unroll
            for (int i = 0; i < PC; ++i) g[i] = 0u;
          } else {
#pragma unroll
            for (int i = 0; i < PC; i += 32) tmem_ld32(taddr + (uint32_t)(c + i), g + i);
            tmem_ld_wait();
          }
#pragma unroll
          for (int i = 0; i < 32; ++i)
            w[i] = sizeof(TO) == 2 ? pack_bf16(__uint_as_float(g[2 * i % PC]), __uint_as_float(g[(2 * i + 1) % PC])) : g[i];
          put_wide(w, full_rows, row_ok, stg, mo, t.n0 + c, (int)row, orow + c, (Nout - (t.n0 + c)) * (int)sizeof(TO));
        }
      }
      tc_fence_before();
      mbar_arrive_cluster(tempty_bar(b) & PEER_MASK);           // the leader waits for both CTAs' epilogues
    }
    if (lane == 0) bulk_wait_all();                              // this lane's stores have landed before the CTA ends
  }

  // ------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();             // no signal of the peer can still be on its way to this CTA
  if (warp == 1) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
  if (tid == 0 && *abort_flag && ar.dev_status) atomicExch(ar.dev_status, (int)CAPMOE_ETIMEOUT);
}

template <int KIND, typename TO>
int launch(const GmmMaps& mp, const GmmArgs& ar, cudaStream_t st) {
  const int pairs = sm_count() / 2;
  if (pairs < 1) return CAPMOE_EUNSUPPORTED;
  cudaError_t err = cudaFuncSetAttribute(k_gmm2<KIND, TO>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<KIND>::SMEM);
  if (err != cudaSuccess) return note_cuda(err);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(GMM_THREADS);
  cfg.dynamicSmemBytes = Shape<KIND>::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see wait_for_previous_kernel()
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  err = cudaLaunchKernelEx(&cfg, k_gmm2<KIND, TO>, mp, ar);
  count_launch(1);
  return note_cuda(err);
}

// Tile counters in the caller's status block: slot i of the launches of one call; cleared by begin_counters.
int32_t* counter(int32_t* dev_status, int i) { return dev_status ? dev_status + 1 + i : nullptr; }
int begin_counters(int32_t* dev_status, int n, cudaStream_t st) {
  return dev_status ? clear_words(dev_status + 1, n, nullptr, 0, st) : CAPMOE_OK;
}

// bf16 [batch, rows, cols] in boxes of 64 columns x box_rows
bool map3(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t batch, uint32_t box_rows) {
  return make_map(m, p, (uint64_t)cols, (uint64_t)rows, (uint64_t)batch, box_rows);
}
bool map2(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, uint32_t box_rows) {
  return make_map(m, p, (uint64_t)cols, (uint64_t)rows, 0, box_rows);
}

int segment_maps(const BaseMaps& base, int lists, const Segments& sg, void* ws, cudaStream_t st) {
  const int rc = note_cuda(launch_chained(k_segment_maps, (unsigned)lists, GMM_MAX_E, 0, st, base, sg, (CUtensorMap*)ws));
  count_launch(1);
  return rc;
}

}  // namespace

// Rows of 16 bytes for TMA; dw's E * n (E * d) rows are 32-bit coordinates.
bool gmm_tc_supported(int E, int d, int n, int dtype) {
  const int64_t lim = (int64_t)1 << 31;
  return dtype == CAPMOE_BF16 && d % 8 == 0 && n % 8 == 0 && (int64_t)E * n < lim && (int64_t)E * d < lim;
}
size_t gmm_tc_map_bytes(int E, int lists) { return (size_t)lists * E * sizeof(CUtensorMap); }

int gmm_tc_fwd(const void* x, const Segments& sg, const void* w, int d, int n, void* y, int32_t* dev_status, cudaStream_t st) {
  if (use_short(sg, SHORT_LIMIT)) {
    const int rc0 = begin_counters(dev_status, 1, st);
    return rc0 != CAPMOE_OK ? rc0 : gmm_short_fwd(x, sg, w, d, n, y, dev_status, counter(dev_status, 0), st);
  }
  GmmMaps mp = {};
  GmmArgs ar = {};
  if (!map2(&mp.a0, x, d, sg.rows, BM) || !map3(&mp.b0, w, d, n, sg.E, 128) || !make_wide_map(&mp.o0, y, n, sg.rows, 2))
    return note_cuda(cudaErrorInvalidValue);
  const int rc = begin_counters(dev_status, 1, st);
  if (rc != CAPMOE_OK) return rc;
  ar.sg = sg; ar.K = d; ar.Nout = n; ar.out[0] = y; ar.dev_status = dev_status; ar.sched = counter(dev_status, 0);
  return launch<FWD, __nv_bfloat16>(mp, ar, st);
}

int gmm_tc_dx(const void* dy, const Segments& sg, const void* w, int d, int n, void* dx, int32_t* dev_status, cudaStream_t st) {
  if (use_short(sg, SHORT_LIMIT)) {
    const int rc0 = begin_counters(dev_status, 1, st);
    return rc0 != CAPMOE_OK ? rc0 : gmm_short_dx(dy, sg, w, d, n, dx, dev_status, counter(dev_status, 0), st);
  }
  GmmMaps mp = {};
  GmmArgs ar = {};
  if (!map2(&mp.a0, dy, n, sg.rows, BM) || !make_mn_map(&mp.b0, w, d, n, sg.E) || !make_wide_map(&mp.o0, dx, d, sg.rows, 2))
    return note_cuda(cudaErrorInvalidValue);
  const int rc = begin_counters(dev_status, 1, st);
  if (rc != CAPMOE_OK) return rc;
  ar.sg = sg; ar.K = n; ar.Nout = d; ar.out[0] = dx; ar.wide_b = mn_wide(d); ar.dev_status = dev_status; ar.sched = counter(dev_status, 0);
  return launch<DX, __nv_bfloat16>(mp, ar, st);
}

int gmm_tc_dw(const void* dy, const void* x, const Segments& sg, int d, int n, bool out_f32, void* dw, void* ws, int32_t* dev_status,
              cudaStream_t st) {
  GmmMaps mp = {};
  GmmArgs ar = {};
  BaseMaps base = {};
  if (!make_mn_map(&base.m[0], dy, n, sg.rows, 0) || !make_mn_map(&base.m[1], x, d, sg.rows, 0) ||
      !make_wide_map(&mp.o0, dw, d, (uint64_t)sg.E * n, out_f32 ? 4 : 2))
    return note_cuda(cudaErrorInvalidValue);
  int rc = begin_counters(dev_status, 1, st);
  if (rc == CAPMOE_OK) rc = segment_maps(base, 2, sg, ws, st);
  if (rc != CAPMOE_OK) return rc;
  ar.sg = sg; ar.out[0] = dw; ar.count = 1; ar.M[0] = n; ar.N[0] = d; ar.ia[0] = 0; ar.ib[0] = 1;
  ar.wide_a = mn_wide(n); ar.wide_b = mn_wide(d);
  ar.maps = (const CUtensorMap*)ws; ar.dev_status = dev_status; ar.sched = counter(dev_status, 0);
  return out_f32 ? launch<DW, float>(mp, ar, st) : launch<DW, __nv_bfloat16>(mp, ar, st);
}

// ws: the maps (gmm_tc_map_bytes(E, 5)), then dg, du and h [rows, F]
int gmm_tc_ffn_grad(const void* x, const void* dy, const Segments& sg, int d, int F, const void* wg, const void* wu,
                    const void* wd, void* dx, void* dwg, void* dwu, void* dwd, void* map_ws, void* hidden, int32_t* dev_status,
                    cudaStream_t st) {
  using B = __nv_bfloat16;
  B* dg = (B*)hidden;
  B* du = dg + (int64_t)sg.rows * F;
  B* h = du + (int64_t)sg.rows * F;
  GmmMaps m1 = {}, m2 = {}, m3 = {};
  BaseMaps base = {};
  const int64_t R = sg.rows;
  if (!map2(&m1.a0, x, d, R, BM) || !map2(&m1.a1, dy, d, R, BM) || !map3(&m1.b0, wg, d, F, sg.E, 64) ||
      !map3(&m1.b1, wu, d, F, sg.E, 64) || !map3(&m1.b2, wd, F, d, sg.E, 64) || !make_store_map(&m1.o0, dg, F, R) ||
      !make_store_map(&m1.o1, du, F, R) || !make_store_map(&m1.o2, h, F, R) ||
      !make_mn_map(&base.m[0], dg, F, R, 0) || !make_mn_map(&base.m[1], du, F, R, 0) || !make_mn_map(&base.m[2], dy, d, R, 0) ||
      !make_mn_map(&base.m[3], x, d, R, 0) || !make_mn_map(&base.m[4], h, F, R, 0) ||
      !make_wide_map(&m2.o0, dwg, d, (uint64_t)sg.E * F, 2) || !make_wide_map(&m2.o1, dwu, d, (uint64_t)sg.E * F, 2) ||
      !make_wide_map(&m2.o2, dwd, F, (uint64_t)sg.E * d, 2) ||
      !map2(&m3.a0, dg, F, R, BM) || !map2(&m3.a1, du, F, R, BM) || !make_mn_map(&m3.b0, wg, d, F, sg.E) ||
      !make_mn_map(&m3.b1, wu, d, F, sg.E) || !make_wide_map(&m3.o0, dx, d, R, 2))
    return note_cuda(cudaErrorInvalidValue);
  int rc = begin_counters(dev_status, 3, st);
  if (rc == CAPMOE_OK) rc = segment_maps(base, MAP_LISTS, sg, map_ws, st);
  if (rc != CAPMOE_OK) return rc;
  GmmArgs a1 = {}, a2 = {}, a3 = {};
  a1.sg = a2.sg = a3.sg = sg;
  a1.dev_status = a2.dev_status = a3.dev_status = dev_status;
  a1.sched = counter(dev_status, 0); a2.sched = counter(dev_status, 1); a3.sched = counter(dev_status, 2);
  a1.K = d; a1.Nout = F; a1.out[0] = dg; a1.out[1] = du; a1.out[2] = h;
  a3.K = F; a3.Nout = d; a3.out[0] = dx; a3.wide_b = mn_wide(d);
  const bool brief = use_short(sg, SHORT_LIMIT);
  rc = brief ? gmm_short_hidden(x, dy, sg, d, F, wg, wu, wd, dg, du, h, dev_status, a1.sched, st) : launch<HID, B>(m1, a1, st);
  if (rc != CAPMOE_OK) return rc;
  rc = brief ? gmm_short_dx2(dg, du, sg, d, F, wg, wu, dx, dev_status, a3.sched, st) : launch<DX2, B>(m3, a3, st);
  if (rc != CAPMOE_OK) return rc;
  a2.count = 3;
  a2.out[0] = dwg; a2.out[1] = dwu; a2.out[2] = dwd;
  a2.M[0] = a2.M[1] = F; a2.M[2] = d;
  a2.N[0] = a2.N[1] = d; a2.N[2] = F;
  a2.ia[0] = 0; a2.ia[1] = 1; a2.ia[2] = 2;
  a2.ib[0] = a2.ib[1] = 3; a2.ib[2] = 4;
  a2.wide_a = (mn_wide(F) ? 3 : 0) | (mn_wide(d) ? 4 : 0);
  a2.wide_b = (mn_wide(d) ? 3 : 0) | (mn_wide(F) ? 4 : 0);
  a2.maps = (const CUtensorMap*)map_ws;
  return launch<DW, B>(m2, a2, st);
}

}  // namespace capmoe
