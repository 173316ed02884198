// Weight gradients of the grouped products in bf16 on tcgen05: dW[e] = sum over the rows r of expert e of p[r] q[r]^T, up
// to three products in one launch.  Persistent, warp-specialised kernel over CTA pairs (cta_group::2), 256 x 256 output
// tiles, TMA-fed operand ring, two fp32 accumulators in tensor memory.
// The reduction runs over rows, so both operands have their output index contiguous ("MN-major"): TMA brings them in as
// boxes of 64 output indices (one 128-byte swizzle row) by 64 rows, and the MMA descriptor says so; nothing is
// transposed in memory.  The rows of an expert are ragged: the tensor maps are copies, one per expert, whose row count
// ends where the expert's rows end (made on the device by k_segment_maps, since the host does not know the offsets),
// so TMA fills the rows behind with zeros and no other expert's row, NaN or not, enters the sum.
// When the tiles are fewer than half the pairs (one or two experts of a rank, thousands of rows each) the reductions are
// split into parts, each a tile of its own with an fp32 output in the workspace, and a second kernel adds the parts in
// their order.
// What bounds it: a tile of an expert with a few hundred rows has only a handful of k-blocks, about as long as its
// epilogue (3200 cycles) and as its share of the HBM writes; 17,500 rows of 64 experts, 2048 x 1024, 268 MB of
// gradients: 87 us for one cold launch (0.46 of the tensor pipe, 0.44 of the peak DRAM rate), about 105 us in a loop at the
// power limit, 84 with operands of zeros, which do not reach it; the FFN's three gradients there 240 us cold.
#include "gmm.cuh"
#include "gmm_tc.cuh"

namespace capmoe {
namespace {

struct DwMaps { CUtensorMap o0, o1, o2; };
struct DwArgs {
  Segments sg;
  void* out[3];                // the outputs as plain pointers, for pieces that do not fill a box
  int count, M[3], N[3];       // products, their sizes: out[p] is [E, M, N]
  int ia[3], ib[3];            // which of the per-expert map lists holds each product's operands
  int split;                   // parts of every reduction, each with an output of its own: out[p] is [split, E, M, N]
  int wide_a, wide_b;          // a bit per product: one box per k-block (see make_mn_map)
  const CUtensorMap* maps;     // [lists][E]
  int32_t* dev_status;
  int32_t* sched;
};

// Tensor maps: list l, expert e = the base map of matrix l with its row count set to the end of e's rows.
constexpr int MAP_LISTS = 5;
struct BaseMaps { CUtensorMap m[MAP_LISTS]; };
__global__ void __launch_bounds__(GMM_MAX_E) k_segment_maps(const __grid_constant__ BaseMaps base, Segments sg, CUtensorMap* maps, int32_t* counter) {
  wait_for_previous_kernel();
  allow_next_kernel();                       // in this order: an early successor reads what came before (gmm.cuh)
  const int e = threadIdx.x, l = blockIdx.x;
  if (counter && e == 0 && l == 0) *counter = 0;
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

constexpr int DW_NST = 5;
constexpr int DW_STAGE = 2 * A_BYTES;                         // 128 columns of each operand by 64 rows: 32 KB
constexpr int DW_STG_OFF = DW_NST * DW_STAGE;
constexpr int DW_TAIL = DW_STG_OFF + EPI_WARPS * WIDE_BYTES;
constexpr int DW_SMEM = DW_TAIL + 1024 + 512 + 2 * (GMM_MAX_E + 1) * 4 + 16 + TR_BYTES;
static_assert(DW_SMEM <= 227 * 1024, "shared memory of a thread block");

// e, product p; row0, rows: output rows of the tile; n0: first output column; k0, num_kb: first row and k-blocks of the
// reduction; oe: which of the output's [split * E] matrices
struct DTile { int e, row0, rows, n0, p, num_kb, k0, oe; };

constexpr int GMM_THREADS = TC_THREADS + 32;             // one more warp: the scheduler

template <typename TO>
__global__ void __launch_bounds__(GMM_THREADS, 1) k_gmm_dw(const __grid_constant__ DwMaps mp, const __grid_constant__ DwArgs ar) {
  constexpr int BM2 = 2 * BM;
  allow_next_kernel();
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (tiles - raw);
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen + DW_TAIL);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 52);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* offs = reinterpret_cast<int*>(gen + DW_TAIL + 512);
  int* ends = offs + (GMM_MAX_E + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank();                      // 0 = leader (issues the MMAs)
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(MAX_STAGES + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (uint32_t)(2 * MAX_STAGES + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (uint32_t)(2 * MAX_STAGES + 2 + b); };
  // A tile lasts as long as its reduction, whose length the host does not know: 0.28 to 0.46 us a k-block for a pair on its
  // own (2^25 rows of one expert, 8 x 8 to 88 x 88), so 400 million rows outlast the usual limit.  Waits for a whole tile get
  // about 2 us more for each k-block that may be in it.
  const long long tile_limit = WAIT_LIMIT_CYCLES + (long long)(ar.sg.rows / BK) * 4096;
  const TileRing ring{bar0 + 8u * RING_BAR, smem_u32(ends + (GMM_MAX_E + 1) + 2) /* 2 * 257 + 2 ints: 16-byte aligned */, rank,
                      abort_flag, tile_limit};

  // set-up that touches no global memory comes before the wait for the previous kernel
  if (tid == 0) {
    for (int s = 0; s < DW_NST; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * EPI_WARPS * 32); }
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
  int per_e = 0;                                                // tiles of one expert
  for (int p = 0; p < ar.count; ++p) per_e += ((ar.M[p] + 255) >> 8) * ((ar.N[p] + 255) >> 8);
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();             // the peer's barriers are initialised and its tensor memory allocated
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int tile_hi = E * per_e * ar.split;
  auto get_tile = [&](int j, bool whole_warp, DTile& t) -> bool {
    int4 a, b;
    if (!ring.get(j, whole_warp, a, b)) return false;
    t.e = a.x; t.row0 = a.y; t.rows = a.z; t.n0 = a.w;
    t.p = b.x; t.num_kb = b.y; t.k0 = b.z; t.oe = b.w;
    return true;
  };

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (both CTAs)
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 0;
      DTile t;
      bool ok = true;
      int mapped = -1;                                          // expert and product whose maps were last acquired
      for (int j = 0; ok; ++j) {
        if (!get_tile(j, false, t)) break;
        const CUtensorMap* ma = ar.maps + (size_t)ar.ia[t.p] * E + t.e;
        const CUtensorMap* mb = ar.maps + (size_t)ar.ib[t.p] * E + t.e;
        if (mapped != t.e * 4 + t.p) {
          asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(ma) : "memory");
          asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(mb) : "memory");
          mapped = t.e * 4 + t.p;
        }
        for (int kb = 0; kb < t.num_kb; ++kb) {
          if (!mbar_wait(empty_bar(s), ph ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t bar = full_bar(s) & PEER_MASK;         // the leader's barrier counts both CTAs' bytes
          if (rank == 0) mbar_expect_tx(full_bar(s), 2 * DW_STAGE);
          const uint32_t a_dst = tiles + (uint32_t)s * DW_STAGE;
          const int r = t.k0 + kb * BK;
          load_mn(a_dst, ma, (ar.wide_a >> t.p) & 1, t.row0 + (int)rank * BM, r, bar);
          load_mn(a_dst + A_BYTES, mb, (ar.wide_b >> t.p) & 1, t.n0 + (int)rank * 128, r, bar);
          if (++s == DW_NST) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (leader CTA only)
    if (rank == 0 && elect_one()) {
      int s = 0;
      uint32_t it = 0, ph = 0;
      const uint32_t idesc = pair_idesc(256, true, true);
      const uint64_t a0 = umma_desc_mn(tiles), b0 = umma_desc_mn(tiles + A_BYTES);
      uint64_t off = 0;
      DTile t;
      bool ok = true;
      for (int j = 0; ok; ++j, ++it) {
        if (!get_tile(j, false, t)) break;
        const uint32_t b = it & 1u, use = it >> 1;
        if (!mbar_wait(tempty_bar(b), (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem_base + b * 256u;
        for (int kb = 0; kb < t.num_kb; ++kb) {
          if (!mbar_wait(full_bar(s), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < BK / UMMA_K; ++k)                 // 16 reduction steps: 16 rows of 128 bytes
            umma2(d, a0 + off + 128 * k, b0 + off + 128 * k, idesc, (kb | k) != 0 ? 1u : 0u);
          umma2_commit_both(empty_bar(s));                      // both CTAs may refill this stage
          off += (uint64_t)(DW_STAGE >> 4);
          if (++s == DW_NST) { s = 0; ph ^= 1u; off = 0; }
        }
        if (ok) umma2_commit_both(tfull_bar(b));
      }
    }
  } else if (warp == 2 + EPI_WARPS) {
    // ------------------------------------------------------------ scheduler (both CTAs)
    if (elect_one()) {
      ring.run(pair, npairs, tile_hi, ar.sched, [&](int tile, int4& a, int4& b) {
        const int part = tile / per_e, e = part / ar.split, s = part - e * ar.split;
        int local = tile - part * per_e, p = 0, nmb = (ar.M[0] + 255) >> 8;
        while (p + 1 < ar.count) {
          const int here = nmb * ((ar.N[p] + 255) >> 8);
          if (local < here) break;
          local -= here;
          nmb = (ar.M[++p] + 255) >> 8;
        }
        const int nb = local / nmb, m0 = (local - nb * nmb) * BM2;
        a = make_int4(e, m0, min(BM2, ar.M[p] - m0), nb * 256);
        const int kbs = (ends[e] - offs[e] + BK - 1) / BK, each = (kbs + ar.split - 1) / ar.split, first = min(s * each, kbs);
        b = make_int4(p, min(each, kbs - first), offs[e] + first * BK, s * E + e);
      });
    }
  } else {
    // ------------------------------------------------------------ epilogue (both CTAs, own 128 rows)
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint32_t it = 0;
    DTile t;
    uint8_t* stg = gen + DW_STG_OFF + (warp - 2) * WIDE_BYTES;
    for (int j = 0;; ++j, ++it) {
      if (!get_tile(j, true, t)) break;
      const uint32_t b = it & 1u, use = it >> 1;
      bool ready = mbar_wait(tfull_bar(b), use & 1u, abort_flag, tile_limit);
      ready = __all_sync(0xffffffffu, ready);
      if (!ready) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + b * 256u;
      const int warp_row0 = (int)rank * BM + quarter * 32;      // first of this warp's 32 rows in the pair's tile
      const bool full_rows = warp_row0 + 32 <= t.rows, row_ok = warp_row0 + lane < t.rows;
      const bool empty_sum = t.num_kb == 0;                     // an expert without rows: zeros
      const int Nout = ar.N[t.p];
      const int64_t row = (int64_t)t.oe * ar.M[t.p] + t.row0 + warp_row0;
      const CUtensorMap* mo = t.p == 0 ? &mp.o0 : t.p == 1 ? &mp.o1 : &mp.o2;
      TO* orow = reinterpret_cast<TO*>(ar.out[t.p]) + (row + lane) * Nout + t.n0;
      constexpr int PC = 128 / (int)sizeof(TO);               // columns of a piece
      bool held = true;
      auto release = [&]() {                                  // this warp has read its last columns
        tc_fence_before();
        mbar_arrive_cluster(tempty_bar(b) & PEER_MASK);       // the leader waits for both CTAs' epilogues
        held = false;
      };
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
        if (held && (c + PC >= half * 128 + 128 || t.n0 + c + PC >= Nout)) release();
#pragma unroll
        for (int i = 0; i < 32; ++i)
          w[i] = sizeof(TO) == 2 ? pack_bf16(__uint_as_float(g[2 * i % PC]), __uint_as_float(g[(2 * i + 1) % PC])) : g[i];
        put_wide(w, full_rows, row_ok, stg, mo, t.n0 + c, (int)row, orow + c, (Nout - (t.n0 + c)) * (int)sizeof(TO));
      }
      if (held) release();
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

// Sum of the parts, in their order.  out[p] [n] from parts [3][split][n], n a multiple of 4.
template <typename TO> struct JoinSet { TO* out[3]; };
template <typename TO>
__global__ void __launch_bounds__(256) k_join_parts(const float* __restrict__ parts, JoinSet<TO> to, int split, int64_t n, int per_product) {
  wait_for_previous_kernel();
  allow_next_kernel();
  const int p = (int)blockIdx.x / per_product;
  const int64_t i = ((int64_t)(blockIdx.x - (unsigned)(p * per_product)) * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  const float* from = parts + (int64_t)p * split * n + i;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0; k < split; ++k) {
    const float4 v = *reinterpret_cast<const float4*>(from + k * n);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  if constexpr (sizeof(TO) == 4) *reinterpret_cast<float4*>(to.out[p] + i) = s;
  else *reinterpret_cast<uint2*>(to.out[p] + i) = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
}
template <typename TO>
int join_parts(const float* parts, int products, const JoinSet<TO>& to, int split, int64_t n, cudaStream_t st) {
  const int per = (int)ceil_div(n, 1024);
  const int rc = note_cuda(launch_chained(k_join_parts<TO>, (unsigned)(products * per), 256, 0, st, parts, to, split, n, per));
  count_launch(1);
  return rc;
}

template <typename TO>
int launch(const DwMaps& mp, const DwArgs& ar, cudaStream_t st) {
  const int pairs = sm_count() / 2;
  if (pairs < 1) return CAPMOE_EUNSUPPORTED;
  cudaError_t err = cudaFuncSetAttribute(k_gmm_dw<TO>, cudaFuncAttributeMaxDynamicSharedMemorySize, DW_SMEM);
  if (err != cudaSuccess) return note_cuda(err);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(GMM_THREADS);
  cfg.dynamicSmemBytes = DW_SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see wait_for_previous_kernel()
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  err = cudaLaunchKernelEx(&cfg, k_gmm_dw<TO>, mp, ar);
  count_launch(1);
  return note_cuda(err);
}

// `counter`: a word to clear on the way, or NULL
int segment_maps(const BaseMaps& base, int lists, const Segments& sg, void* ws, int32_t* counter, cudaStream_t st) {
  const int rc = note_cuda(launch_chained(k_segment_maps, (unsigned)lists, GMM_MAX_E, 0, st, base, sg, (CUtensorMap*)ws, counter));
  count_launch(1);
  return rc;
}

}  // namespace

size_t gmm_dw_parts_bytes(int E, int d, int n, int products, int split) {
  return split > 1 ? (size_t)split * products * E * d * n * sizeof(float) : 0;
}
// A reduction's parts: with fewer tiles than half the pairs, as many as save most, of 8 k-blocks at least on the average of
// the allocated rows.  A k-block takes 0.27 us; joining parts takes a launch, 3 us, and writes and reads them once (6 bytes
// a nanosecond, 1000 times that a microsecond).  One expert, 2048 x 1024, two parts: 16,384 rows 81 us whole, 59 split,
// 4096 rows 26.7 and 24.9, 2048 rows 17.6 and 19.8 (not split); 3 experts of 9000 rows, 104 x 88, 16 parts: 89 and 20.
int gmm_dw_split(int64_t rows, int E, int d, int n, int products) {
  const int64_t pairs = sm_count() / 2, tiles = ceil_div(d, 256) * ceil_div(n, 256) * E * products, kbs = rows / E / BK;
  int best = 1;
  double gain = 0;
  for (int s = 2; s <= 16 && s * tiles <= pairs && kbs >= 8 * s; ++s) {
    const double g = 0.27 * (double)kbs * (s - 1) / s - 3.0 - (double)gmm_dw_parts_bytes(E, d, n, products, s) * 2 / 6e6;
    if (g > gain) { gain = g; best = s; }
  }
  return best;
}
size_t gmm_dw_map_bytes(int E, int lists) { return (size_t)lists * E * sizeof(CUtensorMap); }

int gmm_dw(const void* dy, const void* x, const Segments& sg, int d, int n, bool out_f32, void* dw, void* map_ws, float* parts,
           int split, int32_t* dev_status, int32_t* sched, cudaStream_t st) {
  DwMaps mp = {};
  DwArgs ar = {};
  BaseMaps base = {};
  if (!make_mn_map(&base.m[0], dy, n, sg.rows, 0) || !make_mn_map(&base.m[1], x, d, sg.rows, 0) ||
      !make_wide_map(&mp.o0, split > 1 ? parts : dw, d, (uint64_t)split * sg.E * n, split > 1 || out_f32 ? 4 : 2))
    return note_cuda(cudaErrorInvalidValue);
  int rc = segment_maps(base, 2, sg, map_ws, sched, st);
  if (rc != CAPMOE_OK) return rc;
  ar.sg = sg; ar.split = split; ar.out[0] = split > 1 ? parts : dw; ar.count = 1; ar.M[0] = n; ar.N[0] = d; ar.ia[0] = 0; ar.ib[0] = 1;
  ar.wide_a = mn_wide(n); ar.wide_b = mn_wide(d);
  ar.maps = (const CUtensorMap*)map_ws; ar.dev_status = dev_status; ar.sched = sched;
  if (split == 1) return out_f32 ? launch<float>(mp, ar, st) : launch<__nv_bfloat16>(mp, ar, st);
  if ((rc = launch<float>(mp, ar, st)) != CAPMOE_OK) return rc;
  const int64_t size = (int64_t)sg.E * n * d;
  if (out_f32) return join_parts<float>(parts, 1, {{(float*)dw}}, split, size, st);
  return join_parts<__nv_bfloat16>(parts, 1, {{(__nv_bfloat16*)dw}}, split, size, st);
}

int gmm_dw_ffn_maps(const void* dg, const void* du, const void* dy, const void* x, const void* h, const Segments& sg, int d, int F,
                    void* map_ws, cudaStream_t st) {
  BaseMaps base = {};
  const int64_t R = sg.rows;
  if (!make_mn_map(&base.m[0], dg, F, R, 0) || !make_mn_map(&base.m[1], du, F, R, 0) || !make_mn_map(&base.m[2], dy, d, R, 0) ||
      !make_mn_map(&base.m[3], x, d, R, 0) || !make_mn_map(&base.m[4], h, F, R, 0))
    return note_cuda(cudaErrorInvalidValue);
  return segment_maps(base, MAP_LISTS, sg, map_ws, nullptr, st);
}

int gmm_dw_ffn(const Segments& sg, int d, int F, void* dwg, void* dwu, void* dwd, const void* map_ws, float* parts, int split,
               int32_t* dev_status, int32_t* sched, cudaStream_t st) {
  DwMaps mp = {};
  DwArgs ar = {};
  const int64_t size = (int64_t)sg.E * F * d, step = split * size;
  const bool f = split > 1;
  void *o0 = f ? parts : dwg, *o1 = f ? parts + step : dwu, *o2 = f ? parts + 2 * step : dwd;
  const uint64_t mats = (uint64_t)split * sg.E;
  const int elt = f ? 4 : 2;
  if (!make_wide_map(&mp.o0, o0, d, mats * F, elt) || !make_wide_map(&mp.o1, o1, d, mats * F, elt) ||
      !make_wide_map(&mp.o2, o2, F, mats * d, elt))
    return note_cuda(cudaErrorInvalidValue);
  ar.sg = sg; ar.count = 3; ar.split = split;
  ar.out[0] = o0; ar.out[1] = o1; ar.out[2] = o2;
  ar.M[0] = ar.M[1] = F; ar.M[2] = d;
  ar.N[0] = ar.N[1] = d; ar.N[2] = F;
  ar.ia[0] = 0; ar.ia[1] = 1; ar.ia[2] = 2;
  ar.ib[0] = ar.ib[1] = 3; ar.ib[2] = 4;
  ar.wide_a = (mn_wide(F) ? 3 : 0) | (mn_wide(d) ? 4 : 0);
  ar.wide_b = (mn_wide(d) ? 3 : 0) | (mn_wide(F) ? 4 : 0);
  ar.maps = (const CUtensorMap*)map_ws; ar.dev_status = dev_status; ar.sched = sched;
  if (!f) return launch<__nv_bfloat16>(mp, ar, st);
  const int rc = launch<float>(mp, ar, st);
  if (rc != CAPMOE_OK) return rc;
  using B = __nv_bfloat16;
  return join_parts<B>(parts, 3, {{(B*)dwg, (B*)dwu, (B*)dwd}}, split, size, st);
}

}  // namespace capmoe
