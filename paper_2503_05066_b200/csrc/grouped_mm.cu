// Grouped products of expert-major rows with per-expert weights, and their gradients: host side, and the
// plain-FMA kernels for fp32 storage and for sizes the tensor-core kernels do not take.
//   forward    y[r]   = W[e] x[r]
//   dx         dx[r]  = W[e]^T dy[r]
//   dw         dW[e]  = sum over the rows r of expert e of dy[r] x[r]^T
//   backward of the SwiGLU FFN: g = W_g x, u = W_u x, dh = W_d^T dy, p = sigmoid(g), then
//              dg = dh u p (1 + g (1 - p)), du = dh g p, h = g p u and the products of those with x, dy and
//              the weights.
// All sums are fp32; one rounding to the storage type at each stored matrix.
#include "gmm_simt.cuh"

namespace capmoe {
namespace {

enum { DIR_FWD = 0, DIR_DX = 1 };

template <typename T, int DIR, class GE>
__global__ void __launch_bounds__(GE::SN, GE::BLOCKS)
k_mm_rows(const T* __restrict__ A, const T* __restrict__ W, T* __restrict__ out, Segments sg, int K, int Nout) {
  wait_for_previous_kernel();
  SimtTile<GE>& sm = simt_tile<GE>();
  RowTile t;
  if (!find_row_tile<GE>(sg, blockIdx.x, t)) return;
  const int col0 = blockIdx.y * GE::TN;
  const T* We = W + (int64_t)t.e * Nout * K;
  constexpr int R = GE::R;
  const Share k = share_of(K);
  float acc[1][R][GE::C];
  clear_acc(acc[0]);
  const Dense<T, true> la{A + (int64_t)t.row0 * K + k.k0, K};
  if (DIR == DIR_FWD) tile_product<GE>(la, Dense<T, true>{We + (int64_t)col0 * K + k.k0, K}, t.rows, Nout - col0, k.len, sm, acc[0]);
  else tile_product<GE>(la, Dense<T, false>{We + (int64_t)k.k0 * Nout + col0, Nout}, t.rows, Nout - col0, k.len, sm, acc[0]);
  if (!join_shares(sm, acc)) return;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < GE::C; ++j) {
      const int r = out_row<GE>(i), c = col0 + out_col<GE>(j);
      if (r < t.rows && c < Nout) out[(int64_t)(t.row0 + r) * Nout + c] = from_float<T>(acc[0][i][j]);
    }
}

// Up to three weight gradients of one set of segments in one launch (blockIdx.z = product * E + expert):
// product p is P[p]^T Q[p] with P [rows, M[p]] and Q [rows, N[p]].
template <typename T, typename TO>
struct DwSet { const T* P[3]; const T* Q[3]; TO* out[3]; int M[3], N[3]; };

// Experts with up to DW_DIRECT rows: outer products straight from global memory, without staging and partial tiles (64
// experts, 512 x 512, fp32: 34 us with 1 row, 43 with 4, 58 with 8, 79 with 12; staged 60, 60, 61, 62).
constexpr int DW_DIRECT = 8;
template <typename T, typename TO, class GE>
__global__ void __launch_bounds__(GE::SN, GE::BLOCKS) k_mm_dw(DwSet<T, TO> s, Segments sg) {
  wait_for_previous_kernel();
  SimtTile<GE>& sm = simt_tile<GE>();
  const int p = blockIdx.z / sg.E, e = blockIdx.z - p * sg.E;
  const int M = s.M[p], N = s.N[p];
  const int r0 = blockIdx.x * GE::TM, c0 = blockIdx.y * GE::TN;
  if (r0 >= M || c0 >= N) return;
  const int begin = seg_at(sg, e), n = seg_at(sg, e + 1) - begin;
  constexpr int R = GE::R;
  float acc[R][GE::C];
  clear_acc(acc);
  const Dense<T, false> P{s.P[p] + (int64_t)begin * M + r0, M}, Q{s.Q[p] + (int64_t)begin * N + c0, N};
  if (n <= DW_DIRECT) {
    for (int k = 0; k < n; ++k) {
      float a[R], b[GE::C];
#pragma unroll
      for (int i = 0; i < R; ++i) a[i] = r0 + out_row<GE>(i) < M ? P.at(out_row<GE>(i), k) : 0.f;
#pragma unroll
      for (int j = 0; j < GE::C; ++j) b[j] = c0 + out_col<GE>(j) < N ? Q.at(out_col<GE>(j), k) : 0.f;
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < GE::C; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
    }
  } else {
    tile_product<GE>(P, Q, M - r0, N - c0, n, sm, acc);
  }
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < GE::C; ++j) {
      const int r = r0 + out_row<GE>(i), c = c0 + out_col<GE>(j);
      if (r < M && c < N) s.out[p][((int64_t)e * M + r) * N + c] = from_float<TO>(acc[i][j]);
    }
}

// dg, du and h of the SwiGLU backward pass: three products over d with the elementwise part in registers.
template <typename T, class GE>
__global__ void __launch_bounds__(GE::SN, GE::BLOCKS)
k_ffn_grad_hidden(const T* __restrict__ x, const T* __restrict__ dy, const T* __restrict__ wg, const T* __restrict__ wu,
                  const T* __restrict__ wd, T* __restrict__ dg, T* __restrict__ du, T* __restrict__ h, Segments sg, int d,
                  int F) {
  wait_for_previous_kernel();
  SimtTile<GE>& sm = simt_tile<GE>();
  RowTile t;
  if (!find_row_tile<GE>(sg, blockIdx.x, t)) return;
  const int col0 = blockIdx.y * GE::TN, cols = F - col0;
  const int64_t we = (int64_t)t.e * F * d;
  const Share k = share_of(d);
  const int64_t at = (int64_t)t.row0 * d + k.k0, wat = we + (int64_t)col0 * d + k.k0;
  constexpr int R = GE::R;
  float acc[3][R][GE::C];                               // g, u, dh
  clear_acc(acc[0]); clear_acc(acc[1]); clear_acc(acc[2]);
  tile_product<GE>(Dense<T, true>{x + at, d}, Dense<T, true>{wg + wat, d}, t.rows, cols, k.len, sm, acc[0]);
  tile_product<GE>(Dense<T, true>{x + at, d}, Dense<T, true>{wu + wat, d}, t.rows, cols, k.len, sm, acc[1]);
  tile_product<GE>(Dense<T, true>{dy + at, d}, Dense<T, false>{wd + we + (int64_t)k.k0 * F + col0, F}, t.rows, cols, k.len, sm, acc[2]);
  if (!join_shares(sm, acc)) return;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < GE::C; ++j) {
      const int r = out_row<GE>(i), c = col0 + out_col<GE>(j);
      if (r >= t.rows || c >= F) continue;
      const float gv = acc[0][i][j], uv = acc[1][i][j], dhv = acc[2][i][j];
      const float p = 1.0f / (1.0f + expf(-gv));
      const float a = gv * p;
      const int64_t o = (int64_t)(t.row0 + r) * F + c;
      dg[o] = from_float<T>(dhv * uv * (p + a * (1.0f - p)));
      du[o] = from_float<T>(dhv * a);
      h[o] = from_float<T>(a * uv);
    }
}

// dx = dg W_g + du W_u (weights [E, F, d])
template <typename T, class GE>
__global__ void __launch_bounds__(GE::SN, GE::BLOCKS)
k_ffn_grad_x(const T* __restrict__ dg, const T* __restrict__ du, const T* __restrict__ wg, const T* __restrict__ wu,
             T* __restrict__ dx, Segments sg, int d, int F) {
  wait_for_previous_kernel();
  SimtTile<GE>& sm = simt_tile<GE>();
  RowTile t;
  if (!find_row_tile<GE>(sg, blockIdx.x, t)) return;
  const int col0 = blockIdx.y * GE::TN;
  const Share k = share_of(F);
  const int64_t at = (int64_t)t.row0 * F + k.k0, we = (int64_t)t.e * F * d + (int64_t)k.k0 * d + col0;
  constexpr int R = GE::R;
  float acc[1][R][GE::C];
  clear_acc(acc[0]);
  tile_product<GE>(Dense<T, true>{dg + at, F}, Dense<T, false>{wg + we, d}, t.rows, d - col0, k.len, sm, acc[0]);
  tile_product<GE>(Dense<T, true>{du + at, F}, Dense<T, false>{wu + we, d}, t.rows, d - col0, k.len, sm, acc[0]);
  if (!join_shares(sm, acc)) return;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < GE::C; ++j) {
      const int r = out_row<GE>(i), c = col0 + out_col<GE>(j);
      if (r < t.rows && c < d) dx[(int64_t)(t.row0 + r) * d + c] = from_float<T>(acc[0][i][j]);
    }
}

int launched(cudaError_t err) {
  count_launch(1);
  return note_cuda(err);
}

// These kernels do not let their successor start early (no allow_next_kernel): its blocks would be handed to the SMs
// that happen to have room, several to each, and stay there (a 1024-row fp32 product of 120 blocks, launched back to
// back: 63 us that way, 25 without); letting it start when the sums are done changes nothing.
template <class GE, class... KArgs, class... Args>
int launch_tiles(void (*kernel)(KArgs...), dim3 grid, int split, cudaStream_t st, Args... args) {
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SimtTile<GE>));
  if (err != cudaSuccess) return note_cuda(err);
  cudaLaunchConfig_t cfg = {};
  cfg.dynamicSmemBytes = sizeof(SimtTile<GE>);
  cfg.gridDim = grid;
  cfg.blockDim = dim3(GE::SN);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;           // the blocks that share a reduction
  attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = (unsigned)split;
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 2 : 1;
  return launched(cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...));
}

template <class GE>
dim3 row_grid(const Segments& sg, int cols, int split) {       // every segment rounds up to whole tiles
  return dim3((unsigned)(ceil_div(sg.rows, GE::TM) + sg.E), (unsigned)ceil_div(cols, GE::TN), (unsigned)split);
}
// Geometry by the number of tiles.  128 x 128 tiles when BIG_MIN whole ones per SM exist and the segments fill them (16,305
// rows of 8 experts, 1000 x 1024: y 870 us, dx 885, with 64 x 64 tiles 1070 and 1111; 2919 rows of 8, 848 x 862, with 1 or 2
// per SM: 215 us against 145).  From `large` 64 x 64 ones per SM on, those; else 32-row ones, whose block gets an SM to
// itself when they do not outnumber the SMs (see gmm_simt.cuh; FFN gradients of 236 rows of 45 experts, 41 x 415: 74 us
// with two blocks to an SM, 90 with one).
enum Size { BIG, LARGE, MEDIUM, SMALL };
Size size_of(int64_t tiles64, int64_t tiles32, int large = 2) {
  return tiles64 >= large * sm_count() ? LARGE : tiles32 > sm_count() ? MEDIUM : SMALL;
}
// Row products: the number of 32-row tiles, taking three quarters of the segments that can have rows to have some, each
// ending in half a tile; and, while those would leave half of the SMs without one, into how many parts of at least
// SPLIT_MIN steps the reduction is split.
struct Plan { Size size; int split; };
constexpr int SPLIT_MIN = 32;
constexpr int BIG_MIN = 2;
Plan plan_rows(const Segments& sg, int cols, int K) {
  const int64_t used = ((sg.E < sg.rows ? sg.E : sg.rows) * 3 + 3) / 4, nc = ceil_div(cols, ST);
  const int64_t t32 = ceil_div(sg.rows, 32) + used / 2, tiles32 = (t32 > used ? t32 : used) * nc;
  Plan p = {size_of(ceil_div(sg.rows, ST) * nc, tiles32), 1};
  if (sg.rows / sg.E >= 128 && (int64_t)(sg.rows / 128) * (cols / 128) >= BIG_MIN * sm_count()) p.size = BIG;
  if (p.size == SMALL)
    while (p.split < 8 && tiles32 * p.split * 2 <= sm_count() && K >= p.split * 2 * SPLIT_MIN) p.split *= 2;
  return p;
}
using Big = Geo<128, 1, 128>;
using Large = Geo<64, 4>;
using Medium = Geo<32, 4>;
using Small = Geo<32, 8>;

template <typename T, int DIR, class GE>
int rows_run(const T* a, const T* w, T* out, const Segments& sg, int K, int Nout, int split, cudaStream_t st) {
  return launch_tiles<GE>(k_mm_rows<T, DIR, GE>, row_grid<GE>(sg, Nout, split), split, st, a, w, out, sg, K, Nout);
}
template <typename T, int DIR>
int rows_simt(const void* a, const void* w, void* out, const Segments& sg, int K, int Nout, cudaStream_t st) {
  const Plan p = plan_rows(sg, Nout, K);
  auto run = p.size == BIG ? rows_run<T, DIR, Big> : p.size == LARGE ? rows_run<T, DIR, Large> : p.size == MEDIUM ? rows_run<T, DIR, Medium> : rows_run<T, DIR, Small>;
  return run((const T*)a, (const T*)w, (T*)out, sg, K, Nout, p.split, st);
}

template <typename T, typename TO, class GE>
int dw_run(const DwSet<T, TO>& s, int M, int N, unsigned z, const Segments& sg, cudaStream_t st) {
  return launch_tiles<GE>(k_mm_dw<T, TO, GE>, dim3((unsigned)ceil_div(M, GE::TM), (unsigned)ceil_div(N, GE::TN), z), 1, st, s, sg);
}
template <typename T, typename TO>
int dw_simt(const DwSet<T, TO>& s, int count, const Segments& sg, cudaStream_t st) {
  int M = 0, N = 0;
  int64_t tiles = 0, big = 0;
  for (int p = 0; p < count; ++p) {
    M = s.M[p] > M ? s.M[p] : M;
    N = s.N[p] > N ? s.N[p] : N;
    tiles += ceil_div(s.M[p], ST) * ceil_div(s.N[p], ST) * sg.E;
    big += (int64_t)(s.M[p] / 128) * (s.N[p] / 128) * sg.E;
  }
  // short sums: 64-row tiles from one per SM on (871 rows of 8 experts, 512 x 256: 12.5 us, 14.3 with 32-row tiles)
  Size z = size_of(tiles, 2 * tiles, 1);
  if (sg.rows / sg.E >= 64 && big >= BIG_MIN * sm_count()) z = BIG;
  auto run = z == BIG ? dw_run<T, TO, Big> : z == LARGE ? dw_run<T, TO, Large> : z == MEDIUM ? dw_run<T, TO, Medium> : dw_run<T, TO, Small>;
  return run(s, M, N, (unsigned)(count * sg.E), sg, st);
}

template <typename T, class GE>
int hidden_run(const T* x, const T* dy, const T* wg, const T* wu, const T* wd, T* dg, T* du, T* h, const Segments& sg, int d, int F,
               int split, cudaStream_t st) {
  return launch_tiles<GE>(k_ffn_grad_hidden<T, GE>, row_grid<GE>(sg, F, split), split, st, x, dy, wg, wu, wd, dg, du, h, sg, d, F);
}
template <typename T, class GE>
int dx2_run(const T* dg, const T* du, const T* wg, const T* wu, T* dx, const Segments& sg, int d, int F, int split,
            cudaStream_t st) {
  return launch_tiles<GE>(k_ffn_grad_x<T, GE>, row_grid<GE>(sg, d, split), split, st, dg, du, wg, wu, dx, sg, d, F);
}
template <typename T>
int ffn_grad_simt(const void* x, const void* dy, const Segments& sg, int d, int F, const void* w_gate, const void* w_up,
                  const void* w_down, void* dx, void* dwg, void* dwu, void* dwd, void* ws, cudaStream_t st) {
  T* dg = (T*)ws;
  T* du = dg + (int64_t)sg.rows * F;
  T* h = du + (int64_t)sg.rows * F;
  const T *wg = (const T*)w_gate, *wu = (const T*)w_up, *wd = (const T*)w_down;
  const Plan ph = plan_rows(sg, F, d), px = plan_rows(sg, d, F);
  auto hidden = ph.size <= LARGE ? hidden_run<T, Large> : ph.size == MEDIUM ? hidden_run<T, Medium> : hidden_run<T, Small>;
  auto dx2 = px.size == BIG ? dx2_run<T, Big> : px.size == LARGE ? dx2_run<T, Large> : px.size == MEDIUM ? dx2_run<T, Medium> : dx2_run<T, Small>;
  int rc = hidden((const T*)x, (const T*)dy, wg, wu, wd, dg, du, h, sg, d, F, ph.split, st);
  if (rc == CAPMOE_OK) rc = dx2(dg, du, wg, wu, (T*)dx, sg, d, F, px.split, st);
  if (rc != CAPMOE_OK) return rc;
  DwSet<T, T> s = {{dg, du, (const T*)dy}, {(const T*)x, (const T*)x, h}, {(T*)dwg, (T*)dwu, (T*)dwd}, {F, F, d}, {d, d, F}};
  return dw_simt(s, 3, sg, st);
}

// Checks common to the grouped products.  CAPMOE_OK, or the status to return before anything is enqueued.
int check_shape(const int32_t* offsets, int E, int d, int n, int dtype, int64_t rows) {
  if (E < 1 || d < 1 || n < 1 || rows < 0 || !offsets) return CAPMOE_EINVAL;
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  if (E > GMM_MAX_E || rows > GMM_MAX_ROWS || ceil_div(d, ST) > 65535 || ceil_div(n, ST) > 65535)
    return CAPMOE_EUNSUPPORTED;
  return CAPMOE_OK;
}
size_t align256(size_t b) { return (b + 255) / 256 * 256; }
void* align256(void* p) { return (void*)align256((size_t)p); }
// Parts of the weight gradients' reductions: all that pay when the workspace has room for them behind `parts`, else one.
int split_that_fits(int64_t rows, int E, int d, int n, int products, const uint8_t* parts, const void* ws, size_t ws_bytes) {
  const int split = gmm_dw_split(rows, E, d, n, products);
  const size_t before = (size_t)(parts - (const uint8_t*)ws);
  return before <= ws_bytes && gmm_dw_parts_bytes(E, d, n, products, split) <= ws_bytes - before ? split : 1;
}

}  // namespace
}  // namespace capmoe

using namespace capmoe;

extern "C" int capmoe_grouped_mm(const void* x_rows, const int32_t* expert_offsets, const void* w, int E, int d, int n,
                                 int dtype, void* y, int64_t rows, int32_t* dev_status, void* stream) {
  int rc = check_shape(expert_offsets, E, d, n, dtype, rows);
  if (rc != CAPMOE_OK || rows == 0) return rc;
  if (!usable(x_rows, w, y)) return CAPMOE_EINVAL;
  const Segments sg{expert_offsets, E, (int)rows};
  if (gmm_supported(E, d, n, dtype)) {
    int32_t* counters = counters_of(sg, dev_status);
    if ((rc = begin_counters(counters, 1, as_stream(stream))) != CAPMOE_OK) return rc;
    return gmm_fwd(x_rows, sg, w, d, n, y, dev_status, counter_at(counters, 0), false, as_stream(stream));
  }
  if (dtype == CAPMOE_F32) return rows_simt<float, DIR_FWD>(x_rows, w, y, sg, d, n, as_stream(stream));
  return rows_simt<__nv_bfloat16, DIR_FWD>(x_rows, w, y, sg, d, n, as_stream(stream));
}

extern "C" int capmoe_grouped_mm_dx(const void* dy_rows, const int32_t* expert_offsets, const void* w, int E, int d, int n,
                                    int dtype, void* dx, int64_t rows, int32_t* dev_status, void* stream) {
  int rc = check_shape(expert_offsets, E, d, n, dtype, rows);
  if (rc != CAPMOE_OK || rows == 0) return rc;
  if (!usable(dy_rows, w, dx)) return CAPMOE_EINVAL;
  const Segments sg{expert_offsets, E, (int)rows};
  if (gmm_supported(E, d, n, dtype)) {
    int32_t* counters = counters_of(sg, dev_status);
    if ((rc = begin_counters(counters, 1, as_stream(stream))) != CAPMOE_OK) return rc;
    return gmm_dx(dy_rows, sg, w, d, n, dx, dev_status, counter_at(counters, 0), false, as_stream(stream));
  }
  if (dtype == CAPMOE_F32) return rows_simt<float, DIR_DX>(dy_rows, w, dx, sg, n, d, as_stream(stream));
  return rows_simt<__nv_bfloat16, DIR_DX>(dy_rows, w, dx, sg, n, d, as_stream(stream));
}

extern "C" int capmoe_grouped_mm_dw_workspace_bytes(int E, size_t* bytes) {
  if (!bytes || E < 1) return CAPMOE_EINVAL;
  *bytes = gmm_dw_map_bytes(E, 2) + 256;                     // 256: to align the maps
  return CAPMOE_OK;
}

extern "C" int capmoe_grouped_mm_dw(const void* dy_rows, const void* x_rows, const int32_t* expert_offsets, int E, int d,
                                    int n, int dtype, int out_dtype, void* dw, int64_t rows, void* ws, size_t ws_bytes,
                                    int32_t* dev_status, void* stream) {
  int rc = check_shape(expert_offsets, E, d, n, dtype, rows);
  if (rc != CAPMOE_OK) return rc;
  if (out_dtype != CAPMOE_F32 && out_dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  if (dtype == CAPMOE_F32 && out_dtype != CAPMOE_F32) return CAPMOE_EUNSUPPORTED;
  if (!usable(dw)) return CAPMOE_EINVAL;
  if (rows == 0) return note_cuda(cudaMemsetAsync(dw, 0, (size_t)E * n * d * elt_size(out_dtype), as_stream(stream)));
  if (!usable(dy_rows, x_rows, ws)) return CAPMOE_EINVAL;
  size_t need = 0;
  capmoe_grouped_mm_dw_workspace_bytes(E, &need);
  if (ws_bytes < need) return CAPMOE_EWORKSPACE;
  const Segments sg{expert_offsets, E, (int)rows};
  cudaStream_t st = as_stream(stream);
  if (gmm_supported(E, d, n, dtype)) {
    uint8_t* maps = (uint8_t*)align256(ws);
    uint8_t* parts = maps + align256(gmm_dw_map_bytes(E, 2));
    return gmm_dw(dy_rows, x_rows, sg, d, n, out_dtype == CAPMOE_F32, dw, maps, (float*)parts,
                  split_that_fits(rows, E, d, n, 1, parts, ws, ws_bytes), dev_status, counter_at(dev_status, 0), st);
  }
  if (dtype == CAPMOE_F32)
    return dw_simt(DwSet<float, float>{{(const float*)dy_rows}, {(const float*)x_rows}, {(float*)dw}, {n}, {d}}, 1, sg, st);
  using B = __nv_bfloat16;
  if (out_dtype == CAPMOE_F32)
    return dw_simt(DwSet<B, float>{{(const B*)dy_rows}, {(const B*)x_rows}, {(float*)dw}, {n}, {d}}, 1, sg, st);
  return dw_simt(DwSet<B, B>{{(const B*)dy_rows}, {(const B*)x_rows}, {(B*)dw}, {n}, {d}}, 1, sg, st);
}

extern "C" int capmoe_dw_split_bytes(int64_t rows, int E, int d, int n, int dtype, int products, size_t* bytes) {
  if (!bytes || rows < 0 || E < 1 || d < 1 || n < 1 || products < 1 || products > 3) return CAPMOE_EINVAL;
  const int split = gmm_supported(E, d, n, dtype) ? gmm_dw_split(rows, E, d, n, products) : 1;
  *bytes = split > 1 ? gmm_dw_parts_bytes(E, d, n, products, split) + 512 : 0;    // 512: to align the parts
  return CAPMOE_OK;
}

extern "C" int capmoe_ffn_backward_workspace_bytes(int64_t A_max, int E, int F, int dtype, size_t* bytes) {
  if (!bytes || A_max < 0 || E < 1 || F < 1) return CAPMOE_EINVAL;
  if (dtype != CAPMOE_F32 && dtype != CAPMOE_BF16) return CAPMOE_EUNSUPPORTED;
  *bytes = (size_t)A_max * (size_t)F * elt_size(dtype) * 3 + align256(gmm_dw_map_bytes(E, 5)) + 256;
  return CAPMOE_OK;
}

extern "C" int capmoe_grouped_ffn_backward(const void* x_perm, const void* dy_perm, const int32_t* expert_offsets, int E,
                                           int d, int F, int dtype, const void* w_gate, const void* w_up,
                                           const void* w_down, void* dx_perm, void* dw_gate, void* dw_up, void* dw_down,
                                           int64_t A_max, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream) {
  int rc = check_shape(expert_offsets, E, d, F, dtype, A_max);
  if (rc != CAPMOE_OK) return rc;
  if (!usable(dw_gate, dw_up, dw_down)) return CAPMOE_EINVAL;
  cudaStream_t st = as_stream(stream);
  if (A_max == 0) {
    for (void* dw : {dw_gate, dw_up, dw_down})
      if ((rc = note_cuda(cudaMemsetAsync(dw, 0, (size_t)E * F * d * elt_size(dtype), st))) != CAPMOE_OK) return rc;
    return CAPMOE_OK;
  }
  if (!usable(x_perm, dy_perm, w_gate, w_up, w_down, dx_perm, ws)) return CAPMOE_EINVAL;
  size_t need = 0;
  capmoe_ffn_backward_workspace_bytes(A_max, E, F, dtype, &need);
  if (ws_bytes < need) return CAPMOE_EWORKSPACE;
  const Segments sg{expert_offsets, E, (int)A_max};
  if (gmm_supported(E, d, F, dtype)) {
    uint8_t* maps = (uint8_t*)align256(ws);
    __nv_bfloat16* dg = (__nv_bfloat16*)(maps + align256(gmm_dw_map_bytes(E, 5)));
    __nv_bfloat16 *du = dg + A_max * F, *h = du + A_max * F;
    rc = begin_counters(dev_status, 3, st);
    if (rc == CAPMOE_OK) rc = gmm_dw_ffn_maps(dg, du, dy_perm, x_perm, h, sg, d, F, maps, st);
    if (rc == CAPMOE_OK)
      rc = gmm_hidden(x_perm, dy_perm, sg, d, F, w_gate, w_up, w_down, dg, du, h, dev_status, counter_at(dev_status, 0), true, st);
    if (rc == CAPMOE_OK) rc = gmm_dx2(dg, du, sg, d, F, w_gate, w_up, dx_perm, dev_status, counter_at(dev_status, 1), true, st);
    if (rc != CAPMOE_OK) return rc;
    uint8_t* parts = (uint8_t*)align256(h + A_max * F);
    return gmm_dw_ffn(sg, d, F, dw_gate, dw_up, dw_down, maps, (float*)parts,
                      split_that_fits(A_max, E, d, F, 3, parts, ws, ws_bytes), dev_status, counter_at(dev_status, 2), st);
  }
  if (dtype == CAPMOE_F32)
    return ffn_grad_simt<float>(x_perm, dy_perm, sg, d, F, w_gate, w_up, w_down, dx_perm, dw_gate, dw_up, dw_down, ws, st);
  return ffn_grad_simt<__nv_bfloat16>(x_perm, dy_perm, sg, d, F, w_gate, w_up, w_down, dx_perm, dw_gate, dw_up, dw_down, ws,
                                      st);
}
