// Products of rows ordered by type (see grouped.h): entry points, the choice of tiles, and the sum of the parts of a
// group whose rows were cut.
#include "grouped.h"

namespace sagnn {
namespace {

// dW[g] = the sum of its parts, chunks ascending, in 64 bits (there may be thousands); a group of one part was written by the product itself.
__global__ __launch_bounds__(256) void grouped_join_kernel(const GroupedArgs a, bool four) {
  const int32_t g = blockIdx.y;
  const int64_t lo = grouped_row(a.off, g, a.m), hi = grouped_row(a.off, g + 1, a.m), size = (int64_t)a.kdim * a.nout;
  if (hi <= lo) return;
  const int64_t c0 = lo / a.chunk, c1 = (hi - 1) / a.chunk;
  if (c0 == c1) return;
  if (four) {                                 // (a multiple of four, and aligned so)
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (int64_t)gridDim.x * 1024) {
      const float4 head = *reinterpret_cast<const float4*>(a.partial + (2 * c0 + 1) * size + i);
      double sum[4] = {head.x, head.y, head.z, head.w};
#pragma unroll 4
      for (int64_t c = c0 + 1; c <= c1; ++c) {
        const float4 x = *reinterpret_cast<const float4*>(a.partial + 2 * c * size + i);
        sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
      }
      *reinterpret_cast<float4*>(a.dW + g * size + i) = make_float4((float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]);
    }
    return;
  }
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += (int64_t)gridDim.x * 256) {
    double sum = a.partial[(2 * c0 + 1) * size + i];
#pragma unroll 8
    for (int64_t c = c0 + 1; c <= c1; ++c) sum += a.partial[2 * c * size + i];
    a.dW[g * size + i] = (float)sum;
  }
}

bool valid(int32_t dtype, int32_t prec, int64_t m, int32_t groups, int32_t kdim, int32_t nout) {
  return (dtype == SAGNN_F32 || (dtype == SAGNN_BF16 && prec == SAGNN_GEMM_FP32)) && prec >= SAGNN_GEMM_FP32 && prec <= SAGNN_GEMM_FP32_BF16X3 &&
         m >= 0 && m <= INT32_MAX && groups >= 1 && groups <= SAGNN_GROUPED_MAX && kdim >= 1 && kdim <= SAGNN_GROUPED_MAX_WIDTH &&
         nout >= 1 && nout <= SAGNN_GROUPED_MAX_WIDTH;
}
bool element_aligned(const void* p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == SAGNN_BF16 ? 1u : 3u)) == 0; }

// Whether the kernels that load into LDS directly take an operand: rows of whole granules, offsets inside a tile below 2^31
bool direct_rows(const void* p, int64_t ld, int64_t width) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 && width % 8 == 0 && ld <= (1 << 20);
}

constexpr int64_t kStagedLd = 1 << 20;     // (offsets inside a tile of 256 rows below 2^31)

// Which tiles an operation can have: through registers any (staged: fp32 tensors), straight into LDS bfloat16 ones
enum { kAny = 0, kDirect = 1, kStaged = 2 };

// What a tile costs: how well it feeds the matrix cores (rates of 8192 x 4096 x 4096, 128 x 128 = 1), and how much of the summed index its
// beginning and end are worth.  Small tiles are several to a CU, which hides both; the large ones are alone there.
struct TileCost { double rate, ends; };
TileCost tile_cost(int32_t dtype, int32_t prec, int tile) {
  static constexpr TileCost fp32[kGroupedTiles] = {{1., 48}, {.98, 24}, {.91, 12}, {.95, 8}, {.85, 16}, {0, 0}, {0, 0}, {0, 0}, {.78, 200}};
  static constexpr TileCost rounded[kGroupedTiles] = {{1., 128}, {.76, 128}, {.62, 32}, {.49, 8}, {.25, 16}, {0, 0}, {1.08, 160}, {1.08, 160}, {.18, 200}};
  static constexpr TileCost split[kGroupedTiles] = {{1., 48}, {.87, 24}, {.67, 8}, {.76, 8}, {.65, 8}, {0, 0}, {1.18, 54}, {1.18, 54}, {.46, 200}};
  static constexpr TileCost bf16[kGroupedTiles] = {{1., 128}, {.81, 128}, {.66, 32}, {.66, 32}, {.39, 32}, {1.69, 200}, {0, 0}, {0, 0}, {.26, 200}};
  return dtype == SAGNN_BF16 ? bf16[tile] : prec == SAGNN_GEMM_FP32 ? fp32[tile] : prec == SAGNN_GEMM_BF16 ? rounded[tile] : split[tile];
}

// The tile with the least cost: `rows` rows in `parts` ragged parts by `cols` columns, `times` over, `sum` of the summed index.  Tiles are
// whole, so each part leaves half a tile empty; a launch lasts as long as its fullest CU; and a tile alone on a CU waits for its
// loads.  `whole`: a product of rows.  Bfloat16 results are no place for the sum of several runs, which the largest tile and the thin one would
// need.
int choose_tile(int32_t dtype, int32_t prec, int ways, int64_t rows, int64_t parts, int64_t cols, int64_t times, int64_t sum, bool whole) {
  int best = kTile128;
  double least = 1e300;
  for (int tile = 0; tile < kGroupedTiles; ++tile) {
    const TileCost c = tile_cost(dtype, prec, tile);
    if (c.rate == 0 || (tile == kDirect256 && !(ways & kDirect)) || ((tile == kStaged256x128 || tile == kStaged128x256) && !(ways & kStaged))) continue;
    if (tile == kThin && !whole) continue;
    if (whole && dtype == SAGNN_BF16 && ((tile == kDirect256 && sum > kRunRounded) || (tile == kThin && sum > 8 * kRunBf16))) continue;
    const int64_t h = grouped_tile_rows(tile), w = grouped_tile_cols(tile);
    const int64_t tiles = (ceil_div(rows, h) + (parts < rows ? parts : rows) / 2) * ceil_div(cols, w) * times;
    const double turns = tiles <= 256 ? 1.25 : whole && tiles < 4 * 256 ? (double)ceil_div(tiles, 256) : tiles / 256.;
    const double cost = turns * h * w * (sum + c.ends) / c.rate;
    if (cost < least) {
      least = cost;
      best = tile;
    }
  }
  return best;
}

// Tile and workgroups of the product (fills in a's tiles); < 0 workgroups: more than a launch has
struct Launch { int tile; int64_t blocks; };
Launch plan_rows(GroupedArgs& a, int32_t dtype, int32_t prec) {
  int ways = kAny;
  if (dtype == SAGNN_BF16) {
    if (direct_rows(a.X, a.ldx, a.kdim) && direct_rows(a.W, a.ldw, a.nout) && a.stride_w % 8 == 0 && direct_rows(a.Y, a.ldy, 0) &&
        (!a.mask || direct_rows(a.mask, a.ldmask, 0)))
      ways = kDirect;
  } else if (a.ldx <= kStagedLd && a.ldw <= kStagedLd) {
    ways = kStaged;
  }
  const int tile = choose_tile(dtype, prec, ways, a.m, a.groups, a.nout, 1, a.kdim, true);
  a.run = grouped_run(dtype == SAGNN_BF16 ? SAGNN_GEMM_BF16 : prec, tile == kThin ? ceil_div(a.kdim, 8) : a.kdim);
  a.row_tiles = (int32_t)(a.m / grouped_tile_rows(tile) + a.groups + 1);
  a.col_tiles = (int32_t)ceil_div(a.nout, grouped_tile_cols(tile));
  const int64_t blocks = (int64_t)a.row_tiles * a.col_tiles;
  return {tile, blocks <= INT32_MAX ? blocks : -1};
}

int launch_rows(const GroupedArgs& a, Launch l, int32_t dtype, int32_t prec, bool trans_w, hipStream_t s) {
  if (dtype == SAGNN_BF16) return grouped_bf16(a, l.tile, trans_w, l.blocks, s);
  return prec == SAGNN_GEMM_FP32 ? grouped_fp32(a, l.tile, trans_w, l.blocks, s)
         : prec == SAGNN_GEMM_BF16 ? grouped_fp32_bf16(a, l.tile, trans_w, l.blocks, s)
                                   : grouped_fp32_bf16x3(a, l.tile, trans_w, l.blocks, s);
}

// The weight gradient's tiles and chunks of rows.  Chunks fill the chip where the matrices are small or one group has most rows (170003 x 128 x 128
// in 4 groups, three terms: 83 chunks 95 us, 256 chunks 62); but a group that a chunk's end cuts costs its matrix written twice, read
// twice and written once more, so a chunk has 640 rows or more, and 8192 where the arithmetic is fastest (16 groups of 16384 x
// 2048 x 1024, bfloat16: 16 chunks 191 us, 4 chunks 106), but never fewer than as many as give half the CUs work, or as its sums' runs ask for.
struct TnPlan { int tile; int64_t row_tiles, col_tiles, chunk, chunks; };
TnPlan tn_plan(int64_t m, int32_t groups, int32_t kdim, int32_t nout, int32_t dtype, int32_t prec, int ways) {
  TnPlan p{};
  // (a chunk of 512 rows or a group is what a workgroup has at least)
  const int64_t pairs = groups > m / 512 + 1 ? groups : m / 512 + 1;
  p.tile = choose_tile(dtype, prec, ways, kdim, 0, nout, pairs, m / pairs, false);
  p.row_tiles = ceil_div(kdim, grouped_tile_rows(p.tile));
  p.col_tiles = ceil_div(nout, grouped_tile_cols(p.tile));
  const int64_t tiles = p.row_tiles * p.col_tiles, rare = m / (p.tile == kDirect256 ? 8192 : 640);
  int64_t chunks = 512 / tiles < rare ? 512 / tiles : rare;
  if (chunks < 128 / tiles) chunks = 128 / tiles;
  if (chunks > ceil_div(m, 256)) chunks = ceil_div(m, 256);
  const int64_t longest = grouped_sum_most(dtype == SAGNN_BF16 ? SAGNN_GEMM_BF16 : prec);
  if (chunks < ceil_div(m, longest)) chunks = ceil_div(m, longest);
  if (chunks < 1) chunks = 1;
  p.chunk = round_up((size_t)ceil_div(m > 0 ? m : 1, chunks), 64);
  p.chunks = ceil_div(m > 0 ? m : 1, p.chunk);
  return p;
}
// Room for the plan of any types and modes
size_t tn_ws_bytes(int64_t m, int32_t groups, int32_t kdim, int32_t nout) {
  int64_t chunks = 0;
  auto most = [&](int32_t dtype, int32_t prec, int ways) {
    const int64_t c = tn_plan(m, groups, kdim, nout, dtype, prec, ways).chunks;
    chunks = c > chunks ? c : chunks;
  };
  most(SAGNN_BF16, SAGNN_GEMM_FP32, kAny);
  most(SAGNN_BF16, SAGNN_GEMM_FP32, kDirect);
  for (int32_t prec : {SAGNN_GEMM_FP32, SAGNN_GEMM_BF16, SAGNN_GEMM_FP32_BF16X3}) {
    most(SAGNN_F32, prec, kAny);
    most(SAGNN_F32, prec, kStaged);
  }
  return chunks > 1 ? (size_t)(2 * chunks) * kdim * nout * 4 : 0;
}

Launch plan_weights(GroupedArgs& a, int32_t dtype, int32_t prec) {
  const bool direct = dtype == SAGNN_BF16 && direct_rows(a.X, a.ldx, a.kdim) && direct_rows(a.G, a.ldg, a.nout) && aligned16(a.dW) && aligned16(a.partial);
  const bool staged = dtype == SAGNN_F32 && a.ldx <= kStagedLd && a.ldg <= kStagedLd;
  const TnPlan p = tn_plan(a.m, a.groups, a.kdim, a.nout, dtype, prec, direct ? kDirect : staged ? kStaged : kAny);
  a.chunk = p.chunk;
  a.run = grouped_run(dtype == SAGNN_BF16 ? SAGNN_GEMM_BF16 : prec, p.chunk);
  a.row_tiles = (int32_t)p.row_tiles;
  a.col_tiles = (int32_t)p.col_tiles;
  int64_t pairs = p.chunks + a.groups;
  a.pairs = (int32_t)pairs;
  if (pairs >= kManyPairs) pairs = round_up((size_t)pairs, 8);
  const int64_t blocks = pairs * p.row_tiles * p.col_tiles;
  return {p.tile, blocks <= INT32_MAX ? blocks : -1};
}

int launch_weights(const GroupedArgs& a, Launch l, int32_t dtype, int32_t prec, hipStream_t s) {
  return dtype == SAGNN_BF16 ? grouped_tn_bf16(a, l.tile, l.blocks, s)
         : prec == SAGNN_GEMM_FP32 ? grouped_tn_fp32(a, l.tile, l.blocks, s)
         : prec == SAGNN_GEMM_BF16 ? grouped_tn_fp32_bf16(a, l.tile, l.blocks, s) : grouped_tn_fp32_bf16x3(a, l.tile, l.blocks, s);
}

// The groups whose rows lie in several chunks
int join_weights(const GroupedArgs& a, hipStream_t s) {
  if (a.m <= a.chunk) return SAGNN_OK;
  const bool four = ((int64_t)a.kdim * a.nout & 3) == 0 && aligned16(a.dW) && aligned16(a.partial);
  int64_t wide = ceil_div((int64_t)a.kdim * a.nout, four ? 1024 : 256);
  if (wide > 1024) wide = 1024;
  grouped_join_kernel<<<dim3((uint32_t)wide, (uint32_t)a.groups), 256, 0, s>>>(a, four);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

}  // namespace
}  // namespace sagnn

SAGNN_EXPORT int grouped_gemm_act(int32_t dtype, const void* d_X, int64_t ldx, const void* d_W, int64_t ldw, int64_t stride_w,
                                  int32_t transW, const int32_t* d_off, int32_t n_groups, int64_t m, int32_t kdim, int32_t nout,
                                  int32_t prec, int32_t act, const void* d_mask, int64_t ldmask, void* d_Y, int64_t ldy, void* stream) {
  using namespace sagnn;
  if (!valid(dtype, prec, m, n_groups, kdim, nout) || (transW & ~1) || (act != SAGNN_ACT_IDENTITY && act != SAGNN_ACT_RELU)) return SAGNN_EINVAL;
  if (ldx < kdim || ldy < nout || ldw < (transW ? kdim : nout) || stride_w < 0 || (d_mask && ldmask < nout)) return SAGNN_EINVAL;
  if (m == 0) return SAGNN_OK;
  if (!d_X || !d_W || !d_off || !d_Y) return SAGNN_EINVAL;
  for (const void* p : {d_X, d_W, d_mask, (const void*)d_Y})
    if (!element_aligned(p, dtype)) return SAGNN_EINVAL;
  if (!element_aligned(d_off, SAGNN_F32)) return SAGNN_EINVAL;
  GroupedArgs a{};
  a.X = d_X; a.ldx = ldx; a.W = d_W; a.ldw = ldw; a.stride_w = stride_w; a.off = d_off; a.groups = n_groups;
  a.m = m; a.kdim = kdim; a.nout = nout; a.act = act; a.mask = d_mask; a.ldmask = ldmask; a.Y = d_Y; a.ldy = ldy;
  const Launch l = plan_rows(a, dtype, prec);
  if (l.blocks < 0) return SAGNN_EINVAL;
  return launch_rows(a, l, dtype, prec, transW != 0, (hipStream_t)stream);
}

SAGNN_EXPORT int grouped_gemm_bwd_workspace_bytes(int64_t m, int32_t n_groups, int32_t kdim, int32_t nout, size_t* bytes) {
  using namespace sagnn;
  if (!bytes || !valid(SAGNN_F32, SAGNN_GEMM_FP32, m, n_groups, kdim, nout)) return SAGNN_EINVAL;
  *bytes = tn_ws_bytes(m, n_groups, kdim, nout);
  return SAGNN_OK;
}

SAGNN_EXPORT int grouped_gemm_bwd(int32_t dtype, const void* d_X, int64_t ldx, const void* d_W, int64_t ldw, int64_t stride_w,
                                  const int32_t* d_off, int32_t n_groups, int64_t m, int32_t kdim, int32_t nout, int32_t prec,
                                  const void* d_G, int64_t ldg, const void* d_mask, int64_t ldmask, void* d_dX, int64_t lddx,
                                  float* d_dW, void* d_ws, size_t ws_bytes, void* stream) {
  using namespace sagnn;
  if (!valid(dtype, prec, m, n_groups, kdim, nout) || ldg < nout) return SAGNN_EINVAL;
  if (d_dX && (ldw < nout || stride_w < 0 || lddx < kdim || (d_mask && ldmask < kdim))) return SAGNN_EINVAL;
  if (d_dW && ldx < kdim) return SAGNN_EINVAL;
  if ((m > 0 && (!d_G || (d_dX && !d_W) || (d_dW && !d_X))) || ((m > 0 || d_dW) && !d_off)) return SAGNN_EINVAL;
  for (const void* p : {d_X, d_W, d_G, d_mask, (const void*)d_dX})
    if (!element_aligned(p, dtype)) return SAGNN_EINVAL;
  if (!element_aligned(d_off, SAGNN_F32) || !element_aligned(d_dW, SAGNN_F32) || !element_aligned(d_ws, SAGNN_F32)) return SAGNN_EINVAL;
  if (d_dW && ws_bytes < tn_ws_bytes(m, n_groups, kdim, nout)) return SAGNN_ECAPACITY;
  if (d_dW && !d_ws && tn_ws_bytes(m, n_groups, kdim, nout) > 0) return SAGNN_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  GroupedArgs x{}, w{};
  Launch lx{0, 0}, lw{0, 0};
  if (d_dX && m > 0) {       // (G W^T: the stored W read as the transposed one of a product with kdim and nout exchanged)
    x.off = d_off; x.groups = n_groups; x.m = m;
    x.X = d_G; x.ldx = ldg; x.W = d_W; x.ldw = ldw; x.stride_w = stride_w; x.kdim = nout; x.nout = kdim;
    x.mask = d_mask; x.ldmask = ldmask; x.Y = d_dX; x.ldy = lddx;
    lx = plan_rows(x, dtype, prec);
  }
  if (d_dW) {
    w.off = d_off; w.groups = n_groups; w.m = m;
    w.X = d_X; w.ldx = ldx; w.G = d_G; w.ldg = ldg; w.kdim = kdim; w.nout = nout; w.dW = d_dW; w.partial = (float*)d_ws;
    lw = plan_weights(w, dtype, prec);
  }
  if (lx.blocks < 0 || lw.blocks < 0) return SAGNN_EINVAL;
  int rc = SAGNN_OK;
  if (lx.blocks > 0 && lw.blocks > 0 && lx.tile == kDirect256 && lw.tile == kDirect256 && lx.blocks + lw.blocks <= most_blocks(512)) {
    rc = grouped_bwd_bf16(x, lx.blocks, w, lw.blocks, s);
  } else {
    if (d_dX && m > 0) rc = launch_rows(x, lx, dtype, prec, true, s);
    if (rc == SAGNN_OK && d_dW) rc = launch_weights(w, lw, dtype, prec, s);
  }
  return rc == SAGNN_OK && d_dW ? join_weights(w, s) : rc;
}
