// y = x W^T + bias with 4-bit weights and group scales, for few rows of x: warp MMAs on unpacked codes.
//
// What it cannot do without is reading the codes: 16 outputs x 128 inputs are 1 KB, read once.  A warp streams the tiles of R row
// tiles (16 R outputs) over a part of the inputs through a ring of asynchronous copies, against up to 8 NT
// rows of x, which it reads from the L1 cache in the form of MMA operands.  `split` warps of a block, and the
// S blocks of a cluster where there are too few outputs to fill the GPU, share the inputs; their sums
// meet in shared memory in a fixed order: no workspace, no atomics.
// One row of 8192 x 32768 in bf16: 34.6 us, where the bytes alone take 21.2 at the rate of a copy.  No unit is full: of
// 155 instructions a 1 KB tile 2.3 are issued a clock while an SM has work (58 % of what it can, the ALU pipe 51 %
// busy), and 256 blocks on 148 SMs leave 40 of them with one block where the others have two, 1.9 a clock over the whole
// time.  Short sums are bound by latency: no weight is asked for before the kernel in front is over.  The row tiles
// of a warp share the loads of x.
// Rows that are not on 16-byte boundaries, or whose length is no multiple of eight, are read an element at a time and
// eight at once: 64 rows of 8191 x 8192 in bf16 take 160 us, of 8192 x 8192 21 (on the other kernel).
#include <cooperative_groups.h>

#include "wino_packed.cuh"
#include "wino_spread.h"

namespace wino {

namespace cg = cooperative_groups;

constexpr int kRowsWarps = 8, kRowTiles = 2 /* of a warp */, kRingSlots = 3, kMaxCluster = 4;

template <bool VEC, int DT, int NT, bool SMALL, bool ZEROS>
__global__ void __launch_bounds__(kRowsWarps * 32)
k_linear_rows(const __grid_constant__ LinearArgs a) {
  using In = Input<DT>;
  constexpr int R = kRowTiles, kSums = R * 16 + 1;   // floats of a row of sums: one bank apart
  using Tiles = Ring<R, SMALL, ZEROS>;
  extern __shared__ __align__(128) uint8_t smem[];
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int tiles_K = (a.w.K + 15) / 16;
  const int shared_by = a.split * S, part = rank * a.split + warp % a.split;
  const int unit = (int)(blockIdx.x / S) * (kRowsWarps / a.split) + warp / a.split;    // R row tiles
  const int m0 = blockIdx.y * NT * 8;
  const int c0 = (int)((long)a.w.tiles_C * part / shared_by), c1 = (int)((long)a.w.tiles_C * (part + 1) / shared_by);
  griddep_launch();
  griddep_wait();

  float acc[R][NT][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[r][n][0] = acc[r][n][1] = acc[r][n][2] = acc[r][n][3] = 0.0f;
  if (unit * R < tiles_K) {
    Stream w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = stream_of(a.w, min(unit * R + r, tiles_K - 1));
    const char* row[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) row[n] = a.x + min(m0 + 8 * n + g, a.M - 1) * a.x_row;
    const uint32_t ring = smem_u32(smem) + warp * kRingSlots * Tiles::kSlot, ring_end = ring + kRingSlots * Tiles::kSlot;
    Tiles tiles;
    tiles.start(w, a.w, c0, lane);
#pragma unroll 1
    for (int d = 0; d < kRingSlots; ++d) {
      if (c0 + d < c1) tiles.fill(ring + d * Tiles::kSlot, lane);
      Tiles::commit();
    }
    uint32_t slot = ring;
    for (int c = c0; c < c1; ++c) {
      In x[NT][4];
      load_tile<VEC, DT, NT>(x, row, c, a.w.C, a.z_x, t);
      Tiles::template wait<kRingSlots - 1>();
#pragma unroll
      for (int r = 0; r < R; ++r) tile_mma<SMALL, ZEROS, Tiles, NT>(acc[r], slot, r, a.w, x, a.z_x, lane);
      __syncwarp();          // the slot has been read
      if (tiles.c < c1) tiles.fill(slot, lane);
      Tiles::commit();
      slot = slot + Tiles::kSlot == ring_end ? ring : slot + Tiles::kSlot;
    }
  }
  __syncthreads();           // the rings are read: their place is that of the sums
  float* sums = reinterpret_cast<float*>(smem);           // [warp][row of x][output]
  float* total = sums + kRowsWarps * NT * 8 * kSums;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sums[(warp * NT * 8 + 8 * n + 2 * t + (e & 1)) * kSums + r * 16 + g + 8 * (e >> 1)] = acc[r][n][e];
  __syncthreads();
  // The block's outputs, 32 of a row of x and unit at a time, lane = output.  Where there is a cluster, block
  // `rank` finishes its share of them.
  const int rows = min(NT * 8, a.M - m0), pairs = kRowsWarps / a.split * rows;
  auto finish = [&](int v, int m, float s) {
    const long out = ((long)(blockIdx.x / S) * (kRowsWarps / a.split) + v) * 32 + lane;
    if (out < a.w.K) store_output(a.out, (m0 + m) * a.y_row + out, s, a.bias ? a.bias[out] : 0.0f);
  };
  for (int e = warp; e < pairs; e += kRowsWarps) {
    const int v = e / rows, m = e - v * rows;
    float s = 0.0f;
    for (int i = 0; i < a.split; ++i) s = __fadd_rn(s, sums[((v * a.split + i) * NT * 8 + m) * kSums + lane]);
    if (S > 1) total[(v * NT * 8 + m) * kSums + lane] = s;
    else finish(v, m, s);
  }
  if (S == 1) return;
  cluster.sync();
  for (int e = warp * S + rank; e < pairs; e += kRowsWarps * S) {
    const int v = e / rows, m = e - v * rows;
    float s = 0.0f, part_of[kMaxCluster];
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b)
      part_of[b] = b < S ? cluster.map_shared_rank(total, b)[(v * NT * 8 + m) * kSums + lane] : 0.0f;
#pragma unroll
    for (int b = 0; b < kMaxCluster; ++b) s = __fadd_rn(s, part_of[b]);
    finish(v, m, s);
  }
  cluster.sync();   // no block leaves while another reads its sums
}

namespace {

template <bool VEC, int DT, int NT, bool SMALL, bool ZEROS>
int launch_rows(const LinearArgs& given, int num_sms, cudaStream_t st) {
  LinearArgs a = given;
  const long units = ((a.w.K + 15) / 16 + kRowTiles - 1) / kRowTiles, slices = (a.M + NT * 8 - 1) / (NT * 8);
  // Inputs shared by as many warps as two blocks an SM have: split of a block times S of a cluster.
  const long room = 2l * kRowsWarps * num_sms;
  int S = 1, best = 0;
  a.split = 1;
  for (int split = 1; split <= kRowsWarps; split *= 2)
    for (int s = 1; s <= kMaxCluster; ++s) {
      const int by = split * s;
      if (by > 1 && (units * slices * by > room || by > a.w.tiles_C)) break;
      if (by > best || (by == best && s < S)) best = by, S = s, a.split = split;
    }
  const long blocks = (units + kRowsWarps / a.split - 1) / (kRowsWarps / a.split);
  const dim3 grid((unsigned)(blocks * S), (unsigned)slices);
  constexpr size_t ring = (size_t)kRowsWarps * kRingSlots * Ring<kRowTiles, SMALL, ZEROS>::kSlot;
  constexpr size_t sums = (size_t)2 * kRowsWarps * NT * 8 * (kRowTiles * 16 + 1) * sizeof(float);
  constexpr size_t least = ring > sums ? ring : sums;
  // no more blocks on an SM than its share: while the kernel in front runs they would gather on a few
  const long per_sm = (blocks * S * slices + num_sms - 1) / num_sms;
  const size_t smem = spread_smem(least, per_sm <= 8 ? (int)per_sm : 0);
  auto kernel = k_linear_rows<VEC, DT, NT, SMALL, ZEROS>;
  static DeviceOnce once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return WINO_ERR_CUDA;
  const int rc = set_max_smem(once, dev, kernel, spread_smem(least, 1));
  if (rc != 0) return rc;
  return launch_kernel_cluster(kernel, grid, dim3(kRowsWarps * 32), (unsigned)S, smem, st, true, a);
}

template <bool VEC, int DT, int NT>
int launch_groups(const LinearArgs& a, int num_sms, cudaStream_t st) {
  if (a.w.zeros != nullptr)
    return a.w.group < 128 ? launch_rows<VEC, DT, NT, true, true>(a, num_sms, st)
                           : launch_rows<VEC, DT, NT, false, true>(a, num_sms, st);
  return a.w.group < 128 ? launch_rows<VEC, DT, NT, true, false>(a, num_sms, st)
                         : launch_rows<VEC, DT, NT, false, false>(a, num_sms, st);
}

template <int DT>
int launch_type(const LinearArgs& a, int num_sms, cudaStream_t st) {
  if (a.vec && a.w.C % 8 == 0)
    return a.M <= 8 ? launch_groups<true, DT, 1>(a, num_sms, st) : launch_groups<true, DT, 2>(a, num_sms, st);
  return launch_groups<false, DT, 1>(a, num_sms, st);
}

}  // namespace
int launch_linear(const wino_linear_desc_t& d, const void* x, const float* bias, void* y, int num_sms,
                  cudaStream_t st) {
  LinearArgs a;
  a.w = packed_view(d.w);
  const int size = d.x_dtype == WINO_INT8 ? 1 : d.x_dtype == WINO_FLOAT ? 4 : 2;
  const int align = size == 1 ? 8 : 16;   // of eight elements, as they are loaded
  a.x = (const char*)x; a.x_row = (long)d.x_stride * size;
  a.vec = (reinterpret_cast<uintptr_t>(x) % align == 0 && (d.M == 1 || a.x_row % align == 0)) ? 1 : 0;
  a.bias = bias; a.y_row = d.y_stride; a.M = d.M;
  a.z_x = d.x_dtype == WINO_INT8 ? d.q_x.zero_point : 0;
  const double s_x = d.x_dtype == WINO_INT8 ? (double)d.q_x.scale : 1.0;
  const bool codes = d.y_dtype == WINO_INT8;
  a.out.y = y; a.out.dtype = d.y_dtype;
  a.out.mult = codes ? (float)(s_x / (double)d.q_Y.scale) : (float)s_x;
  a.out.s_Y = codes ? d.q_Y.scale : 1.0f;
  a.out.z_Y = codes ? d.q_Y.zero_point : 0;
  a.out.lo = codes ? (float)(d.q_Y.qmin - d.q_Y.zero_point) : 0.0f;
  a.out.hi = codes ? (float)(d.q_Y.qmax - d.q_Y.zero_point) : 0.0f;
  // The tcgen05 kernel takes some 2 us longer to start and to finish, and less for every weight: a warp MMA
  // goes through the weights once for every 16 rows of x.  us, this / that:  16 rows 8192x8192 16.4 / 15.1,
  // 4096x4096 7.4 / 7.4, 1024x1024 3.5 / 5.0;  32 rows 4096x4096 9.1 / 7.9, 1024 -> 8192 6.9 / 6.7;  64 rows
  // 1024 -> 8192 11.8 / 8.1, 512x512 4.1 / 6.7;  8 rows 8192x8192 12.9 / 14.8.
  const double passes = (d.M + 15) / 16, work = passes * d.w.K * d.w.C;
  if (linear_tc_supported(a, d.x_dtype) && d.M > 8 && work >= (passes == 1 ? 50e6 : 20e6)) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return WINO_ERR_CUDA;
    return launch_linear_tc(a, d.x_dtype, num_sms, dev, st);
  }
  switch (d.x_dtype) {
    case WINO_INT8: return launch_type<WINO_INT8>(a, num_sms, st);
    case WINO_FLOAT: return launch_type<WINO_FLOAT>(a, num_sms, st);
    case WINO_BF16: return launch_type<WINO_BF16>(a, num_sms, st);
    default: return launch_type<WINO_FP16>(a, num_sms, st);
  }
}

}  // namespace wino
