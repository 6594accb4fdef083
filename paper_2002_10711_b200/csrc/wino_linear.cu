// y = x W^T + bias with 4-bit weights and group scales, for few rows of x: warp MMAs on unpacked codes.
//
// Bound by reading the codes: 16 outputs x 128 inputs are 1 KB, read once.  A warp streams the tiles of R row
// tiles (16 R outputs) over a part of the inputs through a ring of asynchronous copies, against up to 8 NT
// rows of x, which it reads from the L1 cache in the form of MMA operands.  `split` warps of a block, and the
// S blocks of a cluster where there are too few outputs to fill the GPU, share the inputs; their sums
// meet in shared memory in a fixed order: no workspace, no atomics.
#include <cooperative_groups.h>

#include "wino_packed.cuh"

namespace wino {

namespace cg = cooperative_groups;

constexpr int kRowsWarps = 8;
#ifndef RING
#define RING 3
#endif

template <int DT, int NT, int R, bool SMALL, bool ZEROS>
__global__ void __launch_bounds__(kRowsWarps * 32)
k_linear_rows(const __grid_constant__ LinearArgs a) {
  using In = Input<DT>;
  constexpr int T = 2 / R;                           // tiles of inputs a slot
  using Tiles = Ring<R, T, SMALL, ZEROS>;
  constexpr int kDepth = RING;
  constexpr int kSums = R * 16 + 1;                  // floats of a row of sums: one bank apart
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
    const char* next[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      row[n] = a.x + min(m0 + 8 * n + g, a.M - 1) * a.x_row;
      next[n] = row[n] + (c0 * 128l + 8 * t) * In::kBytes;
    }
    const uint32_t ring = smem_u32(smem) + warp * kDepth * Tiles::kSlot, ring_end = ring + kDepth * Tiles::kSlot;
    Tiles tiles;
    tiles.start(w, a.w, c0, c1, lane);
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (c0 + d * T < c1) tiles.fill(ring + d * Tiles::kSlot, lane);
      Tiles::commit();
    }
    const int whole = a.vec ? min(c1, a.w.C >> 7) : c0;     // tiles inside the rows of x, and aligned
    uint32_t slot = ring;
    for (int c = c0; c < c1; c += T) {
#pragma unroll
      for (int j = 0; j < T; ++j) {
        if (j > 0 && c + j >= c1) break;
        In x[NT][4];
        if (c + j < whole) {
          load_tile<DT, NT>(x, next);
        } else {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[n][i] = load_input<DT>(row[n], (c + j) * 128 + 32 * i + 8 * t, a.w.C, a.vec, a.z_x);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) next[n] += 128 * In::kBytes;
        if (j == 0) Tiles::template wait<kDepth - 1>();
#pragma unroll
        for (int r = 0; r < R; ++r) tile_mma<SMALL, ZEROS, Tiles, NT>(acc[r], slot, r * T + j, a.w, x, a.z_x, lane);
      }
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
  // outputs of the block: [unit][row of x][16 R]
  const int outputs = kRowsWarps / a.split * NT * 8 * R * 16;
  auto place = [&](int e, int& v, int& m, int& k) {
    k = e % (R * 16);
    m = e / (R * 16) % (NT * 8);
    v = e / (R * 16 * NT * 8);
  };
  auto finish = [&](int v, int m, int k, float s) {
    const long out = ((long)(blockIdx.x / S) * (kRowsWarps / a.split) + v) * R * 16 + k;
    if (m0 + m < a.M && out < a.w.K) store_output(a.out, (m0 + m) * a.y_row + out, s, a.bias ? a.bias[out] : 0.0f);
  };
  for (int e = threadIdx.x; e < outputs; e += kRowsWarps * 32) {
    int v, m, k;
    place(e, v, m, k);
    float s = 0.0f;
    for (int i = 0; i < a.split; ++i) s = __fadd_rn(s, sums[((v * a.split + i) * NT * 8 + m) * kSums + k]);
    if (S > 1) total[(v * NT * 8 + m) * kSums + k] = s;
    else finish(v, m, k, s);
  }
  if (S == 1) return;
  cluster.sync();
  // block `rank` of the cluster finishes its share of the outputs
  for (int e = threadIdx.x * S + rank; e < outputs; e += kRowsWarps * 32 * S) {
    int v, m, k;
    place(e, v, m, k);
    float s = 0.0f;
    for (int b = 0; b < S; ++b) s = __fadd_rn(s, cluster.map_shared_rank(total, b)[(v * NT * 8 + m) * kSums + k]);
    finish(v, m, k, s);
  }
  cluster.sync();   // no block leaves while another reads its sums
}

namespace {

#ifndef WARPS_PER_SM
#define WARPS_PER_SM 16
#endif
template <int DT, int NT, int R, bool SMALL, bool ZEROS>
int launch_rows(const LinearArgs& given, int num_sms, cudaStream_t st) {
  LinearArgs a = given;
  const long units = ((a.w.K + 15) / 16 + R - 1) / R, slices = (a.M + NT * 8 - 1) / (NT * 8);
  if (slices > 65535) return WINO_ERR_UNSUPPORTED;
  // inputs shared by as many warps as it takes to have WARPS_PER_SM of them on every SM
  int shared_by = 1;
  while (shared_by < 64 && units * slices * shared_by < (long)WARPS_PER_SM * num_sms && shared_by * 2 <= a.w.tiles_C) shared_by *= 2;
  a.split = shared_by < kRowsWarps ? shared_by : kRowsWarps;
  const int S = shared_by / a.split;
  const long blocks = (units + kRowsWarps / a.split - 1) / (kRowsWarps / a.split);
  const dim3 grid((unsigned)(blocks * S), (unsigned)slices);
  constexpr int kDepth = RING;
  constexpr size_t ring = (size_t)kRowsWarps * kDepth * Ring<R, 2 / R, SMALL, ZEROS>::kSlot;
  constexpr size_t sums = (size_t)2 * kRowsWarps * NT * 8 * (R * 16 + 1) * sizeof(float);
  constexpr size_t smem = ring > sums ? ring : sums;
  auto kernel = k_linear_rows<DT, NT, R, SMALL, ZEROS>;
  static DeviceOnce once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return WINO_ERR_CUDA;
  const int rc = set_max_smem(once, dev, kernel, smem);
  if (rc != 0) return rc;
  return launch_kernel_cluster(kernel, grid, dim3(kRowsWarps * 32), (unsigned)S, smem, st, true, a);
}

template <int DT, int NT, int R>
int launch_groups(const LinearArgs& a, int num_sms, cudaStream_t st) {
  if (a.w.zeros != nullptr)
    return a.w.group < 128 ? launch_rows<DT, NT, R, true, true>(a, num_sms, st) : launch_rows<DT, NT, R, false, true>(a, num_sms, st);
  return a.w.group < 128 ? launch_rows<DT, NT, R, true, false>(a, num_sms, st) : launch_rows<DT, NT, R, false, false>(a, num_sms, st);
}

template <int DT>
int launch_type(const LinearArgs& a, int num_sms, cudaStream_t st) {
  return a.M <= 8 ? launch_groups<DT, 1, 1>(a, num_sms, st) : launch_groups<DT, 2, 2>(a, num_sms, st);
}

}  // namespace
#ifndef TCMIN
#define TCMIN 9
#endif
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
  if (linear_tc_supported(a, d.x_dtype) && d.M >= TCMIN) {
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
