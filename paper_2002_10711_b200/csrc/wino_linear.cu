// y = x W^T + bias with 4-bit weights and group scales, for few rows of x: warp MMAs on unpacked codes.
//
// Bound by reading the codes: 16 outputs x 128 inputs are 1 KB, read once.  A block owns 16 outputs and
// up to 8 NT rows of x; its eight warps take the 1 KB tiles of its outputs in turn, and where there are
// too few blocks to fill the GPU, the S blocks of a cluster share the tiles.  Sums of warps meet in
// shared memory, those of blocks through the cluster's, in a fixed order: no workspace, no atomics.
#include <cooperative_groups.h>

#include "wino_packed.cuh"

namespace wino {

namespace cg = cooperative_groups;

struct LinearArgs {
  Packed w;
  const char* x;
  long x_row;       // bytes
  Output out;
  long y_row;       // elements
  const float* bias;
  int M, z_x, vec;
};

constexpr int kRowsWarps = 8;

template <int DT, int NT, bool SMALL>
__global__ void __launch_bounds__(kRowsWarps * 32)
k_linear_rows(const __grid_constant__ LinearArgs a) {
  __shared__ float part[kRowsWarps][NT * 8][17];   // [warp][row of x][output], one bank apart
  __shared__ float total[NT * 8][17];
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long tile_K = blockIdx.x / S;
  const int m0 = blockIdx.y * NT * 8;
  griddep_launch();
  griddep_wait();

  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
  const char* row[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) row[n] = a.x + min(m0 + 8 * n + g, a.M - 1) * a.x_row;
  const uint4* codes = a.w.codes + tile_K * a.w.tiles_C * 64 + lane;
  const int step = kRowsWarps * S;
  int c = rank * kRowsWarps + warp;
  uint4 u0, u1;
  Input<DT> x[NT][4];
  auto fetch = [&](int tile) {
    u0 = __ldg(codes + tile * 64l);
    u1 = __ldg(codes + tile * 64l + 32);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[n][i] = load_input<DT>(row[n], tile * 128 + 32 * i + 8 * t, a.w.C, a.vec, a.z_x);
  };
  for (; c < a.w.tiles_C; c += step) {
    fetch(c);
    tile_mma<SMALL, NT>(acc, a.w, tile_K, c, u0, u1, x, a.z_x, g);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    part[warp][8 * n + 2 * t][g] = acc[n][0];
    part[warp][8 * n + 2 * t + 1][g] = acc[n][1];
    part[warp][8 * n + 2 * t][g + 8] = acc[n][2];
    part[warp][8 * n + 2 * t + 1][g + 8] = acc[n][3];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 8 * 16; e += kRowsWarps * 32) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < kRowsWarps; ++v) s = __fadd_rn(s, part[v][e >> 4][e & 15]);
    total[e >> 4][e & 15] = s;
  }
  if (S > 1) cluster.sync();
  else __syncthreads();
  // block `rank` of the cluster finishes its share of the outputs
  for (int e = threadIdx.x * S + rank; e < NT * 8 * 16; e += kRowsWarps * 32 * S) {
    const int m = m0 + (e >> 4);
    const long k = tile_K * 16 + (e & 15);
    float s = 0.0f;
    for (int b = 0; b < S; ++b)
      s = __fadd_rn(s, S > 1 ? cluster.map_shared_rank(&total[0][0], b)[(e >> 4) * 17 + (e & 15)] : total[e >> 4][e & 15]);
    if (m < a.M && k < a.w.K) store_output(a.out, m * a.y_row + k, s, a.bias ? __ldg(a.bias + k) : 0.0f);
  }
  if (S > 1) cluster.sync();   // no block leaves while another reads its sums
}

namespace {

template <int DT, int NT>
int launch_rows(const LinearArgs& a, int num_sms, cudaStream_t st) {
  const long tiles_K = (a.w.K + 15) / 16, slices = (a.M + NT * 8 - 1) / (NT * 8);
  int S = 1;
  while (S < 8 && tiles_K * slices * S < 2l * num_sms && S * kRowsWarps < a.w.tiles_C) S *= 2;
  if (slices > 65535) return WINO_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(tiles_K * S), (unsigned)slices);
  auto kernel = a.w.group < 128 ? k_linear_rows<DT, NT, true> : k_linear_rows<DT, NT, false>;
  return launch_kernel_cluster(kernel, grid, dim3(kRowsWarps * 32), (unsigned)S, 0, st, true, a);
}

template <int DT>
int launch_type(const LinearArgs& a, int num_sms, cudaStream_t st) {
  return a.M <= 8 ? launch_rows<DT, 1>(a, num_sms, st) : launch_rows<DT, 2>(a, num_sms, st);
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
  switch (d.x_dtype) {
    case WINO_INT8: return launch_type<WINO_INT8>(a, num_sms, st);
    case WINO_FLOAT: return launch_type<WINO_FLOAT>(a, num_sms, st);
    case WINO_BF16: return launch_type<WINO_BF16>(a, num_sms, st);
    default: return launch_type<WINO_FP16>(a, num_sms, st);
  }
}

}  // namespace wino
