// Mixture of experts for few tokens, with 4-bit weights: router, gate and up products, down product.
//
// Bound by reading the chosen experts' codes, each once.  Three launches, each starting while the one in
// front of it ends:
//   route  a block per token: its logits, the top_k experts and their weights
//   up     a block per (chosen expert, 16 of its inner values): gate and up products of up to 8 NT of the
//          expert's tokens, h = weight * silu(gate) * up, kept as the sum of two bf16 (three for 32-bit
//          inputs), which the next product takes as it is: 16 (24) significant bits, so that nothing
//          is rounded to the output's type in between
//   down   a block (or cluster) per 16 outputs: the products of every chosen expert, summed over experts in
//          their order; warps share the 1 KB tiles of all experts
// A token chooses an expert at most once, so that an expert's tokens are a set of bits, which every block
// makes for itself from the ids: no counters, no atomics on global memory, sums in a fixed order.
#include <cooperative_groups.h>

#include "wino_packed.cuh"

namespace wino {

namespace cg = cooperative_groups;

constexpr int kMaxExperts = 512, kSliceTokens = 64;
constexpr int kExpertWarps = 8;

struct ExpertsArgs {
  Packed gate, up, down;
  long gate_units, down_units;       // 16-byte units of codes an expert
  long gate_scales, down_scales;     // scales an expert
  const char* x;
  long x_row;                        // bytes
  const char* router;
  const float* router_bias;
  Output out;
  long y_row;                        // elements
  int* ids;
  float* weights;
  uint16_t* h;                       // [parts][rows][h_row]
  long h_plane, h_row;               // elements
  int T, D, I, E, top_k, normalize, vec, vec_router;
};

__device__ __forceinline__ Packed expert_of(Packed w, int e, long units, long scales) {
  w.codes += e * units;
  w.scales += e * scales;
  if (w.zeros) w.zeros += e * scales;
  return w;
}

// ---- router -----------------------------------------------------------------------------
constexpr int kRouteThreads = 512;
template <int DT>
__global__ void __launch_bounds__(kRouteThreads)
k_experts_route(const __grid_constant__ ExpertsArgs a) {
  __shared__ float logits[kMaxExperts];
  const int token = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_launch();
  griddep_wait();
  const char* x = a.x + token * a.x_row;
  for (int e = warp; e < a.E; e += kRouteThreads / 32) {
    const char* r = a.router + (long)e * a.D * Input<DT>::kBytes;
    float s = 0.0f;
    for (int k = lane * 8; k < a.D; k += 256) {
      float xv[8], rv[8];
      to_floats<DT>(load_input<DT>(x, k, a.D, a.vec, 0), xv);
      to_floats<DT>(load_input<DT>(r, k, a.D, a.vec_router, 0), rv);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __fmaf_rn(xv[i], rv[i], s);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, o));
    if (lane == 0) logits[e] = a.router_bias ? __fadd_rn(s, __ldg(a.router_bias + e)) : s;
  }
  __syncthreads();
  if (warp != 0) return;
  constexpr int kPer = kMaxExperts / 32;
  float v[kPer];          // experts 32 i + lane
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = 32 * i + lane;
    v[i] = e < a.E ? logits[e] : -INFINITY;
    nan |= !(v[i] < INFINITY);       // NaN or +inf
    top = fmaxf(top, v[i]);
  }
  nan = __any_sync(0xffffffffu, nan);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float sum = 0.0f;
  if (!a.normalize) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum = __fadd_rn(sum, v[i] > -INFINITY ? expf(__fsub_rn(v[i], top)) : 0.0f);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
  }
  // lane j keeps the j-th choice; `taken`: this lane's experts that are chosen already
  uint32_t taken = 0;
  int my_id = 0;
  float my_l = -INFINITY;
  for (int j = 0; j < a.top_k; ++j) {
    float best = -INFINITY;
    int at = kMaxExperts;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = 32 * i + lane;
      if (e < a.E && !(taken >> i & 1) && (at == kMaxExperts || v[i] > best)) best = v[i], at = e;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float b = __shfl_xor_sync(0xffffffffu, best, o);
      const int n = __shfl_xor_sync(0xffffffffu, at, o);
      if (n < kMaxExperts && (at == kMaxExperts || b > best || (b == best && n < at))) best = b, at = n;
    }
    if (nan) at = j;
    if ((at & 31) == lane) taken |= 1u << (at >> 5);
    if (lane == j) my_id = at, my_l = best;
  }
  float p = lane < a.top_k && my_l > -INFINITY ? expf(__fsub_rn(my_l, top)) : 0.0f;
  if (a.normalize) {
    sum = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
  }
  if (lane < a.top_k) {
    a.ids[(long)token * a.top_k + lane] = my_id;
    a.weights[(long)token * a.top_k + lane] = nan ? __uint_as_float(0x7FC00000u) : p > 0.0f ? __fdiv_rn(p, sum) : 0.0f;
  }
}

// ---- who goes where ---------------------------------------------------------------------
struct Lists {
  unsigned long long tokens[kMaxExperts];   // set of tokens of each expert
  uint16_t expert[kMaxExperts + 1];         // chosen experts, ascending
  uint16_t first[kMaxExperts + 1];          // first row of each chosen expert in h; rows of all behind the last
  int chosen;
};
// All threads; pairs whose weight is 0 are left out.
__device__ __forceinline__ void build_lists(Lists& l, const ExpertsArgs& a) {
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) l.tokens[e] = 0;
  __syncthreads();
  for (int p = threadIdx.x; p < a.T * a.top_k; p += blockDim.x)
    if (__ldg(a.weights + p) != 0.0f) atomicOr(&l.tokens[__ldg(a.ids + p)], 1ull << (p / a.top_k));
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int slots = 0, rows = 0;
    for (int base = 0; base < a.E; base += 32) {
      const int n = base + lane < a.E ? __popcll(l.tokens[base + lane]) : 0;
      const unsigned some = __ballot_sync(0xffffffffu, n != 0);
      int upto = n;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      if (n != 0) {
        const int slot = slots + __popc(some & ((1u << lane) - 1));
        l.expert[slot] = (uint16_t)(base + lane);
        l.first[slot] = (uint16_t)(rows + upto - n);
      }
      slots += __popc(some);
      rows += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) l.chosen = slots, l.first[slots] = (uint16_t)rows;
  }
  __syncthreads();
}
// The n-th token of a set (n below its size).
__device__ __forceinline__ int nth_token(unsigned long long set, int n) {
  const uint32_t lo = (uint32_t)set, hi = (uint32_t)(set >> 32);
  const int c = __popc(lo);
  return n < c ? __fns(lo, 0, n + 1) : 32 + __fns(hi, 0, n - c + 1);
}

// ---- gate and up --------------------------------------------------------------------------
template <int DT, int NT, bool SMALL>
__global__ void __launch_bounds__(kExpertWarps * 32)
k_experts_up(const __grid_constant__ ExpertsArgs a) {
  __shared__ Lists lists;
  __shared__ float part[kExpertWarps][2][NT * 8][17];
  __shared__ float weight[kSliceTokens];
  constexpr int P = Input<DT>::kParts == 3 ? 3 : 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  griddep_launch();
  griddep_wait();
  build_lists(lists, a);
  if ((int)blockIdx.y >= lists.chosen) return;
  const int slot = blockIdx.y, expert = lists.expert[slot];
  const unsigned long long tokens = lists.tokens[expert];
  const int count = __popcll(tokens);
  for (int p = threadIdx.x; p < a.T * a.top_k; p += blockDim.x)
    if (__ldg(a.ids + p) == expert) weight[p / a.top_k] = __ldg(a.weights + p);
  const Packed gate = expert_of(a.gate, expert, a.gate_units, a.gate_scales);
  const Packed up = expert_of(a.up, expert, a.gate_units, a.gate_scales);
  const long tile_K = blockIdx.x;
  const long at = tile_K * gate.tiles_C * 64 + lane;
  for (int n0 = 0; n0 < count; n0 += NT * 8) {
    float acc_g[NT][4], acc_u[NT][4];
    const char* row[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      acc_g[n][0] = acc_g[n][1] = acc_g[n][2] = acc_g[n][3] = 0.0f;
      acc_u[n][0] = acc_u[n][1] = acc_u[n][2] = acc_u[n][3] = 0.0f;
      row[n] = a.x + nth_token(tokens, min(n0 + 8 * n + g, count - 1)) * a.x_row;
    }
    for (int c = warp; c < gate.tiles_C; c += kExpertWarps) {
      const uint4 g0 = __ldg(gate.codes + at + c * 64l), g1 = __ldg(gate.codes + at + c * 64l + 32);
      const uint4 u0 = __ldg(up.codes + at + c * 64l), u1 = __ldg(up.codes + at + c * 64l + 32);
      Input<DT> x[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[n][i] = load_input<DT>(row[n], c * 128 + 32 * i + 8 * t, a.D, a.vec, 0);
      tile_mma<SMALL, NT>(acc_g, gate, tile_K, c, g0, g1, x, 0, g);
      tile_mma<SMALL, NT>(acc_u, up, tile_K, c, u0, u1, x, 0, g);
    }
    __syncthreads();   // the sums of the tokens in front have been read, and `weight` is complete
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        part[warp][0][8 * n + 2 * t + (e & 1)][g + 8 * (e >> 1)] = acc_g[n][e];
        part[warp][1][8 * n + 2 * t + (e & 1)][g + 8 * (e >> 1)] = acc_u[n][e];
      }
    __syncthreads();
    for (int e = threadIdx.x; e < NT * 8 * 16; e += kExpertWarps * 32) {
      const int n = n0 + (e >> 4);
      const int i = (int)tile_K * 16 + (e & 15);
      if (n >= count || i >= a.I) continue;
      float gs = 0.0f, us = 0.0f;
#pragma unroll
      for (int v = 0; v < kExpertWarps; ++v) {
        gs = __fadd_rn(gs, part[v][0][e >> 4][e & 15]);
        us = __fadd_rn(us, part[v][1][e >> 4][e & 15]);
      }
      const float silu = __fdiv_rn(gs, __fadd_rn(1.0f, expf(-gs)));
      float h = keep_nan(__fmul_rn(__fmul_rn(silu, us), weight[nth_token(tokens, n)]));
      uint16_t* to = a.h + (lists.first[slot] + n) * a.h_row + i;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        to[p * a.h_plane] = (uint16_t)(__float_as_uint(h) >> 16);
        h = rest_of_any(h);
      }
    }
  }
}

// ---- down -----------------------------------------------------------------------------------
template <int P, int NT, bool SMALL>
__global__ void __launch_bounds__(kExpertWarps * 32)
k_experts_down(const __grid_constant__ ExpertsArgs a) {
  __shared__ Lists lists;
  extern __shared__ float sums[];    // [warp][T][17], then [T][17]
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  griddep_launch();
  for (int e = threadIdx.x; e < kExpertWarps * a.T * 17; e += blockDim.x) sums[e] = 0.0f;
  griddep_wait();
  build_lists(lists, a);
  float* mine = sums + warp * a.T * 17;
  const long tile_K = blockIdx.x / S;
  const int tiles = a.down.tiles_C;
  for (int u = rank * kExpertWarps + warp; u < lists.chosen * tiles; u += kExpertWarps * S) {
    const int slot = u / tiles, c = u - slot * tiles, expert = lists.expert[slot];
    const unsigned long long tokens = lists.tokens[expert];
    const int count = __popcll(tokens);
    const Packed w = expert_of(a.down, expert, a.down_units, a.down_scales);
    const uint4* codes = w.codes + (tile_K * tiles + c) * 64l + lane;
    const uint4 u0 = __ldg(codes), u1 = __ldg(codes + 32);
    for (int n0 = 0; n0 < count; n0 += NT * 8) {
      float acc[NT][4];
      Planes<P> x[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
        const uint16_t* row = a.h + (lists.first[slot] + min(n0 + 8 * n + g, count - 1)) * a.h_row;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int p = 0; p < P; ++p)
            x[n][i].v[p] = load_input<WINO_BF16>(reinterpret_cast<const char*>(row + p * a.h_plane),
                                                 c * 128 + 32 * i + 8 * t, a.I, true, 0).v;
      }
      tile_mma<SMALL, NT>(acc, w, tile_K, c, u0, u1, x, 0, g);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = n0 + 8 * n + 2 * t + (e & 1);
          if (at < count) {
            float* s = mine + nth_token(tokens, at) * 17 + g + 8 * (e >> 1);
            *s = __fadd_rn(*s, acc[n][e]);
          }
        }
    }
    __syncwarp();
  }
  __syncthreads();
  float* total = sums + kExpertWarps * a.T * 17;
  for (int e = threadIdx.x; e < a.T * 16; e += blockDim.x) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < kExpertWarps; ++v) s = __fadd_rn(s, sums[(v * a.T + (e >> 4)) * 17 + (e & 15)]);
    total[(e >> 4) * 17 + (e & 15)] = s;
  }
  if (S > 1) cluster.sync();
  else __syncthreads();
  for (int e = threadIdx.x * S + rank; e < a.T * 16; e += blockDim.x * S) {
    const int m = e >> 4;
    const long k = tile_K * 16 + (e & 15);
    float s = 0.0f;
    for (int b = 0; b < S; ++b)
      s = __fadd_rn(s, (S > 1 ? cluster.map_shared_rank(total, b) : total)[m * 17 + (e & 15)]);
    if (k < a.D) store_output(a.out, m * a.y_row + k, s, 0.0f);
  }
  if (S > 1) cluster.sync();   // no block leaves while another reads its sums
}

namespace {

template <int DT, int NT>
int launch_slice(const ExpertsArgs& a, int num_sms, cudaStream_t st) {
  constexpr int P = Input<DT>::kParts == 3 ? 3 : 2;
  int rc = launch_kernel(k_experts_route<DT>, dim3((unsigned)a.T), dim3(kRouteThreads), 0, st, true, a);
  if (rc != 0) return rc;
  const long slots = (long)a.T * a.top_k < a.E ? (long)a.T * a.top_k : a.E;
  auto up = a.gate.group < 128 ? k_experts_up<DT, NT, true> : k_experts_up<DT, NT, false>;
  rc = launch_kernel(up, dim3((unsigned)((a.I + 15) / 16), (unsigned)slots), dim3(kExpertWarps * 32), 0, st, true, a);
  if (rc != 0) return rc;
  auto down = a.down.group < 128 ? k_experts_down<P, NT, true> : k_experts_down<P, NT, false>;
  const size_t smem = (size_t)(kExpertWarps + 1) * a.T * 17 * sizeof(float);   // at most 38.25 KB
  const long tiles_K = (a.D + 15) / 16, units = (a.I + 127) / 128 * slots;
  int S = 1;
  while (S < 8 && tiles_K * S < 2l * num_sms && (long)S * kExpertWarps < units) S *= 2;
  return launch_kernel_cluster(down, dim3((unsigned)(tiles_K * S)), dim3(kExpertWarps * 32), (unsigned)S, smem, st,
                               true, a);
}

template <int DT>
int launch_type(const ExpertsArgs& a, int num_sms, cudaStream_t st) {
  return a.T <= 8 ? launch_slice<DT, 1>(a, num_sms, st) : launch_slice<DT, 2>(a, num_sms, st);
}

long h_row_of(int I) { return (I + 7l) / 8 * 8; }
int parts_of(int dtype) { return dtype == WINO_FLOAT ? 3 : 2; }

}  // namespace

size_t experts_workspace(int T, int I, int top_k, int dtype) {
  return (size_t)(T < kSliceTokens ? T : kSliceTokens) * top_k * h_row_of(I) * 2 * parts_of(dtype);
}

int launch_experts(const wino_experts_desc_t& d, const void* x, const void* router, const float* router_bias, void* y,
                   int* ids, float* weights, void* workspace, int num_sms, cudaStream_t st) {
  ExpertsArgs a;
  a.gate = packed_view(d.gate); a.up = packed_view(d.up); a.down = packed_view(d.down);
  a.gate_units = (long)(wino_packed_code_bytes(d.I, d.D) / 16);
  a.down_units = (long)(wino_packed_code_bytes(d.D, d.I) / 16);
  a.gate_scales = (long)wino_packed_scale_count(d.I, d.D, d.gate.group);
  a.down_scales = (long)wino_packed_scale_count(d.D, d.I, d.down.group);
  const int size = d.dtype == WINO_FLOAT ? 4 : 2;
  a.x_row = (long)d.x_stride * size; a.y_row = d.y_stride;
  a.router = (const char*)router; a.router_bias = router_bias;
  a.D = d.D; a.I = d.I; a.E = d.E; a.top_k = d.top_k; a.normalize = d.normalize;
  a.out.dtype = d.dtype; a.out.mult = 1.0f; a.out.s_Y = 1.0f; a.out.lo = a.out.hi = 0.0f; a.out.z_Y = 0;
  a.h = (uint16_t*)workspace; a.h_row = h_row_of(d.I);
  a.vec_router = reinterpret_cast<uintptr_t>(router) % 16 == 0 && ((long)d.D * size) % 16 == 0;
  for (int t0 = 0; t0 < d.T; t0 += kSliceTokens) {
    a.T = d.T - t0 < kSliceTokens ? d.T - t0 : kSliceTokens;
    a.h_plane = (long)a.T * d.top_k * a.h_row;
    a.x = (const char*)x + t0 * a.x_row;
    a.out.y = (char*)y + (long)t0 * a.y_row * size;
    a.ids = ids + (long)t0 * d.top_k; a.weights = weights + (long)t0 * d.top_k;
    a.vec = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.T == 1 || a.x_row % 16 == 0);
    const int rc = d.dtype == WINO_FLOAT ? launch_type<WINO_FLOAT>(a, num_sms, st)
                 : d.dtype == WINO_BF16 ? launch_type<WINO_BF16>(a, num_sms, st)
                                        : launch_type<WINO_FP16>(a, num_sms, st);
    if (rc != 0) return rc;
  }
  return 0;
}

}  // namespace wino
