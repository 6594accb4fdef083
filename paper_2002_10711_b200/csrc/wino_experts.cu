// Mixture of experts for few tokens, with 4-bit weights: router, gate and up products, down product.
//
// What it cannot do without is reading the chosen experts' codes, each once.  Three launches, each starting while the one in
// front of it ends:
//   route  a cluster per token: its logits, the top_k experts and their weights
//   up     a block per chosen expert and up to 8 row tiles of 16 of its inner values: gate and up products of up
//          to 8 NT of the expert's tokens at a time, h = weight * silu(gate) * up, kept as the exact sum of three bf16
//          for 32-bit inputs and for one or two tokens, whose planes take the MMA columns that would stay empty;
//          else of two rounded to nearest, which leave out at most 2^-17 of h, 2.5e-6 of y (rms, replayed with
//          2048 x 1024, 8 experts), where one bf16 would add a rounding of the output's own size
//   down   a block (or cluster) per up to 8 row tiles of outputs: the products of every chosen expert, summed
//          over experts in their order; the warps of a row tile share the tiles of all experts
// Warps stream their tiles through rings of asynchronous copies, as in the linear layer.
// 16 tokens, 8 of 64 experts, 2048 x 1024, bf16: 77 us for the three, where the bytes alone take 28 at the rate of a
// copy.  No unit is full.  up: about 170 instructions a 1 KB tile, 2.2 a clock while an SM has work but 1.6 over the
// whole time, for some 450 items on 296 blocks leave half of the blocks with twice the others' work.  down: about 250 a
// tile, 1.8 a clock; its columns are for eight tokens of an expert, which has 2.3, and h is waited for where it is used.
// One token: 19.0 us, the latency of three kernels in a row.
// A token chooses an expert at most once, so that an expert's tokens are a set of bits, which every block
// makes for itself from the ids: no counters, no atomics on global memory, sums in a fixed order.
#include <cooperative_groups.h>

#include "wino_packed.cuh"
#include "wino_spread.h"

namespace wino {

namespace cg = cooperative_groups;

constexpr int kMaxExperts = 512, kMaxTopK = 16, kSliceTokens = 64;
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
  uint16_t* h;                       // [parts][rows][h_row], bf16
  long h_plane, h_row;               // elements
  int T, D, I, E, top_k, normalize, vec, vec_router, parts;
};

__device__ __forceinline__ Packed expert_of(Packed w, int e, long units, long scales) {
  w.codes += e * units;
  w.scales += e * scales;
  if (w.zeros) w.zeros += e * scales;
  return w;
}

// ---- router -----------------------------------------------------------------------------
// A cluster per token: each block the logits of its share of the experts, a warp at a time; the first
// block ranks them all: an expert's place is the number of experts in front of it.
constexpr int kRouteThreads = 256;
template <int DT>
__global__ void __launch_bounds__(kRouteThreads)
k_experts_route(const __grid_constant__ ExpertsArgs a) {
  using In = Input<DT>;
  __shared__ __align__(16) float logits[kMaxExperts];
  __shared__ float top_l[kMaxTopK];
  __shared__ int top_e[kMaxTopK];
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int token = blockIdx.x / S, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_launch();
  // (behind the last expert: for four at a time)
  if (rank == 0)
    for (int e = a.E + threadIdx.x; e < (a.E + 3) / 4 * 4; e += kRouteThreads) logits[e] = -INFINITY;
  int log_by = 0;          // 2^log_by neighbouring lanes rank one expert
  while (log_by < 5 && a.E << (log_by + 1) <= kRouteThreads) ++log_by;
  auto arrived = cluster.barrier_arrive();         // the first block is there to be written to: waited for below
  griddep_wait();
  const char* x = a.x + token * a.x_row;
  float* to = cluster.map_shared_rank(logits, 0);
  bool waits = true;
  for (int e = rank + S * warp; e < a.E; e += S * (kRouteThreads / 32)) {
    const char* r = a.router + (long)e * a.D * In::kBytes;
    float s = 0.0f;
    auto add = [&](const In& xi, const In& ri) {
      float xv[8], rv[8];
      to_floats<DT>(xi, xv);
      to_floats<DT>(ri, rv);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __fmaf_rn(xv[i], rv[i], s);
    };
    if (a.vec && a.vec_router && a.D % 8 == 0) {
      constexpr int kAtOnce = DT == WINO_FLOAT ? 4 : 8;     // loads of each on the way at a time
#pragma unroll 1
      for (int k = lane * 8; k < a.D; k += kAtOnce * 256) {
        In xi[kAtOnce], ri[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          xi[i].clear(0);
          ri[i].clear(0);
          if (k + 256 * i < a.D) {
            xi[i].load(x + (k + 256 * i) * In::kBytes);
            ri[i].load(r + (k + 256 * i) * In::kBytes);
          }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) add(xi[i], ri[i]);
      }
    } else {
#pragma unroll 1
      for (int k = lane * 8; k < a.D; k += 256) add(load_input<DT>(x, k, a.D, a.vec, 0), load_input<DT>(r, k, a.D, a.vec_router, 0));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, o));
    if (waits) cluster.barrier_wait(std::move(arrived)), waits = false;
    if (lane == 0) to[e] = a.router_bias ? __fadd_rn(s, a.router_bias[e]) : s;
  }
  if (waits) cluster.barrier_wait(std::move(arrived));
  cluster.sync();
  if (rank != 0) return;
  bool odd = false;                       // NaN or +inf
  for (int e0 = 0; e0 < a.E; e0 += kRouteThreads >> log_by) {
    const int e = e0 + (threadIdx.x >> log_by), part = threadIdx.x & ((1 << log_by) - 1);
    const float l = e < a.E ? logits[e] : 0.0f;
    odd |= !(l < INFINITY);
    int place = 0;
    for (int f = part * 4; f < a.E; f += 4 << log_by) {
      const float4 o = *reinterpret_cast<const float4*>(logits + f);
      place += o.x > l || (o.x == l && f < e);
      place += o.y > l || (o.y == l && f + 1 < e);
      place += o.z > l || (o.z == l && f + 2 < e);
      place += o.w > l || (o.w == l && f + 3 < e);
    }
    for (int o = 1; o < 1 << log_by; o *= 2) place += __shfl_xor_sync(0xffffffffu, place, o);
    // (with a NaN about, places mean nothing, and nothing is done with them)
    if (part == 0 && e < a.E && place < a.top_k) top_l[place] = l, top_e[place] = e;
  }
  odd = __syncthreads_or(odd);
  if (warp != 0) return;
  const bool mine = lane < a.top_k;
  if (odd) {
    if (mine) {
      a.ids[(long)token * a.top_k + lane] = lane;
      a.weights[(long)token * a.top_k + lane] = __uint_as_float(0x7FC00000u);
    }
    return;
  }
  const float top = top_l[0];
  auto share = [&](float l) { return l > -INFINITY ? expf(__fsub_rn(l, top)) : 0.0f; };
  const float p = mine ? share(top_l[lane]) : 0.0f;
  float sum = p;
  if (!a.normalize) {
    sum = 0.0f;
    for (int e = lane; e < a.E; e += 32) sum = __fadd_rn(sum, share(logits[e]));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
  if (mine) {
    a.ids[(long)token * a.top_k + lane] = top_e[lane];
    a.weights[(long)token * a.top_k + lane] = p > 0.0f ? __fdiv_rn(p, sum) : 0.0f;
  }
}

// ---- who goes where ---------------------------------------------------------------------
// The chosen experts and their rows of h; pairs (token, expert) whose weight is 0 are left out.
struct Lists {
  unsigned long long tokens[kMaxExperts];   // set of tokens of each expert
  uint16_t slot[kMaxExperts];               // place of each chosen expert
  uint16_t expert[kMaxExperts];             // chosen experts, ascending
  uint16_t first[kMaxExperts + 1];          // first row of each in h; behind the last, the rows of all
  uint8_t token[kSliceTokens * kMaxTopK];   // token of each row
  float weight[kSliceTokens * kMaxTopK];    // weight of each row
  int chosen;
};
// All threads of the block.
__device__ __forceinline__ void build_lists(Lists& l, const ExpertsArgs& a) {
  const int pairs = a.T * a.top_k;
  if (a.T == 1) {
    // the token's choices as they stand, those of weight 0 last
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      const float w = lane < pairs ? a.weights[lane] : 0.0f;
      const int e = lane < pairs ? a.ids[lane] : 0;
      const int chosen = __popc(__ballot_sync(0xffffffffu, w != 0.0f));
      if (lane <= chosen) l.first[lane] = (uint16_t)lane;
      if (lane < chosen) l.expert[lane] = (uint16_t)e, l.token[lane] = 0, l.weight[lane] = w;
      if (lane == 0) l.chosen = chosen;
    }
    __syncthreads();
    return;
  }
  if (pairs <= 32) {
    // a pair per lane of the first warp: the same experts find one another without a table
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
      const float w = lane < pairs ? a.weights[lane] : 0.0f;
      const int id = lane < pairs ? a.ids[lane] : 0;
      const int e = w != 0.0f ? id : kMaxExperts + lane;
      const unsigned same = __match_any_sync(0xffffffffu, e), below = (1u << lane) - 1;
      const bool on = e < kMaxExperts, leads = on && (same & below) == 0;
      // places by expert: how many leaders have smaller ones, and how many pairs
      int slot = 0, first = 0;
      const unsigned leaders = __ballot_sync(0xffffffffu, leads);
      for (int i = 0; i < pairs; ++i) {
        const int o = __shfl_sync(0xffffffffu, e, i);
        if (o < e) slot += leaders >> i & 1, ++first;
      }
      if (on) {
        const int row = first + __popc(same & below);
        l.token[row] = (uint8_t)(lane / a.top_k);
        l.weight[row] = w;
      }
      if (leads) l.expert[slot] = (uint16_t)e, l.first[slot] = (uint16_t)first;
      const int rows = __popc(__ballot_sync(0xffffffffu, on));
      if (lane == 0) l.chosen = __popc(leaders), l.first[__popc(leaders)] = (uint16_t)rows;
    }
    __syncthreads();
    return;
  }
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) l.tokens[e] = 0;
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += blockDim.x)
    if (a.weights[p] != 0.0f) atomicOr(&l.tokens[a.ids[p]], 1ull << (p / a.top_k));
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
        l.slot[base + lane] = (uint16_t)slot;
        l.expert[slot] = (uint16_t)(base + lane);
        l.first[slot] = (uint16_t)(rows + upto - n);
      }
      slots += __popc(some);
      rows += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) l.chosen = slots, l.first[slots] = (uint16_t)rows;
  }
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += blockDim.x) {
    const float w = a.weights[p];
    if (w == 0.0f) continue;
    const int e = a.ids[p], t = p / a.top_k;
    const int row = l.first[l.slot[e]] + __popcll(l.tokens[e] & ((1ull << t) - 1));
    l.token[row] = (uint8_t)t;
    l.weight[row] = w;
  }
  __syncthreads();
}

// ---- gate and up --------------------------------------------------------------------------
constexpr int kUpDepth = 3, kDownDepth = 3, kDownCluster = 4;

// h as the sum of two or three bf16.  Two are rounded to nearest, each: the rest of the first is at most half of its
// last place, 2^(e-8) of an h in [2^e, 2^(e+1)), and what the second leaves at most 2^(e-17), on either side.  (Cut off
// as the three are they would leave up to 2^(e-15), always towards zero.)  Three cut off leave nothing.
__device__ __forceinline__ void store_parts(uint16_t* to, long plane, int parts, float h) {
  if (parts == 2) {
    // beyond the largest bf16 the nearest is infinity: cut off there (infinities and NaN stay what they are)
    const uint16_t first = fabsf(h) <= 0x1.FEp127f ? __bfloat16_as_ushort(__float2bfloat16_rn(h)) : (uint16_t)(__float_as_uint(h) >> 16);
    const float rest = fabsf(h) <= 3.4028235e38f ? __fsub_rn(h, __uint_as_float((uint32_t)first << 16)) : 0.0f;
    to[0] = first;
    to[plane] = __bfloat16_as_ushort(__float2bfloat16_rn(rest));
    return;
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    to[p * plane] = (uint16_t)(__float_as_uint(h) >> 16);
    h = rest_of_any(h);
  }
}

// An item is an expert, 8 / split row tiles, and 8 NT of the expert's tokens; a block takes every
// gridDim.x-th, and has the next one's first tiles on the way while it finishes one.
template <bool VEC, int DT, int NT, bool SMALL, bool ZEROS>
__global__ void __launch_bounds__(kExpertWarps * 32)
k_experts_up(const __grid_constant__ ExpertsArgs a, int log_split) {
  using In = Input<DT>;
  using Tiles = Ring<2, SMALL, ZEROS>;
  __shared__ Lists lists;
  extern __shared__ __align__(128) uint8_t smem[];
  float* sums = reinterpret_cast<float*>(smem + kExpertWarps * kUpDepth * Tiles::kSlot);   // [warp][token][33]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  griddep_launch();
  // what needs no lists, before the wait
  const int split = 1 << log_split;
  const int tiles_K = (a.I + 15) / 16, per_block = kExpertWarps >> log_split, blocks_K = (tiles_K + per_block - 1) / per_block;
  const int part = warp & (split - 1);
  const int c0 = (int)((long)a.gate.tiles_C * part >> log_split), c1 = (int)((long)a.gate.tiles_C * (part + 1) >> log_split);
  const uint32_t ring = smem_u32(smem) + warp * kUpDepth * Tiles::kSlot, ring_end = ring + kUpDepth * Tiles::kSlot;
  int slot = blockIdx.x / blocks_K, block_K = blockIdx.x - slot * blocks_K, n0 = 0;
  griddep_wait();
  build_lists(lists, a);
  Tiles tiles;
  auto begin = [&]() {
    if (slot < lists.chosen) {
      const int tile_K = min(block_K * per_block + (warp >> log_split), tiles_K - 1), expert = lists.expert[slot];
      const Stream from[2] = {stream_of(expert_of(a.gate, expert, a.gate_units, a.gate_scales), tile_K),
                              stream_of(expert_of(a.up, expert, a.gate_units, a.gate_scales), tile_K)};
      tiles.start(from, a.gate, c0, lane);
    }
#pragma unroll 1
    for (int d = 0; d < kUpDepth; ++d) {
      if (slot < lists.chosen && c0 + d < c1) tiles.fill(ring + d * Tiles::kSlot, lane);
      Tiles::commit();
    }
  };
  begin();
  while (slot < lists.chosen) {
    const int first = lists.first[slot], count = lists.first[slot + 1] - first;
    float acc[2][NT][4];
    const char* row[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      acc[0][n][0] = acc[0][n][1] = acc[0][n][2] = acc[0][n][3] = 0.0f;
      acc[1][n][0] = acc[1][n][1] = acc[1][n][2] = acc[1][n][3] = 0.0f;
      row[n] = a.x + lists.token[first + min(n0 + 8 * n + g, count - 1)] * a.x_row;
    }
    In x[NT][4];
    load_tile<VEC, DT, NT>(x, row, c0, a.D, 0, t);
    uint32_t at = ring;
    for (int c = c0; c < c1; ++c) {
      In now[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) now[n][i] = x[n][i];
      load_tile<VEC, DT, NT>(x, row, c + 1, a.D, 0, t);        // one tile ahead
      Tiles::template wait<kUpDepth - 1>();
      tile_mma<SMALL, ZEROS, Tiles, NT>(acc[0], at, 0, a.gate, now, 0, lane);
      tile_mma<SMALL, ZEROS, Tiles, NT>(acc[1], at, 1, a.up, now, 0, lane);
      __syncwarp();            // the slot has been read
      if (c + kUpDepth < c1) tiles.fill(at, lane);
      Tiles::commit();
      at = at + Tiles::kSlot == ring_end ? ring : at + Tiles::kSlot;
    }
    const int this_K = block_K * per_block, this_n0 = n0;
    if ((n0 += NT * 8) >= count) {
      n0 = 0;
      const int item = slot * blocks_K + block_K + gridDim.x;
      slot = item / blocks_K; block_K = item - slot * blocks_K;
    }
    __syncthreads();           // the sums in front have been read
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float* s = sums + (warp * NT * 8 + 8 * n + 2 * t + (e & 1)) * 33 + g + 8 * (e >> 1);
        s[0] = acc[0][n][e];
        s[16] = acc[1][n][e];
      }
    begin();
    __syncthreads();
    for (int e = threadIdx.x; e < per_block * NT * 8 * 16; e += kExpertWarps * 32) {
      const int k = e & 15, m = (e >> 4) % (NT * 8), v = (e >> 4) / (NT * 8);
      const int i = (this_K + v) * 16 + k;
      if (this_n0 + m >= count || i >= a.h_row) continue;      // h_row: I rounded up to eight, zeros behind I
      float gs = 0.0f, us = 0.0f;
      for (int w = 0; w < split; ++w) {
        const float* s = sums + ((v * split + w) * NT * 8 + m) * 33 + k;
        gs = __fadd_rn(gs, s[0]);
        us = __fadd_rn(us, s[16]);
      }
      const float silu = __fdiv_rn(gs, __fadd_rn(1.0f, expf(-gs)));
      const int row_h = first + this_n0 + m;
      const float h = i < a.I ? keep_nan(__fmul_rn(__fmul_rn(silu, us), lists.weight[row_h])) : 0.0f;
      store_parts(a.h + row_h * a.h_row + i, a.h_plane, a.parts, h);
    }
  }
}

// ---- down -----------------------------------------------------------------------------------
// A warp takes two row tiles.  The planes of h stand in columns of their own: with two, the eight columns of an
// MMA are four tokens' upper parts and their lower ones, added up at the end.
template <int P, int NT, bool SMALL, bool ZEROS>
__global__ void __launch_bounds__(kExpertWarps * 32)
k_experts_down(const __grid_constant__ ExpertsArgs a, int log_split, int log_S) {
  using In = Input<WINO_BF16>;
  using Tiles = Ring<2, SMALL, ZEROS>;
  constexpr int kEach = P == 2 ? 4 : 2, kTokens = NT * kEach;      // tokens of an MMA's columns, and at a time
  __shared__ Lists lists;
  extern __shared__ __align__(128) uint8_t smem[];
  float* sums = reinterpret_cast<float*>(smem + kExpertWarps * kDownDepth * Tiles::kSlot);   // [warp][T][33]
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  griddep_launch();
  for (int e = threadIdx.x; e < kExpertWarps * a.T * 33; e += blockDim.x) sums[e] = 0.0f;
  float* mine = sums + warp * a.T * 33;
  const int split = 1 << log_split, per_block = kExpertWarps >> log_split, tiles_K = (a.D + 15) / 16, tiles = a.down.tiles_C;
  const int unit = (int)(blockIdx.x >> log_S) * per_block + (warp >> log_split);     // two row tiles
  const int part = rank * split + (warp & (split - 1)), log_by = log_split + log_S;
  griddep_wait();
  build_lists(lists, a);
  // this warp's part of the tiles of all chosen experts, [expert][tile of inputs]
  const int all = lists.chosen * tiles;
  const int u0 = (int)((long)all * part >> log_by), u1 = unit * 2 < tiles_K ? (int)((long)all * (part + 1) >> log_by) : u0;
  const uint32_t ring = smem_u32(smem) + warp * kDownDepth * Tiles::kSlot, ring_end = ring + kDownDepth * Tiles::kSlot;
  int slot = 0, c = 0, fill_slot = 0, fill_c = 0;
  Tiles from;
  auto start = [&](int s, int at) {
    const Packed w = expert_of(a.down, lists.expert[s], a.down_units, a.down_scales);
    const Stream of[2] = {stream_of(w, unit * 2), stream_of(w, min(unit * 2 + 1, tiles_K - 1))};
    from.start(of, a.down, at, lane);
  };
  if (u0 < u1) {
    slot = fill_slot = u0 / tiles;
    c = fill_c = u0 - slot * tiles;
    start(slot, c);
  }
  auto fill = [&](uint32_t to) {
    from.fill(to, lane);
    if (++fill_c == tiles) {
      fill_c = 0;
      if (++fill_slot < lists.chosen) start(fill_slot, 0);
    }
  };
#pragma unroll 1
  for (int d = 0; d < kDownDepth; ++d) {
    if (u0 + d < u1) fill(ring + d * Tiles::kSlot);
    Tiles::commit();
  }
  float acc[2][NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[0][n][e] = acc[1][n][e] = 0.0f;
  uint32_t at = ring;
  int first = 0, count = 0;
  const char* row[NT];                              // of h: this column's plane and token, of the first ones
  auto enter = [&](int n0) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
      row[n] = reinterpret_cast<const char*>(a.h + min(g / kEach, P - 1) * a.h_plane +
                                             (first + min(n0 + n * kEach + g % kEach, count - 1)) * a.h_row);
  };
  auto expert = [&]() {
    first = lists.first[slot]; count = lists.first[slot + 1] - first;
    enter(0);
  };
  auto multiply = [&]() {
    In x[NT][4];
    load_tile<true, WINO_BF16, NT>(x, row, c, a.I, 0, t);       // (rows of h are filled up to eight values)
    Tiles::template wait<kDownDepth - 1>();
    tile_mma<SMALL, ZEROS, Tiles, NT>(acc[0], at, 0, a.down, x, 0, lane);
    tile_mma<SMALL, ZEROS, Tiles, NT>(acc[1], at, 1, a.down, x, 0, lane);
  };
  if (u0 < u1) expert();
  for (int u = u0; u < u1; ++u) {
    // up to kTokens tokens, sums stay in registers over an expert's tiles
    const bool last = c + 1 == tiles || u + 1 == u1, more = count > kTokens;
    for (int n0 = 0;;) {
      multiply();
      if (last || more) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float v = acc[r][n][e];
              if (P == 3) v = t == 3 ? 0.0f : __fadd_rn(v, 0.0f);
              if (P == 3) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, 1));
              v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, 2));
              const int m = n0 + n * kEach + (P == 2 ? 2 * t : 0) + (e & 1);
              if ((P == 2 ? t < 2 : t == 0) && m < count) {
                float* s = mine + lists.token[first + m] * 33 + r * 16 + g + 8 * (e >> 1);
                *s = __fadd_rn(*s, v);
              }
              acc[r][n][e] = 0.0f;
            }
      }
      if (!more || (n0 += kTokens) >= count) break;
      enter(n0);
    }
    if (more) enter(0);
    __syncwarp();              // the slot has been read, and `mine` is everyone's
    if (u + kDownDepth < u1) fill(at);
    Tiles::commit();
    if (++c == tiles) {
      c = 0;
      ++slot;
      if (u + 1 < u1) expert();
    }
    at = at + Tiles::kSlot == ring_end ? ring : at + Tiles::kSlot;
  }
  __syncthreads();
  // Outputs of the block, 32 of a token and unit at a time, lane = output, summed over the warps that share the
  // unit; a cluster's blocks leave their sums where their first warp's were.
  const int pairs = per_block * a.T;
  auto finish = [&](int v, int m, float s) {
    const long out = ((long)(blockIdx.x >> log_S) * per_block + v) * 32 + lane;
    if (out < a.D) store_output(a.out, m * a.y_row + out, s, 0.0f);
  };
  for (int e = warp; e < pairs; e += kExpertWarps) {
    const int v = e / a.T, m = e - v * a.T;
    float s = 0.0f;
    for (int i = 0; i < split; ++i) s = __fadd_rn(s, sums[((v * split + i) * a.T + m) * 33 + lane]);
    if (S > 1) sums[(v * split * a.T + m) * 33 + lane] = s;
    else finish(v, m, s);
  }
  if (S == 1) return;
  cluster.sync();
  for (int e = warp * S + rank; e < pairs; e += kExpertWarps * S) {
    const int v = e / a.T, m = e - v * a.T;
    float s = 0.0f, of[kDownCluster];
#pragma unroll
    for (int b = 0; b < kDownCluster; ++b) of[b] = b < S ? cluster.map_shared_rank(sums, b)[(v * split * a.T + m) * 33 + lane] : 0.0f;
#pragma unroll
    for (int b = 0; b < kDownCluster; ++b) s = __fadd_rn(s, of[b]);
    finish(v, m, s);
  }
  cluster.sync();   // no block leaves while another reads its sums
}

namespace {

constexpr long kBlocksPerSm = 2;    // of both products: more of them only start more often
// spread_smem for blocks that have Lists in static shared memory besides.
size_t spread_beside_lists(size_t smem, int per) {
  const size_t all = spread_smem(smem + sizeof(Lists), per);
  return all - sizeof(Lists);
}

// Warps that share one row tile's inputs: a power of two up to `most`, no more warps than there are, and
// no more than tiles.
int shared_by(long row_tiles, long tiles, int most, long warps) {
  int n = 1;
  while (n < most && row_tiles * n * 2 <= warps && n * 2 <= tiles) n *= 2;
  return n;
}

int log2_of(int n) {
  int l = 0;
  while (1 << l < n) ++l;
  return l;
}

template <bool VEC, int DT, int NT, bool SMALL, bool ZEROS>
int launch_up(const ExpertsArgs& a, long slots, int num_sms, int dev, cudaStream_t st) {
  constexpr size_t least = (size_t)kExpertWarps * (kUpDepth * Ring<2, SMALL, ZEROS>::kSlot + NT * 8 * 33 * sizeof(float));
  const long tiles_K = (a.I + 15) / 16;
  const int split = shared_by(tiles_K * slots, a.gate.tiles_C, kExpertWarps, kBlocksPerSm * kExpertWarps * num_sms);
  const long items = (tiles_K + kExpertWarps / split - 1) / (kExpertWarps / split) * slots;
  const long most = kBlocksPerSm * num_sms, blocks = items < most ? items : most;
  const size_t smem = spread_beside_lists(least, (int)((blocks + num_sms - 1) / num_sms));
  static DeviceOnce once;
  auto kernel = k_experts_up<VEC, DT, NT, SMALL, ZEROS>;
  const int rc = set_max_smem(once, dev, kernel, spread_beside_lists(least, 1));
  if (rc != 0) return rc;
  return launch_kernel(kernel, dim3((unsigned)blocks), dim3(kExpertWarps * 32), smem, st, true, a, log2_of(split));
}

template <int P, int NT, bool SMALL, bool ZEROS>
int launch_down(const ExpertsArgs& a, long slots, int num_sms, int dev, cudaStream_t st) {
  constexpr size_t ring = (size_t)kExpertWarps * kDownDepth * Ring<2, SMALL, ZEROS>::kSlot;
  const long units = ((a.D + 15) / 16 + 1) / 2;
  const int by = shared_by(units, (a.I + 127l) / 128 * slots, kDownCluster * kExpertWarps, kBlocksPerSm * kExpertWarps * num_sms);
  const int split = by < kExpertWarps ? by : kExpertWarps, S = by / split;
  const long blocks = (units + kExpertWarps / split - 1) / (kExpertWarps / split);
  const long per_sm = (blocks * S + num_sms - 1) / num_sms;
  const size_t smem = spread_beside_lists(ring + (size_t)kExpertWarps * a.T * 33 * sizeof(float), per_sm <= 8 ? (int)per_sm : 0);
  static DeviceOnce once;
  auto kernel = k_experts_down<P, NT, SMALL, ZEROS>;
  const int rc = set_max_smem(once, dev, kernel, spread_beside_lists(ring + (size_t)kExpertWarps * kSliceTokens * 33 * sizeof(float), 1));
  if (rc != 0) return rc;
  return launch_kernel_cluster(kernel, dim3((unsigned)(blocks * S)), dim3(kExpertWarps * 32), (unsigned)S, smem, st,
                               true, a, log2_of(split), log2_of(S));
}

template <int P, int NT>
int launch_down_groups(const ExpertsArgs& a, long slots, int num_sms, int dev, cudaStream_t st) {
  if (a.down.zeros)
    return a.down.group < 128 ? launch_down<P, NT, true, true>(a, slots, num_sms, dev, st)
                              : launch_down<P, NT, false, true>(a, slots, num_sms, dev, st);
  return a.down.group < 128 ? launch_down<P, NT, true, false>(a, slots, num_sms, dev, st)
                            : launch_down<P, NT, false, false>(a, slots, num_sms, dev, st);
}

template <int DT, int NT>
int launch_slice(const ExpertsArgs& a, int num_sms, cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return WINO_ERR_CUDA;
  // blocks that share a token's experts, until a warp has one, while there are SMs for them
  int S = 1;
  while (S < 8 && (long)a.T * S * 2 <= num_sms && S * (kRouteThreads / 32) < a.E) S *= 2;
  int rc = launch_kernel_cluster(k_experts_route<DT>, dim3((unsigned)(a.T * S)), dim3(kRouteThreads), (unsigned)S, 0, st, true, a);
  if (rc != 0) return rc;
  const long slots = (long)a.T * a.top_k < a.E ? (long)a.T * a.top_k : a.E;
  auto up = a.vec && a.D % 8 == 0
                ? (a.gate.group < 128 ? (a.gate.zeros ? launch_up<true, DT, NT, true, true> : launch_up<true, DT, NT, true, false>)
                                      : (a.gate.zeros ? launch_up<true, DT, NT, false, true> : launch_up<true, DT, NT, false, false>))
                : (a.gate.group < 128 ? (a.gate.zeros ? launch_up<false, DT, NT, true, true> : launch_up<false, DT, NT, true, false>)
                                      : (a.gate.zeros ? launch_up<false, DT, NT, false, true> : launch_up<false, DT, NT, false, false>));
  if ((rc = up(a, slots, num_sms, dev, st)) != 0) return rc;
  // columns for as many tokens as an expert may have of very few, else for more than it has as a rule: a
  // warp whose experts have more multiplies again, and the others wait for it
  if (NT == 1 && a.T <= 2) return launch_down_groups<3, 1>(a, slots, num_sms, dev, st);
  if constexpr (Input<DT>::kParts == 3) return launch_down_groups<3, NT == 1 ? 2 : 4>(a, slots, num_sms, dev, st);
  else if (NT == 1 && a.T <= 4) return launch_down_groups<2, 1>(a, slots, num_sms, dev, st);
  else return launch_down_groups<2, NT == 1 ? 2 : 4>(a, slots, num_sms, dev, st);
}

template <int DT>
int launch_type(const ExpertsArgs& a, int num_sms, cudaStream_t st) {
  // 16 of an expert's tokens at a time where it has more than 6 on average
  return (long)a.T * a.top_k <= 6l * a.E || a.T <= 8 ? launch_slice<DT, 1>(a, num_sms, st) : launch_slice<DT, 2>(a, num_sms, st);
}

long h_row_of(int I) { return (I + 7l) / 8 * 8; }
// of h, of a slice of T tokens (one or two: the NT == 1 of launch_type, and its first branch in launch_slice)
int parts_of(int dtype, int T) { return dtype == WINO_FLOAT || T <= 2 ? 3 : 2; }

}  // namespace

size_t experts_workspace(int T, int I, int top_k, int dtype) {
  const int slice = T < kSliceTokens ? T : kSliceTokens;   // a last, smaller one needs less
  return (size_t)slice * top_k * h_row_of(I) * 2 * parts_of(dtype, slice);
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
    a.parts = parts_of(d.dtype, a.T);
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
