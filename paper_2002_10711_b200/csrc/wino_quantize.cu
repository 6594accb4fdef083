// Weights [K][C] -> 4-bit codes, scales and zeros of groups of inputs (and the values the codes stand for).
//
// Bound by memory: w is read once, codes, scales and values written once.  A warp takes 8 outputs x 128
// inputs; lane (g, t) holds of output g the 32 inputs of its 16-byte unit of codes, so that a group's
// extremes are those of four lanes and a unit leaves in one store.  A group longer than 128 inputs is read
// twice, by the same warp one after the other.
// 8192 x 8192 in bf16 with zeros and values: 60.3 us, 77 % of a copy's rate, with three of four issue slots taken
// by 24 instructions a weight (of a lane).  One warp walks a whole group: with one scale for 8192 inputs it is 215 us.
#include "wino_packed.cuh"

namespace wino {

struct QuantizeArgs {
  uint4* codes;
  uint16_t* scales;
  uint8_t* zeros;
  const char* w;
  char* values;
  long w_row;           // bytes
  int K, C, group, tiles_C, groups, scale_f16, vec, vec_values;
};

constexpr int kQuantWarps = 4;

// FULL: rows of w and of the values are aligned to eight elements, and C is a multiple of 128
template <bool FULL, int DT>
__device__ __forceinline__ void load_weights(const QuantizeArgs& a, const char* row, int k, float (&v)[8]) {
  if constexpr (FULL) {
    Input<DT> in;
    in.load(row + (long)k * Input<DT>::kBytes);
    to_floats<DT>(in, v);
    return;
  }
  to_floats<DT>(load_input<DT>(row, k, a.C, a.vec, 0), v);
}

template <bool FULL, int DT>
__device__ __forceinline__ void store_values(const QuantizeArgs& a, char* row, int k, const float (&v)[8]) {
  if constexpr (DT == WINO_FLOAT) {
    float* p = reinterpret_cast<float*>(row) + k;
    if (FULL || (a.vec_values && k + 8 <= a.C)) {
      reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (k + e < a.C) p[e] = v[e];
    }
  } else {
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == WINO_FP16) {
        const __half2 p = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
        h[j] = *reinterpret_cast<const uint32_t*>(&p);
      } else {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        h[j] = *reinterpret_cast<const uint32_t*>(&p);
      }
    }
    uint16_t* p = reinterpret_cast<uint16_t*>(row) + k;
    if (FULL || (a.vec_values && k + 8 <= a.C)) {
      *reinterpret_cast<uint4*>(p) = make_uint4(h[0], h[1], h[2], h[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (k + e < a.C) p[e] = (uint16_t)(h[e >> 1] >> (16 * (e & 1)));
    }
  }
}

struct Range {
  float lo, hi;   // min(w, 0), max(w, 0)
  __device__ __forceinline__ void join(float v) { lo = fminf(lo, v); hi = fmaxf(hi, v); }
  __device__ __forceinline__ void join(const Range& r) { lo = fminf(lo, r.lo); hi = fmaxf(hi, r.hi); }
  // over the four lanes of a row
  __device__ __forceinline__ void join_lanes() {
#pragma unroll
    for (int o = 1; o < 4; o *= 2) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
  }
};

struct Grid { float s, z, inverse; uint16_t bits; };
__device__ __forceinline__ Grid grid_of(const QuantizeArgs& a, const Range& r) {
  Grid q;
  const float span = a.zeros ? __fdiv_rn(__fsub_rn(r.hi, r.lo), 15.0f) : __fdiv_rn(fmaxf(r.hi, -r.lo), 7.0f);
  if (a.scale_f16) {
    q.bits = __half_as_ushort(__float2half_rn(fminf(span, 65504.0f)));
  } else {
    q.bits = __bfloat16_as_ushort(__float2bfloat16_rn(fminf(span, __uint_as_float(0x7F7F0000u))));
  }
  q.s = scale_to_float(q.bits, a.scale_f16);
  q.inverse = q.s > 0.0f ? __frcp_rn(q.s) : 0.0f;
  q.z = a.zeros && q.s > 0.0f ? fminf(fmaxf(rintf(__fdiv_rn(-r.lo, q.s)), 0.0f), 15.0f) : 8.0f;
  return q;
}

// w / s in 32 bits for scales far from the ends of the floats' range, as the reciprocal's product and one
// correction by its exact remainder: with the correctly rounded 1 / s that is the correctly rounded quotient
// (Markstein, Computation of elementary functions on the IBM RISC System/6000 processor, 1990).  Three
// instructions, where a division's special cases and their code took 8192 x 8192 bf16 weights from 60 to 115 us.
__device__ __forceinline__ bool plain_scale(float s) { return s == 0.0f || (s >= 0x1p-100f && s <= 0x1p100f); }
__device__ __forceinline__ float quotient(float w, const Grid& q) {
  const float r = __fmul_rn(w, q.inverse);
  const float rest = fminf(__fmaf_rn(-r, q.s, w), q.s);     // of an infinite r: not a number, and then s
  return __fmaf_rn(rest, q.inverse, r);
}
__device__ __noinline__ float any_quotient(float w, float s) { return __fdiv_rn(w, s); }

template <bool FULL, int DT>
__device__ __forceinline__ uint32_t codes_of(const QuantizeArgs& a, const Grid& q, const float (&v)[8], char* out, int k) {
  uint32_t word = 0;
  float back[8], r[8];
  if (plain_scale(q.s)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = quotient(v[e], q);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = any_quotient(v[e], q.s);
  }
  const float zero = __fadd_rn(kMagic, q.z);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // kMagic + code, clamped as such: the code is in the low bits, what is above them goes with the sum
    const float c = fminf(fmaxf(__fadd_rn(__fadd_rn(r[e], kMagic), q.z), kMagic), kMagic + 15.0f);
    back[e] = __fmul_rn(__fsub_rn(c, zero), q.s);
    word += (uint32_t)__float_as_int(c) * (1u << (4 * (e / 2 + 4 * (e & 1))));
  }
  if (out != nullptr) store_values<FULL, DT>(a, out, k, back);
  return word - (uint32_t)kMagicBits * 0x11111111u;
}

// grid.x: warps over (pairs of half tiles of outputs) x parts of the inputs; span: tiles of inputs that a
// warp takes, whole groups
template <bool FULL, int DT>
__global__ void __launch_bounds__(kQuantWarps * 32, FULL ? 8 : 1)
k_quantize(const __grid_constant__ QuantizeArgs a, int span, int parts) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long unit = blockIdx.x * (long)kQuantWarps + (threadIdx.x >> 5);
  const long half = unit / parts;                 // 8 outputs
  const int first = (int)(unit - half * parts) * span;
  griddep_launch();
  griddep_wait();
  if (half >= 2l * ((a.K + 15) / 16)) return;
  const long k = half * 8 + g;                    // output
  const bool in = k < a.K;
  const char* row = a.w + (in ? k : 0) * a.w_row;
  char* out = a.values != nullptr && in ? a.values + k * (long)a.C * Input<DT>::kBytes : nullptr;
  const long tile_K = half >> 1;
  uint4* codes = a.codes + tile_K * a.tiles_C * 64 + (half & 1) * 32 + lane;
  const long group_at = tile_K * a.groups * 16 + (half & 1) * 8 + g;
  const int last = min(first + span, a.tiles_C);
  auto put = [&](int grp, const Grid& q) {
    if (t == 0 && grp < a.groups) {
      a.scales[group_at + grp * 16l] = in ? q.bits : (uint16_t)0;
      if (a.zeros) a.zeros[group_at + grp * 16l] = in ? (uint8_t)(int)q.z : (uint8_t)8;
    }
  };
  if (a.group <= 128) {
    const int per = a.group / 32;                 // MMA pairs (32 inputs) a group
    for (int c = first; c < last; ++c) {
      float v[4][8];
      Range r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) load_weights<FULL, DT>(a, row, c * 128 + 32 * i + 8 * t, v[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r[i].lo = r[i].hi = 0.0f;
        if (a.zeros) {
#pragma unroll
          for (int e = 0; e < 8; ++e) r[i].join(v[i][e]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) r[i].hi = fmaxf(r[i].hi, fabsf(v[i][e]));
        }
      }
      if (per >= 2) { r[0].join(r[1]); r[2].join(r[3]); }
      if (per == 4) r[0].join(r[2]);
      uint32_t word[4];
      Grid q;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((i & (per - 1)) == 0) {
          r[i].join_lanes();
          q = grid_of(a, r[i]);
          put(per == 1 ? c * 4 + i : per == 2 ? c * 2 + (i >> 1) : c, q);
        }
        if (!in) q.s = q.inverse = 0.0f, q.z = 8.0f;
        word[i] = codes_of<FULL, DT>(a, q, v[i], out, c * 128 + 32 * i + 8 * t);
      }
      codes[c * 64l] = make_uint4(word[0], word[1], word[2], word[3]);
    }
    return;
  }
  const int per = a.group / 128;                  // tiles a group; span is a multiple of it
  for (int c0 = first; c0 < last; c0 += per) {
    const int c1 = min(c0 + per, last);
    Range r;
    r.lo = r.hi = 0.0f;
    for (int c = c0; c < c1; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
        load_weights<FULL, DT>(a, row, c * 128 + 32 * i + 8 * t, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) r.join(v[e]);
      }
    r.join_lanes();
    Grid q = grid_of(a, r);
    put(c0 / per, q);
    if (!in) q.s = q.inverse = 0.0f, q.z = 8.0f;
    for (int c = c0; c < c1; ++c) {
      uint32_t word[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
        load_weights<FULL, DT>(a, row, c * 128 + 32 * i + 8 * t, v);
        word[i] = codes_of<FULL, DT>(a, q, v, out, c * 128 + 32 * i + 8 * t);
      }
      codes[c * 64l] = make_uint4(word[0], word[1], word[2], word[3]);
    }
  }
}

int launch_quantize(const wino_packed_t& o, const void* w, int w_dtype, int64_t w_stride, void* values,
                    cudaStream_t st) {
  QuantizeArgs a;
  a.codes = (uint4*)const_cast<void*>(o.codes_dev);
  a.scales = (uint16_t*)const_cast<void*>(o.scales_dev);
  a.zeros = const_cast<uint8_t*>(o.zeros_dev);
  const int size = w_dtype == WINO_FLOAT ? 4 : 2;
  a.w = (const char*)w; a.w_row = (long)w_stride * size; a.values = (char*)values;
  a.K = o.K; a.C = o.C; a.group = o.group; a.tiles_C = (o.C + 127) / 128;
  a.groups = groups_of(o.C, o.group); a.scale_f16 = o.scale_dtype == WINO_FP16;
  a.vec = reinterpret_cast<uintptr_t>(w) % 16 == 0 && a.w_row % 16 == 0;
  a.vec_values = reinterpret_cast<uintptr_t>(values) % 16 == 0 && ((long)o.C * size) % 16 == 0;
  const long halves = 2l * ((o.K + 15) / 16);
  const int per = o.group <= 128 ? 1 : (int)((o.group + 127l) / 128 < a.tiles_C ? o.group / 128 : a.tiles_C);
  const int span = per, parts = (a.tiles_C + span - 1) / span;
  const long blocks = (halves * parts + kQuantWarps - 1) / kQuantWarps;
  if (blocks > 0x7fffffffl) return WINO_ERR_UNSUPPORTED;
  const bool full = a.vec && (values == nullptr || a.vec_values) && a.C % 128 == 0;
  auto kernel = w_dtype == WINO_FLOAT  ? (full ? k_quantize<true, WINO_FLOAT> : k_quantize<false, WINO_FLOAT>)
                : w_dtype == WINO_BF16 ? (full ? k_quantize<true, WINO_BF16> : k_quantize<false, WINO_BF16>)
                                       : (full ? k_quantize<true, WINO_FP16> : k_quantize<false, WINO_FP16>);
  return launch_kernel(kernel, dim3((unsigned)blocks), dim3(kQuantWarps * 32), 0, st, true, a, span, parts);
}

}  // namespace wino
