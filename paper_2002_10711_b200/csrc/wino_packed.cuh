// Layers with 4-bit weights: how codes become tensor-core operands, and how inputs do.
//
// A code less its zero is an integer of magnitude at most 15, exact in bf16 and in fp16, and so is
// every input of those types; int8 inputs less their zero point (at most 255 in magnitude) are exact
// fp16 integers, and a 32-bit input is the exact sum of three bf16 values of 8 significant bits each (down to 2^-110).
// The products are therefore exact, and the only roundings in front of the output are those of 32-bit sums (and, in
// the experts, that of the inner values between the two products).
//
// Warp MMA m16n8k16, weights as the 16-row operand, up to 8 rows of x as the columns.  Lane (g, t) =
// (lane / 4, lane % 4) holds rows g and g + 8 of A and column g of B at k = 2t, 2t+1, 2t+8, 2t+9.
// Which input stands at which k is free as long as both operands agree: in the pair of MMAs i of a
// 128-input tile lane t's eight k are the inputs 32 i + 8 t + 0..7, so that a lane reads 16 bytes of x
// at once, its codes of the whole tile are one 16-byte unit per row, and no MMA mixes inputs of two
// groups of 32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "wino.h"
#include "wino_launch.h"
#include "wino_ptx.cuh"

namespace wino {

// Packed weights as the kernels see them.
struct Packed {
  const uint4* codes;
  const uint16_t* scales;
  const uint8_t* zeros;   // null: 8
  int K, C, group, tiles_C, groups, scale_f16;
};
inline int groups_of(int C, int group) { return C / group + (C % group != 0); }   // no sum that passes 32 bits
inline Packed packed_view(const wino_packed_t& w) {
  Packed p;
  p.codes = (const uint4*)w.codes_dev; p.scales = (const uint16_t*)w.scales_dev; p.zeros = w.zeros_dev;
  p.K = w.K; p.C = w.C; p.group = w.group; p.tiles_C = (w.C + 127) / 128;
  p.groups = groups_of(w.C, w.group); p.scale_f16 = w.scale_dtype == WINO_FP16;
  return p;
}

__device__ __forceinline__ float scale_to_float(uint16_t s, int f16) {
  return f16 ? __half2float(__ushort_as_half(s)) : __uint_as_float((uint32_t)s << 16);
}

template <uint32_t MASK, uint32_t OR>
__device__ __forceinline__ uint32_t mask_or(uint32_t a) {
  uint32_t d;   // (a & MASK) | OR
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "n"(MASK), "n"(OR));
  return d;
}

// Operand format of the MMAs: F16 = false: bf16.
// Eight codes -> four pairs of (code - zero).  Spliced into the mantissa of 128 (bf16) or 1024 (fp16) a code
// is the exact value 128 + q or 1024 + q, and a subtraction of 128 + zero (1024 + zero) is exact too;
// in fp16 a code four bits further up is 1024 + 16 q, which saves two of the three shifts.
template <bool F16>
__device__ __forceinline__ uint32_t zero_bias(uint32_t zero) {   // both halves: 128 + zero or 1024 + zero
  return (F16 ? 0x64006400u : 0x43004300u) | (zero * 0x00010001u);
}
template <bool F16>
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
  uint32_t d;
  if (F16) asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <bool F16>
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t bias, uint32_t (&a)[4]) {
  if (F16) {
    // (1024 + 16 q) / 16 - (64 + zero); 64 + zero is exact in fp16: (1024 + zero) - 960
    uint32_t bias16, q1, q3;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(bias16) : "r"(0x63806380u), "r"(bias));   // 960 - (1024 + zero)
    const uint32_t w8 = w >> 8;
    a[0] = sub2<true>(mask_or<0x000F000Fu, 0x64006400u>(w), bias);
    q1 = mask_or<0x00F000F0u, 0x64006400u>(w);
    a[2] = sub2<true>(mask_or<0x000F000Fu, 0x64006400u>(w8), bias);
    q3 = mask_or<0x00F000F0u, 0x64006400u>(w8);
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(a[1]) : "r"(q1), "r"(0x2C002C00u), "r"(bias16));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(a[3]) : "r"(q3), "r"(0x2C002C00u), "r"(bias16));
  } else {
#pragma unroll
    for (int p = 0; p < 4; ++p) a[p] = sub2<false>(mask_or<0x000F000Fu, 0x43004300u>(w >> (4 * p)), bias);
  }
}

template <bool F16>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  if (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <bool F16>
__device__ __forceinline__ void mma_16816_from_0(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                 uint32_t b0, uint32_t b1) {
  if (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// Two floats -> a bf16 pair of their leading 8 significant bits (truncated: what is left is exact,
// and nothing overflows), lower half first.
__device__ __forceinline__ uint32_t truncate2(float lo, float hi) {
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632u);
}
__device__ __forceinline__ float rest_of(float v) {
  const float t = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
  return __fsub_rn(v, t);
}
// The same of a value that may be infinite or NaN: nothing is left of those.
__device__ __forceinline__ float rest_of_any(float v) { return fabsf(v) <= 3.4028235e38f ? rest_of(v) : 0.0f; }
// Top 16 bits that keep a NaN one whose payload is all in the lower bits.
__device__ __forceinline__ float keep_nan(float v) { return v == v ? v : __uint_as_float(0x7FFF0000u); }

// Eight consecutive inputs of one row of x, as loaded and as the B operand of two MMAs.  Loads are ordinary
// ones (not of the read-only path): the kernel in front may have written x while this one was starting.
//   PARTS  number of operands whose sum is x;  F16  their format
template <int DT> struct Input;
template <> struct Input<WINO_BF16> {
  static constexpr int kParts = 1, kBytes = 2;
  static constexpr bool kF16 = false;
  uint4 v;
  __device__ __forceinline__ void load(const char* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void clear(int) { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void set(int e, const char* p) {
    const uint32_t h = *reinterpret_cast<const unsigned short*>(p);
    uint32_t& w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
    w |= e & 1 ? h << 16 : h;
  }
  __device__ __forceinline__ void operand(int, uint32_t (&b)[kParts][4]) const {
    b[0][0] = v.x; b[0][1] = v.y; b[0][2] = v.z; b[0][3] = v.w;
  }
};
template <> struct Input<WINO_FP16> : Input<WINO_BF16> {
  static constexpr bool kF16 = true;
};
template <> struct Input<WINO_FLOAT> {
  static constexpr int kParts = 3, kBytes = 4;
  static constexpr bool kF16 = false;
  float v[8];
  __device__ __forceinline__ void load(const char* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void clear(int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
  }
  __device__ __forceinline__ void set(int e, const char* p) { v[e] = *reinterpret_cast<const float*>(p); }
  __device__ __forceinline__ void operand(int, uint32_t (&b)[kParts][4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float lo = keep_nan(v[2 * j]), hi = keep_nan(v[2 * j + 1]);
      const float lo1 = rest_of_any(lo), hi1 = rest_of_any(hi);
      b[0][j] = truncate2(lo, hi);
      b[1][j] = truncate2(lo1, hi1);
      b[2][j] = truncate2(rest_of(lo1), rest_of(hi1));
    }
  }
};
template <> struct Input<WINO_INT8> {
  static constexpr int kParts = 1, kBytes = 1;
  static constexpr bool kF16 = true;
  uint2 v;
  __device__ __forceinline__ void load(const char* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void clear(int z_x) {   // the code of zero
    v.x = v.y = ((uint32_t)z_x & 0xFFu) * 0x01010101u;
  }
  __device__ __forceinline__ void set(int e, const char* p) {
    const uint32_t c = (uint32_t)*reinterpret_cast<const uint8_t*>(p);
    uint32_t& w = e < 4 ? v.x : v.y;
    w = (w & ~(0xFFu << (8 * (e & 3)))) | (c << (8 * (e & 3)));
  }
  __device__ __forceinline__ void operand(int z_x, uint32_t (&b)[kParts][4]) const {
    // code + 128 in the mantissa of 1024, less 1152 + z_x: exact
    const uint32_t bias = (0x6400u + 128u + (uint32_t)z_x) * 0x00010001u;
    const uint32_t lo = v.x ^ 0x80808080u, hi = v.y ^ 0x80808080u;
    b[0][0] = sub2<true>(__byte_perm(lo, 0x64646464u, 0x4140u), bias);
    b[0][1] = sub2<true>(__byte_perm(lo, 0x64646464u, 0x4342u), bias);
    b[0][2] = sub2<true>(__byte_perm(hi, 0x64646464u, 0x4140u), bias);
    b[0][3] = sub2<true>(__byte_perm(hi, 0x64646464u, 0x4342u), bias);
  }
};

// The eight values of an input of real type.
template <int DT>
__device__ __forceinline__ void to_floats(const Input<DT>& in, float (&v)[8]) {
  if constexpr (DT == WINO_FLOAT) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = in.v[e];
  } else {
    const uint32_t w[4] = {in.v.x, in.v.y, in.v.z, in.v.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint16_t h = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      v[e] = DT == WINO_FP16 ? __half2float(__ushort_as_half(h)) : __uint_as_float((uint32_t)h << 16);
    }
  }
}

// Inputs k .. k+7 of the row at `row`, the code of zero beyond C.  vec: rows are aligned to eight elements
// (at most 16 bytes).
template <int DT>
__device__ __forceinline__ Input<DT> load_input(const char* row, int k, int C, bool vec, int z_x) {
  Input<DT> in;
  if (vec && k + 8 <= C) {
    in.load(row + (long)k * Input<DT>::kBytes);
  } else {
    in.clear(z_x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < C) in.set(e, row + (long)(k + e) * Input<DT>::kBytes);
  }
  return in;
}

// The inputs of tile c: x[n][i] of the row at row[n], inputs 128 c + 32 i + 8 t on.
//   VEC  rows are aligned to eight elements and C is a multiple of eight: eight at once, or none
template <bool VEC, int DT, int NT>
__device__ __forceinline__ void load_tile(Input<DT> (&x)[NT][4], const char* const (&row)[NT], int c, int C, int z_x, int t) {
  if (VEC && (c + 1) * 128 <= C) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const char* at = row[n] + (c * 128l + 8 * t) * Input<DT>::kBytes;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[n][i].load(at + 32 * i * Input<DT>::kBytes);
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = c * 128 + 32 * i + 8 * t;
      if constexpr (VEC) {
        x[n][i].clear(z_x);
        if (k < C) x[n][i].load(row[n] + (long)k * Input<DT>::kBytes);
      } else {
        x[n][i] = load_input<DT>(row[n], k, C, false, z_x);
      }
    }
}

// Codes, scales and zeros of one row tile (16 outputs), from its first input on.
struct Stream {
  const uint4* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
};
__device__ __forceinline__ Stream stream_of(const Packed& w, long tile_K) {
  return {w.codes + tile_K * w.tiles_C * 64, w.scales + tile_K * w.groups * 16,
          w.zeros ? w.zeros + tile_K * w.groups * 16 : nullptr};
}

// A warp's ring of weight tiles in shared memory, filled by asynchronous copies several tiles ahead of
// their use: each lane copies the two units of codes it will read itself, some lanes the scales and zeros
// as well (SMALL, groups of 32 or 64 inputs: four or two to a tile; else a group is one or more tiles, and
// every tile brings its scales along).  A slot holds one tile of each of R row tiles.
template <int R, bool SMALL, bool ZEROS> struct Ring {
  static constexpr int kGroups = SMALL ? 4 : 1;       // room for, a tile
  static constexpr int kScales = R * 1024, kZeros = kScales + R * kGroups * 32;
  static constexpr int kSlot = kZeros + (ZEROS ? R * kGroups * 16 : 0);
  const char* codes[R];
  const char* meta[R];     // scales, or zeros, of the row tile
  int c;                   // next tile
  int per;                 // groups a tile (SMALL) or tiles a group
  int groups;
  // this lane's 16 bytes of scales (two lanes a group) or zeros (a lane a group): whether it has some, group of
  // the tile, size of a group, offset in the group, place in the slot
  bool mine;
  int my_group, my_size, my_part;
  uint32_t my_place;

  // the next fill is of tile `from` of `w`
  __device__ __forceinline__ void start(const Stream (&w)[R], const Packed& p, int from, int lane) {
    c = from; groups = p.groups;
    per = SMALL ? (p.group == 32 ? 4 : 2) : p.group >> 7;
    const bool zero = ZEROS && lane >= 2 * kGroups;
    my_group = zero ? lane - 2 * kGroups : lane >> 1;
    mine = my_group < (SMALL ? per : 1);
    my_size = zero ? 16 : 32; my_part = zero ? 0 : 16 * (lane & 1);
    my_place = (zero ? kZeros : kScales) + my_group * my_size + my_part;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      codes[r] = reinterpret_cast<const char*>(w[r].codes + c * 64l + lane);
      meta[r] = (zero ? reinterpret_cast<const char*>(w[r].zeros) : reinterpret_cast<const char*>(w[r].scales)) + my_part;
    }
  }
  __device__ __forceinline__ void fill(uint32_t slot, int lane) {
    const uint32_t to = slot + lane * 16;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + r * 1024), "l"(codes[r]) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + r * 1024 + 512), "l"(codes[r] + 512) : "memory");
    }
    if (mine) {
      const int group = SMALL ? c * per + my_group : per == 1 ? c : c / per;
      // groups behind the last: zeros in place of what is not there
      const bool in = !SMALL || group < groups;
      const int bytes = in ? 16 : 0;
#pragma unroll
      for (int r = 0; r < R; ++r)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot + my_place + r * kGroups * my_size),
                     "l"(meta[r] + (in ? group : 0) * (long)my_size), "r"(bytes) : "memory");
    }
#pragma unroll
    for (int r = 0; r < R; ++r) codes[r] += 1024;
    ++c;
  }
  __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  template <int PENDING> __device__ __forceinline__ static void wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
  }
};

__device__ __forceinline__ uint32_t lds_u16(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint4 lds_u4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}

__device__ __forceinline__ uint32_t word_of(const uint4& u, int i) {
  return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
}

// One 16 x 128 tile of weights, the `index`-th of a ring's slot, against NT x 8 rows of x: acc +=
// scale * (codes - zeros) x, the sum of a group multiplied by its scale (for groups of at least 128: of a
// tile).  x[n][i]: the input of row 8 n + g at 32 i + 8 t.  Two chains of MMAs: one would wait for itself.
template <bool SMALL, bool ZEROS, class Tiles, int NT, class In>
__device__ __forceinline__ void tile_mma(float (&acc)[NT][4], uint32_t slot, int index, const Packed& w, const In (&x)[NT][4],
                                         int z_x, int lane) {
  constexpr bool F16 = In::kF16;
  constexpr int P = In::kParts;
  const uint32_t tile = slot + index * 1024 + lane * 16;
  const uint4 u0 = lds_u4(tile), u1 = lds_u4(tile + 512);
  const uint32_t scales = slot + Tiles::kScales + index * Tiles::kGroups * 32 + (lane >> 2) * 2;
  const uint32_t zeros = slot + Tiles::kZeros + index * Tiles::kGroups * 16 + (lane >> 2);
  float part[NT][2][4], s0, s1;
  uint32_t b0 = zero_bias<F16>(8), b1 = b0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (SMALL || i == 0) {
      const int grp = SMALL ? (w.group == 32 ? i : i >> 1) : 0;   // a group of 64 counts twice
      s0 = scale_to_float((uint16_t)lds_u16(scales + grp * 32), w.scale_f16);
      s1 = scale_to_float((uint16_t)lds_u16(scales + grp * 32 + 16), w.scale_f16);
      if (ZEROS) {
        b0 = zero_bias<F16>(lds_u8(zeros + grp * 16) & 15u);
        b1 = zero_bias<F16>(lds_u8(zeros + grp * 16 + 8) & 15u);
      }
    }
    uint32_t a0[4], a1[4];
    unpack8<F16>(word_of(u0, i), b0, a0);
    unpack8<F16>(word_of(u1, i), b1, a1);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      uint32_t b[P][4];
      x[n][i].operand(z_x, b);
#pragma unroll
      for (int p = P - 1; p >= 0; --p) {
        if ((SMALL || i == 0) && p == P - 1) {
          mma_16816_from_0<F16>(part[n][0], a0[0], a1[0], a0[1], a1[1], b[p][0], b[p][1]);
          mma_16816_from_0<F16>(part[n][1], a0[2], a1[2], a0[3], a1[3], b[p][2], b[p][3]);
        } else {
          mma_16816<F16>(part[n][0], a0[0], a1[0], a0[1], a1[1], b[p][0], b[p][1]);
          mma_16816<F16>(part[n][1], a0[2], a1[2], a0[3], a1[3], b[p][2], b[p][3]);
        }
      }
      if (SMALL || i == 3) {
        acc[n][0] = __fmaf_rn(__fadd_rn(part[n][0][0], part[n][1][0]), s0, acc[n][0]);
        acc[n][1] = __fmaf_rn(__fadd_rn(part[n][0][1], part[n][1][1]), s0, acc[n][1]);
        acc[n][2] = __fmaf_rn(__fadd_rn(part[n][0][2], part[n][1][2]), s1, acc[n][2]);
        acc[n][3] = __fmaf_rn(__fadd_rn(part[n][0][3], part[n][1][3]), s1, acc[n][3]);
      }
    }
  }
}

// One element of y.
struct Output {
  void* y;
  int dtype, z_Y;
  float mult, lo, hi;    // s_x, or s_x / s_Y and code bounds less the zero point
  float s_Y;             // for the bias of integer outputs
};
__device__ __forceinline__ void store_output(const Output& o, long at, float sum, float bias) {
  if (o.dtype == WINO_INT8) {
    const float f = __fmaf_rn(sum, o.mult, (float)((double)bias / (double)o.s_Y));
    const float r = __fadd_rn(fminf(fmaxf(f, o.lo), o.hi), kMagic);
    reinterpret_cast<int8_t*>(o.y)[at] = (int8_t)(magic_to_int(r) + o.z_Y);
    return;
  }
  const float f = __fmaf_rn(sum, o.mult, bias);
  if (o.dtype == WINO_FLOAT) reinterpret_cast<float*>(o.y)[at] = f;
  else if (o.dtype == WINO_BF16) reinterpret_cast<__nv_bfloat16*>(o.y)[at] = __float2bfloat16_rn(f);
  else reinterpret_cast<__half*>(o.y)[at] = __float2half_rn(f);
}

struct LinearArgs {
  Packed w;
  const char* x;
  long x_row;       // bytes
  Output out;
  long y_row;       // elements
  const float* bias;
  int M, z_x, vec;
  int split;        // warps of a block that share a row tile's inputs
};

// The kernel of wino_linear_tc.cu: bf16 and fp16, rows of x on 16-byte boundaries.
bool linear_tc_supported(const LinearArgs& a, int x_dtype);
int launch_linear_tc(const LinearArgs& a, int x_dtype, int num_sms, int device, cudaStream_t st);

}  // namespace wino
