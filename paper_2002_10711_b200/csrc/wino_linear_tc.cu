// y = x W^T + bias with 4-bit weights and group scales on the 5th-generation tensor cores, for bf16 and fp16.
//
// A block owns 128 outputs (the rows of the MMA), NP rows of x (its columns) and a part of the inputs, in
// chunks of 128.  Codes become operands on the way: unpacked in registers (exact, see wino_packed.cuh)
// and stored to tensor memory, from where the MMA reads its A operand; x is the B operand, in shared memory.
// A group's products are accumulated on their own, in a slot of NP columns of tensor memory, and leave it
// multiplied by the output's scale into 32-bit sums in registers: no weight is rounded.
//
//   warps 0-3    epilogue: lane = output; slot -> registers, times the scale, added up
//   warps 4-11   two sets that take chunks in turn: copies of codes and of x several chunks ahead, unpacking;
//                warp w of a set fills lanes 32 (w % 4) .. +31
//   warp 12      tensor-memory owner; issues the MMAs
//
// Codes are copied in the order they are stored (512 consecutive bytes an instruction) to places in which a
// lane finds the four units of its own row without bank conflicts: unit t of row r stands at
// t ^ (r / 2 % 4).  The blocks of a cluster share the inputs and add their sums in a fixed order.
#include <cooperative_groups.h>

#include "wino_packed.cuh"

namespace wino {

namespace cg = cooperative_groups;

namespace {

constexpr int kTcThreads = 13 * 32, kTcStages = 3 /* code stages of a set */, kTcA = 2 /* A buffers */;

__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n"
      ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
        "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Instruction descriptor: D = 32-bit float, A = B = bf16 or fp16, both K-major, M x N.
constexpr uint32_t idesc_f16(bool f16, int M, int N) {
  return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

struct TcShape {
  // chunks whose x is on the way or in use: copies run 2 kTcStages chunks ahead of the MMA at most kTcA behind
  static constexpr int kB = 2 * kTcStages + kTcA;
};
constexpr int tc_columns(int NP, int slots) {
  int n = 32;
  while (n < kTcA * 64 + slots * NP) n *= 2;
  return n;
}
// Slots of sums: four while they fit beside the A buffers.
constexpr int tc_slots(int NP) { return NP <= 64 ? 4 : 3; }

struct TcBars { uint64_t a_full[kTcA], a_empty[kTcA], d_full[4], d_empty[4]; uint32_t tmem, abort; };

template <bool F16, int NP, bool SMALL, bool ZEROS>
__global__ void __launch_bounds__(kTcThreads, NP <= 16 ? 2 : 1)
k_linear_tc(const __grid_constant__ LinearArgs a, int* __restrict__ status) {
  constexpr int kSlots = tc_slots(NP), kB = TcShape::kB, kColumns = tc_columns(NP, kSlots);
  constexpr uint32_t kBytesB = NP * 256, kHalfB = NP * 128;      // a chunk of x: two halves of 64 inputs
  extern __shared__ uint8_t smem_raw[];
  __shared__ TcBars bars;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring_codes = base + kB * kBytesB;               // [set][stage][128 rows][64 bytes]
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles_K = (a.w.K + 15) / 16, block_K = blockIdx.x / S, m0 = blockIdx.y * NP;
  const int first = (int)((long)a.w.tiles_C * rank / S), n = (int)((long)a.w.tiles_C * (rank + 1) / S) - first;   // chunks
  const int parts = SMALL ? 128 / a.w.group : 1;                 // sums a chunk
  volatile uint32_t* abort_p = &bars.abort;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kTcA; ++i) {
      mbar_init(smem_u32(&bars.a_full[i]), 4);
      mbar_init(smem_u32(&bars.a_empty[i]), 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(smem_u32(&bars.d_full[i]), 1);
      mbar_init(smem_u32(&bars.d_empty[i]), 4);
    }
    bars.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // Tensor memory is taken when the kernel in front is over, and the next may start when it is taken: no
  // block holds some while it waits for one that needs some.
  griddep_wait();
  if (warp == 12) tmem_alloc(smem_u32(&bars.tmem), kColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch();
  const uint32_t tmem = bars.tmem, tmem_d = tmem + kTcA * 64;

  float acc[NP];                                                 // epilogue only
  if (warp < 4) {
#pragma unroll
    for (int i = 0; i < NP; ++i) acc[i] = 0.0f;
    // this lane's output among the packed rows, and its scales, fetched eight sums ahead
    const long row_tile = min(block_K * 8 + warp * 2 + (lane >> 4), tiles_K - 1);
    const uint16_t* scales = a.w.scales + row_tile * a.w.groups * 16 + (lane & 15);
    const int per = SMALL ? 1 : a.w.group >> 7, all = n * parts;
    auto scale = [&](int i) -> uint32_t {
      if (i >= all) return 0;
      const int grp = SMALL ? first * parts + i : per == 1 ? first + i : (first + i) / per;
      return scales[min(grp, a.w.groups - 1) * 16l];
    };
    uint32_t next[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) next[i] = scale(i);
    bool ok = true;
    int slot = 0;
    uint32_t phase = 0;
    for (int i0 = 0; i0 < all && ok; i0 += 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (i0 + j >= all || !ok) break;
        const float s = scale_to_float((uint16_t)next[j], a.w.scale_f16);
        next[j] = scale(i0 + j + 8);
        ok = __all_sync(0xffffffffu, mbar_wait<false>(smem_u32(&bars.d_full[slot]), phase, abort_p));
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = tmem_d + slot * NP + ((uint32_t)(warp * 32) << 16);
        if constexpr (NP == 16) {
          uint32_t d[16];
          tmem_ld16(from, d);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bars.d_empty[slot]));
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[i] = __fmaf_rn(__uint_as_float(d[i]), s, acc[i]);
        } else {
#pragma unroll
          for (int col = 0; col < NP; col += 32) {
            uint32_t d[32];
            tmem_ld32(from + col, d);
            tmem_ld_wait();
            if (col + 32 == NP) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(&bars.d_empty[slot]));
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[col + i] = __fmaf_rn(__uint_as_float(d[i]), s, acc[col + i]);
          }
        }
        if (++slot == kSlots) slot = 0, phase ^= 1u;
      }
    }
    if (!ok) *abort_p = 1u;
  } else if (warp < 12) {
    const int set = (warp - 4) >> 2, quad = warp & 3, u = threadIdx.x - 128 - set * 128;
    const uint32_t codes_at = ring_codes + set * kTcStages * 8192 + quad * 2048;
    // copies: instruction k takes rows 8 k .. 8 k + 7 of the warp's 32
    const uint32_t to = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ (lane >> 3 & 3)) << 4));
    const long tile0 = min(block_K * 8 + quad * 2, tiles_K - 1), tile1 = min(block_K * 8 + quad * 2 + 1, tiles_K - 1);
    const uint4* from0 = a.w.codes + tile0 * a.w.tiles_C * 64 + lane;
    const uint4* from1 = a.w.codes + tile1 * a.w.tiles_C * 64 + lane;
    // x: rows u / 16 + 8 k, piece u % 16 of 16 bytes of a chunk's row
    const int xr = u >> 4, piece = u & 15;
    const uint32_t x_to = base + (piece >> 3) * kHalfB + xr * 128 + (((piece & 7) ^ xr) << 4);
    const char* x_from = a.x + (long)(m0 + xr) * a.x_row + piece * 16;
    auto copy = [&](int q, int stage) {
      if (q < n) {
        const long c = first + q;
        const uint32_t s = codes_at + stage * 8192 + to;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from0 + c * 64) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + 512), "l"(from0 + c * 64 + 32) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + 1024), "l"(from1 + c * 64) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + 1536), "l"(from1 + c * 64 + 32) : "memory");
        const uint32_t b = x_to + (q % kB) * kBytesB;
        const int left = (a.w.C - (int)c * 128 - piece * 8) * 2;     // bytes of the row from this piece on
        const int bytes = left < 0 ? 0 : left > 16 ? 16 : left;
        const char* x = bytes > 0 ? x_from + c * 256 : a.x;
#pragma unroll
        for (int k = 0; k < NP / 8; ++k)
          if (m0 + xr + 8 * k < a.M)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(b + k * 1024), "l"(x + (bytes > 0 ? 8l * k * a.x_row : 0l)), "r"(bytes) : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // zeros of this lane's row: up to four of a chunk, a byte each
    const uint8_t* zeros = ZEROS ? a.w.zeros + (lane < 16 ? tile0 : tile1) * a.w.groups * 16 + (lane & 15) : nullptr;
    auto zero = [&](int q) -> uint32_t {
      if (!ZEROS || q >= n) return 0;
      uint32_t z = 0;
      if constexpr (SMALL) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < parts) z |= (uint32_t)zeros[min((first + q) * parts + i, a.w.groups - 1) * 16l] << (8 * i);
      } else {
        const int per = a.w.group >> 7;
        z = zeros[(per == 1 ? first + q : (first + q) / per) * 16l];
      }
      return z;
    };
    uint32_t z[kTcStages];
#pragma unroll
    for (int d = 0; d < kTcStages; ++d) {
      copy(set + 2 * d, d);
      z[d] = zero(set + 2 * d);
    }
    const uint32_t row_at = codes_at + lane * 64, swap = (uint32_t)(lane >> 1 & 3) << 4;
    bool ok = true;
    for (int q0 = set; q0 < n && ok; q0 += 2 * kTcStages) {
#pragma unroll
      for (int d = 0; d < kTcStages; ++d) {
        const int q = q0 + 2 * d;
        if (q >= n || !ok) break;
        asm volatile("cp.async.wait_group %0;" ::"n"(kTcStages - 1) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // x is read by the MMA
        __syncwarp();
        uint4 c[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) c[t] = lds_u4(row_at + d * 8192 + ((uint32_t)(t << 4) ^ swap));
        const int buf = q % kTcA;
        ok = __all_sync(0xffffffffu, mbar_wait<false>(smem_u32(&bars.a_empty[buf]), ((q / kTcA) & 1) ^ 1, abort_p));
        if (!ok) break;
        tc_fence_after();
        const uint32_t a_at = tmem + buf * 64 + ((uint32_t)(quad * 32) << 16);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t r[32];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t bias = zero_bias<F16>(8);
            if (ZEROS) bias = zero_bias<F16>((SMALL ? z[d] >> (8 * (parts == 4 ? 2 * h + i : h)) : z[d]) & 15u);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              uint32_t v[4];
              unpack8<F16>(word_of(c[t], 2 * h + i), bias, v);
#pragma unroll
              for (int p = 0; p < 4; ++p) r[i * 16 + t * 4 + p] = v[p];
            }
          }
          tmem_st32(a_at + h * 32, r);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.a_full[buf]));
        copy(q + 2 * kTcStages, d);
        z[d] = zero(q + 2 * kTcStages);
      }
    }
    if (!ok) *abort_p = 1u;
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    const bool leader = elect_one();
    constexpr uint32_t idesc = idesc_f16(F16, 128, NP);
    const int steps = 8 / parts;                                 // MMAs a sum
    bool ok = true;
    int slot = 0;
    uint32_t phase = 1;
    for (int q = 0; q < n; ++q) {
      const int buf = q % kTcA;
      if (!(ok = __all_sync(0xffffffffu, mbar_wait<false>(smem_u32(&bars.a_full[buf]), (q / kTcA) & 1, abort_p)))) break;
      tc_fence_after();
      const uint64_t desc = make_desc_sw128(base + (q % kB) * kBytesB);
      for (int p = 0; p < parts; ++p) {
        if (!(ok = __all_sync(0xffffffffu, mbar_wait<false>(smem_u32(&bars.d_empty[slot]), phase, abort_p)))) break;
        tc_fence_after();
        if (leader) {
          for (int s = 0; s < steps; ++s) {
            const int k = p * steps + s;                         // inputs 16 k .. +15
            mma_f16_ts(tmem_d + slot * NP, tmem + buf * 64 + k * 8, desc + (uint64_t)((k >> 2) * (kHalfB >> 4) + (k & 3) * 2),
                       idesc, s > 0 ? 1u : 0u);
          }
          mma_commit(smem_u32(&bars.d_full[slot]));
          if (p + 1 == parts) mma_commit(smem_u32(&bars.a_empty[buf]));
        }
        __syncwarp();
        if (++slot == kSlots) slot = 0, phase ^= 1u;
      }
      if (!ok) break;
    }
    // the last commit has arrived
    ok = ok && __all_sync(0xffffffffu, mbar_wait<false>(smem_u32(&bars.a_empty[(n - 1) % kTcA]), ((n - 1) / kTcA) & 1, abort_p));
    if (!ok) *abort_p = 1u;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_p != 0u && threadIdx.x == 0) atomicExch(status, WINO_ERR_TIMEOUT);
  if (warp == 12) {
    tc_fence_after();
    tmem_dealloc(tmem, kColumns);
  }
  const long out = (long)block_K * 128 + warp * 32 + lane;      // epilogue lanes
  if (S == 1) {
    if (warp < 4 && out < a.w.K) {
      const float bias = a.bias ? a.bias[out] : 0.0f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (m0 + i < a.M) store_output(a.out, (m0 + i) * a.y_row + out, acc[i], bias);
    }
    return;
  }
  float* sums = reinterpret_cast<float*>(smem_raw);              // [row of x][output]: the rings have been read
  if (warp < 4)
#pragma unroll
    for (int i = 0; i < NP; ++i) sums[i * 128 + warp * 32 + lane] = acc[i];
  cluster.sync();
  const int rows = min(NP, a.M - m0);
  for (int e = threadIdx.x + rank * kTcThreads; e < rows * 128; e += kTcThreads * S) {
    const long k = (long)block_K * 128 + (e & 127);
    float s = 0.0f;
    for (int b = 0; b < S; ++b) s = __fadd_rn(s, cluster.map_shared_rank(sums, b)[e]);
    if (k < a.w.K) store_output(a.out, (m0 + (e >> 7)) * a.y_row + k, s, a.bias ? a.bias[k] : 0.0f);
  }
  cluster.sync();   // no block leaves while another reads its sums
}

#ifndef TCBLOCKS
#define TCBLOCKS 1
#endif
template <bool F16, int NP, bool SMALL, bool ZEROS>
int launch_tc(const LinearArgs& a, int num_sms, int device, int* status, cudaStream_t st) {
  const long blocks = (a.w.K + 127) / 128, slices = (a.M + NP - 1) / NP;
  if (slices > 65535) return WINO_ERR_UNSUPPORTED;
  const long room = (long)(NP <= 16 ? 2 : 1) * TCBLOCKS * num_sms;
  int S = 1;
  while (S < 8 && blocks * slices * (S + 1) <= room && (S + 1) * 2 <= a.w.tiles_C) ++S;
  constexpr size_t ring = (size_t)TcShape::kB * NP * 256 + 2 * kTcStages * 8192;
  constexpr size_t sums = (size_t)NP * 128 * sizeof(float);
  constexpr size_t smem = (ring > sums ? ring : sums) + 1024;
  static DeviceOnce once;
  auto kernel = k_linear_tc<F16, NP, SMALL, ZEROS>;
  const int rc = set_max_smem(once, device, kernel, smem);
  if (rc != 0) return rc;
  return launch_kernel_cluster(kernel, dim3((unsigned)(blocks * S), (unsigned)slices), dim3(kTcThreads), (unsigned)S, smem, st,
                               true, a, status);
}
template <bool F16, int NP>
int launch_build(const LinearArgs& a, int num_sms, int device, int* status, cudaStream_t st) {
  if (a.w.zeros != nullptr)
    return a.w.group < 128 ? launch_tc<F16, NP, true, true>(a, num_sms, device, status, st)
                           : launch_tc<F16, NP, false, true>(a, num_sms, device, status, st);
  return a.w.group < 128 ? launch_tc<F16, NP, true, false>(a, num_sms, device, status, st)
                         : launch_tc<F16, NP, false, false>(a, num_sms, device, status, st);
}
template <bool F16>
int launch_width(const LinearArgs& a, int num_sms, int device, int* status, cudaStream_t st) {
  return a.M <= 16 ? launch_build<F16, 16>(a, num_sms, device, status, st)
       : a.M <= 32 ? launch_build<F16, 32>(a, num_sms, device, status, st)
                   : launch_build<F16, 64>(a, num_sms, device, status, st);
}

}  // namespace

bool linear_tc_supported(const LinearArgs& a, int x_dtype) {
  return (x_dtype == WINO_BF16 || x_dtype == WINO_FP16) && a.vec;
}

int launch_linear_tc(const LinearArgs& a, int x_dtype, int num_sms, int device, cudaStream_t st) {
  int* status = direct_tc_status_word(device);
  if (status == nullptr) return WINO_ERR_CUDA;
  return x_dtype == WINO_FP16 ? launch_width<true>(a, num_sms, device, status, st)
                              : launch_width<false>(a, num_sms, device, status, st);
}

}  // namespace wino
