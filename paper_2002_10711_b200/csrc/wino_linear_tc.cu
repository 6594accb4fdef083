// y = x W^T + bias with 4-bit weights and group scales on the 5th-generation tensor cores, for bf16 and fp16.
//
// A block owns 128 outputs (the rows of the MMA), NP rows of x (its columns) and a part of the inputs, in
// chunks of 128.  Codes become operands on the way: unpacked in registers (exact, see wino_packed.cuh)
// and stored to tensor memory, from where the MMA reads its A operand; x is the B operand, in shared memory.
// A group's products are accumulated on their own, in a slot of NP columns of tensor memory, and leave it
// multiplied by the output's scale into 32-bit sums in registers: no weight is rounded.
//
//   warps 0-7    epilogue: lane = output; sums of a chunk -> registers, times the scale, added up.  Two sets of four
//                take chunks in turn, or, for 64 rows of x, half of the rows each: one set alone took 500 to
//                900 cycles a chunk, longer than everything else
//   then kSets sets of four warps that take chunks in turn: copies of codes several chunks ahead, unpacking
//                into the set's buffer of tensor memory; warp w of a set fills lanes 32 (w % 4) .. +31
//   then a warp that owns the tensor memory and issues the MMAs, and one whose leader copies x by TMA
//
// 16 rows of 8192 x 8192 in bf16: 15.2 us, 64 with zeros 21.4, where the bytes take 5.4 and 5.7 at the rate of a copy.
// Up to 16 rows no unit is full (2.1 instructions a clock, the ALU pipe 43 % busy); warps wait for memory more than for
// anything else, and 128 blocks leave 20 SMs idle.  Unpacking is the most of the work, seven instructions of the ALU
// pipe for eight codes, which is why twelve of the 22 warps do it, and why x, which needs no conversion, is left to the
// copy engine.  With 64 rows it is the epilogue, 64 sums a chunk and output, whose loads, waits and products follow
// one another.
// Codes are copied in the order they are stored (512 consecutive bytes an instruction) to places in which a
// lane finds the four units of its own row without bank conflicts: unit t of row r stands at
// t ^ (r / 2 % 4).  The blocks of a cluster share the inputs and add their sums in a fixed order.
#include <cooperative_groups.h>

#include "wino_f32x2.cuh"
#include "wino_packed.cuh"

namespace wino {

namespace cg = cooperative_groups;

namespace {

// Unpacking sets: three; two beside more than 16 rows of x, where the epilogue wants more registers than 22 warps leave it
// (what it spilled missed the small L1 cache: 24.7 against 21.4 us for 64 x 8192 x 8192).
constexpr int tc_sets(int NP) { return NP > 16 ? 2 : 3; }
constexpr int kTcStages = 3 /* code stages of a set */;
constexpr int kRing = 8;       // chunks of x in shared memory, and of barriers
constexpr int kEpiWarps = 8;
constexpr int tc_threads(int NP) { return (kEpiWarps + 4 * tc_sets(NP) + 2) * 32; }

template <bool ACCUMULATE>
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint32_t bdesc_lo, uint32_t bdesc_hi, uint32_t idesc) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b64 b;\n"
      "mov.b64 b, {%2, %3};\n"
      "setp.ne.b32 p, %5, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n"
      "}\n"
      ::"r"(d), "r"(a), "r"(bdesc_lo), "r"(bdesc_hi), "r"(idesc), "n"(ACCUMULATE ? 1 : 0)
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

// Chunks in tensor memory, operand and sums (of up to four groups: small groups come with NP at most 32).
constexpr int tc_chunks(int NP, bool small) { return small && NP > 16 ? 2 : 4; }
constexpr int tc_columns(int NP, bool small) {
  int n = 32;
  while (n < tc_chunks(NP, small) * (64 + (small ? 4 : 1) * NP)) n *= 2;
  return n;
}

// full: a chunk's operands are there (its four unpacking warps, the copy of x) and the sums it goes to have been
// read (the epilogue's warps); done: its MMAs are over.  One wait and one commit a chunk: the thread that issues
// them is the only one of its kind, and two more of each a chunk made it the slowest part.
struct TcBars {
  uint64_t full[kRing], done[kRing];
  uint32_t tmem, abort;
};
constexpr int kScaleStages = 8;
// A stage of codes: 128 rows of 64 bytes, and zeros [4 warps][2 row tiles][4 groups][16].
constexpr uint32_t kZerosAt = 8192, kStageBytes = 8192 + 512;

template <bool F16, int NP, bool SMALL, bool ZEROS>
__global__ void __launch_bounds__(tc_threads(NP), 1)
k_linear_tc(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap map_x, int* __restrict__ status) {
  constexpr int kChunks = tc_chunks(NP, SMALL), kColumns = tc_columns(NP, SMALL), kSums = SMALL ? 4 : 1;
  constexpr int kSets = tc_sets(NP), kMmaWarp = kEpiWarps + 4 * kSets, kTcThreads = tc_threads(NP);
  constexpr bool kAlternate = NP <= 32;                          // the epilogue's sets take chunks in turn
  constexpr int kRows = kAlternate ? NP : NP / 2;                // of x, of an epilogue warp
  constexpr uint32_t kBytesX = NP * 256, kHalfX = NP * 128;      // a chunk of x: two halves of 64 inputs
  extern __shared__ uint8_t smem_raw[];
  __shared__ TcBars bars;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring_codes = base + kRing * kBytesX;         // [set][stage]
  const uint32_t scales_at = ring_codes + kSets * kTcStages * kStageBytes;   // [warp][stage][2 row tiles][16]
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles_K = (a.w.K + 15) / 16, block_K = blockIdx.x / S, m0 = blockIdx.y * NP;
  const int first = (int)((long)a.w.tiles_C * rank / S), n = (int)((long)a.w.tiles_C * (rank + 1) / S) - first;   // chunks
  const int parts = SMALL ? 128 / a.w.group : 1;                 // sums a chunk
  volatile uint32_t* abort_p = &bars.abort;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(smem_u32(&bars.full[i]), 4 + 1 + (kAlternate ? 4 : 8));
      mbar_init(smem_u32(&bars.done[i]), 1);
    }
    bars.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_map(&map_x);
  }
  // Tensor memory is taken when the kernel in front is over, and the next may start when it is taken: no
  // block holds some while it waits for one that needs some.
  griddep_wait();
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&bars.tmem), kColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch();
  const uint32_t tmem = bars.tmem, tmem_d = tmem + kChunks * 64;

  F2 acc[kRows / 2];                                             // epilogue only: rows of x 2 i, 2 i + 1
#pragma unroll
  for (int i = 0; i < kRows / 2; ++i) acc[i] = f2_both(0.0f);
  const int quad = warp & 3, epi = warp >> 2;
  if (warp < kEpiWarps) {
    // Scales of the warp's two row tiles, 64 bytes a sum, copied some sums ahead by lanes 0 .. 3.  (Held in
    // registers they would be waited for wherever a register is moved.)
    constexpr int kStep = kAlternate ? 2 : 1;                    // chunks
    const long row_tile = min(block_K * 8 + quad * 2 + (lane >> 1 & 1), tiles_K - 1);
    const int q0 = kAlternate ? epi : 0, per = SMALL ? 1 : a.w.group >> 7;
    const char* from_scales = reinterpret_cast<const char*>(a.w.scales + row_tile * a.w.groups * 16) + (lane & 1) * 16;
    const uint32_t ring = scales_at + warp * kScaleStages * 64;
    int next_q = q0, next_p = 0;
    uint32_t to = 0;
    auto copy = [&]() {
      if (lane < 4 && next_q < n) {
        // (groups behind the last have no inputs: any scale does)
        const int grp = min(SMALL ? (first + next_q) * parts + next_p : per == 1 ? first + next_q : (first + next_q) / per, a.w.groups - 1);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + to + lane * 16), "l"(from_scales + grp * 32l) : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (!SMALL || ++next_p == parts) next_p = 0, next_q += kStep;
      to = (to + 64) % (kScaleStages * 64);
    };
    if (lane == 0)
      for (int i = q0; i < kChunks; i += kStep) mbar_arrive(smem_u32(&bars.full[i]));      // nothing to read yet
    for (int i = 0; i < kScaleStages; ++i) copy();
    bool ok = true;
    uint32_t at = 0;
    for (int q = q0; q < n; q += kStep) {
      ok = __all_sync(0xffffffffu, mbar_wait<false>(smem_u32(&bars.done[q % kRing]), (q / kRing) & 1, abort_p));
      if (!ok) break;
      tc_fence_after();
      for (int p = 0; p < parts; ++p) {
        const uint32_t from = tmem_d + (q % kChunks * kSums + p) * NP + (kAlternate ? 0 : epi * kRows) + ((uint32_t)(quad * 32) << 16);
        uint32_t d[kRows];
        if constexpr (kRows == 32) tmem_ld32(from, d);
        else tmem_ld16(from, d);
        asm volatile("cp.async.wait_group %0;" ::"n"(kScaleStages - 1) : "memory");
        __syncwarp();
        const F2 s = f2_both(scale_to_float((uint16_t)lds_u16(ring + at + lane * 2), a.w.scale_f16));
        at = (at + 64) % (kScaleStages * 64);
        tmem_ld_wait();
        if (p + 1 == parts) tc_fence_before();
        __syncwarp();                      // every lane has its scale, and its sums
        if (p + 1 == parts && lane == 0) mbar_arrive(smem_u32(&bars.full[(q + kChunks) % kRing]));
        copy();
#pragma unroll
        for (int e = 0; e < kRows / 2; ++e) acc[e] = v_fma(f2_bits(d[2 * e], d[2 * e + 1]), s, acc[e]);
      }
    }
    if (!ok) *abort_p = 1u;
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp < kMmaWarp) {
    const int set = (warp - kEpiWarps) >> 2;
    const uint32_t ring = ring_codes + set * kTcStages * kStageBytes, codes_at = ring + quad * 2048, zeros_at = ring + kZerosAt + quad * 128;
    // copies: instruction k takes rows 8 k .. 8 k + 7 of the warp's 32
    const uint32_t to = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ (lane >> 3 & 3)) << 4));
    const long tile0 = min(block_K * 8 + quad * 2, tiles_K - 1), tile1 = min(block_K * 8 + quad * 2 + 1, tiles_K - 1);
    const uint4* from0 = a.w.codes + (tile0 * a.w.tiles_C + first + set) * 64 + lane;
    const uint4* from1 = a.w.codes + (tile1 * a.w.tiles_C + first + set) * 64 + lane;
    // zeros: 16 bytes of row tile lane / 4 and group lane % 4 of the chunk
    const uint8_t* from_zeros = ZEROS ? a.w.zeros + (lane < 4 ? tile0 : tile1) * a.w.groups * 16 : nullptr;
    int ahead = set;                                             // the chunk that is copied next
    auto copy = [&](uint32_t stage) {
      if (ahead < n) {
        const uint32_t s = codes_at + stage + to;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from0) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + 512), "l"(from0 + 32) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + 1024), "l"(from1) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + 1536), "l"(from1 + 32) : "memory");
        if (ZEROS && lane < 8 && (lane & 3) < parts) {
          const int per = SMALL ? 1 : a.w.group >> 7;
          const int grp = SMALL ? (first + ahead) * parts + (lane & 3) : per == 1 ? first + ahead : (first + ahead) / per;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(zeros_at + stage + lane * 16),
                       "l"(from_zeros + min(grp, a.w.groups - 1) * 16l) : "memory");
        }
        from0 += 64 * kSets; from1 += 64 * kSets;
        ahead += kSets;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int d = 0; d < kTcStages; ++d) copy(d * kStageBytes);
    const uint32_t row_at = codes_at + lane * 64, swap = (uint32_t)(lane >> 1 & 3) << 4;
    bool ok = true;
    uint32_t stage = 0;
    for (int q = set; q < n; q += kSets) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kTcStages - 1) : "memory");
      __syncwarp();
      uint4 c[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) c[t] = lds_u4(row_at + stage + ((uint32_t)(t << 4) ^ swap));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t r[32];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t bias = zero_bias<F16>(8);
          if (ZEROS) bias = zero_bias<F16>(lds_u8(zeros_at + stage + (lane >> 4) * 64 + (SMALL ? (parts == 4 ? 2 * h + i : h) : 0) * 16 + (lane & 15)) & 15u);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            uint32_t v[4];
            unpack8<F16>(word_of(c[t], 2 * h + i), bias, v);
#pragma unroll
            for (int p = 0; p < 4; ++p) r[i * 16 + t * 4 + p] = v[p];
          }
        }
        if (h == 0 && q >= kChunks) {        // what was there has been multiplied
          const int before = q - kChunks;
          ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&bars.done[before % kRing]), (before / kRing) & 1, abort_p));
          if (!ok) break;
          tc_fence_after();
        }
        tmem_st32(tmem + q % kChunks * 64 + h * 32 + ((uint32_t)(quad * 32) << 16), r);
      }
      if (!ok) break;
      __syncwarp();
      copy(stage);                        // every lane has read its part
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.full[q % kRing]));
      stage = stage == (kTcStages - 1) * kStageBytes ? 0 : stage + kStageBytes;
    }
    if (!ok) *abort_p = 1u;
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kMmaWarp) {
    // One thread: what it does between two chunks is what a chunk takes at least, so its MMAs are laid out in a
    // row and it waits for no other lane.
    if (elect_one()) {
      constexpr uint32_t idesc = idesc_f16(F16, 128, NP);
      const uint64_t desc0 = make_desc_sw128(base);
      const uint32_t desc_hi = (uint32_t)(desc0 >> 32);
      bool ok = true;
      for (int q = 0; q < n; ++q) {
        const int at = q % kRing, to = q % kChunks;
        if (!(ok = mbar_wait<false>(smem_u32(&bars.full[at]), (q / kRing) & 1, abort_p))) break;
        tc_fence_after();
        const uint32_t desc = (uint32_t)desc0 + at * (kBytesX >> 4), from = tmem + to * 64, sum0 = tmem_d + to * kSums * NP;
#pragma unroll
        for (int k = 0; k < 8; ++k) {                            // inputs 16 k .. +15
          const uint32_t b = desc + (k >> 2) * (kHalfX >> 4) + (k & 3) * 2;
          const bool begins = SMALL ? (parts == 4 ? k % 2 == 0 : k % 4 == 0) : k == 0;
          const uint32_t d = sum0 + (SMALL ? (parts == 4 ? k / 2 : k / 4) * NP : 0);
          if (begins) mma_f16_ts<false>(d, from + k * 8, b, desc_hi, idesc);
          else mma_f16_ts<true>(d, from + k * 8, b, desc_hi, idesc);
        }
        mma_commit(smem_u32(&bars.done[at]));
      }
      // the last commit has arrived
      ok = ok && mbar_wait<false>(smem_u32(&bars.done[(n - 1) % kRing]), ((n - 1) / kRing) & 1, abort_p);
      if (!ok) *abort_p = 1u;
    }
  } else if (lane == 0) {
    bool ok = true;
    int q = 0;
    for (; q < n; ++q) {
      const int at = q % kRing;
      const uint32_t bar = smem_u32(&bars.full[at]), to = base + at * kBytesX;
      if (q >= kRing && !(ok = mbar_wait(smem_u32(&bars.done[at]), ((q / kRing) & 1) ^ 1, abort_p))) break;
      mbar_expect_tx(bar, kBytesX);
      tma_load_2d(to, &map_x, bar, (first + q) * 128, m0);
      tma_load_2d(to + kHalfX, &map_x, bar, (first + q) * 128 + 64, m0);
    }
    if (!ok) {
      // A wait elsewhere ran out: the copies under way get time to land before the block ends.
      *abort_p = 1u;
      const long long t0 = clock64();
      while (clock64() - t0 < 10000000ll) __nanosleep(1000);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_p != 0u && threadIdx.x == 0) atomicExch(status, WINO_ERR_TIMEOUT);
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kColumns);
  }
  // Sums by way of shared memory, where the rings were: [row of x][output].  A short loop then finishes them:
  // laid out in a row, the code for 64 results of any type is 60 KB, and fetching it took 6 us.
  float* sums = reinterpret_cast<float*>(smem_raw);
  auto put = [&](bool add) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      uint32_t v[2];
      f2_split(acc[i / 2], v[0], v[1]);
      float* to = sums + ((kAlternate ? 0 : epi * kRows) + i) * 128 + quad * 32 + lane;
      *to = add ? __fadd_rn(*to, __uint_as_float(v[i & 1])) : __uint_as_float(v[i & 1]);
    }
  };
  if (warp < 4 || (!kAlternate && warp < kEpiWarps)) put(false);
  if (kAlternate) {
    __syncthreads();
    if (warp >= 4 && warp < kEpiWarps) put(true);
  }
  if (S > 1) cluster.sync();
  else __syncthreads();
  const int rows = min(NP, a.M - m0), k = threadIdx.x & 127, by = kTcThreads / 128 * S;
  const long out = (long)block_K * 128 + k;
  if (out < a.w.K && threadIdx.x < kTcThreads / 128 * 128) {
    const float bias = a.bias ? a.bias[out] : 0.0f;
#pragma unroll 1
    for (int m = threadIdx.x / 128 * S + rank; m < rows; m += by) {
      float s = 0.0f;
      if (S == 1) {
        s = sums[m * 128 + k];
      } else {
        float v[8];
#pragma unroll
        for (int b = 0; b < 8; ++b) v[b] = b < S ? cluster.map_shared_rank(sums, b)[m * 128 + k] : 0.0f;
#pragma unroll
        for (int b = 0; b < 8; ++b) s = __fadd_rn(s, v[b]);
      }
      store_output(a.out, (m0 + m) * a.y_row + out, s, bias);
    }
  }
  if (S > 1) cluster.sync();   // no block leaves while another reads its sums
}

template <bool F16, int NP, bool SMALL, bool ZEROS>
int launch_tc(const LinearArgs& a, int num_sms, int device, int* status, cudaStream_t st) {
  const long blocks = (a.w.K + 127) / 128, slices = (a.M + NP - 1) / NP;
  // blocks that share the inputs, while there are SMs for them and two chunks for each; of clusters of more than
  // four, one to an SM, the GPU holds no more than fourteen at once (2048 x 2048: 10 us in sixteen of eight)
  const int most = blocks * slices <= 14 ? 8 : 4;
  int S = 1;
  while (S < most && blocks * slices * (S + 1) <= num_sms && (S + 1) * 2 <= a.w.tiles_C) ++S;
  constexpr size_t ring = (size_t)kRing * NP * 256 + tc_sets(NP) * kTcStages * kStageBytes + kEpiWarps * kScaleStages * 64;
  constexpr size_t sums = (size_t)NP * 128 * sizeof(float);
  constexpr size_t smem = (ring > sums ? ring : sums) + 1024;
  CUtensorMap map_x;
  int rc = encode_rows_16bit(&map_x, a.x, F16, (uint64_t)a.w.C, (uint64_t)a.M, (uint64_t)a.x_row, 64, NP);
  if (rc != 0) return rc;
  static DeviceOnce once;
  auto kernel = k_linear_tc<F16, NP, SMALL, ZEROS>;
  if ((rc = set_max_smem(once, device, kernel, smem)) != 0) return rc;
  return launch_kernel_cluster(kernel, dim3((unsigned)(blocks * S), (unsigned)slices), dim3(tc_threads(NP)), (unsigned)S, smem, st,
                               true, a, map_x, status);
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
  if (a.M <= 16) return launch_build<F16, 16>(a, num_sms, device, status, st);
  if (a.M <= 32 || a.w.group < 128) return launch_build<F16, 32>(a, num_sms, device, status, st);
  // (64 rows of x and small groups would take more than 512 columns of tensor memory)
  return a.w.zeros ? launch_tc<F16, 64, false, true>(a, num_sms, device, status, st)
                   : launch_tc<F16, 64, false, false>(a, num_sms, device, status, st);
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
