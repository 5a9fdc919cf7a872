// Tiles of C = A B^T with both operands' K contiguous, for fp16 and 8-bit integer elements: what the orthogonalised updates
// and the 8-bit experts multiply with.
//
// A K-tile is 128 bytes of every row (64 fp16 or 128 int8), two MFMA steps of 64 bytes; byte for byte the two types are the
// same tile: v_mfma_f32_16x16x32_f16 and v_mfma_i32_16x16x64_i8 take 16 bytes of a row per lane. Operands go global -> LDS
// with direct loads through a ring of stages. A row's 16-byte chunk c lies at chunk c ^ (row & 7), so that the 16 rows of a
// fragment read cover all banks evenly.
#pragma once
#include "grouped_gemm.h"

namespace pcmoe {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

struct F16 {
  typedef floatx4 acc;
  static constexpr int size = 2;
  static __device__ __forceinline__ acc mfma(const Chunk& a, const Chunk& b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  }
};
struct I8 {
  typedef int32x4 acc;
  static constexpr int size = 1;
  static __device__ __forceinline__ acc mfma(const Chunk& a, const Chunk& b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(int32x4, a), __builtin_bit_cast(int32x4, b), c, 0, 0, 0);
  }
};

constexpr int NT_ROWB = 128;  // bytes of a tile row

template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct NtShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int NW = WM * WN, NT = 64 * NW;
  static constexpr int WTM = BM / WM, WTN = BN / WN;      // a wavefront's part of the tile
  static constexpr int FM = WTM / 16, FN = WTN / 16;
  static constexpr int IA = BM / 8 / NW, IB = BN / 8 / NW;  // direct loads (8 rows each) per wavefront and K-tile
  static constexpr int A_BYTES = BM * NT_ROWB, STAGE = (BM + BN) * NT_ROWB, LDS = STAGES * STAGE;
  static_assert(IA * 8 * NW == BM && IB * 8 * NW == BN, "tiles split evenly over the wavefronts");
};

// K loop of one tile. load_a(kt, j, dst) and load_b(kt, j, dst) issue the direct load of rows 8 j .. 8 j + 7 of K-tile kt
// to LDS address dst: lane l brings row 8 j + (l >> 3), chunk (l & 7) ^ (l >> 3) (nt_lane). Accumulators hold, in lane (q =
// lane >> 4, i = lane & 15), row i of the fragment and its columns 4 q .. 4 q + 3. `live`: this wavefront has something to
// compute (uniform); the others load and synchronise with it.
template <typename S, typename E, typename LA, typename LB>
__device__ __forceinline__ void nt_loop(char* smem, int ktiles, bool live, LA&& load_a, LB&& load_b,
                                        typename E::acc (&acc)[S::FM][S::FN]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN;
  const int q = lane >> 4, li = lane & 15;
  const uint32_t base = lds_addr(smem);
  const auto issue = [&](int kt) {
    const uint32_t st = base + (kt % S::STAGES) * S::STAGE;
#pragma unroll
    for (int j = 0; j < S::IA; ++j) load_a(kt, wave + S::NW * j, st + (wave + S::NW * j) * 1024);
#pragma unroll
    for (int j = 0; j < S::IB; ++j) load_b(kt, wave + S::NW * j, st + S::A_BYTES + (wave + S::NW * j) * 1024);
  };
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = typename E::acc{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < S::STAGES - 1; ++s)
    if (s < ktiles) issue(s);
  for (int kt = 0; kt < ktiles; ++kt) {
    if (kt + S::STAGES - 2 < ktiles) wait_vmcnt<(S::STAGES - 2) * (S::IA + S::IB)>();
    else wait_vmcnt<0>();
    // every wavefront's loads of kt have landed, and its reads of the stage that is filled next are done
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (kt + S::STAGES - 1 < ktiles) issue(kt + S::STAGES - 1);
    if (!live) continue;
    const char* As = smem + (kt % S::STAGES) * S::STAGE;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = li * NT_ROWB + (((4 * s + q) ^ (li & 7)) << 4);
      Chunk a[S::FM], b[S::FN];
#pragma unroll
      for (int i = 0; i < S::FM; ++i) a[i] = ld_chunk(As + (wm * S::WTM + 16 * i) * NT_ROWB + at);
#pragma unroll
      for (int j = 0; j < S::FN; ++j) b[j] = ld_chunk(As + S::A_BYTES + (wn * S::WTN + 16 * j) * NT_ROWB + at);
#pragma unroll
      for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = E::mfma(b[j], a[i], acc[i][j]);
    }
  }
  __syncthreads();  // the operands' LDS is free
}
// Byte offset of a lane's chunk within a direct load whose rows are ld bytes apart.
__device__ __forceinline__ int nt_lane(int ld) {
  const int l = threadIdx.x & 63;
  return (l >> 3) * ld + (((l & 7) ^ (l >> 3)) << 4);
}

// The one buffer or the other, in scalar registers (`second` is uniform).
__device__ __forceinline__ int32x4 pick_rsrc(bool second, const int32x4& a, const int32x4& b) {
  int32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(second ? b[i] : a[i]);
  return r;
}

// Workgroup bid of `total` on 8 XCDs (bid % 8 picks the XCD): consecutive results share an XCD and its L2.
__device__ __forceinline__ int xcd_order(int bid, int total) {
  const int x = bid & 7, q = total >> 3, r = total & 7;
  return x * q + min(x, r) + (bid >> 3);
}

}  // namespace pcmoe
