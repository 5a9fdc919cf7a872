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
  static __device__ __forceinline__ void mfma_agpr(acc& c, const Chunk& a, const Chunk& b) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0"
                 : "+a"(c)
                 : "v"(__builtin_bit_cast(int32x4, a)), "v"(__builtin_bit_cast(int32x4, b)));
  }
};
struct I8 {
  typedef int32x4 acc;
  static constexpr int size = 1;
  static __device__ __forceinline__ acc mfma(const Chunk& a, const Chunk& b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(int32x4, a), __builtin_bit_cast(int32x4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ void mfma_agpr(acc& c, const Chunk& a, const Chunk& b) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0"
                 : "+a"(c)
                 : "v"(__builtin_bit_cast(int32x4, a)), "v"(__builtin_bit_cast(int32x4, b)));
  }
};

constexpr int NT_ROWB = 128;  // bytes of a tile row

template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int TOGETHER_ = 1>
struct NtShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int TOGETHER = TOGETHER_;              // K-tiles between two barriers of the ring
  static constexpr int NW = WM * WN, NT = 64 * NW;
  static constexpr int WTM = BM / WM, WTN = BN / WN;      // a wavefront's part of the tile
  static constexpr int FM = WTM / 16, FN = WTN / 16;
  static constexpr int IA = BM / 8 / NW, IB = BN / 8 / NW;  // direct loads (8 rows each) per wavefront and K-tile
  static constexpr int A_BYTES = BM * NT_ROWB, STAGE = (BM + BN) * NT_ROWB, LDS = STAGES * STAGE;
  // one wavefront per SIMD with outputs of 128 columns: nt_pipe
  static constexpr bool PIPE = BM >= 128 && BN == 256 && NW == 4 && STAGES == 2;
  static_assert(IA * 8 * NW == BM && IB * 8 * NW == BN, "tiles split evenly over the wavefronts");
};

// Where a direct load takes its rows from: lane l brings row l >> 3 of eight, chunk (l & 7) ^ (l >> 3) (nt_lane).
struct NtSrc {
  int32x4 rsrc;
  int off;
};

// K loop of one tile. src_a(kt, j) and src_b(kt, j) name rows 8 j .. 8 j + 7 of K-tile kt. Accumulators hold, in lane (q =
// lane >> 4, i = lane & 15), row i of the fragment and its columns 4 q .. 4 q + 3. `live`: this wavefront has something to
// compute (uniform); the others load and synchronise with it.
template <typename S, typename E, typename LA, typename LB>
__device__ __forceinline__ void nt_ring(char* smem, int ktiles, bool live, LA&& src_a, LB&& src_b,
                                        typename E::acc (&acc)[S::FM][S::FN]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN;
  const int q = lane >> 4, li = lane & 15;
  const uint32_t base = lds_addr(smem);
  const auto issue = [&](int kt) {
    const uint32_t st = base + (kt % S::STAGES) * S::STAGE;
#pragma unroll
    for (int j = 0; j < S::IA; ++j) {
      const NtSrc a = src_a(kt, wave + S::NW * j);
      dma16(a.rsrc, st + (wave + S::NW * j) * 1024, a.off);
    }
#pragma unroll
    for (int j = 0; j < S::IB; ++j) {
      const NtSrc b = src_b(kt, wave + S::NW * j);
      dma16(b.rsrc, st + S::A_BYTES + (wave + S::NW * j) * 1024, b.off);
    }
  };
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = typename E::acc{0, 0, 0, 0};
  constexpr int G = S::TOGETHER, AHEAD = S::STAGES - G, LOADS = S::IA + S::IB;
  static_assert(S::STAGES % G == 0 && (AHEAD - G) * LOADS < 64, "whole groups of K-tiles, waited for by count");
#pragma unroll
  for (int s = 0; s < AHEAD; ++s)
    if (s < ktiles) issue(s);
  for (int k0 = 0; k0 < ktiles; k0 += G) {
    if (k0 + AHEAD <= ktiles) wait_vmcnt<(AHEAD - G) * LOADS>();
    else wait_vmcnt<0>();
    // every wavefront's loads of these K-tiles have landed, and its reads of the stages that are filled next are done
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (k0 + AHEAD + g < ktiles) issue(k0 + AHEAD + g);
    if (!live) continue;
#pragma unroll
    for (int s = 0; s < 2 * G; ++s) {
      if (G > 1 && k0 + s / 2 >= ktiles) break;
      const char* As = smem + ((k0 + s / 2) % S::STAGES) * S::STAGE;
      const int at = li * NT_ROWB + (((4 * (s & 1) + q) ^ (li & 7)) << 4);
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

// The same for 256 x 256 tiles with one wavefront per SIMD (accumulators in AGPRs). Nothing else hides a stall of a
// wavefront, so its loop is ordered by hand: while the MFMAs of a 64-byte step run, the fragments of the next step are read
// into other registers, one read after every fourth MFMA, and during a K-tile's second step the 16 direct loads of the K-tile
// after the next are issued. One barrier per K-tile, between its steps: by then every wavefront has read the K-tile's last
// fragments (its stage is free), and its loads of the next K-tile, issued a whole K-tile ago, have landed. Loads past the
// last K-tile are issued with an offset past every range: a branch around them would make the compiler move accumulators.
// 8192 x 14336 x 8192 bytes of K, products alone: 1,320 TFLOP/s fp16 and 2,650 TOP/s int8, against 980 and 1,980 of the
// 128 x 128 tiles, and 1,260 and 2,460 of the same loop with eight wavefronts of 128 x 64, whose fragments pass LDS 1.5 times
// as often.
// A workgroup that goes on to another tile calls nt_fill for it before the epilogue of the last one, so that its first two
// K-tiles are under way meanwhile; `behind` says that the wavefront has issued at least 16 stores since.
template <typename S, typename LA, typename LB>
__device__ __forceinline__ void nt_load(uint32_t base, int ktiles, int kt, int l, LA&& src_a, LB&& src_b) {
  constexpr int OOR = 0x7fffffff;  // no operand has 2^31 bytes
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & (S::NW - 1);  // what of a row's number is l's, is known
  const uint32_t st = base + (kt & 1) * S::STAGE;
  const NtSrc s = l < S::IA ? src_a(kt, wave + S::NW * l) : src_b(kt, wave + S::NW * (l - S::IA));
  const uint32_t dst = l < S::IA ? st + (wave + S::NW * l) * 1024 : st + S::A_BYTES + (wave + S::NW * (l - S::IA)) * 1024;
  dma16(s.rsrc, dst, kt < ktiles ? s.off : OOR);
}
template <typename S, typename LA, typename LB>
__device__ __forceinline__ void nt_fill(char* smem, int ktiles, LA&& src_a, LB&& src_b) {
  const uint32_t base = lds_addr(smem);
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int l = 0; l < S::IA + S::IB; ++l) nt_load<S>(base, ktiles, kt, l, src_a, src_b);
}
template <typename S, typename E, typename LA, typename LB>
__device__ __forceinline__ void nt_pipe(char* smem, int ktiles, bool live, bool behind, LA&& src_a, LB&& src_b,
                                        typename E::acc (&acc)[S::FM][S::FN]) {
  static_assert(S::STAGES == 2, "two stages");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
  const uint32_t base = lds_addr(smem);
  constexpr int LOADS = S::IA + S::IB, NF = S::FM + S::FN, NM = S::FM * S::FN;
  constexpr int RS = NM / NF, LS = NM / LOADS;  // MFMAs for each read, and for each load
  const auto load = [&](int kt, int l) { nt_load<S>(base, ktiles, kt, l, src_a, src_b); };
  const int at0 = li * NT_ROWB + ((q ^ (li & 7)) << 4), at1 = li * NT_ROWB + (((4 + q) ^ (li & 7)) << 4);
  const char* a0 = smem + wm * S::WTM * NT_ROWB;
  const char* b0 = smem + S::A_BYTES + wn * S::WTN * NT_ROWB;
  Chunk fa[2][S::FM], fb[2][S::FN];
  // read t of step s of K-tile kt, in the order in which the MFMAs take them: A's first, B's, A's others
  const auto read = [&](int kt, int s, int t) {
    const int st = (kt & 1) * S::STAGE + (s ? at1 : at0);
    if (t == 0) fa[s][0] = ld_chunk(a0 + st);
    else if (t <= S::FN) fb[s][t - 1] = ld_chunk(b0 + st + 16 * (t - 1) * NT_ROWB);
    else fa[s][t - S::FN] = ld_chunk(a0 + st + 16 * (t - S::FN) * NT_ROWB);
  };
  const auto barrier = [] {
    wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = typename E::acc{0, 0, 0, 0};
  if (behind) wait_vmcnt<16>();  // the loads are older than the last 16 stores
  else wait_vmcnt<0>();
  asm volatile("s_barrier" ::: "memory");
  if (!live) {
    for (int kt = 0; kt < ktiles; ++kt) {
      barrier();
#pragma unroll
      for (int l = 0; l < LOADS; ++l) load(kt + 2, l);
    }
  } else {
#pragma unroll
    for (int t = 0; t < NF; ++t) read(0, 0, t);
    for (int kt = 0; kt < ktiles; ++kt) {
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        E::mfma_agpr(acc[m / S::FN][m % S::FN], fb[0][m % S::FN], fa[0][m / S::FN]);
        if (m % RS == 0 && m / RS < NF) read(kt, 1, m / RS);
        __builtin_amdgcn_sched_barrier(0);
      }
      barrier();
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        E::mfma_agpr(acc[m / S::FN][m % S::FN], fb[1][m % S::FN], fa[1][m / S::FN]);
        if (m % RS == 0 && m / RS < NF) read(kt + 1, 0, m / RS);
        if (m % LS == LS / 2 && m / LS < LOADS) load(kt + 2, m / LS);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  wait_vmcnt<0>();  // the loads past the last K-tile have landed before the LDS is used again
  asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");  // the last MFMAs' results are ready to read
  __syncthreads();
}

template <typename S, typename E, typename LA, typename LB>
__device__ __forceinline__ void nt_loop(char* smem, int ktiles, bool live, LA&& src_a, LB&& src_b,
                                        typename E::acc (&acc)[S::FM][S::FN]) {
  if constexpr (S::PIPE) {
    nt_fill<S>(smem, ktiles, src_a, src_b);
    nt_pipe<S, E>(smem, ktiles, live, false, src_a, src_b, acc);
  } else {
    nt_ring<S, E>(smem, ktiles, live, src_a, src_b, acc);
  }
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
