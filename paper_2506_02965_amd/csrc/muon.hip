// Update of the experts' matrices by their orthogonalised momentum.
//
// m <- mu m + g, u = g + mu m or m, X = u / (|u|_F + eps); then a fixed number of Newton-Schulz steps
//   A = X X^T,  P = a + b A + c A^2,  X <- P X,
// taken with X's rows no longer than its columns' number (of a tall matrix X is the transpose), and p <- p (1 - lr wd) -
// lr scale X. A step of an m x n matrix takes m^2 n (A, half of a symmetric product) + m^3 (A^2, the other) + 2 m^2 n
// operations, all on the fp16 matrix cores: bound by them, and at small sizes by the launches in a row.
//
// Six matrices of 4096 x 14336: 14.4 ms, of which A = X X^T takes 1.26 a time (1,150 TFLOP/s of what the definition needs), X
// <- P X 2.41 (1,200), a product of 4096^3 0.40; momentum, norm and the first X 1.42 at the memory's rate.
//
// All three are products of two K-contiguous operands: A = X X^T reads X, A^2 reads A = A^T, and P X reads P and X^T. So X is
// kept in both orientations, each written by the epilogue that makes it. Of a symmetric product only the tiles on and above
// the diagonal are computed; each is stored twice. The last step's epilogue updates the parameters.
//
// X, A and P are held in fp16 after powers of two that keep them below 2^15: |X| never passes the polynomial's largest value
// on [0, 1], which the host knows. Eleven bits leave X some 2^-10 of its size off (muon_group has figures); in the precise form
// each is held in two fp16 parts (22 bits) and three products are added up, smallest first. Sums are fp32, the momentum fp32,
// the norm fp64.
#include "nt_gemm.h"
#include "expert_ops.h"

#include <algorithm>
#include <cmath>

namespace pcmoe {

namespace {

typedef _Float16 f16;

constexpr int SUM_BLOCKS = 64;  // partial sums of squares of a matrix

struct MuonArgs {
  void* w[3];
  const void* g[3];
  int G;             // experts: matrices of a tensor
  int mat0;          // the first matrix of this pass, of [gate, up, down][G]
  int d, f;
  float *master, *m; // [3][G][f d]
  double* part;      // [matrices of a pass][SUM_BLOCKS]
  float mu;
  int nesterov;
  double eps;
  f16 *x, *xt;       // [matrices of a pass][parts][m][n], [..][parts][n][m]
  float s0;          // power of two of the first X
  int wide_first;    // gate and up are wide (f <= d)
};

__device__ __forceinline__ void momentum(const MuonArgs& a, float g, float& m) { m = a.mu * m + g; }
__device__ __forceinline__ float update_of(const MuonArgs& a, float g, float m) {
  return a.nesterov ? g + a.mu * m : m;
}

// m <- mu m + g, and partial sums of u^2. blockIdx.y: the matrix.
template <typename T>
__global__ __launch_bounds__(256) void muon_momentum_kernel(MuonArgs a) {
  constexpr int EP = EPC<T>::value;
  const int mat = a.mat0 + (int)blockIdx.y;
  const int64_t n = (int64_t)a.d * a.f / EP;  // chunks
  const Chunk* g = (const Chunk*)a.g[mat / a.G] + (size_t)(mat % a.G) * n;
  float* mm = a.m + (size_t)mat * a.d * a.f;
  double sum = 0.;
  const int64_t per = (n + SUM_BLOCKS - 1) / SUM_BLOCKS, c1 = min((int64_t)n, per * (blockIdx.x + 1));
  for (int64_t c = per * blockIdx.x + threadIdx.x; c < c1; c += 256) {
    float gv[EP];
    chunk_to_f<T>(ld_chunk_nt(g + c), gv);
#pragma unroll
    for (int h = 0; h < EP; h += 4) {
      float mv[4];
      chunk_to_f<float>(ld_chunk(mm + c * EP + h), mv);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        momentum(a, gv[h + e], mv[e]);
        const double u = (double)update_of(a, gv[h + e], mv[e]);
        sum += u * u;
      }
      st_chunk(mm + c * EP + h, f_to_chunk<float>(mv));
    }
  }
  __shared__ double s[256];
  s[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) s[threadIdx.x] += s[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.part[(size_t)blockIdx.y * SUM_BLOCKS + blockIdx.x] = s[0];
}

// fp16 parts of a value: its rounding, and the rounding of the rest.
__device__ __forceinline__ f16 part_of(float v, bool second) {
  const f16 hi = (f16)v;
  return second ? (f16)(v - (float)hi) : hi;
}

// X = s0 u / (|u| + eps) in both orientations, by tiles of 64 x 64 of the matrix as it is stored.
template <typename T, bool PRECISE>
__global__ __launch_bounds__(256) void muon_normalise_kernel(MuonArgs a) {
  constexpr int EP = EPC<T>::value;
  // the last rows of the last matrices first: they are what the pass before this left in the last-level cache
  const int here = (int)gridDim.y - 1 - (int)blockIdx.y, mat = a.mat0 + here, tensor = mat / a.G;
  const int rows = tensor == 2 ? a.d : a.f, cols = tensor == 2 ? a.f : a.d;
  const int l = (int)gridDim.x - 1 - (int)blockIdx.x, tr = l / (cols / 64), tc = l % (cols / 64);
  __shared__ double norm2;
  __shared__ f16 tile[PRECISE ? 2 : 1][64][72];
  const size_t at = (size_t)mat * a.d * a.f, part = (size_t)a.d * a.f, at_x = here * part * (PRECISE ? 2 : 1);
  const T* g = (const T*)a.g[tensor] + (size_t)(mat % a.G) * a.d * a.f;
  const bool flip = rows > cols;  // stored tall: X is the transpose
  f16* straight = flip ? a.xt : a.x;
  f16* turned = flip ? a.x : a.xt;
  constexpr int PER_ROW = 64 / EP, TASKS = 64 * PER_ROW / 256;
  Chunk gc[TASKS], mc[TASKS][EP / 4];  // on their way while the norm is formed
#pragma unroll
  for (int k = 0; k < TASKS; ++k) {
    const int task = threadIdx.x + 256 * k, r = task / PER_ROW, c = (task % PER_ROW) * EP;
    const size_t src = (size_t)(tr * 64 + r) * cols + tc * 64 + c;
    gc[k] = ld_chunk(g + src);
#pragma unroll
    for (int h = 0; h < EP / 4; ++h) mc[k][h] = ld_chunk(a.m + at + src + 4 * h);
  }
  if (threadIdx.x < 64) {
    double s = a.part[(size_t)here * SUM_BLOCKS + threadIdx.x];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (threadIdx.x == 0) norm2 = s;
  }
  __syncthreads();
  const double inv = (double)a.s0 / (sqrt(norm2) + a.eps);
#pragma unroll
  for (int k = 0; k < TASKS; ++k) {
    const int task = threadIdx.x + 256 * k, r = task / PER_ROW, c = (task % PER_ROW) * EP;
    float gv[EP], mv[EP];
    chunk_to_f<T>(gc[k], gv);
#pragma unroll
    for (int h = 0; h < EP / 4; ++h) chunk_to_f<float>(mc[k][h], mv + 4 * h);
#pragma unroll
    for (int p = 0; p < (PRECISE ? 2 : 1); ++p)
#pragma unroll
      for (int e = 0; e < EP; ++e)
        tile[p][r][c + e] = part_of((float)((double)update_of(a, gv[e], mv[e]) * inv), p != 0);
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < (PRECISE ? 2 : 1); ++p)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int task = threadIdx.x + 256 * k, r = task >> 3, c = (task & 7) * 8;
      st_chunk(straight + at_x + p * part + (size_t)(tr * 64 + r) * cols + tc * 64 + c,
               *reinterpret_cast<const Chunk*>(&tile[p][r][c]));
      half8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile[p][c + e][r];
      st_chunk(turned + at_x + p * part + (size_t)(tc * 64 + r) * rows + tr * 64 + c, __builtin_bit_cast(Chunk, v));
    }
}

// One product of every matrix: out = alpha P Q^T (+ beta D + diag on the diagonal), P [M][K], Q [N][K], D and out [M][N]; in the
// precise form each matrix is followed by its second part.
struct NsArgs {
  const f16 *p, *q, *d;
  f16 *out, *out_t;        // out, and its transpose [N][M]
  int M, N, K, mats;
  int whole;               // tiles that are not split into quarters
  float alpha, beta, diag;
  float* partial;          // NS_PARTIAL: [ksplit][mats][M][N]
  int ksplit;
  // a second product of the same shape by the same P, in the same launch
  const f16* q2;
  f16* out2;
  float alpha2;
  // last step: parameters in place of out
  void* w[3];
  float* master;
  int mat0, G, dtype;
  int flip_up, flip_down;  // gate and up, down are stored transposed to X
  float decay, step;       // p <- decay p - step X
};

// Stores: one tile and its mirror, both orientations, the parameters, or a part of a symmetric product's sums over K. (That of the
// parameters spills 276 bytes a lane in the 256 x 256 tiles, whose results take 256 registers meanwhile.)
enum NsMode { NS_SYMMETRIC, NS_BOTH, NS_LAST, NS_PARTIAL };

// LDS of an epilogue: a wavefront's part transposed, [WTN][WTM] fp16 with rows of PITCH words, or for parameters stored
// transposed to X half of it in fp32. Rows an odd multiple of 4 words apart spread the writes over all banks.
template <typename S, int MODE>
struct NsLds {
  static constexpr int PITCH = S::WTM / 2 + 4, PITCH32 = S::WTM + 4;
  static constexpr int WAVE = MODE == NS_LAST ? S::WTN / 2 * PITCH32 * 4 : S::WTN * PITCH * 4;
  static constexpr int BYTES = S::LDS > S::NW * WAVE ? S::LDS : S::NW * WAVE;
};

// Two column blocks of a fragment row (four consecutive columns a lane each) -> eight consecutive columns a lane: of the first
// block in the even rows of 16 lanes, of the second in the odd ones, starting at column 8 (q >> 1).
__device__ __forceinline__ void join_columns(const floatx4& a, const floatx4& b, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[e]), __float_as_uint(b[e]), false, false);
    v[e] = __uint_as_float(r[0]);
    v[4 + e] = __uint_as_float(r[1]);
  }
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b, bool second) {
  return (uint32_t)__builtin_bit_cast(uint16_t, part_of(a, second)) |
         (uint32_t)__builtin_bit_cast(uint16_t, part_of(b, second)) << 16;
}

// The tile of matrix `mat` whose first row and column are m0 and n0.
template <typename S, int MODE, bool PRECISE>
__device__ __forceinline__ void product_tile(const NsArgs& a, char* smem, int mat, bool other, int m0, int n0, int split = 0) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
  const int ld = a.K * 2;
  constexpr int PARTS = PRECISE ? 2 : 1;
  // Both parts of a matrix are one buffer, so that choosing between them is an offset. (A row past the first part's end, of which
  // nothing is stored, reads the second's.)
  const uint32_t p_part = (uint32_t)a.M * ld, q_part = (uint32_t)a.N * ld;
  const int32x4 rp = make_rsrc(a.p + mat * ((size_t)PARTS * a.M * a.K), PARTS * p_part);
  const int32x4 rq = make_rsrc((other ? a.q2 : a.q) + mat * ((size_t)PARTS * a.N * a.K), PARTS * q_part);
  const int kts = a.K / 64, at = nt_lane(ld);
  // the wavefronts' parts lie on either side of a matrix's end, not across it: the sides are multiples of 128
  const bool live = m0 + wm * S::WTM < a.M && n0 + wn * S::WTN < a.N;
  typename F16::acc acc[S::FM][S::FN];
  // K-tiles kt: of a precise product first P1 Q2, then P2 Q1, then P1 Q1
  const int all = PRECISE ? 3 * kts : kts;
  const int k0 = MODE == NS_PARTIAL ? all * split / a.ksplit : 0, k1 = MODE == NS_PARTIAL ? all * (split + 1) / a.ksplit : all;
  nt_loop<S, F16>(
      smem, k1 - k0, live,
      [&](int kt, int j) {
        if (MODE == NS_PARTIAL) kt += k0;
        const int seg = PRECISE ? (kt >= 2 * kts ? 2 : kt >= kts ? 1 : 0) : 0;
        return NtSrc{rp, (m0 + 8 * j) * ld + at + (kt - seg * kts) * NT_ROWB + (PRECISE && seg == 1 ? (int)p_part : 0)};
      },
      [&](int kt, int j) {
        if (MODE == NS_PARTIAL) kt += k0;
        const int seg = PRECISE ? (kt >= 2 * kts ? 2 : kt >= kts ? 1 : 0) : 0;
        return NtSrc{rq, (n0 + 8 * j) * ld + at + (kt - seg * kts) * NT_ROWB + (PRECISE && seg == 0 ? (int)q_part : 0)};
      },
      acc);
  if (!live) return;
  const int mr = m0 + wm * S::WTM, nc = n0 + wn * S::WTN;  // the wavefront's part
  const size_t part = (size_t)a.M * a.N;                     // elements of a part of the result

  if constexpr (MODE == NS_PARTIAL) {
    float* to = a.partial + ((size_t)split * a.mats + mat) * part;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
      for (int j = 0; j < S::FN; ++j)
        *reinterpret_cast<floatx4*>(to + (size_t)(mr + 16 * i + li) * a.N + nc + 16 * j + 4 * q) = acc[i][j];
  } else if constexpr (MODE == NS_LAST) {
    const int tensor = (a.mat0 + mat) / a.G;
    const size_t at_w = (size_t)((a.mat0 + mat) % a.G) * part;
    float* mp = a.master ? a.master + (size_t)tensor * a.G * part + at_w : nullptr;
    void* const w = tensor == 0 ? a.w[0] : tensor == 1 ? a.w[1] : a.w[2];
    float* wf = (float*)w + at_w;
    bf16* wb = (bf16*)w + at_w;
    // with the parameters' type and whether there is a master copy known, so that nothing in the loops branches
    const auto keep = [&] {  // the accumulators stay where they are until a path takes them
#pragma unroll
      for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) asm volatile("" : "+a"(acc[i][j]));
    };
    const auto update = [&](auto f32, auto has_master) {
      constexpr bool F32 = decltype(f32)::value, MASTER = decltype(has_master)::value;
      // eight consecutive parameters from element o on
      const auto fetch = [&](size_t o, Chunk (&c)[2]) {
        if constexpr (F32 || MASTER) {
          const float* from = (MASTER ? mp : wf) + o;
          c[0] = ld_chunk(from);
          c[1] = ld_chunk(from + 4);
        } else {
          c[0] = c[1] = ld_chunk(wb + o);
        }
      };
      const auto store = [&](size_t o, const Chunk (&c)[2], const float (&x)[8]) {
        float p[8];
        if constexpr (F32 || MASTER) {
          chunk_to_f<float>(c[0], p);
          chunk_to_f<float>(c[1], p + 4);
        } else {
          chunk_to_f<bf16>(c[0], p);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = a.decay * p[e] - a.step * (a.alpha * x[e]);
        if constexpr (MASTER) {
          st_chunk(mp + o, f_to_chunk<float>(p));
          st_chunk(mp + o + 4, f_to_chunk<float>(p + 4));
        }
        if constexpr (F32) {
          st_chunk(wf + o, f_to_chunk<float>(p));
          st_chunk(wf + o + 4, f_to_chunk<float>(p + 4));
        } else {
          st_chunk(wb + o, f_to_chunk<bf16>(p));
        }
      };
      if (!(tensor == 2 ? a.flip_down : a.flip_up)) {
        keep();
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          const size_t o = (size_t)(mr + 16 * i + li) * a.N + nc + 16 * (q & 1) + 8 * (q >> 1);
          Chunk c[S::FN / 2][2];
#pragma unroll
          for (int j = 0; j < S::FN / 2; ++j) fetch(o + 32 * j, c[j]);
#pragma unroll
          for (int j = 0; j < S::FN / 2; ++j) {
            float v[8];
            join_columns(acc[i][2 * j], acc[i][2 * j + 1], v);
            store(o + 32 * j, c[j], v);
          }
        }
      } else {
        constexpr int PITCH = NsLds<S, MODE>::PITCH32, CH = S::WTM / 8;
        float* st = reinterpret_cast<float*>(smem + wave * NsLds<S, MODE>::WAVE);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          keep();
#pragma unroll
          for (int i = 0; i < S::FM; ++i, __builtin_amdgcn_sched_barrier(0))
#pragma unroll
            for (int j = 0; j < S::FN / 2; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) st[(16 * j + 4 * q + e) * PITCH + 16 * i + li] = acc[i][half * (S::FN / 2) + j][e];
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          constexpr int ALL = S::WTN / 2 * CH, TASKS = (ALL + 63) / 64, AHEAD = TASKS < 4 ? TASKS : 4;
#pragma unroll 1
          for (int k0 = 0; k0 < TASKS; k0 += AHEAD) {
            Chunk c[AHEAD][2];
            size_t o[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
              const int task = lane + 64 * (k0 + k);
              o[k] = (size_t)(nc + half * (S::WTN / 2) + task / CH) * a.M + mr + (task % CH) * 8;
              if (ALL % 64 == 0 || task < ALL) fetch(o[k], c[k]);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
              const int task = lane + 64 * (k0 + k);
              if (ALL % 64 != 0 && task >= ALL) continue;
              const float* from = st + (task / CH) * PITCH + (task % CH) * 8;
              float v[8];
              chunk_to_f<float>(ld_chunk(from), v);
              chunk_to_f<float>(ld_chunk(from + 4), v + 4);
              store(o[k], c[k], v);
            }
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    };
    if (a.dtype == MOE_F32) {
      if (mp) update(std::true_type{}, std::true_type{});
      else update(std::true_type{}, std::false_type{});
    } else {
      if (mp) update(std::false_type{}, std::true_type{});
      else update(std::false_type{}, std::false_type{});
    }
    return;
  } else {
    f16* out = (other ? a.out2 : a.out) + mat * PARTS * part;
    f16* out_t = (MODE == NS_SYMMETRIC ? (other ? a.out2 : a.out) : a.out_t) + mat * PARTS * part;
    const float alpha = other ? a.alpha2 : a.alpha;
    const f16* d0 = MODE == NS_SYMMETRIC && a.d ? a.d + mat * PARTS * part : nullptr;
    const bool turn = MODE == NS_BOTH || m0 != n0;
    constexpr int PITCH = NsLds<S, MODE>::PITCH;
    uint32_t* st = reinterpret_cast<uint32_t*>(smem + wave * NsLds<S, MODE>::WAVE);
    const bool odd = lane & 1;
    const uint32_t sel_lo = odd ? 0x01000504u : 0x05040100u, sel_hi = odd ? 0x03020706u : 0x07060302u;
#pragma unroll 1
    for (int p = 0; p < (PRECISE ? 2 : 1); ++p) {
      float by = alpha;
      int row = li;
      if (PRECISE) asm volatile("" : "+v"(by), "+v"(row));  // keeps what both parts compute from being kept in registers
#pragma unroll
      for (int i = 0; i < S::FM; ++i) {
        __builtin_amdgcn_sched_barrier(0);  // one row of blocks out of the accumulators at a time: more would spill
        floatx4 x[S::FN];
#pragma unroll
        for (int j = 0; j < S::FN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j][e] = by * acc[i][j][e];
        if (d0) {
          typedef _Float16 half4 __attribute__((ext_vector_type(4)));
          const int m = mr + 16 * i + row;
          const size_t o = (size_t)m * a.N + nc + 4 * q;
          half4 dv[S::FN], d1[S::FN];
#pragma unroll
          for (int j = 0; j < S::FN; ++j) {
            dv[j] = *reinterpret_cast<const half4*>(d0 + o + 16 * j);
            if (PRECISE) d1[j] = *reinterpret_cast<const half4*>(d0 + part + o + 16 * j);
          }
#pragma unroll
          for (int j = 0; j < S::FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[j][e] += a.beta * ((float)dv[j][e] + (PRECISE ? (float)d1[j][e] : 0.f));
              if (m == nc + 16 * j + 4 * q + e) x[j][e] += a.diag;
            }
        }
        // by rows, from registers
#pragma unroll
        for (int j = 0; j < S::FN / 2; ++j) {
          float v[8];
          join_columns(x[2 * j], x[2 * j + 1], v);
          Chunk c;
#pragma unroll
          for (int e = 0; e < 4; ++e) c.w[e] = pack_f16(v[2 * e], v[2 * e + 1], p != 0);
          st_chunk(out + p * part + (size_t)(mr + 16 * i + row) * a.N + nc + 32 * j + 16 * (q & 1) + 8 * (q >> 1), c);
        }
        // by columns, through LDS: neighbouring lanes (rows m and m + 1) exchange halves, the even one keeps columns 0 and 1 of
        // its four, the odd one 2 and 3
        if (!turn) continue;
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
          const uint32_t c01 = pack_f16(x[j][0], x[j][1], p != 0), c23 = pack_f16(x[j][2], x[j][3], p != 0);
          const uint32_t keep = odd ? c23 : c01, give = odd ? c01 : c23;
          const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0xb1, 0xf, 0xf, true);
          uint32_t* to = st + (16 * j + 4 * q + (odd ? 2 : 0)) * PITCH + 8 * i + (row >> 1);
          to[0] = __builtin_amdgcn_perm(got, keep, sel_lo);
          to[PITCH] = __builtin_amdgcn_perm(got, keep, sel_hi);
        }
      }
      if (!turn) continue;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      constexpr int CH = S::WTM / 8;
#pragma unroll
      for (int k = 0; k < S::WTN * CH / 64; ++k) {
        const int task = lane + 64 * k, r = task / CH, c = task % CH;
        st_chunk(out_t + p * part + (size_t)(nc + r) * a.M + mr + 8 * c, ld_chunk(st + r * PITCH + 4 * c));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// 256 x 256 tiles with one wavefront per SIMD, 128 x 128 tiles two workgroups a CU, and the quarters of 256 x 256 tiles, which
// share a launch with them. While all tiles are multiplied at once a launch is bound by latencies, the more K-tiles on their way
// the better: 64 x 64 tiles, and 32 x 32 tiles with up to 18 K-tiles (three matrices of 384 rows, K = 384 in two parts: 7.0 us a
// launch, with 64 x 64 tiles of four or eight wavefronts 10.4 and 8.1; an empty launch is 1.5).
typedef NtShape<256, 256, 2, 2, 2> NsLarge;
typedef NtShape<128, 128, 2, 2, 4> NsQuarter;
typedef NtShape<128, 128, 2, 2, 2> NsSmall;
typedef NtShape<64, 64, 4, 2, 8, 2> NsTiny;
typedef NtShape<32, 32, 2, 1, 18, 6> NsTiniest;

// Tile l of a grid of `tm` x `tn` tiles of every matrix (for symmetric products, of those on and above the diagonal).
template <int MODE>
__device__ __forceinline__ void ns_tile(const NsArgs& a, int l, int tm, int tn, int& mat, bool& other, int& mt, int& nt) {
  constexpr bool SYM = MODE == NS_SYMMETRIC || MODE == NS_PARTIAL;
  const int per = SYM ? tm * (tm + 1) / 2 : tm * tn;
  other = MODE == NS_SYMMETRIC && l >= per * a.mats;
  if (other) l -= per * a.mats;
  mat = l / per;
  l -= mat * per;
  if (SYM) {  // nt >= mt, by columns: nt (nt + 1) / 2 tiles stand before column nt
    nt = (int)((sqrtf(8.f * (float)l + 1.f) - 1.f) * 0.5f);
    while (nt * (nt + 1) / 2 > l) --nt;
    while ((nt + 1) * (nt + 2) / 2 <= l) ++nt;
    mt = l - nt * (nt + 1) / 2;
  } else {  // eight row tiles at a time, so that neighbours share both operands
    const int blk = l / (8 * tn), rem = l - blk * 8 * tn, rows = min(8, tm - 8 * blk);
    nt = rem / rows;
    mt = 8 * blk + rem % rows;
  }
  mat = __builtin_amdgcn_readfirstlane(mat);
  mt = __builtin_amdgcn_readfirstlane(mt);
  nt = __builtin_amdgcn_readfirstlane(nt);
}

template <typename S, int MODE, bool PRECISE>
__global__ __launch_bounds__(S::NT) void muon_product_kernel(NsArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tm = (a.M + S::BM - 1) / S::BM, tn = (a.N + S::BN - 1) / S::BN;
  int mat, mt, nt;
  bool other;
  if constexpr (MODE == NS_PARTIAL) {
    const int l = xcd_order(blockIdx.x, (int)gridDim.x), tile = l / a.ksplit;
    ns_tile<MODE>(a, tile, tm, tn, mat, other, mt, nt);
    product_tile<S, MODE, PRECISE>(a, smem, mat, other, mt * S::BM, nt * S::BN, l - tile * a.ksplit);
  } else if (!S::PIPE || (int)blockIdx.x < a.whole) {
    ns_tile<MODE>(a, xcd_order(blockIdx.x, S::PIPE ? a.whole : (int)gridDim.x), tm, tn, mat, other, mt, nt);
    product_tile<S, MODE, PRECISE>(a, smem, mat, other, mt * S::BM, nt * S::BN);
  } else {  // a quarter of one of the last tiles
    const int l = xcd_order(blockIdx.x - a.whole, (int)gridDim.x - a.whole);
    ns_tile<MODE>(a, a.whole + l / 4, tm, tn, mat, other, mt, nt);
    const int m0 = mt * S::BM + (l >> 1 & 1) * (S::BM / 2), n0 = nt * S::BN + (l & 1) * (S::BN / 2);
    if (m0 >= a.M || n0 >= a.N || (MODE == NS_SYMMETRIC && m0 > n0)) return;  // below the diagonal: the mirror of another
    product_tile<NsQuarter, MODE, PRECISE>(a, smem, mat, other, m0, n0);
  }
}

// The parts of a symmetric product's sums added up in order, times alpha: a 32 x 32 block on or above the diagonal, and its
// mirror. blockIdx.y: the matrix.
template <bool PRECISE>
__global__ __launch_bounds__(256) void muon_join_kernel(NsArgs a) {
  constexpr int PARTS = PRECISE ? 2 : 1;
  __shared__ float block[32][33];
  int bc = (int)((sqrtf(8.f * (float)blockIdx.x + 1.f) - 1.f) * 0.5f);
  while (bc * (bc + 1) / 2 > (int)blockIdx.x) --bc;
  while ((bc + 1) * (bc + 2) / 2 <= (int)blockIdx.x) ++bc;
  const int br = blockIdx.x - bc * (bc + 1) / 2, mat = blockIdx.y, r = threadIdx.x >> 3, c = 4 * (threadIdx.x & 7);
  const size_t part = (size_t)a.M * a.N;
  const float* from = a.partial + mat * part + (size_t)(32 * br + r) * a.N + 32 * bc + c;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.ksplit; ++s) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(from + (size_t)s * a.mats * part);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += v[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) block[r][c + e] = a.alpha * sum[e];
  __syncthreads();
  f16* out = a.out + mat * PARTS * part;
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    const uint2 straight = {pack_f16(block[r][c], block[r][c + 1], p != 0), pack_f16(block[r][c + 2], block[r][c + 3], p != 0)};
    const uint2 turned = {pack_f16(block[c][r], block[c + 1][r], p != 0), pack_f16(block[c + 2][r], block[c + 3][r], p != 0)};
    *reinterpret_cast<uint2*>(out + p * part + (size_t)(32 * br + r) * a.N + 32 * bc + c) = straight;
    if (br != bc) *reinterpret_cast<uint2*>(out + p * part + (size_t)(32 * bc + r) * a.N + 32 * br + c) = turned;
  }
}

template <typename S, int MODE>
int64_t ns_tiles(const NsArgs& a) {
  const int64_t tm = (a.M + S::BM - 1) / S::BM, tn = (a.N + S::BN - 1) / S::BN;
  return (MODE == NS_SYMMETRIC ? tm * (tm + 1) / 2 * (a.q2 ? 2 : 1) : MODE == NS_PARTIAL ? tm * (tm + 1) / 2 * a.ksplit : tm * tn) *
         a.mats;
}

template <typename S, int MODE, bool PRECISE>
hipError_t ns_launch(const char* name, NsArgs a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kern = muon_product_kernel<S, MODE, PRECISE>;
  constexpr int lds = S::PIPE && NsLds<NsQuarter, MODE>::BYTES > NsLds<S, MODE>::BYTES ? NsLds<NsQuarter, MODE>::BYTES : NsLds<S, MODE>::BYTES;
  if (hipError_t e = lds_limit_once((const void*)kern, lds, done); e != hipSuccess) return e;
  int64_t tiles = ns_tiles<S, MODE>(a);
  a.whole = (int)tiles;
  if (S::PIPE) {
    // A last round of few tiles is split into quarters, which take about 0.4 of a tile's time each (six matrices of 4096 rows, 816
    // tiles of 3.2 rounds, K = 14336: 1402 us, 1236 with the last 48 in quarters; K = 4096: 425, 394).
    const int64_t cus = device_cus(), rest = tiles % cus;
    if (4 * rest <= 2 * cus) {
      a.whole = (int)(tiles - rest);
      tiles += 3 * rest;
    }
  }
  KernelTimer kt(name, s);
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(S::NT), lds, s, a);
  return hipGetLastError();
}
// Rounds of n 256 x 256 tiles, a last one of few tiles in quarters.
double rounds_of(int64_t n, int64_t cus) {
  const int64_t rest = n % cus;
  return (double)(n / cus) + (rest == 0 ? 0. : 4 * rest <= cus ? 0.4 : 4 * rest <= 2 * cus ? 0.8 : 1.);
}

template <int MODE>
hipError_t ns_product(const char* name, const NsArgs& a, bool precise, hipStream_t s) {
  const auto go = [&](auto shape) {
    using S = decltype(shape);
    return precise ? ns_launch<S, MODE, true>(name, a, s) : ns_launch<S, MODE, false>(name, a, s);
  };
  // Rounds of the chip, each priced by a tile's time: 4 units of the 128 x 128 tile's work at 1.4 times its rate (a last round in
  // quarters 0.4 or 0.8 of that), two such tiles at once, the smaller ones where both cost the same. 48 matrices of 1024 x 2816: A 170
  // and 204 us, P 82 and 94, X 346 and 407; 27 of 1024 x 1536 (A and P cost the same) 74 and 73, 58 and 52, X 122 and 142.
  // The prices hold for 16 K-tiles and more. Where there are four to six, storing is most of a tile's time, which they leave out: 24
  // matrices of 384 x 2176 take the larger tiles at 46.5 and 58.4 us for X and the parameters (128 x 128 tiles: 38.0 and 44.5), 24
  // of 256 x 2560 at 32.2 for the parameters (24.6).
  const int64_t cus = device_cus();
  const double large = rounds_of(ns_tiles<NsLarge, MODE>(a), cus) * 4 / 1.4;
  const int64_t n = ns_tiles<NsSmall, MODE>(a);
  const double small = n <= cus ? 1.1 : (double)((n + 2 * cus - 1) / (2 * cus)) * 2;  // alone on a CU a tile is faster
  if (ns_tiles<NsTiniest, MODE>(a) <= cus) return go(NsTiniest{});
  if (ns_tiles<NsTiny, MODE>(a) <= cus) return go(NsTiny{});
  return large < small ? go(NsLarge{}) : go(NsSmall{});
}

hipError_t ns_gram_split(const NsArgs& a, bool tiniest, bool precise, hipStream_t s) {
  const auto go = [&](auto shape) {
    using S = decltype(shape);
    return precise ? ns_launch<S, NS_PARTIAL, true>("muon_gram", a, s) : ns_launch<S, NS_PARTIAL, false>("muon_gram", a, s);
  };
  if (hipError_t e = tiniest ? go(NsTiniest{}) : go(NsTiny{}); e != hipSuccess) return e;
  const int tm = a.M / 32;
  const dim3 grid((unsigned)(tm * (tm + 1) / 2), a.mats);
  KernelTimer kt("muon_join", s);
  if (precise) hipLaunchKernelGGL(muon_join_kernel<true>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(muon_join_kernel<false>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

// Matrices taken at a time, from X to the parameters: as few as fill the chip, since the workspace is theirs alone (192 matrices
// of 1408 x 2048: twelve at a time 0.45 GB and 19.2 ms, all 7.1 GB and 19.0 ms; 48 of 1024 x 2816: 24 at a time 2.65 ms, all
// 2.70). The least number whose symmetric products take a round of the chip and, 3% aside, no more rounds in all than all
// matrices at once (a last round in quarters: 0.4, or 0.8 of a round), the last pass at least half full.
int muon_pass(int m, int mats) {
  const int64_t tm = (m + 255) / 256, tiles = tm * (tm + 1) / 2, cus = 256;
  const auto cost = [&](int64_t n) { return rounds_of(n * tiles, cus); };
  for (int n = 1; n < mats; ++n) {
    const int last = mats % n;
    if (n * tiles * 10 < cus * 9 || (last && 2 * last < n)) continue;
    if ((mats / n) * cost(n) + cost(last) <= 1.03 * cost(mats)) return n;
  }
  return mats;
}

// A = X X^T of few rows and long K would leave most CUs idle while some walk over all of K: its sums are split over K, and joined
// by a second launch. Both ways priced by a workgroup's time: 0.2 us a K-tile of 32 x 32 tiles, 0.33 of 64 x 64 tiles, all at
// once, and 4 for the second launch (two parts of two fp32 experts, 2048 x 256: 238 -> 209 us an update of six steps; four of
// 4096 x 128: 298 -> 214).
struct GramSplit {
  int parts;    // 1: not split
  bool tiniest; // 32 x 32 tiles
};
GramSplit gram_split(int m, int n, int mats, bool precise) {
  const int64_t cus = 256, kts = n / 64 * (precise ? 3 : 1);
  const auto tiles = [&](int b) { return (int64_t)((m + b - 1) / b) * ((m + b - 1) / b + 1) / 2 * mats; };
  GramSplit best{1, true};
  if (tiles(64) > cus) return best;
  double time = kts * (tiles(32) <= cus ? 0.2 : 0.33);
  for (int b : {32, 64}) {
    const int64_t s = std::min(cus / tiles(b), kts / 8);
    const double t = kts * (b == 32 ? 0.2 : 0.33) / s + 4;
    if (s >= 2 && t < time) {
      best = {(int)s, b == 32};
      time = t;
    }
  }
  return best;
}

struct MuonLayout {
  int mats, m, n;
  int pass;  // matrices taken at a time
  GramSplit split;
  size_t x, xt[2], a, r, b[3], partial, bytes;  // the partial sums of squares come first
};
MuonLayout muon_layout(const moe_desc& d, bool precise) {
  MuonLayout l{};
  l.mats = 3 * (d.local_count + d.n_shared);
  l.m = std::min(d.d_model, d.d_ff);
  l.n = std::max(d.d_model, d.d_ff);
  l.pass = muon_pass(l.m, l.mats);
  const size_t parts = precise ? 2 : 1;
  const size_t all_x = (size_t)l.pass * l.m * l.n, all_a = (size_t)l.pass * l.m * l.m;
  size_t at = align256(sizeof(double) * l.pass * SUM_BLOCKS);
  const auto take = [&](size_t n) {
    const size_t here = at;
    at += align256(parts * n * 2);
    return here;
  };
  l.x = take(all_x);
  for (size_t& o : l.xt) o = take(all_x);
  l.a = take(all_a);
  l.r = take(all_a);
  for (size_t& o : l.b) o = take(all_a);
  l.split = gram_split(l.m, l.n, l.pass, precise);
  l.partial = at;
  if (l.split.parts > 1) at += align256((size_t)l.split.parts * all_a * sizeof(float));
  l.bytes = at;
  return l;
}

// Largest |poly| over [0, top], poly = t (c0 + c1 t^2 + c2 t^4).
double largest(double c0, double c1, double c2, double top) {
  const auto at = [&](double t) { return std::fabs(t * (c0 + t * t * (c1 + t * t * c2))); };
  double most = at(top);
  // extrema: c0 + 3 c1 s + 5 c2 s^2 = 0 with s = t^2
  const double disc = 9 * c1 * c1 - 20 * c0 * c2;
  double roots[2] = {-1., -1.};
  if (c2 != 0 && disc >= 0) {
    roots[0] = (-3 * c1 + std::sqrt(disc)) / (10 * c2);
    roots[1] = (-3 * c1 - std::sqrt(disc)) / (10 * c2);
  } else if (c2 == 0 && c1 != 0) {
    roots[0] = -c0 / (3 * c1);
  }
  for (double s : roots)
    if (s > 0 && s < top * top) most = std::max(most, at(std::sqrt(s)));
  return most;
}
// Largest |c0 + c1 s + c2 s^2| over s in [0, top^2]: of the factor by which a step multiplies a singular value.
double largest_factor(double c0, double c1, double c2, double top) {
  const double s1 = top * top;
  double most = std::max(std::fabs(c0), std::fabs(c0 + s1 * (c1 + s1 * c2)));
  if (c2 != 0) {
    const double s = -c1 / (2 * c2);
    if (s > 0 && s < s1) most = std::max(most, std::fabs(c0 + s * (c1 + s * c2)));
  }
  return most;
}
// Steps that are taken on A before X is formed again, after `done` of `steps`. A group of g steps costs m^2 n + 2 m^2 n + (4 g -
// 3) m^3 operations, g steps one by one g (3 m^2 n + m^3): a longer group saves where n is above m. It also multiplies what
// rounding has done to A's small eigenvalues by a^2 a step. Off the 64-bit X of random matrices with four directions 0.5 / 3 /
// 20 times the others' size (1024 x 2816): one by one 0.9e-3 / 1.9e-3 / 9.9e-3, groups of 2, 2, 1: 1.3e-3 / 1.6e-3 / 8.2e-3, of
// 2, 3: 1.1e-3 / 3.3e-3 / 9.5e-3, of five: 1e-3 / 0.1 (a simulation). In two parts: 1.2e-6 / 1.6e-6 / 8.1e-6, 1.7e-6 / 1.2e-6 /
// 5.7e-6, 1.4e-6 / 3.6e-6 / 6.9e-6 (fp32 products 3.5e-6 / 2.3e-6 / 1.2e-5). Two at first, when A's eigenvalues span most, then
// three, and two at most in the precise form.
int muon_group(const MuonLayout& l, bool precise, int done, int steps) {
  if (2 * l.n < 3 * l.m) return 1;
  return std::min(done == 0 || precise ? 2 : 3, steps - done);
}
// The power of two that takes values of up to `top` below 2^15.
double two_to(double top) {
  int e = 0;
  std::frexp(std::max(top, 1e-6), &e);  // top <= 2^e
  return std::ldexp(1.0, 15 - e);
}

}  // namespace

double muon_growth(const moe_muon& o) {
  double top = 1., most = 1.;
  for (int i = 0; i < o.steps && most <= 1e6; ++i) {
    top = largest(o.a, o.b, o.c, top);
    most = std::max(most, top);
  }
  return most;
}

size_t update_muon_ws_bytes(const moe_desc& d, bool precise) { return muon_layout(d, precise).bytes; }

// Matrices mat0 .. mat0 + mats - 1.
static hipError_t muon_run(const moe_desc& d, const moe_muon& o, const MuonLayout& l, int mat0, int mats, void* wg, void* wu,
                           void* wd, const void* gg, const void* gu, const void* gd, float* master, float* m, void* ws,
                           hipStream_t s) {
  char* base = (char*)ws;
  MuonArgs a{};
  a.w[0] = wg; a.w[1] = wu; a.w[2] = wd;
  a.g[0] = gg; a.g[1] = gu; a.g[2] = gd;
  a.G = d.local_count + d.n_shared;
  a.mat0 = mat0;
  a.d = d.d_model;
  a.f = d.d_ff;
  a.master = master;
  a.m = m;
  a.part = (double*)base;
  a.mu = o.momentum;
  a.nesterov = o.nesterov;
  a.eps = (double)o.eps;
  a.x = (f16*)(base + l.x);
  a.xt = (f16*)(base + l.xt[0]);
  double sx = two_to(1.0);
  a.s0 = (float)sx;
  const bool bf = d.dtype == MOE_BF16;
  {
    KernelTimer kt("muon_momentum", s);
    const dim3 grid(SUM_BLOCKS, mats);
    if (bf) hipLaunchKernelGGL(muon_momentum_kernel<bf16>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(muon_momentum_kernel<float>, grid, dim3(256), 0, s, a);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  {
    KernelTimer kt("muon_normalise", s);
    const dim3 grid((unsigned)((size_t)(a.d / 64) * (a.f / 64)), mats);
    if (o.precise) {
      if (bf) hipLaunchKernelGGL((muon_normalise_kernel<bf16, true>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((muon_normalise_kernel<float, true>), grid, dim3(256), 0, s, a);
    } else {
      if (bf) hipLaunchKernelGGL((muon_normalise_kernel<bf16, false>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((muon_normalise_kernel<float, false>), grid, dim3(256), 0, s, a);
    }
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;

  f16 *xt[2] = {a.xt, (f16*)(base + l.xt[1])}, *A = (f16*)(base + l.a), *R = (f16*)(base + l.r);
  f16* buf[3];
  for (int i = 0; i < 3; ++i) buf[i] = (f16*)(base + l.b[i]);
  double top = 1.0;   // of X's singular values
  int turn = 0;
  for (int done = 0; done < o.steps;) {
    const int group = muon_group(l, o.precise != 0, done, o.steps);
    const bool last = done + group == o.steps;
    // A = X X^T
    NsArgs n{};
    n.mats = mats;
    n.M = n.N = l.m;
    n.K = l.n;
    n.p = n.q = a.x;
    n.out = A;
    double sa = two_to(top * top);
    n.alpha = (float)(sa / (sx * sx));
    if (l.split.parts > 1) {
      n.ksplit = l.split.parts;
      n.partial = (float*)(base + l.partial);
      if (hipError_t e = ns_gram_split(n, l.split.tiniest, o.precise, s); e != hipSuccess) return e;
    } else if (hipError_t e = ns_product<NS_SYMMETRIC>("muon_gram", n, o.precise, s); e != hipSuccess) {
      return e;
    }
    n.K = l.m;
    f16 *P = nullptr, *Q = nullptr;
    double sp = 0, sq = 0, tq = 1.0;
    for (int i = 0; i < group; ++i) {
      // P = a + b A + c A^2, in a buffer that is neither Q nor the last P
      const double tp = largest_factor(o.a, o.b, o.c, top);
      sp = two_to(tp);
      f16* next = buf[0];
      for (f16* f : buf)
        if (f != P && f != Q) next = f;
      NsArgs v = n;
      v.p = v.q = v.d = A;
      v.out = P = next;
      v.alpha = (float)((double)o.c * sp / (sa * sa));
      v.beta = (float)((double)o.b * sp / sa);
      v.diag = (float)((double)o.a * sp);
      if (hipError_t e = ns_product<NS_SYMMETRIC>("muon_poly", v, o.precise, s); e != hipSuccess) return e;
      // R = P A unless X is formed next, and Q <- P Q
      v = n;
      v.p = P;
      const bool more = i + 1 < group;
      const double tr = tp * top * top, sr = two_to(tr), sq2 = two_to(tp * tq);
      f16* q_out = nullptr;
      for (f16* f : buf)
        if (f != P && f != Q) q_out = f;
      if (more) {
        v.q = A;
        v.out = R;
        v.alpha = (float)(sr / (sp * sa));
        if (Q) {
          v.q2 = Q;
          v.out2 = q_out;
          v.alpha2 = (float)(sq2 / (sp * sq));
        }
      } else if (Q) {
        v.q = Q;
        v.out = q_out;
        v.alpha = (float)(sq2 / (sp * sq));
      }
      if (more || Q) {
        if (hipError_t e = ns_product<NS_SYMMETRIC>("muon_chain", v, o.precise, s); e != hipSuccess) return e;
      }
      top = largest(o.a, o.b, o.c, top);
      if (more) {  // A <- P R, the Gram matrix of P X
        v = n;
        v.p = P;
        v.q = R;
        v.out = A;
        sa = two_to(top * top);
        v.alpha = (float)(sa / (sp * sr));
        if (hipError_t e = ns_product<NS_SYMMETRIC>("muon_chain", v, o.precise, s); e != hipSuccess) return e;
      }
      tq *= tp;
      sq = Q ? sq2 : sp;
      Q = Q ? q_out : P;
    }
    // X <- Q X
    n.N = l.n;
    n.p = Q;
    n.q = xt[turn];
    const double sn = last ? 1.0 : two_to(top);
    n.alpha = (float)(sn / (sq * sx));
    if (last) {
      for (int t = 0; t < 3; ++t) n.w[t] = a.w[t];
      n.flip_up = a.f > a.d;
      n.flip_down = a.d > a.f;
      n.master = master;
      n.G = a.G;
      n.mat0 = mat0;
      n.dtype = d.dtype;
      n.decay = (float)(1.0 - (double)o.lr * (double)o.weight_decay);
      n.step = (float)((double)o.lr * (double)o.scale);
      if (hipError_t e = ns_product<NS_LAST>("muon_update", n, o.precise, s); e != hipSuccess) return e;
    } else {
      n.out = a.x;
      turn ^= 1;
      n.out_t = xt[turn];
      if (hipError_t e = ns_product<NS_BOTH>("muon_step", n, o.precise, s); e != hipSuccess) return e;
    }
    sx = sn;
    done += group;
  }
  return hipSuccess;
}

hipError_t launch_expert_update_muon(const moe_desc& d, const moe_muon& o, void* wg, void* wu, void* wd, const void* gg,
                                     const void* gu, const void* gd, float* master, float* m, void* ws, hipStream_t s) {
  const MuonLayout l = muon_layout(d, o.precise != 0);
  for (int mat0 = 0; mat0 < l.mats; mat0 += l.pass) {
    const int mats = std::min(l.pass, l.mats - mat0);
    if (hipError_t e = muon_run(d, o, l, mat0, mats, wg, wu, wd, gg, gu, gd, master, m, ws, s); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pcmoe
