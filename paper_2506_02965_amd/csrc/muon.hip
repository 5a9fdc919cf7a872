// Update of the experts' matrices by their orthogonalised momentum.
//
// m <- mu m + g, u = g + mu m or m, X = u / (|u|_F + eps); then a fixed number of Newton-Schulz steps
//   A = X X^T,  B = b A + c A^2,  X <- a X + B X,
// taken with X's rows no longer than its columns' number (of a tall matrix X is the transpose), and p <- p (1 - lr wd) -
// lr scale X. A step of an m x n matrix takes m^2 n (A, half of a symmetric product) + m^3 (A^2, the other) + 2 m^2 n
// operations, all on the fp16 matrix cores: bound by them, and at small sizes by the launches in a row.
//
// All three are products of two K-contiguous operands: A = X X^T reads X, A^2 reads A = A^T, and B X reads B and X^T. So X is
// kept in both orientations, each written by the epilogue that makes it. Of a symmetric product only the tiles on and above
// the diagonal are computed; each is stored twice. The last step's epilogue updates the parameters.
//
// X, A and B are held in fp16 after a power of two that keeps them below 2^15: |X| never passes the polynomial's largest value
// on [0, 1], which the host knows. Eleven bits leave X some 2^-11 of its size off; in the precise form each is held in two
// fp16 parts (22 bits) and three products are added up, smallest first. Sums are fp32, the momentum fp32, the norm fp64.
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
  int d, f;
  float *master, *m; // [3][G][f d]
  double* part;      // [3 G][SUM_BLOCKS]
  float mu;
  int nesterov;
  double eps;
  f16 *x, *xt;       // [3 G][m][n], [3 G][n][m], then the second parts
  size_t plane;      // elements of a part
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
  const int mat = blockIdx.y;
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
  if (threadIdx.x == 0) a.part[(size_t)mat * SUM_BLOCKS + blockIdx.x] = s[0];
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
  const int mat = blockIdx.y, tensor = mat / a.G;
  const int rows = tensor == 2 ? a.d : a.f, cols = tensor == 2 ? a.f : a.d;
  const int tr = blockIdx.x / (cols / 64), tc = blockIdx.x % (cols / 64);
  __shared__ double norm2;
  __shared__ f16 tile[PRECISE ? 2 : 1][64][72];
  const size_t at = (size_t)mat * a.d * a.f;
  if (threadIdx.x < 64) {
    double s = a.part[(size_t)mat * SUM_BLOCKS + threadIdx.x];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (threadIdx.x == 0) norm2 = s;
  }
  __syncthreads();
  const double inv = (double)a.s0 / (sqrt(norm2) + a.eps);
  const T* g = (const T*)a.g[tensor] + (size_t)(mat % a.G) * a.d * a.f;
  const bool flip = rows > cols;  // stored tall: X is the transpose
  f16* straight = flip ? a.xt : a.x;
  f16* turned = flip ? a.x : a.xt;
  constexpr int PER_ROW = 64 / EP;
#pragma unroll
  for (int k = 0; k < 64 * PER_ROW / 256; ++k) {
    const int task = threadIdx.x + 256 * k, r = task / PER_ROW, c = (task % PER_ROW) * EP;
    const size_t src = (size_t)(tr * 64 + r) * cols + tc * 64 + c;
    float gv[EP], mv[EP];
    chunk_to_f<T>(ld_chunk(g + src), gv);
#pragma unroll
    for (int h = 0; h < EP; h += 4) chunk_to_f<float>(ld_chunk(a.m + at + src + h), mv + h);
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
      st_chunk(straight + p * a.plane + at + (size_t)(tr * 64 + r) * cols + tc * 64 + c,
               *reinterpret_cast<const Chunk*>(&tile[p][r][c]));
      half8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile[p][c + e][r];
      st_chunk(turned + p * a.plane + at + (size_t)(tc * 64 + r) * rows + tr * 64 + c, __builtin_bit_cast(Chunk, v));
    }
}

// One product of every matrix: out = alpha P Q^T + beta D, P [M][K], Q [N][K], D and out [M][N].
struct NsArgs {
  const f16 *p, *q, *d;
  f16 *out, *out_t;        // out, and its transpose [N][M]
  size_t p_mat, q_mat, o_mat;        // elements of a matrix
  size_t p_plane, q_plane, o_plane;  // ... of a part
  int M, N, K, mats;
  float alpha, beta;
  // last step: parameters in place of out
  void* w[3];
  float* master;
  int G, dtype;
  int flip[3];             // the tensor is stored transposed to X
  float decay, step;       // p <- decay p - step X
};

enum NsMode { NS_SYMMETRIC, NS_BOTH, NS_LAST };  // stores: one tile and its mirror, both orientations, the parameters

template <typename S, int MODE, bool PRECISE>
__global__ __launch_bounds__(S::NT) void muon_product_kernel(NsArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tm = (a.M + S::BM - 1) / S::BM, tn = (a.N + S::BN - 1) / S::BN;
  const int per = MODE == NS_SYMMETRIC ? tm * (tm + 1) / 2 : tm * tn;
  const int L = xcd_order(blockIdx.x, per * a.mats);
  const int mat = L / per;
  int l = L - mat * per, mt, nt;
  if (MODE == NS_SYMMETRIC) {  // nt >= mt, by columns: nt (nt + 1) / 2 tiles stand before column nt
    nt = (int)((sqrtf(8.f * (float)l + 1.f) - 1.f) * 0.5f);
    while (nt * (nt + 1) / 2 > l) --nt;
    while ((nt + 1) * (nt + 2) / 2 <= l) ++nt;
    mt = l - nt * (nt + 1) / 2;
  } else {  // eight row tiles at a time, so that neighbours share both operands
    const int blk = l / (8 * tn), rem = l - blk * 8 * tn, rows = min(8, tm - 8 * blk);
    nt = rem / rows;
    mt = 8 * blk + rem % rows;
  }
  const int m0 = mt * S::BM, n0 = nt * S::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
  const int ld = a.K * 2;
  const f16 *p0 = a.p + mat * a.p_mat, *q0 = a.q + mat * a.q_mat;
  const uint32_t p_bytes = (uint32_t)a.M * ld, q_bytes = (uint32_t)a.N * ld;
  const int32x4 rp = make_rsrc(p0, p_bytes), rq = make_rsrc(q0, q_bytes);
  int32x4 rp1 = rp, rq1 = rq;
  if (PRECISE) {
    rp1 = make_rsrc(p0 + a.p_plane, p_bytes);
    rq1 = make_rsrc(q0 + a.q_plane, q_bytes);
  }
  const int kts = a.K / 64, at = nt_lane(ld);
  // the wavefronts' parts lie on either side of a matrix's end, not across it: both are multiples of 64
  const bool live = m0 + wm * S::WTM < a.M && n0 + wn * S::WTN < a.N;
  typename F16::acc acc[S::FM][S::FN];
  // K-tiles kt: of a precise product first P1 Q2, then P2 Q1, then P1 Q1
  nt_loop<S, F16>(
      smem, PRECISE ? 3 * kts : kts, live,
      [&](int kt, int j, uint32_t dst) {
        const int seg = PRECISE ? (kt >= 2 * kts ? 2 : kt >= kts ? 1 : 0) : 2;
        dma16(PRECISE ? pick_rsrc(seg == 1, rp, rp1) : rp, dst, (m0 + 8 * j) * ld + at + (PRECISE ? kt - seg * kts : kt) * NT_ROWB);
      },
      [&](int kt, int j, uint32_t dst) {
        const int seg = PRECISE ? (kt >= 2 * kts ? 2 : kt >= kts ? 1 : 0) : 2;
        dma16(PRECISE ? pick_rsrc(seg == 0, rq, rq1) : rq, dst, (n0 + 8 * j) * ld + at + (PRECISE ? kt - seg * kts : kt) * NT_ROWB);
      },
      acc);
  if (!live) return;

  // Epilogue, per wavefront: 32 rows at a time go through LDS in fp32, are combined with D and stored by rows of 16-byte
  // chunks, then read again by columns for the transposed store.
  constexpr int PITCH = S::WTN + 4;
  float* st = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
  static_assert(S::NW * 32 * PITCH * 4 <= S::LDS, "the staging fits the operands' LDS");
  const int tensor = mat / max(a.G, 1), flip = MODE == NS_LAST ? a.flip[tensor] : 0;
#pragma unroll
  for (int part = 0; part < S::FM / 2; ++part) {
    const int mr = m0 + wm * S::WTM + 32 * part, nc = n0 + wn * S::WTN;
#pragma unroll
    for (int i = 0; i < S::FM; ++i) {
      if (i / 2 != part) continue;
#pragma unroll
      for (int j = 0; j < S::FN; ++j)
        *reinterpret_cast<floatx4*>(st + (16 * (i & 1) + li) * PITCH + 16 * j + 4 * q) = acc[i][j];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    constexpr int CH = S::WTN / 8;  // 8-column chunks of a row
#pragma unroll
    for (int k = 0; k < 32 * CH / 64; ++k) {
      const int task = lane + 64 * k, r = task / CH, c = (task % CH) * 8;
      float v[8];
      chunk_to_f<float>(ld_chunk(st + r * PITCH + c), v);
      chunk_to_f<float>(ld_chunk(st + r * PITCH + c + 4), v + 4);
      const size_t o = mat * a.o_mat + (size_t)(mr + r) * a.N + nc + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= a.alpha;
      if (a.d) {
        const half8 dv = __builtin_bit_cast(half8, ld_chunk(a.d + o));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += a.beta * (float)dv[e];
        if (PRECISE) {
          const half8 d1 = __builtin_bit_cast(half8, ld_chunk(a.d + a.o_plane + o));
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += a.beta * (float)d1[e];
        }
      }
      if (MODE != NS_LAST) {
#pragma unroll
        for (int p = 0; p < (PRECISE ? 2 : 1); ++p) {
          half8 h;
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = part_of(v[e], p != 0);
          st_chunk(a.out + p * a.o_plane + o, __builtin_bit_cast(Chunk, h));
        }
      }
      st_chunk(st + r * PITCH + c, f_to_chunk<float>(v));
      st_chunk(st + r * PITCH + c + 4, f_to_chunk<float>(v + 4));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (MODE == NS_LAST) {
      // rows of the parameters: X's rows, or its columns where the tensor is stored transposed
      const int inner = flip ? 4 : CH, outer = flip ? S::WTN : 32;
      for (int k = 0; k < outer * inner / 64; ++k) {
        const int task = lane + 64 * k, r = task / inner, c = (task % inner) * 8;
        float v[8], p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = flip ? st[(c + e) * PITCH + r] : st[r * PITCH + c + e];
        const size_t in = (size_t)(mat % a.G) * a.o_mat +
                          (flip ? (size_t)(nc + r) * a.M + mr + c : (size_t)(mr + r) * a.N + nc + c);
        float* mp = a.master ? a.master + (size_t)tensor * a.G * a.o_mat + in : nullptr;
        float* wf = (float*)a.w[tensor] + in;
        bf16* wb = (bf16*)a.w[tensor] + in;
        if (mp || a.dtype == MOE_F32) {
          const float* from = mp ? mp : wf;
          chunk_to_f<float>(ld_chunk(from), p);
          chunk_to_f<float>(ld_chunk(from + 4), p + 4);
        } else {
          chunk_to_f<bf16>(ld_chunk(wb), p);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = a.decay * p[e] - a.step * v[e];
        if (mp) {
          st_chunk(mp, f_to_chunk<float>(p));
          st_chunk(mp + 4, f_to_chunk<float>(p + 4));
        }
        if (a.dtype == MOE_F32) {
          st_chunk(wf, f_to_chunk<float>(p));
          st_chunk(wf + 4, f_to_chunk<float>(p + 4));
        } else {
          st_chunk(wb, f_to_chunk<bf16>(p));
        }
      }
    } else if (MODE == NS_BOTH || mt != nt) {
#pragma unroll
      for (int k = 0; k < S::WTN * 4 / 64; ++k) {
        const int task = lane + 64 * k, r = task >> 2, c = (task & 3) * 8;
        const size_t o = mat * a.o_mat + (size_t)(nc + r) * a.M + mr + c;
#pragma unroll
        for (int p = 0; p < (PRECISE ? 2 : 1); ++p) {
          half8 h;
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = part_of(st[(c + e) * PITCH + r], p != 0);
          st_chunk(a.out_t + p * a.o_plane + o, __builtin_bit_cast(Chunk, h));
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

typedef NtShape<128, 128, 2, 2, 2> NsSmall;

template <typename S, int MODE, bool PRECISE>
hipError_t ns_launch(const char* name, const NsArgs& a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kern = muon_product_kernel<S, MODE, PRECISE>;
  if (hipError_t e = lds_limit_once((const void*)kern, S::LDS, done); e != hipSuccess) return e;
  const int64_t tm = (a.M + S::BM - 1) / S::BM, tn = (a.N + S::BN - 1) / S::BN;
  const int64_t tiles = (MODE == NS_SYMMETRIC ? tm * (tm + 1) / 2 : tm * tn) * a.mats;
  KernelTimer kt(name, s);
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(S::NT), S::LDS, s, a);
  return hipGetLastError();
}
template <int MODE>
hipError_t ns_product(const char* name, const NsArgs& a, bool precise, hipStream_t s) {
  return precise ? ns_launch<NsSmall, MODE, true>(name, a, s) : ns_launch<NsSmall, MODE, false>(name, a, s);
}

struct MuonLayout {
  int mats, m, n;
  size_t x_plane, a_plane;  // elements of a part of X and of A
  size_t part, x, xt, a, b, bytes;
};
MuonLayout muon_layout(const moe_desc& d, bool precise) {
  MuonLayout l{};
  l.mats = 3 * (d.local_count + d.n_shared);
  l.m = std::min(d.d_model, d.d_ff);
  l.n = std::max(d.d_model, d.d_ff);
  const size_t parts = precise ? 2 : 1;
  l.x_plane = (size_t)l.mats * l.m * l.n;
  l.a_plane = (size_t)l.mats * l.m * l.m;
  l.x = align256(sizeof(double) * l.mats * SUM_BLOCKS);
  l.xt = l.x + align256(parts * l.x_plane * 2);  // two of them, in turn
  l.a = l.xt + 2 * align256(parts * l.x_plane * 2);
  l.b = l.a + align256(parts * l.a_plane * 2);
  l.bytes = l.b + align256(parts * l.a_plane * 2);
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

hipError_t launch_expert_update_muon(const moe_desc& d, const moe_muon& o, void* wg, void* wu, void* wd, const void* gg,
                                     const void* gu, const void* gd, float* master, float* m, void* ws, hipStream_t s) {
  const MuonLayout l = muon_layout(d, o.precise != 0);
  char* base = (char*)ws;
  MuonArgs a{};
  a.w[0] = wg; a.w[1] = wu; a.w[2] = wd;
  a.g[0] = gg; a.g[1] = gu; a.g[2] = gd;
  a.G = d.local_count + d.n_shared;
  a.d = d.d_model;
  a.f = d.d_ff;
  a.master = master;
  a.m = m;
  a.part = (double*)base;
  a.mu = o.momentum;
  a.nesterov = o.nesterov;
  a.eps = (double)o.eps;
  a.x = (f16*)(base + l.x);
  a.xt = (f16*)(base + l.xt);
  a.plane = l.x_plane;
  double sx = two_to(1.0);
  a.s0 = (float)sx;
  const bool bf = d.dtype == MOE_BF16;
  {
    KernelTimer kt("muon_momentum", s);
    const dim3 grid(SUM_BLOCKS, l.mats);
    if (bf) hipLaunchKernelGGL(muon_momentum_kernel<bf16>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(muon_momentum_kernel<float>, grid, dim3(256), 0, s, a);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  {
    KernelTimer kt("muon_normalise", s);
    const dim3 grid((unsigned)((size_t)(a.d / 64) * (a.f / 64)), l.mats);
    if (o.precise) {
      if (bf) hipLaunchKernelGGL((muon_normalise_kernel<bf16, true>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((muon_normalise_kernel<float, true>), grid, dim3(256), 0, s, a);
    } else {
      if (bf) hipLaunchKernelGGL((muon_normalise_kernel<bf16, false>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((muon_normalise_kernel<float, false>), grid, dim3(256), 0, s, a);
    }
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;

  f16* xt[2] = {a.xt, (f16*)(base + l.xt + (l.a - l.xt) / 2)};
  f16 *A = (f16*)(base + l.a), *B = (f16*)(base + l.b);
  const size_t mn = (size_t)l.m * l.n, mm = (size_t)l.m * l.m;
  double top = 1.0;
  for (int step = 0; step < o.steps; ++step) {
    const double sa = two_to(top * top), next = largest(o.a, o.b, o.c, top);
    // B's largest eigenvalue: |b s^2 + c s^4| over [0, top]
    double tb = std::fabs(top * top * (o.b + o.c * top * top));
    if (o.c != 0 && -o.b / (2 * o.c) > 0 && -o.b / (2 * o.c) < top * top) tb = std::max(tb, std::fabs(o.b * o.b / (4 * (double)o.c)));
    const double sb = two_to(tb), sn = two_to(next);
    NsArgs n{};
    n.mats = l.mats;
    n.M = n.N = l.m;
    n.K = l.n;
    n.p = n.q = a.x;
    n.p_mat = n.q_mat = mn;
    n.p_plane = n.q_plane = l.x_plane;
    n.out = n.out_t = A;
    n.o_mat = mm;
    n.o_plane = l.a_plane;
    n.alpha = (float)(sa / (sx * sx));
    if (hipError_t e = ns_product<NS_SYMMETRIC>("muon_gram", n, o.precise, s); e != hipSuccess) return e;
    n.K = l.m;
    n.p = n.q = n.d = A;
    n.p_mat = n.q_mat = mm;
    n.p_plane = n.q_plane = l.a_plane;
    n.out = n.out_t = B;
    n.alpha = (float)((double)o.c * sb / (sa * sa));
    n.beta = (float)((double)o.b * sb / sa);
    if (hipError_t e = ns_product<NS_SYMMETRIC>("muon_square", n, o.precise, s); e != hipSuccess) return e;
    const bool last = step == o.steps - 1;
    n.N = l.n;
    n.p = B;
    n.q = xt[step & 1];
    n.q_mat = mn;
    n.q_plane = l.x_plane;
    n.d = a.x;
    n.out = a.x;
    n.out_t = xt[(step + 1) & 1];
    n.o_mat = mn;
    n.o_plane = l.x_plane;
    n.alpha = (float)((last ? 1.0 : sn) / (sb * sx));
    n.beta = (float)((double)o.a * (last ? 1.0 : sn) / sx);
    if (last) {
      for (int t = 0; t < 3; ++t) {
        n.w[t] = a.w[t];
        n.flip[t] = (t == 2 ? a.d > a.f : a.f > a.d) ? 1 : 0;
      }
      n.master = master;
      n.G = a.G;
      n.dtype = d.dtype;
      n.decay = (float)(1.0 - (double)o.lr * (double)o.weight_decay);
      n.step = (float)((double)o.lr * (double)o.scale);
      if (hipError_t e = ns_product<NS_LAST>("muon_update", n, o.precise, s); e != hipSuccess) return e;
    } else {
      if (hipError_t e = ns_product<NS_BOTH>("muon_step", n, o.precise, s); e != hipSuccess) return e;
    }
    sx = sn;
    top = next;
  }
  return hipSuccess;
}

}  // namespace pcmoe
