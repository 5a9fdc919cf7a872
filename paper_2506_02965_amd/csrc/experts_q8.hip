// Experts in 8-bit integers: weights with a scale for each output channel, rows of x and of H with a scale for each token.
//
// A row v is held as scale = fp32(m / 127), m = max|v|, and codes rint(127 v / m), ties to even. G = sx sg (x . g) with the
// sum over codes exact in int32 (127^2 K stays below 2^31), U likewise, H = silu(G) U in fp32, which is held in 8 bits per
// row again once the whole row is there, and y = sh sd (h . d). So a call is four launches: rows of x to codes, gate and up,
// rows of H to codes, down.
//
// Bound by the int8 matrix cores for long prompts; H passes memory once in fp32 and once in codes.
#include "nt_gemm.h"
#include "expert_ops.h"

#include <algorithm>
#include <cstdlib>

namespace pcmoe {

namespace {

constexpr int Q8_THREADS = 256;

__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }
// Largest magnitude bits over the workgroup (of fp32 numbers: infinities and NaN are above all finite ones).
__device__ __forceinline__ uint32_t block_max_bits(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max_u32(v, (uint32_t)__shfl_xor((int)v, o, 64));
  __shared__ uint32_t s[Q8_THREADS / 64];
  __syncthreads();  // the values of the last call have been read
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < Q8_THREADS / 64; ++w) v = max_u32(v, s[w]);
  return v;
}

// What turns a row's values into codes. Quotients 127 v / m of bf16 numbers that are not ties lie 2^-17 or more away from
// one, so that the fp32 quotient, corrected once by its exact remainder, decides them as the real one does; fp32 weights
// need fp64 for the same.
struct RowCodes {
  float m, inv;    // the largest magnitude, scaled into [1, 2), and its reciprocal
  int shift;       // power of two that does so
  double dm, dinv;
  bool ok, zero;
};
__device__ __forceinline__ RowCodes row_codes(uint32_t bits) {
  RowCodes r;
  const float m = __uint_as_float(bits);
  r.ok = bits < 0x7f800000u;
  r.zero = bits == 0;
  r.shift = r.ok && !r.zero ? -ilogbf(m) : 0;
  r.m = r.ok && !r.zero ? ldexpf(m, r.shift) : 1.f;
  r.inv = __builtin_amdgcn_rcpf(r.m);
  r.dm = (double)r.m;
  r.dinv = 1.0 / r.dm;
  return r;
}
__device__ __forceinline__ float row_scale(uint32_t bits) {
  return bits < 0x7f800000u ? (float)((double)__uint_as_float(bits) / 127.0) : __uint_as_float(0x7fc00000u);
}
template <bool F64>
__device__ __forceinline__ int code_of(const RowCodes& r, float v) {
  const float x = ldexpf(v, r.shift);
  float q;
  if (F64) {
    const double a = 127.0 * (double)x, t = a * r.dinv;
    q = (float)rint(fma(fma(-t, r.dm, a), r.dinv, t));
  } else {
    const float a = 127.f * x, t = a * r.inv;
    q = rintf(__builtin_fmaf(__builtin_fmaf(-t, r.m, a), r.inv, t));
  }
  return r.ok ? (int)q : 0;
}

// A row of K values to codes and scale, by the whole workgroup. SRC: bf16 or float; F64: exact quotients of fp32 values. The
// first KEEP chunks of a thread stay in registers; what a longer row has beyond them is read again.
template <typename SRC, bool F64, int KEEP>
__device__ __forceinline__ void code_row(const SRC* v, int K, int8_t* codes, float* scale) {
  constexpr int EP = EPC<SRC>::value;
  const int n = K / EP;
  uint32_t top = 0;
  const auto look = [&](const Chunk& c) {
    float x[EP];
    chunk_to_f<SRC>(c, x);
#pragma unroll
    for (int e = 0; e < EP; ++e) top = max_u32(top, __float_as_uint(x[e]) & 0x7fffffffu);
  };
  Chunk kept[KEEP];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    const int c = threadIdx.x + i * Q8_THREADS;
    kept[i] = c < n ? ld_chunk(v + c * EP) : zero_chunk();
  }
#pragma unroll
  for (int i = 0; i < KEEP; ++i) look(kept[i]);
  for (int c = threadIdx.x + KEEP * Q8_THREADS; c < n; c += Q8_THREADS) look(ld_chunk(v + c * EP));
  top = block_max_bits(top);
  const RowCodes r = row_codes(top);
  const auto put = [&](int c, const Chunk& from) {
    float x[EP];
    chunk_to_f<SRC>(from, x);
    uint32_t w[EP / 4];
#pragma unroll
    for (int e = 0; e < EP; ++e) {
      if (e % 4 == 0) w[e / 4] = 0;
      w[e / 4] |= (uint32_t)(code_of<F64>(r, x[e]) & 255) << (8 * (e % 4));
    }
    if constexpr (EP == 8) *reinterpret_cast<uint2*>(codes + c * EP) = uint2{w[0], w[1]};
    else *reinterpret_cast<uint32_t*>(codes + c * EP) = w[0];
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    const int c = threadIdx.x + i * Q8_THREADS;
    if (c < n) put(c, kept[i]);
  }
  for (int c = threadIdx.x + KEEP * Q8_THREADS; c < n; c += Q8_THREADS) put(c, ld_chunk(v + c * EP));
  if (threadIdx.x == 0) *scale = row_scale(top);
}

template <typename T>
__global__ __launch_bounds__(Q8_THREADS) void q8_pack_kernel(const T* w, int64_t rows, int cols, int8_t* codes, float* scales) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    code_row<T, std::is_same<T, float>::value, 4>(w + r * cols, cols, codes + r * cols, scales + r);
}

template <typename T>
__global__ __launch_bounds__(Q8_THREADS) void q8_unpack_kernel(const int8_t* codes, const float* scales, int64_t rows, int cols,
                                                               T* w) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float s = scales[r];
    for (int c = threadIdx.x; c < cols / 16; c += Q8_THREADS) {
      const Chunk q = ld_chunk(codes + r * cols + 16 * c);
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = (float)(int8_t)(q.w[e / 4] >> (8 * (e % 4))) * s;
#pragma unroll
      for (int e = 0; e < 16; e += EPC<T>::value) st_chunk(w + r * cols + 16 * c + e, f_to_chunk<T>(v + e));
    }
  }
}

struct Q8Args {
  GemmArgs ga;        // T, k, d, f, Eloc, S, rows_cap, offsets, mt_prefix, n_tiles
  const void *x, *xp;
  int8_t* xq;         // [T k + T][d]: codes of x_perm, then of x
  float* sx;
  float* h;           // [R][f]
  int8_t* hq;
  float* sh;          // [R]
  const int8_t *wg, *wu, *wd;
  const float *sg, *su, *sd;
  bf16* y;            // [R][d]
  int32_t *prefix, *tail;  // [G + 1] each; no tails: null
  int bm;             // rows of an m-tile
};

// Codes of the rows of x_perm and x; the last workgroup makes the m-tile prefix of the groups, with tails (last m-tiles of at
// most half their rows) in a prefix of their own where they take another tile.
__global__ __launch_bounds__(Q8_THREADS) void q8_rows_x_kernel(Q8Args a) {
  const int r = blockIdx.x;
  if (r == (int)gridDim.x - 1) {
    if (threadIdx.x >= 128) return;
    const int lane = threadIdx.x & 63, tails = threadIdx.x >> 6;  // the second wavefront: the tails
    if (tails && !a.tail) return;
    int32_t* out = tails ? a.tail : a.prefix;
    const int G = a.ga.Eloc + a.ga.S;
    int carry = 0;
    if (lane == 0) out[0] = 0;
    for (int g0 = 0; g0 < G; g0 += 64) {
      const int g = g0 + lane;
      const int rows = g < a.ga.Eloc ? a.ga.offsets[g + 1] - a.ga.offsets[g] : g < G ? a.ga.T : 0;
      const int rem = rows % a.bm, is_tail = a.tail && rem > 0 && 2 * rem <= a.bm ? 1 : 0;
      int v = tails ? is_tail : (rows + a.bm - 1) / a.bm - is_tail;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
      }
      v += carry;
      carry = __builtin_amdgcn_readlane(v, 63);
      if (g < G) out[g + 1] = v;
    }
    return;
  }
  const bool routed = r < a.ga.rows_cap;
  if (routed && r >= a.ga.offsets[a.ga.Eloc]) return;
  const bf16* v = routed ? (const bf16*)a.xp + (size_t)r * a.ga.d : (const bf16*)a.x + (size_t)(r - a.ga.rows_cap) * a.ga.d;
  code_row<bf16, false, 2>(v, a.ga.d, a.xq + (size_t)r * a.ga.d, a.sx + r);
}
template <int KEEP>
__global__ __launch_bounds__(Q8_THREADS) void q8_rows_h_kernel(Q8Args a) {
  const int r = blockIdx.x;
  if (r < a.ga.rows_cap && r >= a.ga.offsets[a.ga.Eloc]) return;
  code_row<float, false, KEEP>(a.h + (size_t)r * a.ga.f, a.ga.f, a.hq + (size_t)r * a.ga.f, a.sh + r);
}

// 1 / (1 + exp(-g)) with the hardware's exponential and reciprocal. The exponential of a product rounded to fp32 alone would be
// |g| roundings off; what the product rounds away is put back.
__device__ __forceinline__ float sigmoid_of(float g) {
  const float t = -1.44269504f * g, r = __builtin_fmaf(-1.44269504f, g, -t) + -1.925963e-8f * g;
  const float e = __builtin_amdgcn_exp2f(fminf(t, 126.f));
  return __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(e, 0.693147181f * r, e));
}

// Gate and up (DOWN = false): half of a wavefront's columns are gate rows, the other half the up rows of the same columns of
// H. Down: y.
template <typename S, bool DOWN>
__device__ __forceinline__ void q8_tile(const Q8Args& a, const TileIdx& ti, int m0, char* smem) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
  const int d = a.ga.d, f = a.ga.f, K = DOWN ? f : d;
  const bool routed = ti.g < a.ga.Eloc;
  const int shared = ti.g - a.ga.Eloc;
  // the group's first row: in the row space, and among the codes of x
  const size_t rs = routed ? (size_t)ti.row0 : (size_t)a.ga.rows_cap + (size_t)shared * a.ga.T;
  const size_t rx = routed ? (size_t)ti.row0 : (size_t)a.ga.rows_cap;
  const int8_t* ap = DOWN ? a.hq + rs * f : a.xq + rx * d;
  const float* sa = DOWN ? a.sh + rs : a.sx + rx;
  const int32x4 ra = make_rsrc(ap, (uint32_t)((size_t)ti.rows * K));
  const size_t wat = (size_t)ti.g * f * d;
  const uint32_t w_bytes = (uint32_t)((size_t)f * d);
  const int32x4 rb0 = make_rsrc((DOWN ? a.wd : a.wg) + wat, w_bytes), rb1 = make_rsrc((DOWN ? a.wd : a.wu) + wat, w_bytes);
  constexpr int HALF = S::WTN / 2;
  const int n0 = DOWN ? ti.nt * S::BN : ti.nt * (S::BN / 2);  // first column of the output
  const int at = nt_lane(K);
  const bool live = m0 + wm * S::WTM < ti.rows && (!DOWN || n0 + wn * S::WTN < d);
  I8::acc acc[S::FM][S::FN];
  nt_loop<S, I8>(
      smem, K / NT_ROWB, live,
      [&](int kt, int j) { return NtSrc{ra, (m0 + 8 * j) * K + at + kt * NT_ROWB}; },
      [&](int kt, int j) {
        if (DOWN) return NtSrc{rb0, (n0 + 8 * j) * K + at + kt * NT_ROWB};
        const int r = 8 * j, w = r / S::WTN, in = r % S::WTN;
        return NtSrc{pick_rsrc(in >= HALF, rb0, rb1), (n0 + w * HALF + in % HALF) * K + at + kt * NT_ROWB};
      },
      acc);
  if (!live) return;
#pragma unroll
  for (int i = 0; i < S::FM; ++i) {
    const int m = m0 + wm * S::WTM + 16 * i + li;
    if (m >= ti.rows) continue;
    const float s = sa[m];
    if (DOWN) {
#pragma unroll
      for (int j = 0; j < S::FN; ++j) {
        const int n = n0 + wn * S::WTN + 16 * j + 4 * q;
        const floatx4 sw = *reinterpret_cast<const floatx4*>(a.sd + (size_t)ti.g * d + n);
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (float)acc[i][j][e] * (s * sw[e]);
        *reinterpret_cast<uint2*>(a.y + (rs + m) * d + n) = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
      }
    } else {
#pragma unroll
      for (int j = 0; j < S::FN / 2; ++j) {
        const int n = n0 + wn * HALF + 16 * j + 4 * q;
        const floatx4 sg = *reinterpret_cast<const floatx4*>(a.sg + (size_t)ti.g * f + n);
        const floatx4 su = *reinterpret_cast<const floatx4*>(a.su + (size_t)ti.g * f + n);
        floatx4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float g = (float)acc[i][j][e] * (s * sg[e]), u = (float)acc[i][j + S::FN / 2][e] * (s * su[e]);
          o[e] = g * sigmoid_of(g) * u;
        }
        *reinterpret_cast<floatx4*>(a.h + (rs + m) * f + n) = o;
      }
    }
  }
}

// A tail (at most half of the rows) of a 256-row tile takes a tile of 128 rows.
template <typename S, bool DOWN>
__global__ __launch_bounds__(S::NT) void q8_gemm_kernel(Q8Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  TileIdx ti;
  if (!decode_tile<true>(a.ga, blockIdx.x, ti)) return;
  const int m0 = ti.mt * S::BM;
  if constexpr (S::PIPE && S::BM == 256) {
    if (2 * (ti.rows - m0) <= S::BM) {
      q8_tile<NtShape<S::BM / 2, S::BN, 2, 2, 2>, DOWN>(a, ti, m0, smem);
      return;
    }
  }
  q8_tile<S, DOWN>(a, ti, m0, smem);
}

typedef NtShape<256, 256, 2, 2, 2> Q8Large;
typedef NtShape<64, 128, 2, 2, 3> Q8b;
typedef NtShape<64, 128, 2, 2, 2> Q8c;
typedef NtShape<32, 128, 1, 4, 4> Q8d;
typedef NtShape<128, 128, 2, 2, 4> Q8e;
typedef NtShape<64, 64, 2, 2, 4> Q8f;
typedef NtShape<64, 256, 2, 4, 2> Q8g;
typedef NtShape<32, 64, 1, 2, 4> Q8h;
typedef NtShape<128, 256, 2, 2, 2> Q8p;
typedef NtShape<64, 256, 1, 4, 3> Q8q;
typedef NtShape<128, 128, 2, 4, 2> Q8r;
typedef NtShape<128, 128, 2, 2, 2> Q8Small;

struct Q8Layout {
  size_t sx, prefix, tail, h, hq, sh, bytes;
};
Q8Layout q8_layout(const moe_desc& d) {
  Q8Layout l;
  const size_t rx = (size_t)d.T * d.top_k + (d.n_shared ? d.T : 0), R = (size_t)rows_total(d);
  l.sx = align256(rx * d.d_model);
  l.prefix = l.sx + align256(rx * 4);
  l.tail = l.prefix + align256((d.local_count + d.n_shared + 1) * 4);
  l.h = l.tail + align256((d.local_count + d.n_shared + 1) * 4);
  l.hq = l.h + align256(R * d.d_ff * 4);
  l.sh = l.hq + align256(R * d.d_ff);
  l.bytes = l.sh + align256(R * 4);
  return l;
}

template <typename S, bool DOWN>
hipError_t q8_gemm(const char* name, const moe_desc& d, Q8Args a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kern = q8_gemm_kernel<S, DOWN>;
  if (hipError_t e = lds_limit_once((const void*)kern, S::LDS, done); e != hipSuccess) return e;
  a.ga.n_tiles = DOWN ? (d.d_model + S::BN - 1) / S::BN : d.d_ff / (S::BN / 2);
  const int64_t most = std::min((int64_t)d.T * d.top_k / S::BM + d.local_count,
                                (int64_t)d.local_count * ((d.T + S::BM - 1) / S::BM)) +
                       (int64_t)d.n_shared * ((d.T + S::BM - 1) / S::BM);
  KernelTimer kt(name, s);
  // every XCD takes its share of the tiles and of the tails, each rounded up: at most two tiles more than an eighth of all
  hipLaunchKernelGGL(kern, dim3((unsigned)(most * a.ga.n_tiles / 8 * 8 + 16)), dim3(S::NT), S::LDS, s, a);
  return hipGetLastError();
}

unsigned row_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

}  // namespace

size_t ffn_q8_ws_bytes(const moe_desc& d) { return q8_layout(d).bytes; }

hipError_t launch_q8_pack(int n, int rows, int cols, int dtype, const void* w, void* codes, void* scales, hipStream_t s) {
  const int64_t all = (int64_t)n * rows;
  KernelTimer kt("q8_pack", s);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(q8_pack_kernel<bf16>, dim3(row_grid(all)), dim3(Q8_THREADS), 0, s, (const bf16*)w, all, cols, (int8_t*)codes,
                       (float*)scales);
  else
    hipLaunchKernelGGL(q8_pack_kernel<float>, dim3(row_grid(all)), dim3(Q8_THREADS), 0, s, (const float*)w, all, cols,
                       (int8_t*)codes, (float*)scales);
  return hipGetLastError();
}

hipError_t launch_q8_unpack(int n, int rows, int cols, int dtype, const void* codes, const void* scales, void* w,
                            hipStream_t s) {
  const int64_t all = (int64_t)n * rows;
  KernelTimer kt("q8_unpack", s);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(q8_unpack_kernel<bf16>, dim3(row_grid(all)), dim3(Q8_THREADS), 0, s, (const int8_t*)codes,
                       (const float*)scales, all, cols, (bf16*)w);
  else
    hipLaunchKernelGGL(q8_unpack_kernel<float>, dim3(row_grid(all)), dim3(Q8_THREADS), 0, s, (const int8_t*)codes,
                       (const float*)scales, all, cols, (float*)w);
  return hipGetLastError();
}

hipError_t launch_ffn_q8(const moe_desc& d, const void* x, const void* xp, const int32_t* offsets, const Q8Weights& gate,
                         const Q8Weights& up, const Q8Weights& down, void* yp, void* ws, hipStream_t s) {
  const Q8Layout l = q8_layout(d);
  char* base = (char*)ws;
  Q8Args a{};
  a.ga.T = d.T;
  a.ga.k = d.top_k;
  a.ga.d = d.d_model;
  a.ga.f = d.d_ff;
  a.ga.Eloc = d.local_count;
  a.ga.S = d.n_shared;
  a.ga.rows_cap = d.T * d.top_k;
  a.ga.offsets = offsets;
  a.prefix = (int32_t*)(base + l.prefix);
  a.ga.mt_prefix = a.prefix;
  a.tail = nullptr;
  a.x = x;
  a.xp = xp;
  a.xq = (int8_t*)base;
  a.sx = (float*)(base + l.sx);
  a.h = (float*)(base + l.h);
  a.hq = (int8_t*)(base + l.hq);
  a.sh = (float*)(base + l.sh);
  a.wg = (const int8_t*)gate.codes;
  a.wu = (const int8_t*)up.codes;
  a.wd = (const int8_t*)down.codes;
  a.sg = (const float*)gate.scales;
  a.su = (const float*)up.scales;
  a.sd = (const float*)down.scales;
  a.y = (bf16*)yp;
  // rows per expert
  const double rows = (double)d.T * d.top_k / d.n_experts;
  bool large = rows >= 192;
  const char* e = getenv("Q8_TILE");
  const char shape = e ? e[0] : large ? 'l' : 's';
  large = shape == 'l';
  a.bm = large ? 256 : 128;
  if (shape == 'b' || shape == 'c' || shape == 'f' || shape == 'g' || shape == 'q') a.bm = 64;
  if (shape == 'd' || shape == 'h') a.bm = 32;
  if (large) a.ga.mt_tail = a.tail = (int32_t*)(base + l.tail);
  const int rx = d.T * d.top_k + (d.n_shared ? d.T : 0);
  {
    KernelTimer kt("q8_rows_x", s);
    hipLaunchKernelGGL(q8_rows_x_kernel, dim3(rx + 1), dim3(Q8_THREADS), 0, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const auto gemm = [&](const char* name, auto down) {
    constexpr bool D = decltype(down)::value;
    switch (shape) {
      case 'l': return q8_gemm<Q8Large, D>(name, d, a, s);
      case 'b': return q8_gemm<Q8b, D>(name, d, a, s);
      case 'c': return q8_gemm<Q8c, D>(name, d, a, s);
      case 'd': return q8_gemm<Q8d, D>(name, d, a, s);
      case 'e': return q8_gemm<Q8e, D>(name, d, a, s);
      case 'f': return q8_gemm<Q8f, D>(name, d, a, s);
      case 'g': return q8_gemm<Q8g, D>(name, d, a, s);
      case 'p': return q8_gemm<Q8p, D>(name, d, a, s);
      case 'q': return q8_gemm<Q8q, D>(name, d, a, s);
      case 'r': return q8_gemm<Q8r, D>(name, d, a, s);
      case 'h': return q8_gemm<Q8h, D>(name, d, a, s);
    }
    return q8_gemm<Q8Small, D>(name, d, a, s);
  };
  if (hipError_t e = gemm("q8_gate_up", std::false_type{}); e != hipSuccess) return e;
  {
    KernelTimer kt("q8_rows_h", s);
    const auto rows_h = [&](auto keep) {
      hipLaunchKernelGGL(q8_rows_h_kernel<decltype(keep)::value>, dim3((unsigned)rows_total(d)), dim3(Q8_THREADS), 0, s, a);
    };
    if (d.d_ff <= 4 * 4 * Q8_THREADS) rows_h(std::integral_constant<int, 4>{});
    else rows_h(std::integral_constant<int, 16>{});
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return gemm("q8_down", std::true_type{});
}

}  // namespace pcmoe
