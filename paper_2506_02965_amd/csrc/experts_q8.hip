// Experts in 8-bit integers: weights with a scale for each output channel, rows of x and of H with a scale for each token.
//
// A row v is held as scale = fp32(m / 127), m = max|v|, and codes rint(127 v / m), ties to even. G = sx sg (x . g) with the
// sum over codes exact in int32 (127^2 K stays below 2^31), U likewise, H = silu(G) U in fp32, which is held in 8 bits per
// row again once the whole row is there, and y = sh sd (h . d). So a call is four launches: rows of x to codes, gate and up,
// rows of H to codes, down.
//
// Bound by the int8 matrix cores for long prompts (8192 tokens, 4096, 14336, 8 experts, 2 a token: gate and up 1,775 us, 2,170
// TOP/s; down 905, 2,130), where H passes memory once in fp32 and once in codes (210 us), and by the weights for few rows (24
// tokens, 2048, 1408, 64 experts: 64 + 34 us, 5.4 and 5.1 TB/s).
#include "nt_gemm.h"
#include "expert_ops.h"

#include <algorithm>
#include <cmath>

namespace pcmoe {

namespace {

constexpr int Q8_THREADS = 256;

__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }
// Largest magnitude bits over a row's threads, a wavefront or the workgroup (of fp32 numbers: infinities and NaN are above all
// finite ones).
template <int THREADS>
__device__ __forceinline__ uint32_t row_max_bits(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max_u32(v, (uint32_t)__shfl_xor((int)v, o, 64));
  if constexpr (THREADS > 64) {
    __shared__ uint32_t s[THREADS / 64];
    __syncthreads();  // the values of the last call have been read
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v = max_u32(v, s[w]);
  }
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

// A row of K values to codes and scale, by THREADS threads: the workgroup, or a wavefront where a row is at most four chunks a
// lane. SRC: bf16 or float; F64: exact quotients of fp32 values. The first KEEP chunks of a thread stay in registers; what a
// longer row has beyond them is read again.
template <typename SRC, bool F64, int KEEP, int THREADS>
__device__ __forceinline__ void code_row(const SRC* v, int K, int8_t* codes, float* scale) {
  constexpr int EP = EPC<SRC>::value;
  const int n = K / EP, t = threadIdx.x % THREADS;
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
    const int c = t + i * THREADS;
    kept[i] = c < n ? ld_chunk(v + c * EP) : zero_chunk();
  }
#pragma unroll
  for (int i = 0; i < KEEP; ++i) look(kept[i]);
  for (int c = t + KEEP * THREADS; c < n; c += THREADS) look(ld_chunk(v + c * EP));
  top = row_max_bits<THREADS>(top);
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
    const int c = t + i * THREADS;
    if (c < n) put(c, kept[i]);
  }
  for (int c = t + KEEP * THREADS; c < n; c += THREADS) put(c, ld_chunk(v + c * EP));
  if (t == 0) *scale = row_scale(top);
}

// Rows a workgroup works on at once where they are short: a row's wavefronts share nothing with the others'.
constexpr int ROWS = Q8_THREADS / 64;
template <typename T>
constexpr int short_row = 4 * 64 * EPC<T>::value;  // columns of the longest row that a wavefront takes

template <typename T, bool SHORT>
__global__ __launch_bounds__(Q8_THREADS) void q8_pack_kernel(const T* w, int64_t rows, int cols, int8_t* codes, float* scales) {
  constexpr int AT_ONCE = SHORT ? ROWS : 1;
  for (int64_t r = (int64_t)blockIdx.x * AT_ONCE + (SHORT ? threadIdx.x / 64 : 0); r < rows; r += (int64_t)gridDim.x * AT_ONCE)
    code_row<T, std::is_same<T, float>::value, 4, SHORT ? 64 : Q8_THREADS>(w + r * cols, cols, codes + r * cols, scales + r);
}

// 16 codes a thread.
template <typename T>
__global__ __launch_bounds__(Q8_THREADS) void q8_unpack_kernel(const int8_t* codes, const float* scales, int64_t rows, int cols,
                                                               T* w) {
  const int per_row = cols / 16;
  const int64_t all = rows * per_row, step = (int64_t)gridDim.x * Q8_THREADS;
  for (int64_t i = (int64_t)blockIdx.x * Q8_THREADS + threadIdx.x; i < all; i += step) {
    const float s = scales[i / per_row];
    const Chunk q = ld_chunk(codes + 16 * i);
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = (float)(int8_t)(q.w[e / 4] >> (8 * (e % 4))) * s;
#pragma unroll
    for (int e = 0; e < 16; e += EPC<T>::value) st_chunk(w + 16 * i + e, f_to_chunk<T>(v + e));
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
  int32_t *prefix, *tail, *mid, *few;  // [G + 1] each: m-tiles of 256 rows but the tails, tails, m-tiles of 128 and of 64 rows
};

// Codes of the rows of x_perm and x; the last workgroup makes the m-tile prefixes of the groups, a wavefront each.
template <bool SHORT>
__global__ __launch_bounds__(Q8_THREADS) void q8_rows_x_kernel(Q8Args a, int rows_x) {
  if (blockIdx.x == gridDim.x - 1) {
    const int lane = threadIdx.x & 63, which = threadIdx.x >> 6, bm = which < 2 ? 256 : which == 2 ? 128 : 64;
    int32_t* out = which == 0 ? a.prefix : which == 1 ? a.tail : which == 2 ? a.mid : a.few;
    const int G = a.ga.Eloc + a.ga.S;
    int carry = 0;
    if (lane == 0) out[0] = 0;
    for (int g0 = 0; g0 < G; g0 += 64) {
      const int g = g0 + lane;
      const int rows = g < a.ga.Eloc ? a.ga.offsets[g + 1] - a.ga.offsets[g] : g < G ? a.ga.T : 0;
      const int rem = rows % 256, is_tail = which < 2 && rem > 0 && rem <= 128 ? 1 : 0;
      int v = which == 1 ? is_tail : (rows + bm - 1) / bm - is_tail;
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
  const int r = SHORT ? blockIdx.x * ROWS + threadIdx.x / 64 : blockIdx.x;
  const bool routed = r < a.ga.rows_cap;
  if (r >= rows_x || (routed && r >= a.ga.offsets[a.ga.Eloc])) return;
  const bf16* v = routed ? (const bf16*)a.xp + (size_t)r * a.ga.d : (const bf16*)a.x + (size_t)(r - a.ga.rows_cap) * a.ga.d;
  code_row<bf16, false, SHORT ? 4 : 2, SHORT ? 64 : Q8_THREADS>(v, a.ga.d, a.xq + (size_t)r * a.ga.d, a.sx + r);
}
// Codes of the rows of H.
template <int KEEP, bool SHORT>
__global__ __launch_bounds__(Q8_THREADS) void q8_rows_h_kernel(Q8Args a, int64_t rows) {
  constexpr int AT_ONCE = SHORT ? ROWS : 1;
  const int64_t routed = a.ga.offsets[a.ga.Eloc];
  for (int64_t r = (int64_t)blockIdx.x * AT_ONCE + (SHORT ? threadIdx.x / 64 : 0); r < rows; r += (int64_t)gridDim.x * AT_ONCE)
    if (r >= a.ga.rows_cap || r < routed)
      code_row<float, false, KEEP, SHORT ? 64 : Q8_THREADS>(a.h + r * a.ga.f, a.ga.f, a.hq + r * a.ga.f, a.sh + r);
}

// 1 / (1 + exp(-g)) with the hardware's exponential and reciprocal. The exponential of a product rounded to fp32 alone would be
// |g| roundings off; what the product rounds away is put back. g stops where the result is one, and where it is 2^-126: the products
// of numbers next to the end of fp32's range would be infinite, and what they round away not a number.
__device__ __forceinline__ float sigmoid_of(float g) {
  g = __builtin_amdgcn_fmed3f(g, -87.3f, 128.f);
  const float t = -1.44269504f * g, r = __builtin_fmaf(-1.44269504f, g, -t) + -1.925963e-8f * g;
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(e, 0.693147181f * r, e));
}

// A tile's operands. Gate and up (DOWN = false): half of a wavefront's columns are gate rows, the other half the up rows of the
// same columns of H. Down: columns of y.
template <typename S, bool DOWN>
struct Q8Tile {
  static constexpr int HALF = S::WTN / 2;
  int32x4 ra, rb0, rb1;
  int K, m0, n0, at;
  size_t rs;         // the group's first row in the row space
  const float* sa;   // its rows' scales
  int g, rows;
  __device__ __forceinline__ Q8Tile(const Q8Args& a, const TileIdx& ti, int first) {
    const int d = a.ga.d, f = a.ga.f;
    K = DOWN ? f : d;
    g = ti.g;
    rows = ti.rows;
    m0 = first;
    n0 = DOWN ? ti.nt * S::BN : ti.nt * (S::BN / 2);  // first column of the output
    const bool routed = g < a.ga.Eloc;
    rs = routed ? (size_t)ti.row0 : (size_t)a.ga.rows_cap + (size_t)(g - a.ga.Eloc) * a.ga.T;
    const size_t rx = routed ? (size_t)ti.row0 : (size_t)a.ga.rows_cap;  // among the codes of x
    sa = DOWN ? a.sh + rs : a.sx + rx;
    ra = make_rsrc(DOWN ? a.hq + rs * f : a.xq + rx * d, (uint32_t)((size_t)rows * K));
    const size_t w = (size_t)g * f * d;
    rb0 = make_rsrc((DOWN ? a.wd : a.wg) + w, (uint32_t)((size_t)f * d));
    rb1 = DOWN ? rb0 : make_rsrc(a.wu + w, (uint32_t)((size_t)f * d));
    at = nt_lane(K);
  }
  __device__ __forceinline__ NtSrc a_rows(int kt, int j) const { return {ra, (m0 + 8 * j) * K + at + kt * NT_ROWB}; }
  __device__ __forceinline__ NtSrc b_rows(int kt, int j) const {
    if (DOWN) return {rb0, (n0 + 8 * j) * K + at + kt * NT_ROWB};
    const int r = 8 * j, w = r / S::WTN, in = r % S::WTN;
    return {pick_rsrc(in >= HALF, rb0, rb1), (n0 + w * HALF + in % HALF) * K + at + kt * NT_ROWB};
  }
  // Whether this wavefront has something to compute, and whether all its rows and columns are there.
  __device__ __forceinline__ bool live(const Q8Args& a) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return m0 + wave / S::WN * S::WTM < rows && (!DOWN || n0 + wave % S::WN * S::WTN < a.ga.d);
  }
  __device__ __forceinline__ bool full() const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return m0 + wave / S::WN * S::WTM + S::WTM <= rows;
  }
};

// Scales and stores of a tile. `meanwhile` is called between the loads of the scales and everything else.
template <typename S, bool DOWN, typename F>
__device__ __forceinline__ void q8_store(const Q8Args& a, const Q8Tile<S, DOWN>& t, I8::acc (&acc)[S::FM][S::FN], bool live,
                                         F&& meanwhile) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
  const int d = a.ga.d, f = a.ga.f, HALF = S::WTN / 2;
  const int m = t.m0 + wm * S::WTM + li, n = t.n0 + wn * (DOWN ? S::WTN : HALF) + 4 * q;
  float s[S::FM];
  floatx4 sw[S::FN];  // down: of the columns; else gate's, then up's
  if (live) {
#pragma unroll
    for (int i = 0; i < S::FM; ++i) s[i] = m + 16 * i < t.rows ? t.sa[m + 16 * i] : 0.f;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
      const float* from = DOWN ? a.sd + (size_t)t.g * d + n + 16 * j
                               : (j < S::FN / 2 ? a.sg : a.su) + (size_t)t.g * f + n + 16 * (j % (S::FN / 2));
      sw[j] = *reinterpret_cast<const floatx4*>(from);
    }
    // Waited for here. Left open, they would be waited for where the compiler cannot count what was issued since: with all of
    // the next tile's loads, and all of this one's stores.
#pragma unroll
    for (int i = 0; i < S::FM; ++i) asm volatile("" : "+v"(s[i]));
#pragma unroll
    for (int j = 0; j < S::FN; ++j) asm volatile("" : "+v"(sw[j]));
  }
  meanwhile();
  if (!live) return;
#pragma unroll
  for (int i = 0; i < S::FM; ++i) {
    if constexpr (S::PIPE) __builtin_amdgcn_sched_barrier(0);  // one row of blocks out of the accumulators at a time
    if (m + 16 * i >= t.rows) continue;
    if (DOWN) {
#pragma unroll
      for (int j = 0; j < S::FN; ++j) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (float)acc[i][j][e] * (s[i] * sw[j][e]);
        *reinterpret_cast<uint2*>(a.y + (t.rs + m + 16 * i) * d + n + 16 * j) = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
      }
    } else {
#pragma unroll
      for (int j = 0; j < S::FN / 2; ++j) {
        floatx4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float g = (float)acc[i][j][e] * (s[i] * sw[j][e]);
          const float u = (float)acc[i][j + S::FN / 2][e] * (s[i] * sw[j + S::FN / 2][e]);
          o[e] = g * sigmoid_of(g) * u;
        }
        *reinterpret_cast<floatx4*>(a.h + (t.rs + m + 16 * i) * f + n + 16 * j) = o;
      }
    }
  }
}

// One tile a workgroup.
template <typename S, bool DOWN>
__global__ __launch_bounds__(S::NT) void q8_gemm_kernel(Q8Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  TileIdx ti;
  if (!decode_tile<true>(a.ga, blockIdx.x, ti)) return;
  const Q8Tile<S, DOWN> t(a, ti, ti.mt * S::BM);
  const bool live = t.live(a);
  I8::acc acc[S::FM][S::FN];
  nt_loop<S, I8>(
      smem, t.K / NT_ROWB, live, [&](int kt, int j) { return t.a_rows(kt, j); }, [&](int kt, int j) { return t.b_rows(kt, j); },
      acc);
  q8_store<S, DOWN>(a, t, acc, live, [] {});
}

// Workgroups that stay, one a CU, and walk over the tiles of their XCD: 256 x 256, and 128 x 256 for tails (a group's last rows,
// at most 128), which come after the others. The next tile's first loads are issued before a tile is stored.
template <bool DOWN>
__global__ __launch_bounds__(256) void q8_walk_kernel(Q8Args a) {
  typedef NtShape<256, 256, 2, 2, 2> S;
  typedef NtShape<128, 256, 2, 2, 2> St;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int* const plan = reinterpret_cast<int*>(smem + S::LDS);  // prefix of the tiles, of the tails, row offsets: 512 each
  const int G = a.ga.Eloc + a.ga.S, lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < 512; i += 256) {
    plan[i] = i <= G ? a.prefix[i] : 0x7fffffff;
    plan[512 + i] = i <= G ? a.tail[i] : 0x7fffffff;
    plan[1024 + i] = i <= a.ga.Eloc ? a.ga.offsets[i] : 0;
  }
  __syncthreads();
  const int nt = a.ga.n_tiles, x = blockIdx.x & 7, stride = gridDim.x >> 3;
  const int body = __builtin_amdgcn_readfirstlane(plan[G]) * nt, tails = __builtin_amdgcn_readfirstlane(plan[512 + G]) * nt;
  const int nb = body / 8 + (x < body % 8 ? 1 : 0), nx = tails / 8 + (x < tails % 8 ? 1 : 0);  // of this XCD
  const int b0 = x * (body / 8) + min(x, body % 8), t0 = x * (tails / 8) + min(x, tails % 8);
  // Tile i of this XCD; false past the last.
  const auto decode = [&](int i, TileIdx& ti, bool& tail) __attribute__((always_inline)) {
    if (i >= nb + nx) return false;
    tail = i >= nb;
    const int L = tail ? t0 + i - nb : b0 + i;
    const int* pre = plan + (tail ? 512 : 0);
    const int mt = L / nt;   // among all m-tiles of its kind
    int g = 0;               // the last group whose prefix is at most mt
    for (int s = 0; s < G; s += 64) g += __popcll(__ballot(s + lane >= 1 && s + lane < G && pre[s + lane] <= mt));
    g = __builtin_amdgcn_readfirstlane(g);
    ti.g = g;
    const bool routed = g < a.ga.Eloc;
    ti.row0 = routed ? __builtin_amdgcn_readfirstlane(plan[1024 + g]) : 0;
    ti.rows = routed ? __builtin_amdgcn_readfirstlane(plan[1024 + g + 1]) - ti.row0 : a.ga.T;
    const int first = __builtin_amdgcn_readfirstlane(plan[g]), count = __builtin_amdgcn_readfirstlane(plan[g + 1]) - first;
    if (tail) {
      ti.mt = count;  // after the group's others
      ti.nt = L - mt * nt;
    } else {  // m-tiles in bunches of GROUP_M per n-tile
      const int l = L - first * nt, blk = l / (GROUP_M * nt), rem = l - blk * GROUP_M * nt, n = min(GROUP_M, count - blk * GROUP_M);
      ti.nt = rem / n;
      ti.mt = blk * GROUP_M + rem % n;
    }
    ti.mt = __builtin_amdgcn_readfirstlane(ti.mt);
    ti.nt = __builtin_amdgcn_readfirstlane(ti.nt);
    return true;
  };
  const auto fill = [&](const TileIdx& ti, bool tail) __attribute__((always_inline)) {
    if (tail) {
      const Q8Tile<St, DOWN> t(a, ti, ti.mt * 256);
      nt_fill<St>(smem, t.K / NT_ROWB, [&](int kt, int j) { return t.a_rows(kt, j); }, [&](int kt, int j) { return t.b_rows(kt, j); });
    } else {
      const Q8Tile<S, DOWN> t(a, ti, ti.mt * 256);
      nt_fill<S>(smem, t.K / NT_ROWB, [&](int kt, int j) { return t.a_rows(kt, j); }, [&](int kt, int j) { return t.b_rows(kt, j); });
    }
  };
  TileIdx ti, next;
  bool tail = false, next_tail = false, behind = false;
  int i = blockIdx.x >> 3;
  bool more = decode(i, ti, tail);
  if (more) fill(ti, tail);
  while (more) {
    i += stride;
    const bool there = decode(i, next, next_tail);
    const auto tile = [&](auto shape) __attribute__((always_inline)) {
      using Sh = decltype(shape);
      const Q8Tile<Sh, DOWN> t(a, ti, ti.mt * 256);
      const bool live = t.live(a);
      I8::acc acc[Sh::FM][Sh::FN];
      nt_pipe<Sh, I8>(
          smem, t.K / NT_ROWB, live, behind, [&](int kt, int j) { return t.a_rows(kt, j); },
          [&](int kt, int j) { return t.b_rows(kt, j); }, acc);
      q8_store<Sh, DOWN>(a, t, acc, live, [&]() __attribute__((always_inline)) {
        if (there) fill(next, next_tail);
      });
      behind = live && t.full();
    };
    if (tail) tile(St{});
    else tile(S{});
    more = there;
    ti = next;
    tail = next_tail;
  }
}

typedef NtShape<128, 128, 2, 4, 2> Q8Mid;   // two workgroups a CU
typedef NtShape<64, 128, 2, 4, 3> Q8Few;

struct Q8Layout {
  size_t sx, prefix, tail, mid, few, h, hq, sh, bytes;
};
Q8Layout q8_layout(const moe_desc& d) {
  Q8Layout l;
  const size_t rx = (size_t)d.T * d.top_k + (d.n_shared ? d.T : 0), R = (size_t)rows_total(d);
  l.sx = align256(rx * d.d_model);
  l.prefix = l.sx + align256(rx * 4);
  l.tail = l.prefix + align256((d.local_count + d.n_shared + 1) * 4);
  const size_t plan = l.tail - l.prefix;
  l.mid = l.tail + plan;
  l.few = l.mid + plan;
  l.h = l.few + plan;
  l.hq = l.h + align256(R * d.d_ff * 4);
  l.sh = l.hq + align256(R * d.d_ff);
  l.bytes = l.sh + align256(R * 4);
  return l;
}

// An upper bound of the m-tiles of bm rows, and what to expect of them: half a tile of each group is empty.
int64_t most_tiles(const moe_desc& d, int bm) {
  const int64_t of_all = (d.T + bm - 1) / bm;
  return std::min((int64_t)d.T * d.top_k / bm + d.local_count, d.local_count * of_all) + d.n_shared * of_all;
}
double mean_rows(const moe_desc& d) {
  return ((double)d.T * d.top_k / d.n_experts * d.local_count + (double)d.T * d.n_shared) / (d.local_count + d.n_shared);
}
double expected_tiles(const moe_desc& d, int bm) {
  return (d.local_count + d.n_shared) * (mean_rows(d) / bm + 0.5);
}

// Which tiles a contraction takes.
//   Few rows a group: 64 x 128, two workgroups of eight wavefronts a CU with two K-tiles of weights on their way each. Fewer than
//   64 rows, or so few tiles that 128 x 128 ones would leave CUs idle.
//   Else by the rounds of the chip and what a tile costs (us): 1.55 a K-tile and 10 for the 256 x 256 tiles, 1.15 and 3 for the
//   128 x 128 tiles, two at once.
// us of gate and up / down for 64-row, 128-row and 256-row tiles (d, f, experts: rows an expert):
//   4096, 14336, 8:  6: 161/83  172/113  188/145;  75: 237/128  196/124  216/156;  250: 427/240  369/246  335/198;
//                    500: 783/413  623/346  522/322
//   1024, 2816, 16:  32: 22/15  23/19  32/25;  97: 28/15  27/22  35/28;  375: 72/35  62/31  69/44
//   2048, 1408, 64:  12: 71/39  76/41  86/46;  96: 103/60  98/54  107/56;  384: 259/156  224/140  222/129
// (64 x 128 with four wavefronts: 97 rows of 1024, 2816, 16: 31/18. 64 x 256, 128 x 64, 64 x 64, 32 x 128 and four stages of 128 x
// 128 tiles, one workgroup a CU, were slower in most cells.)
enum Q8Tiles { Q8_FEW, Q8_MID, Q8_LARGE };
Q8Tiles pick_tiles(const moe_desc& d, bool down) {
  const double kts = (down ? d.d_ff : d.d_model) / 128., cus = device_cus(), n = down ? d.d_model : 2. * d.d_ff;
  const double large = expected_tiles(d, 256) * std::ceil(n / 256), mid = expected_tiles(d, 128) * std::ceil(n / 128);
  if (mean_rows(d) < 64 || mid <= cus) return Q8_FEW;
  return std::ceil(large / cus) * (1.55 * kts + 10) <= std::ceil(mid / (2 * cus)) * (1.15 * kts + 3) ? Q8_LARGE : Q8_MID;
}

template <typename S, bool DOWN>
hipError_t q8_gemm(const char* name, const moe_desc& d, Q8Args a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kern = q8_gemm_kernel<S, DOWN>;
  if (hipError_t e = lds_limit_once((const void*)kern, S::LDS, done); e != hipSuccess) return e;
  a.ga.n_tiles = DOWN ? (d.d_model + S::BN - 1) / S::BN : d.d_ff / (S::BN / 2);
  KernelTimer kt(name, s);
  hipLaunchKernelGGL(kern, dim3((unsigned)((most_tiles(d, S::BM) * a.ga.n_tiles + 7) / 8 * 8)), dim3(S::NT), S::LDS, s, a);
  return hipGetLastError();
}
template <bool DOWN>
hipError_t q8_walk(const char* name, const moe_desc& d, Q8Args a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kern = q8_walk_kernel<DOWN>;
  constexpr int lds = NtShape<256, 256, 2, 2, 2>::LDS + 3 * 512 * 4;
  if (hipError_t e = lds_limit_once((const void*)kern, lds, done); e != hipSuccess) return e;
  a.ga.n_tiles = DOWN ? (d.d_model + 255) / 256 : d.d_ff / 128;
  KernelTimer kt(name, s);
  hipLaunchKernelGGL(kern, dim3(std::max(8, device_cus() / 8 * 8)), dim3(256), lds, s, a);
  return hipGetLastError();
}

unsigned row_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

}  // namespace

size_t ffn_q8_ws_bytes(const moe_desc& d) { return q8_layout(d).bytes; }

hipError_t launch_q8_pack(int n, int rows, int cols, int dtype, const void* w, void* codes, void* scales, hipStream_t s) {
  const int64_t all = (int64_t)n * rows;
  KernelTimer kt("q8_pack", s);
  const auto go = [&](auto t) {
    using T = decltype(t);
    if (cols <= short_row<T>)
      hipLaunchKernelGGL((q8_pack_kernel<T, true>), dim3(row_grid((all + ROWS - 1) / ROWS)), dim3(Q8_THREADS), 0, s,
                         (const T*)w, all, cols, (int8_t*)codes, (float*)scales);
    else
      hipLaunchKernelGGL((q8_pack_kernel<T, false>), dim3(row_grid(all)), dim3(Q8_THREADS), 0, s, (const T*)w, all, cols,
                         (int8_t*)codes, (float*)scales);
  };
  if (dtype == MOE_BF16) go(bf16{});
  else go(float{});
  return hipGetLastError();
}

hipError_t launch_q8_unpack(int n, int rows, int cols, int dtype, const void* codes, const void* scales, void* w,
                            hipStream_t s) {
  const int64_t all = (int64_t)n * rows;
  const unsigned grid = row_grid((all * (cols / 16) + Q8_THREADS - 1) / Q8_THREADS);
  KernelTimer kt("q8_unpack", s);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(q8_unpack_kernel<bf16>, dim3(grid), dim3(Q8_THREADS), 0, s, (const int8_t*)codes,
                       (const float*)scales, all, cols, (bf16*)w);
  else
    hipLaunchKernelGGL(q8_unpack_kernel<float>, dim3(grid), dim3(Q8_THREADS), 0, s, (const int8_t*)codes,
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
  a.tail = (int32_t*)(base + l.tail);
  a.mid = (int32_t*)(base + l.mid);
  a.few = (int32_t*)(base + l.few);
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
  const int rx = d.T * d.top_k + (d.n_shared ? d.T : 0);
  {
    KernelTimer kt("q8_rows_x", s);
    if (d.d_model <= short_row<bf16>)
      hipLaunchKernelGGL(q8_rows_x_kernel<true>, dim3((rx + ROWS - 1) / ROWS + 1), dim3(Q8_THREADS), 0, s, a, rx);
    else
      hipLaunchKernelGGL(q8_rows_x_kernel<false>, dim3(rx + 1), dim3(Q8_THREADS), 0, s, a, rx);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const auto gemm = [&](const char* name, auto down) {
    constexpr bool D = decltype(down)::value;
    const Q8Tiles tiles = pick_tiles(d, D);
    a.ga.mt_prefix = tiles == Q8_FEW ? a.few : a.mid;
    if (tiles == Q8_LARGE) return q8_walk<D>(name, d, a, s);
    return tiles == Q8_MID ? q8_gemm<Q8Mid, D>(name, d, a, s) : q8_gemm<Q8Few, D>(name, d, a, s);
  };
  if (hipError_t e = gemm("q8_gate_up", std::false_type{}); e != hipSuccess) return e;
  {
    KernelTimer kt("q8_rows_h", s);
    const int64_t rows = rows_total(d);
    const auto rows_h = [&](auto keep, auto is_short) {
      constexpr bool SHORT = decltype(is_short)::value;
      const unsigned grid = row_grid(SHORT ? (rows + ROWS - 1) / ROWS : rows);
      hipLaunchKernelGGL((q8_rows_h_kernel<decltype(keep)::value, SHORT>), dim3(grid), dim3(Q8_THREADS), 0, s, a, rows);
    };
    if (d.d_ff <= short_row<float>) rows_h(std::integral_constant<int, 4>{}, std::true_type{});
    else if (d.d_ff <= 4 * 4 * Q8_THREADS) rows_h(std::integral_constant<int, 4>{}, std::false_type{});
    else rows_h(std::integral_constant<int, 16>{}, std::false_type{});
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return gemm("q8_down", std::true_type{});
}

}  // namespace pcmoe
