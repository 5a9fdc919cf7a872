// What stands between two layers of a stack: r = alpha x + gamma * post(y), h = pre(r), and the adjoint of both.
//
// RMS: N(v) = v / sqrt(mean(v^2) + eps) * w; LAYER: the same of v - mean(v). With vhat = N(v) / w and a = dN w,
// dv = (a - vhat mean(a vhat) [- mean(a)]) / sqrt(...). Both passes are bound by memory: every row is read once, kept in
// registers and written once. Row sums are fp64, those of products with gradients fp64 sums of a chunk's in fp32, so that none
// overflows whose row and gradients do not, and means are kept in two fp32 parts, so that one far from zero costs no digits;
// everything else is fp32, rounded once on the way out.
// 16384 x 2048 bf16 with a post norm and a gate: 268 MB in 44 us alone and 51 among other passes. Adjoint of 8192 x 4096: 403 MB
// in 67 + 5; of 777 x 1024 fp32 with layer norms 10 + 4, two launches and a row's three sums one after the other.
#include "expert_ops.h"

#include <algorithm>

namespace pcmoe {

namespace {

constexpr int kMaxWaves = 16;

struct NormArgs {
  int T, d, cpr;        // tokens, columns, 16-byte chunks of a row
  int pre, post;        // moe_norm_kind
  int gate_rows;        // tokens that share a gate row
  int groups;           // gate rows (1 without a gate)
  float alpha;
  double eps, inv_d;
  const void *x, *y, *w_post, *gate, *w_pre;
  void *r, *h;
  // adjoint
  const void *dr, *dh;
  void *dx, *dy;
  float *dw_post, *dgate, *dw_pre;
  float* part;          // partial sums [3][n_part][d]: dw_pre, dw_post, dgate
  int n_part;           // workgroups
  int parts;            // workgroups of a gate row (0: workgroups of whole gate rows)
  int direct;           // the only workgroup writes the sums themselves
};

// Sum over a wavefront, in every lane: DPP within 16 lanes, then the four row sums from scalar registers.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double lane_of(double v, int l) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, l);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), l);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double sum64(double v) {
  v += dpp<0xb1>(v);   // lanes 1 apart
  v += dpp<0x4e>(v);   // 2 apart
  v += dpp<0x141>(v);  // mirrored within 8
  v += dpp<0x140>(v);  // mirrored within 16
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// Sums of N fp64 values over the workgroup's wavefronts. Consecutive calls alternate between two halves of `lds`: a wavefront that
// writes a half again has passed the barrier that the others reach after reading it.
constexpr int kMaxSums = 3;
struct Sums {
  double v[kMaxSums];
};
struct SumLds {
  Sums s[2][kMaxWaves];
};
template <int N>
__device__ __forceinline__ Sums block_sum(Sums v, SumLds& lds, int& turn) {
#pragma unroll
  for (int k = 0; k < N; ++k) v.v[k] = sum64(v.v[k]);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return v;
  Sums* at = lds.s[turn];
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) at[threadIdx.x >> 6].v[k] = v.v[k];
  __syncthreads();
  Sums t{};
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int k = 0; k < N; ++k) t.v[k] += at[w].v[k];
  turn ^= 1;
  return t;
}

// A value that all lanes hold, in a scalar register where S.
template <bool S = true>
__device__ __forceinline__ float uniform(float v) {
  return S ? __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))) : v;
}

// A mean as two fp32 parts. v - hi is exact where v is within a factor of two of it, so that v - mean is off by its own rounding
// only, however far the mean is above the deviation (rounded to fp32 alone, a mean of 1e4 deviations would move every v of the
// row by up to 2^-11 of one).
struct Mean {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ Mean() {}
  __device__ __forceinline__ explicit Mean(double m) : hi((float)m), lo((float)(m - (double)(float)m)) {}
  template <bool S>
  __device__ __forceinline__ Mean in() const {
    Mean m;
    m.hi = uniform<S>(hi);
    m.lo = uniform<S>(lo);
    return m;
  }
  __device__ __forceinline__ float from(float v) const { return (v - hi) - lo; }  // v - mean
};

// A power of two that takes a chunk's differences from the mean, of which q is the sum of squares, to about one, and back: their
// products with gradients are added up in fp32 within a chunk, where those of rows above 1e19 could overflow.
struct Scale {
  int e;
  __device__ __forceinline__ explicit Scale(double q) : e(max(-100, min(120, (((__double2hiint(q) >> 20) & 0x7ff) - 1023) >> 1))) {}
  __device__ __forceinline__ float down() const { return __int_as_float((127 - e) << 23); }
  __device__ __forceinline__ double up() const { return __hiloint2double((1023 + e) << 20, 0); }
};

// 1 / sqrt(v) to fp32: the hardware's estimate (23 bits) and a Newton step, in fp64 for its range.
__device__ __forceinline__ float rsqrt_of(double v) {
  const double y = __builtin_amdgcn_rsq(v);
  return y == 0. ? 0.f : (float)(y * fma(-0.5 * v * y, y, 1.5));  // an infinite sum
}

// The chunk of a thread's i-th piece, and whether the row has it.
#define PIECE(i) const int c = threadIdx.x + (i) * blockDim.x; const bool in = c < a.cpr

template <typename T, int CPT, int NT>
__global__ __launch_bounds__(NT) void residual_norm_kernel(NormArgs a) {
  constexpr int EP = EPC<T>::value;
  __shared__ SumLds lds;
  int turn = 0;
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    const size_t row = (size_t)t * a.cpr;
    const Chunk* gate = a.gate ? (const Chunk*)a.gate + (size_t)(t / a.gate_rows) * a.cpr : nullptr;
    float v[CPT][EP];
    if (a.y) {
      Chunk yc[CPT], xc[CPT], gc[CPT];
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        yc[i] = in ? ld_chunk((const Chunk*)a.y + row + c) : zero_chunk();
        xc[i] = in ? ld_chunk((const Chunk*)a.x + row + c) : zero_chunk();
        gc[i] = gate && in ? ld_chunk(gate + c) : zero_chunk();
      }
      Mean mean;
      float rstd = 1.f;
      if (a.post == MOE_NORM_LAYER) {
        Sums s{};
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          float y[EP];
          chunk_to_f<T>(yc[i], y);
#pragma unroll
          for (int e = 0; e < EP; ++e) s.v[0] += (double)y[e];
        }
        mean = Mean(block_sum<1>(s, lds, turn).v[0] * a.inv_d);
      }
      if (a.post != MOE_NORM_NONE) {
        Sums s{};
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          PIECE(i);
          float y[EP];
          chunk_to_f<T>(yc[i], y);
          if (in)
#pragma unroll
            for (int e = 0; e < EP; ++e) s.v[0] += (double)mean.from(y[e]) * (double)mean.from(y[e]);
        }
        rstd = rsqrt_of(block_sum<1>(s, lds, turn).v[0] * a.inv_d + a.eps);
      }
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        float x[EP], y[EP], g[EP], w[EP];
        chunk_to_f<T>(xc[i], x);
        chunk_to_f<T>(yc[i], y);
        chunk_to_f<T>(gc[i], g);
        chunk_to_f<T>(a.w_post && in ? ld_chunk((const Chunk*)a.w_post + c) : zero_chunk(), w);
#pragma unroll
        for (int e = 0; e < EP; ++e) {
          float n = mean.from(y[e]) * rstd;
          if (a.w_post) n *= w[e];
          if (gate) n *= g[e];
          v[i][e] = a.alpha * x[e] + n;
        }
        if (in) st_chunk((Chunk*)a.r + row + c, f_to_chunk<T>(v[i]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        chunk_to_f<T>(in ? ld_chunk((const Chunk*)a.x + row + c) : zero_chunk(), v[i]);
      }
    }
    if (a.pre == MOE_NORM_NONE) continue;
    Mean mean;
    if (a.pre == MOE_NORM_LAYER) {
      Sums s{};
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        if (in)
#pragma unroll
          for (int e = 0; e < EP; ++e) s.v[0] += (double)v[i][e];
      }
      mean = Mean(block_sum<1>(s, lds, turn).v[0] * a.inv_d);
    }
    Sums s{};
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      PIECE(i);
      if (in)
#pragma unroll
        for (int e = 0; e < EP; ++e) s.v[0] += (double)mean.from(v[i][e]) * (double)mean.from(v[i][e]);
    }
    const float rstd = rsqrt_of(block_sum<1>(s, lds, turn).v[0] * a.inv_d + a.eps);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      PIECE(i);
      if (!in) continue;
      float o[EP], w[EP];
      if (a.w_pre) chunk_to_f<T>(ld_chunk((const Chunk*)a.w_pre + c), w);
#pragma unroll
      for (int e = 0; e < EP; ++e) {
        o[e] = mean.from(v[i][e]) * rstd;
        if (a.w_pre) o[e] *= w[e];
      }
      st_chunk((Chunk*)a.h + row + c, f_to_chunk<T>(o));
    }
  }
}

// Adjoint. A workgroup walks over the rows of a part of a gate row's tokens (or over whole gate rows) and keeps the sums over
// tokens of its columns in registers; norm_sums_kernel adds the workgroups' up in a fixed order.
template <typename T, int CPT, int NT, bool PRE, bool POST>
__global__ __launch_bounds__(NT) void residual_norm_bwd_kernel(NormArgs a) {
  constexpr int EP = EPC<T>::value;
  __shared__ SumLds lds;
  int turn = 0;
  const bool need_y = a.y && (POST || a.gate);
  // Row sums in scalar registers where vector registers are short (8192 x 7168 bf16 176 -> 168 us; 8192 x 4096 96 -> 98).
  constexpr bool SCALAR = CPT * EP > 8;
  const bool lr = PRE && a.pre == MOE_NORM_LAYER, ly = POST && a.post == MOE_NORM_LAYER;
  float s_pre[CPT][EP], s_post[CPT][EP], s_gate[CPT][EP];
  Chunk wpre[CPT], wpost[CPT], gc[CPT];
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    PIECE(i);
    wpre[i] = PRE && a.w_pre && in ? ld_chunk((const Chunk*)a.w_pre + c) : zero_chunk();
    wpost[i] = POST && a.w_post && in ? ld_chunk((const Chunk*)a.w_post + c) : zero_chunk();
#pragma unroll
    for (int e = 0; e < EP; ++e) s_pre[i][e] = s_post[i][e] = 0.f;
  }
  // gate rows of this workgroup, and its tokens of each
  int g0, g1, first, last;
  if (a.parts) {
    g0 = blockIdx.x / a.parts;
    g1 = g0 + 1;
    const int p = blockIdx.x - g0 * a.parts;
    first = (int)((int64_t)a.gate_rows * p / a.parts);
    last = (int)((int64_t)a.gate_rows * (p + 1) / a.parts);
  } else {
    g0 = (int)((int64_t)a.groups * blockIdx.x / a.n_part);
    g1 = (int)((int64_t)a.groups * (blockIdx.x + 1) / a.n_part);
    first = 0;
    last = a.gate_rows;
  }
  for (int g = g0; g < g1; ++g) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      PIECE(i);
      gc[i] = a.gate && in ? ld_chunk((const Chunk*)a.gate + (size_t)g * a.cpr + c) : zero_chunk();
#pragma unroll
      for (int e = 0; e < EP; ++e) s_gate[i][e] = 0.f;
    }
    // the next row's chunks are loaded while a row is worked on
    Chunk next[4][CPT];
    const auto fetch = [&](int t, bool there) {
      const size_t row = (size_t)t * a.cpr;
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        const bool ld = in && there;
        next[0][i] = a.dr && ld ? ld_chunk((const Chunk*)a.dr + row + c) : zero_chunk();
        next[1][i] = PRE && ld ? ld_chunk((const Chunk*)a.dh + row + c) : zero_chunk();
        next[2][i] = PRE && ld ? ld_chunk((const Chunk*)a.r + row + c) : zero_chunk();
        next[3][i] = need_y && ld ? ld_chunk((const Chunk*)a.y + row + c) : zero_chunk();
      }
    };
    const int t1 = g * a.gate_rows + last;
    fetch(g * a.gate_rows + first, first < last);
    for (int t = g * a.gate_rows + first; t < t1; ++t) {
      const size_t row = (size_t)t * a.cpr;
      Chunk drc[CPT], dhc[CPT], rc[CPT], yc[CPT];
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        drc[i] = next[0][i];
        dhc[i] = next[1][i];
        rc[i] = next[2][i];
        yc[i] = next[3][i];
      }
      fetch(t + 1, t + 1 < t1);
      // row sums: of r and y (LAYER), then of their squares with those of a = dh w_pre
      Mean mr, my;
      float ma = 0.f, rr = 1.f, ry = 1.f, car = 0.f;
      if (lr || ly) {
        Sums s{};
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          float r[EP], y[EP], dh[EP], w[EP];
          chunk_to_f<T>(rc[i], r);
          chunk_to_f<T>(yc[i], y);
          chunk_to_f<T>(dhc[i], dh);
          chunk_to_f<T>(wpre[i], w);
          float fa = 0.f;
#pragma unroll
          for (int e = 0; e < EP; ++e) {
            if (lr) s.v[0] += (double)r[e];
            if (ly) s.v[1] += (double)y[e];
            if (lr) fa += a.w_pre ? dh[e] * w[e] : dh[e];
          }
          s.v[2] += (double)fa;
        }
        s = block_sum<3>(s, lds, turn);
        if (lr) mr = Mean(s.v[0] * a.inv_d).template in<SCALAR>();
        if (ly) my = Mean(s.v[1] * a.inv_d).template in<SCALAR>();
        if (lr) ma = (float)(s.v[2] * a.inv_d);
      }
      if (PRE || POST) {
        Sums s{};
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          PIECE(i);
          float r[EP], y[EP], dh[EP], w[EP];
          chunk_to_f<T>(rc[i], r);
          chunk_to_f<T>(yc[i], y);
          chunk_to_f<T>(dhc[i], dh);
          chunk_to_f<T>(wpre[i], w);
          if (!in) continue;
          if (PRE) {
            double q = 0.;
#pragma unroll
            for (int e = 0; e < EP; ++e) {
              r[e] = mr.from(r[e]);
              q += (double)r[e] * (double)r[e];
            }
            s.v[0] += q;
            const Scale by(q);
            float f = 0.f;
#pragma unroll
            for (int e = 0; e < EP; ++e) f += (a.w_pre ? dh[e] * w[e] : dh[e]) * (r[e] * by.down());
            s.v[2] += (double)f * by.up();
          }
          if (POST)
#pragma unroll
            for (int e = 0; e < EP; ++e) s.v[1] += (double)my.from(y[e]) * (double)my.from(y[e]);
        }
        s = block_sum<PRE ? 3 : 2>(s, lds, turn);
        if (PRE) rr = uniform<SCALAR>(rsqrt_of(s.v[0] * a.inv_d + a.eps));
        if (POST) ry = uniform<SCALAR>(rsqrt_of(s.v[1] * a.inv_d + a.eps));
        if (PRE) car = uniform<SCALAR>((float)(s.v[2] * a.inv_d * (double)rr));  // mean(a rhat)
      }
      float b[CPT][EP];  // gradient of r, then of post(y)
      Sums s{};
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        float dr[EP], dh[EP], r[EP], y[EP], w[EP], wp[EP], gt[EP], o[EP];
        chunk_to_f<T>(drc[i], dr);
        chunk_to_f<T>(dhc[i], dh);
        chunk_to_f<T>(rc[i], r);
        chunk_to_f<T>(yc[i], y);
        chunk_to_f<T>(wpre[i], w);
        chunk_to_f<T>(wpost[i], wp);
        chunk_to_f<T>(gc[i], gt);
        float fb = 0.f, fm = 0.f;
#pragma unroll
        for (int e = 0; e < EP; ++e) {
          float gr = dr[e];
          if (PRE) {
            const float rhat = mr.from(r[e]) * rr;
            gr += (((a.w_pre ? dh[e] * w[e] : dh[e]) - ma) - rhat * car) * rr;
            s_pre[i][e] += dh[e] * rhat;
          }
          o[e] = a.alpha * gr;
          const float yhat = my.from(y[e]) * ry;
          if (a.gate) s_gate[i][e] += gr * (POST && a.w_post ? yhat * wp[e] : yhat);
          b[i][e] = a.gate ? gr * gt[e] : gr;
          if (POST) {
            s_post[i][e] += b[i][e] * yhat;
            if (a.w_post) b[i][e] *= wp[e];
            if (in) {
              fb += b[i][e] * yhat;
              if (ly) fm += b[i][e];
            }
          }
        }
        if (POST) {
          s.v[0] += (double)fb;
          if (ly) s.v[1] += (double)fm;
        }
        if (in) st_chunk((Chunk*)a.dx + row + c, f_to_chunk<T>(o));
      }
      if (!a.dy) continue;
      if (POST) {
        s = ly ? block_sum<2>(s, lds, turn) : block_sum<1>(s, lds, turn);
        const float cy = (float)(s.v[0] * a.inv_d), mb = (float)(s.v[1] * a.inv_d);
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          float y[EP];
          chunk_to_f<T>(yc[i], y);
#pragma unroll
          for (int e = 0; e < EP; ++e) b[i][e] = ((b[i][e] - mb) - my.from(y[e]) * ry * cy) * ry;
        }
      }
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        if (in) st_chunk((Chunk*)a.dy + row + c, f_to_chunk<T>(b[i]));
      }
    }
    if (a.gate) {
      float* out = a.parts > 1 ? a.part + ((size_t)2 * a.n_part + blockIdx.x) * a.d : a.dgate + (size_t)g * a.d;
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        if (!in) continue;
#pragma unroll
        for (int e = 0; e < EP; e += 4) st_chunk(out + c * EP + e, f_to_chunk<float>(&s_gate[i][e]));
      }
    }
  }
  float* o_pre = a.direct ? a.dw_pre : a.part + (size_t)blockIdx.x * a.d;
  float* o_post = a.direct ? a.dw_post : a.part + ((size_t)a.n_part + blockIdx.x) * a.d;
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    PIECE(i);
    if (!in) continue;
#pragma unroll
    for (int e = 0; e < EP; e += 4) {
      if (PRE && a.dw_pre) st_chunk(o_pre + c * EP + e, f_to_chunk<float>(&s_pre[i][e]));
      if (POST && a.dw_post) st_chunk(o_post + c * EP + e, f_to_chunk<float>(&s_post[i][e]));
    }
  }
}
#undef PIECE

// Sums of the workgroups' partial rows. blockIdx.y: dw_pre, dw_post, then the gate rows; a workgroup adds SUM_COLS columns,
// four a thread, by SHARES shares of the rows.
constexpr int SUM_COLS = 32, SHARES = 256 / (SUM_COLS / 4);
__global__ __launch_bounds__(256) void norm_sums_kernel(NormArgs a, int first) {
  const int which = blockIdx.y + first;
  float* out = which == 0 ? a.dw_pre : which == 1 ? a.dw_post : a.dgate + (size_t)(which - 2) * a.d;
  if (!out) return;  // uniform
  const int n = which < 2 ? a.n_part : a.parts;
  const float* part = a.part + ((size_t)min(which, 2) * a.n_part + (which < 2 ? 0 : (size_t)(which - 2) * a.parts)) * a.d;
  const int quad = threadIdx.x % (SUM_COLS / 4), share = threadIdx.x / (SUM_COLS / 4);
  const int col = blockIdx.x * SUM_COLS + 4 * quad;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p = share; p < n; p += SHARES * 8) {  // eight loads at a time
    Chunk c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      c[k] = p + SHARES * k < n ? ld_chunk(part + (size_t)(p + SHARES * k) * a.d + col) : zero_chunk();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float v[4];
      chunk_to_f<float>(c[k], v);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
  }
  __shared__ float sums[SHARES][SUM_COLS];
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[share][4 * quad + e] = s[e];
  __syncthreads();
  if (threadIdx.x < SUM_COLS) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < SHARES; ++k) v[k % 4] += sums[k][threadIdx.x];
    out[blockIdx.x * SUM_COLS + threadIdx.x] = (v[0] + v[1]) + (v[2] + v[3]);
  }
}

constexpr int kMaxParts = 512;

NormArgs norm_args(const moe_desc& d, const moe_norm& n, const void* y, const void* w_post, const void* gate,
                   const void* w_pre) {
  NormArgs a{};
  a.T = d.T;
  a.d = d.d_model;
  a.cpr = d.d_model * (int)elem_bytes(d) / 16;
  a.pre = n.pre;
  a.post = n.post;
  a.groups = gate ? n.gate_groups : 1;
  a.gate_rows = d.T / a.groups;
  a.alpha = n.residual_scale;
  a.eps = (double)n.eps;
  a.inv_d = 1.0 / d.d_model;
  a.y = y;
  a.w_post = w_post;
  a.gate = gate;
  a.w_pre = w_pre;
  return a;
}

// 16-byte chunks per thread (a power of two) and threads of a workgroup of at most `most`, for rows of cpr chunks. `most` is
// raised to 1024 for rows that would need more than four; the longest fp32 rows (of up to 5,760 chunks; bf16 rows end at 4,080)
// then take eight.
struct Shape {
  int p, nt, most;
};
Shape row_shape(int cpr, int most) {
  if (cpr > 4 * most) most = 1024;
  int p = 1;
  while ((cpr + p - 1) / p > most) p *= 2;
  return {p, ((cpr + p - 1) / p + 63) / 64 * 64, most};
}
template <int MOST, typename F>
void row_kernels(int dtype, const Shape& sh, F&& f) {
  const auto one = [&](auto t) {
    const auto with = [&](auto p) {
      if (sh.most == MOST) f(t, p, std::integral_constant<int, MOST>{});
      else f(t, std::integral_constant<int, (decltype(p)::value < 4 ? 4 : decltype(p)::value)>{}, std::integral_constant<int, 1024>{});
    };
    if (sh.p == 1) with(std::integral_constant<int, 1>{});
    else if (sh.p == 2) with(std::integral_constant<int, 2>{});
    else if (sh.p == 4) with(std::integral_constant<int, 4>{});
    else if constexpr (std::is_same<decltype(t), float>::value) f(t, std::integral_constant<int, 8>{}, std::integral_constant<int, 1024>{});
  };
  if (dtype == MOE_BF16) one(bf16{});
  else one(float{});
}

}  // namespace

size_t norm_bwd_ws_bytes(const moe_desc& d) {
  return (size_t)3 * std::min(d.T, kMaxParts) * d.d_model * sizeof(float);
}

hipError_t launch_residual_norm(const moe_desc& d, const moe_norm& n, const void* x, const void* y, const void* w_post,
                                const void* gate, const void* w_pre, void* r, void* h, hipStream_t s) {
  NormArgs a = norm_args(d, n, y, w_post, gate, w_pre);
  a.x = x;
  a.r = r;
  a.h = h;
  if (!y && n.pre == MOE_NORM_NONE) return hipSuccess;  // r is x
  const Shape sh = row_shape(a.cpr, d.T >= 1024 ? 256 : 1024);
  KernelTimer kt("residual_norm", s);
  const auto go = [&](auto t, auto p, auto most) {
    hipLaunchKernelGGL((residual_norm_kernel<decltype(t), decltype(p)::value, decltype(most)::value>), dim3(a.T),
                       dim3(sh.nt), 0, s, a);
  };
  if (d.T >= 1024) row_kernels<256>(d.dtype, sh, go);
  else row_kernels<1024>(d.dtype, sh, go);
  return hipGetLastError();
}

hipError_t launch_residual_norm_bwd(const moe_desc& d, const moe_norm& n, const void* dr, const void* dh, const void* y,
                                    const void* r, const void* w_post, const void* gate, const void* w_pre, void* dx,
                                    void* dy, float* dw_post, float* dgate, float* dw_pre, void* ws, hipStream_t s) {
  NormArgs a = norm_args(d, n, y, w_post, gate, w_pre);
  a.dr = dr;
  a.dh = dh;
  a.r = const_cast<void*>(r);
  a.dx = dx;
  a.dy = dy;
  a.dw_post = w_post ? dw_post : nullptr;
  a.dgate = gate ? dgate : nullptr;
  a.dw_pre = w_pre ? dw_pre : nullptr;
  a.part = (float*)ws;
  // Workgroups: a row each while there are few, which leaves most of them to run at once (777 x 1024 fp32, a row / two / four /
  // eight: 14.0 / 15.0 / 17.3 / 26 us). One or two rows: a single workgroup, which needs no second launch.
  const int want = a.T <= 2 ? 1 : std::min(kMaxParts, a.T);
  a.parts = a.groups <= want ? std::min(want / a.groups, a.gate_rows) : 0;
  a.n_part = a.parts ? a.groups * a.parts : want;
  a.direct = a.n_part == 1;
  const Shape sh = row_shape(a.cpr, 512);
  {
    KernelTimer kt("residual_norm_bwd", s);
    row_kernels<512>(d.dtype, sh, [&](auto t, auto p, auto most) {
      using T = decltype(t);
      constexpr int C = decltype(p)::value, NT = decltype(most)::value;
      const auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(a.n_part), dim3(sh.nt), 0, s, a); };
      const bool pre = n.pre != MOE_NORM_NONE, post = y && n.post != MOE_NORM_NONE;
      if (pre && post) go(residual_norm_bwd_kernel<T, C, NT, true, true>);
      else if (pre) go(residual_norm_bwd_kernel<T, C, NT, true, false>);
      else if (post) go(residual_norm_bwd_kernel<T, C, NT, false, true>);
      else go(residual_norm_bwd_kernel<T, C, NT, false, false>);
    });
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const bool weights = !a.direct && (a.dw_pre || a.dw_post), gates = gate && a.parts > 1;
  if (weights || gates) {
    const int first = weights ? 0 : 2, rows = (weights ? 2 : 0) + (gates ? a.groups : 0);
    KernelTimer kt("residual_norm_sums", s);
    hipLaunchKernelGGL(norm_sums_kernel, dim3(a.d / SUM_COLS, rows), dim3(256), 0, s, a, first);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pcmoe
