// What stands between two layers of a stack: r = alpha x + gamma * post(y), h = pre(r), and the adjoint of both.
//
// RMS: N(v) = v / sqrt(mean(v^2) + eps) * w; LAYER: the same of v - mean(v). With vhat = N(v) / w and a = dN w,
// dv = (a - vhat mean(a vhat) [- mean(a)]) / sqrt(...). Both passes are bound by memory: every row is read once and written once
// (what the adjoint uses again of its longest rows comes from the L2). Row sums are fp64, those of products with gradients fp64
// sums of a chunk's in fp32, so that none of finite rows overflows (with gradients up to 1e37), and means are kept in two fp32
// parts, so that one far from zero costs no digits; everything else is fp32, rounded once on the way out.
// 16384 x 2048 bf16 with a post norm and a gate: 268 MB in 44 us alone and 51 among other passes. Adjoint of 8192 x 4096: 403 MB
// in 68 + 5; of 777 x 1024 fp32 with layer norms 11 + 4, two launches and a row's three sums one after the other.
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

// A mean as two fp32 parts. v - hi is exact where v is within a factor of two of it, so that v - mean is off by its own rounding
// only, however far the mean is above the deviation (rounded to fp32 alone, a mean of 1e4 deviations would move every v of the
// row by up to 2^-11 of one).
struct Mean {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ Mean() {}
  __device__ __forceinline__ explicit Mean(double m) : hi((float)m), lo((float)(m - (double)(float)m)) {}
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

template <typename T>
__device__ __forceinline__ Chunk ones() {
  Chunk c;
#pragma unroll
  for (int i = 0; i < 4; ++i) c.w[i] = std::is_same<T, float>::value ? 0x3f800000u : 0x3f803f80u;
  return c;
}
// What goes into v is computed here. Sums that are used much later would be formed there, and their operands kept until then.
template <typename V>
__device__ __forceinline__ void settle(V& v) {
  asm volatile("" : "+v"(v));
}
// What was unpacked from a chunk is unpacked again after this, not kept.
__device__ __forceinline__ void forget(Chunk& c) {
  asm volatile("" : "+v"(c.w[0]), "+v"(c.w[1]), "+v"(c.w[2]), "+v"(c.w[3]));
}
// Loads of the next chunk stay behind this.
__device__ __forceinline__ void next_chunk() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Adjoint. A workgroup walks over the rows of a part of a gate row's tokens (or over whole gate rows) and keeps two sums over
// tokens of its columns in registers; norm_sums_kernel adds the workgroups' up in a fixed order. With g the gradient of r they are
// dh rhat and, of a gate row's tokens, c = g yhat: the gate's gradient is w_post c, that of w_post the sum of gate c over gate rows.
//
// What else a row needs is kept in registers as far as they go; nothing is spilled to memory but a few words where stated:
//   up to 1024 chunks (8,192 bf16, 4,096 fp32)   the row, the next row's loads, weights and gate; a third sum (w_post's) if MANY
//   up to 2048, 512 threads of up to four chunks  the row; weights and gate come from the L2 for every row
//   above, 1024 threads of up to six              the sums alone; each of a row's rounds loads its chunks again, from the L2
// us, before (all of it in registers for every length, up to 3.7 KB a lane spilled) and now, of 6 T d elements through memory at
// the copy's rate: bf16 with post norm and gate 4096 x 12288 1,265 -> 193 (117), 4096 x 16384 1,461 -> 272 (156), 2048 x 28672
// 1,923 -> 334 (136), without 490 -> 124, 573 -> 170, 1,066 -> 172; fp32 with 4096 x 8192 329 -> 216 (156), 2048 x 20480 1,775 ->
// 385 (194). The rounds' dependent loads and sums bound them; the two norms' rounds are one after the other.
// One-chunk bf16 rows with two workgroups a CU (128 registers, 12 bytes spilled): 8192 x 2560 with layer norms 109 -> 82. The
// longest bf16 rows spill 44 bytes.
template <typename T, int CPT, int NT, bool PRE, bool POST, bool MANY>
__global__ __launch_bounds__(NT, (CPT == 1 && sizeof(T) == 2 && !MANY ? 4 : 1))
void residual_norm_bwd_kernel(NormArgs a) {
  constexpr int EP = EPC<T>::value, N = CPT * EP, BYTES = CPT * 16;
  constexpr bool BF16 = std::is_same<T, bf16>::value;
  constexpr bool KEEP = NT <= 512;                  // a row's chunks stay in registers; else they are loaded again (from the L2)
  constexpr bool AHEAD = KEEP && BYTES <= 32;       // the next row's are on their way while a row is worked on
  constexpr bool KEEP_W = BYTES <= 32;              // weights and gate stay too
  constexpr bool KEEP_B = POST && KEEP && BYTES <= 48;  // the gradient of post(y) stays until its row sums are there
  constexpr bool LONG = !KEEP || N > 16;            // chunk after chunk, nothing moved from one to another
  constexpr bool FORGET = BF16 && N > 16, FORGET_W = FORGET || (BF16 && MANY && N > 8);  // values are unpacked where they are used
  __shared__ SumLds lds;
  int turn = 0;
  const bool need_y = a.y && (POST || a.gate);
  const bool lr = PRE && a.pre == MOE_NORM_LAYER, ly = POST && a.post == MOE_NORM_LAYER;
  // Sums over tokens: dh rhat, and g yhat of the present gate row, from which the gate's gradient (by w_post) and w_post's (by the
  // gate, summed over gate rows) are made
  float s_pre[CPT][EP], s_y[CPT][EP], s_post[MANY ? CPT : 1][EP];
  Chunk wk[3][KEEP_W ? CPT : 1];
  // chunk c of row t of p
  const auto ld = [&](const void* p, int t, int c, bool there) {
    return buf_ld16(buf_rsrc(p ? (const char*)p + (size_t)t * (uint32_t)(a.cpr * 16) : nullptr, p && there ? a.cpr * 16 : 0), c * 16);
  };
  const auto st = [&](void* p, int t, int c, const Chunk& v) {
    typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{v.w[0], v.w[1], v.w[2], v.w[3]},
                                           buf_rsrc((char*)p + (size_t)t * (uint32_t)(a.cpr * 16), a.cpr * 16), c * 16, 0, 0);
  };
  // chunk c of w_pre (0), w_post (1) or row g of the gate (2); ones where there is none
  const auto ld_w = [&](int k, int g, int c) {
    const void* p = k == 0 ? (PRE ? a.w_pre : nullptr) : k == 1 ? (POST ? a.w_post : nullptr) : a.gate;
    return p ? ld(p, k == 2 ? g : 0, c, true) : ones<T>();
  };
  const auto put_sums = [&](float* out, int c, const float* v) {  // a chunk's columns
#pragma unroll
    for (int e = 0; e < EP; e += 4) st_chunk((float*)((char*)out + (uint32_t)(c * EP * 4)) + e, f_to_chunk<float>(v + e));
  };
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    if constexpr (KEEP_W)
#pragma unroll
      for (int k = 0; k < 2; ++k) wk[k][i] = ld_w(k, 0, threadIdx.x + i * blockDim.x);
#pragma unroll
    for (int e = 0; e < EP; ++e) s_pre[i][e] = 0.f;
    if (MANY)
#pragma unroll
      for (int e = 0; e < EP; ++e) s_post[i][e] = 0.f;
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
  float* const o_pre = a.direct ? a.dw_pre : a.part + (size_t)blockIdx.x * a.d;
  float* const o_post = a.direct ? a.dw_post : a.part + ((size_t)a.n_part + blockIdx.x) * a.d;
  for (int g = g0; g < g1; ++g) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      if constexpr (KEEP_W) wk[2][i] = ld_w(2, g, threadIdx.x + i * blockDim.x);
#pragma unroll
      for (int e = 0; e < EP; ++e) s_y[i][e] = 0.f;
    }
    const int t1 = g * a.gate_rows + last;
    Chunk kept[4][KEEP ? CPT : 1], next[4][AHEAD ? CPT : 1];
    // chunk i of row t of dr (0), dh (1), r (2) or y (3)
    const auto load = [&](int k, int t, int i, bool there) {
      const void* p = k == 0 ? a.dr : k == 1 ? (PRE ? a.dh : nullptr) : k == 2 ? (PRE ? a.r : nullptr) : need_y ? a.y : nullptr;
      return ld(p, t, threadIdx.x + i * blockDim.x, there);
    };
    const auto fetch = [&](auto& to, int t, bool there) {
#pragma unroll
      for (int i = 0; i < (KEEP ? CPT : 0); ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) to[k][i] = load(k, t, i, there);
    };
    if constexpr (AHEAD) fetch(next, g * a.gate_rows + first, first < last);
    for (int t = g * a.gate_rows + first; t < t1; ++t) {
      if constexpr (AHEAD) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < CPT; ++i) kept[k][i] = next[k][i];
        fetch(next, t + 1, t + 1 < t1);
      } else if constexpr (KEEP) {
        fetch(kept, t, true);
      }
      const auto part = [&](int k, int i, float (&v)[EP]) {
        if constexpr (KEEP && FORGET) forget(kept[k][i]);
        if constexpr (KEEP) chunk_to_f<T>(kept[k][i], v);
        else chunk_to_f<T>(load(k, t, i, true), v);
      };
      const auto weight = [&](int k, int i, float (&v)[EP]) {
        if constexpr (KEEP_W) {
          if constexpr (FORGET_W) forget(wk[k][i]);
          chunk_to_f<T>(wk[k][i], v);
        } else {
          chunk_to_f<T>(ld_w(k, g, threadIdx.x + i * blockDim.x), v);
        }
      };
      // row sums: of r and y (LAYER), then of their squares with those of a = dh w_pre
      Mean mr, my;
      float ma = 0.f, rr = 1.f, ry = 1.f, car = 0.f;
      if (lr || ly) {
        Sums s{};
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          if constexpr (LONG) next_chunk();
          float r[EP], y[EP], dh[EP], w[EP];
          part(2, i, r);
          part(3, i, y);
          part(1, i, dh);
          weight(0, i, w);
          float fa = 0.f;
#pragma unroll
          for (int e = 0; e < EP; ++e) {
            if (lr) s.v[0] += (double)r[e];
            if (ly) s.v[1] += (double)y[e];
            if (lr) fa += dh[e] * w[e];
          }
          s.v[2] += (double)fa;
          if constexpr (LONG) { settle(s.v[0]); settle(s.v[1]); settle(s.v[2]); }
        }
        s = block_sum<3>(s, lds, turn);
        if (lr) mr = Mean(s.v[0] * a.inv_d);
        if (ly) my = Mean(s.v[1] * a.inv_d);
        if (lr) ma = (float)(s.v[2] * a.inv_d);
      }
      if (PRE || POST) {
        Sums s{};
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          PIECE(i);
          if constexpr (LONG) next_chunk();
          float r[EP], y[EP], dh[EP], w[EP];
          part(2, i, r);
          part(3, i, y);
          part(1, i, dh);
          weight(0, i, w);
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
            for (int e = 0; e < EP; ++e) f += dh[e] * w[e] * (r[e] * by.down());
            s.v[2] += (double)f * by.up();
          }
          if (POST)
#pragma unroll
            for (int e = 0; e < EP; ++e) s.v[1] += (double)my.from(y[e]) * (double)my.from(y[e]);
          if constexpr (LONG) { settle(s.v[0]); settle(s.v[1]); settle(s.v[2]); }
        }
        s = block_sum<PRE ? 3 : 2>(s, lds, turn);
        if (PRE) rr = rsqrt_of(s.v[0] * a.inv_d + a.eps);
        if (POST) ry = rsqrt_of(s.v[1] * a.inv_d + a.eps);
        if (PRE) car = (float)(s.v[2] * a.inv_d * (double)rr);  // mean(a rhat)
      }
      // The gradient g of r; that of post(y) is g by the gate, and by w_post, b.
      const auto grad = [&](int i, float (&gr)[EP], float (&rhat)[EP]) {
        float dh[EP], r[EP], w[EP];
        part(0, i, gr);
        if (!PRE) return;
        part(1, i, dh);
        part(2, i, r);
        weight(0, i, w);
#pragma unroll
        for (int e = 0; e < EP; ++e) {
          rhat[e] = mr.from(r[e]) * rr;
          gr[e] += ((dh[e] * w[e] - ma) - rhat[e] * car) * rr;
          rhat[e] *= dh[e];
        }
      };
      const auto factor = [&](int i, float (&f)[EP]) {  // gate w_post
        float gt[EP], wp[EP];
        weight(2, i, gt);
        weight(1, i, wp);
#pragma unroll
        for (int e = 0; e < EP; ++e) f[e] = gt[e] * wp[e];
      };
      const auto put_dx = [&](int i, const float (&gr)[EP]) {
        float o[EP];
#pragma unroll
        for (int e = 0; e < EP; ++e) o[e] = a.alpha * gr[e];
        st(a.dx, t, threadIdx.x + i * blockDim.x, f_to_chunk<T>(o));
      };
      const auto put_dy = [&](int i, const float (&b)[EP]) { st(a.dy, t, threadIdx.x + i * blockDim.x, f_to_chunk<T>(b)); };
      float b[KEEP_B ? CPT : 1][EP];
      Sums s{};
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        PIECE(i);
        if constexpr (LONG) next_chunk();
        float gr[EP], rhat[EP], y[EP], f[EP];
        grad(i, gr, rhat);
        if (PRE)
#pragma unroll
          for (int e = 0; e < EP; ++e) s_pre[i][e] += rhat[e];
        part(3, i, y);
        factor(i, f);
        float (&bi)[EP] = b[KEEP_B ? i : 0];
        float fb = 0.f, fm = 0.f;
#pragma unroll
        for (int e = 0; e < EP; ++e) {
          const float gy = gr[e] * (my.from(y[e]) * ry);
          s_y[i][e] += gy;
          bi[e] = gr[e] * f[e];
          if (POST) {
            fb += gy * f[e];
            if (ly) fm += bi[e];
          }
        }
        if (POST && in) {
          s.v[0] += (double)fb;
          if (ly) s.v[1] += (double)fm;
        }
        if constexpr (LONG) {
          settle(s.v[0]);
          settle(s.v[1]);
#pragma unroll
          for (int e = 0; e < EP; ++e) {
            if (PRE) settle(s_pre[i][e]);
            settle(s_y[i][e]);
          }
        }
        // dx may take the place of dr or dh: with POST and without KEEP they are read once more before it is written
        if (KEEP || !POST) put_dx(i, gr);
        if (!POST && a.dy) put_dy(i, bi);
      }
      if (!POST) continue;
      s = ly ? block_sum<2>(s, lds, turn) : block_sum<1>(s, lds, turn);
      const float cy = (float)(s.v[0] * a.inv_d), mb = (float)(s.v[1] * a.inv_d);
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        if constexpr (LONG) next_chunk();
        float gr[EP], rhat[EP], y[EP], f[EP];
        float (&bi)[EP] = b[KEEP_B ? i : 0];
        part(3, i, y);
        if constexpr (!KEEP_B) {
          grad(i, gr, rhat);
          factor(i, f);
#pragma unroll
          for (int e = 0; e < EP; ++e) bi[e] = gr[e] * f[e];
        }
#pragma unroll
        for (int e = 0; e < EP; ++e) bi[e] = ((bi[e] - mb) - my.from(y[e]) * ry * cy) * ry;
        if (!KEEP) put_dx(i, gr);
        put_dy(i, bi);
      }
    }
    if (!POST && !a.gate) continue;
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      PIECE(i);
      if (!in) continue;
      float gt[EP], wp[EP], v[EP];
      chunk_to_f<T>(KEEP_W ? wk[2][KEEP_W ? i : 0] : ld_w(2, g, c), gt);
      chunk_to_f<T>(KEEP_W ? wk[1][KEEP_W ? i : 0] : ld_w(1, g, c), wp);
      if (a.gate) {
        float* out = a.parts > 1 ? a.part + ((size_t)2 * a.n_part + blockIdx.x) * a.d : a.dgate + (size_t)g * a.d;
#pragma unroll
        for (int e = 0; e < EP; ++e) v[e] = s_y[i][e] * wp[e];
        put_sums(out, c, v);
      }
      if (!POST || !a.dw_post) continue;
#pragma unroll
      for (int e = 0; e < EP; ++e) v[e] = s_y[i][e] * gt[e];
      if constexpr (MANY) {
#pragma unroll
        for (int e = 0; e < EP; ++e) s_post[i][e] += v[e];
        if (g + 1 < g1) continue;
#pragma unroll
        for (int e = 0; e < EP; ++e) v[e] = s_post[i][e];
      }
      if (!MANY && g > g0) {  // to the sum so far, which this thread wrote
#pragma unroll
        for (int e = 0; e < EP; e += 4) {
          float was[4];
          chunk_to_f<float>(ld_chunk(o_post + c * EP + e), was);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[e + k] += was[k];
        }
      }
      put_sums(o_post, c, v);
    }
  }
  if (!PRE || !a.dw_pre) return;
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    PIECE(i);
    if (in) put_sums(o_pre, c, s_pre[i]);
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
  {
    KernelTimer kt("residual_norm_bwd", s);
    const bool pre = n.pre != MOE_NORM_NONE, post = y && n.post != MOE_NORM_NONE;
    const auto with = [&](auto t, auto p, auto most, auto many) {
      using T = decltype(t);
      constexpr int C = decltype(p)::value, NT = decltype(most)::value;
      constexpr bool M = decltype(many)::value;
      const int nt = ((a.cpr + C - 1) / C + 63) / 64 * 64;
      const auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(a.n_part), dim3(nt), 0, s, a); };
      if (pre && post) go(residual_norm_bwd_kernel<T, C, NT, true, true, M>);
      else if (pre) go(residual_norm_bwd_kernel<T, C, NT, true, false, false>);
      else if (post) go(residual_norm_bwd_kernel<T, C, NT, false, true, M>);
      else go(residual_norm_bwd_kernel<T, C, NT, false, false, false>);
    };
    constexpr std::integral_constant<int, 512> half;
    constexpr std::integral_constant<int, 1024> whole;
    const auto shapes = [&](auto t) {
      using T = decltype(t);
      const auto few = [&](auto p) {
        if (a.parts) with(t, p, half, std::false_type{});
        else with(t, p, half, std::true_type{});
      };
      // whole gate rows of a workgroup: what w_post's gradient has so far is added to in memory, a gate row at a time
      const auto more = [&](auto p, auto most) { with(t, p, most, std::false_type{}); };
      if (a.cpr <= 512) few(std::integral_constant<int, 1>{});
      else if (a.cpr <= 2 * 512) few(std::integral_constant<int, 2>{});
      else if (a.cpr <= 3 * 512) more(std::integral_constant<int, 3>{}, half);
      else if (a.cpr <= 4 * 512) more(std::integral_constant<int, 4>{}, half);
      else if (a.cpr <= 3 * 1024) more(std::integral_constant<int, 3>{}, whole);
      else if (a.cpr <= 4 * 1024) more(std::integral_constant<int, 4>{}, whole);
      else if constexpr (std::is_same<T, float>::value) more(std::integral_constant<int, 6>{}, whole);  // at most 5,760
    };
    if (d.dtype == MOE_BF16) shapes(bf16{});
    else shapes(float{});
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
