// Gating (Alg. 7: scores, softmax, TopKIndices, w = p[I]) and its adjoint on the data owner.
//
// Scores are accumulated in fp64 (MFMA or FMA) from the products of the stored inputs (exact in fp64) and rounded once to
// fp32. The order of a score's sum follows the tiling, which goes by the batch size and the device's CU count: equal
// calls give equal bits, and where fp64 holds the sum exactly (bf16 inputs, as long as no product is smaller than about
// 2^-37 of the sum) so do other batches; else a score can differ in its last fp32 bit, in about one of 10^8, and a
// selection that hangs on that bit with it. Selection happens at wavefront level: k rounds of a 64-lane maximum over
// order-preserving keys, ties to the lowest expert index.
#include "expert_ops.h"
#include <math.h>
#include <algorithm>

namespace pcmoe {

typedef double doublex4 __attribute__((ext_vector_type(4)));

// Wavefront maximum of unsigned keys on the vector ALU (DPP: row shifts, then row broadcasts), in every lane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#define PCMOE_DPP_MAX(ctrl, rows) \
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false))
  PCMOE_DPP_MAX(0x111, 0xf);  // row_shr 1, 2, 4, 8: lane 15 of each row of 16 holds the row's maximum
  PCMOE_DPP_MAX(0x112, 0xf);
  PCMOE_DPP_MAX(0x114, 0xf);
  PCMOE_DPP_MAX(0x118, 0xf);
  PCMOE_DPP_MAX(0x142, 0xa);  // row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
  PCMOE_DPP_MAX(0x143, 0xc);
#undef PCMOE_DPP_MAX
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Order-preserving key of a score: larger score, larger key; -0 and +0 share one; 0 (below every number's) for a
// NaN, which is never selected.
__device__ __forceinline__ uint32_t score_key(float f) {
  const uint32_t u = __float_as_uint(f);
  if (f != f) return 0u;
  if (f == 0.f) return 0x80000000u;
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) {
  return k == 0u ? -INFINITY : __uint_as_float((k >> 31) ? (k & 0x7fffffffu) : ~k);
}

// ------------------------------------------------------------------------- gated selection
// Selection by scores with a balance bias within limited expert groups. An expert's score s is softmax(l) or sigmoid(l) of
// its fp32 score l above, its choice value s + bias; both are formed in fp64, so that which of two close experts is chosen
// does not hang on the last bits of an exponential. (Without a bias the experts rank by l itself, the same order.)
constexpr int NO_EXPERT = 0x7fffffff;  // index of a slot that no expert fills

struct GateArgs {
  const float* bias;  // [E] or null
  float scale;
  int sigmoid, groups, keep, top, group_size;
  int group_mul;      // e / group_size = e * group_mul >> 16 for e < 256
  int lane_shift;     // 2^lane_shift = lanes of a wavefront per group, the largest power of two up to 64 / groups
};

// Order-preserving key of a choice value: 0 for what is never chosen (NaN, -inf), -0 and +0 alike.
__device__ __forceinline__ uint64_t choice_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  if (!(v > -INFINITY)) return 0ull;
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
// The value of another lane, by the vector ALU's lane shifts (a shuffle through LDS costs ten times as long).
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp_f64(double v, double otherwise = 0.0) {
  const uint64_t u = (uint64_t)__double_as_longlong(v), w = (uint64_t)__double_as_longlong(otherwise);
  const uint32_t lo = __builtin_amdgcn_update_dpp((int)w, (int)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp((int)(w >> 32), (int)(u >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double readlane_f64(double v, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return __longlong_as_double((long long)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32) |
                                          (uint32_t)__builtin_amdgcn_readlane((int)u, lane)));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  v += dpp_f64<0x111>(v);  // row_shr 1, 2, 4, 8: lane 15 of each row of 16 holds the row's sum
  v += dpp_f64<0x112>(v);
  v += dpp_f64<0x114>(v);
  v += dpp_f64<0x118>(v);
  v += dpp_f64<0x142, 0xa>(v);  // row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
  v += dpp_f64<0x143, 0xc>(v);
  return readlane_f64(v, 63);
}
__device__ __forceinline__ double sum8_f64(double v) {  // of lanes 0 .. 7
  v += dpp_f64<0x111>(v);
  v += dpp_f64<0x112>(v);
  v += dpp_f64<0x114>(v);
  return readlane_f64(v, 7);
}
// The largest of fp32 numbers (NaN passed over; -inf where there is none), in every lane.
__device__ __forceinline__ float wave_max_dpp(float v) {
#define PCMOE_DPP_FMAX(ctrl, rows) \
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp((int)0xff800000, (int)__float_as_uint(v), ctrl, rows, 0xf, false)))
  PCMOE_DPP_FMAX(0x111, 0xf);
  PCMOE_DPP_FMAX(0x112, 0xf);
  PCMOE_DPP_FMAX(0x114, 0xf);
  PCMOE_DPP_FMAX(0x118, 0xf);
  PCMOE_DPP_FMAX(0x142, 0xa);
  PCMOE_DPP_FMAX(0x143, 0xc);
#undef PCMOE_DPP_FMAX
  return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// NT tokens at once, whose chains of dependent instructions fill each other's waits: v[n][qq] is token n's score of expert
// lane + 64 qq (-inf past E). row[n] is LDS that only this wavefront uses, E doubles of it. Token n's results go to idx + n
// * step and gw + n * step, as long as n < valid.
template <int QE, int NT>
__device__ __forceinline__ void gated_select(const float (&v)[NT][QE], int E, int k, int renorm, const GateArgs& ga,
                                             double* const (&row)[NT], int valid, size_t step,
                                             int32_t* __restrict__ idx, float* __restrict__ gw) {
  const int lane = threadIdx.x & 63;
  const bool need = ga.bias || (ga.groups > 1 && ga.top == 2);  // are scores of all the experts needed?
  double z[NT];                                                  // softmax: the largest logit and the sum over E
  float m[NT];
  double sc[NT][QE];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    z[n] = 1.0;
    m[n] = 0.f;
    if (!ga.sigmoid && (need || !renorm)) {
      float mm = v[n][0];
#pragma unroll
      for (int qq = 1; qq < QE; ++qq) mm = fmaxf(mm, v[n][qq]);
      m[n] = wave_max_dpp(mm);
      double zz = 0.0;
#pragma unroll
      for (int qq = 0; qq < QE; ++qq) {
        // nothing of a masked or NaN expert; the maximum may be +inf
        sc[n][qq] = v[n][qq] > -INFINITY ? (v[n][qq] == m[n] ? 1.0 : exp((double)v[n][qq] - (double)m[n])) : 0.0;
        zz += sc[n][qq];
      }
      z[n] = wave_sum_f64(zz);
    }
  }
  uint64_t key[NT][QE];
  double worth[NT][QE];  // what a group's value is made of
#pragma unroll
  for (int qq = 0; qq < QE; ++qq) {
    const int e = lane + 64 * qq;
    const double bias = ga.bias && e < E ? (double)ga.bias[e] : 0.0;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      double c = (double)v[n][qq];
      worth[n][qq] = c;
      if (need) {
        worth[n][qq] = ga.sigmoid ? 1.0 / (1.0 + exp(-c)) : sc[n][qq] / z[n];
        if (ga.bias) {
          worth[n][qq] += bias;
          c = worth[n][qq];
        }
      }
      key[n][qq] = e < E && v[n][qq] > -INFINITY ? choice_key(c) : 0ull;
    }
  }
  if (ga.groups > 1) {
    // 2^lane_shift lanes find the largest and the second largest value of a group
    const int g = lane >> ga.lane_shift, lanes = 1 << ga.lane_shift;
    double a[NT], b[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int qq = 0; qq < QE; ++qq)
        if (lane + 64 * qq < E) row[n][lane + 64 * qq] = key[n][qq] ? worth[n][qq] : -INFINITY;
      a[n] = b[n] = -INFINITY;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (g < ga.groups)
      for (int o = lane & (lanes - 1); o < ga.group_size; o += lanes) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const double w = row[n][g * ga.group_size + o];
          b[n] = fmax(b[n], fmin(a[n], w));
          a[n] = fmax(a[n], w);
        }
      }
    auto merge = [&](int n, double a2, double b2) {
      b[n] = fmax(fmax(b[n], b2), fmin(a[n], a2));
      a[n] = fmax(a[n], a2);
    };
    // lane pairs, quads (quad_perm), halves of 8 and 16 lanes (mirrors: the lanes merged so far are equal)
    if (ga.lane_shift >= 1)
#pragma unroll
      for (int n = 0; n < NT; ++n) merge(n, dpp_f64<0xb1>(a[n]), dpp_f64<0xb1>(b[n]));
    if (ga.lane_shift >= 2)
#pragma unroll
      for (int n = 0; n < NT; ++n) merge(n, dpp_f64<0x4e>(a[n]), dpp_f64<0x4e>(b[n]));
    if (ga.lane_shift >= 3)
#pragma unroll
      for (int n = 0; n < NT; ++n) merge(n, dpp_f64<0x141>(a[n]), dpp_f64<0x141>(b[n]));
    if (ga.lane_shift >= 4)
#pragma unroll
      for (int n = 0; n < NT; ++n) merge(n, dpp_f64<0x140>(a[n]), dpp_f64<0x140>(b[n]));
    if (ga.lane_shift >= 5)
#pragma unroll
      for (int n = 0; n < NT; ++n) merge(n, __shfl_xor(a[n], 16, 64), __shfl_xor(b[n], 16, 64));
    uint64_t mine[NT];
    int ahead[NT];  // groups that come before the lane's: of equals, the lower index first
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (ga.top == 2 && b[n] > -INFINITY) a[n] += b[n];
      mine[n] = choice_key(a[n]);
      ahead[n] = 0;
    }
    for (int h = 0; h < ga.groups; ++h) {
      const int l = h << ga.lane_shift;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint64_t o = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine[n] >> 32), l) << 32) |
                           (uint32_t)__builtin_amdgcn_readlane((int)mine[n], l);
        ahead[n] += o > mine[n] || (o == mine[n] && h < g);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint64_t open = __ballot(g < ga.groups && ahead[n] < ga.keep);
#pragma unroll
      for (int qq = 0; qq < QE; ++qq)
        if (!((open >> (((((lane + 64 * qq) * ga.group_mul) >> 16) << ga.lane_shift) & 63)) & 1)) key[n][qq] = 0ull;
    }
  }
  int myi[NT];
  float myl[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    myi[n] = NO_EXPERT;
    myl[n] = -INFINITY;
  }
  for (int j = 0; j < k; ++j) {
    // the largest upper word; the lower words are compared only where several lanes hold it
    uint32_t hi[NT], low[NT];
    bool one[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      hi[n] = (uint32_t)(key[n][0] >> 32);
#pragma unroll
      for (int qq = 1; qq < QE; ++qq) hi[n] = max(hi[n], (uint32_t)(key[n][qq] >> 32));
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) hi[n] = wave_max_u32(hi[n]);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      int holders = 0;
      low[n] = 0u;
#pragma unroll
      for (int qq = 0; qq < QE; ++qq) {
        const bool is = (uint32_t)(key[n][qq] >> 32) == hi[n];
        holders += __popcll(__ballot(is));
        low[n] = is ? max(low[n], (uint32_t)key[n][qq]) : low[n];
      }
      one[n] = holders == 1;
      if (!one[n]) low[n] = wave_max_u32(low[n]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      int best = NO_EXPERT;
      float l = -INFINITY;
#pragma unroll
      for (int qq = QE - 1; qq >= 0; --qq) {
        const uint64_t bl = __ballot((uint32_t)(key[n][qq] >> 32) == hi[n] && (one[n] || (uint32_t)key[n][qq] == low[n]));
        const int ln = __builtin_ctzll(bl | 0x8000000000000000ull);
        const float lv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[n][qq]), ln));
        best = bl ? 64 * qq + ln : best;
        l = bl ? lv : l;
      }
      // nothing is left to choose from (a key above 0 has bits in its upper word)
      if (hi[n] == 0u) {
        best = NO_EXPERT;
        l = -INFINITY;
      }
#pragma unroll
      for (int qq = 0; qq < QE; ++qq)
        if (lane + 64 * qq == best) key[n][qq] = 0ull;
      if (lane == j) {
        myi[n] = best;
        myl[n] = l;
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const bool filled = lane < k && myi[n] != NO_EXPERT;
    if (!ga.sigmoid && renorm) m[n] = wave_max_dpp(myl[n]);  // the largest of the chosen: the others' exponentials stay finite
    double s = ga.sigmoid ? 1.0 / (1.0 + exp(-(double)myl[n]))
                          : (myl[n] == m[n] ? 1.0 : exp((double)myl[n] - (double)m[n])) / z[n];
    if (!filled) s = 0.0;
    if (renorm) {
      const double t = sum8_f64(s);
      s = t == 0.0 ? 0.0 : s / t;  // every chosen score underflows (or nothing is chosen): no weight
    }
    if (lane < k && n < valid) {
      idx[n * step + lane] = myi[n];
      gw[n * step + lane] = (float)(s * (double)ga.scale);
    }
  }
}

// Scores of NTOK = TB * TT tokens against all E experts on the fp64 matrix cores, then top-k and gate weights.
// The WE x WK wavefronts split the experts into WE runs of 16 * NET and d into WK ranges of column steps (4 chunks
// each); the WK fp64 partial sums of a score are added in a fixed order, the bias is added in fp64 and the result is
// rounded once to fp32. Each lane feeds one 16-byte chunk of its token row and of its expert row (8 bf16 / 4 fp32
// consecutive k) into 8 / 4 MFMAs: MFMA s takes element s of every lane, so lane group q contributes
// k = 4*EPC*c + EPC*q + s (the same mapping on both operands).
//   TB = 16: v_mfma_f64_16x16x4f64, 16 tokens x 16 experts.
//   TB = 4:  v_mfma_f64_4x4x4_4b_f64, its four blocks one group of 4 tokens against 4 x 4 experts.
//   TB = 1:  one token on v_fma_f64; lane group q's partial sums are added across the groups at the end.
// All three do about 16 multiply-adds per cycle and SIMD (a 16 x 16 x 4 product takes 64 cycles, measured), and the
// vector ALU does not run beside an fp64 MFMA: the bound is the products and, at 8 cycles each, the conversions to
// fp64 (T = 16384, E = 64, d = 2048: 4.3 GFLOP, 56 us of products, 86 us measured, 108 before). A workgroup's
// products run on one CU, so a short batch takes workgroups of few tokens: 16 tokens x 64 experts x d = 2048 alone
// are 14 us of a CU's fp64 rate, whatever the token count. Long batches take TT token tiles per wavefront: an expert
// chunk is then converted once for TT products, a token chunk once for NET.
// PF column steps of loads are in flight per wavefront.
// MODE says what becomes of the scores. SCORES: they are all there is to do, and a workgroup takes the 16 NET WE experts
// from 16 NET WE blockIdx.y on.
enum { ROUTE = 0, GATED = 1, SCORES = 2 };
template <typename T, int MODE, int TB, int TT, int NET, int WE, int WK, int PF>
__global__ __launch_bounds__(64 * WE * WK) void route_fwd_kernel(const T* __restrict__ x, const T* __restrict__ wr,
                                                              const float* __restrict__ bias, int bias_div, int Tn,
                                                              int d, int E, int k, int renorm,
                                                              float* __restrict__ logits, int32_t* __restrict__ idx,
                                                              float* __restrict__ gw, GateArgs ga) {
  const int ld = E;  // row length of logits and bias
  if constexpr (MODE == SCORES) {
    const int eb = blockIdx.y * 16 * NET * WE;
    wr += (size_t)eb * d;
    logits += eb;
    if (bias) bias += eb;
    E = min(E - eb, 16 * NET * WE);
  }
  constexpr int EP = EPC<T>::value;        // elements per 16-byte chunk
  constexpr int EW = 16 * NET * WE + 1;    // padded expert stride of the partial-sum table
  constexpr int NTOK = TB * TT;
  constexpr int W = WE * WK;
  extern __shared__ double part[];         // [WK][NTOK][EW]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int we = wave % WE, wk = wave / WE;
  const int i = lane & 15, q = lane >> 4;
  const int t0 = blockIdx.x * NTOK;
  const int e0 = we * 16 * NET;
  // Column steps [s0, s1) of this wavefront.
  const int steps = d / (4 * EP);
  const int s0 = (int)((long)steps * wk / WK), s1 = (int)((long)steps * (wk + 1) / WK);
  const T* xrow[TT];
  const T* wrow[NET];
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) {
    const int t = t0 + tt * TB + (TB == 16 ? i : TB == 4 ? (lane & 3) : 0);
    xrow[tt] = x + (size_t)(t < Tn ? t : Tn - 1) * d + EP * q;  // rows past the end: a valid row, never used
  }
#pragma unroll
  for (int et = 0; et < NET; ++et) {
    const int e = e0 + 16 * et + i;
    wrow[et] = wr + (size_t)(e < E ? e : E - 1) * d + EP * q;   // as above
  }
  typedef typename std::conditional<TB == 16, doublex4, double>::type Acc;
  // CH independent accumulator chains per product (column steps alternate between them), added in chain order
  // at the end: back-to-back MFMAs on one accumulator wait for each other.
  constexpr int CH = TT * NET >= 8 ? 1 : TT * NET >= 4 ? 2 : 4;
  Acc acc[CH][TT][NET];
#pragma unroll
  for (int ch = 0; ch < CH; ++ch)
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
      for (int et = 0; et < NET; ++et) {
        if constexpr (TB == 16) acc[ch][tt][et] = doublex4{0.0, 0.0, 0.0, 0.0};
        else acc[ch][tt][et] = 0.0;
      }
  Chunk xc[PF][TT], wc[PF][NET];
  auto load = [&](int st, Chunk (&xb)[TT], Chunk (&wb)[NET]) {
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) xb[tt] = ld_chunk(xrow[tt] + st * 4 * EP);
#pragma unroll
    for (int et = 0; et < NET; ++et) wb[et] = ld_chunk(wrow[et] + st * 4 * EP);
  };
  auto compute = [&](const Chunk (&xb)[TT], const Chunk (&wb)[NET]) {
    float xf[TT][EP], wf[NET][EP];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) chunk_to_f<T>(xb[tt], xf[tt]);
#pragma unroll
    for (int et = 0; et < NET; ++et) chunk_to_f<T>(wb[et], wf[et]);
#pragma unroll
    for (int s = 0; s < EP; ++s) {
      double xd[TT], wd[NET];
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) xd[tt] = (double)xf[tt][s];
#pragma unroll
      for (int et = 0; et < NET; ++et) wd[et] = (double)wf[et][s];
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int et = 0; et < NET; ++et) {
          Acc& a = acc[s % CH][tt][et];
          if constexpr (TB == 16) a = __builtin_amdgcn_mfma_f64_16x16x4f64(xd[tt], wd[et], a, 0, 0, 0);
          else if constexpr (TB == 4) a = __builtin_amdgcn_mfma_f64_4x4x4f64(wd[et], xd[tt], a, 0, 0, 0);
          else a = fma(xd[tt], wd[et], a);
        }
    }
  };
#pragma unroll
  for (int u = 0; u < PF; ++u)
    if (s0 + u < s1) load(s0 + u, xc[u], wc[u]);
  for (int st = s0; st < s1; st += PF) {
#pragma unroll
    for (int u = 0; u < PF; ++u) {
      if (st + u < s1) {
        compute(xc[u], wc[u]);
        if (st + u + PF < s1) load(st + u + PF, xc[u], wc[u]);
      }
    }
  }
  // 16x16x4: register r of lane group q holds D[token 4r + q][expert i]. 4x4x4: lane l holds token l & 3 and expert
  // 4 * ((l >> 2) & 3) + (l >> 4). One token: every lane group holds its own columns' sum for expert i.
#pragma unroll
  for (int tt = 0; tt < TT; ++tt)
#pragma unroll
    for (int et = 0; et < NET; ++et) {
      Acc a = acc[0][tt][et];
#pragma unroll
      for (int ch = 1; ch < CH; ++ch) a += acc[ch][tt][et];
      if constexpr (TB == 16) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          part[(wk * NTOK + tt * 16 + 4 * r + q) * EW + e0 + 16 * et + i] = a[r];
      } else if constexpr (TB == 4) {
        part[(wk * NTOK + tt * 4 + (lane & 3)) * EW + e0 + 16 * et + (lane & 12) + q] = a;
      } else {
        a += __shfl_xor(a, 16, 64);
        a += __shfl_xor(a, 32, 64);
        if (q == 0) part[(wk * NTOK + tt) * EW + e0 + 16 * et + i] = a;
      }
    }
  __syncthreads();

  // Each wavefront finishes tokens wave, wave + W, ...: fixed-order sum of the WK partials, bias, one rounding, then
  // k rounds of the wavefront maximum over order-preserving keys (lowest expert index among equal scores).
  constexpr int QE = (16 * NET * WE + 63) / 64;  // experts per lane: lane, lane + 64, ...
  // the score of expert lane + 64 qq of a token (which is also stored)
  auto score_of = [&](int row, int qq) -> float {
    const int e = lane + 64 * qq, tt = t0 + row;
    if (e >= E) return -INFINITY;
    double sum = part[row * EW + e];
#pragma unroll
    for (int w = 1; w < WK; ++w) sum += part[(w * NTOK + row) * EW + e];
    if (bias) sum += (double)bias[(size_t)(tt / bias_div) * ld + e];
    const float L = (float)sum;
    logits[(size_t)tt * ld + e] = L;
    return L;
  };
  if constexpr (MODE == SCORES) {
    for (int row = wave; row < NTOK && t0 + row < Tn; row += W)
#pragma unroll
      for (int qq = 0; qq < QE; ++qq) (void)score_of(row, qq);
    return;
  }
  if constexpr (MODE == GATED) {
    // as many tokens at once as the wavefront has, up to 4 (us at 1 / 2 / 4: T = 16,384, d = 128, E = 64, groups and bias
    // 35.5 / 32.9 / 31.8; T = 8192, d = 2048, E = 256 166 / 163.3 / 162.5)
    constexpr int NT = NTOK >= 4 * W ? 4 : NTOK >= 2 * W ? 2 : 1;
    for (int row = wave; row < NTOK && t0 + row < Tn; row += NT * W) {
      float v[NT][QE];
      double* lds[NT];
      int valid = 0;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = row + n * W;
        lds[n] = part + r * EW;
        const bool in = t0 + r < Tn;
        valid += in;
#pragma unroll
        for (int qq = 0; qq < QE; ++qq) v[n][qq] = in ? score_of(r, qq) : -INFINITY;
      }
      gated_select<QE, NT>(v, E, k, renorm, ga, lds, valid, (size_t)W * k, idx + (size_t)(t0 + row) * k,
                           gw + (size_t)(t0 + row) * k);
    }
    return;
  }
  for (int row = wave; row < NTOK; row += W) {
    const int tt = t0 + row;
    if (tt >= Tn) break;
    uint32_t key[QE];
    float v[QE];
#pragma unroll
    for (int qq = 0; qq < QE; ++qq) {
      v[qq] = score_of(row, qq);
      key[qq] = lane + 64 * qq < E ? score_key(v[qq]) : 0u;
    }
    float myv = -INFINITY;
    int myi = 0;
    for (int j = 0; j < k; ++j) {
      uint32_t m = key[0];
#pragma unroll
      for (int qq = 1; qq < QE; ++qq) m = max(m, key[qq]);
      m = wave_max_u32(m);
      int best = 0x7fffffff;  // no selectable score is left (NaN scores only)
      if (m != 0u) {
#pragma unroll
        for (int qq = QE - 1; qq >= 0; --qq) {
          const uint64_t b = __ballot(key[qq] == m);
          if (b) best = 64 * qq + __builtin_ctzll(b);
        }
      }
#pragma unroll
      for (int qq = 0; qq < QE; ++qq)
        if (lane + 64 * qq == best) key[qq] = 0u;
      if (lane == j) {
        myv = key_score(m);
        myi = best;
      }
    }
    const float m = __shfl(myv, 0, 64);  // the largest score of the token
    const float ex = (lane < k) ? expf(myv - m) : 0.f;
    float zp = ex;
    if (!renorm) {
      zp = 0.f;
#pragma unroll
      for (int qq = 0; qq < QE; ++qq)
        if (lane + 64 * qq < E) zp += expf(v[qq] - m);
    }
    zp = wave_sum(zp);
    if (lane < k) {
      idx[(size_t)tt * k + lane] = myi;
      gw[(size_t)tt * k + lane] = ex / zp;
    }
  }
}

template <typename T, int MODE, int TB, int TT, int NET, int WE, int WK, int PF>
static hipError_t route_fwd_run(const moe_desc& d, const void* x, const void* wr, const float* bias, int div,
                                float* logits, int32_t* idx, float* w, const GateArgs& ga, hipStream_t s) {
  constexpr int NTOK = TB * TT;
  constexpr size_t LDS = (size_t)WK * NTOK * (16 * NET * WE + 1) * sizeof(double);
  static_assert(LDS <= 160 * 1024, "partial-sum table");
  auto kern = route_fwd_kernel<T, MODE, TB, TT, NET, WE, WK, PF>;
  if (LDS > 65536) {
    static std::atomic<uint64_t> lds_set{0};
    if (hipError_t e = lds_limit_once((const void*)kern, (int)LDS, lds_set); e != hipSuccess) return e;
  }
  KernelTimer kt(MODE == SCORES ? "gate_scores" : MODE == GATED ? "route_gated" : "route_fwd", s);
  const dim3 grid((d.T + NTOK - 1) / NTOK, MODE == SCORES ? (d.n_experts + 16 * NET * WE - 1) / (16 * NET * WE) : 1);
  hipLaunchKernelGGL(kern, grid, dim3(64 * WE * WK), LDS, s, (const T*)x, (const T*)wr, bias,
                     div, d.T, d.d_model, d.n_experts, d.top_k, d.renormalize, logits, idx, w, ga);
  return hipGetLastError();
}

template <typename T, int MODE>
static hipError_t route_fwd_t(const moe_desc& d, const void* x, const void* wr, const float* bias, int bg,
                              float* logits, int32_t* idx, float* w, const GateArgs& ga, hipStream_t s) {
  const int E = d.n_experts;
  const int div = d.T / (bg > 0 ? bg : 1);
  // Tokens per workgroup: the fewest (1, 4, 16 or 32) whose workgroups are at most one per CU, since a workgroup costs
  // its padded tokens' products and a second round costs as much as the first. Measured on MI355X (d = 2048, E = 64;
  // us for 1 / 4 / 16 / 32 tokens): T = 24 12 / 14 / - / -, T = 300 22 / 15 / 26 / 43, T = 3000 - / 48 / 26 / 43,
  // T = 8192 - / - / 50 / 44; the 16-token workgroups of 4 wavefronts used before took 36, 37, 37 and 57.
  // Past one round of 32 tokens a full one costs 0.9 of two rounds of 16, but a last round that is nearly empty as much
  // as a full one: 32 tokens are taken while their rounds cost less (bf16, E = 64, d = 2048, us for 16 / 32 tokens:
  // T = 8300 68 / 80, 12,288 69 / 80, 16,384 88 / 82, 16,500 108 / 119, 24,576 128 / 121). With up to 32 bf16 experts
  // 16 tokens of 4 wavefronts are always the better past one round (E = 32, T = 16,384, d = 128: 12.1 / 15.3, T = 8300,
  // d = 2048: 36 / 47).
  // Wavefronts: as many as fit the LDS table and, at 16 of them, 128 VGPRs without spills; 4 to a workgroup of 16 tokens
  // in long batches, where several workgroups share a CU.
#define RT(TB, TT, NET, WE, WK, PF) \
  return route_fwd_run<T, MODE, TB, TT, NET, WE, WK, PF>(d, x, wr, bias, div, logits, idx, w, ga, s)
  const int cus = device_cus();
  const int r16 = (d.T + 16 * cus - 1) / (16 * cus), r32 = (r16 + 1) / 2;  // rounds of 16 and of 32 tokens per CU
  const bool by32 = r32 == 1 || ((E > 32 || d.dtype == MOE_F32) && 20 * r32 <= 11 * r16);
  const int tok = d.T <= cus ? 1 : d.T <= 4 * cus ? 4 : r16 == 1 ? 16 : by32 ? 32 : 64;  // 64: 16, in a long batch
  if (E <= 16) {
    if (tok == 1) RT(1, 1, 1, 1, 16, 4);
    if (tok == 4) RT(4, 1, 1, 1, 16, 4);
    if (tok == 16) RT(16, 1, 1, 1, 16, 4);
    RT(16, 1, 1, 1, 8, 4);  // one expert tile: 32 tokens per workgroup measured slower (28 against 30 us at d = 4096)
  } else if (E <= 32) {
    if (tok == 1) RT(1, 1, 2, 1, 16, 4);
    if (tok == 4) RT(4, 1, 2, 1, 16, 4);
    if (tok == 16) RT(16, 1, 2, 1, 8, 3);
    if (tok == 32) RT(16, 2, 2, 1, 8, 2);
    RT(16, 1, 2, 1, 4, 4);
  } else if (E <= 64) {
    if (tok == 1) RT(1, 1, 4, 1, 16, 2);
    if (tok == 4) RT(4, 1, 4, 1, 16, 2);
    if (tok == 16) RT(16, 1, 4, 1, 8, 2);
    if (tok == 32) RT(16, 2, 4, 1, 8, 2);
    RT(16, 1, 4, 1, 4, 2);
  } else if (E <= 128) {
    if (tok == 1) RT(1, 1, 4, 2, 8, 2);
    if (tok == 4) RT(4, 1, 4, 2, 8, 2);
    if (tok == 32) RT(16, 2, 4, 2, 4, 2);
    RT(16, 1, 4, 2, 4, 2);
  } else {
    if (tok == 1) RT(1, 1, 4, 4, 4, 2);
    if (tok == 4) RT(4, 1, 4, 4, 4, 2);
    if (tok == 32) RT(16, 2, 4, 4, 2, 2);
    RT(16, 1, 4, 4, 2, 2);
  }
#undef RT
}

hipError_t launch_route_fwd(const moe_desc& d, const void* x, const void* wr, const float* bias, int bg,
                            float* logits, int32_t* idx, float* w, hipStream_t s) {
  const GateArgs none{};
  if (d.dtype == MOE_BF16) return route_fwd_t<bf16, ROUTE>(d, x, wr, bias, bg, logits, idx, w, none, s);
  return route_fwd_t<float, ROUTE>(d, x, wr, bias, bg, logits, idx, w, none, s);
}

// Selection from scores that are there: one wavefront per token.
template <int QE>
__global__ __launch_bounds__(256) void gate_select_kernel(const float* __restrict__ logits, int Tn, int E, int k, int renorm,
                                                          int32_t* __restrict__ idx, float* __restrict__ gw, GateArgs ga) {
  __shared__ double values[4][64 * QE];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * 4 + w;
  if (t >= Tn) return;
  float v[1][QE];
#pragma unroll
  for (int qq = 0; qq < QE; ++qq) v[0][qq] = lane + 64 * qq < E ? logits[(size_t)t * E + lane + 64 * qq] : -INFINITY;
  double* row[1] = {values[w]};
  gated_select<QE, 1>(v, E, k, renorm, ga, row, 1, 0, idx + (size_t)t * k, gw + (size_t)t * k);
}

template <typename T>
static hipError_t route_gated_t(const moe_desc& d, const void* x, const void* wr, const float* bias, int bg,
                                float* logits, int32_t* idx, float* w, const GateArgs& ga, hipStream_t s) {
  const int E = d.n_experts, div = d.T / bg, cus = device_cus();
  // The fused kernel holds all the experts' scores of its tokens in one workgroup, on one CU. Where its workgroups would
  // leave CUs idle, or fill a last round badly, the scores are spread over them instead, in tiles of fewer experts, and
  // selected from by a second launch. The estimates: us of a tile's products at d = 2048 times the tiles that the busiest CU
  // gets, and 4 us around one launch, 6.5 around two; the fused kernel's tile is as wide as its padded experts (multiples
  // of 16) and has the tokens that route_fwd_t gives it. us, fused / spread (bf16, top-4, groups and bias), T, d, E:
  //   1, 2048, 64 11.6 / 8.7;  1, 4096, 200 56.7 / 12.7;  1, 512, 200 13.1 / 8.4;  17, 256, 256 10.9 / 9.0;
  //   64, 2048, 64 12.1 / 8.9;  200, 4096, 200 58.0 / 20.4;  465, 4096, 200 73.3 / 29.3;  1000, 2048, 64 15.1 / 12.8;
  //   2048, 2048, 64 26.2 / 17.5;  2048, 4096, 200 159 / 79.4;  2048, 256, 256 21.7 / 15.0; fp32 1, 4096, 200 104 / 16.6;
  //   fused instead: 1, 1408, 16 5.9 / 8.3;  1000, 2560, 32 11.9 / 13.9;  4096, 2048, 64 26.8 / 27.2;
  //   8192, 2048, 256 156 / 165.
  const double per = d.d_model / 2048.0;
  const auto rounds = [&](int tokens, int experts) {
    return (double)(((int64_t)((d.T + tokens - 1) / tokens) * ((E + experts - 1) / experts) + cus - 1) / cus);
  };
  const int wide = E <= 16 ? 16 : E <= 32 ? 32 : E <= 64 ? 64 : E <= 128 ? 128 : 256;
  const double fused = 4 + per * (wide / 16) *
                               (d.T <= cus       ? 1.65
                                : d.T <= 4 * cus ? 2.5
                                                 : std::min(5.5 * rounds(16, wide), 9.7 * rounds(32, wide)));
  static constexpr struct {
    int tokens, experts;
    double us;
  } tiles[] = {{1, 16, 2.5}, {4, 16, 4}, {16, 16, 7}, {16, 32, 12}, {32, 32, 21}, {32, 64, 40}};
  int pick = -1;
  double best = fused;
  for (int i = 0; i < 6; ++i) {
    const double us = 6.5 + per * tiles[i].us * rounds(tiles[i].tokens, tiles[i].experts);
    if (us < best) {
      best = us;
      pick = i;
    }
  }
  const bool spread = pick >= 0;
  hipError_t e = hipSuccess;
#define GS(TB, TT, NET, WK, PF) \
  e = route_fwd_run<T, SCORES, TB, TT, NET, 1, WK, PF>(d, x, wr, bias, div, logits, nullptr, nullptr, ga, s)
  switch (pick) {
    case 0: GS(1, 1, 1, 16, 4); break;
    case 1: GS(4, 1, 1, 16, 4); break;
    case 2: GS(16, 1, 1, 16, 4); break;
    case 3: GS(16, 1, 2, 8, 3); break;
    case 4: GS(16, 2, 2, 8, 2); break;
    case 5: GS(16, 2, 4, 8, 2); break;
  }
#undef GS
  if (!spread) return route_fwd_t<T, GATED>(d, x, wr, bias, bg, logits, idx, w, ga, s);
  if (e != hipSuccess) return e;
  KernelTimer kt("gate_select", s);
  const dim3 grid((d.T + 3) / 4);
#define GSEL(QE) \
  hipLaunchKernelGGL(gate_select_kernel<QE>, grid, dim3(256), 0, s, logits, d.T, E, d.top_k, d.renormalize, idx, w, ga)
  if (E <= 64) GSEL(1);
  else if (E <= 128) GSEL(2);
  else GSEL(4);
#undef GSEL
  return hipGetLastError();
}

hipError_t launch_route_gated(const moe_desc& d, const moe_gate& g, const void* x, const void* wr, const float* bias,
                              int bg, const float* select_bias, float* logits, int32_t* idx, float* w, hipStream_t s) {
  const int size = d.n_experts / g.n_groups;
  int lane_shift = 0;
  while ((2 << lane_shift) * g.n_groups <= 64) ++lane_shift;
  const GateArgs ga{select_bias, g.scale, g.score == MOE_SCORE_SIGMOID, g.n_groups, g.topk_groups, g.group_top, size,
                    (65536 + size - 1) / size, lane_shift};
  if (d.dtype == MOE_BF16) return route_gated_t<bf16>(d, x, wr, bias, bg, logits, idx, w, ga, s);
  return route_gated_t<float>(d, x, wr, bias, bg, logits, idx, w, ga, s);
}

// ------------------------------------------------------------------------------ backward

// dscores per token (one wavefront per token).
__global__ __launch_bounds__(256) void route_dlogits_kernel(int Tn, int E, int k, int renorm,
                                                            const float* __restrict__ logits,
                                                            const int32_t* __restrict__ idx,
                                                            const float* __restrict__ gw,
                                                            const float* __restrict__ dgate,
                                                            float* __restrict__ dl) {
  const int lane = threadIdx.x & 63;
  const int wave = (blockIdx.x * blockDim.x + threadIdx.x) >> 6;
  const int nwaves = (gridDim.x * blockDim.x) >> 6;
  for (int t = wave; t < Tn; t += nwaves) {
    float wj = 0.f, gj = 0.f;
    int ij = -1;
    if (lane < k) {
      wj = gw[(size_t)t * k + lane];
      gj = dgate[(size_t)t * k + lane];
      ij = idx[(size_t)t * k + lane];
    }
    if (renorm) {
      const float sgw = wave_sum(wj * gj);
      for (int e0 = 0; e0 < E; e0 += 64) {
        int e = e0 + lane;
        float val = 0.f;
        for (int jj = 0; jj < k; ++jj) {
          int i2 = __shfl(ij, jj, 64);
          float w2 = __shfl(wj, jj, 64), g2 = __shfl(gj, jj, 64);
          if (e == i2) val = w2 * (g2 - sgw);
        }
        if (e < E) dl[(size_t)t * E + e] = val;
      }
    } else {
      // p over all E experts (up to 4 per lane); g = dgate scattered onto E
      constexpr int NQ = 4;  // E <= 256
      float p[NQ], g[NQ], M = -INFINITY, zp = 0.f, spg = 0.f;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int e = lane + 64 * n;
        p[n] = e < E ? logits[(size_t)t * E + e] : -INFINITY;
        M = fmaxf(M, p[n]);
      }
      M = wave_max(M);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        p[n] = lane + 64 * n < E ? expf(p[n] - M) : 0.f;
        zp += p[n];
        g[n] = 0.f;
      }
      const float Z = wave_sum(zp);
      for (int jj = 0; jj < k; ++jj) {
        const int i2 = __builtin_amdgcn_readlane(ij, jj);
        const float g2 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gj), jj));
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          if (lane + 64 * n == i2) g[n] = g2;
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        p[n] = p[n] / Z;
        spg += p[n] * g[n];
      }
      const float S = wave_sum(spg);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
        if (lane + 64 * n < E) dl[(size_t)t * E + lane + 64 * n] = p[n] * (g[n] - S);
    }
  }
}

// ... of the gated routing. With w_j the returned weight of slot j, g_j its gradient, c the scale:
//   renormalised: dl_j = w_j (g_j - sum_i w_i g_i / c), for sigmoid scores times (1 - s_j);
//   sigmoid:      dl_j = w_j (1 - s_j) g_j;       softmax: dl_e = p_e (c g_e - sum_i c p_i g_i) over all the experts.
// 1 - s is formed as sigmoid(-l), which does not cancel. Slots that no expert fills give nothing.
// A wavefront takes 8 tokens: first a lane per slot (lane 8 n + j has slot j of token n), so that the loads' latencies are
// paid once for all of them, then the rows one by one, a lane per expert (T = 16,384, E = 64, top-6: 6.6 us, 8.2 with a
// wavefront per token). DENSE, which reads whole rows of scores: one token (T = 1500, E = 8: 3.9 us, 10 with eight).
template <bool DENSE>
__global__ __launch_bounds__(256) void gate_dlogits_kernel(int Tn, int E, int k, int renorm, int sigmoid, float scale,
                                                           const float* __restrict__ logits,
                                                           const int32_t* __restrict__ idx,
                                                           const float* __restrict__ gw,
                                                           const float* __restrict__ dgate, float* __restrict__ dl) {
  const float per_scale = 1.f / scale;
  constexpr int NQ = 4, TW = DENSE ? 1 : 8;  // E <= 256; tokens of a wavefront
  const int lane = threadIdx.x & 63;
  const int t0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * TW;
  if (t0 >= Tn) return;
  const int t = t0 + (lane >> 3), j = lane & 7;
  const size_t slot = (size_t)t * k + j;
  float wj = 0.f, gj = 0.f, lj = 0.f;
  int ij = NO_EXPERT;
  if (lane < 8 * TW && t < Tn && j < k) ij = idx[slot];
  const bool filled = (unsigned)ij < (unsigned)E;
  if (filled) {
    wj = gw[slot];
    gj = dgate[slot];
    if (sigmoid) lj = logits[(size_t)t * E + ij];
  }
  float val = DENSE ? scale * gj : gj;  // what the slot adds to its expert
  if constexpr (!DENSE) {
    if (renorm) {
      // g - (sum w g) / c, each operation rounded by itself: where one expert is chosen the two cancel
#pragma clang fp contract(off)
      float s = wj * gj;
      s += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(s), 0xb1, 0xf, 0xf, false));   // lane pairs,
      s += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(s), 0x4e, 0xf, 0xf, false));   // quads,
      s += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(s), 0x141, 0xf, 0xf, false));  // eights
      s *= per_scale;
      val -= s;
    }
    val *= wj;
    if (sigmoid && filled) val /= 1.f + expf(lj);
  }
  for (int n = 0; n < TW && t0 + n < Tn; ++n) {
    const size_t row = (size_t)(t0 + n) * E;
    float out[NQ] = {0.f, 0.f, 0.f, 0.f};
    for (int jj = 0; jj < k; ++jj) {
      const int i2 = __builtin_amdgcn_readlane(ij, 8 * n + jj);
      const float g2 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(val), 8 * n + jj));
#pragma unroll
      for (int q = 0; q < NQ; ++q)
        if (lane + 64 * q == i2) out[q] = g2;
    }
    if constexpr (DENSE) {
      float p[NQ], m = -INFINITY, zp = 0.f, spg = 0.f;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        p[q] = lane + 64 * q < E ? logits[row + lane + 64 * q] : -INFINITY;
        m = fmaxf(m, p[q]);
      }
      m = wave_max_dpp(m);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        p[q] = p[q] > -INFINITY ? (p[q] == m ? 1.f : expf(p[q] - m)) : 0.f;
        zp += p[q];
      }
      const float z = wave_sum(zp);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        p[q] = z == 0.f ? 0.f : p[q] / z;  // z = 0: every expert is masked
        spg += p[q] * out[q];
      }
      spg = wave_sum(spg);
#pragma unroll
      for (int q = 0; q < NQ; ++q) out[q] = p[q] * (out[q] - spg);
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q)
      if (lane + 64 * q < E) dl[row + lane + 64 * q] = out[q];
  }
}

// Partial dW_router over one chunk of tokens, part[chunk][e][c] = sum_{t in chunk} dl[t][e] * x[t][c], as an
// fp32 MFMA contraction (v_mfma_f32_16x16x4f32, tokens as K). Lane (q, i) of a wavefront loads JJ contiguous
// columns c0 + JJ*i .. + JJ-1 of token rows t + q (one coalesced load of the row segment per 16 lanes) and
// feeds column c0 + JJ*i + jj of MFMA number jj; its A operand is dl[t + q][16 et + i]. 8 token-steps of 4
// tokens are loaded before their MFMAs.
template <typename T, int JJ>
struct alignas(JJ * sizeof(T) < 16 ? JJ * sizeof(T) : 16) XRow {  // tensors are 16-byte aligned
  T v[JJ];
};

// JJ columns per lane: 4 for up to 16 experts (narrower workgroups, so that 256 of them need only 64 token
// chunks of partial sums: measured 9 us against 12 us for 8 columns and 128 chunks at T=4096, d=1024), 8 up to 32.
// For more experts, fewer while the accumulators (JJ x NET tiles) fit.
constexpr int dw_cols_per_lane(int net) { return net == 1 ? 4 : net <= 2 ? 8 : 16 / net; }

template <typename T, int NET, int JJ>
__global__ __launch_bounds__(256) void route_dw_partial_kernel(int Tn, int d, int E, int tok_per_chunk,
                                                               const T* __restrict__ x,
                                                               const float* __restrict__ dl,
                                                               float* __restrict__ part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int q = lane >> 4, i = lane & 15;
  const int c0 = (blockIdx.x * 4 + wave) * 16 * JJ;  // first column of this wavefront
  if (c0 >= d) return;                               // d is a multiple of 16 * JJ: all or nothing
  const int chunk = blockIdx.y;
  const int tb = chunk * tok_per_chunk;
  const int te = min(Tn, tb + tok_per_chunk);
  floatx4 acc[JJ][NET];
#pragma unroll
  for (int jj = 0; jj < JJ; ++jj)
#pragma unroll
    for (int et = 0; et < NET; ++et) acc[jj][et] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int t0 = tb; t0 < te; t0 += 32) {
    XRow<T, JJ> xv[8];
    float a[8][NET];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int t = t0 + 4 * u + q;
      const bool ok = t < te;
      if (ok) xv[u] = *reinterpret_cast<const XRow<T, JJ>*>(x + (size_t)t * d + c0 + JJ * i);
      else xv[u] = XRow<T, JJ>{};
#pragma unroll
      for (int et = 0; et < NET; ++et) {
        const int e = 16 * et + i;
        a[u][et] = (ok && e < E) ? dl[(size_t)t * E + e] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int jj = 0; jj < JJ; ++jj) {
        const float b = to_f(xv[u].v[jj]);
#pragma unroll
        for (int et = 0; et < NET; ++et)
          acc[jj][et] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u][et], b, acc[jj][et], 0, 0, 0);
      }
  }
  // register r of lane group q holds D[expert 16 et + 4q + r][n = i], column c0 + JJ*i + jj
#pragma unroll
  for (int et = 0; et < NET; ++et)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = 16 * et + 4 * q + r;
      if (e >= E) continue;
      float* o = part + ((size_t)chunk * E + e) * d + c0 + JJ * i;
#pragma unroll
      for (int jj = 0; jj < JJ; ++jj) o[jj] = acc[jj][et][r];
    }
}

// The same partial sums for more than 32 experts and many tokens. A wavefront holds 64 experts x 16 groups of N columns
// (16 bytes of x) and steps through its tokens 4 at a time with one 16-byte load of dl (lane (q, i): token t + q, experts
// 4 i .. 4 i + 3, one per MFMA row) and one of x (its columns of token t + q) per 4 N MFMAs, 16 tokens ahead of the MFMAs.
// Bound by the fp32 MFMAs. Bit for bit the sums of the narrow kernel. Both launches, narrow and wide: T = 8192, d = 2048,
// E = 256 181 and 96 us (56 us of MFMA at the peak rate); T = 16384, E = 64 78 and 62.
template <typename T, bool VEC>
__global__ __launch_bounds__(256, 2) void route_dw_wide_kernel(int Tn, int d, int E, int tok_per_chunk, int col_blocks,
                                                               const T* __restrict__ x, const float* __restrict__ dl,
                                                               float* __restrict__ part) {
  constexpr int N = EPC<T>::value, U = 4;
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int groups = (E + 63) >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  // a workgroup's wavefronts: the expert groups of one column block first (they read the same x)
  const int cb = wave / groups, eg = wave - cb * groups;
  if (cb >= col_blocks) return;
  const int c0 = (cb * 16 + i) * N, e0 = eg * 64 + 4 * i;
  const int tb = blockIdx.y * tok_per_chunk, te = min(Tn, tb + tok_per_chunk);
  floatx4 acc[N][4];
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int m = 0; m < 4; ++m) acc[s][m] = floatx4{0.f, 0.f, 0.f, 0.f};
  struct Buf {
    Chunk x[U];
    float a[U][4];
  };
  // the chunk's rows of x and dl as buffers: tokens past its end read as zeros
  const auto xr = buf_rsrc(x + (size_t)tb * d, (size_t)(te - tb) * d * sizeof(T));
  const auto gr = buf_rsrc(dl + (size_t)tb * E, (size_t)(te - tb) * E * 4);
  int xo = (q * d + c0) * (int)sizeof(T), go = (q * E + e0) * 4;
  auto load = [&](Buf& b) {  // the next 4 U tokens
#pragma unroll
    for (int u = 0; u < U; ++u) {
      b.x[u] = buf_ld16(xr, xo);
      if (VEC) {
        const Chunk v = buf_ld16(gr, e0 < E ? go : kBufPast);
#pragma unroll
        for (int m = 0; m < 4; ++m) b.a[u][m] = __uint_as_float(v.w[m]);
      } else {
#pragma unroll
        for (int m = 0; m < 4; ++m)
          b.a[u][m] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(gr, e0 + m < E ? go + 4 * m : kBufPast, 0, 0));
      }
      xo += 4 * d * (int)sizeof(T);
      go += 16 * E;
    }
  };
  auto mul = [&](const Buf& b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float xf[N];
      chunk_to_f<T>(b.x[u], xf);
#pragma unroll
      for (int s = 0; s < N; ++s)
#pragma unroll
        for (int m = 0; m < 4; ++m)
          acc[s][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.a[u][m], xf[s], acc[s][m], 0, 0, 0);
    }
  };
  Buf b0, b1;
  load(b0);
  for (int t0 = tb; t0 < te; t0 += 8 * U) {
    load(b1);
    __builtin_amdgcn_sched_barrier(0);
    mul(b0);
    __builtin_amdgcn_sched_barrier(0);
    load(b0);
    __builtin_amdgcn_sched_barrier(0);
    mul(b1);
    __builtin_amdgcn_sched_barrier(0);
  }
  // register r of lane (q, i), MFMA (s, m): expert 64 eg + 4 (4 q + r) + m, column c0 + s
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int e = eg * 64 + 4 * (4 * q + r) + m;
      if (e >= E) continue;
      float* o = part + ((size_t)blockIdx.y * E + e) * d + c0;
#pragma unroll
      for (int s = 0; s < N; s += 4)
        *reinterpret_cast<float4*>(o + s) = float4{acc[s][m][r], acc[s + 1][m][r], acc[s + 2][m][r], acc[s + 3][m][r]};
    }
}

// dW_router[o] = sum over chunks of part[chunk][o], in a fixed order: thread (g, o) of a workgroup sums
// the chunks g, g + 16, g + 32, ... in turn, then the 16 partial sums of an output are added in g order.
constexpr int RED_G = 16;  // chunk lanes per output
__global__ __launch_bounds__(256) void route_dw_reduce_kernel(int n4, int nchunks, const float4* __restrict__ part,
                                                              float4* __restrict__ out) {
  __shared__ float4 red[RED_G][256 / RED_G];
  const int g = threadIdx.x / (256 / RED_G), ol = threadIdx.x % (256 / RED_G);
  const int o = blockIdx.x * (256 / RED_G) + ol;
  float4 s = float4{0.f, 0.f, 0.f, 0.f};
  if (o < n4)
    for (int c = g; c < nchunks; c += RED_G) {
      const float4 v = part[(size_t)c * n4 + o];
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  red[g][ol] = s;
  __syncthreads();
  if (g == 0 && o < n4) {
    float4 t = red[0][ol];
    for (int h = 1; h < RED_G; ++h) {
      const float4 v = red[h][ol];
      t.x += v.x;
      t.y += v.y;
      t.z += v.z;
      t.w += v.w;
    }
    out[o] = t;
  }
}

// Column blocks of a wavefront's 16 chunks (route_dw_wide_kernel).
static int dw_wide_cols(const moe_desc& d) { return (int)(d.d_model * elem_bytes(d) / 256); }

static int dw_net(int E) { return E <= 16 ? 1 : E <= 32 ? 2 : E <= 64 ? 4 : E <= 128 ? 8 : 16; }

// Token chunks of the weight-gradient contraction, a multiple of 32 tokens each: as many as give the narrow kernel about
// 256 workgroups for up to 16 experts and 1024 above (4 wavefronts x 16 x JJ columns each). The chunk is the length of an
// fp32 accumulator and so sets the error of dW_router (T = 8192, d = 2048, E = 256: 3.0e-7 of its norm over 256 tokens,
// 4.1e-7 over 512): the wide kernel takes the same chunks, though it would fill the chip with fewer. Chunks of 32 tokens
// are too short for its loop body, which then runs once, from cold instruction caches; more than 64 experts, whose
// narrow kernel reads x several times, gain all the same once there are two of its wavefronts per SIMD (both launches,
// us for narrow / wide: E = 256, bf16, T = 4096, d = 512 47 / 39, T = 1000, d = 1024 26.6 / 28.3; E = 128, T = 4096,
// d = 1024 42.8 / 36.4, T = 2048, d = 512 24.1 / 25.5; E = 64, T = 2048, d = 2048 27.3 / 26.2, T = 3000, d = 1024
// 24.7 / 25.0; E = 33, T = 3000, d = 2048 25.8 / 28.8).
static void route_bwd_chunks(const moe_desc& d, int* nch, int* tpc, bool* wide) {
  const int E = d.n_experts;
  const int wg_cols = 64 * dw_cols_per_lane(dw_net(E));
  const int ncol = (d.d_model + wg_cols - 1) / wg_cols;
  const int maxch = (d.T + 31) / 32;
  const int want = ((E <= 16 ? 256 : 1024) + ncol - 1) / ncol;
  const int n = std::max(std::min(want, maxch), 1);
  const int per = ((d.T + n - 1) / n + 31) / 32 * 32;
  *tpc = per;
  *nch = (d.T + per - 1) / per;
  const int waves = dw_wide_cols(d) * ((E + 63) / 64) * *nch;  // of the wide kernel
  *wide = E > 32 && (per >= 64 || (E > 64 && waves >= 2048));
}

size_t route_bwd_ws_bytes(const moe_desc& d) {
  int nch, tpc;
  bool wide;
  route_bwd_chunks(d, &nch, &tpc, &wide);
  return align256((size_t)nch * d.n_experts * d.d_model * sizeof(float));
}

// dW_router = dlogits^T x of bf16 tokens on v_mfma_f32_16x16x32_bf16: the gradients of the scores as three bf16 numbers that
// add up to each fp32 one exactly (8 + 8 + 8 bits), so the products are those of the fp32 contraction. Three of them take a
// third of its time by the rates of large products, 1,586 and 154 TFLOP/s (T = 16,384, E = 64, d = 2048: 4.3 GFLOP, 28 us in
// fp32, 8 for three bf16 products; the tokens' 67 MB take 14; 21.7 us measured). A workgroup holds 128 columns x 16 NET experts; its wavefronts take the chunk's tokens 32 at a time in turn, with
// accumulators of their own, which meet in LDS half the columns at a time and are added in wavefront order.
//   tokens as K: lane (q, i) loads 16 bytes of tokens 8 q .. 8 q + 7 and turns the 8 x 8 block into operands of its columns
//   8 i + s, s = 0 .. 7, by byte permutes; row i of expert tile m is expert NET i + m, so that a token's gradients of a
//   lane's NET experts are one load. Tokens and experts past the end read as zeros.
// An infinite x makes NaN where a part of the gradient is 0; the fp32 contraction makes it only where the gradient is.
constexpr int GDW_W = 8;
template <int NET, bool VEC>
__global__ __launch_bounds__(64 * GDW_W, 2) void gate_dw_kernel(int Tn, int d, int E, int tok_per_chunk,
                                                                const bf16* __restrict__ x, const float* __restrict__ dl,
                                                                float* __restrict__ part) {
  __shared__ float4 red[GDW_W][16 * NET][16];
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = blockIdx.x * 128, e0 = blockIdx.y * 16 * NET;
  const int tb = blockIdx.z * tok_per_chunk, te = min(Tn, tb + tok_per_chunk);
  const auto xr = buf_rsrc(x + (size_t)tb * d + c0, ((size_t)(te - tb) * d - c0) * 2);
  const auto gr = buf_rsrc(dl + (size_t)tb * E, (size_t)(te - tb) * E * 4);
  const int el = e0 + NET * i;  // the lane's first expert
  floatx4 acc[8][NET];
#pragma unroll
  for (int s = 0; s < 8; ++s)
#pragma unroll
    for (int m = 0; m < NET; ++m) acc[s][m] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int t0 = 32 * w; t0 < te - tb; t0 += 32 * GDW_W) {
    Chunk xv[8];
    uint32_t g[8][NET];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = t0 + 8 * q + j;
      xv[j] = buf_ld16(xr, t < te - tb ? (t * d + 8 * i) * 2 : kBufPast);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int o = ((t0 + 8 * q + j) * E + el) * 4;
      if constexpr (VEC && NET == 4) {
        const Chunk c = buf_ld16(gr, el < E ? o : kBufPast);
#pragma unroll
        for (int m = 0; m < NET; ++m) g[j][m] = c.w[m];
      } else {
#pragma unroll
        for (int m = 0; m < NET; ++m)
          g[j][m] = __builtin_amdgcn_raw_buffer_load_b32(gr, el + m < E ? o + 4 * m : kBufPast, 0, 0);
      }
    }
    Chunk a[NET][3];
#pragma unroll
    for (int m = 0; m < NET; ++m)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        uint32_t hi[2], mid[2], low[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          hi[b] = g[2 * p + b][m];
          // an infinity or a NaN is all in the first part (of a NaN the upper half might be an infinity's)
          const bool special = (hi[b] & 0x7f800000u) == 0x7f800000u;
          if (special && (hi[b] & 0x7fffffu)) hi[b] = 0x7fc00000u;
          mid[b] = special ? 0u : __float_as_uint(__uint_as_float(hi[b]) - __uint_as_float(hi[b] & 0xffff0000u));
          low[b] = __float_as_uint(__uint_as_float(mid[b]) - __uint_as_float(mid[b] & 0xffff0000u));
        }
        a[m][0].w[p] = __builtin_amdgcn_perm(hi[1], hi[0], 0x07060302u);
        a[m][1].w[p] = __builtin_amdgcn_perm(mid[1], mid[0], 0x07060302u);
        a[m][2].w[p] = __builtin_amdgcn_perm(low[1], low[0], 0x07060302u);
      }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      Chunk b;
#pragma unroll
      for (int p = 0; p < 4; ++p)
        b.w[p] = __builtin_amdgcn_perm(xv[2 * p + 1].w[s / 2], xv[2 * p].w[s / 2], s % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int n = 2; n >= 0; --n)
#pragma unroll
        for (int m = 0; m < NET; ++m)
          acc[s][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[m][n]),
                                                              __builtin_bit_cast(bf16x8, b), acc[s][m], 0, 0, 0);
    }
  }
  // register r of lane (q, i), product (s, m): expert e0 + NET (4 q + r) + m, column c0 + 8 i + s
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h) __syncthreads();
#pragma unroll
    for (int m = 0; m < NET; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        red[w][NET * (4 * q + r) + m][i] =
            float4{acc[4 * h][m][r], acc[4 * h + 1][m][r], acc[4 * h + 2][m][r], acc[4 * h + 3][m][r]};
    __syncthreads();
    for (int u = threadIdx.x; u < 16 * NET * 16; u += 64 * GDW_W) {
      const int e = u >> 4, n = u & 15;
      if (e0 + e >= E) break;
      float4 v = red[0][e][n];
#pragma unroll
      for (int k = 1; k < GDW_W; ++k) {
        const float4 o = red[k][e][n];
        v.x += o.x;
        v.y += o.y;
        v.z += o.z;
        v.w += o.w;
      }
      *reinterpret_cast<float4*>(part + ((size_t)blockIdx.z * E + e0 + e) * d + c0 + 8 * n + 4 * h) = v;
    }
  }
}

static void route_dw_sum(const moe_desc& d, int nch, const float* part, float* dwr, hipStream_t s) {
  KernelTimer kt("route_dw_reduce", s);
  const int n4 = d.n_experts * d.d_model / 4;
  const int blocks = (n4 + 256 / RED_G - 1) / (256 / RED_G);
  hipLaunchKernelGGL(route_dw_reduce_kernel, dim3(blocks), dim3(256), 0, s, n4, nch, (const float4*)part, (float4*)dwr);
}

static unsigned token_blocks(const moe_desc& d) { return std::min((d.T + 3) / 4, 4096); }

// dW_router from the gradients of the scores.
template <typename T>
static hipError_t route_dw_t(const moe_desc& d, const void* x, const float* dl, float* dwr, void* ws, hipStream_t s) {
  const int E = d.n_experts;
  int nch, tpc;
  bool wide;
  route_bwd_chunks(d, &nch, &tpc, &wide);
  // one chunk (up to 32 tokens, or column blocks enough to fill the chip): its sums are the result, without the sum over
  // chunks and its launch (6 us)
  float* part = nch == 1 ? dwr : (float*)ws;
  {
    KernelTimer kt("route_dw_partial", s);
    if (wide) {
      const int cb = dw_wide_cols(d);
      const dim3 grid((cb * ((E + 63) / 64) + 3) / 4, nch);
      if (E % 4 == 0)
        hipLaunchKernelGGL((route_dw_wide_kernel<T, true>), grid, dim3(256), 0, s, d.T, d.d_model, E, tpc, cb,
                           (const T*)x, dl, part);
      else
        hipLaunchKernelGGL((route_dw_wide_kernel<T, false>), grid, dim3(256), 0, s, d.T, d.d_model, E, tpc, cb,
                           (const T*)x, dl, part);
    } else {
      const int wg_cols = 64 * dw_cols_per_lane(dw_net(E));
      const dim3 grid((d.d_model + wg_cols - 1) / wg_cols, nch);
#define RB_LAUNCH(NET)                                                                                       \
  hipLaunchKernelGGL((route_dw_partial_kernel<T, NET, dw_cols_per_lane(NET)>), grid, dim3(256), 0, s, d.T, \
                     d.d_model, E, tpc, (const T*)x, dl, part)
      if (E <= 16) RB_LAUNCH(1);
      else if (E <= 32) RB_LAUNCH(2);
      else if (E <= 64) RB_LAUNCH(4);
      else if (E <= 128) RB_LAUNCH(8);
      else RB_LAUNCH(16);
#undef RB_LAUNCH
    }
  }
  if (nch > 1) route_dw_sum(d, nch, part, dwr, s);
  return hipGetLastError();
}

// ... of bf16 tokens for the gated routing. Chunks of tokens: as many as give each CU a workgroup, at least a step of 32
// tokens for each wavefront, and no more than the workspace holds.
static hipError_t gate_dw(const moe_desc& d, const void* x, const float* dl, float* dwr, void* ws, hipStream_t s) {
  const int E = d.n_experts, net = E <= 16 ? 1 : E <= 32 ? 2 : 4;
  const int cols = d.d_model / 128, groups = (E + 16 * net - 1) / (16 * net);
  int most, tpc;
  bool wide;
  route_bwd_chunks(d, &most, &tpc, &wide);
  const int want = std::min({device_cus() / (cols * groups), d.T / (32 * GDW_W), most});
  const int per = (d.T + std::max(want, 1) - 1) / std::max(want, 1);
  tpc = (per + 31) / 32 * 32;
  const int nch = (d.T + tpc - 1) / tpc;
  float* part = nch == 1 ? dwr : (float*)ws;
  {
    KernelTimer kt("gate_dw", s);
    const dim3 grid(cols, groups, nch);
#define GD_LAUNCH(NET, VEC)                                                                                       \
  hipLaunchKernelGGL((gate_dw_kernel<NET, VEC>), grid, dim3(64 * GDW_W), 0, s, d.T, d.d_model, E, tpc, (const bf16*)x, \
                     dl, part)
    if (net == 1) GD_LAUNCH(1, false);
    else if (net == 2) GD_LAUNCH(2, false);
    else if (E % 4) GD_LAUNCH(4, false);
    else GD_LAUNCH(4, true);
#undef GD_LAUNCH
  }
  if (nch > 1) route_dw_sum(d, nch, part, dwr, s);
  return hipGetLastError();
}

static hipError_t route_dw(const moe_desc& d, const void* x, const float* dl, float* dwr, void* ws, hipStream_t s) {
  if (d.dtype == MOE_BF16) return route_dw_t<bf16>(d, x, dl, dwr, ws, s);
  return route_dw_t<float>(d, x, dl, dwr, ws, s);
}

hipError_t launch_route_bwd(const moe_desc& d, const void* x, const float* logits, const int32_t* idx,
                            const float* w, const float* dgate, float* dl, float* dwr, void* ws, hipStream_t s) {
  {
    KernelTimer kt("route_dlogits", s);
    hipLaunchKernelGGL(route_dlogits_kernel, dim3(token_blocks(d)), dim3(256), 0, s, d.T, d.n_experts, d.top_k,
                       d.renormalize, logits, idx, w, dgate, dl);
  }
  return route_dw(d, x, dl, dwr, ws, s);
}

hipError_t launch_route_gated_bwd(const moe_desc& d, const moe_gate& g, const void* x, const float* logits,
                                  const int32_t* idx, const float* w, const float* dgate, float* dl, float* dwr,
                                  void* ws, hipStream_t s) {
  {
    KernelTimer kt("gate_dlogits", s);
    const bool sigmoid = g.score == MOE_SCORE_SIGMOID, dense = !d.renormalize && !sigmoid;
    hipLaunchKernelGGL(dense ? gate_dlogits_kernel<true> : gate_dlogits_kernel<false>,
                       dim3(dense ? (d.T + 3) / 4 : (d.T + 31) / 32), dim3(256), 0, s, d.T, d.n_experts, d.top_k,
                       d.renormalize, (int)sigmoid, g.scale, logits, idx, w, dgate, dl);
  }
  return d.dtype == MOE_BF16 ? gate_dw(d, x, dl, dwr, ws, s) : route_dw_t<float>(d, x, dl, dwr, ws, s);
}

}  // namespace pcmoe
