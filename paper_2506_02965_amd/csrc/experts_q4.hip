// SwiGLU experts over few rows with 4-bit weights, and the packing of such weights.
//
// A weight is code * scale: the code one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (the E2M1 element of the OCP
// microscaling formats, which gfx950 converts to bf16 two at a time, exactly), the scale a bf16 number for each group of
// 32, 64 or 128 consecutive k of a weight row. A group's sum runs on v_mfma_f32_16x16x32_bf16 over the codes themselves;
// the scale multiplies that sum in fp32, so the weights are never rounded to anything. fp32 activations are split into
// three bf16 numbers that add up to them exactly, three products in place of one.
//
// Layout: blocks of 16 weight rows x 128 k, 1 KB in the order in which a wavefront feeds them to the MFMA: lane (q, i)
// holds 16 bytes of row i, dword s of them k = 32 s + 8 q .. + 7, so one 16-byte load per lane is four operands.
#include "expert_ops.h"

#include <algorithm>
#include <cmath>

namespace pcmoe {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ----------------------------------------------------------------------------------------------- packing

// Codes of eight values in units of their scale s: the nearest of the magnitudes, ties to the even code.
//   fp32: by comparisons with the midpoints times s, which are exact, so they decide on the quotient itself.
//   bf16: two 8-bit significands' quotient is a midpoint exactly or at least 2^-17 away from it, so the fp32 quotient (one
//   correction of v * rcp(s): exact where the quotient has few bits) decides, in the hardware's conversion. A third of the
//   instructions: the comparisons bound the packing (344 us for 470 M weights, 3.4 TB/s).
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float s, float) {
  uint32_t d = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = fabsf(v[e]);
    const uint32_t c = (a > 0.25f * s) + (a >= 0.75f * s && a > 0.f) + (a > 1.25f * s) + (a >= 1.75f * s && a > 0.f) +
                       (a > 2.5f * s) + (a >= 3.5f * s && a > 0.f) + (a > 5.f * s);
    d |= (c | (v[e] < 0.f ? 8u : 0u)) << (4 * e);
  }
  return d;
}
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float s, bf16) {
  const float up = s < 0x1p-60f ? 0x1p64f : 1.f;  // keeps the reciprocal of a tiny scale finite
  const float su = s * up, r = s > 0.f ? __builtin_amdgcn_rcpf(su) : 0.f;
  float t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float vu = v[e] * up, t0 = vu * r;
    t[e] = fmaf(fmaf(-t0, su, vu), r, t0);
  }
  uint32_t d = 0;
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[0], t[1], 1.0f, 0);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[2], t[3], 1.0f, 1);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[4], t[5], 1.0f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, t[6], t[7], 1.0f, 3);
}

// One 16 x 128 block per wavefront and turn: lane (q, i) reads the eight k of each dword, the four lanes of a row share each
// group's largest value. Magnitudes are compared as integers, which orders infinities and NaN above every number.
template <typename T>
__global__ __launch_bounds__(256) void q4_pack_kernel(int64_t blocks, int kb, int group, const T* __restrict__ w,
                                                      char* __restrict__ codes, bf16* __restrict__ scales) {
  constexpr int XC = 8 / EPC<T>::value;
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15, per = group / 32;  // dwords of a group
  const int64_t b = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (b >= blocks) return;
  const int64_t nb = b / kb;
  const int k0 = (int)(b - nb * kb);
  const T* src = w + ((nb * 16 + i) * kb + k0) * 128 + 8 * q;
  float v[4][8];
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int c = 0; c < XC; ++c)
      chunk_to_f<T>(ld_chunk_nt(src + 32 * s + c * EPC<T>::value), v[s] + c * EPC<T>::value);
  uint32_t top[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint32_t t = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(v[s][e]) & 0x7fffffffu);
    t = max(t, (uint32_t)__shfl_xor((int)t, 16, 64));
    top[s] = max(t, (uint32_t)__shfl_xor((int)t, 32, 64));
  }
  if (per >= 2) {
    top[0] = top[1] = max(top[0], top[1]);
    top[2] = top[3] = max(top[2], top[3]);
  }
  if (per == 4) top[0] = top[1] = top[2] = top[3] = max(top[0], top[2]);
  Chunk out;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    // a group with a NaN or an infinity: its scale, and with it every product, is NaN
    const bf16 sb = top[s] < 0x7f800000u ? f2bf(__uint_as_float(top[s]) * (1.f / 6.f)) : (bf16)0x7fc0;
    out.w[s] = codes_of(v[s], bf2f(sb), T{});
    if (q == 0 && s % per == 0) scales[((nb * kb + k0) * (4 / per) + s / per) * 16 + i] = sb;
  }
  st_chunk(codes + b * 1024 + lane * 16, out);
}

// Two codes, byte B of the dword, as bf16 numbers.
template <int B>
__device__ __forceinline__ uint32_t codes2(uint32_t d) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, B));
}
__device__ __forceinline__ Chunk codes8(uint32_t d) {
  Chunk c;
  c.w[0] = codes2<0>(d);
  c.w[1] = codes2<1>(d);
  c.w[2] = codes2<2>(d);
  c.w[3] = codes2<3>(d);
  return c;
}

template <typename T>
__global__ __launch_bounds__(256) void q4_unpack_kernel(int64_t blocks, int kb, int group, const char* __restrict__ codes,
                                                        const bf16* __restrict__ scales, T* __restrict__ w) {
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b >= blocks) return;
  const int64_t nb = b / kb;
  const int k0 = (int)(b - nb * kb), per = group / 32;
  const Chunk in = ld_chunk(codes + b * 1024 + lane * 16);
  T* dst = w + ((nb * 16 + i) * kb + k0) * 128 + 8 * q;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const float sc = bf2f(scales[((nb * kb + k0) * (4 / per) + s / per) * 16 + i]);
    float v[8];
    chunk_to_f<bf16>(codes8(in.w[s]), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= sc;
#pragma unroll
    for (int c = 0; c < 8 / EPC<T>::value; ++c)
      st_chunk(dst + 32 * s + c * EPC<T>::value, f_to_chunk<T>(v + c * EPC<T>::value));
  }
}

// ----------------------------------------------------------------------------------------------- experts

struct Q4Args {
  int T, f, d, Eloc, S, n_blocks;
  int walk;                // q4_short_kernel: column blocks of a workgroup
  int64_t shared0;         // T * k: first row of the shared experts in the row space
  const int32_t* offsets;  // [Eloc + 1]
  const void* x;           // [T, d]: rows of the shared experts
  const void* xp;          // [T * k, d]
  void* h;                 // H [R, f] ...
  int64_t h_low;           // ... of bf16 in two parts, the second this many bytes on
  void* y;                 // [R, d]
  const char* codes[2];    // gate, up; or down
  const bf16* scales[2];
};

// Inclusive sum over the lanes (DPP: shifts within rows of 16, then row broadcasts).
__device__ __forceinline__ int wave_scan(int v) {
#define PCMOE_DPP_ADD(ctrl, rows) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
  PCMOE_DPP_ADD(0x111, 0xf);  // row_shr 1, 2, 4, 8
  PCMOE_DPP_ADD(0x112, 0xf);
  PCMOE_DPP_ADD(0x114, 0xf);
  PCMOE_DPP_ADD(0x118, 0xf);
  PCMOE_DPP_ADD(0x142, 0xa);  // row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
  PCMOE_DPP_ADD(0x143, 0xc);
#undef PCMOE_DPP_ADD
  return v;
}

// Workgroup -> (group, chunk of its rows, column block), from the offsets alone. Lane l counts the chunks of groups l,
// l + 64, ... Consecutive tiles, the row chunks of one column block first, stay on one XCD, whose L2 serves a block's
// repeated reads.
struct Q4Tile {
  int g, row0, rows, ch, nb;
};
__device__ __forceinline__ bool q4_tile(const Q4Args& p, int bid, int chunk, Q4Tile& t) {
  constexpr int NS = 8;  // at most 511 groups
  const int G = p.Eloc + p.S, lane = threadIdx.x & 63, ns = (G + 63) >> 6;
  int lo[NS], n[NS], incl[NS], total = 0;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    lo[s] = n[s] = 0;
    if (s < ns) {
      const int g = 64 * s + lane;
      lo[s] = g < p.Eloc ? p.offsets[g] : 0;
      n[s] = g < p.Eloc ? p.offsets[g + 1] - lo[s] : g < G ? p.T : 0;
    }
  }
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    incl[s] = 0;
    if (s < ns) {
      incl[s] = wave_scan((n[s] + chunk - 1) / chunk) + total;
      total = __builtin_amdgcn_readlane(incl[s], 63);
    }
  }
  total *= p.n_blocks;
  const int x = bid & 7, lb = bid >> 3, qt = total >> 3, r = total & 7;
  if (lb >= qt + (x < r ? 1 : 0)) return false;
  const int L = x * qt + min(x, r) + lb;
  int before = 0;  // groups whose tiles all come before L
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < ns) before += __popcll(__ballot(incl[s] * p.n_blocks <= L));  // entries past G only repeat the total
  const int gl = before & 63;
  int first = 0, nch = 1;
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < ns && s == before >> 6) {
      t.g = before;
      t.row0 = __builtin_amdgcn_readlane(lo[s], gl);
      t.rows = __builtin_amdgcn_readlane(n[s], gl);
      nch = (t.rows + chunk - 1) / chunk;
      first = __builtin_amdgcn_readlane(incl[s], gl) - nch;
    }
  const int l = L - first * p.n_blocks;
  t.nb = __builtin_amdgcn_readfirstlane(l / nch);
  t.ch = __builtin_amdgcn_readfirstlane(l - t.nb * nch);
  return true;
}

// Eight activations as bf16 parts that add up to them, NP of them, and as they are loaded, XC chunks:
//   bf16 tensors: one part (B = 1) of x; two (B = 2) of H, which the gate/up kernel holds in fp32 and then stores as two bf16
//     arrays, its rounding and the rounding of the rest. Rounded to bf16 alone, H adds as much error to an output as the
//     output's own rounding (2.3e-3 in place of 1.7e-3 of the outputs' norm).
//   fp32 tensors: three parts, exact (truncated: 8 + 8 + 8 bits), made of two chunks. Infinities and NaN stay in the first.
template <typename T, int B>
struct Acts {
  static constexpr bool F32 = std::is_same<T, float>::value;
  static constexpr int NP = F32 ? 3 : B, XC = F32 ? 2 : B;
  Chunk c[XC];
  __device__ __forceinline__ void parts(Chunk (&out)[NP]) const {
    if constexpr (!F32) {
#pragma unroll
      for (int n = 0; n < NP; ++n) out[n] = c[n];
    } else {
#pragma unroll
      for (int p = 0; p < 4; ++p) {  // pairs of values
        uint32_t part[3][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t u = c[p / 2].w[2 * (p % 2) + e];
          const bool special = (u & 0x7f800000u) == 0x7f800000u;
          uint32_t hi = u & 0xffff0000u;
          if (special && (u & 0x7fffffu)) hi = 0x7fc00000u;
          const float r = special ? 0.f : __uint_as_float(u) - __uint_as_float(hi);
          const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
          part[0][e] = hi;
          part[1][e] = mid;
          part[2][e] = __float_as_uint(r - __uint_as_float(mid));
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) out[n].w[p] = (part[n][0] >> 16) | (part[n][1] & 0xffff0000u);
      }
    }
  }
};

// 16 or 2 bytes at byte voff + soff of a buffer, soff wave-uniform; zeros where voff is past the end.
__device__ __forceinline__ Chunk buf_ld16_at(__amdgpu_buffer_rsrc_t r, int voff, int soff) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(Chunk, __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0)));
}
__device__ __forceinline__ uint32_t buf_ld2_at(__amdgpu_buffer_rsrc_t r, int voff, int soff) {
  return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, voff, soff, 0);
}

// The scales of a block's 16 weight rows for the SG groups of a step. Lane (q, i) has read row i's scale of group q % SG;
// out[z] is row i's scale of group z in every lane.
template <int SG>
__device__ __forceinline__ void spread_scales(uint32_t v, float (&out)[SG]) {
  if constexpr (SG == 1) {
    out[0] = __uint_as_float(v << 16);
  } else {
    uint32_t lo = v << 16, hi = lo;  // rows of 16 lanes hold groups 0 1 0 1 or 0 1 2 3
    if constexpr (SG == 4) {
      const auto h = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);  // 0 1 0 1 and 2 3 2 3
      lo = h[0];
      hi = h[1];
    }
    const auto a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false);  // 0 0 0 0 and 1 1 1 1
    out[0] = __uint_as_float(a[0]);
    out[1] = __uint_as_float(a[1]);
    if constexpr (SG == 4) {
      const auto b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
      out[2] = __uint_as_float(b[0]);
      out[3] = __uint_as_float(b[1]);
    }
  }
}

__device__ __forceinline__ float silu_of(float g, bf16) { return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
__device__ __forceinline__ float silu_of(float g, float) { return g / (1.f + expf(-g)); }

// The second part of a bf16 H: the rest of its rounding; 0 where h rounds to an infinity (inf - inf makes products NaN).
__device__ __forceinline__ bf16 h_rest(float h) {
  const float rest = h - bf2f(f2bf(h));
  return fabsf(rest) < INFINITY ? f2bf(rest) : (bf16)0;
}

// Up to 16 rows of a group against 16 NB columns of the output (GU: of gate and of up): the KS wavefronts take a part of K
// each, 128 k at a time, read rows and weights straight into MFMA operands and share nothing until their sums meet in LDS
// and are added in wavefront order. SG = 128 / group. Bound by the round trips of the loads: a wavefront's steps are few, so
// the next one's loads, issued behind a step's products, are all that is in flight.
constexpr int KS = 8;
template <typename T, bool GU, int NB, int SG>
__global__ __launch_bounds__(64 * KS) void q4_split_kernel(Q4Args p) {
  typedef Acts<T, GU ? 1 : 2> X;
  constexpr int NM = GU ? 2 : 1, NP = X::NP, XC = X::XC, XB = sizeof(T);
  __shared__ __align__(16) floatx4 red[KS][NM * NB][64];
  Q4Tile t;
  if (!q4_tile(p, blockIdx.x, 16, t)) return;
  const int lane = threadIdx.x & 63, q = lane >> 4, li = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = GU ? p.d : p.f, N = GU ? p.f : p.d, units = K / 128, KB = K * XB;
  const bool routed = t.g < p.Eloc;
  const int64_t rs = routed ? (int64_t)t.row0 : p.shared0 + (int64_t)(t.g - p.Eloc) * p.T;
  const char* xb = GU ? (routed ? (const char*)p.xp + (int64_t)t.row0 * KB : (const char*)p.x) : (const char*)p.h + rs * KB;
  const int m0 = t.ch * 16, m_rows = min(t.rows - m0, 16);
  // rows past the last read as zeros; of bf16 H also the second array
  const __amdgpu_buffer_rsrc_t xr[2] = {buf_rsrc(xb + (int64_t)m0 * KB, (size_t)m_rows * KB),
                                        buf_rsrc(xb + (GU ? 0 : p.h_low) + (int64_t)m0 * KB, (size_t)m_rows * KB)};
  const int u0 = (int)((int64_t)units * w / KS), u1 = (int)((int64_t)units * (w + 1) / KS);
  const int nb0 = t.nb * NB;  // first 16-column block
  __amdgpu_buffer_rsrc_t cr[NM], sr[NM];
#pragma unroll
  for (int a = 0; a < NM; ++a) {
    const int64_t blk = ((int64_t)t.g * (N / 16) + nb0) * units;
    cr[a] = buf_rsrc(p.codes[a] + blk * 1024, (size_t)NB * units * 1024);
    sr[a] = buf_rsrc((const char*)p.scales[a] + blk * SG * 32, (size_t)NB * units * SG * 32);
  }
  struct Stage {
    Chunk c[NM][NB];
    uint32_t s[NM][NB];
    X x[4];
  } st;
  auto load = [&](int u) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int c = 0; c < XC; ++c)
        st.x[s].c[c] = buf_ld16_at(xr[X::F32 ? 0 : c], li * KB + (32 * s + 8 * q) * XB + (X::F32 ? 16 * c : 0), u * 128 * XB);
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int o = i * units + u;
        st.c[a][i] = buf_ld16_at(cr[a], lane * 16, o * 1024);
        st.s[a][i] = buf_ld2_at(sr[a], (q % SG) * 32 + 2 * li, o * SG * 32);
      }
  };
  floatx4 acc[NM][NB];
#pragma unroll
  for (int a = 0; a < NM; ++a)
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[a][i] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (u0 < u1) load(u0);
  for (int u = u0; u < u1; ++u) {
    Chunk xs[4][NP];
#pragma unroll
    for (int s = 0; s < 4; ++s) st.x[s].parts(xs[s]);
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        float sc[SG];
        spread_scales<SG>(st.s[a][i], sc);
#pragma unroll
        for (int z = 0; z < SG; ++z) {
          floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = z * 4 / SG; s < (z + 1) * 4 / SG; ++s) {
            const Chunk wv = codes8(st.c[a][i].w[s]);
#pragma unroll
            for (int n = 0; n < NP; ++n)
              sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xs[s][n]),
                                                            __builtin_bit_cast(bf16x8, wv), sum, 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[a][i][r] = fmaf(sc[z], sum[r], acc[a][i][r]);
        }
        asm volatile("" : "+v"(acc[a][i]));  // due here, as in q4_rows_kernel
      }
    __builtin_amdgcn_sched_barrier(0);
    if (u + 1 < u1) load(u + 1);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int a = 0; a < NM; ++a)
#pragma unroll
    for (int i = 0; i < NB; ++i) red[w][a * NB + i][lane] = acc[a][i];
  __syncthreads();
  if (w >= NB) return;
  floatx4 v[NM];  // rows 4 q .. 4 q + 3, column li of block w
#pragma unroll
  for (int a = 0; a < NM; ++a) {
    v[a] = red[0][a * NB + w][lane];
#pragma unroll
    for (int k = 1; k < KS; ++k) v[a] += red[k][a * NB + w][lane];
  }
  const int col = (nb0 + w) * 16 + li;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (4 * q + r >= m_rows) break;
    const int64_t row = rs + m0 + 4 * q + r;
    if constexpr (GU) {
      const float h = silu_of(v[0][r], T{}) * v[NM - 1][r];
      ((T*)p.h)[row * p.f + col] = from_f<T>(h);
      if constexpr (std::is_same<T, bf16>::value) ((bf16*)((char*)p.h + p.h_low))[row * p.f + col] = h_rest(h);
    } else {
      ((T*)p.y)[row * p.d + col] = from_f<T>(v[0][r]);
    }
  }
}

// Codes and scales of a wavefront's columns for one step of 128 k, and the step's products of ML row blocks. The rows lie in
// LDS as the NP parts that the MFMAs take, PLANE bytes each: 256 bytes a row, 16-byte chunk c of row r at c ^ (r & 15), so
// that the 16 rows of an operand read fall on different banks. A read runs while the products of the one before do.
template <int NM, int NF, int SG>
struct Q4Step {
  Chunk c[NM][NF];
  uint32_t s[NM][NF];
  // block i of 16 columns, step u: `blk` is i * units + u, `past` 0 or kBufPast (zeros)
  __device__ __forceinline__ void load(int a, int i, __amdgpu_buffer_rsrc_t cr, __amdgpu_buffer_rsrc_t sr, int blk, int past) {
    const int lane = threadIdx.x & 63;
    c[a][i] = buf_ld16_at(cr, lane * 16 | past, blk * 1024);
    s[a][i] = buf_ld2_at(sr, (((lane >> 4) % SG) * 32 + 2 * (lane & 15)) | past, blk * SG * 32);
  }
  template <int NP, int ML, int MT>
  __device__ __forceinline__ void mul(const char* xs, int plane, floatx4 (&acc)[NM][NF][MT]) const {
    const int lane = threadIdx.x & 63, q = lane >> 4, li = lane & 15;
    Chunk xf[2][ML][NP];
    auto read = [&](int k, Chunk (&f)[ML][NP]) {
#pragma unroll
      for (int m = 0; m < ML; ++m)
#pragma unroll
        for (int n = 0; n < NP; ++n) f[m][n] = ld_chunk(xs + n * plane + (16 * m + li) * 256 + (((4 * k + q) ^ li) << 4));
    };
    read(0, xf[0]);
    float sc[NM][NF][SG];
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NF; ++i) spread_scales<SG>(s[a][i], sc[a][i]);
    floatx4 sum[NM][NF][ML];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k < 3) read(k + 1, xf[(k + 1) & 1]);
      const int z = k * SG / 4;
#pragma unroll
      for (int a = 0; a < NM; ++a)
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          const Chunk wv = codes8(c[a][i].w[k]);
#pragma unroll
          for (int m = 0; m < ML; ++m) {
            if (k % (4 / SG) == 0) sum[a][i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NP; ++n)
              sum[a][i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xf[k & 1][m][n]),
                                                                     __builtin_bit_cast(bf16x8, wv), sum[a][i][m], 0, 0, 0);
          }
        }
      if ((k + 1) % (4 / SG) == 0) {
#pragma unroll
        for (int a = 0; a < NM; ++a)
#pragma unroll
          for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int m = 0; m < ML; ++m)
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[a][i][m][r] = fmaf(sc[a][i][z], sum[a][i][m][r], acc[a][i][m][r]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the sums are due here: left alone, the compiler moves the scaling past the next branch, with every product live
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int m = 0; m < ML; ++m) asm volatile("" : "+v"(acc[a][i][m]));
  }
};

// Item j of 256 of a step's rows: eight activations of row r, columns 8 c .. 8 c + 7, into LDS as above.
template <int NP, typename X>
__device__ __forceinline__ void put_acts(char* xs, int plane, int it, const X& x) {
  const int r = it >> 4;
  Chunk part[NP];
  x.parts(part);
#pragma unroll
  for (int n = 0; n < NP; ++n) st_chunk(xs + n * plane + r * 256 + (((it & 15) ^ (r & 15)) << 4), part[n]);
}

// Up to 16 MT rows of a group against 64 NF columns of the output: the four wavefronts split the columns (16 NF each; GU: of
// gate and of up) and share the rows, which pass through LDS 128 k at a time in two stages, as the bf16 parts that the MFMAs
// take. One barrier per step; the next steps' rows and codes are loaded while this one is multiplied.
template <typename T, bool GU, int MT, int NF, int SG, int D>
__global__ __launch_bounds__(256, 2) void q4_rows_kernel(Q4Args p) {
  static_assert(D % 2 == 0, "the steps of a round alternate between two LDS stages");
  typedef Acts<T, GU ? 1 : 2> X;
  constexpr int NM = GU ? 2 : 1, NP = X::NP, XC = X::XC, XB = sizeof(T), ROWS = 16 * MT;
  constexpr int PLANE = ROWS * 256;
  __shared__ __align__(16) char xs[2][NP * PLANE];
  Q4Tile t;
  if (!q4_tile(p, blockIdx.x, ROWS, t)) return;
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, li = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = GU ? p.d : p.f, N = GU ? p.f : p.d, units = K / 128, KB = K * XB;
  const bool routed = t.g < p.Eloc;
  const int64_t rs = routed ? (int64_t)t.row0 : p.shared0 + (int64_t)(t.g - p.Eloc) * p.T;
  const char* xb = GU ? (routed ? (const char*)p.xp + (int64_t)t.row0 * KB : (const char*)p.x) : (const char*)p.h + rs * KB;
  const int m0 = t.ch * ROWS, m_rows = min(t.rows - m0, ROWS);
  // rows past the last read as zeros; of bf16 H also the second array
  const __amdgpu_buffer_rsrc_t xr[2] = {buf_rsrc(xb + (int64_t)m0 * KB, (size_t)m_rows * KB),
                                        buf_rsrc(xb + (GU ? 0 : p.h_low) + (int64_t)m0 * KB, (size_t)m_rows * KB)};
  const int nb0 = (t.nb * 4 + w) * NF;  // the wavefront's first 16-column block
  __amdgpu_buffer_rsrc_t cr[NM], sr[NM];
#pragma unroll
  for (int a = 0; a < NM; ++a) {
    const int64_t blk = ((int64_t)t.g * (N / 16) + nb0) * units;
    cr[a] = buf_rsrc(p.codes[a] + blk * 1024, (size_t)NF * units * 1024);
    sr[a] = buf_rsrc((const char*)p.scales[a] + blk * SG * 32, (size_t)NF * units * SG * 32);
  }
  typedef Q4Step<NM, NF, SG> Weights;
  auto load_w = [&](int u, Weights& st) {  // steps past the end read zeros
    const int past = u < units ? 0 : kBufPast;
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NF; ++i) st.load(a, i, cr[a], sr[a], u < units ? i * units + u : 0, past);
  };
  // eight activations of row r, columns 8 c .. 8 c + 7 of the step: thread tid takes (r, c) = item tid + 256 j
  auto load_x = [&](int u, X (&x)[MT]) {
    const int so = u < units ? u * 128 * XB : 0;
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int it = tid + 256 * j;
#pragma unroll
      for (int c = 0; c < XC; ++c)
        x[j].c[c] = buf_ld16_at(xr[X::F32 ? 0 : c],
                                u < units ? (it >> 4) * KB + 8 * (it & 15) * XB + (X::F32 ? 16 * c : 0) : kBufPast, so);
    }
  };
  auto put_x = [&](int stage, const X (&x)[MT]) {
#pragma unroll
    for (int j = 0; j < MT; ++j) put_acts<NP>(xs[stage], PLANE, tid + 256 * j, x[j]);
  };
  floatx4 acc[NM][NF][MT];
#pragma unroll
  for (int a = 0; a < NM; ++a)
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[a][i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
  Weights wt[D];
  X xv[D][MT];
#pragma unroll
  for (int j = 0; j < D - 1; ++j) {
    load_x(j, xv[j]);
    load_w(j, wt[j]);
    __builtin_amdgcn_sched_barrier(0);
  }
  put_x(0, xv[0]);
  auto loop = [&](auto ml) {
    for (int u0 = 0; u0 < units; u0 += D) {
#pragma unroll
      for (int j = 0; j < D; ++j) {
        if (u0 + j >= units) break;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // stage j is filled, the other one was left
        load_x(u0 + j + D - 1, xv[(j + D - 1) % D]);
        load_w(u0 + j + D - 1, wt[(j + D - 1) % D]);
        __builtin_amdgcn_sched_barrier(0);
        wt[j].template mul<NP, decltype(ml)::value>(xs[j & 1], PLANE, acc);
        put_x((j + 1) & 1, xv[(j + 1) % D]);
      }
    }
  };
  // Row blocks past the chunk's rows are left out, in halves of the chunk, by a loop of its own (a branch inside one loop
  // has its sides' conversions hoisted, and spills).
  if (MT >= 2 && m_rows <= 8 * MT) loop(std::integral_constant<int, (MT + 1) / 2>{});
  else loop(std::integral_constant<int, MT>{});
  // Through LDS, so that the stores are 16 bytes a lane and whole rows of the workgroup's columns: a lane's own values are
  // four rows of one column (by themselves 771 x 128, f = 5888, 24 experts, top-8 takes 87 us of gate/up, most of it stores).
  constexpr int CB = 64 * NF * XB, PITCH = CB + 16;  // bytes of a row
  constexpr int PARTS = GU && !X::F32 ? 2 : 1;       // of H
  static_assert(PARTS * ROWS * PITCH <= (int)sizeof(xs), "the output tile");
  char* out = xs[0];
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = acc[0][i][m][r];
        if constexpr (GU) v = silu_of(v, T{}) * acc[NM - 1][i][m][r];
        T* o = reinterpret_cast<T*>(out + (16 * m + 4 * q + r) * PITCH + ((w * NF + i) * 16 + li) * XB);
        *o = from_f<T>(v);
        if constexpr (PARTS == 2) o[ROWS * PITCH / XB] = h_rest(v);
      }
  __syncthreads();
  constexpr int PER = CB / 16;  // 16-byte chunks of a row
#pragma unroll
  for (int n = 0; n < PARTS; ++n)
    for (int c = tid; c < ROWS * PER; c += 256) {
      const int r = c / PER, o = (c - r * PER) * 16;
      if (r >= m_rows) break;
      char* dst = GU ? (char*)p.h + n * p.h_low + (rs + m0 + r) * p.f * XB : (char*)p.y + (rs + m0 + r) * p.d * XB;
      st_chunk(dst + (int64_t)t.nb * CB + o, ld_chunk(out + (n * ROWS + r) * PITCH + o));
    }
}

// K of up to 256 (U = 1 or 2 steps): the group's rows stay in LDS and the four wavefronts, with 16 NF columns each, walk over
// p.walk blocks of 64 NF columns, the next block's weights loading meanwhile. Nothing is shared after the rows are there:
// each wavefront turns its outputs in LDS of its own. In q4_rows_kernel, whose workgroup ends after one block, finding the
// tile and waiting for the first loads were most of such a workgroup's time (771 tokens, d = 128, f = 5888, 24 experts, top-8:
// gate/up 70 us there, 50 here; with the second part of H 84 and 65).
template <typename T, bool GU, int MT, int NF, int SG, int U>
__global__ __launch_bounds__(256, 2) void q4_short_kernel(Q4Args p) {
  typedef Acts<T, GU ? 1 : 2> X;
  constexpr int NM = GU ? 2 : 1, NP = X::NP, XC = X::XC, XB = sizeof(T), ROWS = 16 * MT, PLANE = ROWS * 256;
  constexpr int CB = 16 * NF * XB, PITCH = CB + 16;  // bytes of a wavefront's output row
  constexpr int PARTS = GU && !X::F32 ? 2 : 1;       // of H
  __shared__ __align__(16) char xs[U][NP * PLANE];
  __shared__ __align__(16) char turn[4][PARTS * ROWS * PITCH];
  Q4Tile t;
  if (!q4_tile(p, blockIdx.x, ROWS, t)) return;
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, li = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int N = GU ? p.f : p.d, units = U, KB = U * 128 * XB;
  const bool routed = t.g < p.Eloc;
  const int64_t rs = routed ? (int64_t)t.row0 : p.shared0 + (int64_t)(t.g - p.Eloc) * p.T;
  const char* xb = GU ? (routed ? (const char*)p.xp + (int64_t)t.row0 * KB : (const char*)p.x) : (const char*)p.h + rs * KB;
  const int m0 = t.ch * ROWS, m_rows = min(t.rows - m0, ROWS);
  // rows past the last read as zeros; of bf16 H also the second array
  const __amdgpu_buffer_rsrc_t xr[2] = {buf_rsrc(xb + (int64_t)m0 * KB, (size_t)m_rows * KB),
                                        buf_rsrc(xb + (GU ? 0 : p.h_low) + (int64_t)m0 * KB, (size_t)m_rows * KB)};
  // column blocks b0 .. b1 of 64 NF columns
  const int b0 = t.nb * p.walk, b1 = min(b0 + p.walk, N / (64 * NF));
  typedef Q4Step<NM, NF, SG> Weights;
  __amdgpu_buffer_rsrc_t cr[NM], sr[NM];
#pragma unroll
  for (int a = 0; a < NM; ++a) {
    const int64_t blk = ((int64_t)t.g * (N / 16) + (b0 * 4 + w) * NF) * units;
    const size_t n = ((size_t)(b1 - b0 - 1) * 4 + 1) * NF * units;
    cr[a] = buf_rsrc(p.codes[a] + blk * 1024, n * 1024);
    sr[a] = buf_rsrc((const char*)p.scales[a] + blk * SG * 32, n * SG * 32);
  }
  auto load_w = [&](int b, Weights (&st)[U]) {
    const int past = b < b1 ? 0 : kBufPast;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int a = 0; a < NM; ++a)
#pragma unroll
        for (int i = 0; i < NF; ++i) st[u].load(a, i, cr[a], sr[a], b < b1 ? ((b - b0) * 4 * NF + i) * units + u : 0, past);
  };
  Weights wt[2][U];
  {
    X x[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        const int it = tid + 256 * j;
#pragma unroll
        for (int c = 0; c < XC; ++c)
          x[u][j].c[c] = buf_ld16_at(xr[X::F32 ? 0 : c], (it >> 4) * KB + 8 * (it & 15) * XB + (X::F32 ? 16 * c : 0), u * 128 * XB);
      }
    load_w(b0, wt[0]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < MT; ++j) put_acts<NP>(xs[u], PLANE, tid + 256 * j, x[u][j]);
  }
  __syncthreads();
  char* out = turn[w];
  for (int bb = b0; bb < b1; bb += 2) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int b = bb + j;
      if (b >= b1) break;
      load_w(b + 1, wt[j ^ 1]);
      __builtin_amdgcn_sched_barrier(0);
      floatx4 acc[NM][NF][MT];
#pragma unroll
      for (int a = 0; a < NM; ++a)
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[a][i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < U; ++u) wt[j][u].template mul<NP, MT>(xs[u], PLANE, acc);
      const int col = (b * 4 + w) * 16 * NF;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 16 * m + 4 * q + r;
            float v = acc[0][i][m][r];
            if constexpr (GU) v = silu_of(v, T{}) * acc[NM - 1][i][m][r];
            T* o = reinterpret_cast<T*>(out + row * PITCH + (16 * i + li) * XB);
            *o = from_f<T>(v);
            if constexpr (PARTS == 2) o[ROWS * PITCH / XB] = h_rest(v);
          }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      constexpr int PER = CB / 16;  // 16-byte chunks of a row
#pragma unroll
      for (int c = 0; c < PARTS * ROWS * PER / 64; ++c) {
        const int n = c / (ROWS * PER / 64), r = (c * 64 + lane) / PER - n * ROWS, o = (c * 64 + lane) % PER * 16;
        char* dst = GU ? (char*)p.h + n * p.h_low + (rs + m0 + r) * p.f * XB : (char*)p.y + (rs + m0 + r) * p.d * XB;
        if (r < m_rows) st_chunk(dst + (int64_t)col * XB + o, ld_chunk(out + (n * ROWS + r) * PITCH + o));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// ------------------------------------------------------------------------- host side

// Upper bound on the row chunks: each routed chunk holds at least one row, and all but one per group are full.
int64_t chunks_of(const moe_desc& d, int chunk) {
  const int64_t slots = (int64_t)d.T * d.top_k;
  return std::min(slots, (slots + (int64_t)d.local_count * (chunk - 1)) / chunk) +
         (int64_t)d.n_shared * ((d.T + chunk - 1) / chunk);
}

template <typename T, bool GU, int NB, int SG>
hipError_t q4_run_split(const moe_desc& d, Q4Args a, hipStream_t s) {
  a.n_blocks = (GU ? d.d_ff : d.d_model) / (16 * NB);
  const unsigned grid = (unsigned)((chunks_of(d, 16) * a.n_blocks + 7) / 8 * 8);
  KernelTimer kt(GU ? "q4_gate_up" : "q4_down", s);
  hipLaunchKernelGGL((q4_split_kernel<T, GU, NB, SG>), dim3(grid), dim3(64 * KS), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool GU, int MT, int NF, int SG, int D>
hipError_t q4_run_rows(const moe_desc& d, Q4Args a, hipStream_t s) {
  a.n_blocks = (GU ? d.d_ff : d.d_model) / (64 * NF);
  const unsigned grid = (unsigned)((chunks_of(d, 16 * MT) * a.n_blocks + 7) / 8 * 8);
  KernelTimer kt(GU ? "q4_gate_up" : "q4_down", s);
  hipLaunchKernelGGL((q4_rows_kernel<T, GU, MT, NF, SG, D>), dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool GU, int MT, int SG, int U>
hipError_t q4_run_short(const moe_desc& d, Q4Args a, hipStream_t s) {
  constexpr int NF = 2;
  const int blocks = (GU ? d.d_ff : d.d_model) / (64 * NF);
  // four workgroups per CU, as long as each has a block
  const int64_t chunks = chunks_of(d, 16 * MT);
  a.walk = (int)std::max<int64_t>(1, std::min<int64_t>(blocks, chunks * blocks / (4 * device_cus())));
  a.n_blocks = (blocks + a.walk - 1) / a.walk;
  const unsigned grid = (unsigned)((chunks * a.n_blocks + 7) / 8 * 8);
  KernelTimer kt(GU ? "q4_gate_up" : "q4_down", s);
  hipLaunchKernelGGL((q4_short_kernel<T, GU, MT, NF, SG, U>), dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Which kernel a projection takes, by the rows that an active expert can expect (the counts stay on the device; a shard's
// share of the slots, experts equally likely):
//   * K up to 256: the walking kernel, 16-row chunks up to 16 rows, 32-row chunks above;
//   * up to 12 rows where the shared-rows kernel would be bound by the chain of its steps (0.45 and 0.36 us each, gate/up
//     and down, and 2 us around them) rather than by reading the weights (5.5 TB/s), and K is long enough to split: K split
//     over 8 wavefronts. 64 columns to a workgroup from 280 workgroups of 32 on (gate/up: and more than 2 rows), which
//     share their reads of the rows; 32 below, and in the down projection 16 where there are less than 160 of 32;
//   * else shared rows. Gate/up: 16-row chunks up to 8 rows, 32-row chunks above. Down, whose K is the long one: 16-row
//     chunks of 64 columns with four steps in flight, or, where that leaves two workgroups per CU, of 128 columns with two.
// us of split 32 / split 64 / rows 16 / rows 32 (down: rows 16 / rows 16 x 128), group 64, at T, d, f, E, k, shared:
//   gate/up:  1, 2048, 1408, 64, 6, 2    9.9 / 10.0 / 12.0 / 13.1     down:  7.8 /  7.7 /  9.0 / 10.3
//             1, 4096, 14336, 8, 2      25.8 / 25.7 / 26.4 / 29.1           21.6 / 24.1 / 44.9 / 65.7
//             8, 1024, 2816, 16, 2      10.6 / 11.2 / 10.2 / 10.7            9.0 /  9.1 / 12.2 / 15.1
//             16, 2048, 1408, 64, 6, 2  35.2 / 35.4 / 34.5 / 40.7           35.0 / 28.4 / 23.6 / 20.8
//             16, 4096, 1408, 8, 2      15.3 / 14.0 / 18.2 / 19.7           13.6 / 10.3 / 10.5 / 10.5
//             24, 4096, 14336, 8, 2     91.5 / 88.2 / 86.8 / 88.2           91.3 / 63.8 / 59.2 / 72.0
//             48, 4096, 14336, 8, 2    105.2 / 92.4 / 94.0 / 92.5          127.4 / 92.4 / 75.6 / 79.0
//             64, 1024, 2816, 16, 2     16.1 / 15.1 / 12.9 / 13.1           13.8 / 11.3 / 12.5 / 15.0
//             128, 4096, 14336, 8, 2   188   / 145  / 135  / 124           269   / 162  / 122  / 104
//             400, 1024, 1408, 16, 2    23.8 / 19.5 / 14.3 / 14.0           27.0 / 18.4 / 13.6 / 12.4
//             777, 1024, 2816, 16, 2    65.1 / 56.0 / 34.3 / 31.1           72.7 / 46.3 / 32.0 / 27.9
//             1000, 4096, 4096, 8, 2   312   / 222  / 188  / 157           482   / 276  / 186  / 142
//             254, 128, 6912, 8, 4                                          31.3 / 21.8 / 21.8 / 28.9
// (32 rows x 128 columns of the down projection: 80.5, 84.1, 119, 16.0, 27.9, 140 us for 24, 48, 128,
// 400, 777 and 1000 tokens.) Split 16 / 32 / 64, down: 1, 640, 11392, 6, 6 11.7 / 14.7 / 18.1; 14, 128, 14208, 8, 4 22.9 / 24.1
// / 26.4; 4, 1024, 2816, 16, 2 8.9 / 7.8 / 8.7; 2, 4096, 4096, 8, 2 13.4 / 12.3 / 10.9; 1, 4096, 14336, 8, 2 30.5 / 21.6 / 24.1.
// Sixteen wavefronts were no faster than eight (23.1, 12.0, 10.8, 18.9 and 32.0 us for these with 16 columns).
// Walking / rows 32: gate/up 771, 128, 5888, 24, 8 65 / 84; 700, 256, 14336, 4, 2 49 / 49; walking / rows 16 x 128: down 451,
// 4096, 128, 256, 8, 2 31 / 51; 451, 4096, 256, 64, 8, 2 32 / 41.
// The second part of H is a second array written and read: with one part (2.3e-3 of the outputs' norm off in place of 1.7e-3)
// both projections of 24, 4096, 14336, 8, 2 took 134 us in place of 146, of 777, 1024, 2816, 16, 2 51 in place of 59, of 771,
// 128, 5888, 24, 8 the gate/up 50 in place of 65.
// Measured and not kept: 32- / 64- / 128-row chunks of gate/up (groups of 32: 777, 1024, 2816, 16, 2 37.2 / 38.3 / 43.2, 1000,
// 4096, 4096, 8, 2 188 / 178 / 211; groups of 64: the first 32.6 / 38.4 / 84.2), and, with H in one part, four wavefronts of a
// split, deeper prefetch in the split, non-temporal loads of the codes (equal, and worse where calls follow each other), the walking
// kernel for K of up to 1024 with a chunk's rows held in LDS whole (rows 32 / walking, gate/up: 777, 1024, 2816, 16, 2 37.7 /
// 39.6; 1500, 1024, 4096, 8, 2 83.9 / 81.3; 777, 512, 2048, 32, 4 29.7 / 25.8; down 777, 2048, 768, 64, 6 32.8 / 36.5), four
// steps in flight of 32-row chunks (gate/up of the first 49.5 against 38.7), a group's scalings among the next one's products
// (equal). So neither waits nor their order bind many rows, but the instructions: an MFMA takes 18 cycles of a SIMD, its 4
// scalings (groups of 32) 18, both together 27 to 29.
struct Q4Pick {
  double active, rows;  // experts with a row, and their rows
  int units;    // steps of 128 k
  bool split;   // K over the wavefronts
};
Q4Pick q4_rule(const moe_desc& d, int group, bool gate_up) {
  const double share = (double)d.top_k / d.n_experts;
  const double active = d.local_count * (1 - std::pow(1 - share, d.T)) + d.n_shared;
  const double rows = d.T * (share * d.local_count + d.n_shared) / active;
  const int units = (gate_up ? d.d_model : d.d_ff) / 128;
  const double bytes = active * (gate_up ? 2 : 1) * d.d_ff * d.d_model * (0.5 + 2.0 / group);
  const double chain = 2 + (gate_up ? 0.45 : 0.36) * units;
  const bool split = units >= 6 && rows <= 12 && chain > bytes / 5.5e6;
  return {active, rows, units, split};
}

template <typename T, bool GU, int SG>
hipError_t q4_pick(const moe_desc& d, const Q4Args& a, hipStream_t s) {
  const Q4Pick k = q4_rule(d, 128 / SG, GU);
  if (k.units == 1) return k.rows <= 16 ? q4_run_short<T, GU, 1, SG, 1>(d, a, s) : q4_run_short<T, GU, 2, SG, 1>(d, a, s);
  if (k.units == 2) return k.rows <= 16 ? q4_run_short<T, GU, 1, SG, 2>(d, a, s) : q4_run_short<T, GU, 2, SG, 2>(d, a, s);
  if (k.split) {
    const double wgs = k.active * ((GU ? d.d_ff : d.d_model) / 32);
    if (!GU && wgs < 160) return q4_run_split<T, false, 1, SG>(d, a, s);
    return wgs < 280 || (GU && k.rows <= 2) ? q4_run_split<T, GU, 2, SG>(d, a, s) : q4_run_split<T, GU, 4, SG>(d, a, s);
  }
  if constexpr (GU) {
    return k.rows <= 8 ? q4_run_rows<T, GU, 1, 1, SG, 2>(d, a, s) : q4_run_rows<T, GU, 2, 1, SG, 2>(d, a, s);
  } else {
    const bool wide = chunks_of(d, 16) * (d.d_model / 128) >= 2 * device_cus();
    return wide ? q4_run_rows<T, GU, 1, 2, SG, 2>(d, a, s) : q4_run_rows<T, GU, 1, 1, SG, 4>(d, a, s);
  }
}

template <typename T, int SG>
hipError_t q4_both(const moe_desc& d, Q4Args a, const Q4Weights& gate, const Q4Weights& up, const Q4Weights& down,
                   hipStream_t s) {
  a.codes[0] = (const char*)gate.codes;
  a.codes[1] = (const char*)up.codes;
  a.scales[0] = (const bf16*)gate.scales;
  a.scales[1] = (const bf16*)up.scales;
  if (hipError_t e = q4_pick<T, true, SG>(d, a, s); e != hipSuccess) return e;
  a.codes[0] = a.codes[1] = (const char*)down.codes;
  a.scales[0] = a.scales[1] = (const bf16*)down.scales;
  return q4_pick<T, false, SG>(d, a, s);
}

template <typename T>
hipError_t q4_ffn(const moe_desc& d, int group, const Q4Args& a, const Q4Weights& gate, const Q4Weights& up,
                  const Q4Weights& down, hipStream_t s) {
  if (group == 32) return q4_both<T, 4>(d, a, gate, up, down, s);
  if (group == 64) return q4_both<T, 2>(d, a, gate, up, down, s);
  return q4_both<T, 1>(d, a, gate, up, down, s);
}

}  // namespace

// H, of bf16 in two arrays
static size_t h_bytes(const moe_desc& d) { return align256((size_t)rows_total(d) * d.d_ff * elem_bytes(d)); }
size_t ffn_q4_ws_bytes(const moe_desc& d) { return h_bytes(d) * (d.dtype == MOE_BF16 ? 2 : 1); }

hipError_t launch_ffn_q4(const moe_desc& d, int group, const void* x, const void* xp, const int32_t* offsets,
                         const Q4Weights& gate, const Q4Weights& up, const Q4Weights& down, void* yp, void* ws,
                         hipStream_t s) {
  Q4Args a{};
  a.T = d.T;
  a.f = d.d_ff;
  a.d = d.d_model;
  a.Eloc = d.local_count;
  a.S = d.n_shared;
  a.shared0 = (int64_t)d.T * d.top_k;
  a.offsets = offsets;
  a.x = x;
  a.xp = xp;
  a.h = ws;
  a.h_low = d.dtype == MOE_BF16 ? (int64_t)h_bytes(d) : 0;
  a.y = yp;
  if (d.dtype == MOE_BF16) return q4_ffn<bf16>(d, group, a, gate, up, down, s);
  return q4_ffn<float>(d, group, a, gate, up, down, s);
}

hipError_t launch_q4_pack(int n, int rows, int cols, int group, int dtype, const void* w, void* codes, void* scales,
                          hipStream_t s) {
  const int64_t blocks = (int64_t)n * (rows / 16) * (cols / 128);
  const dim3 grid((unsigned)((blocks + 3) / 4));
  KernelTimer kt("q4_pack", s);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(q4_pack_kernel<bf16>, grid, dim3(256), 0, s, blocks, cols / 128, group, (const bf16*)w,
                       (char*)codes, (bf16*)scales);
  else
    hipLaunchKernelGGL(q4_pack_kernel<float>, grid, dim3(256), 0, s, blocks, cols / 128, group, (const float*)w,
                       (char*)codes, (bf16*)scales);
  return hipGetLastError();
}

hipError_t launch_q4_unpack(int n, int rows, int cols, int group, int dtype, const void* codes, const void* scales,
                            void* w, hipStream_t s) {
  const int64_t blocks = (int64_t)n * (rows / 16) * (cols / 128);
  const dim3 grid((unsigned)((blocks + 3) / 4));
  KernelTimer kt("q4_unpack", s);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(q4_unpack_kernel<bf16>, grid, dim3(256), 0, s, blocks, cols / 128, group, (const char*)codes,
                       (const bf16*)scales, (bf16*)w);
  else
    hipLaunchKernelGGL(q4_unpack_kernel<float>, grid, dim3(256), 0, s, blocks, cols / 128, group, (const char*)codes,
                       (const bf16*)scales, (float*)w);
  return hipGetLastError();
}

}  // namespace pcmoe
