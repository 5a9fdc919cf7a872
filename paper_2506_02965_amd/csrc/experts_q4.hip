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

namespace pcmoe {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ----------------------------------------------------------------------------------------------- packing

// Code of a value with |value| = a in units of its scale s: nearest of the eight magnitudes, ties to the even code. The
// midpoints times s are exact in fp32, so the comparisons decide on the quotient itself.
__device__ __forceinline__ uint32_t e2m1(float v, float s) {
  const float a = fabsf(v);
  uint32_t c = (a > 0.25f * s) + (a >= 0.75f * s && a > 0.f) + (a > 1.25f * s) + (a >= 1.75f * s && a > 0.f) +
               (a > 2.5f * s) + (a >= 3.5f * s && a > 0.f) + (a > 5.f * s);
  return c | (v < 0.f ? 8u : 0u);
}

// One wavefront per 16 x 128 block: lane (q, i) reads the eight k of each dword, the four lanes of a row share each
// group's largest value.
template <typename T>
__global__ __launch_bounds__(256) void q4_pack_kernel(int64_t blocks, int kb, int group, const T* __restrict__ w,
                                                      char* __restrict__ codes, bf16* __restrict__ scales) {
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b >= blocks) return;
  const int64_t nb = b / kb;
  const int k0 = (int)(b - nb * kb);
  const T* src = w + ((nb * 16 + i) * kb + k0) * 128 + 8 * q;
  float v[4][8];
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int c = 0; c < 8 / EPC<T>::value; ++c)
      chunk_to_f<T>(ld_chunk(src + 32 * s + c * EPC<T>::value), v[s] + c * EPC<T>::value);
  float top[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    float t = 0.f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t = fmaxf(t, fabsf(v[s][e]));
      bad |= !(fabsf(v[s][e]) < INFINITY);
    }
    if (bad) t = INFINITY;
    t = fmaxf(t, __shfl_xor(t, 16, 64));
    top[s] = fmaxf(t, __shfl_xor(t, 32, 64));
  }
  const int per = group / 32;  // dwords of a group
  if (per >= 2) {
    top[0] = top[1] = fmaxf(top[0], top[1]);
    top[2] = top[3] = fmaxf(top[2], top[3]);
  }
  if (per == 4) top[0] = top[1] = top[2] = top[3] = fmaxf(top[0], top[2]);
  Chunk out;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    // a group with a NaN or an infinity: its scale, and with it every product, is NaN
    const bf16 sb = top[s] < INFINITY ? f2bf(top[s] / 6.f) : (bf16)0x7fc0;
    const float sc = bf2f(sb);
    uint32_t d = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) d |= e2m1(v[s][e], sc) << (4 * e);
    out.w[s] = d;
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
  int64_t shared0;         // T * k: first row of the shared experts in the row space
  const int32_t* offsets;  // [Eloc + 1]
  const void* x;           // [T, d]: rows of the shared experts
  const void* xp;          // [T * k, d]
  void* h;                 // [R, f]
  void* y;                 // [R, d]
  const char* codes[2];    // gate, up; or down
  const bf16* scales[2];
};

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
      int v = (n[s] + chunk - 1) / chunk;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
      }
      incl[s] = v + total;
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

// The bf16 parts of eight activations: the numbers themselves, or three bf16 that add up to each fp32 number (truncated:
// 8 + 8 + 8 bits). Infinities and NaN stay in the first part.
template <typename T> struct Parts;
template <> struct Parts<bf16> { static constexpr int N = 1; };
template <> struct Parts<float> { static constexpr int N = 3; };
template <typename T>
struct XChunk {
  Chunk c[8 / EPC<T>::value];
};
__device__ __forceinline__ void split(const XChunk<bf16>& x, Chunk (&out)[1]) { out[0] = x.c[0]; }
__device__ __forceinline__ void split(const XChunk<float>& x, Chunk (&out)[3]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {  // pairs of values
    uint32_t part[3][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t u = x.c[p / 2].w[2 * (p % 2) + e];
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

__device__ __forceinline__ float silu_of(float g, bf16) { return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)); }
__device__ __forceinline__ float silu_of(float g, float) { return g / (1.f + expf(-g)); }

template <typename T>
__device__ __forceinline__ void store4(T* p, const floatx4& v) {
  if constexpr (std::is_same<T, bf16>::value)
    *reinterpret_cast<uint2*>(p) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else
    *reinterpret_cast<floatx4*>(p) = v;
}

// Up to 16 MT rows of a group against 16 NB columns of the output (GU: of gate and of up). The four wavefronts take a
// quarter of K each, 128 k at a time with D steps of loads in flight; their sums meet in LDS and are added in wavefront
// order. SG = 128 / group.
constexpr int Q4_W = 4;
template <typename T, bool GU, int MT, int NB, int SG, int D>
__global__ __launch_bounds__(64 * Q4_W) void q4_split_kernel(Q4Args p) {
  constexpr int NM = GU ? 2 : 1, NP = Parts<T>::N, XC = 8 / EPC<T>::value;
  __shared__ __align__(16) floatx4 red[Q4_W][NM * NB * MT][64];
  Q4Tile t;
  if (!q4_tile(p, blockIdx.x, 16 * MT, t)) return;
  const int lane = threadIdx.x & 63, q = lane >> 4, li = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = GU ? p.d : p.f, N = GU ? p.f : p.d, units = K / 128, KB = K * (int)sizeof(T);
  const bool routed = t.g < p.Eloc;
  const int64_t rs = routed ? (int64_t)t.row0 : p.shared0 + (int64_t)(t.g - p.Eloc) * p.T;
  const char* xb = GU ? (routed ? (const char*)p.xp + (int64_t)t.row0 * KB : (const char*)p.x) : (const char*)p.h + rs * KB;
  const int m0 = t.ch * 16 * MT, m_rows = min(t.rows - m0, 16 * MT);
  const auto xr = buf_rsrc(xb + (int64_t)m0 * KB, (size_t)m_rows * KB);
  const int u0 = (int)((int64_t)units * w / Q4_W), u1 = (int)((int64_t)units * (w + 1) / Q4_W);
  const int nb0 = t.nb * NB;  // first 16-column block
  const char* cb[NM];
  const char* sb[NM];
#pragma unroll
  for (int a = 0; a < NM; ++a) {
    const int64_t blk = ((int64_t)t.g * (N / 16) + nb0) * units;
    cb[a] = p.codes[a] + blk * 1024 + lane * 16;
    sb[a] = (const char*)p.scales[a] + blk * SG * 32 + q * 8;
  }
  struct Stage {
    Chunk c[NM][NB];
    uint2 s[NM][NB][SG];
    XChunk<T> x[4][MT];
  };
  auto load = [&](int u, Stage& st) {
    if (u >= u1) return;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int c = 0; c < XC; ++c)
          st.x[s][m].c[c] = buf_ld16(xr, (16 * m + li) * KB + (u * 128 + 32 * s + 8 * q) * (int)sizeof(T) + 16 * c);
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int64_t o = (int64_t)i * units + u;
        st.c[a][i] = ld_chunk(cb[a] + o * 1024);
#pragma unroll
        for (int z = 0; z < SG; ++z) st.s[a][i][z] = *reinterpret_cast<const uint2*>(sb[a] + (o * SG + z) * 32);
      }
  };
  floatx4 acc[NM][NB][MT];
#pragma unroll
  for (int a = 0; a < NM; ++a)
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[a][i][m] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto mul = [&](const Stage& st) {
    Chunk xs[4][MT][NP];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int m = 0; m < MT; ++m) split(st.x[s][m], xs[s][m]);
#pragma unroll
    for (int a = 0; a < NM; ++a)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int z = 0; z < SG; ++z) {
          floatx4 sum[MT];
#pragma unroll
          for (int m = 0; m < MT; ++m) sum[m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = z * 4 / SG; s < (z + 1) * 4 / SG; ++s) {
            const Chunk wv = codes8(st.c[a][i].w[s]);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int n = 0; n < NP; ++n)
                sum[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv),
                                                                 __builtin_bit_cast(bf16x8, xs[s][m][n]), sum[m], 0, 0, 0);
          }
          const uint2 sv = st.s[a][i][z];
          const floatx4 sc = {__uint_as_float(sv.x << 16), __uint_as_float(sv.x & 0xffff0000u),
                              __uint_as_float(sv.y << 16), __uint_as_float(sv.y & 0xffff0000u)};
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[a][i][m][r] = fmaf(sc[r], sum[m][r], acc[a][i][m][r]);
        }
  };
  Stage st[D];
#pragma unroll
  for (int j = 0; j < D; ++j) load(u0 + j, st[j]);
  for (int u = u0; u < u1; u += D) {
#pragma unroll
    for (int j = 0; j < D; ++j)
      if (u + j < u1) {
        mul(st[j]);
        load(u + j + D, st[j]);
      }
  }
#pragma unroll
  for (int a = 0; a < NM; ++a)
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int m = 0; m < MT; ++m) red[w][(a * NB + i) * MT + m][lane] = acc[a][i][m];
  __syncthreads();
  for (int it = w; it < NB * MT; it += Q4_W) {
    const int i = it / MT, m = it - i * MT;
    if (16 * m + li >= m_rows) continue;
    floatx4 v[NM];
#pragma unroll
    for (int a = 0; a < NM; ++a) {
      v[a] = red[0][a * NB * MT + it][lane];
#pragma unroll
      for (int k = 1; k < Q4_W; ++k) v[a] += red[k][a * NB * MT + it][lane];
    }
    const int64_t row = rs + m0 + 16 * m + li;
    const int col = (nb0 + i) * 16 + 4 * q;
    if constexpr (GU) {
      floatx4 h;
#pragma unroll
      for (int r = 0; r < 4; ++r) h[r] = silu_of(v[0][r], T{}) * v[NM - 1][r];
      store4((T*)p.h + row * p.f + col, h);
    } else {
      store4((T*)p.y + row * p.d + col, v[0]);
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

template <typename T, bool GU, int MT, int NB, int SG, int D>
hipError_t q4_run(const moe_desc& d, Q4Args a, hipStream_t s) {
  a.n_blocks = (GU ? d.d_ff : d.d_model) / (16 * NB);
  const unsigned grid = (unsigned)((chunks_of(d, 16 * MT) * a.n_blocks + 7) / 8 * 8);
  KernelTimer kt(GU ? "q4_gate_up" : "q4_down", s);
  hipLaunchKernelGGL((q4_split_kernel<T, GU, MT, NB, SG, D>), dim3(grid), dim3(64 * Q4_W), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool GU, int SG>
hipError_t q4_pick(const moe_desc& d, const Q4Args& a, hipStream_t s) {
  const int64_t groups = std::min<int64_t>((int64_t)d.T * d.top_k, d.local_count) + d.n_shared;
  const int64_t rows = rows_total(d) / std::max<int64_t>(1, groups);
  if (rows <= 16) return q4_run<T, GU, 1, 2, SG, 2>(d, a, s);
  return q4_run<T, GU, 2, 2, SG, 1>(d, a, s);
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

size_t ffn_q4_ws_bytes(const moe_desc& d) { return align256((size_t)rows_total(d) * d.d_ff * elem_bytes(d)); }

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
