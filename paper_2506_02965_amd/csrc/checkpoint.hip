// Activations that the expert forward saves for its backward, kept in 8 bits between the two.
//
// A block of 32 consecutive columns of a row of G|U shares one power of two 2^e, the smallest with max|v| <= 127 2^e, and
// a value is kept as the integer rint(v / 2^e): at most 2^(e-1) off, and the value that it stands for, code * 2^e, is a
// bf16 number (at most 7 significant bits), so reading a checkpoint rounds nothing. (-126 <= e <= 121: the largest finite
// numbers are kept as 127 * 2^121, since 64 * 2^122 would be an infinity.) H is not kept; it is formed again as
// silu(G) U from the values kept, so that the backward uses one consistent point.
// Checkpoint: codes [R, 2f] int8, then exponents [R, 2f / 32] (e + 127), then the forward's tile plan as it is.
#include "expert_ops.h"

#include <algorithm>

namespace pcmoe {

namespace {

constexpr int QB = 32;         // columns of a block
constexpr int CK_THREADS = 256;
// 16-byte chunks in flight per thread. Both kernels are bound by the memory (T = 8192, f = 14,336, 2 slots: 1.4 GB in 297 us
// and 1.9 GB in 323 us in turn, 4.8 and 5.9 TB/s; the first 249 us at best). What they read is read for the last time until its buffer is written again, so it is read
// non-temporally (34 and 16 us less). us of both at 1 / 2 / 4 / 8 chunks: 654 / 567 / 595 / 608.
constexpr int CK_UNROLL = 2;

struct CkptArgs {
  int64_t units;         // work items of 16 saved bytes
  int per_row;           // ... of a row
  int64_t shared0;       // first row of the shared experts, T * k
  const int32_t* n_loc;  // rows of the hosted experts
  int f;
  char* saved;           // G|U, H, plan
  char* codes;
  uint8_t* exps;
  int64_t h_off;         // H within saved
  int64_t plan_off;      // the plan within saved ...
  char* plan;            // ... and within the checkpoint
  int plan_chunks;       // its 16-byte chunks
};

// Lane exchange within groups of 4 (DPP) and 8.
__device__ __forceinline__ float xor_max(float v, int lanes) {
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0xb1, 0xf, 0xf, true)));
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x4e, 0xf, 0xf, true)));
  if (lanes == 8) v = fmaxf(v, __shfl_xor(v, 4, 64));
  return v;
}

__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// The items of a workgroup: CK_UNROLL x 256 consecutive ones. f(unit index within the row, row).
template <typename F>
__device__ __forceinline__ void ckpt_items(const CkptArgs& a, F&& f) {
  const int64_t base = (int64_t)blockIdx.x * (CK_THREADS * CK_UNROLL);
  const int64_t row0 = base / a.per_row;  // uniform
  const unsigned c0 = (unsigned)(base - row0 * a.per_row) + threadIdx.x;
#pragma unroll
  for (int i = 0; i < CK_UNROLL; ++i) {
    const unsigned c = c0 + i * CK_THREADS, r = c / (unsigned)a.per_row;
    f(i, row0 + r, (int)(c - r * a.per_row), base + threadIdx.x + i * CK_THREADS < a.units);
  }
}

template <typename T>
__global__ __launch_bounds__(CK_THREADS) void ckpt_pack_kernel(CkptArgs a, int blocks) {
  constexpr int EP = EPC<T>::value, LANES = QB / EP;
  if ((int)blockIdx.x >= blocks) {
    for (int i = threadIdx.x; i < a.plan_chunks; i += CK_THREADS)
      st_chunk(a.plan + 16 * (size_t)i, ld_chunk(a.saved + a.plan_off + 16 * (size_t)i));
    return;
  }
  const int64_t n_loc = *a.n_loc;
  Chunk v[CK_UNROLL];
  int64_t at[CK_UNROLL];  // first element of the item; -1: none
  ckpt_items(a, [&](int i, int64_t row, int u, bool in) {
    at[i] = in && (row < n_loc || row >= a.shared0) ? row * 2 * a.f + (int64_t)u * EP : -1;
    v[i] = at[i] >= 0 ? ld_chunk_nt(a.saved + at[i] * sizeof(T)) : zero_chunk();
  });
#pragma unroll
  for (int i = 0; i < CK_UNROLL; ++i) {
    float x[EP];
    chunk_to_f<T>(v[i], x);
    float top = 0.f;
#pragma unroll
    for (int s = 0; s < EP; ++s) top = fmaxf(top, is_finite(x[s]) ? fabsf(x[s]) : 0.f);
    top = xor_max(top, LANES);
    // biased exponent of 2^e: 127 = 1.984375 * 2^6, whose mantissa bits are 0x7e0000
    const int eb = min(max((int)((__float_as_uint(top) + 0x1ffffu) >> 23) - 6, 1), 127 + 121);
    const float inv = __uint_as_float((uint32_t)(254 - eb) << 23);
    uint32_t w[EP / 4];
#pragma unroll
    for (int s = 0; s < EP; ++s) {
      // -128 stands for NaN
      const int q = is_finite(x[s]) ? (int)__builtin_amdgcn_fmed3f(rintf(x[s] * inv), -127.f, 127.f) : -128;
      if (s % 4 == 0) w[s / 4] = 0;
      w[s / 4] |= (uint32_t)(q & 255) << (8 * (s % 4));
    }
    if (at[i] < 0) continue;
    if constexpr (EP == 8) *reinterpret_cast<uint2*>(a.codes + at[i]) = uint2{w[0], w[1]};
    else *reinterpret_cast<uint32_t*>(a.codes + at[i]) = w[0];
    if (threadIdx.x % LANES == 0) a.exps[at[i] / QB] = (uint8_t)eb;
  }
}

// silu(g) u of a backward's saved H, to the accuracy of its type.
template <typename T> __device__ __forceinline__ float swiglu(float g, float u);
template <> __device__ __forceinline__ float swiglu<bf16>(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * u;
}
template <> __device__ __forceinline__ float swiglu<float>(float g, float u) { return g / (1.f + expf(-g)) * u; }

template <typename T>
__global__ __launch_bounds__(CK_THREADS) void ckpt_unpack_kernel(CkptArgs a, int blocks) {
  constexpr int EP = EPC<T>::value;
  if ((int)blockIdx.x >= blocks) {
    for (int i = threadIdx.x; i < a.plan_chunks; i += CK_THREADS)
      st_chunk(a.saved + a.plan_off + 16 * (size_t)i, ld_chunk(a.plan + 16 * (size_t)i));
    return;
  }
  const int64_t n_loc = *a.n_loc;
  uint32_t w[CK_UNROLL][2][EP / 4];
  int eb[CK_UNROLL][2];
  int64_t row[CK_UNROLL];
  int col[CK_UNROLL];
  ckpt_items(a, [&](int i, int64_t r, int u, bool in) {
    row[i] = in && (r < n_loc || r >= a.shared0) ? r : -1;
    col[i] = u * EP;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      eb[i][p] = 127;
#pragma unroll
      for (int s = 0; s < EP / 4; ++s) w[i][p][s] = 0;
      if (row[i] < 0) continue;
      const int64_t e = r * 2 * a.f + (int64_t)p * a.f + col[i];
      if constexpr (EP == 8) {
        const uint64_t t = __builtin_nontemporal_load(reinterpret_cast<const uint64_t*>(a.codes + e));
        w[i][p][0] = (uint32_t)t;
        w[i][p][1] = (uint32_t)(t >> 32);
      } else {
        w[i][p][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(a.codes + e));
      }
      eb[i][p] = a.exps[e / QB];
    }
  });
#pragma unroll
  for (int i = 0; i < CK_UNROLL; ++i) {
    if (row[i] < 0) continue;
    float x[2][EP], h[EP];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float step = __uint_as_float((uint32_t)eb[i][p] << 23);
#pragma unroll
      for (int s = 0; s < EP; ++s) {
        const int q = (int)(int8_t)(w[i][p][s / 4] >> (8 * (s % 4)));
        x[p][s] = q == -128 ? __uint_as_float(0x7fc00000u) : (float)q * step;
      }
    }
#pragma unroll
    for (int s = 0; s < EP; ++s) h[s] = swiglu<T>(x[0][s], x[1][s]);
    char* gu = a.saved + (row[i] * 2 * a.f + col[i]) * sizeof(T);
    st_chunk(gu, f_to_chunk<T>(x[0]));
    st_chunk(gu + (size_t)a.f * sizeof(T), f_to_chunk<T>(x[1]));
    st_chunk(a.saved + a.h_off + (row[i] * a.f + col[i]) * sizeof(T), f_to_chunk<T>(h));
  }
}

size_t gu_bytes(const moe_desc& d) { return align256((size_t)rows_total(d) * 2 * d.d_ff * elem_bytes(d)); }
size_t plan_off(const moe_desc& d) { return gu_bytes(d) + align256((size_t)rows_total(d) * d.d_ff * elem_bytes(d)); }
size_t codes_bytes(const moe_desc& d) { return align256((size_t)rows_total(d) * 2 * d.d_ff); }
size_t exps_bytes(const moe_desc& d) { return align256((size_t)rows_total(d) * 2 * d.d_ff / QB); }

CkptArgs ckpt_args(const moe_desc& d, const int32_t* offsets, void* saved, void* ckpt) {
  CkptArgs a{};
  a.shared0 = (int64_t)d.T * d.top_k;
  a.n_loc = offsets + d.local_count;
  a.f = d.d_ff;
  a.saved = (char*)saved;
  a.codes = (char*)ckpt;
  a.exps = (uint8_t*)ckpt + codes_bytes(d);
  a.h_off = (int64_t)gu_bytes(d);
  a.plan_off = (int64_t)plan_off(d);
  a.plan = (char*)ckpt + codes_bytes(d) + exps_bytes(d);
  a.plan_chunks = (int)((ffn_saved_bytes(d) - plan_off(d)) / 16);
  return a;
}

template <typename K>
hipError_t ckpt_run(const char* name, K kern, const moe_desc& d, CkptArgs a, int cols, hipStream_t s) {
  a.per_row = cols * (int)elem_bytes(d) / 16;
  a.units = rows_total(d) * a.per_row;
  const int64_t blocks = (a.units + CK_THREADS * CK_UNROLL - 1) / (CK_THREADS * CK_UNROLL);
  KernelTimer kt(name, s);
  hipLaunchKernelGGL(kern, dim3((unsigned)blocks + 1), dim3(CK_THREADS), 0, s, a, (int)blocks);
  return hipGetLastError();
}

}  // namespace

size_t ffn_ckpt_bytes(const moe_desc& d) {
  return codes_bytes(d) + exps_bytes(d) + (ffn_saved_bytes(d) - plan_off(d));
}

hipError_t launch_ffn_checkpoint(const moe_desc& d, const int32_t* offsets, const void* saved, void* ckpt,
                                 hipStream_t s) {
  const CkptArgs a = ckpt_args(d, offsets, const_cast<void*>(saved), ckpt);
  if (d.dtype == MOE_BF16) return ckpt_run("ffn_checkpoint", ckpt_pack_kernel<bf16>, d, a, 2 * d.d_ff, s);
  return ckpt_run("ffn_checkpoint", ckpt_pack_kernel<float>, d, a, 2 * d.d_ff, s);
}

hipError_t launch_ffn_restore(const moe_desc& d, const int32_t* offsets, const void* ckpt, void* saved, hipStream_t s) {
  const CkptArgs a = ckpt_args(d, offsets, saved, const_cast<void*>(ckpt));
  if (d.dtype == MOE_BF16) return ckpt_run("ffn_restore", ckpt_unpack_kernel<bf16>, d, a, d.d_ff, s);
  return ckpt_run("ffn_restore", ckpt_unpack_kernel<float>, d, a, d.d_ff, s);
}

}  // namespace pcmoe
