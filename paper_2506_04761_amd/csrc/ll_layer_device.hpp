// Device-side building blocks of the operators around a token mixer: guarded vector loads, the
// activations in fp32, and sums across the lanes of a wave.
#pragma once

#include <utility>

#include "ll_device.hpp"

namespace ll {

template <typename T, int N>
struct VecN {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef type loose __attribute__((aligned(sizeof(T))));  // at any element
};

// N adjacent elements at p, of which the first n are inputs (the others read as zero, and are not
// touched): `vec` says that rows are aligned for whole vectors (then n is 0 or N).
template <typename T, int N>
__device__ inline typename VecN<T, N>::type load_n(const T* p, int n, bool vec) {
  typename VecN<T, N>::type v = {};
  if (vec) {
    if (n > 0) v = *reinterpret_cast<const typename VecN<T, N>::type*>(p);
  } else if (n == N) {
    v = *reinterpret_cast<const typename VecN<T, N>::loose*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) v[i] = p[i];
  }
  return v;
}

template <typename T, int N>
__device__ inline void store_n(T* p, const float* f, int n, bool vec) {
  typename VecN<T, N>::type v;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = from_f32<T>(f[i]);
  if (vec) {
    if (n > 0) *reinterpret_cast<typename VecN<T, N>::type*>(p) = v;
  } else if (n == N) {
    *reinterpret_cast<typename VecN<T, N>::loose*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = v[i];
  }
}

// N adjacent parameters at p, or `value` without any; the first n are inputs, the others zero.  `vec`: 16-byte aligned.
template <int N>
__device__ inline void load_params(const float* p, int n, float value, bool vec, float* f) {
  if (p && vec && n == N && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
      for (int j = 0; j < 4 && i + j < N; ++j) f[i + j] = v[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = i < n ? (p ? p[i] : value) : 0.0f;
  }
}

// Element n of row `row` at `base` (the same for all lanes: a uniform address plus a lane's 32-bit offset).
template <typename T>
__device__ inline T load_at(const T* base, int row, int64_t stride, int n) {
  return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + (unsigned(row) * unsigned(stride) + unsigned(n)) * unsigned(sizeof(T)));
}
// 1 / (1 + e^-v); v_exp_f32 and v_rcp_f32 are each within 1 ulp.
__device__ inline float sigmoidf(float v) { return __builtin_amdgcn_rcpf(1.0f + fast_exp2(-kLog2e * v)); }
__device__ inline float silu(float v) { return v * sigmoidf(v); }
// d silu / dv, given p = sigmoid(v)
__device__ inline float silu_grad(float v, float p) { return p * (1.0f + v * (1.0f - p)); }

// softplus(v) = max(v, 0) + log1p(e), e = exp(-|v|) in [0, 1].  log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3;
// atanh(s) = s (1 + q r(q)), q = s^2, with r a cubic fitted to a relative error of 4.5e-9 over q in [0, 1/9].
// A small e keeps its relative precision (log(1 + e) would lose it, and step sizes are mostly small).
__device__ inline float softplusf(float v) {
  const float e = fast_exp2(-kLog2e * __builtin_fabsf(v));
  const float s = e * __builtin_amdgcn_rcpf(2.0f + e);
  const float q = s * s;
  float p = 0.14012232f;
  p = fmaf(p, q, 0.13999569f);
  p = fmaf(p, q, 0.20010850f);
  p = fmaf(p, q, 0.33333206f);
  p = fmaf(p, q, 1.0f);
  return fmaf(s + s, p, v > 0.0f ? v : 0.0f);
}

// The lanes of one wave exchange data through LDS without a workgroup barrier: the LDS serves a
// wave's accesses in order, so only the compiler has to keep theirs.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// f(0), f(1), .. with the index as a compile-time constant (DPP controls need one).
template <int... I, typename F>
__device__ inline void unrolled(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}

template <int CTRL>
__device__ inline float dpp_mov(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Lane M of each row of 16 lanes, seen by the whole row (an operand modifier: no instruction of its own
// where the compiler folds it into the product).
template <int M>
__device__ inline float row_bcast(float v) {
  return dpp_mov<0x150 + M>(v);
}

// One token of a backward scan for four states: g_i += c_i dy, then sum_i b_i g_i and, with H, sum_i c_i h_i, where
// b_i and c_i are lane M + i of each row of `b` and `c`: DPP operands, in multiply-adds that the compiler does not form
// by itself.  A register needs two wait states between its write and its use as a DPP operand; the compiler does not
// see into the block, so it waits itself.  Every g_i is written before the last input is read (early clobber): an input of
// the same value needs a register of its own.
template <int M, bool H>
__device__ inline void grad_token(float* g, float b, float c, float dy, const float* h, float& bg, float& ch) {
#define LL_DPP(op, d, s, v, m) op " " d ", " s ", " v " row_newbcast:" m " row_mask:0xf bank_mask:0xf\n\t"
  if (H) {
    asm("s_nop 1\n\t"
        LL_DPP("v_fmac_f32_dpp", "%0", "%7", "%8", "%13") LL_DPP("v_fmac_f32_dpp", "%1", "%7", "%8", "%14")
        LL_DPP("v_fmac_f32_dpp", "%2", "%7", "%8", "%15") LL_DPP("v_fmac_f32_dpp", "%3", "%7", "%8", "%16")
        LL_DPP("v_mul_f32_dpp", "%5", "%7", "%9", "%13") LL_DPP("v_mul_f32_dpp", "%4", "%6", "%0", "%13")
        LL_DPP("v_fmac_f32_dpp", "%5", "%7", "%10", "%14") LL_DPP("v_fmac_f32_dpp", "%4", "%6", "%1", "%14")
        LL_DPP("v_fmac_f32_dpp", "%5", "%7", "%11", "%15") LL_DPP("v_fmac_f32_dpp", "%4", "%6", "%2", "%15")
        LL_DPP("v_fmac_f32_dpp", "%5", "%7", "%12", "%16") LL_DPP("v_fmac_f32_dpp", "%4", "%6", "%3", "%16")
        : "+&v"(g[0]), "+&v"(g[1]), "+&v"(g[2]), "+&v"(g[3]), "=&v"(bg), "=&v"(ch)
        : "v"(b), "v"(c), "v"(dy), "v"(h[0]), "v"(h[1]), "v"(h[2]), "v"(h[3]), "n"(M), "n"(M + 1), "n"(M + 2), "n"(M + 3));
  } else {
    asm("s_nop 1\n\t"
        LL_DPP("v_fmac_f32_dpp", "%0", "%6", "%7", "%8") LL_DPP("v_fmac_f32_dpp", "%1", "%6", "%7", "%9")
        LL_DPP("v_fmac_f32_dpp", "%2", "%6", "%7", "%10") LL_DPP("v_fmac_f32_dpp", "%3", "%6", "%7", "%11")
        LL_DPP("v_mul_f32_dpp", "%4", "%5", "%0", "%8") LL_DPP("v_fmac_f32_dpp", "%4", "%5", "%1", "%9")
        LL_DPP("v_fmac_f32_dpp", "%4", "%5", "%2", "%10") LL_DPP("v_fmac_f32_dpp", "%4", "%5", "%3", "%11")
        : "+&v"(g[0]), "+&v"(g[1]), "+&v"(g[2]), "+&v"(g[3]), "=&v"(bg)
        : "v"(b), "v"(c), "v"(dy), "n"(M), "n"(M + 1), "n"(M + 2), "n"(M + 3));
    ch = 0.0f;
  }
#undef LL_DPP
}

// Sums over the 16 lanes of each row of 16 values: lane m of a row holds the total of v[m].  Halves of a row
// are paired, then quads, then lanes of a quad; each step adds two values' pairs and keeps one of them in each
// half of the lanes, the first two with the write mask of the add itself (33 instructions for 16 sums).
__device__ inline float sum_lanes16(const float (&v)[16]) {
  float w[8], x[4];
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %8, %8 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %1, %9, %9 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %2, %10, %10 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %3, %11, %11 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %4, %12, %12 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %5, %13, %13 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %6, %14, %14 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %7, %15, %15 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %0, %16, %16 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %1, %17, %17 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %2, %18, %18 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %3, %19, %19 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %4, %20, %20 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %5, %21, %21 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %6, %22, %22 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
      "v_add_f32_dpp %7, %23, %23 row_ror:8 row_mask:0xf bank_mask:0xc"
      : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7])
      : "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]), "v"(v[8]), "v"(v[9]),
        "v"(v[10]), "v"(v[11]), "v"(v[12]), "v"(v[13]), "v"(v[14]), "v"(v[15]));
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %4, %4 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %1, %5, %5 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %2, %6, %6 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %3, %7, %7 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
      "v_add_f32_dpp %0, %8, %8 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
      "v_add_f32_dpp %1, %9, %9 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
      "v_add_f32_dpp %2, %10, %10 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
      "v_add_f32_dpp %3, %11, %11 row_half_mirror row_mask:0xf bank_mask:0xa"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
      : "v"(w[0]), "v"(w[1]), "v"(w[2]), "v"(w[3]), "v"(w[4]), "v"(w[5]), "v"(w[6]), "v"(w[7]));
  const int lane = threadIdx.x;
  const bool b1 = lane & 2, b0 = lane & 1;
  const float k0 = b1 ? x[2] : x[0], o0 = b1 ? x[0] : x[2], k1 = b1 ? x[3] : x[1], o1 = b1 ? x[1] : x[3];
  const float y0 = k0 + dpp_mov<0x4E>(o0), y1 = k1 + dpp_mov<0x4E>(o1);  // quad_perm 2,3,0,1
  const float k = b0 ? y1 : y0, o = b0 ? y0 : y1;
  return k + dpp_mov<0xB1>(o);  // quad_perm 1,0,3,2
}

// Sums over the four rows of 16 lanes of four values: row r of the result holds the total of y_r.
__device__ inline float sum_rows4(float y0, float y1, float y2, float y3) {
  auto swap32 = [](float& a, float& b) {
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    a = __builtin_bit_cast(float, (unsigned)s[0]);
    b = __builtin_bit_cast(float, (unsigned)s[1]);
  };
  auto swap16 = [](float& a, float& b) {
    const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    a = __builtin_bit_cast(float, (unsigned)s[0]);
    b = __builtin_bit_cast(float, (unsigned)s[1]);
  };
  swap32(y0, y2);
  swap32(y1, y3);
  float s02 = y0 + y2, s13 = y1 + y3;
  swap16(s02, s13);
  return s02 + s13;
}

}  // namespace ll
