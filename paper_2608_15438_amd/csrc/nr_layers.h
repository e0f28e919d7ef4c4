// Layers of an encoder in training (k_linear.hip, k_norm.hip, k_hold.hip):
// argument structs, launch wrappers, and device helpers for the element types
// and for activations held in 8 bits.  Not part of the ABI.
#pragma once

#include "nr_internal.h"

namespace nr {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline size_t layer_elem(int dtype) { return dtype == NR_F32 ? 4 : 2; }
inline int64_t hold_ld(int64_t d) { return (d + 31) / 32 * 32; }

// A matrix operand whose rows are held in 8 bits (hold != 0) or in the type
struct LayerMat {
  const void *p;
  int64_t ld;            // elements of the type, or bytes of q
  int hold;
  const uint8_t *scale;  // [rows x ld / 32] when held
  bool padded;           // zeros from the width up to ld
};

struct LinearArgs {
  int64_t m;
  int n, k;
  int act;
  const void *x;
  int64_t ldx;
  const void *w;
  int64_t ldw;
  const void *bias, *res;
  int64_t ldr;
  void *y;
  int64_t ldy;
  void *pre;
  int64_t ldp;
  int pre_hold;
  uint8_t *pre_scale;
};

struct LinearGradArgs {
  int64_t m;
  int n, k;
  int act;
  const void *dy;
  int64_t lddy;
  LayerMat x;
  const void *w;
  int64_t ldw;
  LayerMat pre;
  void *dx;
  int64_t lddx;
  void *dw;
  int64_t lddw;
  void *db;
};

struct NormArgs {
  int64_t m;
  int d;
  float eps;
  const void *x;
  int64_t ldx;
  const void *g, *b;
  void *y;
  int64_t ldy;
  float *mean, *rstd;  // or NULL
  int x_hold, y_hold;
  uint8_t *xq, *xs, *yq, *ys;
};

struct NormGradArgs {
  int64_t m;
  int d;
  const void *dy;
  int64_t lddy;
  LayerMat x;
  const float *mean, *rstd;
  const void *g, *add;
  int64_t ldadd;
  void *dx;
  int64_t lddx;
  void *dg, *db;
};

size_t linear_ws(const LinearArgs &a, int dtype);
hipError_t launch_linear(const LinearArgs &a, int dtype, void *ws, hipStream_t s);
size_t linear_grad_ws(const LinearGradArgs &a, int dtype);
hipError_t launch_linear_grad(const LinearGradArgs &a, int dtype, void *ws, hipStream_t s);
hipError_t launch_norm(const NormArgs &a, int dtype, hipStream_t s);
size_t norm_grad_ws(const NormGradArgs &a);
hipError_t launch_norm_grad(const NormGradArgs &a, int dtype, void *ws, hipStream_t s);
hipError_t launch_hold(const void *x, int64_t ldx, int64_t m, int d, int dtype, int hold,
                       uint8_t *q, uint8_t *scale, hipStream_t s);
hipError_t launch_read(const uint8_t *q, const uint8_t *scale, int64_t m, int d, int hold,
                       int dtype, void *y, int64_t ldy, hipStream_t s);
// out[c] = sum over r of partial[r][c] (rows of d floats), rounded to the type; the
// rows are added in a fixed order.  Two such sums in one launch; out NULL: not
// wanted
hipError_t launch_col_join(const float *p0, void *out0, const float *p1, void *out1, int64_t rows,
                           int d, int dtype, hipStream_t s);

// ---------------------------------------------------------------- elements

template <class T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <class T>
__device__ __forceinline__ T from_f32(float v) { return (T)v; }   // to nearest, ties to even

// eight elements of a row from column c0 on, zero past d: one 16-byte access (two
// for fp32) wherever the row starts, which costs nothing on a 16-byte boundary
// and little off it
template <class T>
__device__ __forceinline__ void load8(const T *row, int c0, int d, float (&v)[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  if (c0 + 8 <= d) {
    t8 a;
    __builtin_memcpy(&a, row + c0, sizeof a);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(a[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c0 + i < d ? to_f32(row[c0 + i]) : 0.0f;
  }
}

template <class T>
__device__ __forceinline__ void store8(T *row, int c0, int d, const float (&v)[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  if (c0 + 8 <= d) {
    t8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = from_f32<T>(v[i]);
    __builtin_memcpy(row + c0, &a, sizeof a);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i < d) row[c0 + i] = from_f32<T>(v[i]);
  }
}

// eight elements as they are in memory
template <class T>
struct Raw8 {
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 v;
  __device__ __forceinline__ void load(const T *row, int c0, int d) {
    if (c0 + 8 <= d) {
      __builtin_memcpy(&v, row + c0, sizeof v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c0 + i < d ? row[c0 + i] : (T)0.0f;
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return to_f32(v[i]); }
};

// ---------------------------------------------------------------- 8 bits

__device__ __forceinline__ float hold_scale(uint8_t s) {
  return s == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)s << 23);
}

// the scale byte of a group from the bits of its largest magnitude (a NaN's
// bits are above infinity's, so one integer maximum finds both).  half: the
// type is fp16
__device__ __forceinline__ int hold_byte(uint32_t amax, int hold, bool half) {
  if (amax >= 0x7f800000u) return 255;
  const int top = hold == NR_HOLD_I8 ? 6 : 8;
  int e = (int)(amax >> 23) - 127 - top;   // of zero and subnormals: below the range
  e = e < -126 ? -126 : e > 121 ? 121 : e;
  const float v = __uint_as_float(amax) * __uint_as_float((uint32_t)(127 - e) << 23);
  e += hold == NR_HOLD_I8 ? v >= 127.5f : v > 448.0f;
  const int hi = hold == NR_HOLD_I8 ? (half ? 9 : 121) : (half ? 7 : 119);
  return (e > hi ? hi : e) + 127;
}

// four elements under a scale byte, in the bytes of a word
__device__ __forceinline__ uint32_t hold_pack4(float a, float b, float c, float d, int byte,
                                               int hold) {
  if (byte == 255) return 0u;
  const float r = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
  if (hold == NR_HOLD_I8) {
    auto q = [r](float x) {
      return (uint32_t)(int)fminf(fmaxf(rintf(x * r), -127.0f), 127.0f) & 0xffu;
    };
    return q(a) | q(b) << 8 | q(c) << 16 | q(d) << 24;
  }
  auto q = [r](float x) { return fminf(fmaxf(x * r, -448.0f), 448.0f); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(q(a), q(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q(c), q(d), w, true);
}

// and back
__device__ __forceinline__ void hold_unpack4(uint32_t w, float s, int hold, float *v) {
  if (hold == NR_HOLD_I8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i)) * s;
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = lo[0] * s, v[1] = lo[1] * s, v[2] = hi[0] * s, v[3] = hi[1] * s;
  }
}

// eight held elements, as the type has them: fp16's subnormals round, so that a kernel
// that reads what is held in place finds the values of the tensor that reads it out
template <class T>
__device__ __forceinline__ void unpack8(uint2 w, uint8_t scale, int hold, float (&v)[8]) {
  const float s = hold_scale(scale);
  hold_unpack4(w.x, s, hold, v);
  hold_unpack4(w.y, s, hold, v + 4);
  if constexpr (__is_same(T, f16_t))
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(from_f32<T>(v[i]));
}

// eight elements of a held row from column c0 (a multiple of 8) on; the row's q
// bytes start on a 16-byte boundary and are padded to whole groups
template <class T>
__device__ __forceinline__ void read8(const uint8_t *q, const uint8_t *scale, int c0, int hold,
                                      float (&v)[8]) {
  unpack8<T>(*reinterpret_cast<const uint2 *>(q + c0), scale[c0 >> 5], hold, v);
}

// eight elements v of a row at column c0, whose group the four lanes l ^ 1, l ^ 2
// and l ^ 3 hold together: q bytes, and the scale by the first of them.  All
// four lanes call it together
__device__ __forceinline__ void write8(uint8_t *q, uint8_t *scale, int c0, int hold, bool half,
                                       const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
    m = m > b ? m : b;
  }
  uint32_t o = xor_lane<1>(m);
  m = m > o ? m : o;
  o = xor_lane<2>(m);
  m = m > o ? m : o;
  const int byte = hold_byte(m, hold, half);
  *reinterpret_cast<uint2 *>(q + c0) =
      make_uint2(hold_pack4(v[0], v[1], v[2], v[3], byte, hold),
                 hold_pack4(v[4], v[5], v[6], v[7], byte, hold));
  if ((c0 & 31) == 0) scale[c0 >> 5] = (uint8_t)byte;
}

// ---------------------------------------------------------------- activations

// Phi(z) = erfc(-z / sqrt 2) / 2, and e = exp(-z^2 / 2).  EXACT (fp32 results): the
// library's erfc.  The 16-bit types take Phi(-a) exp(a^2 / 2) for a = |z| as a
// polynomial in t = 1 / (1 + 0.3 a) without a constant term (the form of Abramowitz
// and Stegun 7.1.26), its six coefficients fitted here to the RELATIVE error over a
// <= 13.5 (a weighted minimax): below 2^-17.7 up to a = 3, 2^-15.8 up to 6 and 2^-15.3
// up to 13.2, where e leaves fp32's normal range and only subnormal results are
// lost; Phi itself is off by at most 5.3e-7.  Half a step of fp16 is 2^-12 of a value
// or more, so the small results of the negative side round as the large ones do.  (The
// published five coefficients bound the absolute error, 1.5e-7, alone: z Phi(z) at
// -11.75 is 3 % off with them, eight steps of bf16.)  The sixth
// term costs no time: 65,536 x 1024 -> 4096 bf16 with gelu 742 to 748 us, with five 742
// to 754
template <bool EXACT>
__device__ __forceinline__ float normal_cdf(float z, float &e) {
  if constexpr (EXACT) {
    e = expf(-0.5f * z * z);
    return 0.5f * erfcf(z * -0.70710678118654752f);
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3f, 1.0f));
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);   // log2(e) / 2
    float p = fmaf(t, -0.080316348f, 0.22519063f);
    p = fmaf(t, p, -0.026678644f);
    p = fmaf(t, p, 0.14896143f);
    p = fmaf(t, p, 0.11268393f);
    p = fmaf(t, p, 0.12015860f);
    const float h = p * t * e;   // Phi(-|z|)
    return z < 0.0f ? h : 1.0f - h;
  }
}

// The 16-bit types take the hardware's exponential and reciprocal (a few 2^-23 of the
// result; half a step of fp16 is 2^-12 of it), fp32 the library's
template <bool EXACT>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (EXACT) return 1.0f / (1.0f + expf(-z));
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

template <bool EXACT>
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == NR_ACT_RELU) return z > 0.0f || z != z ? z : 0.0f;   // a NaN stays one
  if (act == NR_ACT_GELU) {
    float e;
    return z * normal_cdf<EXACT>(z, e);
  }
  if (act == NR_ACT_SILU) return z * logistic<EXACT>(z);
  return z;
}

template <bool EXACT>
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == NR_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  if (act == NR_ACT_GELU) {
    float e;
    const float c = normal_cdf<EXACT>(z, e);
    return fmaf(z * e, 0.39894228040143268f, c);
  }
  if (act == NR_ACT_SILU) {
    const float p = logistic<EXACT>(z);
    return p * fmaf(z, 1.0f - p, 1.0f);
  }
  return 1.0f;
}

}  // namespace nr
