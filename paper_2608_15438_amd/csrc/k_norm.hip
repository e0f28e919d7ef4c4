// Layer norm of rows and its gradients: with mu and rs the mean and 1 / sqrt of
// the variance (about that mean, plus eps) of a row, xh = (x - mu) rs,
//   y = xh g + b,   u = dy g,
//   dx = rs (u - mean(u) - xh mean(u xh)) + add,   dg = sum dy xh,   db = sum dy.
// All sums in fp32.  A block of 256 threads takes a row, eight elements per
// thread at a time.
#include "nr_layers.h"

namespace nr {

// sums over the 256 threads, the same in all of them
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float (*red)[4]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    for (int m = 1; m < WAVE; m <<= 1) v[i] += __shfl_xor(v[i], m);
  __syncthreads();
  if (lane_id() == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[i][threadIdx.x / WAVE] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (red[i][0] + red[i][1]) + (red[i][2] + red[i][3]);
}

// eight elements of a row of the type, or of one held in 8 bits
template <class T>
__device__ __forceinline__ void row8(const LayerMat &a, int64_t r, int c0, int d, float (&v)[8]) {
  if (a.hold)
    read8<T>((const uint8_t *)a.p + r * a.ld, a.scale + r * (a.ld / 32), c0, a.hold, v);
  else
    load8((const T *)a.p + r * a.ld, c0, d, v);
}

template <class T>
__global__ void __launch_bounds__(256) k_norm(NormArgs a) {
  __shared__ float red[1][4];
  constexpr bool half = __is_same(T, f16_t);
  const int d = a.d, dp = (d + 31) / 32 * 32;
  for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
    const T *x = (const T *)a.x + r * a.ldx;
    float v[8], s[1] = {0.0f};
    for (int c = threadIdx.x * 8; c < d; c += 2048) {
      load8(x, c, d, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[i];
    }
    block_sum(s, red);
    const float mu = s[0] / (float)d;
    s[0] = 0.0f;
    for (int c = threadIdx.x * 8; c < d; c += 2048) {
      load8(x, c, d, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += c + i < d ? (v[i] - mu) * (v[i] - mu) : 0.0f;
    }
    block_sum(s, red);
    const float rs = 1.0f / sqrtf(s[0] / (float)d + a.eps);
    if (threadIdx.x == 0 && a.mean) {
      a.mean[r] = mu;
      a.rstd[r] = rs;
    }
    for (int c = threadIdx.x * 8; c < dp; c += 2048) {
      float g[8], b[8];
      load8(x, c, d, v);
      if (a.x_hold) write8(a.xq + r * dp, a.xs + r * (dp / 32), c, a.x_hold, half, v);
      if (a.g) load8((const T *)a.g, c, d, g);
      if (a.b) load8((const T *)a.b, c, d, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = (v[i] - mu) * rs * (a.g ? g[i] : 1.0f) + (a.b ? b[i] : 0.0f);
        v[i] = c + i < d ? to_f32(from_f32<T>(v[i])) : 0.0f;
      }
      store8((T *)a.y + r * a.ldy, c, d, v);
      if (a.y_hold) write8(a.yq + r * dp, a.ys + r * (dp / 32), c, a.y_hold, half, v);
    }
  }
}

template <class T>
__global__ void __launch_bounds__(256) k_norm_dx(NormGradArgs a) {
  __shared__ float red[2][4];
  const int d = a.d;
  for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
    const T *dy = (const T *)a.dy + r * a.lddy;
    const float mu = a.mean[r], rs = a.rstd[r];
    float x[8], u[8], g[8], s[2] = {0.0f, 0.0f};
    for (int c = threadIdx.x * 8; c < d; c += 2048) {
      row8<T>(a.x, r, c, d, x);
      load8(dy, c, d, u);
      if (a.g) load8((const T *)a.g, c, d, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c + i >= d) continue;
        if (a.g) u[i] *= g[i];
        s[0] += u[i];
        s[1] += u[i] * ((x[i] - mu) * rs);
      }
    }
    block_sum(s, red);
    const float m1 = s[0] / (float)d, m2 = s[1] / (float)d;
    for (int c = threadIdx.x * 8; c < d; c += 2048) {
      row8<T>(a.x, r, c, d, x);
      load8(dy, c, d, u);
      if (a.g) load8((const T *)a.g, c, d, g);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        u[i] = rs * ((a.g ? u[i] * g[i] : u[i]) - m1 - (x[i] - mu) * rs * m2);
      if (a.add) {
        load8((const T *)a.add + r * a.ldadd, c, d, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] += x[i];
      }
      store8((T *)a.dx + r * a.lddx, c, d, u);
    }
  }
}

// Column sums over `rows` rows per block: dy xh, and dy
template <class T>
__global__ void __launch_bounds__(256) k_norm_cols(NormGradArgs a, int64_t rows, float *pg,
                                                   float *pb) {
  const int c0 = (blockIdx.y * 256 + threadIdx.x) * 8;
  if (c0 >= a.d) return;
  const int64_t r0 = (int64_t)blockIdx.x * rows, r1 = r0 + rows < a.m ? r0 + rows : a.m;
  float sg[8] = {}, sb[8] = {};
  for (int64_t r = r0; r < r1; ++r) {
    const float mu = a.mean[r], rs = a.rstd[r];
    float x[8], u[8];
    row8<T>(a.x, r, c0, a.d, x);
    load8((const T *)a.dy + r * a.lddy, c0, a.d, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sg[i] += u[i] * ((x[i] - mu) * rs);
      sb[i] += u[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c0 + i < a.d) {
      pg[(int64_t)blockIdx.x * a.d + c0 + i] = sg[i];
      pb[(int64_t)blockIdx.x * a.d + c0 + i] = sb[i];
    }
}

// 64 columns per block; each of sixteen threads of a column adds every
// sixteenth row, then the sixteen sums in order
template <class T>
__global__ void __launch_bounds__(1024) k_col_join(const float *partial, int64_t rows, int64_t ld,
                                                   int d, T *out) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float v = 0.0f;
  if (c < d)
    for (int64_t r = w; r < rows; r += 16) v += partial[r * ld + c];
  s[w][lane] = v;
  __syncthreads();
  if (w == 0 && c < d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += s[i][lane];
    out[c] = from_f32<T>(v);
  }
}

hipError_t launch_col_join(const float *partial, int64_t rows, int64_t ld, int d, int dtype,
                           void *out, hipStream_t s) {
  const dim3 g((d + 63) / 64), b(1024);
  if (dtype == NR_F32)
    hipLaunchKernelGGL(k_col_join<float>, g, b, 0, s, partial, rows, ld, d, (float *)out);
  else if (dtype == NR_BF16)
    hipLaunchKernelGGL(k_col_join<bf16_t>, g, b, 0, s, partial, rows, ld, d, (bf16_t *)out);
  else
    hipLaunchKernelGGL(k_col_join<f16_t>, g, b, 0, s, partial, rows, ld, d, (f16_t *)out);
  return hipGetLastError();
}

static unsigned row_grid(int64_t m) { return (unsigned)(m < 1 << 20 ? m : 1 << 20); }

template <class T>
static hipError_t norm_t(const NormArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(k_norm<T>, dim3(row_grid(a.m)), dim3(256), 0,
                     s, a);
  return hipGetLastError();
}

hipError_t launch_norm(const NormArgs &a, int dtype, hipStream_t s) {
  if (a.m <= 0) return hipSuccess;
  if (dtype == NR_F32) return norm_t<float>(a, s);
  if (dtype == NR_BF16) return norm_t<bf16_t>(a, s);
  return norm_t<f16_t>(a, s);
}

// rows per block of the column sums: at most 1024 blocks of rows
static int64_t col_rows(int64_t m) {
  const int64_t r = (m + 1023) / 1024;
  return r < 32 ? 32 : r;
}

size_t norm_grad_ws(const NormGradArgs &a) {
  if (!a.dg && !a.db) return 0;
  const int64_t nb = (a.m + col_rows(a.m) - 1) / col_rows(a.m);
  return sizeof(float) * (size_t)(2 * nb) * a.d;
}

template <class T>
static hipError_t norm_grad_t(const NormGradArgs &a, int dtype, float *ws, hipStream_t s) {
  if (a.dx && a.m > 0)
    hipLaunchKernelGGL(k_norm_dx<T>, dim3(row_grid(a.m)), dim3(256), 0, s, a);
  if (a.dg || a.db) {
    const int64_t rows = col_rows(a.m), nb = (a.m + rows - 1) / rows;
    float *pg = ws, *pb = ws + nb * a.d;
    if (nb > 0)
      hipLaunchKernelGGL(k_norm_cols<T>, dim3((unsigned)nb, (a.d + 2047) / 2048), dim3(256), 0, s,
                         a, rows, pg, pb);
    hipError_t er = hipSuccess;
    if (a.dg) er = launch_col_join(pg, nb, a.d, a.d, dtype, a.dg, s);
    if (a.db && er == hipSuccess) er = launch_col_join(pb, nb, a.d, a.d, dtype, a.db, s);
    if (er != hipSuccess) return er;
  }
  return hipGetLastError();
}

hipError_t launch_norm_grad(const NormGradArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == NR_F32) return norm_grad_t<float>(a, dtype, (float *)ws, s);
  if (dtype == NR_BF16) return norm_grad_t<bf16_t>(a, dtype, (float *)ws, s);
  return norm_grad_t<f16_t>(a, dtype, (float *)ws, s);
}

}  // namespace nr
