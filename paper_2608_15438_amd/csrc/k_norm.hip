// Layer norm of rows and its gradients: with mu and rs the mean and 1 / sqrt of
// the variance (about that mean, plus eps) of a row, xh = (x - mu) rs,
//   y = xh g + b,   u = dy g,
//   dx = rs (u - mean(u) - xh mean(u xh)) + add,   dg = sum dy xh,   db = sum dy.
// All sums in fp32.  What bounds both is memory: a row is read once and kept in
// registers, G lanes a row (16, 64 or the block's 256), NV vectors of eight
// elements a lane.  The backward pass keeps the column sums of dy xh and dy in
// registers too, over all the rows that a group of lanes takes; a block's groups
// meet in LDS, the blocks' sums in a second kernel, in a fixed order.  65,536 x 1536
// bf16: forward 77 us (403 MB, 5.2 TB/s), backward with `add` 178 and 7 for the
// column sums (805 MB, 4.5 TB/s).  Rows wider than 8192 take 64 elements a lane, and
// their backward kernel spills 196 B a lane (16 bits 44): 8192 rows of 16,384 fp32 220 us
// forward, 449 backward (4.9 and 3.6 TB/s), bf16 163 and 370; of 8192 98 and 177, 52 and
// 180.
#include <type_traits>

#include "nr_layers.h"

namespace nr {

constexpr int NORM_BLOCKS = 1024;   // blocks of the backward pass, at most

// sums over a group of G lanes, the same in all of them
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float (*red)[4]) {
  auto add = [&](auto m) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      v[i] += __uint_as_float(xor_lane<decltype(m)::value>(__float_as_uint(v[i])));
  };
  add(std::integral_constant<int, 1>{});
  add(std::integral_constant<int, 2>{});
  add(std::integral_constant<int, 4>{});
  add(std::integral_constant<int, 8>{});
  if constexpr (G >= 64) {
    add(std::integral_constant<int, 16>{});
    add(std::integral_constant<int, 32>{});
  }
  if constexpr (G == 256) {
    __syncthreads();   // the last sums have been read
    if (lane_id() == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[i][threadIdx.x / WAVE] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (red[i][0] + red[i][1]) + (red[i][2] + red[i][3]);
  }
}

template <class T, int G, int NV>
__global__ void __launch_bounds__(256) k_norm(NormArgs a) {
  __shared__ float red[1][4];
  constexpr bool half = __is_same(T, f16_t);
  constexpr int RPB = 256 / G;
  const int d = a.d, dp = (d + 31) / 32 * 32, l = threadIdx.x % G;
  Raw8<T> g[NV], b[NV];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = (n * G + l) * 8;
    if (a.g) g[n].load((const T *)a.g, c, d);
    if (a.b) b[n].load((const T *)a.b, c, d);
  }
  const float inv = 1.0f / (float)d;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.m; r0 += (int64_t)gridDim.x * RPB) {
    const int64_t r = r0 + threadIdx.x / G;
    if (r >= a.m) continue;   // a whole group of lanes; with G = 256 none
    Raw8<T> x[NV];
    float s[1] = {0.0f};
#pragma unroll
    for (int n = 0; n < NV; ++n) x[n].load((const T *)a.x + r * a.ldx, (n * G + l) * 8, d);
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += x[n][i];
    group_sum<G>(s, red);
    const float mu = s[0] * inv;
    s[0] = 0.0f;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = x[n][i] - mu;
        s[0] += (n * G + l) * 8 + i < d ? v * v : 0.0f;
      }
    group_sum<G>(s, red);
    const float rs = 1.0f / sqrtf(s[0] * inv + a.eps);
    if (l == 0 && a.mean) {
      a.mean[r] = mu;
      a.rstd[r] = rs;
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * G + l) * 8;
      if (c >= dp) continue;   // a whole quad
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = x[n][i];
      if (a.x_hold) write8(a.xq + r * dp, a.xs + r * (dp / 32), c, a.x_hold, half, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = (v[i] - mu) * rs;
        if (a.g) v[i] *= g[n][i];
        if (a.b) v[i] += b[n][i];
      }
      store8((T *)a.y + r * a.ldy, c, d, v);
      if (a.y_hold) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < d ? to_f32(from_f32<T>(v[i])) : 0.0f;
        write8(a.yq + r * dp, a.ys + r * (dp / 32), c, a.y_hold, half, v);
      }
    }
  }
}

template <class T, int G, int NV>
__global__ void __launch_bounds__(256) k_norm_grad(NormGradArgs a, float *pg, float *pb) {
  __shared__ float red[2][4];
  constexpr int RPB = 256 / G;
  __shared__ float cols[RPB > 1 ? RPB - 1 : 1][RPB > 1 ? G * 8 : 1];
  const int d = a.d, l = threadIdx.x % G, grp = threadIdx.x / G;
  const float inv = 1.0f / (float)d;
  Raw8<T> g[NV];
  float sg[NV][8], sb[NV][8];
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    if (a.g) g[n].load((const T *)a.g, (n * G + l) * 8, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) sg[n][i] = sb[n][i] = 0.0f;
  }
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.m; r0 += (int64_t)gridDim.x * RPB) {
    const int64_t r = r0 + grp;
    if (r >= a.m) continue;   // a whole group of lanes; with G = 256 none
    float x[NV][8];
    Raw8<T> dy[NV], add[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int c = (n * G + l) * 8;
      dy[n].load((const T *)a.dy + r * a.lddy, c, d);
      if (!a.x.hold) {
        load8((const T *)a.x.p + r * a.x.ld, c, d, x[n]);
      } else if (c < a.x.ld) {
        read8<T>((const uint8_t *)a.x.p + r * a.x.ld, a.x.scale + r * (a.x.ld / 32), c, a.x.hold,
                 x[n]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[n][i] = 0.0f;
      }
      if (a.add) add[n].load((const T *)a.add + r * a.ldadd, c, d);
    }
    const float mu = a.mean[r], rs = a.rstd[r];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int i = 0; i < 8; ++i) {   // past d dy is zero, and so is what it makes
        x[n][i] = (n * G + l) * 8 + i < d ? (x[n][i] - mu) * rs : 0.0f;
        const float v = dy[n][i], u = a.g ? v * g[n][i] : v;
        sg[n][i] += v * x[n][i];
        sb[n][i] += v;
        s[0] += u;
        s[1] += u * x[n][i];
      }
    if (!a.dx) continue;
    group_sum<G>(s, red);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = a.g ? dy[n][i] * g[n][i] : dy[n][i];
        v[i] = rs * (u - m1 - x[n][i] * m2);
        if (a.add) v[i] += add[n][i];
      }
      store8((T *)a.dx + r * a.lddx, (n * G + l) * 8, d, v);
    }
  }
  // the block's groups, in order, eight columns per lane at a time
  auto put = [&](float (&v)[8], float *out, int c) {
    if constexpr (RPB > 1) {
      __syncthreads();
      if (grp > 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) cols[grp - 1][i * G + l] = v[i];
      __syncthreads();
      if (grp > 0) return;
#pragma unroll
      for (int q = 0; q < RPB - 1; ++q)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += cols[q][i * G + l];
    }
    store8(out + (int64_t)blockIdx.x * d, c, d, v);
  };
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int c = (n * G + l) * 8;
    if (a.dg) put(sg[n], pg, c);
    if (a.db) put(sb[n], pb, c);
  }
}

// 64 columns per block; each of sixteen threads of a column adds every
// sixteenth row, then the sixteen sums in order
template <class T>
__global__ void __launch_bounds__(1024) k_col_join(const float *p0, T *out0, const float *p1,
                                                   T *out1, int64_t rows, int d) {
  __shared__ float s[16][64];
  const float *p = blockIdx.y ? p1 : p0;
  T *out = blockIdx.y ? out1 : out0;
  if (!out) return;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float v = 0.0f;
  if (c < d) {
#pragma unroll 8
    for (int64_t r = w; r < rows; r += 16) v += p[r * d + c];
  }
  s[w][lane] = v;
  __syncthreads();
  if (w == 0 && c < d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += s[i][lane];
    out[c] = from_f32<T>(v);
  }
}

template <class T>
static void col_join_t(const float *p0, void *o0, const float *p1, void *o1, int64_t rows, int d,
                       hipStream_t s) {
  hipLaunchKernelGGL(k_col_join<T>, dim3((d + 63) / 64, o1 ? 2 : 1), dim3(1024), 0, s, p0, (T *)o0,
                     p1, (T *)o1, rows, d);
}

hipError_t launch_col_join(const float *p0, void *out0, const float *p1, void *out1, int64_t rows,
                           int d, int dtype, hipStream_t s) {
  if (dtype == NR_F32) col_join_t<float>(p0, out0, p1, out1, rows, d, s);
  else if (dtype == NR_BF16) col_join_t<bf16_t>(p0, out0, p1, out1, rows, d, s);
  else col_join_t<f16_t>(p0, out0, p1, out1, rows, d, s);
  return hipGetLastError();
}

// Calls f(G, NV) with the lanes per row and vectors per lane that hold d elements:
// 16 lanes up to 256, a wave up to 2048 (a row of a wave needs no barrier), the
// block beyond
template <class F>
static void with_shape(int d, F f) {
  using std::integral_constant;
#define NR_SHAPE(g, nv) return f(integral_constant<int, g>{}, integral_constant<int, nv>{})
  if (d <= 128) NR_SHAPE(16, 1);
  if (d <= 256) NR_SHAPE(16, 2);
  if (d <= 512) NR_SHAPE(64, 1);
  if (d <= 1024) NR_SHAPE(64, 2);
  if (d <= 1536) NR_SHAPE(64, 3);
  if (d <= 2048) NR_SHAPE(64, 4);
  if (d <= 4096) NR_SHAPE(256, 2);
  if (d <= 8192) NR_SHAPE(256, 4);
  NR_SHAPE(256, 8);
#undef NR_SHAPE
}

template <class T>
static hipError_t norm_t(const NormArgs &a, hipStream_t s) {
  with_shape(a.d, [&](auto g, auto nv) {
    constexpr int G = decltype(g)::value, NV = decltype(nv)::value;
    const int64_t blocks = (a.m + 256 / G - 1) / (256 / G);
    hipLaunchKernelGGL((k_norm<T, G, NV>), dim3((unsigned)(blocks < 2048 ? blocks : 2048)),
                       dim3(256), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_norm(const NormArgs &a, int dtype, hipStream_t s) {
  if (a.m <= 0) return hipSuccess;
  if (dtype == NR_F32) return norm_t<float>(a, s);
  if (dtype == NR_BF16) return norm_t<bf16_t>(a, s);
  return norm_t<f16_t>(a, s);
}

// blocks of the backward pass: at least eight rows per group of lanes, where
// the rows suffice for 256 blocks so
static int64_t grad_blocks(int64_t m, int d) {
  int64_t per = 1;
  with_shape(d, [&](auto g, auto) { per = 256 / decltype(g)::value; });
  int64_t b = (m + 8 * per - 1) / (8 * per);
  const int64_t most = (m + per - 1) / per;
  if (b < 256) b = 256;
  if (b > most) b = most;
  return b < NORM_BLOCKS ? b : NORM_BLOCKS;
}

size_t norm_grad_ws(const NormGradArgs &a) {
  return a.dg || a.db ? sizeof(float) * (size_t)(2 * grad_blocks(a.m, a.d)) * a.d : 0;
}

template <class T>
static hipError_t norm_grad_t(const NormGradArgs &a, int dtype, float *ws, hipStream_t s) {
  const int64_t nb = grad_blocks(a.m, a.d);
  float *pg = ws, *pb = ws + nb * a.d;
  if (nb > 0)
    with_shape(a.d, [&](auto g, auto nv) {
      hipLaunchKernelGGL((k_norm_grad<T, decltype(g)::value, decltype(nv)::value>),
                         dim3((unsigned)nb), dim3(256), 0, s, a, pg, pb);
    });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !(a.dg || a.db)) return e;
  return launch_col_join(pg, a.dg, pb, a.db, nb, a.d, dtype, s);
}

hipError_t launch_norm_grad(const NormGradArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == NR_F32) return norm_grad_t<float>(a, dtype, (float *)ws, s);
  if (dtype == NR_BF16) return norm_grad_t<bf16_t>(a, dtype, (float *)ws, s);
  return norm_grad_t<f16_t>(a, dtype, (float *)ws, s);
}

}  // namespace nr
