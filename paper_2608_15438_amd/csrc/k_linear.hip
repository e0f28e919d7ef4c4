// A layer of an encoder and its gradients:
//   z = x w^T + bias,  y = act(z) + residual,
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum over the rows of dz.
// Three products over the same tile kernel, out[i][j] = sum over k of A B:
//   y   i = row, j = output, k = input:   both operands have k along their rows
//   dx  i = row, j = input, k = output:   w has j along its rows
//   dw  i = output, j = input, k = row:   both have i or j along their rows
// A block of 256 threads owns a 64 x 64 tile, each wave a 32 x 32 quarter, in
// blocks of 16 x 16 of the fp32 matrix cores.  j takes the place of the
// instruction's rows, so that a lane holds four neighbouring elements of a row
// of the output.  Where the tiles are few and k long, k is cut and the parts'
// fp32 sums are added in order by a second kernel with the same epilogue.
#include "nr_layers.h"

namespace nr {

typedef float v4f __attribute__((ext_vector_type(4)));

struct GemmArgs {
  int64_t I, K, kchunk;  // k of a part, a multiple of the K-tile
  int J;
  LayerMat A, B;         // B may be held in 8 bits where j runs along its rows
  float *part;           // [parts][I][ldp] sums of the parts, or NULL
  int64_t ldp;
  int vec;               // outputs (and residual) can be accessed four elements at a time
  void *out;             // without the layer's epilogue: [I][ldo]
  int64_t ldo;
  LinearArgs lin;
};

template <class T>
__device__ __forceinline__ void store4(T *p, const float (&v)[4], int n, bool vec) {
  if (vec && n >= 4) {
    typedef T t4 __attribute__((ext_vector_type(4)));
    t4 o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = from_f32<T>(v[r]);
    *reinterpret_cast<t4 *>(p) = o;
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < n) p[r] = from_f32<T>(v[r]);
  }
}

template <class T>
__device__ __forceinline__ void load4(const T *p, float (&v)[4], int n, bool vec) {
  if (vec && n >= 4) {
    typedef T t4 __attribute__((ext_vector_type(4)));
    const t4 o = *reinterpret_cast<const t4 *>(p);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = to_f32(o[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = r < n ? to_f32(p[r]) : 0.0f;
  }
}

// The epilogue of 16 rows x 32 columns in a wave: lane l holds row l % 16,
// columns j0 + 16 b + 4 (l / 16) + r.  The whole wave calls it together (a
// group held in 8 bits lies in four lanes); ok: the lane's row is inside
template <class T, bool LIN>
__device__ __forceinline__ void finish(const GemmArgs &a, int64_t i, int j0, bool ok,
                                       float (&v)[2][4]) {
  constexpr bool exact = sizeof(T) == 4;
  const int c = j0 + 4 * (lane_id() >> 4);
  if constexpr (!LIN) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if (ok && c + 16 * b < a.J)
        store4((T *)a.out + i * a.ldo + c + 16 * b, v[b], a.J - c - 16 * b, a.vec);
  } else {
    const LinearArgs &l = a.lin;
    if (l.bias) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = c + 16 * b + r;
          if (j < a.J) v[b][r] += to_f32(((const T *)l.bias)[j]);
        }
    }
    if (l.pre_hold) {
      float z[2][4];
      uint32_t m = 0;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[b][r] = c + 16 * b + r < a.J ? to_f32(from_f32<T>(v[b][r])) : 0.0f;
          const uint32_t u = __float_as_uint(z[b][r]) & 0x7fffffffu;
          m = m > u ? m : u;
        }
      uint32_t o = xor_lane<16>(m);
      m = m > o ? m : o;
      o = xor_lane<32>(m);
      m = m > o ? m : o;
      const int byte = hold_byte(m, l.pre_hold, __is_same(T, f16_t));
      if (ok && j0 < a.J) {
        uint8_t *q = (uint8_t *)l.pre + i * l.ldp + c;
#pragma unroll
        for (int b = 0; b < 2; ++b)
          *reinterpret_cast<uint32_t *>(q + 16 * b) =
              hold_pack4(z[b][0], z[b][1], z[b][2], z[b][3], byte, l.pre_hold);
        if (lane_id() < 16) l.pre_scale[i * (l.ldp / 32) + j0 / 32] = (uint8_t)byte;
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int cb = c + 16 * b, n = a.J - cb;
      if (!ok || n <= 0) continue;
      if (l.pre && !l.pre_hold) store4((T *)l.pre + i * l.ldp + cb, v[b], n, a.vec);
      float s[4] = {};
      if (l.res) load4((const T *)l.res + i * l.ldr + cb, s, n, a.vec);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] += act_value<exact>(v[b][r], l.act);
      store4((T *)l.y + i * l.ldy + cb, s, n, a.vec);
    }
  }
}

constexpr int GT = 64, GK = 16;

// four elements (along the operand's rows) of a K-tile: where k runs along the
// rows, row `o` of the tile's side and k0..; otherwise row k and columns o..
template <class T, bool KC, bool HELD>
__device__ __forceinline__ void stage4(const LayerMat &m, int64_t o, int64_t nO, int64_t k,
                                       int64_t kend, float (&v)[4]) {
  const int64_t row = KC ? o : k, rows = KC ? nO : kend;
  const int64_t col = KC ? k : o, cols = KC ? kend : nO;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = 0.0f;
  if (row >= rows) return;
  if constexpr (HELD) {
    if (col < cols) {
      hold_unpack4(*reinterpret_cast<const uint32_t *>((const uint8_t *)m.p + row * m.ld + col),
                   hold_scale(m.scale[row * (m.ld / 32) + col / 32]), m.hold, v);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = to_f32(from_f32<T>(v[r]));
    }
  } else {
    const T *p = (const T *)m.p + row * m.ld + col;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (col + r < cols) v[r] = to_f32(p[r]);
  }
}

template <class T, bool IK, bool JK, bool HELD, bool LIN>
__global__ void __launch_bounds__(256) k_gemm(GemmArgs a) {
  __shared__ float As[GK][GT + 4], Bs[GK][GT + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wi = 32 * (wave & 1), wj = 32 * (wave >> 1);
  const int64_t tj = (a.J + GT - 1) / GT, tiles = (a.I + GT - 1) / GT * tj;
  const int64_t k0 = (int64_t)blockIdx.y * a.kchunk;
  const int64_t k1 = k0 + a.kchunk < a.K ? k0 + a.kchunk : a.K;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t i0 = t / tj * GT;
    const int j0 = (int)(t % tj) * GT;
    v4f acc[2][2];   // [i][j]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int64_t k = k0; k < k1; k += GK) {
      float va[4], vb[4];
      const int oi = IK ? tid / 4 : 4 * (tid % 16), ki = IK ? 4 * (tid % 4) : tid / 16;
      const int oj = JK ? tid / 4 : 4 * (tid % 16), kj = JK ? 4 * (tid % 4) : tid / 16;
      stage4<T, IK, false>(a.A, i0 + oi, a.I, k + ki, k1, va);
      stage4<T, JK, HELD>(a.B, j0 + oj, a.J, k + kj, k1, vb);
      __syncthreads();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        As[IK ? ki + r : ki][IK ? oi : oi + r] = va[r];
        Bs[JK ? kj + r : kj][JK ? oj : oj + r] = vb[r];
      }
      __syncthreads();
#pragma unroll
      for (int kk = 0; kk < GK; kk += 4) {
        const int kr = kk + (lane >> 4), c = lane & 15;
        float av[2], bv[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          av[u] = As[kr][wi + 16 * u + c];
          bv[u] = Bs[kr][wj + 16 * u + c];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(bv[j], av[i], acc[i][j], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t row = i0 + wi + 16 * i + (lane & 15);
      float v[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[j][r] = acc[i][j][r];
      if (a.part) {
        float *p = a.part + ((int64_t)blockIdx.y * a.I + row) * a.ldp + j0 + wj + 4 * (lane >> 4);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (row < a.I && j0 + wj < a.ldp)
            *reinterpret_cast<float4 *>(p + 16 * j) = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
      } else {
        finish<T, LIN>(a, row, j0 + wj, row < a.I, v);
      }
    }
  }
}

// The parts' sums, in order, and the epilogue: a wave per 16 rows x 32 columns
template <class T, bool LIN>
__global__ void __launch_bounds__(256) k_gemm_join(GemmArgs a, int parts) {
  const int lane = threadIdx.x & 63;
  const int64_t gj = (a.J + 31) / 32, units = (a.I + 15) / 16 * gj;
  for (int64_t u = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE; u < units;
       u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / gj * 16 + (lane & 15);
    const int j0 = (int)(u % gj) * 32;
    const int64_t at = (row < a.I ? row : a.I - 1) * a.ldp + j0 + 4 * (lane >> 4);
    float v[2][4] = {};
    for (int s = 0; s < parts; ++s)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float4 p = *reinterpret_cast<const float4 *>(a.part + (int64_t)s * a.I * a.ldp + at +
                                                           16 * b);
        v[b][0] += p.x, v[b][1] += p.y, v[b][2] += p.z, v[b][3] += p.w;
      }
    finish<T, LIN>(a, row, j0, row < a.I, v);
  }
}

// dz = dy act'(pre) of `rows` rows per block, rounded to the type (dz NULL: not
// wanted), and its column sums over them (part NULL: not wanted).  The 256
// threads are 256 / ct rows of ct threads, eight columns each
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_act_grad(LinearGradArgs a, int64_t rows, int ct, T *dz,
                                                  int64_t ldz, float *part) {
  __shared__ float red[256][9];
  constexpr bool exact = sizeof(T) == 4;
  const int tc = threadIdx.x % ct, tr = threadIdx.x / ct, rt = 256 / ct;
  const int c0 = (blockIdx.y * ct + tc) * 8;
  const int64_t r0 = (int64_t)blockIdx.x * rows, r1 = r0 + rows < a.m ? r0 + rows : a.m;
  float s[8] = {};
  if (c0 < a.n)
    for (int64_t r = r0 + tr; r < r1; r += rt) {
      float v[8], z[8];
      load8<T, VEC>((const T *)a.dy + r * a.lddy, c0, a.n, v);
      if (a.act != NR_ACT_NONE) {
        if (a.pre.hold)
          read8<T>((const uint8_t *)a.pre.p + r * a.pre.ld, a.pre.scale + r * (a.pre.ld / 32), c0,
                a.pre.hold, z);
        else
          load8<T, VEC>((const T *)a.pre.p + r * a.pre.ld, c0, a.n, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= act_slope<exact>(z[i], a.act);
      }
      if (dz) store8<T, true>(dz + r * ldz, c0, a.n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += c0 + i < a.n ? v[i] : 0.0f;
    }
  if (!part) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) red[threadIdx.x][i] = s[i];
  __syncthreads();
  if (tr == 0 && c0 < a.n) {
    for (int u = 1; u < rt; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += red[u * ct + tc][i];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i < a.n) part[(int64_t)blockIdx.x * a.n + c0 + i] = s[i];
  }
}

// ---------------------------------------------------------------- host

static int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
static bool aligned(const void *p, int64_t ld, size_t e, size_t to) {
  return !p || (reinterpret_cast<uintptr_t>(p) % to == 0 && ld * e % to == 0);
}

struct Split {
  int parts;
  int64_t kchunk;
};
// Parts of k: enough for two blocks per CU, each of at least 128 of k
static Split split_of(int64_t I, int J, int64_t K) {
  const int64_t tiles = up(I, GT) / GT * (up(J, GT) / GT);
  int64_t parts = tiles > 0 ? (512 + tiles - 1) / tiles : 1;
  const int64_t most = K / 128 < 64 ? K / 128 : 64;
  if (tiles >= 256 || most < 2) parts = 1;
  else if (parts > most) parts = most;
  const int64_t kc = up((K + parts - 1) / parts, GK);
  return {K > 0 ? (int)((K + kc - 1) / kc) : 1, kc > 0 ? kc : GK};
}
static size_t part_bytes(int64_t I, int J, int64_t K) {
  const Split sp = split_of(I, J, K);
  return sp.parts > 1 ? sizeof(float) * (size_t)sp.parts * I * up(J, 32) : 0;
}

template <class T, bool IK, bool JK, bool LIN>
static hipError_t gemm(GemmArgs a, float *ws, hipStream_t s) {
  if (a.I <= 0) return hipSuccess;
  const Split sp = split_of(a.I, a.J, a.K);
  a.kchunk = sp.kchunk;
  a.part = sp.parts > 1 ? ws : nullptr;
  a.ldp = up(a.J, 32);
  const int64_t tiles = up(a.I, GT) / GT * (up(a.J, GT) / GT);
  const dim3 g((unsigned)(tiles < 1 << 22 ? tiles : 1 << 22), sp.parts);
  if constexpr (!JK) {
    if (a.B.hold)
      hipLaunchKernelGGL((k_gemm<T, IK, JK, true, LIN>), g, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_gemm<T, IK, JK, false, LIN>), g, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((k_gemm<T, IK, JK, false, LIN>), g, dim3(256), 0, s, a);
  }
  if (sp.parts > 1) {
    const int64_t blocks = (up(a.I, 16) / 16 * (up(a.J, 32) / 32) + 3) / 4;
    hipLaunchKernelGGL((k_gemm_join<T, LIN>), dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)),
                       dim3(256), 0, s, a, sp.parts);
  }
  return hipGetLastError();
}

size_t linear_ws(int64_t m, int n, int k, int dtype) { return part_bytes(m, n, k); }

template <class T>
static hipError_t linear_t(const LinearArgs &l, void *ws, hipStream_t s) {
  GemmArgs a{};
  a.I = l.m, a.J = l.n, a.K = l.k;
  a.A = LayerMat{l.x, l.ldx, 0, nullptr};
  a.B = LayerMat{l.w, l.ldw, 0, nullptr};
  a.vec = aligned(l.y, l.ldy, sizeof(T), 4 * sizeof(T)) &&
          aligned(l.res, l.ldr, sizeof(T), 4 * sizeof(T)) &&
          (l.pre_hold || aligned(l.pre, l.ldp, sizeof(T), 4 * sizeof(T)));
  a.lin = l;
  return gemm<T, true, true, true>(a, (float *)ws, s);
}

hipError_t launch_linear(const LinearArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == NR_F32) return linear_t<float>(a, ws, s);
  if (dtype == NR_BF16) return linear_t<bf16_t>(a, ws, s);
  return linear_t<f16_t>(a, ws, s);
}

// Work space of the gradients: dz, the column sums of its blocks, and the
// products' parts (dx and dw one after the other in the same place)
struct GradPlan {
  bool act, dz;          // the pass over dy runs; it writes dz
  int64_t rows, nb, ldz; // rows per block of that pass, its blocks, dz's row stride
  int ct;
  size_t at_part, at_prod, bytes;
};
static GradPlan grad_plan(const LinearGradArgs &a, int dtype) {
  GradPlan p{};
  p.dz = a.act != NR_ACT_NONE && (a.dx || a.dw);
  p.act = p.dz || a.db;
  p.ct = 1;
  while (p.ct < 256 && p.ct * 8 < a.n) p.ct *= 2;
  const int64_t rt = 256 / p.ct;
  p.rows = up((a.m + 1023) / 1024, rt);
  if (p.rows < 8 * rt) p.rows = 8 * rt;
  p.nb = (a.m + p.rows - 1) / p.rows;
  p.ldz = up(a.n, 32);
  size_t off = 0;
  if (p.dz) off += up((size_t)a.m * p.ldz * layer_elem(dtype), 256);
  p.at_part = off;
  if (a.db) off += up(sizeof(float) * (size_t)p.nb * a.n, 256);
  p.at_prod = off;
  const size_t px = a.dx ? part_bytes(a.m, a.k, a.n) : 0, pw = a.dw ? part_bytes(a.n, a.k, a.m) : 0;
  p.bytes = off + (px > pw ? px : pw);
  return p;
}

size_t linear_grad_ws(const LinearGradArgs &a, int dtype) { return grad_plan(a, dtype).bytes; }

template <class T>
static hipError_t linear_grad_t(const LinearGradArgs &l, int dtype, char *ws, hipStream_t s) {
  const GradPlan p = grad_plan(l, dtype);
  T *dz = p.dz ? (T *)ws : nullptr;
  float *part = l.db ? (float *)(ws + p.at_part) : nullptr;
  float *prod = (float *)(ws + p.at_prod);
  if (p.act && l.m > 0) {
    const bool vec = aligned(l.dy, l.lddy, sizeof(T), 16) &&
                     (l.act == NR_ACT_NONE || l.pre.hold ||
                      aligned(l.pre.p, l.pre.ld, sizeof(T), 16));
    const dim3 g((unsigned)p.nb, (l.n + 8 * p.ct - 1) / (8 * p.ct));
    hipLaunchKernelGGL((vec ? k_act_grad<T, true> : k_act_grad<T, false>), g, dim3(256), 0, s, l,
                       p.rows, p.ct, dz, p.ldz, part);
  }
  hipError_t e = hipGetLastError();
  if (l.db && e == hipSuccess) e = launch_col_join(part, p.nb, l.n, l.n, dtype, l.db, s);
  const LayerMat z = p.dz ? LayerMat{dz, p.ldz, 0, nullptr} : LayerMat{l.dy, l.lddy, 0, nullptr};
  if (l.dx && e == hipSuccess) {
    GemmArgs a{};
    a.I = l.m, a.J = l.k, a.K = l.n;
    a.A = z;
    a.B = LayerMat{l.w, l.ldw, 0, nullptr};
    a.out = l.dx, a.ldo = l.lddx;
    a.vec = aligned(l.dx, l.lddx, sizeof(T), 4 * sizeof(T));
    e = gemm<T, true, false, false>(a, prod, s);
  }
  if (l.dw && e == hipSuccess) {
    GemmArgs a{};
    a.I = l.n, a.J = l.k, a.K = l.m;
    a.A = z;
    a.B = l.x;
    a.out = l.dw, a.ldo = l.lddw;
    a.vec = aligned(l.dw, l.lddw, sizeof(T), 4 * sizeof(T));
    e = gemm<T, false, false, false>(a, prod, s);
  }
  return e;
}

hipError_t launch_linear_grad(const LinearGradArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == NR_F32) return linear_grad_t<float>(a, dtype, (char *)ws, s);
  if (dtype == NR_BF16) return linear_grad_t<bf16_t>(a, dtype, (char *)ws, s);
  return linear_grad_t<f16_t>(a, dtype, (char *)ws, s);
}

}  // namespace nr
