// A layer of an encoder and its gradients:
//   z = x w^T + bias,  y = act(z) + residual,
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum over the rows of dz.
// Three products over the same tile kernel, out[i][j] = sum over k of A B:
//   y   i = row, j = output, k = input:   both operands have k along their rows
//   dx  i = row, j = input, k = output:   w has j along its rows
//   dw  i = output, j = input, k = row:   both have i or j along their rows
// j takes the place of the matrix instruction's rows, so that a lane holds four
// neighbouring elements of a row of the output.  Where the tiles are few and k
// long, k is cut and the parts' fp32 sums are added in order by a second kernel
// with the same epilogue.
#include <cmath>
#include <type_traits>

#include "nr_layers.h"

namespace nr {

typedef float v4f __attribute__((ext_vector_type(4)));

struct GemmArgs {
  int64_t I, K, kchunk;  // k of a part, a multiple of the K-tiles
  int J;
  LayerMat A, B;         // B may be held in 8 bits where j runs along its rows
  int64_t grid;          // blocks, a multiple of 8
  int parts;
  float *part;           // [parts][I][ldp] sums of the parts, or NULL
  int64_t ldp;
  void *out;             // without the layer's epilogue: [I][ldo]
  int64_t ldo;
  LinearArgs lin;
};

// The epilogue of eight columns of a row from j on (a multiple of 8), with their
// bias and residual.  A group held in 8 bits lies in the lanes of a quad, which
// call it together; ok: the row is inside
template <class T, bool LIN>
__device__ __forceinline__ void finish(const GemmArgs &a, int64_t i, int j, bool ok,
                                       float (&v)[8], const Raw8<T> &bias, const Raw8<T> &res) {
  if constexpr (!LIN) {
    if (ok) store8((T *)a.out + i * a.ldo, j, a.J, v);
  } else {
    constexpr bool exact = sizeof(T) == 4;
    const LinearArgs &l = a.lin;
    if (l.bias) {
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] += bias[r];
    }
    if (l.pre_hold) {
      float u[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) u[r] = j + r < a.J ? to_f32(from_f32<T>(v[r])) : 0.0f;
      if (ok && j < l.ldp)   // the rows of q are whole groups, so a quad is in or out
        write8((uint8_t *)l.pre + i * l.ldp, l.pre_scale + i * (l.ldp / 32), j, l.pre_hold,
               __is_same(T, f16_t), u);
    } else if (l.pre && ok) {
      store8((T *)l.pre + i * l.ldp, j, a.J, v);
    }
    if (!ok) return;
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = act_value<exact>(v[r], l.act);
    if (l.res) {
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] += res[r];
    }
    store8((T *)l.y + i * l.ldy, j, a.J, v);
  }
}

// ---------------------------------------------------------------- the tiles
//
// The 16-bit types go to the matrix cores as they are; a float goes as three
// bf16 (its upper eight significant bits, the next eight, and the rest), and a
// product of two floats as the six products of parts that are above 2^-24 of
// it.  The matrix cores make 16 bf16 products in the time of one fp32 product,
// so six still leave 2.7 times the rate, and what is dropped is of the size of
// the rounding that an fp32 product has anyway.
template <class T>
struct Tile {
  typedef T E;
  static constexpr int P = 1, BK = 64;
};
template <>
struct Tile<float> {
  typedef bf16_t E;
  static constexpr int P = 3, BK = 32;
};

typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v4f mma(bf16x8 a, bf16x8 b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(f16x8 a, f16x8 b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ const uint4 zero_chunk = {0, 0, 0, 0};

// One operand's K-tile: BK of k by R of its side, in chunks of eight elements
// (16 bytes of LDS), read from memory into registers and, a K-tile later, put
// into LDS.
//   KC (k along the operand's rows): [R][BK]; the chunks of a row are exchanged
//     by the row's number, so that the lanes that LDS serves together (a quarter
//     of a wave, by fours: 0-3, 12-15, 20-23, 24-27, and so on) find theirs on
//     different banks.
//   otherwise: [BK][R]; pairs of chunks (the sixteen columns of a block) are
//     exchanged by k, and a block is read transposed (ds_read_b64_tr_b16: sixteen
//     lanes give the addresses of four rows of sixteen columns, and lane t
//     receives the four elements of column t).
template <class T, int R, bool KC, bool HELD, int NT = 256, int BK_ = Tile<T>::BK>
struct Operand {
  typedef typename Tile<T>::E E;
  typedef E E8 __attribute__((ext_vector_type(8)));
  static constexpr int BK = BK_, P = Tile<T>::P;
  static constexpr int N = R * BK / 8 / NT;       // chunks per thread
  static constexpr int CPR = (KC ? BK : R) / 8;   // chunks per row of the tile in memory
  static constexpr int PLANE = R * BK * 2, BYTES = P * PLANE;
  static_assert(N >= 1 && N * NT * 8 == R * BK, "whole chunks per thread");

  uint4 raw[N][sizeof(T) / 2];   // what the thread has read; of held rows:
  uint2 q[N];
  uint32_t scale[N];

  // where chunk c of a row lies, and (the exchange being its own inverse) the
  // chunk that lies at place c
  static __device__ __forceinline__ int swap(int row, int c) {
    if constexpr (KC && BK == 128) return c ^ (row & 15);
    else if constexpr (KC && BK == 64) return c ^ (row & 7);
    else if constexpr (KC) return c ^ ((row >> 3) & 1) << 1;
    else if constexpr (R >= 128) return c ^ (((row & 3) | ((row >> 3) & 1) << 2) << 1);
    else return c ^ ((row & 3) << 1);
  }
  static __device__ __forceinline__ int slot(int row, int c) { return row * CPR + swap(row, c); }

  // eight elements from p on as they are in memory, at any alignment of the
  // element; of a chunk that reaches past the row's end at n, zeros from there
  // on.  room: elements from p to the matrix's last, beyond which nothing is read
  static __device__ __forceinline__ void load(uint4 (&o)[sizeof(T) / 2], const T *p, int n,
                                              int64_t room) {
    constexpr int W = 2 * sizeof(T);   // words of a chunk
    uint32_t v[W];
    if (room >= 8) {
      __builtin_memcpy(v, p, sizeof v);
    } else {   // the last chunk of the last row
#pragma unroll
      for (int w = 0; w < W; ++w) v[w] = 0;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        uint32_t x = 0;
        __builtin_memcpy(&x, p + i, sizeof(T));
        x <<= sizeof(T) == 2 ? 16 * (i & 1) : 0;
        const int at = sizeof(T) == 2 ? i >> 1 : i;
#pragma unroll
        for (int w = 0; w < W; ++w) v[w] |= w == at ? x : 0;
      }
    }
    if (n < 8)
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (sizeof(T) == 2) v[w] = 2 * w + 1 < n ? v[w] : 2 * w < n ? v[w] & 0xffffu : 0;
        else v[w] = w < n ? v[w] : 0;
      }
    __builtin_memcpy(o, v, sizeof v);
  }

  // [o0, o0 + R) x [k, k + BK) of a matrix whose rows have `width` elements.  Past
  // kend, and past nO where the side runs along the rows, zeros; rows of a KC
  // operand past nO repeat the last (their outputs are dropped).  FULL: nothing is
  // past an end
  template <bool FULL>
  __device__ __forceinline__ void fetch(const LayerMat &m, int64_t o0, int64_t nO, int64_t k,
                                        int64_t kend, int64_t K) {
    int tid = threadIdx.x;
    // the addresses of tiles at an end are found where they are needed: kept over
    // the whole loop they would cost the registers that the products need
    if constexpr (!FULL) asm volatile("" : "+v"(tid));
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = tid + NT * u;
      int64_t row = (KC ? o0 : k) + e / CPR;
      const int64_t col = (KC ? k : o0) + 8 * (e % CPR), cols = KC ? kend : nO;
      bool in = true;
      if constexpr (!FULL && KC) row = row < nO ? row : nO - 1;
      if constexpr (!FULL && !KC) in = row < kend;
      if constexpr (HELD) {
        q[u] = make_uint2(0, 0);
        scale[u] = 127;
        if (FULL || (in && col < m.ld)) {   // padded to whole groups, zeros behind the width
          q[u] = *reinterpret_cast<const uint2 *>((const uint8_t *)m.p + row * m.ld + col);
          scale[u] = m.scale[row * (m.ld / 32) + col / 32];
        }
      } else if constexpr (FULL) {
        __builtin_memcpy(raw[u], (const T *)m.p + row * m.ld + col, 8 * sizeof(T));
      } else {
        __builtin_memset(raw[u], 0, 8 * sizeof(T));
        if (in && col < cols) {
          const int64_t at = row * m.ld + col;
          load(raw[u], (const T *)m.p + at, cols - col < 8 ? (int)(cols - col) : 8,
               ((KC ? nO : K) - 1) * m.ld + (KC ? K : nO) - at);
        }
      }
    }
  }

  __device__ __forceinline__ void stash(char *lds, int hold) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = threadIdx.x + NT * u;
      char *at = lds + slot(e / CPR, e % CPR) * 16;
      if constexpr (sizeof(T) == 2 && !HELD) {
        *reinterpret_cast<uint4 *>(at) = raw[u][0];
      } else {
        float v[8];
        if constexpr (HELD) {
          const float s = hold_scale((uint8_t)scale[u]);
          hold_unpack4(q[u].x, s, hold, v);
          hold_unpack4(q[u].y, s, hold, v + 4);
        } else {
          __builtin_memcpy(v, raw[u], 32);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {   // each part is the rest, rounded to nearest
          E8 o;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i] = from_f32<E>(v[i]);
            if (p + 1 < P) v[i] -= to_f32(o[i]);
          }
          *reinterpret_cast<E8 *>(at + p * PLANE) = o;
        }
      }
    }
  }

  // The same straight from memory into LDS, for rows that lie on 16-byte
  // boundaries and whole chunks: a wave's 64 chunks go to 1 KB in a row, so each
  // lane reads the chunk that belongs in its place.  offset: the lane's bytes
  // from the tile's first element, found once; a side past nO repeats its last
  // row or chunk (outputs that are dropped)
  static __device__ __forceinline__ void dma_offsets(const LayerMat &m, int64_t o0, int64_t nO,
                                                     uint32_t (&offset)[N]) {
    const int64_t left = nO - o0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int e = threadIdx.x + NT * u;
      int row = e / CPR, c = swap(row, e % CPR);
      if (KC) row = row < left ? row : (int)left - 1;
      else c = 8 * c < left ? c : (int)((left - 1) / 8);
      offset[u] = (uint32_t)(row * m.ld + 8 * c) * (uint32_t)sizeof(T);
    }
  }
  // (in asm, so that the compiler does not wait for them before every read of LDS;
  // arrived() does, once a K-tile.  m0 holds the LDS address; the load follows its
  // writing by a wait state).  k of the chunks from `left` on: zeros
  template <bool FULL>
  static __device__ __forceinline__ void dma(const T *base, const uint32_t (&offset)[N],
                                             uint32_t lds, int left) {
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds + threadIdx.x / WAVE * 1024);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if constexpr (FULL) {
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :: "{m0}"(at + NT * 16 * u), "v"(offset[u]), "s"(base) : "memory");
      } else {
        const char *p = (const char *)base + offset[u];
        const int e = threadIdx.x + NT * u;
        if ((KC ? 8 * swap(e / CPR, e % CPR) : e / CPR) >= left) p = (const char *)&zero_chunk;
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     :: "{m0}"(at + NT * 16 * u), "v"(p) : "memory");
      }
    }
  }

  // of a 16 x 16 x 32 block from b0 of the side and k = 32 s on: lane l has side
  // b0 + l % 16, k = 32 s + 8 (l / 16) and the seven after it
  static __device__ __forceinline__ E8 frag(const char *lds, int p, int b0, int s) {
    const int t = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    lds += p * PLANE;
    if constexpr (KC) {
      return *reinterpret_cast<const E8 *>(lds + slot(b0 + t, 4 * s + g) * 16);
    } else {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const int k = 32 * s + 8 * g + (t >> 2), c = b0 / 8 + ((t & 3) >> 1), in = 8 * (t & 1);
      const s16x4 lo =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(lds + slot(k, c) * 16 + in));
      const s16x4 hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(lds + slot(k + 4, c) * 16 + in));
      return __builtin_bit_cast(E8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Eight neighbouring outputs of row i as plain chains of fp32 (the columns of `bad`;
// the others stay as they are), for those that came out infinite or as no number: the
// parts of an infinity (or of a float above the largest bf16) make NaN of what is an
// infinity or a number.  The eight chains run side by side, with vector loads; all
// that are no number end.  Slow all the same: 4096 x 1024 -> 1024 y 69 us, with every x
// infinite 2800, one row of them 350; dw 69, with any row infinite (a term of every sum)
// 1300
template <bool IK, bool JK, bool HELD>
__device__ __forceinline__ void plain_chains(const LayerMat &A, const LayerMat &B, int64_t i,
                                             int j, int J, int64_t k0, int64_t k1, uint32_t bad,
                                             float (&v)[8]) {
  float s[8] = {};
#pragma unroll
  for (int r = 0; r < 8; ++r) bad &= j + r < J ? ~0u : ~(1u << r);
  auto open = [&]() {   // a wanted chain that may still change
    bool o = false;
#pragma unroll
    for (int r = 0; r < 8; ++r) o = o || ((bad >> r & 1) && s[r] == s[r]);
    return o;
  };
  constexpr int U = JK ? 4 : 1;   // k at a time
#pragma unroll 1
  for (int64_t k = k0; k < k1 && open(); k += U) {
    int at = j;
    // the addresses are found anew each time: kept over the loop they would cost
    // registers that the products need
    asm volatile("" : "+v"(at));
    if constexpr (JK) {
      static_assert(IK && !HELD, "both along k");
      const float *a = (const float *)A.p + i * A.ld + k;
      const bool whole = k + U <= k1;
      float x[U] = {};
      if (whole) __builtin_memcpy(x, a, sizeof x);
      else
        for (int u = 0; u < U - 1; ++u) x[u] = k + u < k1 ? a[u] : 0.0f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float *b = (const float *)B.p + (at + r < J ? at + r : J - 1) * B.ld + k;
        if (whole) {
          float w[U];
          __builtin_memcpy(w, b, sizeof w);
#pragma unroll
          for (int u = 0; u < U; ++u) s[r] = fmaf(x[u], w[u], s[r]);
        } else {
          for (int u = 0; u < U - 1; ++u)
            if (k + u < k1) s[r] = fmaf(x[u], b[u], s[r]);
        }
      }
    } else {
      const float x = ((const float *)A.p)[IK ? i * A.ld + k : k * A.ld + i];
      float w[8];
      if constexpr (HELD) {   // (rows of whole groups)
        unpack8<float>(*reinterpret_cast<const uint2 *>((const uint8_t *)B.p + k * B.ld + at),
                       B.scale[k * (B.ld / 32) + at / 32], B.hold, w);
      } else {
        load8((const float *)B.p + k * B.ld, at, J, w);
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = fmaf(x, w[r], s[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) v[r] = bad >> r & 1 ? s[r] : v[r];
}

// A wave's outputs, rows i0.. and columns j0.., or their parts' sums, sixteen rows at
// a time by way of LDS: there a lane has four columns of a row in each block,
// and eight neighbouring ones for the epilogue, so that a row's outputs are
// written whole.  The residual of the next rows is asked for before these are
// finished.  lds: the wave's own 1 KB per block of columns; the chunks of four
// floats are exchanged by the row's number against bank conflicts
template <class T, int NI, int NJ, bool IK, bool JK, bool HELD, bool LIN>
__device__ __forceinline__ void write_tile(const GemmArgs &a, const v4f (&acc)[NI][NJ], char *lds,
                                           int64_t i0, int64_t j0, int part, int64_t k0,
                                           int64_t k1) {
  constexpr int W = 16 * NJ, CH = W / 4, LPR = W / 8;    // columns, chunks and lanes of a row
  constexpr int RPS = WAVE / LPR, NS = 16 / RPS;         // rows per step, steps
  const int lane = threadIdx.x & (WAVE - 1), c = 2 * (lane % LPR);
  const int64_t j = j0 + 4 * c;
  float4 *buf = reinterpret_cast<float4 *>(lds);
  const bool inner = j < a.J;
  Raw8<T> bias, res[2][NS];
  auto residual = [&](int p) {
    if constexpr (LIN)
      if (a.lin.res)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const int64_t i = i0 + 16 * p + s * RPS + lane / LPR;
          if (i < a.I && inner)
            res[p & 1][s].load((const T *)a.lin.res + i * a.lin.ldr, (int)j, a.J);
        }
  };
  if constexpr (LIN)
    if (a.lin.bias) bias.load((const T *)a.lin.bias, (int)j, a.J);
  residual(0);
#pragma unroll
  for (int p = 0; p < NI; ++p) {
    if (p + 1 < NI) residual(p + 1);
#pragma unroll
    for (int b = 0; b < NJ; ++b) {
      const int row = lane & 15, ch = 4 * b + (lane >> 4);
      buf[row * CH + (ch ^ (row & 7))] =
          make_float4(acc[p][b][0], acc[p][b][1], acc[p][b][2], acc[p][b][3]);
    }
    // a wave's LDS accesses are carried out in order
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int row = s * RPS + lane / LPR;
      const float4 x = buf[row * CH + (c ^ (row & 7))], y = buf[row * CH + ((c + 1) ^ (row & 7))];
      float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      const int64_t i = i0 + 16 * p + row;
      if constexpr (sizeof(T) == 4) {
        uint32_t bad = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) bad |= fabsf(v[r]) < INFINITY ? 0u : 1u << r;
        if (bad && i < a.I)
          plain_chains<IK, JK, HELD>(a.A, a.B, i, (int)j, a.J, k0, k1, bad, v);
      }
      if (a.part) {
        if (i < a.I && j < a.ldp) {
          float4 *o = reinterpret_cast<float4 *>(a.part + ((int64_t)part * a.I + i) * a.ldp + j);
          o[0] = make_float4(v[0], v[1], v[2], v[3]);
          o[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
      } else {
        finish<T, LIN>(a, i, (int)j, i < a.I, v, bias, res[p & 1][s]);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Which tile comes t-th: groups of eight rows of tiles, a group's tiles column by
// column, so that the tiles that are worked on together need few distinct rows of
// either operand (64 tiles: 8 by 8)
__device__ __forceinline__ void tile_at(int64_t t, int64_t ti, int64_t tj, int64_t &i, int64_t &j) {
  const int64_t g = t / (8 * tj), r = t - g * 8 * tj, h = ti - 8 * g < 8 ? ti - 8 * g : 8;
  j = r / h;
  i = 8 * g + r - j * h;
}

// The products of a K-tile in LDS
template <class OA, class OB, int NI, int NJ>
__device__ __forceinline__ void multiply(const char *la, const char *lb, int wi, int wj,
                                         v4f (&acc)[NI][NJ]) {
  constexpr int P = OA::P;
#pragma unroll
  for (int s = 0; s < OA::BK / 32; ++s) {
    typename OA::E8 fi[P][NI], fj[P][NJ];
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
      for (int i = 0; i < NI; ++i) fi[p][i] = OA::frag(la, p, wi + 16 * i, s);
#pragma unroll
      for (int j = 0; j < NJ; ++j) fj[p][j] = OB::frag(lb, p, wj + 16 * j, s);
    }
#pragma unroll
    for (int q = P - 1; q >= 0; --q)       // the small products first
#pragma unroll
      for (int p = 0; p <= q; ++p)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = mma(fj[q - p][j], fi[p][i], acc[i][j]);
  }
}

// A block of 256 threads owns an S x S tile, each wave a quarter of it in blocks of
// 16 x 16.  The next K-tile is read into registers while this one is multiplied.
// Blocks go to the eight XCDs in turn: each XCD takes a run of neighbouring tiles,
// of one part of k after the other, so that their operands meet in its L2 (dw of
// 65,536 rows, 128 x 256, fp32, whose two tiles would otherwise keep to two XCDs: 122
// -> 44 us).  Tiles of 64 x 64 take K-tiles twice as long: what they lack is loads
// under way.  What bounds it, of floats: two barriers a K-tile with the splitting
// between them, the matrix cores busy 53 % of the cycles: 65,536 x 1024 -> 1024 730 to
// 757 us, 182 to 188 TFLOP/s (the library's fp32 product there 142); with the next
// K-tile stored behind the products instead of ahead of them 815.  (A held operand's
// second and third parts are zero and multiplied all the same.)
template <class T, int S>
struct RegTile {
  static constexpr int BK = S == 64 ? 2 * Tile<T>::BK : Tile<T>::BK;
  static constexpr int BYTES = Tile<T>::P * 2 * S * BK * 2;
};
template <class T, int S, bool IK, bool JK, bool HELD, bool LIN>
__device__ __forceinline__ void gemm_body(const GemmArgs &a, char *lds, int64_t block) {
  constexpr int TI = S, TJ = S, BK = RegTile<T, S>::BK;
  typedef Operand<T, TI, IK, false, 256, BK> OA;
  typedef Operand<T, TJ, JK, HELD, 256, BK> OB;
  constexpr int NI = TI / 32, NJ = TJ / 32;
  const int wave = threadIdx.x / WAVE;
  const int wi = TI / 2 * (wave & 1), wj = TJ / 2 * (wave >> 1);
  const int64_t ti = (a.I + TI - 1) / TI, tj = (a.J + TJ - 1) / TJ, tiles = ti * tj;
  const int64_t units = tiles * a.parts, per = (units + 7) / 8;
  for (int64_t u = block; u < 8 * per; u += a.grid) {
    const int64_t unit = (u & 7) * per + (u >> 3);
    if (unit >= units) continue;   // the whole block together
    const int part = (int)(unit / tiles);
    const int64_t k0 = part * a.kchunk, k1 = k0 + a.kchunk < a.K ? k0 + a.kchunk : a.K;
    int64_t i0, j0;
    tile_at(unit - part * tiles, ti, tj, i0, j0);
    i0 *= TI, j0 *= TJ;
    const bool inside = i0 + TI <= a.I && j0 + TJ <= a.J;
    OA fa;
    OB fb;
    auto fetch = [&](int64_t k) {
      if (inside && k + BK <= k1) {
        fa.template fetch<true>(a.A, i0, a.I, k, k1, a.K);
        fb.template fetch<true>(a.B, j0, a.J, k, k1, a.K);
      } else {
        fa.template fetch<false>(a.A, i0, a.I, k, k1, a.K);
        fb.template fetch<false>(a.B, j0, a.J, k, k1, a.K);
      }
    };
    auto stash = [&]() {
      fa.stash(lds, 0);
      fb.stash(lds + OA::BYTES, a.B.hold);
    };
    v4f acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    if (k0 < k1) fetch(k0);
    for (int64_t k = k0; k < k1; k += BK) {
      __syncthreads();   // the K-tile before, and the tile before, have been read
      stash();
      __syncthreads();
      if (k + BK < k1) fetch(k + BK);
      multiply<OA, OB>(lds, lds + OA::BYTES, wi, wj, acc);
    }
    __syncthreads();   // the last K-tile has been read
    write_tile<T, NI, NJ, IK, JK, HELD, LIN>(a, acc, lds + wave * 1024 * NJ, i0 + wi, j0 + wj,
                                             part, k0, k1);
  }
}

template <class T, int S, bool IK, bool JK, bool HELD, bool LIN>
__global__ void __launch_bounds__(256, 2) k_gemm(GemmArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[RegTile<T, S>::BYTES];
  gemm_body<T, S, IK, JK, HELD, LIN>(a, lds, blockIdx.x);
}

// dx and dw in one launch, where both take small tiles
template <class T, bool HELD>
__global__ void __launch_bounds__(256, 2) k_gemm_two(GemmArgs x, GemmArgs w) {
  __shared__ __attribute__((aligned(16))) char lds[RegTile<T, 64>::BYTES];
  if (blockIdx.x < w.grid) gemm_body<T, 64, false, false, HELD, false>(w, lds, blockIdx.x);
  else gemm_body<T, 64, true, false, false, false>(x, lds, blockIdx.x - w.grid);
}

// The same for 16-bit operands whose rows lie on 16-byte boundaries: K-tiles go
// straight from memory into LDS, NB - 1 of them ahead of the products.  Two blocks
// of four waves share a CU, and one reads its operands from LDS, or makes its
// epilogue, while the other multiplies; a block goes on to its next tile with that
// tile's first K-tiles already under way.  128 x 128 tiles take k 64 at a time, whole
// lines of rows that run along k (32 at a time the 8192^3 product took 1053 us, 64
// 945, the library 679 to 707); 256 x 128 tiles, two thirds of the traffic, take 32, for
// products with an operand that runs along its side (dw of 65,536 rows, 4096 x 1024:
// 443 us, 1.24 PFLOP/s, and a join of 8; in 128 x 128 549 with the join.  Its kernel spills
// 24 B a lane at 256 registers).  What bounds it is waits for operands, and the
// epilogue: the matrix cores are busy 40 % of the cycles in 65,536 x 1024 -> 4096, 35 %
// with bias and gelu, 50 % in its dx, 74 % in its dw and 68 % in 8192^3 (the library's
// kernel 93 %), at 1.6 to 2.0 of 2.4 GHz.  Tried and slower: one block of eight waves, 256
// x 256, operands half a K-tile ahead (1141 TFLOP/s at k = 8192, but its epilogue
// stands alone: 740 us for 65,536 x 1024 -> 4096, here 645 to 670); operands from LDS a
// K-tile ahead with 128 x 128 tiles (1003 / 945 us)
template <class T, int TI, int TJ, int BK, int NB, bool IK, bool JK, bool LIN>
__global__ void __launch_bounds__(256, 2) k_gemm_dma(GemmArgs a) {
  constexpr int NI = TI / 32, NJ = TJ / 32;
  typedef Operand<T, TI, IK, false, 256, BK> OA;
  typedef Operand<T, TJ, JK, false, 256, BK> OB;
  typedef typename OA::E8 E8;
  constexpr int BUF = OA::BYTES + OB::BYTES;
  __shared__ __attribute__((aligned(16))) char lds[NB * BUF];
  const uint32_t la = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  const int wave = threadIdx.x / WAVE;
  const int wi = TI / 2 * (wave & 1), wj = TJ / 2 * (wave >> 1);
  const int64_t ti = (a.I + TI - 1) / TI, tj = (a.J + TJ - 1) / TJ, tiles = ti * tj;
  const int64_t units = tiles * a.parts, per = (units + 7) / 8;
  int part = 0;
  int64_t k0 = 0, k1 = 0;       // the unit's
  int in = 0, out = 0;          // LDS buffers to fill and to read next
  int64_t i0 = 0, j0 = 0, left = 0;   // the tile; k of it not yet asked for
  uint32_t oa[OA::N], ob[OB::N];
  const T *pa = nullptr, *pb = nullptr;
  const int64_t sa = IK ? BK : BK * a.A.ld, sb = JK ? BK : BK * a.B.ld;
  auto next = [](int &b) { b = b == (NB - 1) * BUF ? 0 : b + BUF; };
  auto fetch = [&](auto full) {
    OA::template dma<decltype(full)::value>(pa, oa, la + in, (int)left);
    OB::template dma<decltype(full)::value>(pb, ob, la + in + OA::BYTES, (int)left);
    pa += sa;
    pb += sb;
    left -= BK;
    next(in);
  };
  auto fetch_any = [&]() {
    if (left >= BK) fetch(std::true_type{});
    else if (left > 0) fetch(std::false_type{});
  };
  // the block's next unit from its u-th on (-1: none left), its first NB - 1 K-tiles
  // asked for
  auto begin = [&](int64_t u) -> int64_t {
    for (; u < 8 * per; u += a.grid) {
      const int64_t unit = (u & 7) * per + (u >> 3);
      if (unit >= units) continue;
      part = (int)(unit / tiles);
      k0 = part * a.kchunk;
      k1 = k0 + a.kchunk < a.K ? k0 + a.kchunk : a.K;
      tile_at(unit - part * tiles, ti, tj, i0, j0);
      i0 *= TI, j0 *= TJ;
      OA::dma_offsets(a.A, i0, a.I, oa);
      OB::dma_offsets(a.B, j0, a.J, ob);
      pa = (const T *)a.A.p + (IK ? i0 * a.A.ld + k0 : k0 * a.A.ld + i0);
      pb = (const T *)a.B.p + (JK ? j0 * a.B.ld + k0 : k0 * a.B.ld + j0);
      left = k1 - k0;
#pragma unroll
      for (int b = 1; b < NB; ++b) fetch_any();
      return u;
    }
    return -1;
  };
  // the wave's own reads into LDS are done but for the last `but`, its reads of
  // LDS too; then the other waves' as well
  auto arrived = [](auto but) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(but)::value) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  std::integral_constant<int, 0> ALL;
  std::integral_constant<int, (NB - 2) * (OA::N + OB::N)> BUT_LAST;
  int64_t u = begin(blockIdx.x);
  while (u >= 0) {
    v4f acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&]() {
      constexpr int H = BK / 32;
      E8 fi[H][NI], fj[H][NJ];
#pragma unroll
      for (int s = 0; s < H; ++s) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) fj[s][j] = OB::frag(lds + out + OA::BYTES, 0, wj + 16 * j, s);
#pragma unroll
        for (int i = 0; i < NI; ++i) fi[s][i] = OA::frag(lds + out, 0, wi + 16 * i, s);
      }
      __builtin_amdgcn_sched_barrier(0);
      // the wave that multiplies before the other block's: dw of 65,536 rows, 4096 x
      // 1024, 505 -> 450 us, dx 568 -> 555 (128 x 128 tiles lose 1 %)
      if constexpr (TI == 256) __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int s = 0; s < H; ++s)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = mma(fj[s][j], fi[s][i], acc[i][j]);
      if constexpr (TI == 256) __builtin_amdgcn_s_setprio(0);
      next(out);
    };
    const int64_t nk = (k1 - k0 + BK - 1) / BK;
    int64_t n = 0;
    while (left >= BK) {   // a whole K-tile is still to be asked for
      arrived(BUT_LAST);
      fetch(std::true_type{});
      multiply();
      ++n;
    }
    for (; n < nk; ++n) {   // the last ones
      arrived(ALL);
      fetch_any();
      multiply();
    }
    arrived(ALL);   // the last K-tile has been read
    // the next tile's first K-tiles come while this one is finished; the third
    // buffer is free for that
    const int64_t i1 = i0 + wi, j1 = j0 + wj, ka = k0, kb = k1;
    const int done = part;
    u = begin(u + a.grid);
    write_tile<T, NI, NJ, IK, JK, false, LIN>(a, acc, lds + in + wave * 1024 * NJ, i1, j1, done,
                                              ka, kb);
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): nothing is under way into registers
  }
}

// The parts' sums and the epilogue, eight columns of a row per thread.  Many parts
// are added by four waves, every fourth part each (their loads wait for one
// another), whose sums the first then adds in order
constexpr int JOIN_ONE = 8;   // parts that one thread adds
template <class T, bool LIN>
__device__ __forceinline__ void join_body(const GemmArgs &a, int64_t block, int64_t blocks) {
  __shared__ float4 red[3][2][WAVE];
  const int64_t per = a.ldp / 8, units = a.I * per;   // whole quads per row
  const bool four = a.parts > JOIN_ONE;
  const int chain = four ? threadIdx.x / WAVE : 0, step = four ? 4 : 1;
  const int width = four ? WAVE : 256, at = threadIdx.x % width;
  for (int64_t u0 = block * width; u0 < units; u0 += blocks * width) {
    const int64_t u = u0 + at, i = u / per;
    const int j = (int)(u - i * per) * 8;
    float v[8] = {};
    Raw8<T> bias, res;
    if (u < units) {
      if constexpr (LIN) {
        if (a.lin.bias) bias.load((const T *)a.lin.bias, j, a.J);
        if (a.lin.res) res.load((const T *)a.lin.res + i * a.lin.ldr, j, a.J);
      }
#pragma unroll 4
      for (int s = chain; s < a.parts; s += step) {
        const float4 *p =
            reinterpret_cast<const float4 *>(a.part + ((int64_t)s * a.I + i) * a.ldp + j);
        const float4 x = p[0], y = p[1];
        v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
      }
    }
    if (four) {
      __syncthreads();   // the units before have been added
      if (chain > 0) {
        red[chain - 1][0][at] = make_float4(v[0], v[1], v[2], v[3]);
        red[chain - 1][1][at] = make_float4(v[4], v[5], v[6], v[7]);
      }
      __syncthreads();
      if (chain > 0) continue;
#pragma unroll
      for (int c = 0; c < 3; ++c) {
        const float4 x = red[c][0][at], y = red[c][1][at];
        v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
      }
    }
    if (u < units) finish<T, LIN>(a, i, j, true, v, bias, res);
  }
}

template <class T>
__global__ void __launch_bounds__(256) k_linear_join(GemmArgs a) {
  join_body<T, true>(a, blockIdx.x, gridDim.x);
}

// rows of d elements with a stride of ld, as rows with a stride of ldo (a multiple
// of 8), zeros behind d
template <class T>
__global__ void __launch_bounds__(256) k_pad_rows(const T *x, int64_t ld, int64_t m, int d, T *out,
                                                  int64_t ldo) {
  const int64_t per = ldo / 8, units = m * per;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units;
       u += (int64_t)gridDim.x * 256) {
    const int64_t r = u / per;
    const int c = (int)(u - r * per) * 8;
    Raw8<T> v;
    v.load(x + r * ld, c, d);
    *reinterpret_cast<typename Raw8<T>::t8 *>(out + r * ldo + c) = v.v;
  }
}

// What is left of the gradients: bx blocks join dx, bw join dw, the others add up
// the column sums of dz, sixteen columns each (sixteen threads of a column add
// every sixteenth row, then the sixteen sums in order)
template <class T>
__global__ void __launch_bounds__(256) k_grad_join(GemmArgs x, GemmArgs w, int64_t bx, int64_t bw,
                                                   const float *cols, int64_t rows, int n, T *db) {
  __shared__ float red[16][17];
  int64_t b = blockIdx.x;
  if (b < bx + bw) {
    const bool first = b < bx;
    return join_body<T, false>(first ? x : w, first ? b : b - bx, first ? bx : bw);
  }
  b -= bx + bw;
  const int c = (int)b * 16 + (threadIdx.x & 15), q = threadIdx.x >> 4;
  float v = 0.0f;
  if (c < n) {
#pragma unroll 8
    for (int64_t r = q; r < rows; r += 16) v += cols[r * n + c];
  }
  red[q][threadIdx.x & 15] = v;
  __syncthreads();
  if (q == 0 && c < n) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += red[i][threadIdx.x];
    db[c] = from_f32<T>(v);
  }
}

constexpr int ACT_THREADS = 512;
// dz = dy act'(pre) of `rows` rows per block, rounded to the type, zeros from n up to
// ldz (a multiple of 32; dz NULL: not wanted), and its column sums over them (part
// NULL: not wanted).  The threads are ACT_THREADS / ct rows of ct threads, eight
// columns each.
// The rounding of dz is a choice.  In the 16-bit types it is an operand of the matrix
// cores, which take 16 bits, as every tensor of such a network between two of its
// layers is; the column sums take it unrounded.  It adds one rounding of independent
// size to that of the outputs themselves: dx and dw of a bf16 gelu layer are 0.0024 off
// in the 2-norm (fp16 0.00030), where rounding exact ones gives 0.0017 (0.00021); z, kept in
// the type too, has 0.0001 of that.  dz in two parts (it and the rest, both in the type),
// was measured: 0.0017 again, for 16,384 x 1024 -> 1024 with gelu 108 -> 167 us, 65,536 x
// 1024 -> 4096 1306 -> 2302, in the product of dx alone 111 -> 147 and 1330 -> 1970.  With no
// activation and with relu dz is exact (dy or 0)
template <class T>
__global__ void __launch_bounds__(ACT_THREADS) k_act_grad(LinearGradArgs a, int64_t rows, int ct,
                                                          T *dz, int64_t ldz, float *part) {
  __shared__ float red[ACT_THREADS][9];
  constexpr bool exact = sizeof(T) == 4;
  const int tc = threadIdx.x % ct, tr = threadIdx.x / ct, rt = ACT_THREADS / ct;
  const int c0 = (blockIdx.y * ct + tc) * 8;
  const int64_t r0 = (int64_t)blockIdx.x * rows, r1 = r0 + rows < a.m ? r0 + rows : a.m;
  float s[8] = {};
  constexpr int B = 4;   // rows under way
  if (c0 < ldz)
    for (int64_t r = r0 + tr; r < r1; r += B * rt) {
      Raw8<T> v[B], z[B];
      uint2 zq[B];
      uint8_t zs[B];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int64_t rb = r + b * rt < r1 ? r + b * rt : r;
        v[b].load((const T *)a.dy + rb * a.lddy, c0, a.n);
        if (a.act == NR_ACT_NONE) continue;
        if (a.pre.hold) {   // (its rows are padded as dz's are)
          zq[b] = *reinterpret_cast<const uint2 *>((const uint8_t *)a.pre.p + rb * a.pre.ld + c0);
          zs[b] = a.pre.scale[rb * (a.pre.ld / 32) + (c0 >> 5)];
        } else {
          z[b].load((const T *)a.pre.p + rb * a.pre.ld, c0, a.n);
        }
      }
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if (r + b * rt >= r1) break;
        float d[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = v[b][i];
        if (a.act != NR_ACT_NONE) {
          if (a.pre.hold) {
            unpack8<T>(zq[b], zs[b], a.pre.hold, y);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = z[b][i];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] *= act_slope<exact>(y[i], a.act);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[i] = c0 + i < a.n ? d[i] : 0.0f;   // (a slope of what is behind the width)
          s[i] += d[i];
        }
        if (dz) store8(dz + (r + b * rt) * ldz, c0, (int)ldz, d);
      }
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

// How a product is cut: the tile's side (256: 256 x 128), and parts of k.  The
// cheapest by an estimate of its time in us, from what was measured on MI355X: a
// block takes its tile's products at `rate` / 256 (TFLOP/s) where blocks share a
// CU, at `alone` / 256 where it has one to itself, but at least `step` for each
// K-tile of bk, and all of them together the operands' bytes at `stream` TB/s;
// parts cost a launch, and their sums' way through memory.  Measured, us, the
// chosen one last: y of 10,000 x 1536 -> 512 fp32 in 128 x 128 156, 64 x 64 129, 128 x
// 128 in four parts 114; bf16 700 x 2000 -> 900 64 x 64 36, 128 x 128 25, in four parts
// 18; 4096 x 512 -> 512 128 x 128 13, 64 x 64 9.5; 48 x 4096 -> 4096 64 x 64 in eight
// parts 18.6, 128 x 128 in eight 14.7; 16,384 x 512 -> 512 64 x 64 24, 128 x 128 17.4; dx of
// 65,536 x 4096 -> 1024 128 x 128 578, 256 x 128 560; dw of 65,536 rows, 4096 x 1024, 128 x
// 128 in two parts 549, 256 x 128 in four 452
enum { PROD_Y, PROD_DX, PROD_DW };
struct Split {
  int side, parts;
  int64_t kchunk;
  double us;   // the estimate, without a launch's fixed time
};
static Split split_of(int64_t I, int J, int64_t K, int dtype, int prod, bool large = true) {
  struct Kind {
    int side, ti, tj, bk;
    double rate, alone, step, stream;
  };
  const double small = prod == PROD_DW ? 280 : 390;
  static constexpr Kind f32[2] = {{64, 64, 64, 64, 130, 105, 1.6, 2.9},
                                  {128, 128, 128, 32, 190, 110, 1.8, 2.9}};
  // (256 x 128 only where an operand is read along its side: 32 of k of a row that
  // runs along k are half a line)
  const Kind h16[3] = {{256, 256, 128, 32, 1000, 830, 0.45, 4.0},
                       {128, 128, 128, 64, 950, 850, 0.85, 4.0},
                       {64, 64, 64, 128, small, 0.8 * small, 1.5, 2.9}};
  // !large: 16-bit operands that cannot go straight into LDS
  const int skip = !large ? 2 : prod == PROD_Y ? 1 : 0;
  const Kind *kind = dtype == NR_F32 ? f32 : h16 + skip;
  const int kinds = dtype == NR_F32 ? 2 : 3 - skip;
  const double mbytes = 1e-6 * (dtype == NR_F32 ? 4 : 2) * ((double)I + J) * (double)K;
  Split best{64, 1, 128, INFINITY};
  for (int q = 0; q < kinds; ++q, ++kind) {
    const double tiles =
        (double)(up(I, kind->ti) / kind->ti) * (double)(up(J, kind->tj) / kind->tj);
    for (int want = 1; want <= 256; want *= 2) {
      if (want > 1 && (K < 256 * want || tiles * want > 2048)) break;
      const int64_t kc = K > 0 ? up((K + want - 1) / want, 128) : 128;
      const int parts = K > 0 ? (int)((K + kc - 1) / kc) : 1;
      const double block = 2e-6 * 256 * kind->ti * kind->tj * kc;
      const int64_t per_cu = (int64_t)((tiles * parts + 255) / 256);
      const double busy = per_cu / 2 * 2 * block / kind->rate + per_cu % 2 * block / kind->alone;
      const double wait = (per_cu + 1) / 2 * kind->step * (double)((kc + kind->bk - 1) / kind->bk);
      const double us = std::fmax(std::fmax(busy, wait), mbytes / kind->stream) +
                        (parts > 1 ? 5.0 + 1.25e-6 * parts * (double)I * J : 0.0);
      if (us < best.us) best = Split{kind->side, parts, kc, us};
    }
  }
  return best;
}
static size_t part_bytes(const Split &sp, int64_t I, int J) {
  return sp.parts > 1 ? up(sizeof(float) * (size_t)sp.parts * I * up(J, 32), 256) : 0;
}

// an operand that can go straight into LDS: whole chunks (or zeros up to the row
// stride) in rows on 16-byte boundaries, a tile of them within 2^32 bytes
static bool direct(const LayerMat &m, int64_t width) {
  return !m.hold && aligned(m.p, m.ld, 2, 16) && m.ld < (int64_t)1 << 22 &&
         (width % 8 == 0 || m.padded);
}

// Rows that lie off the 16-byte boundaries can be read, but not straight into LDS,
// and a load across two lines costs two: us of bf16 products in 64 x 64 tiles at widths
// of 1024 / 1023, 16,384 rows: y 70 / 119, dx 74 / 108, dw 71 / 170.  So 16-bit operands are
// copied to padded rows first (k_pad_rows: 4 us, and 4 bytes an element at some 5
// TB/s) where large tiles with the copies are estimated to be faster than small
// ones by way of registers, which take half as long again for such rows, and twice
// as long where they run along the side: us with copies / without, y of 65,536 x
// 1001 -> 301 112 / 145, 2000 x 1001 -> 2001 31 / 44, its dx 34 / 62, dw 33 / 64; dw of
// 16,384 x 333 -> 300 33 / 34.  Rows that are off only because the matrix starts off
// (all by the same bytes, their chunks whole) cost the small tiles less: 10 us and, next
// to their estimate, 1.0 (y), 0.9 (dx) or 0.75 (dw) of it with one such operand, 1.3, 1.2
// and 0.97 with two (measured at 17 sizes from 1000 x 2048 -> 2048 on).  us with copies /
// without, of 16,384 x 1024 -> 1024: x off y 57 / 92, dw 55 / 97; w off y 48 / 84, dx 41 /
// 82; all of them off 61 / 122, 52 / 120, 67 / 130; dw of 65,536 rows, 256 x 1024, x off
// 102 / 90, of 100,000 rows, 128 x 512, 61 / 43
enum { ON_LINES, OFF_START, OFF_ROWS };
static int off_lines(const LayerMat &m, int64_t width) {
  if (direct(m, width)) return ON_LINES;
  LayerMat at0 = m;
  at0.p = nullptr;
  return direct(at0, width) ? OFF_START : OFF_ROWS;
}
static bool copies_pay(const Split &large, const Split &small, int prod, int off_a, int off_b,
                       int64_t elements) {
  static constexpr double rows[3] = {1.4, 2.0, 2.0}, one[3] = {1.0, 0.9, 0.75},
                          two[3] = {1.3, 1.2, 0.97};   // by product
  const int copies = (off_a != ON_LINES) + (off_b != ON_LINES);
  const double without = off_a == OFF_ROWS || off_b == OFF_ROWS
                             ? rows[prod] * small.us
                             : 10.0 + (copies == 1 ? one[prod] : two[prod]) * small.us;
  return large.us + 4.0 * copies + 8e-7 * (double)elements < without;
}

static int64_t tile_grid(const GemmArgs &a, int ti, int tj) {
  const int64_t n = up(up(a.I, ti) / ti * (up(a.J, tj) / tj) * a.parts, 8);
  return n < 1 << 20 ? n : 1 << 20;   // blocks take further tiles in turn
}

static void place(GemmArgs &a, const Split &sp, void *ws) {
  a.kchunk = sp.kchunk;
  a.parts = sp.parts;
  a.part = sp.parts > 1 ? (float *)ws : nullptr;
  a.ldp = up(a.J, 32);
}
static int64_t join_blocks(const GemmArgs &a) {
  if (a.parts < 2) return 0;
  const int64_t width = a.parts > JOIN_ONE ? WAVE : 256;
  const int64_t b = (a.I * (a.ldp / 8) + width - 1) / width;
  return b < 1 << 20 ? b : 1 << 20;
}

template <class T, int S, bool IK, bool JK, bool LIN>
static void gemm_reg(GemmArgs &a, hipStream_t s) {
  a.grid = tile_grid(a, S, S);
  const dim3 g((unsigned)a.grid);
  if constexpr (!IK) {
    if (a.B.hold) {
      hipLaunchKernelGGL((k_gemm<T, S, IK, JK, true, LIN>), g, dim3(256), 0, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((k_gemm<T, S, IK, JK, false, LIN>), g, dim3(256), 0, s, a);
}

template <class T, bool IK, bool JK, bool LIN>
static void gemm(GemmArgs &a, int side, hipStream_t s) {
  if (a.I <= 0) return;
  if constexpr (sizeof(T) == 2) {
    if (side >= 128 && direct(a.A, IK ? a.K : a.I) && direct(a.B, JK ? a.K : a.J)) {
      const int64_t n = tile_grid(a, side, 128);
      a.grid = n < 512 ? n : 512;   // two blocks a CU
      const dim3 g((unsigned)a.grid);
      if constexpr (!JK) {
        if (side == 256) {
          hipLaunchKernelGGL((k_gemm_dma<T, 256, 128, 32, 3, IK, JK, LIN>), g, dim3(256), 0, s, a);
          return;
        }
      }
      hipLaunchKernelGGL((k_gemm_dma<T, 128, 128, 64, 2, IK, JK, LIN>), g, dim3(256), 0, s, a);
      return;
    }
  }
  if constexpr (sizeof(T) == 4) {
    if (side == 128) {
      gemm_reg<T, 128, IK, JK, LIN>(a, s);
      return;
    }
  }
  gemm_reg<T, 64, IK, JK, LIN>(a, s);
}

// Work space of the forward pass: copies of x and w with padded rows, and the parts
struct LinearPlan {
  Split sp;
  bool copy_x, copy_w;   // 16-bit operands of large tiles that cannot go straight into LDS
  size_t at_w, at_part, bytes;
};
static LayerMat plain_mat(const void *p, int64_t ld) { return LayerMat{p, ld, 0, nullptr, false}; }
static LinearPlan linear_plan(const LinearArgs &a, int dtype) {
  LinearPlan p{};
  p.sp = split_of(a.m, a.n, a.k, dtype, PROD_Y);
  const int x_off = off_lines(plain_mat(a.x, a.ldx), a.k);
  const int w_off = off_lines(plain_mat(a.w, a.ldw), a.k);
  if (dtype != NR_F32 && a.m > 0 && p.sp.side >= 128 && (x_off || w_off)) {
    const Split small = split_of(a.m, a.n, a.k, dtype, PROD_Y, false);
    const bool pay = copies_pay(p.sp, small, PROD_Y, x_off, w_off,
                                ((x_off ? a.m : 0) + (w_off ? a.n : 0)) * a.k);
    p.copy_x = pay && x_off;
    p.copy_w = pay && w_off;
    if (!pay) p.sp = small;
  }
  const int64_t ldk = up(a.k, 32);
  size_t off = 0;
  if (p.copy_x) off += up((size_t)a.m * ldk * 2, 256);
  p.at_w = off;
  if (p.copy_w) off += up((size_t)a.n * ldk * 2, 256);
  p.at_part = off;
  p.bytes = off + part_bytes(p.sp, a.m, a.n);
  return p;
}

size_t linear_ws(const LinearArgs &a, int dtype) { return linear_plan(a, dtype).bytes; }

template <class T>
static LayerMat padded(const void *x, int64_t ld, int64_t m, int d, char *at, hipStream_t s) {
  const int64_t ldo = up(d, 32), blocks = (m * (ldo / 8) + 255) / 256;
  hipLaunchKernelGGL(k_pad_rows<T>, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)),
                     dim3(256), 0, s, (const T *)x, ld, m, d, (T *)at, ldo);
  return LayerMat{at, ldo, 0, nullptr, true};
}

template <class T>
static hipError_t linear_t(const LinearArgs &l, int dtype, char *ws, hipStream_t s) {
  if (l.m <= 0) return hipSuccess;
  const LinearPlan p = linear_plan(l, dtype);
  GemmArgs a{};
  a.I = l.m, a.J = l.n, a.K = l.k;
  a.A = plain_mat(l.x, l.ldx);
  a.B = plain_mat(l.w, l.ldw);
  if (p.copy_x) a.A = padded<T>(l.x, l.ldx, l.m, l.k, ws, s);
  if (p.copy_w) a.B = padded<T>(l.w, l.ldw, l.n, l.k, ws + p.at_w, s);
  a.lin = l;
  place(a, p.sp, ws + p.at_part);
  gemm<T, true, true, true>(a, p.sp.side, s);
  if (a.parts > 1)
    hipLaunchKernelGGL(k_linear_join<T>, dim3((unsigned)join_blocks(a)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == NR_F32) return linear_t<float>(a, dtype, (char *)ws, s);
  if (dtype == NR_BF16) return linear_t<bf16_t>(a, dtype, (char *)ws, s);
  return linear_t<f16_t>(a, dtype, (char *)ws, s);
}

// Work space of the gradients: dz, the column sums of its blocks, copies of w and x
// with padded rows, and the parts of the two products
struct GradPlan {
  Split sx, sw;
  bool act, dz;          // the pass over dy runs; it writes dz
  int64_t rows, nb, ldz; // rows per block of that pass, its blocks, dz's row stride
  int ct;
  bool copy_w, copy_x;
  size_t at_cols, at_cw, at_cx, at_x, at_w, bytes;
};
static GradPlan grad_plan(const LinearGradArgs &a, int dtype) {
  GradPlan p{};
  // dz is written where it is another than dy, and as a padded copy of dy; w is
  // copied for dx, x (or what is held of it) for dw
  if (a.dx) p.sx = split_of(a.m, a.k, a.n, dtype, PROD_DX);
  if (a.dw) p.sw = split_of(a.n, a.k, a.m, dtype, PROD_DW);
  p.dz = a.act != NR_ACT_NONE && (a.dx || a.dw);
  const bool h16 = dtype != NR_F32 && a.m > 0;
  const int z_off = p.dz ? ON_LINES : off_lines(plain_mat(a.dy, a.lddy), a.n);
  auto choose = [&](Split &sp, int64_t I, int J, int64_t K, int prod, int off, int64_t elements) {
    if (!h16 || sp.side < 128 || !(z_off || off)) return false;
    const Split small = split_of(I, J, K, dtype, prod, false);
    if (copies_pay(sp, small, prod, z_off, off, (z_off ? a.m * a.n : 0) + (off ? elements : 0)))
      return true;
    sp = small;
    return false;
  };
  const int w_off = off_lines(plain_mat(a.w, a.ldw), a.k), x_off = off_lines(a.x, a.k);
  const bool cx = a.dx && choose(p.sx, a.m, a.k, a.n, PROD_DX, w_off, (int64_t)a.n * a.k);
  const bool cw = a.dw && choose(p.sw, a.n, a.k, a.m, PROD_DW, x_off, a.m * a.k);
  p.copy_w = cx && w_off;
  p.copy_x = cw && x_off;
  if (z_off && (cx || cw)) p.dz = true;
  p.act = p.dz || a.db;
  p.ct = 4;   // whole groups of 32 columns
  while (p.ct < 256 && p.ct * 8 < a.n) p.ct *= 2;
  // blocks of the pass: some thousand in all, at most 512 of them along the rows
  const int64_t rt = ACT_THREADS / p.ct, across = (a.n + 8 * p.ct - 1) / (8 * p.ct);
  int64_t blocks = 1024 / across;
  blocks = blocks > 512 ? 512 : blocks;
  p.rows = up((a.m + blocks - 1) / blocks, 4 * rt);
  if (a.m < blocks * 4 * rt) p.rows = up((a.m + 255) / 256, rt);   // few rows: spread them
  if (p.rows < rt) p.rows = rt;
  p.nb = (a.m + p.rows - 1) / p.rows;
  p.ldz = up(a.n, 32);
  size_t off = 0;
  if (p.dz) off += up((size_t)a.m * p.ldz * layer_elem(dtype), 256);
  p.at_cols = off;
  if (a.db) off += up(sizeof(float) * (size_t)p.nb * a.n, 256);
  p.at_cw = off;
  if (p.copy_w) off += up((size_t)a.n * up(a.k, 32) * 2, 256);
  p.at_cx = off;
  if (p.copy_x) off += up((size_t)a.m * up(a.k, 32) * 2, 256);
  p.at_x = off;
  if (a.dx) off += part_bytes(p.sx, a.m, a.k);
  p.at_w = off;
  if (a.dw) off += part_bytes(p.sw, a.n, a.k);
  p.bytes = off;
  return p;
}

size_t linear_grad_ws(const LinearGradArgs &a, int dtype) { return grad_plan(a, dtype).bytes; }

template <class T>
static hipError_t linear_grad_t(const LinearGradArgs &l, int dtype, char *ws, hipStream_t s) {
  const GradPlan p = grad_plan(l, dtype);
  T *dz = p.dz ? (T *)ws : nullptr;
  float *cols = l.db ? (float *)(ws + p.at_cols) : nullptr;
  if (p.act && l.m > 0) {
    const dim3 g((unsigned)p.nb, (l.n + 8 * p.ct - 1) / (8 * p.ct));
    hipLaunchKernelGGL(k_act_grad<T>, g, dim3(ACT_THREADS), 0, s, l, p.rows, p.ct, dz, p.ldz, cols);
  }
  const LayerMat z = p.dz ? LayerMat{dz, p.ldz, 0, nullptr, true} : plain_mat(l.dy, l.lddy);
  GemmArgs x{}, w{};
  x.I = l.m, x.J = l.k, x.K = l.n;
  x.A = z, x.B = plain_mat(l.w, l.ldw);
  x.out = l.dx, x.ldo = l.lddx;
  w.I = l.n, w.J = l.k, w.K = l.m;
  w.A = z, w.B = l.x;
  w.out = l.dw, w.ldo = l.lddw;
  const bool dx = l.dx && l.m > 0, dw = l.dw;
  if (dx) place(x, p.sx, ws + p.at_x);
  if (dw) place(w, p.sw, ws + p.at_w);
  if (p.copy_w) x.B = padded<T>(l.w, l.ldw, l.n, l.k, ws + p.at_cw, s);
  if (p.copy_x && l.x.hold) {
    const int64_t ld = up(l.k, 32);   // its padding is zeros
    const hipError_t e = launch_read((const uint8_t *)l.x.p, l.x.scale, l.m, (int)ld, l.x.hold,
                                     dtype, ws + p.at_cx, ld, s);
    if (e != hipSuccess) return e;
    w.B = LayerMat{ws + p.at_cx, ld, 0, nullptr, true};
  } else if (p.copy_x) {
    w.B = padded<T>(l.x.p, l.x.ld, l.m, l.k, ws + p.at_cx, s);
  }
  if (dx && dw && p.sx.side == 64 && p.sw.side == 64) {
    x.grid = tile_grid(x, 64, 64), w.grid = tile_grid(w, 64, 64);
    const dim3 g((unsigned)(x.grid + w.grid));
    if (w.B.hold) hipLaunchKernelGGL((k_gemm_two<T, true>), g, dim3(256), 0, s, x, w);
    else hipLaunchKernelGGL((k_gemm_two<T, false>), g, dim3(256), 0, s, x, w);
  } else {
    if (dx) gemm<T, true, false, false>(x, p.sx.side, s);
    if (dw) gemm<T, false, false, false>(w, p.sw.side, s);
  }
  const int64_t bx = dx ? join_blocks(x) : 0, bw = dw ? join_blocks(w) : 0;
  const int64_t bc = l.db ? (l.n + 15) / 16 : 0;
  if (bx + bw + bc > 0)
    hipLaunchKernelGGL(k_grad_join<T>, dim3((unsigned)(bx + bw + bc)), dim3(256), 0, s, x, w, bx,
                       bw, cols, p.nb, l.n, (T *)l.db);
  return hipGetLastError();
}

hipError_t launch_linear_grad(const LinearGradArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == NR_F32) return linear_grad_t<float>(a, dtype, (char *)ws, s);
  if (dtype == NR_BF16) return linear_grad_t<bf16_t>(a, dtype, (char *)ws, s);
  return linear_grad_t<f16_t>(a, dtype, (char *)ws, s);
}

}  // namespace nr
