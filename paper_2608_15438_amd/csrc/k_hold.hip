// Activations in 8 bits between a forward pass and its backward pass.  A row is
// cut into groups of 32; a group is held as q 2^e with one power of two, so
// that q 2^e is exact in fp32 and bf16 and the backward pass multiplies by just
// what was held.  A thread takes eight elements (16 bytes of a 16-bit type), four
// lanes a group; the largest magnitude meets in two VALU exchanges.  Memory bounds
// both: 65,536 x 1536 bf16 62 us in, 54 us out (305 MB each, 4.9 and 5.7 TB/s).
#include "nr_layers.h"

namespace nr {

template <class T>
__global__ void __launch_bounds__(256) k_act_hold(const T *x, int64_t ldx, int64_t m, int d,
                                                  int hold, uint8_t *q, uint8_t *scale) {
  const int64_t ldq = (d + 31) / 32 * 32;
  const int64_t units = m * (ldq / 8), step = (int64_t)gridDim.x * 256;
  // a multiple of four units per row: the lanes of a group leave the loop together
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += step) {
    const int64_t row = u / (ldq / 8);
    const int c0 = (int)(u - row * (ldq / 8)) * 8;
    float v[8];
    load8(x + row * ldx, c0, d, v);
    write8(q + row * ldq, scale + row * (ldq / 32), c0, hold, __is_same(T, f16_t),
           v);
  }
}

template <class T>
__global__ void __launch_bounds__(256) k_act_read(const uint8_t *q, const uint8_t *scale,
                                                  int64_t m, int d, int hold, T *y, int64_t ldy) {
  const int64_t ldq = (d + 31) / 32 * 32;
  const int64_t units = m * (ldq / 8), step = (int64_t)gridDim.x * 256;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += step) {
    const int64_t row = u / (ldq / 8);
    const int c0 = (int)(u - row * (ldq / 8)) * 8;
    float v[8];
    read8<T>(q + row * ldq, scale + row * (ldq / 32), c0, hold, v);
    store8(y + row * ldy, c0, d, v);
  }
}

static unsigned hold_grid(int64_t m, int d) {
  const int64_t blocks = (m * (hold_ld(d) / 8) + 255) / 256;
  return (unsigned)(blocks < 1 << 20 ? blocks : 1 << 20);
}

template <class T>
static hipError_t hold_t(const void *x, int64_t ldx, int64_t m, int d, int hold, uint8_t *q,
                         uint8_t *scale, hipStream_t s) {
  hipLaunchKernelGGL(k_act_hold<T>, dim3(hold_grid(m, d)), dim3(256), 0, s, (const T *)x, ldx, m,
                     d, hold, q, scale);
  return hipGetLastError();
}

template <class T>
static hipError_t read_t(const uint8_t *q, const uint8_t *scale, int64_t m, int d, int hold,
                         void *y, int64_t ldy, hipStream_t s) {
  hipLaunchKernelGGL(k_act_read<T>, dim3(hold_grid(m, d)), dim3(256), 0, s, q, scale, m, d, hold,
                     (T *)y, ldy);
  return hipGetLastError();
}

hipError_t launch_hold(const void *x, int64_t ldx, int64_t m, int d, int dtype, int hold,
                       uint8_t *q, uint8_t *scale, hipStream_t s) {
  if (m <= 0) return hipSuccess;
  if (dtype == NR_F32) return hold_t<float>(x, ldx, m, d, hold, q, scale, s);
  if (dtype == NR_BF16) return hold_t<bf16_t>(x, ldx, m, d, hold, q, scale, s);
  return hold_t<f16_t>(x, ldx, m, d, hold, q, scale, s);
}

hipError_t launch_read(const uint8_t *q, const uint8_t *scale, int64_t m, int d, int hold,
                       int dtype, void *y, int64_t ldy, hipStream_t s) {
  if (m <= 0) return hipSuccess;
  if (dtype == NR_F32) return read_t<float>(q, scale, m, d, hold, y, ldy, s);
  if (dtype == NR_BF16) return read_t<bf16_t>(q, scale, m, d, hold, y, ldy, s);
  return read_t<f16_t>(q, scale, m, d, hold, y, ldy, s);
}

}  // namespace nr
