// Rows to 8-bit blocks and back, and weights packed for the block products (the rule
// and the layouts are in pod_block8.h).
//
// Both conversions are streams: 4 or 2 bytes an entry on one side, 1 + 1/128 on the
// other.  Sixteen lanes own a block of a row, eight consecutive entries each, so a
// wavefront reads four blocks with two 16-byte loads a lane (fp32), finds each maximum
// with four exchanges and writes 8 bytes a lane.  65536 rows of 3001 in fp32: stored in 228 us (4.3 TB/s, rows of an odd
// number of floats straddle lines), restored to bf16 in 110 us (5.4 TB/s; a large copy reaches 5.15).
#include "pod_block8.h"

namespace pod {
namespace b8 {
namespace {

// The (row, block) pairs a group of sixteen lanes works on: `first`, first + step, ...
struct Units {
  int64_t row, row_step;
  int32_t blk, blk_step, nb;
  __device__ Units(int64_t first, int64_t step, int32_t nb) : nb(nb) {
    row = first / nb, blk = (int32_t)(first - row * nb);
    row_step = step / nb, blk_step = (int32_t)(step - row_step * nb);
  }
  __device__ void next() {
    row += row_step, blk += blk_step;
    if (blk >= nb) blk -= nb, ++row;
  }
};

template <class T>
__global__ __launch_bounds__(256) void block8_store_kernel(int64_t rows, int32_t cols, int32_t nb, const T *__restrict__ x,
                                                           int64_t ldx, uint8_t *__restrict__ q, uint8_t *__restrict__ scale) {
  const int lane = threadIdx.x & 15, at = 8 * lane;
  const int64_t groups = (int64_t)gridDim.x * 16;
  Units u((int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), groups, nb);
  for (; u.row < rows; u.next()) {  // (the sixteen lanes of a group leave together)
    float v[8];
    load_row<8>(v, x + u.row * ldx, u.blk * kBlock + at, cols, (u.blk + 1) * kBlock <= cols);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, finite_bits(v[i]));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 16));
    const int e = exponent_of(m);
    const float inv = power(-e);
    const u32x2 c = {codes4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), codes4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
    *reinterpret_cast<u32x2 *>(q + (u.row * nb + u.blk) * kBlock + at) = c;
    if (lane == 0) scale[u.row * nb + u.blk] = (uint8_t)(e + 127);
  }
}

template <class T>
__global__ __launch_bounds__(256) void block8_restore_kernel(int64_t rows, int32_t cols, int32_t nb, const uint8_t *__restrict__ q,
                                                             const uint8_t *__restrict__ scale, T *__restrict__ y, int64_t ldy) {
  const int at = 8 * (threadIdx.x & 15);
  const int64_t groups = (int64_t)gridDim.x * 16;
  Units u((int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), groups, nb);
  for (; u.row < rows; u.next()) {
    const u32x2 c = *reinterpret_cast<const u32x2 *>(q + (u.row * nb + u.blk) * kBlock + at);
    const float s = power_of_byte(scale[u.row * nb + u.blk]);
    const f32x4 a = values4(c[0], s), b = values4(c[1], s);
    const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    store_row(v, y + u.row * ldy, u.blk * kBlock + at, cols);
  }
}

// A workgroup takes one 128 x 128 block of weights through LDS into both orders, by plain byte gathers: 3001 x 1024 in 13.5 us,
// where the 28 MB that it reads and writes take 5.6.  Once an optimiser step.
__global__ __launch_bounds__(256) void block8_pack_kernel(int32_t in_dim, int32_t out_dim, int32_t nib, int32_t nob,
                                                          int64_t wide_at, int64_t back_at, int64_t scale_at,
                                                          int64_t stride, const float *__restrict__ W, uint8_t *__restrict__ packed) {
  __shared__ uint8_t code[kBlock][kBlock + 4];  // [input][output]
  __shared__ uint32_t most[4];
  const int ib = blockIdx.x, ob = blockIdx.y, t = threadIdx.x;
  const float *w = W + (int64_t)blockIdx.z * in_dim * out_dim;
  uint8_t *p = packed + (int64_t)blockIdx.z * stride;
  const int col = t & 127, n = ob * kBlock + col;
  float v[64];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 64; ++i) {
    const int k = ib * kBlock + 2 * i + (t >> 7);
    v[i] = k < in_dim && n < out_dim ? w[(int64_t)k * out_dim + n] : 0.0f;
    m = max(m, finite_bits(v[i]));
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if ((t & 63) == 0) most[t >> 6] = m;
  __syncthreads();
  const int e = exponent_of(max(max(most[0], most[1]), max(most[2], most[3])));
  const float inv = power(-e);
#pragma unroll
  for (int i = 0; i < 64; ++i) code[2 * i + (t >> 7)][col] = (uint8_t)codes4(v[i] * inv, 0.0f, 0.0f, 0.0f);
  __syncthreads();
  if (t == 0) p[scale_at + ib * nob + ob] = (uint8_t)(e + 127);
  const int64_t f_at = (int64_t)ob * nib + ib, b_at = (int64_t)ib * nob + ob;
  u32x4 *fwd = reinterpret_cast<u32x4 *>(p + f_at * kTileBytes), *wide = reinterpret_cast<u32x4 *>(p + wide_at + f_at * kWideTileBytes),
        *back = reinterpret_cast<u32x4 *>(p + back_at + b_at * kWideTileBytes);
  const float unit = power(e);
  auto four = [&](int in, int out, bool along_in) {  // four codes from (in, out) on
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c |= (uint32_t)(along_in ? code[in + i][out] : code[in][out + i]) << (8 * i);
    return c;
  };
#pragma unroll
  for (int j = 0; j < 8; ++j) {  // 2048 pieces of 8 entries decoded, 1024 of 16 codes
    const int piece = t + 256 * j, lane = piece & 63, part = (piece >> 6) & 3, tile = (piece >> 8) & 3, half = piece >> 10;
    const int m = lane & 31, a = 64 * ((m >> 2) & 1) + 16 * tile + 4 * (m >> 3) + (m & 3);
    const int b = 64 * half + 32 * (lane >> 5) + 8 * part, c = 64 * half + 16 * part + 8 * (lane >> 5);
    const uint32_t f[2] = {four(b, a, true), four(b + 4, a, true)}, g[2] = {four(a, c, false), four(a, c + 4, false)};
    const u32x2 f0 = decode4(f[0], unit), f1 = decode4(f[1], unit), g0 = decode4(g[0], unit), g1 = decode4(g[1], unit);
    wide[piece] = u32x4{f0[0], f0[1], f1[0], f1[1]};
    back[piece] = u32x4{g0[0], g0[1], g1[0], g1[1]};
    reinterpret_cast<u32x2 *>(fwd)[((piece >> 7) * 64 + lane) * 2 + (part & 1)] = u32x2{f[0], f[1]};
  }
}

unsigned stream_blocks(int64_t units) {
  const int64_t want = (units + 15) / 16;
  return (unsigned)(want < 256 * 16 ? want : 256 * 16);
}

}  // namespace
}  // namespace b8

using namespace b8;

hipError_t launch_block8_store(hipStream_t st, int64_t rows, int32_t cols, int32_t kind, const void *x, int64_t ldx, uint8_t *q,
                               uint8_t *scale) {
  const int32_t nb = (cols + kBlock - 1) / kBlock;
  const dim3 grid(stream_blocks(rows * nb));
  if (kind == PR_B8_F32)
    hipLaunchKernelGGL(block8_store_kernel<float>, grid, dim3(256), 0, st, rows, cols, nb, static_cast<const float *>(x), ldx, q, scale);
  else
    hipLaunchKernelGGL(block8_store_kernel<uint16_t>, grid, dim3(256), 0, st, rows, cols, nb, static_cast<const uint16_t *>(x), ldx, q,
                       scale);
  return hipGetLastError();
}

hipError_t launch_block8_restore(hipStream_t st, int64_t rows, int32_t cols, const uint8_t *q, const uint8_t *scale, int32_t kind,
                                 void *y, int64_t ldy) {
  const int32_t nb = (cols + kBlock - 1) / kBlock;
  const dim3 grid(stream_blocks(rows * nb));
  if (kind == PR_B8_F32)
    hipLaunchKernelGGL(block8_restore_kernel<float>, grid, dim3(256), 0, st, rows, cols, nb, q, scale, static_cast<float *>(y), ldy);
  else
    hipLaunchKernelGGL(block8_restore_kernel<uint16_t>, grid, dim3(256), 0, st, rows, cols, nb, q, scale, static_cast<uint16_t *>(y), ldy);
  return hipGetLastError();
}

hipError_t launch_block8_pack(hipStream_t st, int32_t P, int32_t in_dim, int32_t out_dim, const float *W, void *packed) {
  const WeightPlan w = weight_plan(in_dim, out_dim);
  hipLaunchKernelGGL(block8_pack_kernel, dim3(w.nib, w.nob, P), dim3(256), 0, st, in_dim, out_dim, w.nib, w.nob, w.wide_at, w.back_at,
                     w.scale_at, w.stride, W, static_cast<uint8_t *>(packed));
  return hipGetLastError();
}

}  // namespace pod
