// 8-bit blocks: 128 columns of a row (128 x 128 of a weight matrix) are e4m3 numbers
// that share a power-of-two scale 2^e, kept as the byte e + 127.
//
// e is the smallest exponent for which the largest finite magnitude m of the block
// fits, m <= 448 2^e, within [kMinExp, kMaxExp]; 0 for a block of zeros.  A power of
// two costs nothing to apply: the matrix instructions take the byte itself, x 2^-e is
// exact, and q 2^e is exact in bf16 (four significant bits; kMinExp keeps the smallest
// of them, 2^(e - 9), a normal number).
//
// Operand layout.  Products are formed transposed, as everywhere in this library: the
// weights are the matrix instruction's A operand (32 output features), 32 batch rows the B
// operand, so a lane owns one batch row, lane % 32.  The weights' 128 features of a block
// are dealt to four tiles such that a lane's accumulators are 64 CONSECUTIVE features of
// its row, 64 (lane / 32) + 16 t + j for accumulator j of tile t: accumulator row m of a
// tile holds feature 64 (m / 4 % 2) + 16 t + 4 (m / 8) + m % 4.
// In the contraction a lane holds the 32 inputs 64 s + 32 (lane / 32) .. + 31 of either half
// s of a block: one 32 x 32 x 64 instruction in 8 bits, or four 32 x 32 x 16 ones on the
// decoded bytes.  (Any order of the inputs is right as long as both operands keep it, and
// the scale is the same for all 128.)  Input gradients, whose rows are bf16, have the inputs
// 64 s + 16 p + 8 (lane / 32) .. + 7 in part p of half s instead.
#pragma once

#include "pod_internal.h"

namespace pod {
namespace b8 {

constexpr int kBlock = 128;
constexpr int kMinExp = -117, kMaxExp = 120;
constexpr int kTileBytes = 16384;            // 128 features x 128 inputs: [half][tile of 32 features][16 of 32 inputs][lane][16 bytes]
constexpr int kWideTileBytes = 32768;        // the same decoded to bf16: [half][tile][8 of 32 inputs][lane][16 bytes]

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// values that need not start on a boundary of their own size
struct __attribute__((packed, aligned(4))) F32x4At4 { f32x4 v; };
struct __attribute__((packed, aligned(2))) U32x4At2 { u32x4 v; };

// bits of the largest finite magnitude -> exponent of the block
__device__ inline int exponent_of(uint32_t m) {
  // 448 = 1.75 * 2^8: the exponent field goes up by one from the first fraction above .75 on
  const int e = min(max((int)((m + 0x1fffffu) >> 23) - 127 - 8, kMinExp), kMaxExp);
  return m == 0 ? 0 : e;
}
__device__ inline float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ inline float power_of_byte(uint32_t b) { return __uint_as_float(b << 23); }

// magnitude bits of a finite number, 0 of the others
__device__ inline uint32_t finite_bits(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}

// four scaled values (at most 448 in magnitude, or infinite or NaN) -> four codes
__device__ inline uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// four codes times a power of two -> two pairs of bf16, exactly
__device__ inline u32x2 decode4(uint32_t q, float scale) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, true))};
}

// four codes times a power of two -> fp32
__device__ inline f32x4 values4(uint32_t q, float scale) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q, scale, true);
  return f32x4{a[0], a[1], b[0], b[1]};
}

__device__ inline uint32_t pack_bf16(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// 16 bytes of a row from `at` on, zeros behind its end, in two steps and without a branch that would make each load wait for the
// one before it: the load, moved back to where the row has 16 bytes, and the shift once it has arrived.  Rows of fewer entries are
// read one by one (short_piece).
template <class T>
__device__ inline int piece_start(int at, int len) { return max(min(at, len - (int)(16 / sizeof(T))), 0); }
template <class T>
__device__ inline u32x4 request_piece(const T *row, int at, int len) {
  return reinterpret_cast<const U32x4At2 *>(row + piece_start<T>(at, len))->v;
}
template <class T>
__device__ inline u32x4 short_piece(const T *row, int len) {
  constexpr int kN = 16 / sizeof(T), kIn = 4 / sizeof(T);  // entries of a piece, of a dword
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kN - 1; ++i)
    if (i < len) v[i / kIn] |= (sizeof(T) == 2 ? (uint32_t)row[i] : __builtin_bit_cast(uint32_t, (float)row[i])) << (16 * (i % kIn));
  return v;
}
template <class T>
__device__ inline u32x4 settle_piece(u32x4 v, int at, int len) {
  const int d = at - piece_start<T>(at, len);  // entries in front of the wanted ones
  const int dwords = sizeof(T) == 4 ? d : d >> 1;
  v = dwords & 2 ? u32x4{v[2], v[3], 0, 0} : v;
  v = dwords & 1 ? u32x4{v[1], v[2], v[3], 0} : v;
  if (sizeof(T) == 2)
    v = d & 1 ? u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16} : v;
  return dwords > 3 ? u32x4{0, 0, 0, 0} : v;
}

// N consecutive elements from `at` on of a row of `len`, zeros behind its end; any alignment of the element's own size.
__device__ inline void spread(float *v, const u32x4 &t, const float *) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(t[j]);
}
__device__ inline void spread(float *v, const u32x4 &t, const uint16_t *) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(t[j] << 16);
    v[2 * j + 1] = __uint_as_float(t[j] & 0xffff0000u);
  }
}
template <int N>
__device__ inline void load_row(float *v, const float *row, int at, int len, bool) {
  if (at + N <= len) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4 t = reinterpret_cast<const F32x4At4 *>(row + at + i)->v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = t[j];
    }
  } else {  // (nothing is done to a value on its way: the loads wait for each other no more than the others)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = at + i < len ? row[at + i] : 0.0f;
  }
}
template <int N>
__device__ inline void load_row(float *v, const uint16_t *row, int at, int len, bool whole) {  // whole: [at, at + N) of every lane is in the row
  u32x4 t[N / 8];
  if (whole) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) t[i] = reinterpret_cast<const U32x4At2 *>(row + at + i * 8)->v;
  } else if (len >= 8) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) t[i] = request_piece(row, at + i * 8, len);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) t[i] = settle_piece<uint16_t>(t[i], at + i * 8, len);
  } else {
    const u32x4 s = short_piece(row, len);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) t[i] = settle_piece<uint16_t>(s, at + i * 8, len);
  }
#pragma unroll
  for (int i = 0; i < N / 8; ++i) spread(v + i * 8, t[i], row);
}

// The same way out.
template <int N>
__device__ inline void store_row(const float (&v)[N], float *row, int at, int len) {
  if (at + N <= len) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      reinterpret_cast<F32x4At4 *>(row + at + i)->v = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at + i < len) row[at + i] = v[i];
  }
}
template <int N>
__device__ inline void store_row(const float (&v)[N], uint16_t *row, int at, int len) {
  if (at + N <= len) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
      reinterpret_cast<U32x4At2 *>(row + at + i)->v = u32x4{pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3]),
                                                           pack_bf16(v[i + 4], v[i + 5]), pack_bf16(v[i + 6], v[i + 7])};
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at + i < len) reinterpret_cast<__bf16 *>(row)[at + i] = (__bf16)v[i];
  }
}

// Packed weights of one agent: tiles [out block][in block] of codes for the 8-bit product, the same decoded to bf16 (exactly),
// tiles [in block][out block] decoded for the input gradients, and the scale bytes [in block][out block] of the codes.
// Decoded weights take LDS and L2 twice the bytes that decoding in registers would, in kernels those do not bound, and
// leave the vector pipe to the activations.
struct WeightPlan {
  int32_t in_dim, out_dim, nib, nob;  // and their numbers of blocks
  int64_t wide_at, back_at, scale_at, stride;  // bytes
};
inline WeightPlan weight_plan(int32_t in_dim, int32_t out_dim) {
  WeightPlan w;
  w.in_dim = in_dim, w.out_dim = out_dim;
  w.nib = (in_dim + kBlock - 1) / kBlock, w.nob = (out_dim + kBlock - 1) / kBlock;
  const int64_t tiles = (int64_t)w.nib * w.nob;
  w.wide_at = tiles * kTileBytes;
  w.back_at = w.wide_at + tiles * kWideTileBytes;
  w.scale_at = w.back_at + tiles * kWideTileBytes;
  w.stride = (w.scale_at + tiles + 255) / 256 * 256;
  return w;
}

}  // namespace b8

// rows [rows, ldx] in fp32 or bf16 -> codes [rows, 128 nb] and scale bytes [rows, nb]; and back
hipError_t launch_block8_store(hipStream_t st, int64_t rows, int32_t cols, int32_t kind, const void *x, int64_t ldx, uint8_t *q,
                               uint8_t *scale);
hipError_t launch_block8_restore(hipStream_t st, int64_t rows, int32_t cols, const uint8_t *q, const uint8_t *scale, int32_t kind,
                                 void *y, int64_t ldy);
hipError_t launch_block8_pack(hipStream_t st, int32_t P, int32_t in_dim, int32_t out_dim, const float *W, void *packed);

// y = act(x W + b) over `rows` rows of each of P agents.
struct Block8Linear {
  int32_t P, in_dim, out_dim, tanh;
  int64_t rows;
  int32_t x_kind;
  const void *x;
  const uint8_t *x_scale;
  int64_t ldx;
  const void *packed;
  const float *bias;  // or null
  int32_t y_kind;
  void *y;
  uint8_t *y_scale;
  int64_t ldy;
};
hipError_t launch_block8_linear(hipStream_t st, const Block8Linear &a);

// Its gradients: dx (unless null), dW, db.  y: the layer's outputs as blocks, null where its activation is the identity.
struct Block8Grads {
  int32_t P, in_dim, out_dim;
  int64_t rows;
  int32_t dy_kind;
  const void *dy;
  int64_t lddy;
  const uint8_t *y, *y_scale, *x, *x_scale;
  const void *packed;
  int32_t dx_kind;
  void *dx;
  int64_t lddx;
  float *dW, *db;
  float *parts;
};
// Bytes of `parts` for these rows, and for any number of rows up to them.
size_t block8_grads_scratch(int32_t P, int64_t rows, int32_t in_dim, int32_t out_dim);
size_t block8_grads_most_scratch(int32_t P, int64_t rows, int32_t in_dim, int32_t out_dim);
hipError_t launch_block8_grads(hipStream_t st, const Block8Grads &a);

}  // namespace pod
