// Pieces of a product of 32-row tiles with 128 features of packed 8-bit weights: operands
// from each kind of rows, the matrix instructions of a block of 128 inputs, and the way out.
#pragma once

#include <type_traits>
#include <utility>

#include "pod_block8.h"
#include "pod_tile.h"

namespace pod {
namespace b8 {

// What the rows are: blocks, plain rows that go through the rule of the blocks on their way in, or gradients behind an
// activation whose output is kept as blocks (g = bf16(dy (1 - y^2)), or bf16(dy) where there is none).
enum { kBlocks = 0, kF32 = 1, kBf16 = 2, kGradF32 = 3, kGradBf16 = 4 };

struct Product {
  int64_t rows;          // of one agent
  int32_t ins, outs, nib, nob, act;
  const void *x;
  const uint8_t *x_scale;
  const uint8_t *out, *out_scale;  // the layer's output blocks (gradients only, or null)
  int64_t ldx;           // elements
  const uint8_t *w, *w_scale;  // tiles of codes and their scale bytes, or decoded tiles
  int64_t w_stride;
  const float *bias;
  void *y;
  uint8_t *y_scale;
  int64_t ldy;
  int32_t x_size, y_size;

  __device__ void to_agent(int p) {
    const int64_t first = p * rows;
    x = static_cast<const uint8_t *>(x) + first * ldx * x_size;
    if (x_scale) x_scale += first * nib;
    if (out) out += first * nib * kBlock, out_scale += first * nib;
    w += p * w_stride;
    if (w_scale) w_scale += p * w_stride;
    if (bias) bias += (int64_t)p * outs;
    y = static_cast<uint8_t *>(y) + first * ldy * y_size;
    if (y_scale) y_scale += first * nob;
  }
};

// Which of eight runs of rows a workgroup is for that follows the XCD it is on (x & 7).  Where there are fewer than eight, the
// workgroups of one tile or agent after the other start on the XCD behind the last one's, or half of the chip would stay idle.
__device__ inline int place_of(unsigned x, int runs, int64_t of) {
  return (int)((x + (runs < 8 ? (uint32_t)(of * (8 - runs)) : 0u)) & 7u);
}

// f(0) .. f(N - 1) with constant arguments: straight-line code whatever its length.
template <class F, int... I>
__device__ inline void each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ inline void each(F f) {
  each(f, std::make_integer_sequence<int, N>());
}

__device__ inline i32x8 join(const u32x4 &lo, const u32x4 &hi) {
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// A lane's 2 x 32 inputs of a block of a row: codes and their scale byte, or decoded, 8 inputs a part.
template <bool IN8>
struct Operand;
template <>
struct Operand<true> {
  i32x8 half[2];
  uint32_t scale;
};
template <>
struct Operand<false> {
  u32x4 part[8];
};

__device__ inline void set_codes(Operand<true> &o, const i32x8 (&half)[2], uint32_t byte) {
  o.half[0] = half[0], o.half[1] = half[1], o.scale = byte;
}
// part p (8 inputs) of a half's codes, decoded
__device__ inline u32x4 decode_part(const i32x8 &codes, int p, float scale) {
  const u32x2 a = decode4((uint32_t)codes[2 * p], scale), b = decode4((uint32_t)codes[2 * p + 1], scale);
  return u32x4{a[0], a[1], b[0], b[1]};
}
__device__ inline void set_codes(Operand<false> &o, const i32x8 (&half)[2], uint32_t byte) {
  const float s = power_of_byte(byte);
#pragma unroll
  for (int i = 0; i < 8; ++i) o.part[i] = decode_part(half[i >> 2], i & 3, s);
}

// The larger of two lanes 32 apart, in both.
__device__ inline uint32_t max_of_two(uint32_t m) {
  const auto a = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return max(a[0], a[1]);
}

// The rule of the blocks on a block's 2 x 64 values of a row (lanes 32 apart share a row).
__device__ inline void encode64(const float (&v)[64], uint32_t (&codes)[16], uint32_t &byte) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 64; ++i) m = max(m, finite_bits(v[i]));
  const int e = exponent_of(max_of_two(m));
  const float inv = power(-e);
#pragma unroll
  for (int i = 0; i < 16; ++i) codes[i] = codes4(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
  byte = (uint32_t)(e + 127);
}

// dy (1 - y^2), y in blocks (y^2 has 8 bits: one rounding)
__device__ inline void times_derivative(float *v, uint32_t codes, float scale) {
  const f32x4 y = values4(codes, scale);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] *= fmaf(-y[j], y[j], 1.0f);
}

// Block ib of a row; h = lane / 32.
template <int SRC, bool IN8>
__device__ inline void load_operand(Operand<IN8> &o, const Product &a, int64_t row, int ib, int h) {
  const int at = ib * kBlock + 32 * h;
  if constexpr (SRC == kBlocks) {
    const i32x8 *p = reinterpret_cast<const i32x8 *>(static_cast<const uint8_t *>(a.x) + row * a.ldx + at);
    const i32x8 half[2] = {p[0], p[2]};
    set_codes(o, half, a.x_scale[row * a.nib + ib]);
  } else {
    typedef std::conditional_t<SRC == kF32 || SRC == kGradF32, float, uint16_t> T;
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    float v[64];
    if constexpr (SRC == kF32 || SRC == kBf16) {
#pragma unroll
      for (int s = 0; s < 2; ++s) load_row<32>(v + 32 * s, x, at + 64 * s, a.ins, (ib + 1) * kBlock <= a.ins);
      uint32_t c[16], byte;
      encode64(v, c, byte);
      i32x8 half[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) half[i >> 3][i & 7] = (int)c[i];
      set_codes(o, half, byte);
    } else {
      static_assert(!IN8, "gradients are bf16 operands");
      constexpr int kN = 16 / sizeof(T), kEach = 8 / kN;  // entries of a piece, pieces of eight inputs
      u32x4 raw[8 * kEach];
      auto at_of = [&](int i) { return ib * kBlock + 16 * (i / kEach) + 8 * h + kN * (i % kEach); };
      if ((ib + 1) * kBlock <= a.ins) {
#pragma unroll
        for (int i = 0; i < 8 * kEach; ++i) raw[i] = reinterpret_cast<const U32x4At2 *>(x + at_of(i))->v;
      } else {
#pragma unroll
        for (int i = 0; i < 8 * kEach; ++i) raw[i] = a.ins >= kN ? request_piece(x, at_of(i), a.ins) : short_piece(x, a.ins);
#pragma unroll
        for (int i = 0; i < 8 * kEach; ++i) raw[i] = settle_piece<T>(raw[i], at_of(i), a.ins);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int from = ib * kBlock + 16 * i + 8 * h;
#pragma unroll
        for (int j = 0; j < kEach; ++j) spread(v + 8 * i + kN * j, raw[kEach * i + j], x);
        if (a.out) {
          const u32x2 c = *reinterpret_cast<const u32x2 *>(a.out + row * a.nib * kBlock + from);
          const float s = power_of_byte(a.out_scale[row * a.nib + ib]);
          times_derivative(v + 8 * i, c[0], s);
          times_derivative(v + 8 * i + 4, c[1], s);
        }
        o.part[i] = u32x4{pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]), pack_bf16(v[8 * i + 4], v[8 * i + 5]),
                          pack_bf16(v[8 * i + 6], v[8 * i + 7])};
      }
    }
  }
}

// 32 features x 32 rows.  In 8 bits an instruction has 64 inputs, at twice the rate, and its sum of eight neighbouring products
// keeps 13 bits below the largest of them (what it adds up behind that is fp32): at most 1.5e-5 of the sum of magnitudes on random
// numbers, 1.5e-6 in the mean, for results that are rounded to bf16 or 8 bits (1.3e-3 and 2e-2 in the 2-norm).  Against the
// unrounded result they are as far off as with fp32 sums, to four digits (bf16) and six (blocks); 6e-4 of the codes, whose sums lie
// next to a border between two, are the neighbouring ones, 7e-4 of the results in the 2-norm.  Decoded to bf16 the products and
// sums are fp32's, at half the rate: 262144 x 512 x 512 with its restore 169 -> 228 us, 65536 x 1024 x 1024 85 -> 122.
// (32 x 32 tiles: 16 x 16 x 128 reads twice the registers for the same work and reaches 3870 TFLOP/s where this one has 4940
// with a wavefront to each SIMD and its operands in registers.)
template <int SEL>
__device__ inline void multiply8(f32x16 &c, const i32x8 &w, uint32_t w_scale, const i32x8 &x, uint32_t x_scale) {
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, SEL, (int)w_scale, SEL, (int)x_scale);
}
__device__ inline void multiply16(f32x16 &c, const u32x4 &w, const u32x4 &x) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
}

// One block of inputs; w: the lane's first piece of the weights' tile.
__device__ inline void multiply_block(f32x16 (&acc)[4], const u32x4 *w, uint32_t w_scale, const Operand<true> &x) {
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int f = 0; f < 4; ++f) multiply8<0>(acc[f], join(w[128 * (4 * s + f)], w[128 * (4 * s + f) + 64]), w_scale, x.half[s], x.scale);
}
__device__ inline void multiply_block(f32x16 (&acc)[4], const u32x4 *w, uint32_t, const Operand<false> &x) {
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int p = 0; p < 4; ++p) multiply16(acc[f], w[64 * (4 * (4 * s + f) + p)], x.part[4 * s + p]);
}

// Sums start from the bias.
__device__ inline void start_sums(f32x16 (&acc)[4], const Product &a, int ob, int h) {
  float b[64];
#pragma unroll
  for (int i = 0; i < 64; ++i) b[i] = 0.0f;
  if (a.bias) load_row<64>(b, a.bias, ob * kBlock + 64 * h, a.outs, (ob + 1) * kBlock <= a.outs);
#pragma unroll
  for (int i = 0; i < 64; ++i) acc[i >> 4][i & 15] = b[i];
}

// Sums are complete here.  (Left alone, the compiler moves a row tile's matrix instructions behind the way out of the tile
// before it, and keeps every operand until then.)
__device__ inline void hold(f32x16 (&acc)[4]) {
#pragma unroll
  for (int f = 0; f < 4; ++f) asm volatile("" : "+v"(acc[f]));
}

// tanh z = 1 - 2 / (e^2z + 1) is off by up to 2^-22 of ONE, whatever z: e^2z + 1 has no digits of a small z.  A result that is
// rounded to bf16 is therefore z itself below 2^-7, off by z^2 / 3, at most 2.1e-5 of it; from there on 2^-22 is at most 3.1e-5
// of it (bf16's own rounding: 3.9e-3).  Two operations an entry: 65536 x 1024 x 1024 90 -> 92 us, 64 agents x 1000 x 301 x 256
// 29 -> 30.5 us; a branch would hardly ever be left out, 64 sums of 32 rows have a small one nearly always.
constexpr float kTanhIsItself = 0.0078125f;
__device__ inline float tanh_to_bf16(float z) {
  const float t = tile::tanh_from_scaled(z * tile::kTwoLog2e);
  return fabsf(z) < kTanhIsItself ? z : t;
}

// Blocks whose sums all lie below 1/2 keep the relative precision of their smallest entries with the odd Taylor polynomial up to
// z^9 (9e-6 of the value at 1/2).  In a block with a larger sum 2^-22 is at most an eighth of half the smallest step of its codes.
// (A branch by rows: 262144 x 512 x 512 with larger sums as before it.)
constexpr float kSmallSums = 0.5f;
__device__ inline float tanh_small(float z) {
  const float z2 = z * z;
  return fmaf(z2 * z, fmaf(z2, fmaf(z2, fmaf(z2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), z);
}

// A row's 2 x 64 sums: the largest |sum|, in both lanes.  (A maximum ignores NaN by itself, and infinite sums have finite tanh.)
__device__ inline float largest_sum(const f32x16 (&acc)[4]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 64; ++i) m = fmaxf(m, fabsf(acc[i >> 4][i & 15]));
  return __uint_as_float(max_of_two(__float_as_uint(m)));
}

// One row's 64 sums to codes.  tanh is monotonic: a block's largest |tanh| is that of its largest |sum|, which is known before
// any of them; from 1/2 on 2^-e tanh(z) = 2^-e - 2 2^-e / (e^2z + 1) is then one operation behind the reciprocal.  (A value may
// be rounded to 2^-20 of itself above the largest one's: 448 still.)
__device__ inline void encode_sums(const f32x16 (&acc)[4], bool act, uint32_t (&codes)[16], uint32_t &byte) {
  if (!act) {
    float v[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = acc[i >> 4][i & 15];
    encode64(v, codes, byte);
    return;
  }
  const float m = largest_sum(acc);
  const bool small = m < kSmallSums;
  const int e = exponent_of(__float_as_uint(small ? tanh_small(m) : tile::tanh_from_scaled(m * tile::kTwoLog2e)));
  const float inv = power(-e), minus2 = -2.0f * inv;
  byte = (uint32_t)(e + 127);
  if (small) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = tanh_small(acc[i >> 2][4 * (i & 3) + j]) * inv;
      codes[i] = codes4(v[0], v[1], v[2], v[3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = fmaf(minus2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(acc[i >> 2][4 * (i & 3) + j] * tile::kTwoLog2e) + 1.0f), inv);
    codes[i] = codes4(v[0], v[1], v[2], v[3]);
  }
}
// A value by itself (of a block too: few rows, whose largest value is found behind the activation).
template <int OUT>
__device__ inline float activate(float z, bool act) {
  return !act ? z : OUT == PR_B8_BF16 ? tanh_to_bf16(z) : tile::tanh_accurate(z);
}

// Activation and the way out of one row's 64 sums.  All lanes have to come here (blocks: two of them share a maximum).
template <int OUT>
__device__ inline void finish(const f32x16 (&acc)[4], const Product &a, int64_t row, int ob, int h) {
  const int at = ob * kBlock + 64 * h;
  if constexpr (OUT == PR_B8_BLOCKS) {
    uint32_t c[16], byte;
    encode_sums(acc, a.act, c, byte);
    if (row >= a.rows) return;
    u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(a.y) + row * a.ldy + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = u32x4{c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3]};
    if (h == 0) a.y_scale[row * a.nob + ob] = (uint8_t)byte;
  } else {
    float v[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = activate<OUT>(acc[i >> 4][i & 15], a.act);
    typedef std::conditional_t<OUT == PR_B8_F32, float, uint16_t> T;
    if (row < a.rows) store_row(v, static_cast<T *>(a.y) + row * a.ldy, at, a.outs);
  }
}

}  // namespace b8
}  // namespace pod
