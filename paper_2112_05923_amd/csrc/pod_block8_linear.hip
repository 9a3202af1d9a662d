// One layer on 8-bit blocks: y = act(x W + b), and with the roles of the weights' sides
// exchanged the input gradients dx = g W^T of its backward pass (layouts: pod_block8.h).
#include <algorithm>
#include <cstddef>

#include "pod_block8.h"
#include "pod_block8_product.h"
#include "pod_tile.h"

namespace pod {
namespace b8 {
namespace {

// A wavefront has 32 rows x 128 features; operands straight from memory.  What the kernels below do not take: rows so far apart
// that 32 of them span 2 GiB, many plain rows of fewer than 8 entries or too many for a launch, gradients of many rows behind
// more than 1024 outputs.
template <int SRC, bool IN8, int OUT>
__global__ __launch_bounds__(256) void linear_kernel(Product a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ob = blockIdx.y, h = lane >> 5;
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + wave) * 32;
  if (row0 >= a.rows) return;
  a.to_agent(blockIdx.z);
  f32x16 acc[4];
  start_sums(acc, a, ob, h);
  const int64_t row = row0 + (lane & 31), from = min(row, a.rows - 1);
  for (int ib = 0; ib < a.nib; ++ib) {
    Operand<IN8> x;
    load_operand<SRC>(x, a, from, ib, h);
    const uint8_t *w = a.w + ((int64_t)ob * a.nib + ib) * (IN8 ? kTileBytes : kWideTileBytes);
    multiply_block(acc, reinterpret_cast<const u32x4 *>(w) + lane, IN8 ? a.w_scale[ib * a.nob + ob] : 0, x);
  }
  hold(acc);
  finish<OUT>(acc, a, row, ob, h);
}

// Few rows: the weights are what has to be read, and many compute units have to read them.  A workgroup of sixteen wavefronts
// has 32 rows x 32 features (128 where they become blocks, which share a maximum), the blocks of inputs dealt to its wavefronts,
// whose sums meet in LDS.  Bound: latency, a launch and three round trips (1 row of 3001 inputs in fp32 to 1024 outputs 9 us, on
// 32 compute units; 48 rows of 301 in bf16 to 512 6 us).  Gradients as the rows spill 14 (bf16) and 36 (fp32) registers.
template <int SRC, bool IN8, int OUT>
__global__ __launch_bounds__(1024) void linear_few_kernel(Product a) {
  constexpr int kTiles = OUT == PR_B8_BLOCKS ? 4 : 1, kSplits = 16 / kTiles, kPitch = 65;
  __shared__ float sums[16][16 * kPitch];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = lane >> 5;
  const int ob = blockIdx.y * kTiles / 4, f = OUT == PR_B8_BLOCKS ? wave & 3 : blockIdx.y & 3, split = wave / kTiles;
  a.to_agent(blockIdx.z);
  const int64_t row0 = (int64_t)blockIdx.x * 32, from = min(row0 + (lane & 31), a.rows - 1);
  f32x16 acc;
#pragma unroll
  for (int j = 0; j < 16; ++j) acc[j] = 0.0f;
  for (int ib = split; ib < a.nib; ib += kSplits) {
    const u32x4 *w = reinterpret_cast<const u32x4 *>(a.w + ((int64_t)ob * a.nib + ib) * (IN8 ? kTileBytes : kWideTileBytes)) + lane;
    Operand<IN8> x;
    if constexpr (IN8) {
      i32x8 wf[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) wf[s] = join(w[128 * (4 * s + f)], w[128 * (4 * s + f) + 64]);
      const uint32_t scale = a.w_scale[ib * a.nob + ob];
      load_operand<SRC>(x, a, from, ib, h);
#pragma unroll
      for (int s = 0; s < 2; ++s) multiply8<0>(acc, wf[s], scale, x.half[s], x.scale);
    } else {
      u32x4 wf[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) wf[i] = w[64 * (4 * (4 * (i >> 2) + f) + (i & 3))];
      load_operand<SRC>(x, a, from, ib, h);
#pragma unroll
      for (int i = 0; i < 8; ++i) multiply16(acc, wf[i], x.part[i]);
    }
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) sums[wave][j * kPitch + lane] = acc[j];
  __syncthreads();
  // entry (feature, row): register feature % 16 of tile feature / 16 % 4, lane 32 (feature / 64) + row
  const int row = t >> 5;
  auto total = [&](int feature, int tile) {
    float z = a.bias && ob * kBlock + feature < a.outs ? a.bias[ob * kBlock + feature] : 0.0f;
#pragma unroll
    for (int s = 0; s < kSplits; ++s) z += sums[s * kTiles + tile][(feature & 15) * kPitch + 32 * (feature >> 6) + row];
    return activate<OUT>(z, a.act);
  };
  if constexpr (OUT == PR_B8_BLOCKS) {
    const int at = 4 * (t & 31);
    float v[4];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = total(at + i, (at + i) >> 4 & 3);
      m = max(m, finite_bits(v[i]));
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    const int e = exponent_of(m);
    const float inv = power(-e);
    if (row0 + row >= a.rows) return;
    uint8_t *y = static_cast<uint8_t *>(a.y) + (row0 + row) * a.ldy + ob * kBlock;
    *reinterpret_cast<uint32_t *>(y + at) = codes4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    if ((t & 31) == 0) a.y_scale[(row0 + row) * a.nob + ob] = (uint8_t)(e + 127);
  } else {
    const int feature = 64 * ((t >> 4) & 1) + 16 * f + (t & 15), n = ob * kBlock + feature;
    const float v = total(feature, 0);
    if (row0 + row >= a.rows || n >= a.outs) return;
    if constexpr (OUT == PR_B8_F32) static_cast<float *>(a.y)[(row0 + row) * a.ldy + n] = v;
    else static_cast<__bf16 *>(a.y)[(row0 + row) * a.ldy + n] = (__bf16)v;
  }
}

// 64 lanes x 16 bytes from `base` (uniform) + `offset` (a lane's own) straight into LDS (its first 64 KiB, kCopyReach: the address's
// register has 16 bits of it); waited for by arrived().  Kernels that copy have one LDS object, which starts at 0, and what they
// copy into in front.
constexpr int kCopyReach = 65536;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void copy_to_lds(const uint8_t *base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// This wavefront's copies are complete; with the barrier everybody's are, and everybody is past what it read before.
__device__ inline void arrived() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// The same where this wavefront has asked for LATER more accesses since its copies (they complete in the order they were asked for).
template <int LATER>
__device__ inline void arrived_before() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Lanes of a wavefront exchange data through LDS here: its accesses are carried out in order, but the compiler, which sees one
// lane, would keep what that lane read before.
__device__ inline void exchange() { asm volatile("" ::: "memory"); }
__device__ inline void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ inline uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p;
}

// Piece c (16 bytes) of row r lies at place c ^ swizzle(r) of the row's 128 bytes in LDS: the 16 rows that lanes read the same
// piece of are on all banks.
__device__ inline int swizzle(int r) { return (r >> 1) & 7; }

// What lane groups (16 lanes) 0, 1, 2, 3 have of two registers a, b: a0 a1 a2 a3, b0 b1 b2 b3 -> a0 b0 a2 b2, a1 b1 a3 b3.
__device__ inline void swap16(uint32_t &a, uint32_t &b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0], b = r[1];
}
__device__ inline void swap16(u32x4 &a, u32x4 &b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u = a[i], v = b[i];
    swap16(u, v);
    a[i] = u, b[i] = v;
  }
}

// A tile's 32 rows x 128 features out through `room` (2 KiB of LDS, the wavefront's own), 16 rows x 128 bytes at a time and
// whole lines to memory.  A lane has 4 kSize pieces of 16 bytes of its row; swapped between lane groups, each of them is of the
// first 16 rows in all lanes, or of the others.  row0 is uniform; 32 rows of y span less than 2^31 bytes (lines_fit).
constexpr int kRoomBytes = 16 * 128;
template <int OUT>
inline constexpr int kSizeOf = OUT == PR_B8_F32 ? 4 : OUT == PR_B8_BF16 ? 2 : 1;

// Returns whether the tile was whole: it then took kLineStores accesses.
template <int OUT>
inline constexpr int kLineStores = 4 * kSizeOf<OUT>;
template <int OUT>
__device__ inline bool write_lines(u32x4 (&piece)[4 * kSizeOf<OUT>], const Product &a, int64_t row0, int ob, int lane, uint8_t *room) {
  constexpr int kSize = kSizeOf<OUT>;
  const int left = (int)min(a.rows - row0, (int64_t)32), r = lane & 15, odd = (lane >> 4) & 1, h = lane >> 5;
  uint8_t *y = static_cast<uint8_t *>(a.y) + (row0 * a.ldy + ob * kBlock) * kSize;
  const uint32_t pitch = (uint32_t)(a.ldy * kSize);
  const bool whole = left == 32 && (OUT == PR_B8_BLOCKS || (ob + 1) * kBlock <= a.outs);
#pragma unroll
  for (int i = 0; i < 2 * kSize; ++i) swap16(piece[2 * i], piece[2 * i + 1]);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int pass = 0; pass < kSize; ++pass) {  // pieces 8 pass .. 8 pass + 7 of the rows
      if (OUT != PR_B8_BLOCKS && ob * kBlock + 16 / kSize * 8 * pass >= a.outs) break;
      exchange();
      if (kSize == 1 || h == pass * 2 / kSize) {
#pragma unroll
        for (int i = 0; i < 2 * kSize; ++i) {
          const int c = 4 * kSize * h + 2 * i + odd;
          if (kSize < 4 || i >> 2 == (pass & 1))
            *reinterpret_cast<u32x4 *>(room + r * 128 + ((c & 7) ^ swizzle(r)) * 16) = piece[2 * i + t];
        }
      }
      exchange();
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = 8 * j + (lane >> 3), c = 8 * pass + ((lane & 7) ^ swizzle(row));
        const u32x4 out = *reinterpret_cast<const u32x4 *>(room + j * 1024 + lane * 16);
        uint8_t *to = y + (uint32_t)((16 * t + row) * pitch + 16 * c);
        const int col = ob * kBlock + 16 / kSize * c;
        if (whole) {
          reinterpret_cast<U32x4At2 *>(to)->v = out;
          continue;
        }
        if (16 * t + row >= left) continue;
        if constexpr (OUT == PR_B8_BLOCKS) {
          *reinterpret_cast<u32x4 *>(to) = out;
        } else if (col + 16 / kSize <= a.outs) {
          reinterpret_cast<U32x4At2 *>(to)->v = out;
        } else if constexpr (OUT == PR_B8_F32) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (col + i < a.outs) reinterpret_cast<uint32_t *>(to)[i] = out[i];
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (col + i < a.outs) reinterpret_cast<uint16_t *>(to)[i] = (uint16_t)(out[i >> 1] >> (16 * (i & 1)));
        }
      }
    }
  }
  return whole;
}
inline bool lines_fit(const Product &a) { return a.ldy * a.y_size < (int64_t)1 << 26; }

template <int OUT, int TILES = 4>
__device__ inline bool finish_lines(const f32x16 (&acc)[4], const Product &a, int64_t row0, int ob, int lane, uint8_t *room) {
  if (row0 >= a.rows) return false;
  constexpr int kSize = kSizeOf<OUT>;
  u32x4 piece[4 * kSize];
  if constexpr (OUT == PR_B8_BLOCKS) {
    uint32_t c[16], byte;
    encode_sums(acc, a.act, c, byte);
#pragma unroll
    for (int i = 0; i < 16; ++i) piece[i >> 2][i & 3] = c[i];
    if (lane < 32 && row0 + lane < a.rows) (a.y_scale + row0 * a.nob + ob)[(uint32_t)(lane * a.nob)] = (uint8_t)byte;
  } else {
#pragma unroll
    for (int i = 0; i < 16 * kSize; ++i) {
      constexpr int kIn = 4 / kSize;  // entries of a dword
      if (kIn * i >> 4 >= TILES) {
        piece[i >> 2][i & 3] = 0;
        continue;
      }
      const float v = activate<OUT>(acc[kIn * i >> 4][kIn * i & 15], a.act);
      piece[i >> 2][i & 3] = OUT == PR_B8_F32 ? __float_as_uint(v) : pack_bf16(v, activate<OUT>(acc[(kIn * i + 1) >> 4][(kIn * i + 1) & 15], a.act));
    }
  }
  return write_lines<OUT>(piece, a, row0, ob, lane, room);
}

// The scale bytes of a row, one of a dword each.
template <int NIB>
__device__ inline uint32_t load_scales(const uint8_t *p) {
  struct __attribute__((packed)) Two { uint16_t v; };
  struct __attribute__((packed)) Four { uint32_t v; };
  if constexpr (NIB == 1) return p[0];
  if constexpr (NIB == 2) return reinterpret_cast<const Two *>(p)->v;
  if constexpr (NIB == 3) return reinterpret_cast<const Two *>(p)->v | (uint32_t)p[2] << 16;
  if constexpr (NIB == 4) return reinterpret_cast<const Four *>(p)->v;
}

constexpr int kVectorMayPass = 0x406;  // scheduling fence for all but vector, transcendental and scalar instructions

// acc += the products of NIB blocks with 32 rows whose codes are in registers.  The weights' pieces lie one behind the other in
// LDS (`w`: the lane's first); each is requested two (decoded: four) before the one in use, 64 (32) cycles of matrix work apart.
// Scale bytes: one of a dword per block of inputs.  used(ib): block ib of the rows has been through its products.
template <int TILES, int NIB, class Used>
__device__ inline void multiply_resident(f32x16 (&acc)[4], const u32x4 *w, uint32_t w_scales, const i32x8 (&x)[NIB][2], uint32_t x_scales,
                                         Used used, std::true_type) {
  constexpr int kAhead = 2, kPieces = 2 * TILES * NIB;
  i32x8 ring[kAhead + 1];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) ring[n] = join(w[128 * n], w[128 * n + 64]);
  each<kPieces>([&](auto piece) {
    constexpr int n = piece, ib = n / (2 * TILES), s = n / TILES % 2, f = n % TILES;
    if constexpr (n + kAhead < kPieces) ring[(n + kAhead) % (kAhead + 1)] = join(w[128 * (n + kAhead)], w[128 * (n + kAhead) + 64]);
    multiply8<ib>(acc[f], ring[n % (kAhead + 1)], w_scales, x[ib][s], x_scales);
    if constexpr ((n + 1) % (2 * TILES) == 0) used(std::integral_constant<int, ib>());
    __builtin_amdgcn_sched_barrier(kVectorMayPass);
  });
}
template <int TILES, int NIB, class Used>
__device__ inline void multiply_resident(f32x16 (&acc)[4], const u32x4 *w, uint32_t, const i32x8 (&x)[NIB][2], uint32_t x_scales, Used used,
                                         std::false_type) {
  constexpr int kAhead = 4, kPieces = 8 * TILES * NIB;
  u32x4 ring[kAhead + 1], part[4];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) ring[n] = w[64 * n];
  each<kPieces>([&](auto piece) {  // half n / (4 TILES), tile of features n / 4 % TILES, eight of the lane's 32 inputs n % 4
    constexpr int n = piece, ib = n / (8 * TILES), s = n / (4 * TILES) % 2, f = n / 4 % TILES, p = n & 3;
    if constexpr (f == 0) part[p] = decode_part(x[ib][s], p, power_of_byte((x_scales >> (8 * ib)) & 255));
    if constexpr (n + kAhead < kPieces) ring[(n + kAhead) % (kAhead + 1)] = w[64 * (n + kAhead)];
    multiply16(acc[f], ring[n % (kAhead + 1)], part[p]);
    if constexpr ((n + 1) % (8 * TILES) == 0) used(std::integral_constant<int, ib>());
    __builtin_amdgcn_sched_barrier(kVectorMayPass);
  });
}

// Up to 512 inputs: the weights of up to 1024 / NIB features (half of that decoded) stay in LDS, and no barrier stands between
// two rows.  A wavefront owns 32 rows at a time, with their codes in registers for all feature blocks; a block's registers take
// the next rows' codes as soon as the last feature block is through with them.  Two wavefronts share a SIMD.  Workgroups for
// the other features of the same rows (`slabs`) are on the same XCD at the same time.  262144 x 512 x 512, blocks to blocks:
// 95 to 104 us, 1.4 PFLOP/s and 2.8 TB/s; matrix and vector pipe (tanh: two transcendentals an entry) are busy 36 % of the time
// each, mostly one after the other in a wavefront.
// Heads of up to 16 TILES outputs have them in the first TILES tiles of their one block (64 further ones, of the lanes above
// 32, are zeros that come along); the other tiles are left out, of the products, of LDS and of the activation: 262144 x 512 x 30
// to fp32 79 -> 48 us, 3.4 TB/s.  One workgroup lives on a compute unit, by its share of the rows, and 256 registers are not
// enough for four blocks of inputs to fp32: 51, 42 and 23 of them are spilled with four tiles, two and one, 22 MB of writes beside
// the 31 of that result; with one tile 144 bytes a lane of an array lie in memory for any number of inputs.
constexpr int kResidentWaves = 8, kResidentRows = 32, kResidentBytes = 131072;
constexpr int kHead = kBlock + 4;  // floats per block of features in LDS: 128 biases, the scale bytes of its weights, the tickets

template <bool IN8, int OUT, int NIB, int TILES>
__global__ __launch_bounds__(512, 2) void linear_resident_kernel(Product a, int32_t slab_blocks, int32_t slabs, int32_t groups) {
  constexpr int kBytes = (IN8 ? kTileBytes : kWideTileBytes) / 4 * TILES, kUnit = (IN8 ? kTileBytes : kWideTileBytes) / 8 / 16;  // (tile of a half)
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int i = blockIdx.x >> 3, slab = i % slabs, group = i / slabs * 8 + place_of(blockIdx.x, groups, blockIdx.z);
  if (group >= groups) return;
  a.to_agent(blockIdx.z);
  const int ob0 = slab * slab_blocks, blocks = min(slab_blocks, a.nob - ob0);
  // The workgroup's row tiles are handed out to its wavefronts one at a time (a fixed share each: the first wavefront is done
  // after two thirds of the last one's time).
  auto row_of_ticket = [&](int k) {
    return ((int64_t)(k / kResidentWaves) * groups + group) * (kResidentWaves * kResidentRows) + k % kResidentWaves * kResidentRows;
  };
  int64_t row0 = row_of_ticket(wave), next_row0;
  uint8_t *room = lds + wave * kRoomBytes;
  float *head = reinterpret_cast<float *>(lds + kResidentWaves * kRoomBytes);
  int *tickets = reinterpret_cast<int *>(head) + kBlock + 1;
  if (threadIdx.x == 0) *tickets = kResidentWaves;
  uint8_t *weights = lds + kResidentWaves * kRoomBytes + slab_blocks * kHead * 4;

  i32x8 x[NIB][2];
  uint32_t scales;
  // Memory likes 16 rows x 64 bytes an instruction, the products 32 rows: lane groups swap pieces when they have arrived.
  u32x4 raw[NIB][2][2];  // [half][16 rows]
  auto request = [&](int64_t from, int ib) {
    from = min(from, a.rows - 1);
    const int last = (int)min(a.rows - 1 - from, (int64_t)(kResidentRows - 1));
    const uint8_t *p = static_cast<const uint8_t *>(a.x) + from * (NIB * kBlock) + ib * kBlock;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t at = (uint32_t)(min(16 * t + (lane & 15), last) * (NIB * kBlock) + 16 * (lane >> 4));
      raw[ib][0][t] = *reinterpret_cast<const u32x4 *>(p + at);
      raw[ib][1][t] = *reinterpret_cast<const u32x4 *>(p + at + 64);
    }
  };
  auto request_scales = [&](int64_t from) {
    from = min(from, a.rows - 1);
    const int last = (int)min(a.rows - 1 - from, (int64_t)(kResidentRows - 1));
    scales = load_scales<NIB>(a.x_scale + from * NIB + (uint32_t)(min(lane & 31, last) * NIB));
  };
#pragma unroll
  for (int ib = 0; ib < NIB; ++ib) request(row0, ib);
  request_scales(row0);
  {
    // (once, through registers: copies straight to LDS reach its first 64 KiB only; every workgroup from another place on, or
    // all of them ask one channel of the L2 at a time)
    const u32x4 *w = reinterpret_cast<const u32x4 *>(a.w + (int64_t)ob0 * NIB * kBytes);
    u32x4 *to = reinterpret_cast<u32x4 *>(weights);
    const int tiles = blocks * NIB, first = group % tiles;
    static_assert(kBytes % 8192 == 0, "whole pieces for 512 threads");
    constexpr int kPieces = kBytes / 16 / 512;
    auto place = [](int i) { return TILES == 4 ? i : i / (TILES * kUnit) * (4 * kUnit) + i % (TILES * kUnit); };
    for (int t = 0; t < tiles; t += 4) {
      u32x4 v[4][kPieces];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t + i < tiles)
#pragma unroll
          for (int j = 0; j < kPieces; ++j) v[i][j] = w[(t + i + first) % tiles * (8 * kUnit) + place(j * 512 + threadIdx.x)];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t + i < tiles)
#pragma unroll
          for (int j = 0; j < kPieces; ++j) to[(t + i + first) % tiles * (kBytes / 16) + j * 512 + threadIdx.x] = v[i][j];
    }
    for (int j = threadIdx.x; j < blocks * kBlock; j += 512) {
      const int n = ob0 * kBlock + j;
      head[j / kBlock * kHead + j % kBlock] = a.bias && n < a.outs ? a.bias[n] : 0.0f;
    }
    if (IN8 && threadIdx.x < blocks) {
      uint32_t s = 0;
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib) s |= (uint32_t)a.w_scale[ib * a.nob + ob0 + threadIdx.x] << (8 * ib);
      head[threadIdx.x * kHead + kBlock] = __uint_as_float(s);
    }
  }
  __syncthreads();

  auto features = [&](int ob, auto last) {
    const float *b = head + ob * kHead;
    f32x16 acc[4];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(b + 64 * h + 4 * j);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j >> 2][4 * (j & 3) + e] = v[e];
    }
    multiply_resident<TILES, NIB>(acc, reinterpret_cast<const u32x4 *>(weights + ob * NIB * kBytes) + lane, __float_as_uint(b[kBlock]), x, scales,
                           [&](auto ib) {
                             if constexpr (decltype(last)::value) request(next_row0, ib);
                           },
                           std::integral_constant<bool, IN8>());
    hold(acc);
    if constexpr (decltype(last)::value) request_scales(next_row0);
    finish_lines<OUT, TILES>(acc, a, row0, ob0 + ob, lane, room);
  };
  for (; row0 < a.rows; row0 = next_row0) {
    int ticket = 0;
    if (lane == 0) ticket = atomicAdd(tickets, 1);
    next_row0 = row_of_ticket(__builtin_amdgcn_readfirstlane(ticket));
#pragma unroll
    for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        swap16(raw[ib][s][0], raw[ib][s][1]);
        x[ib][s] = join(raw[ib][s][0], raw[ib][s][1]);
      }
    for (int ob = 0; ob < blocks - 1; ++ob) features(ob, std::false_type());
    features(blocks - 1, std::true_type());
  }
}

template <bool IN8, int OUT, int NIB, int TILES = 4>
hipError_t launch_resident(hipStream_t st, int32_t P, const Product &a) {
  if constexpr (TILES == 4 && OUT != PR_B8_BLOCKS) {
    if constexpr (!IN8)
      if (a.outs <= 16) return launch_resident<IN8, OUT, NIB, 1>(st, P, a);
    if (a.outs <= 32) return launch_resident<IN8, OUT, NIB, 2>(st, P, a);
  }
  constexpr int kBytes = NIB * (IN8 ? kTileBytes : kWideTileBytes) / 4 * TILES, kMost = kResidentBytes / kBytes;
  constexpr auto kernel = linear_resident_kernel<IN8, OUT, NIB, TILES>;
  const hipError_t e = allow_full_lds<kernel>();
  if (e != hipSuccess) return e;
  const int32_t slabs = (a.nob + kMost - 1) / kMost, blocks = (a.nob + slabs - 1) / slabs;
  const size_t lds = kResidentWaves * kRoomBytes + (size_t)blocks * (kHead * 4 + kBytes);
  const int64_t tiles = (a.rows + kResidentWaves * kResidentRows - 1) / (kResidentWaves * kResidentRows);
  int64_t groups = std::max<int64_t>(1, compute_units() / ((int64_t)slabs * P));
  if (groups > tiles) groups = tiles;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((groups + 7) / 8 * 8 * slabs), 1, P), dim3(512), lds, st, a, blocks, slabs, (int32_t)groups);
  return hipGetLastError();
}

// More inputs.  A wavefront keeps 64 rows x 128 features in its accumulators, so a piece of the weights read from LDS feeds two
// matrix instructions of 64 cycles.  Nothing passes through registers on its way to LDS: four wavefronts share the weights, in
// two stages of 16 KiB (128 inputs in 8 bits, 64 decoded) with a barrier per stage; a wavefront's own rows have 8 KiB that are
// refilled as soon as they are in registers.  Rows and results go between memory and LDS in whole lines: 16 rows x 4 pieces of
// 16 bytes take a compute unit 100 cycles an instruction, 8 rows x 128 bytes a fifth.  Two workgroups live on a compute unit.
// The feature blocks of the same rows follow each other on one XCD, whose L2 then has the rows.  65536 x 1024 x 1024, blocks to
// bf16: 92 us, 1.5 PFLOP/s, matrix pipe busy 38 %; what is left are the barriers and the way out of 128 features at a time.
constexpr int kTilesRows = 256;
constexpr int kStageBytes = 16384, kRowsBytes = 64 * kBlock;

template <bool IN8, int OUT>
__global__ __launch_bounds__(256, 2) void linear_tiles_kernel(Product a, int32_t row_tiles) {
  constexpr int kStages = IN8 ? 1 : 2;  // of a block of inputs
  struct Lds {
    uint8_t ring[2][kStageBytes], own[4][kRowsBytes];
  };
  static_assert(sizeof(Lds) <= kCopyReach, "copies reach all of it");
  __shared__ __attribute__((aligned(16))) Lds lds;
  auto &ring = lds.ring;
  auto &own = lds.own;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, r32 = lane & 31;
  const int i = blockIdx.x >> 3, ob = i % a.nob, tile = i / a.nob * 8 + place_of(blockIdx.x, row_tiles, blockIdx.z);
  if (tile >= row_tiles) return;
  a.to_agent(blockIdx.z);
  const int64_t row0 = (int64_t)tile * kTilesRows + 64 * wave, last = a.rows - 1 - row0;  // (negative: no row is this wavefront's)
  const int64_t base_row = last < 0 ? 0 : row0;
  // rows as they are copied: 8 rows x 128 bytes an instruction, in the order of the places in LDS
  const uint8_t *x = static_cast<const uint8_t *>(a.x) + base_row * a.ldx;
  uint32_t x_at[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int r = 8 * j + (lane >> 3);
    x_at[j] = (uint32_t)(last < 0 ? 0 : min((int64_t)r, last)) * (uint32_t)a.ldx + 16 * ((lane & 7) ^ swizzle(r));
  }
  const uint8_t *xs[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) xs[t] = a.x_scale + (base_row + (last < 0 ? 0 : min((int64_t)(32 * t + r32), last))) * a.nib;
  const uint8_t *w = a.w + (int64_t)ob * a.nib * kStages * kStageBytes + wave * (kStageBytes / 4);
  const uint32_t ring_at = lds_address(&ring[0][0]) + wave * (kStageBytes / 4), own_at = lds_address(&own[wave][0]);
  auto copy_weights = [&](int stage) {
#pragma unroll
    for (int j = 0; j < kStageBytes / 4096; ++j)
      copy_to_lds(w + (int64_t)stage * kStageBytes + 1024 * j, lane * 16, ring_at + (stage & 1) * kStageBytes + 1024 * j);
  };
  auto copy_rows = [&](int ib) {
#pragma unroll
    for (int j = 0; j < 8; ++j) copy_to_lds(x + ib * kBlock, x_at[j], own_at + 1024 * j);
  };
  copy_weights(0);
  copy_rows(0);
  uint32_t scale[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) scale[t] = xs[t][0];
  f32x16 acc[2][4];
  start_sums(acc[0], a, ob, h);
#pragma unroll
  for (int f = 0; f < 4; ++f) acc[1][f] = acc[0][f];
  const int stages = a.nib * kStages;
  for (int ib = 0; ib < a.nib; ++ib) {
    arrived();
    i32x8 half[2][2];
    uint32_t now[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4 *p = reinterpret_cast<const u32x4 *>(&own[wave][(32 * t + r32) * kBlock]);
#pragma unroll
      for (int s = 0; s < 2; ++s) half[t][s] = join(p[(4 * s + 2 * h) ^ swizzle(r32)], p[(4 * s + 2 * h + 1) ^ swizzle(r32)]);
      now[t] = scale[t];
    }
    if (kStages * ib + 1 < stages) copy_weights(kStages * ib + 1);
    if (ib + 1 < a.nib) {
      reads_done();
      copy_rows(ib + 1);
#pragma unroll
      for (int t = 0; t < 2; ++t) scale[t] = xs[t][ib + 1];
    }
    if constexpr (IN8) {
      const u32x4 *wl = reinterpret_cast<const u32x4 *>(ring[ib & 1]) + lane;
      const uint32_t ws = a.w_scale[ib * a.nob + ob];
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const i32x8 wf = join(wl[128 * n], wl[128 * n + 64]);
#pragma unroll
        for (int t = 0; t < 2; ++t) multiply8<0>(acc[t][n & 3], wf, ws, half[t][n >> 2], now[t]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s == 1) {
          arrived();
          if (ib + 1 < a.nib) copy_weights(2 * ib + 2);
        }
        const u32x4 *wl = reinterpret_cast<const u32x4 *>(ring[s]) + lane;
        u32x4 part[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int p = 0; p < 4; ++p) part[t][p] = decode_part(half[t][s], p, power_of_byte(now[t]));
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          const u32x4 wf = wl[64 * n];
#pragma unroll
          for (int t = 0; t < 2; ++t) multiply16(acc[t][n >> 2], wf, part[t][n & 3]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) hold(acc[t]);
#pragma unroll
  for (int t = 0; t < 2; ++t) finish_lines<OUT>(acc[t], a, row0 + 32 * t, ob, lane, own[wave]);
}

// Plain rows, many of them.  A workgroup encodes 128 rows, a block of inputs at a time, for up to four blocks of features (fp32
// results; two for bf16 and blocks, so that rows are encoded twice for 512 features): eight lanes share a row (8 rows x 128 bytes
// an instruction: whole lines), the codes go to LDS, where every wavefront reads the rows it multiplies.  A wavefront has one block of features and 32 TILES rows; its weights come from L2 straight into
// registers, half a block of inputs ahead, and nobody else in the workgroup but the wavefront with its other rows wants them.
// One barrier a block; rows are requested a block ahead.  131009 rows of 301 in fp32 to 512 features in blocks: 160 (every
// wavefront encoding its own rows for its block of features, a lane a row) -> 128 us, where the bytes take 45; vector pipe busy
// 38 %, matrix pipe 9 %: 250 registers leave a workgroup of eight wavefronts alone on a compute unit, with nobody beside its round trips (a workgroup
// that goes on to its next tile, whose rows it requests early, spills and is slower: 150 us).
constexpr int kPlainRows = 128;

// The largest of eight neighbouring lanes, in all of them.
__device__ inline uint32_t max_of_eight(uint32_t m) {
  constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141;  // quads 1 0 3 2 and 2 3 0 1; eight lanes back to front
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, kSwap1, 15, 15, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, kSwap2, 15, 15, true));
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, kMirror8, 15, 15, true));
}

template <class T, bool IN8, int OUT, int WAVES, int TILES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void linear_plain_kernel(Product a, int32_t row_tiles, int32_t groups) {
  constexpr int kObs = WAVES * TILES / 4;                 // blocks of features of a workgroup
  constexpr int kEights = kPlainRows / WAVES / 8;         // of rows that a wavefront encodes
  constexpr int kPieces = sizeof(T), kIn = 16 / sizeof(T);  // of 16 bytes that a lane has of a row, their entries
  __shared__ __attribute__((aligned(16))) uint8_t codes[2][kPlainRows * kBlock], rooms[WAVES][kRoomBytes], bytes[2][kPlainRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, r32 = lane & 31;
  const int i = blockIdx.x >> 3, tile = i / groups * 8 + place_of(blockIdx.x, row_tiles, blockIdx.z);
  if (tile >= row_tiles) return;
  a.to_agent(blockIdx.z);
  const int64_t row0 = (int64_t)tile * kPlainRows;
  const int wanted = i % groups * kObs + wave % kObs;
  const bool idle = wanted >= a.nob;  // (encodes all the same)
  const int ob = idle ? a.nob - 1 : wanted;
  const int first = wave / kObs * (32 * TILES);  // of the workgroup's rows, to multiply
  const int part = lane & 7, enc0 = wave * (8 * kEights) + (lane >> 3);
  const T *row[kEights];
#pragma unroll
  for (int e = 0; e < kEights; ++e) row[e] = static_cast<const T *>(a.x) + min(row0 + enc0 + 8 * e, a.rows - 1) * a.ldx;
  u32x4 raw[kEights][kPieces];
  auto request = [&](int ib) {
#pragma unroll
    for (int e = 0; e < kEights; ++e)
#pragma unroll
      for (int k = 0; k < kPieces; ++k) raw[e][k] = request_piece(row[e], ib * kBlock + (8 * k + part) * kIn, a.ins);
  };
  auto encode = [&](int ib, int to) {
    if ((ib + 1) * kBlock > a.ins) {
#pragma unroll
      for (int e = 0; e < kEights; ++e)
#pragma unroll
        for (int k = 0; k < kPieces; ++k) raw[e][k] = settle_piece<T>(raw[e][k], ib * kBlock + (8 * k + part) * kIn, a.ins);
    }
#pragma unroll
    for (int e = 0; e < kEights; ++e) {
      float v[16];
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
#pragma unroll
        for (int j = 0; j < kIn; ++j)
          v[k * kIn + j] = __uint_as_float(sizeof(T) == 4 ? raw[e][k][j & 3] : j & 1 ? raw[e][k][j >> 1] & 0xffff0000u : raw[e][k][j >> 1] << 16);
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) m = max(m, finite_bits(v[j]));
      const int exp = exponent_of(max_of_eight(m)), r = enc0 + 8 * e;
      const float inv = power(-exp);
      uint32_t c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = codes4(v[4 * j] * inv, v[4 * j + 1] * inv, v[4 * j + 2] * inv, v[4 * j + 3] * inv);
      uint8_t *at = &codes[to][r * kBlock];
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int col = (8 * k + part) * kIn;
        uint8_t *p = at + (((col >> 4) ^ swizzle(r)) << 4) + (col & 15);
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t *>(p) = c[k];
        else *reinterpret_cast<u32x2 *>(p) = u32x2{c[2 * k], c[2 * k + 1]};
      }
      if (part == 0) bytes[to][r] = (uint8_t)(exp + 127);
    }
  };
  const int32_t tile_bytes = IN8 ? kTileBytes : kWideTileBytes;
  const u32x4 *w = reinterpret_cast<const u32x4 *>(a.w + (int64_t)ob * a.nib * tile_bytes) + lane;
  // Weights under way: the four tiles of half a block in 8 bits, four parts of a tile decoded
  constexpr int kRing = 4, kSteps = IN8 ? 8 : 32;  // pieces under way, and of a block
  i32x8 ring8[IN8 ? kRing : 1];
  u32x4 ring16[IN8 ? 1 : kRing];
  auto request_weights = [&](const u32x4 *from, int n, int place) {
    if constexpr (IN8) ring8[place] = join(from[128 * n], from[128 * n + 64]);
    else ring16[place] = from[64 * n];
  };
  request(0);
#pragma unroll
  for (int n = 0; n < kRing; ++n) request_weights(w, n, n);
  f32x16 acc[TILES][4];
  start_sums(acc[0], a, ob, h);
#pragma unroll
  for (int t = 1; t < TILES; ++t)
#pragma unroll
    for (int f = 0; f < 4; ++f) acc[t][f] = acc[0][f];
  encode(0, 0);
  if (a.nib > 1) request(1);
  for (int ib = 0; ib < a.nib; ++ib) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (all codes of this block are written, those of the one before are read)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int at = ib & 1;
    i32x8 half[TILES];
    uint32_t byte[TILES];
    auto read_half = [&](int s) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int r = first + 32 * t + r32;
        const u32x4 *p = reinterpret_cast<const u32x4 *>(&codes[at][r * kBlock]);
        half[t] = join(p[(4 * s + 2 * h) ^ swizzle(r)], p[(4 * s + 2 * h + 1) ^ swizzle(r)]);
        byte[t] = bytes[at][r];
      }
    };
    const u32x4 *now = w + (int64_t)ib * (tile_bytes / 16), *next = ib + 1 < a.nib ? now + tile_bytes / 16 : now;
    const uint32_t ws = IN8 ? a.w_scale[ib * a.nob + ob] : 0;
    u32x4 x16[TILES][4];
    each<kSteps>([&](auto step) {
      constexpr int n = step;
      if constexpr (n % (kSteps / 2) == 0) read_half(n / (kSteps / 2));
      if constexpr (IN8) {
#pragma unroll
        for (int t = 0; t < TILES; ++t) multiply8<0>(acc[t][n & 3], ring8[n % kRing], ws, half[t], byte[t]);
      } else {
        if constexpr ((n & 15) < 4) {
#pragma unroll
          for (int t = 0; t < TILES; ++t) x16[t][n & 3] = decode_part(half[t], n & 3, power_of_byte(byte[t]));
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) multiply16(acc[t][(n >> 2) & 3], ring16[n % kRing], x16[t][n & 3]);
      }
      request_weights(n + kRing < kSteps ? now : next, (n + kRing) % kSteps, n % kRing);
      __builtin_amdgcn_sched_barrier(kVectorMayPass);
    });
    __builtin_amdgcn_sched_barrier(0);
    if (ib + 1 < a.nib) {
      encode(ib + 1, at ^ 1);
      if (ib + 2 < a.nib) request(ib + 2);
    }
  }
  if (idle) return;
#pragma unroll
  for (int t = 0; t < TILES; ++t) hold(acc[t]);
#pragma unroll
  for (int t = 0; t < TILES; ++t) finish_lines<OUT>(acc[t], a, row0 + first + 32 * t, ob, lane, rooms[wave]);
}

// A launch has fewer than 2^32 threads: 2 for each row and block of features here (4 wavefronts for 128 rows and one, 8 for two).
// With a billion rows of more than one block linear_kernel has them on another axis.
inline bool plain_fits(const Product &a) { return (a.rows + 8 * kPlainRows) * (a.nob == 1 ? 1 : (a.nob + 1) / 2 * 2) < (int64_t)1 << 31; }

template <class T, bool IN8, int OUT>
hipError_t launch_plain(hipStream_t st, int32_t P, const Product &a) {
  const int64_t tiles = (a.rows + kPlainRows - 1) / kPlainRows;
  auto go = [&](auto kernel, int obs, int waves) {
    const int32_t groups = (a.nob + obs - 1) / obs;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + 7) / 8 * 8 * groups), 1, P), dim3(64 * waves), 0, st, a, (int32_t)tiles, groups);
    return hipGetLastError();
  };
  // the more features share a workgroup the less often rows are encoded, unless that leaves compute units without one
  auto fills = [&](int obs) { return a.nob > obs / 2 && tiles * P * ((a.nob + obs - 1) / obs) >= compute_units(); };
  if constexpr (!IN8)
    if (fills(4)) return go(linear_plain_kernel<T, IN8, OUT, 8, 2>, 4, 8);
  if (fills(2)) return go(linear_plain_kernel<T, IN8, OUT, 8, 1>, 2, 8);
  return go(linear_plain_kernel<T, IN8, OUT, 4, 1>, 1, 4);
}

// Input gradients of many rows.  A wavefront forms g for its 32 rows and up to 128 NB outputs of the layer once, in registers
// (they are the products' operand as they stand), and takes them through all inputs, whose weights pass through LDS, 32 KiB (a
// block of either side) at a time and one ahead, for eight wavefronts.  With more than 512 outputs a wavefront needs a SIMD's
// registers for itself.  Where rows alone do not fill the compute units the inputs are dealt to several workgroups too.
// 131072 x 512 x 512 in bf16: 101 to 110 us, 650 TFLOP/s, where the bytes (335 MB) take 67 and the products 28 alone.  240
// registers leave one workgroup on a compute unit, so its 512 go in two rounds, each of which forms g, multiplies and stores in step.
// 65537 x 512 x 30: 29 us, where the bytes take 15: 140 registers leave one on a compute unit there too, and the last of 257, of
// a single row, has a round of its own.
template <class T, int OUT, int NB>
__global__ __launch_bounds__(NB <= 4 ? 512 : 256, NB <= 4 ? 2 : 1) void input_grads_kernel(Product a, int32_t slab_blocks) {
  constexpr int kWaves = NB <= 4 ? 8 : 4, kPart = kWideTileBytes / kWaves;
  struct Lds {
    uint8_t ring[2][kWideTileBytes], rooms[kWaves][kRoomBytes];
  };
  static_assert(offsetof(Lds, rooms) <= kCopyReach, "copies reach the ring");
  __shared__ __attribute__((aligned(16))) Lds lds;
  auto &ring = lds.ring;
  auto &rooms = lds.rooms;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  a.to_agent(blockIdx.z);
  a.act = 0;  // (as launched: told here, the way out has no activation to form and leave out)
  const int64_t row0 = ((int64_t)blockIdx.x * kWaves + wave) * 32;
  const uint32_t ring_at = lds_address(&ring[0][0]) + wave * kPart;
  const int ob0 = blockIdx.y * slab_blocks, ob1 = min(ob0 + slab_blocks, a.nob);
  const uint8_t *w = a.w + (int64_t)ob0 * a.nib * kWideTileBytes + wave * kPart;
  auto copy_weights = [&](int stage) {
#pragma unroll
    for (int j = 0; j < kPart / 1024; ++j)
      copy_to_lds(w + (int64_t)stage * kWideTileBytes + 1024 * j, lane * 16, ring_at + (stage & 1) * kWideTileBytes + 1024 * j);
  };
  copy_weights(0);
  u32x4 g[NB][8];
  {
    // 16 rows x 64 bytes an instruction; lane groups then swap what they have of each other's rows
    const int64_t from = min(row0, a.rows - 1);
    const int last = (int)min(a.rows - 1 - from, (int64_t)31);
    int row[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) row[t] = min(16 * t + (lane & 15), last);
    const int group = lane >> 4;
    const T *dy = static_cast<const T *>(a.x) + from * a.ldx;
    const uint8_t *y = a.out ? a.out + from * a.nib * kBlock : nullptr, *ys = a.out ? a.out_scale + from * a.nib : nullptr;
    const int own = min(lane & 31, last);
    // which 16 bytes of 64 a lane group asks for: after the swap lanes 32 h .. have pieces h and 2 + h
    const int order = ((group & 1) << 1) | (group >> 1);
    each<NB>([&](auto block) {
      constexpr int ib = block;
      if (ib < a.nib) {
        const bool whole = (ib + 1) * kBlock <= a.ins, longs = ib > 0 || a.ins >= (int)(16 / sizeof(T));
        u32x4 code[2][2];  // [half][rows]
        float scale = 0.0f;
        if (y) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t)
              code[s][t] = *reinterpret_cast<const u32x4 *>(y + (uint32_t)(row[t] * a.nib + ib) * kBlock + 64 * s + 16 * group);
          scale = power_of_byte(ys[(uint32_t)(own * a.nib + ib)]);
        }
        float v[2][2][16];  // [half][parts 2 i, 2 i + 1][..]
        if constexpr (sizeof(T) == 2) {
          u32x4 raw[2][2][2];
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                const int col = ib * kBlock + 64 * s + 32 * c + 8 * order;
                const T *p = dy + row[t] * a.ldx;
                raw[s][c][t] = longs ? request_piece(p, col, a.ins) : short_piece(p, a.ins);
              }
            }
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              if (!whole) {
#pragma unroll
                for (int t = 0; t < 2; ++t) raw[s][c][t] = settle_piece<T>(raw[s][c][t], ib * kBlock + 64 * s + 32 * c + 8 * order, a.ins);
              }
              swap16(raw[s][c][0], raw[s][c][1]);
#pragma unroll
              for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  v[s][c][8 * q + 2 * i] = __uint_as_float(raw[s][c][q][i] << 16);
                  v[s][c][8 * q + 2 * i + 1] = __uint_as_float(raw[s][c][q][i] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            u32x4 pieces[4][2];
#pragma unroll
            for (int part = 0; part < 4; ++part)
#pragma unroll
              for (int t = 0; t < 2; ++t)
                pieces[part][t] = longs ? request_piece(dy + row[t] * a.ldx, ib * kBlock + 64 * s + 16 * part + 4 * group, a.ins) : short_piece(dy + row[t] * a.ldx, a.ins);
#pragma unroll
            for (int part = 0; part < 4; ++part) {
              u32x4 (&raw)[2] = pieces[part];
              if (!whole) {
#pragma unroll
                for (int t = 0; t < 2; ++t) raw[t] = settle_piece<float>(raw[t], ib * kBlock + 64 * s + 16 * part + 4 * group, a.ins);
              }
              swap16(raw[0], raw[1]);  // 4 of the 8 inputs each
#pragma unroll
              for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[s][part >> 1][8 * (part & 1) + 4 * q + i] = __uint_as_float(raw[q][i]);
            }
          }
        }
        if (y) {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            swap16(code[s][0], code[s][1]);  // 16 codes of parts 2 h and 2 h + 1; lanes 32 apart want 8 of each part
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              u32x4 &c = code[s][q];
              const auto a0 = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false), a1 = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
              // [0]: part q (of lanes below 32), [1]: part 2 + q
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                times_derivative(&v[s][k][8 * q], a0[k], scale);
                times_derivative(&v[s][k][8 * q + 4], a1[k], scale);
              }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float *p = &v[i >> 2][(i >> 1) & 1][8 * (i & 1)];
          g[ib][i] = u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
        }
      }
    });
  }
  const int stages = (ob1 - ob0) * a.nib;
  int stage = 0;
  bool stored = false;  // since the copies of this stage: a whole tile
  for (int ob = ob0; ob < ob1; ++ob) {
    f32x16 acc[4];
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[f][j] = 0.0f;
    each<NB>([&](auto block) {
      constexpr int ib = block;
      if (ib < a.nib) {
        if (stored) arrived_before<kLineStores<OUT>>();
        else arrived();
        stored = false;
        if (stage + 1 < stages) copy_weights(stage + 1);
        const u32x4 *wl = reinterpret_cast<const u32x4 *>(ring[stage & 1]) + lane;
        constexpr int kAhead = 4;
        u32x4 next[kAhead + 1];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) next[n] = wl[64 * n];
        each<32>([&](auto piece) {
          constexpr int n = piece;
          if constexpr (n + kAhead < 32) next[(n + kAhead) % (kAhead + 1)] = wl[64 * (n + kAhead)];
          multiply16(acc[(n >> 2) & 3], next[n % (kAhead + 1)], g[ib][4 * (n >> 4) + (n & 3)]);
          __builtin_amdgcn_sched_barrier(kVectorMayPass);
        });
        ++stage;
      }
    });
    hold(acc);
    stored = finish_lines<OUT>(acc, a, row0, ob, lane, rooms[wave]);
  }
}

// Rows that a workgroup for 32 rows x 32 features serves best: the weights are what has to be read.  Of several agents those
// with up to 128 rows each; more of them are a long launch of workgroups that have few blocks of inputs to split (64 agents x
// 1000 rows of 301 to 256 outputs: 80 us, in tiles 31; 57 agents x 1 row of 1024 to 1024: 14 us this way).
bool few_rows(int32_t P, int64_t rows) { return rows <= 128 || P * rows <= 1024; }

template <class T, int OUT>
bool launch_input_grads(hipStream_t st, int32_t P, const Product &a) {
  // (g of more than 512 outputs takes a workgroup of few rows, of which there are many, longer than its products: 995 x 1024 x
  // 1024 32 us that way, 25 this)
  if ((few_rows(P, a.rows) && (a.nib <= 4 || a.rows < 256)) || a.nib > 8 || !lines_fit(a)) return false;
  const int per = a.nib <= 4 ? 256 : 128;
  const int64_t groups = (a.rows + per - 1) / per;
  const int32_t slabs = (int32_t)std::max<int64_t>(1, std::min<int64_t>(a.nob, compute_units() / (groups * P))), blocks = (a.nob + slabs - 1) / slabs;
  const dim3 grid((unsigned)groups, (a.nob + blocks - 1) / blocks, P), block(2 * per);
  if (a.nib == 1) hipLaunchKernelGGL((input_grads_kernel<T, OUT, 1>), grid, block, 0, st, a, blocks);
  else if (a.nib == 2) hipLaunchKernelGGL((input_grads_kernel<T, OUT, 2>), grid, block, 0, st, a, blocks);
  else if (a.nib <= 4) hipLaunchKernelGGL((input_grads_kernel<T, OUT, 4>), grid, block, 0, st, a, blocks);
  else hipLaunchKernelGGL((input_grads_kernel<T, OUT, 8>), grid, block, 0, st, a, blocks);
  return true;
}

template <int SRC, bool IN8, int OUT>
hipError_t launch_rows(hipStream_t st, int32_t P, const Product &a) {
  if constexpr (SRC == kGradF32 || SRC == kGradBf16)
    if (launch_input_grads<std::conditional_t<SRC == kGradF32, float, uint16_t>, OUT>(st, P, a)) return hipGetLastError();
  if constexpr (SRC == kBlocks)
    if (!few_rows(P, a.rows) && lines_fit(a)) {
      // Resident weights are paid for at the start: with several blocks of features by the second tile of a workgroup's rows only
      // (to bf16, resident and in tiles: 5000 x 512 x 512 17 and 12.5 us, 26861 x 256 x 256 15 and 12.4, 60000 x 256 x 256 17.8
      // and 16.5; one block, 20000 x 128 x 128 8.6 and 9.2, 1577 x 256 x 75 10.6 and 13.1)
      if (a.nob == 1 || P * ((a.rows + 255) / 256) > compute_units()) {
        if (a.nib == 1) return launch_resident<IN8, OUT, 1>(st, P, a);
        if (a.nib == 2) return launch_resident<IN8, OUT, 2>(st, P, a);
        if (a.nib == 3) return launch_resident<IN8, OUT, 3>(st, P, a);
        if (a.nib == 4) return launch_resident<IN8, OUT, 4>(st, P, a);
      }
      const int32_t tiles = (int32_t)((a.rows + kTilesRows - 1) / kTilesRows);
      hipLaunchKernelGGL((linear_tiles_kernel<IN8, OUT>), dim3((unsigned)((tiles + 7) / 8 * 8 * a.nob), 1, P), dim3(256), 0, st, a, tiles);
      return hipGetLastError();
    }
  bool few = few_rows(P, a.rows);
  if constexpr (SRC == kF32 || SRC == kBf16) {
    // (one block of features, and workgroups of 128 rows for less than half of the compute units: 3758 rows of 1261 to 128 outputs
    // in bf16 32 us that way, 21 this; with more features rows are encoded too often, 3000 x 900 x 512 24 us that way, 32 this)
    few = few || (a.nob == 1 && a.nib >= 4 && P * ((a.rows + kPlainRows - 1) / kPlainRows) < compute_units() / 2);
    if (!few && a.ins >= 8 && lines_fit(a) && plain_fits(a)) return launch_plain<std::conditional_t<SRC == kF32, float, uint16_t>, IN8, OUT>(st, P, a);
  }
  if (few) {
    const int split = OUT == PR_B8_BLOCKS ? 1 : 4;
    hipLaunchKernelGGL((linear_few_kernel<SRC, IN8, OUT>), dim3((unsigned)((a.rows + 31) / 32), a.nob * split, P), dim3(1024), 0, st, a);
    return hipGetLastError();
  }
  // (blocks to blocks have left by now: their rows are close together)
  if constexpr (SRC != kBlocks || OUT != PR_B8_BLOCKS)
    hipLaunchKernelGGL((linear_kernel<SRC, IN8, OUT>), dim3((unsigned)((a.rows + 127) / 128), a.nob, P), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int SRC>
hipError_t launch_out(hipStream_t st, int32_t P, const Product &a, int32_t y_kind) {
  if (y_kind == PR_B8_F32) return launch_rows<SRC, false, PR_B8_F32>(st, P, a);
  if (y_kind == PR_B8_BF16) return launch_rows<SRC, true, PR_B8_BF16>(st, P, a);
  return launch_rows<SRC, true, PR_B8_BLOCKS>(st, P, a);
}

template <int SRC>
hipError_t launch_back(hipStream_t st, int32_t P, const Product &a, int32_t dx_kind) {
  if (dx_kind == PR_B8_F32) return launch_rows<SRC, false, PR_B8_F32>(st, P, a);
  return launch_rows<SRC, false, PR_B8_BF16>(st, P, a);
}

}  // namespace
}  // namespace b8

using namespace b8;

hipError_t launch_block8_linear(hipStream_t st, const Block8Linear &l) {
  const WeightPlan w = weight_plan(l.in_dim, l.out_dim);
  const uint8_t *packed = static_cast<const uint8_t *>(l.packed);
  Product a = {};
  a.rows = l.rows, a.ins = l.in_dim, a.outs = l.out_dim, a.nib = w.nib, a.nob = w.nob, a.act = l.tanh;
  a.x = l.x, a.x_scale = l.x_scale, a.ldx = l.x_kind == PR_B8_BLOCKS ? (int64_t)w.nib * kBlock : l.ldx;
  a.w = packed, a.w_scale = packed + w.scale_at, a.w_stride = w.stride;
  if (l.y_kind == PR_B8_F32) a.w += w.wide_at;  // (decoded)
  a.bias = l.bias;
  a.y = l.y, a.y_scale = l.y_scale, a.ldy = l.y_kind == PR_B8_BLOCKS ? (int64_t)w.nob * kBlock : l.ldy;
  a.x_size = l.x_kind == PR_B8_F32 ? 4 : l.x_kind == PR_B8_BF16 ? 2 : 1;
  a.y_size = l.y_kind == PR_B8_F32 ? 4 : l.y_kind == PR_B8_BF16 ? 2 : 1;
  if (l.x_kind == PR_B8_BLOCKS) return launch_out<kBlocks>(st, l.P, a, l.y_kind);
  if (l.x_kind == PR_B8_F32) return launch_out<kF32>(st, l.P, a, l.y_kind);
  return launch_out<kBf16>(st, l.P, a, l.y_kind);
}

hipError_t launch_block8_input_grads(hipStream_t st, const Block8Grads &l) {
  const WeightPlan w = weight_plan(l.in_dim, l.out_dim);
  const uint8_t *packed = static_cast<const uint8_t *>(l.packed);
  Product a = {};
  a.rows = l.rows, a.ins = l.out_dim, a.outs = l.in_dim, a.nib = w.nob, a.nob = w.nib, a.act = 0;
  a.x = l.dy, a.ldx = l.lddy, a.out = l.y, a.out_scale = l.y_scale;
  a.w = packed + w.back_at, a.w_stride = w.stride;
  a.y = l.dx, a.ldy = l.lddx;
  a.x_size = l.dy_kind == PR_B8_F32 ? 4 : 2;
  a.y_size = l.dx_kind == PR_B8_F32 ? 4 : 2;
  if (l.dy_kind == PR_B8_F32) return launch_back<kGradF32>(st, l.P, a, l.dx_kind);
  return launch_back<kGradBf16>(st, l.P, a, l.dx_kind);
}

}  // namespace pod
