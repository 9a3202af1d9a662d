// Backward pass of a layer on 8-bit blocks: dW = x^T g and db = sum_r g from the
// checkpoints (dx = g W^T is a product like the forward one, pod_block8_linear.hip).
//
// The contraction runs over rows, the slow axis of both operands.  A workgroup owns a tile
// of dW and a run of rows; runs (but a single one) are added up by a second launch, in a
// fixed order, so results do not depend on the schedule.  32 rows at a time are decoded (x) or formed (g) on their
// way from registers to LDS, row by row as they lie in memory, and the transposing LDS
// read hands each lane eight rows of its column.  Rows are requested two stages ahead.
//
// 131072 x 512 x 512 in bf16: 109 to 120 us, 600 TFLOP/s, 2.4 TB/s, and 11 us for the sums of its 64 runs.  Matrix pipe, vector
// pipe (decoding x, forming g) and LDS are busy 30 to 45 % of the time each, one stage's work between two barriers; nothing but
// their order bounds it.  Every tile of dW decodes x and forms g again: 27238 x 736 x 736 from fp32, 104 us, does so six and
// three times.  Of the 256 x 128 tile those from fp32 with an activation spill 10 or 11 registers, from bf16 with an activation and
// ragged outputs 3.
#include <algorithm>

#include "pod_block8.h"
#include "pod_block8_product.h"

namespace pod {

hipError_t launch_block8_input_grads(hipStream_t st, const Block8Grads &l);

namespace b8 {
namespace {

constexpr int kStage = 32;  // rows

typedef short i16x4 __attribute__((ext_vector_type(4)));

// Stages of 32 rows x COLS bf16 in LDS: where column `col` is.  A row's 64-byte units are swapped by its lowest two bits (the
// four rows that 16 lanes of a transposing read take 32 bytes of are then on banks of their own, and so are the two rows that 16
// lanes write 128 bytes of), and the 16-byte pieces of a unit by its lowest bit.
template <int COLS>
__device__ inline int stage_at(int row, int col) {
  const int swap = COLS >= 128 ? ((row & 1) << 1) | ((row >> 1) & 1) : 0;
  return row * (2 * COLS) + (((col >> 5) ^ swap) << 6) + ((((col >> 3) & 3) ^ (row & 1)) << 4) + 2 * (col & 7);
}

struct WeightGrads {
  Product a;  // rows dy of `ins` outputs of the layer; outs: its inputs
  const uint8_t *x, *x_scale;
  int32_t tiles_k, tiles, runs;
  int64_t run;
  float *parts, *db_parts;
  int32_t P;
};

template <class T, bool ACT, bool WHOLE, int TK, int TN, int WK, int WN>
__global__ __launch_bounds__(64 * WK * WN, 2) void weight_grads_kernel(WeightGrads d) {
  constexpr int kThreads = 64 * WK * WN, kK = 32 * TK * WK, kN = 32 * TN * WN;
  // A thread's share of a stage: pieces of 16 bytes of one row, so far apart that eight threads read 128 bytes side by side.
  constexpr int kXRow = 8, kXShare = kK / 128;                          // 16 codes of x from each block
  constexpr int kGPiece = 16 / sizeof(T), kGRow = 8 <= kN / kGPiece ? 8 : kN / kGPiece, kGShare = kN / (kGRow * kGPiece);
  constexpr int kGThreads = kStage * kGRow, kXBytes = kStage * kK * 2, kGBytes = kStage * kN * 2;
  static_assert(kN <= kBlock, "one scale for a row's outputs");
  constexpr int kAhead = 2, kRound = kAhead % 2 ? 2 * kAhead : kAhead;  // stages under way; stages of the loop's body
  static_assert(kStage * kXRow == kThreads && kGThreads <= kThreads && kK % kBlock == 0, "shares are whole");
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][kXBytes + kGBytes];
  Product &a = d.a;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int bi = blockIdx.x >> 3, tile = bi % d.tiles, p = blockIdx.z;
  const int part = bi / d.tiles * 8 + place_of(blockIdx.x, d.runs, (int64_t)p * d.tiles + tile);
  if (part >= d.runs) return;
  const int k0 = tile % d.tiles_k * kK, n0 = tile / d.tiles_k * kN, xb = (a.outs + kBlock - 1) / kBlock;
  const int64_t r0 = part * d.run, r1 = min(r0 + d.run, a.rows), first = p * a.rows;
  const T *dy = static_cast<const T *>(a.x) + first * a.ldx;
  const uint8_t *x8 = d.x + first * xb * kBlock, *x8_scale = d.x_scale + first * xb;
  const uint8_t *out = ACT ? a.out + first * a.nib * kBlock : nullptr, *out_scale = ACT ? a.out_scale + first * a.nib : nullptr;

  const int xrow = t / kXRow, xcol = t % kXRow * 16, grow = t / kGRow % kStage, gcol = t % kGRow * kGPiece;
  const bool has_g = kGThreads == kThreads || t < kGThreads;
  const int nblocks = min(xb - (k0 >> 7), kXShare);  // of x that are there
  struct Raw {
    u32x4 x[kXShare], g[kGShare];
    uint32_t y[kGShare][kGPiece / 4], x_scale[kXShare], y_scale;
  };
  // (rows behind the run are zero; blocks behind x's last one are that one again, and what they give is not stored)
  auto request = [&](Raw &w, int64_t from) {
    const int rows = (int)max(min(r1 - from, (int64_t)kStage), (int64_t)0);
    from = min(from, r1 - 1);
    const int last = (int)min(r1 - 1 - from, (int64_t)(kStage - 1)), xr = min(xrow, last), gr = min(grow, last);
    const uint8_t *x = x8 + from * (xb * kBlock) + k0 + (uint32_t)(xr * (xb * kBlock) + xcol), *xs = x8_scale + from * xb + (k0 >> 7);
#pragma unroll
    for (int i = 0; i < kXShare; ++i) {
      const int block = min(i, nblocks - 1);
      w.x[i] = *reinterpret_cast<const u32x4 *>(x + block * kBlock);
      w.x_scale[i] = xs[(uint32_t)(xr * xb + block)];
    }
    const T *g = dy + from * a.ldx + gr * a.ldx;
    if (WHOLE) {
#pragma unroll
      for (int i = 0; i < kGShare; ++i) w.g[i] = reinterpret_cast<const U32x4At2 *>(g + n0 + gcol + i * kGRow * kGPiece)->v;
    } else if (a.ins >= kGPiece) {
#pragma unroll
      for (int i = 0; i < kGShare; ++i) w.g[i] = request_piece(g, n0 + gcol + i * kGRow * kGPiece, a.ins);
    } else {
#pragma unroll
      for (int i = 0; i < kGShare; ++i) w.g[i] = short_piece(g, a.ins);
    }
    if constexpr (ACT) {  // (blocks are whole: columns behind the last output are there)
      const uint8_t *y = out + from * (a.nib * kBlock) + n0 + (uint32_t)(gr * (a.nib * kBlock) + gcol);
#pragma unroll
      for (int i = 0; i < kGShare; ++i) {
        if constexpr (kGPiece == 8) {
          const u32x2 v = *reinterpret_cast<const u32x2 *>(y + i * kGRow * kGPiece);
          w.y[i][0] = v[0], w.y[i][kGPiece / 4 - 1] = v[1];
        } else {
          w.y[i][0] = *reinterpret_cast<const uint32_t *>(y + i * kGRow * kGPiece);
        }
      }
      w.y_scale = (out_scale + from * a.nib + (n0 >> 7))[(uint32_t)(gr * a.nib)];
    }
    if (rows < kStage) {
      if (xrow >= rows)
#pragma unroll
        for (int i = 0; i < kXShare; ++i) w.x[i] = u32x4{0, 0, 0, 0};
      if (grow >= rows)
#pragma unroll
        for (int i = 0; i < kGShare; ++i) w.g[i] = u32x4{0, 0, 0, 0};
    }
  };
  auto stage = [&](const Raw &w, uint8_t *to) {
#pragma unroll
    for (int i = 0; i < kXShare; ++i) {
      const float s = power_of_byte(w.x_scale[i]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x2 c = decode4(w.x[i][2 * j], s), e = decode4(w.x[i][2 * j + 1], s);
        *reinterpret_cast<u32x4 *>(to + stage_at<kK>(xrow, i * kBlock + xcol + 8 * j)) = u32x4{c[0], c[1], e[0], e[1]};
      }
    }
    if (!has_g) return;
    const float ys = ACT ? power_of_byte(w.y_scale) : 0.0f;
#pragma unroll
    for (int i = 0; i < kGShare; ++i) {
      float v[kGPiece];
      spread(v, WHOLE || n0 + kN <= a.ins ? w.g[i] : settle_piece<T>(w.g[i], n0 + gcol + i * kGRow * kGPiece, a.ins), static_cast<const T *>(nullptr));
      if constexpr (ACT) {
#pragma unroll
        for (int j = 0; j < kGPiece / 4; ++j) times_derivative(v + 4 * j, w.y[i][j], ys);
      }
      uint32_t g[kGPiece / 2];
#pragma unroll
      for (int j = 0; j < kGPiece / 2; ++j) g[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
      uint8_t *at = to + kXBytes + stage_at<kN>(grow, gcol + i * kGRow * kGPiece);
      if constexpr (kGPiece == 8) *reinterpret_cast<u32x4 *>(at) = u32x4{g[0], g[1], g[2], g[3]};
      else *reinterpret_cast<u32x2 *>(at) = u32x2{g[0], g[1]};
    }
  };
  f32x16 acc[TK][TN];
#pragma unroll
  for (int i = 0; i < TK; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  // lanes 16 q .. of a transposing read: columns 16 (q % 2) .. + 15 of a tile, rows 8 (q / 2) .. + 3, and + 4 .. + 7
  const int col16 = 16 * ((lane >> 4) & 1) + 4 * (lane & 3), row8 = 8 * (lane >> 5) + ((lane & 15) >> 2);
  const int xw = 32 * TK * (wave % WK), gw = 32 * TN * (wave / WK);
  auto four = [&](auto cols, const uint8_t *from, int row, int col) {
    typedef __attribute__((address_space(3))) i16x4 *Ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(from + stage_at<decltype(cols)::value>(row, col)));
  };
  auto column = [&](auto cols, const uint8_t *from, int row, int col) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(four(cols, from, row, col), four(cols, from, row + 4, col), 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // db: a wavefront has 32 columns of g, a lane half of the rows of one
  float sum = 0.0f;
  const bool sums = k0 == 0 && wave < kN / 32;
  auto products = [&](const uint8_t *from) {
    if (sums) {
#pragma unroll
      for (int s = 0; s < kStage / 8; ++s) {
        const i16x4 v = four(std::integral_constant<int, kN>(), from + kXBytes, 8 * s + row8 - 4 * (lane >> 5), 32 * wave + col16);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += __uint_as_float((uint32_t)(uint16_t)v[j] << 16);
      }
    }
#pragma unroll
    for (int s = 0; s < kStage / 16; ++s) {
      bf16x8 x[TK], g[TN];
#pragma unroll
      for (int i = 0; i < TK; ++i) x[i] = column(std::integral_constant<int, kK>(), from, 16 * s + row8, xw + 32 * i + col16);
#pragma unroll
      for (int j = 0; j < TN; ++j) g[j] = column(std::integral_constant<int, kN>(), from + kXBytes, 16 * s + row8, gw + 32 * j + col16);
#pragma unroll
      for (int i = 0; i < TK; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], g[j], acc[i][j], 0, 0, 0);
    }
  };
  // all writes of the present stage are done, and all reads of the one before
  auto meet = [] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  Raw raw[kAhead];
  each<kAhead>([&](auto i) { request(raw[i], r0 + i * kStage); });
  stage(raw[0], lds[0]);
  for (int64_t r = r0; r < r1; r += kRound * kStage)
    each<kRound>([&](auto i) {
      meet();
      request(raw[i % kAhead], r + (i + kAhead) * kStage);
      products(lds[i & 1]);
      stage(raw[(i + 1) % kAhead], lds[(i + 1) & 1]);
    });
  const int ins = a.outs, outs = a.ins;  // of the layer
  float *w = d.parts + ((int64_t)part * d.P + p) * ins * outs;
#pragma unroll
  for (int i = 0; i < TK; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int k = k0 + xw + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3), n = n0 + gw + 32 * j + (lane & 31);
        if (k < ins && n < outs) w[(int64_t)k * outs + n] = acc[i][j][e];
      }
  if (!sums) return;
  sum += __shfl_xor(sum, 32);
  const int n = n0 + 32 * wave + (lane & 31);
  if (lane < 32 && n < outs) d.db_parts[((int64_t)part * d.P + p) * outs + n] = sum;
}

// out[i] = sum over the runs; dW and db in one launch.  A workgroup has 256 / SPLITS entries, and SPLITS threads for the runs of
// one, whose sums are added up in order: few entries of many runs would leave compute units idle (228 runs of 15390, the gradients
// of 65537 x 512 x 30: 6 us).
template <int SPLITS>
__global__ __launch_bounds__(256) void join_kernel(int32_t runs, int64_t nw, int64_t nb, const float *__restrict__ parts,
                                                   const float *__restrict__ db_parts, float *__restrict__ dW, float *__restrict__ db) {
  constexpr int kEntries = 256 / SPLITS;
  __shared__ float sums[SPLITS][kEntries];
  const int entry = threadIdx.x % kEntries, split = threadIdx.x / kEntries;
  int64_t i = (int64_t)blockIdx.x * kEntries + entry;
  const float *from = parts;
  float *to = dW;
  int64_t n = nw;
  if (i >= nw) from = db_parts, to = db, n = nb, i -= nw;
  float s = 0.0f;
  if (i < n) {
#pragma unroll 8
    for (int r = split; r < runs; r += SPLITS) s += from[r * n + i];
  }
  if constexpr (SPLITS > 1) {
    sums[split][entry] = s;
    __syncthreads();
    if (split > 0) return;
#pragma unroll
    for (int k = 1; k < SPLITS; ++k) s += sums[k][entry];
  }
  if (i < n) to[i] = s;
}

constexpr int64_t kMostZeros = (int64_t)1 << 30;

void launch_join(hipStream_t st, int32_t runs, int64_t nw, int64_t nb, const float *parts, const float *db_parts, float *dW, float *db) {
  const int64_t n = nw + nb;
  auto go = [&](auto kernel, int entries) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((n + entries - 1) / entries)), dim3(256), 0, st, runs, nw, nb, parts, db_parts, dW, db);
  };
  if (runs <= 4 || n >= 256 * 1024) go(join_kernel<1>, 256);
  else if (n >= 32 * 1024) go(join_kernel<4>, 64);
  else go(join_kernel<16>, 16);
}

// Tiles of dW (inputs x outputs) and runs of rows: two workgroups for each compute unit, none with fewer than 128 rows.  Tiles
// of 256 x 128 do the most products for each row they form; where rows are few, or inputs, tiles of 128 x 128 (1024 x 512 x 512
// 17.5 -> 11.5 us, 92311 x 64 x 64 28.5 -> 14 us).
struct Plan {
  int32_t tile_k, tile_n, tiles_k, tiles_n, runs;
  int64_t rows;
};
constexpr int kTileNarrow = 32, kRunRows = 128, kWorkgroups = 512;
int64_t tile_plan(Plan &p, int32_t P, int32_t in_dim, int32_t out_dim, int32_t tile_k) {  // how many tiles that makes
  p.tile_k = tile_k, p.tile_n = out_dim <= kTileNarrow ? kTileNarrow : 128;
  p.tiles_k = (in_dim + p.tile_k - 1) / p.tile_k, p.tiles_n = (out_dim + p.tile_n - 1) / p.tile_n;
  return (int64_t)p.tiles_k * p.tiles_n * P;
}
int64_t runs_wanted(int64_t tiles, int64_t most) { return std::max<int64_t>(1, std::min(kWorkgroups / tiles, most)); }
Plan plan_of(int32_t P, int64_t rows, int32_t in_dim, int32_t out_dim) {
  Plan p = {};
  int64_t tiles = tile_plan(p, P, in_dim, out_dim, 256);
  if (rows == 0) return p;
  const int64_t most = (rows + kRunRows - 1) / kRunRows;
  if (p.tile_n == 128 && (in_dim <= 128 || tiles * most < kWorkgroups)) tiles = tile_plan(p, P, in_dim, out_dim, 128);
  const int64_t want = runs_wanted(tiles, most);
  p.rows = ((rows + want - 1) / want + kStage - 1) / kStage * kStage;
  p.runs = (int32_t)((rows + p.rows - 1) / p.rows);
  return p;
}
// At least the runs of any number of rows up to `rows` (more rows have fewer runs where they take the larger tiles).
int64_t most_runs(int32_t P, int64_t rows, int32_t in_dim, int32_t out_dim) {
  if (rows == 0) return 0;
  Plan p = {};
  const int64_t most = (rows + kRunRows - 1) / kRunRows, large = tile_plan(p, P, in_dim, out_dim, 256);
  if (p.tile_n != 128) return runs_wanted(large, most);
  const int64_t small = tile_plan(p, P, in_dim, out_dim, 128);
  if (in_dim <= 128) return runs_wanted(small, most);
  const int64_t in_small_tiles = std::min((kWorkgroups - 1) / large, most);  // parts of rows that small tiles are taken for
  return std::max(runs_wanted(small, in_small_tiles), in_small_tiles < most ? runs_wanted(large, most) : 1);
}
size_t scratch_of(int64_t runs, int32_t P, int32_t in_dim, int32_t out_dim) {
  return runs > 1 ? (size_t)runs * P * ((size_t)in_dim * out_dim + out_dim) * 4 : 0;
}

template <class T>
void launch_weight_grads(hipStream_t st, const WeightGrads &d, const Plan &p) {
  const dim3 grid((unsigned)((d.runs + 7) / 8 * 8 * d.tiles), 1, d.P);
  auto go = [&](auto act, auto whole) {
    constexpr bool kAct = decltype(act)::value, kWhole = decltype(whole)::value;
    if (p.tile_n == kTileNarrow)
      hipLaunchKernelGGL((weight_grads_kernel<T, kAct, kWhole, 2, 1, 4, 1>), grid, dim3(256), 0, st, d);
    else if (p.tile_k == 128)
      hipLaunchKernelGGL((weight_grads_kernel<T, kAct, kWhole, 2, 2, 2, 2>), grid, dim3(256), 0, st, d);
    else
      hipLaunchKernelGGL((weight_grads_kernel<T, kAct, kWhole, 4, 2, 2, 2>), grid, dim3(256), 0, st, d);
  };
  auto with = [&](auto act) {
    if (d.a.ins % p.tile_n == 0) go(act, std::true_type());
    else go(act, std::false_type());
  };
  if (d.a.out) with(std::true_type());
  else with(std::false_type());
}

}  // namespace
}  // namespace b8

using namespace b8;

// (a single run's sums are the results themselves)
size_t block8_grads_scratch(int32_t P, int64_t rows, int32_t in_dim, int32_t out_dim) {
  return scratch_of(plan_of(P, rows, in_dim, out_dim).runs, P, in_dim, out_dim);
}
size_t block8_grads_most_scratch(int32_t P, int64_t rows, int32_t in_dim, int32_t out_dim) {
  return scratch_of(most_runs(P, rows, in_dim, out_dim), P, in_dim, out_dim);
}

hipError_t launch_block8_grads(hipStream_t st, const Block8Grads &l) {
  if (l.dx && l.rows > 0) {
    const hipError_t e = launch_block8_input_grads(st, l);
    if (e != hipSuccess) return e;
  }
  const WeightPlan w = weight_plan(l.in_dim, l.out_dim);
  const Plan plan = plan_of(l.P, l.rows, l.in_dim, l.out_dim);
  const int64_t nw = (int64_t)l.P * l.in_dim * l.out_dim, nb = (int64_t)l.P * l.out_dim;
  const bool one = plan.runs == 1;  // its sums are the results
  float *parts = one ? l.dW : l.parts, *db_parts = one ? l.db : l.parts + plan.runs * nw;
  if (plan.runs > 0) {
    WeightGrads d = {};
    d.a.rows = l.rows, d.a.ins = l.out_dim, d.a.outs = l.in_dim, d.a.nib = w.nob, d.a.nob = w.nib;
    d.a.x = l.dy, d.a.ldx = l.lddy, d.a.out = l.y, d.a.out_scale = l.y_scale;
    d.x = l.x, d.x_scale = l.x_scale, d.tiles_k = plan.tiles_k, d.tiles = plan.tiles_k * plan.tiles_n, d.runs = plan.runs, d.run = plan.rows;
    d.parts = parts, d.db_parts = db_parts, d.P = l.P;
    if (l.dy_kind == PR_B8_F32) launch_weight_grads<float>(st, d, plan);
    else launch_weight_grads<uint16_t>(st, d, plan);
  }
  if (plan.runs > 1) launch_join(st, plan.runs, nw, nb, l.parts, db_parts, l.dW, l.db);
  if (plan.runs == 0) {  // zeros: sums of no runs, 2^30 entries a launch (which has fewer than 2^32 threads; runs keep dW below 2^24)
    for (int64_t at = 0; at < nw; at += kMostZeros)
      launch_join(st, 0, std::min(nw - at, kMostZeros), at == 0 ? nb : 0, nullptr, nullptr, l.dW + at, l.db);
  }
  return hipGetLastError();
}

}  // namespace pod
