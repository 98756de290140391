// Products of a few rows with a matrix held in 4 bits (include/msi.h,
// msi_q4_*): y[r][o] = sum_c x[r][c] scale[o][c / G] (code[o][c] - 8) (+ add[r][o]).
//
// Arithmetic.  code - 8 and x are bf16 numbers as they stand, so the matrix
// instruction multiplies them exactly; a group's G products are added in fp32,
// the sum is multiplied by the group's scale (fp16, exact in fp32) and added to
// the row's total, also fp32.  Nothing is rounded to fewer bits before the
// output.  The order of the sums is fixed by the shape, the number of rows among it,
// and by the number of SMs (how many warps share a tile's columns).
//
// Floor: the codes and scales, read once (n_out n_in (1/2 + 2/G) bytes), for 2,048
// weights (a step) 181 to 198 cycles of a quarter of an SM's share of memory (6,790
// GB/s, 1.92 GHz).  Beside it, up to 8 rows, 175 instructions, of them 92 on the integer
// pipe at 2 cycles: 56 shifts and logic operations that make operands of the codes, the
// rest addresses.  Neither is busy throughout: 4 rows, 2,048 to 100,003 take 25 us, 4.3
// TB/s, 290 cycles a step, the integer pipe busy for 58 % of them; the rest is waiting.
// 16 rows, 8,192 to 32,768: 43.3 us, 3.3 TB/s, 386 cycles a step, no pipe busy for more
// than half; what they wait for the counters do not show.  Small matrices 3.3 us, a
// launch and two dependent loads.  (mma.sync rather than tcgen05: the operands are made
// in registers and the rows are few; as bf16 in shared memory the weights would go
// through it at four times their size.)
//
// More than 32 rows go through in groups of 32, each of which reads and unpacks all
// weights again, and mma.sync is no more than 0.3 of the tensor cores' rate: 4,096 to
// 2,048 with 64, 512, 4,096 rows 13, 80, 593 us (80, 108, 116 TFLOP/s), 8,192 to 32,768
// with 512 1.32 ms (208 TFLOP/s).
#include "kernels.cuh"

#include <cuda_fp16.h>

namespace msi {
namespace {

// Packed form: tiles of 16 outputs, cut into turns of two steps of 128 columns; the
// turns of all tiles for the same columns follow one another, then those of the next
// columns (tiles go through the columns side by side, and what all of them read
// together is one stretch of memory).  A step holds 1,024 bytes of codes as the
// lanes of one warp take them, two 16-byte vectors a lane, then the step's scales,
// 128 / G of each output.
//   codes: vector v of lane (g = lane / 4, t = lane % 4): the words of columns
//     64 v + 8 t .. + 7 of outputs g and g + 8, then those 32 columns further on;
//   word: column 2 i of the eight in bits 4 i .., column 2 i + 1 in bits 16 + 4 i ..;
//   scales: for each g, for each group: outputs g and g + 8.
// Columns past n_in and outputs past n_out have the code 8 and the scale 0.
constexpr int kQ4Rows = 16, kQ4Step = 128, kQ4StepCodes = 1024;
constexpr int q4_step_bytes(int group) { return kQ4StepCodes + kQ4Rows * 2 * (kQ4Step / group); }

struct Q4Args {
  const uint8_t* packed;
  int n_in, n_out, turns, tiles;
  int rows;
  const __nv_bfloat16* x;
  long long x_stride;
  const __nv_bfloat16* add;
  long long add_stride;
  void* out;
  long long out_stride;
  int out_f32;
  int stall;             // what CTA (0, 0) waits for in vain (msi_q4_inject_stall), 0: nothing
  long long wait_limit;  // cycles
};

constexpr int kQ4Warps = 8;  // most warps of a CTA

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// Codes of columns 2 i, 2 i + 1 less 8, as bf16, the well-known way: a code as the last
// bits of a number whose unit they are (under the high byte 0x43 it is 128 + q), less
// what was added.
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, int i) {
  uint32_t v, r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(w >> (4 * i)), "r"(0x000f000fu), "r"(0x43004300u));  // (a & b) | c
  // v - 136, exact
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(0x3f803f80u), "r"(0xc308c308u));
  return r;
}

constexpr long long kQ4WaitCycles = 4000000000LL;  // ~2 s

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// The products of one step: a tile of 16 outputs, as the rows of the matrix
// instruction, times NT tiles of 8 rows of x, as its columns.  LIVE: all four
// times 32 columns are there; else the first `live` of them.  x(j, n): the vector
// of 8 columns, of the j-th 32, that the lane has of tile n.
template <int NT, int GN, bool LIVE, class X>
__device__ __forceinline__ void q4_step(float (&total)[NT][4], const uint8_t* at, X x, int live, int lane) {
  float sum[NT][4];
  uint4 c;
  uint32_t sc[GN];
  const uint8_t* p = at + kQ4StepCodes + (lane >> 2) * (GN * 4);
  if constexpr (GN == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    sc[0] = v.x, sc[1] = v.y, sc[2] = v.z, sc[3] = v.w;
  } else if constexpr (GN == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    sc[0] = v.x, sc[1] = v.y;
  } else {
    sc[0] = *reinterpret_cast<const uint32_t*>(p);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (!LIVE && j >= live) break;  // a group's columns are live together
    uint4 v[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) v[n] = x(j, n);
    if (j % 2 == 0) c = *reinterpret_cast<const uint4*>(at + (j / 2) * 512 + lane * 16);
    const uint32_t lo = (j & 1) ? c.z : c.x, hi = (j & 1) ? c.w : c.y;
    const uint32_t a0[4] = {q4_pair(lo, 0), q4_pair(hi, 0), q4_pair(lo, 1), q4_pair(hi, 1)};
    const uint32_t a1[4] = {q4_pair(lo, 2), q4_pair(hi, 2), q4_pair(lo, 3), q4_pair(hi, 3)};
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (j % (4 / GN) == 0) mma_bf16(sum[n], a0, v[n].x, v[n].y, zero);
      else mma_bf16(sum[n], a0, v[n].x, v[n].y, sum[n]);
      mma_bf16(sum[n], a1, v[n].z, v[n].w, sum[n]);
    }
    if (j % (4 / GN) == 4 / GN - 1) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&sc[j / (4 / GN)]));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        total[n][0] = fmaf(sum[n][0], f.x, total[n][0]);
        total[n][1] = fmaf(sum[n][1], f.x, total[n][1]);
        total[n][2] = fmaf(sum[n][2], f.y, total[n][2]);
        total[n][3] = fmaf(sum[n][3], f.y, total[n][3]);
      }
    }
  }
}

__device__ __forceinline__ void q4_store(const Q4Args& a, int row, int to, float v) {
  if (to >= a.n_out) return;
  if (a.add != nullptr) v += __bfloat162float(a.add[(size_t)row * a.add_stride + to]);
  if (a.out_f32)
    static_cast<float*>(a.out)[(size_t)row * a.out_stride + to] = v;
  else
    static_cast<__nv_bfloat16*>(a.out)[(size_t)row * a.out_stride + to] = __float2bfloat16(v);
}

// A CTA takes a tile of 16 outputs; its warps share the columns of the matrix
// and add their totals up in shared memory.  The packed steps come through a ring
// of each warp's own in shared memory, by bulk copies: these pass L1 by, where
// loads return in order, so that the rows of x, which the SM's CTAs share there,
// are not held up by the steps that are on their way (by cp.async 16 x 8,192 to
// 32,768 takes 62 us or more).  GN: groups of a step.
//
// A copy that does not arrive within the wait's limit makes the CTA's outputs NaN.
// (An injected stall: the first CTA's first warp, at its second turn if it has one.)
template <int NT, int GN, int STAGES>
__global__ void __launch_bounds__(256, NT == 1 ? 3 : NT == 2 ? 2 : 1) q4_linear_kernel(const __grid_constant__ Q4Args a) {
  constexpr int kCols = NT * 8, kPitch = kQ4Rows + 1;
  constexpr int kBytes = kQ4StepCodes + kQ4Rows * 2 * GN, kTurn = 2 * kBytes;
  extern __shared__ __align__(128) uint8_t s_ring[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const int tile = blockIdx.x, row0 = blockIdx.y * kCols;
  uint8_t* ring = s_ring + warp * (STAGES * kTurn);

  float total[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) total[n][i] = 0.0f;

  const int t0 = (int)((long long)a.turns * warp / warps), turns = (int)((long long)a.turns * (warp + 1) / warps) - t0;
  const size_t pitch = (size_t)a.tiles * kTurn;  // of a turn
  const uint8_t* w = a.packed + t0 * pitch + (size_t)tile * kTurn;
  const __nv_bfloat16* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)  // past the last row: the last one again, not stored
    x[n] = a.x + (size_t)min(row0 + n * 8 + g, a.rows - 1) * a.x_stride + 8 * t;
  uint64_t* full = reinterpret_cast<uint64_t*>(s_ring + warps * (STAGES * kTurn)) + warp * STAGES;
  if (lane == 0) {
    const int stall = a.stall != 0 && tile + row0 + warp == 0 ? min(turns, STAGES) - 1 : -1;
    for (int d = 0; d < STAGES; ++d) mbar_init(full + d, d == stall ? 2 : 1);
    mbar_fence_init();
  }
  __syncwarp();
  int fetched = 0;
  const auto fetch = [&](int slot) {  // the next turn
    if (lane == 0 && fetched < turns) {
      mbar_arrive_expect_tx(full + slot, kTurn);
      bulk_load(ring + slot * kTurn, w, kTurn, full + slot);
      w += pitch;
    }
    ++fetched;
  };
#pragma unroll
  for (int d = 0; d < STAGES - 1; ++d) fetch(d);
  // rows of x a step ahead: their latency passes beside a step's products
  const int last = a.n_in - 32;
  const auto load_x = [&](uint4 (&b)[4][NT], int step) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = min(step * kQ4Step + 32 * j, last);  // past the end: not used
#pragma unroll
      for (int n = 0; n < NT; ++n) b[j][n] = __ldg(reinterpret_cast<const uint4*>(x[n] + col));
    }
  };
  uint4 b0[4][NT], b1[4][NT];
  load_x(b0, 2 * t0);
  int slot = 0, phase = 0, late = 0;
  for (int i = 0; i < turns; ++i) {
    if (!mbar_wait_warp(full + slot, phase, &late, a.wait_limit)) break;
    fetch(slot == 0 ? STAGES - 1 : slot - 1);  // what was read before the wait, by all lanes
    const uint8_t* at = ring + slot * kTurn;
    const int step = 2 * (t0 + i), live = (a.n_in - step * kQ4Step) >> 5;  // the same for the warp
    load_x(b1, step + 1);
    const auto x0 = [&](int j, int n) { return b0[j][n]; };
    const auto x1 = [&](int j, int n) { return b1[j][n]; };
    if (live >= 8) {
      q4_step<NT, GN, true>(total, at, x0, 4, lane);
      load_x(b0, step + 2);
      q4_step<NT, GN, true>(total, at + kBytes, x1, 4, lane);
    } else {
      q4_step<NT, GN, false>(total, at, x0, live, lane);
      q4_step<NT, GN, false>(total, at + kBytes, x1, live - 4, lane);
    }
    if (++slot == STAGES) slot = 0, phase ^= 1;
  }
  late = __any_sync(0xffffffffu, late);
  if (late) {  // copies in flight still land in the ring
    for (int d = 0; d < STAGES; ++d) {
      int again = 0;
      mbar_wait_warp(full + slot, phase, &again, kDrainCycles);
      if (++slot == STAGES) slot = 0, phase ^= 1;
    }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) total[n][i] = __int_as_float(0x7fc00000);
  }
  __syncthreads();  // the rings are free: the warps' totals go there
  float(*s_sum)[kCols][kPitch] = reinterpret_cast<float(*)[kCols][kPitch]>(s_ring);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float(*o)[kPitch] = &s_sum[warp][n * 8 + 2 * t];
      o[0][g] = total[n][0];
      o[1][g] = total[n][1];
      o[0][g + 8] = total[n][2];
      o[1][g + 8] = total[n][3];
    }
  __syncthreads();
  const int cols = min(kCols, a.rows - row0);
  for (int e = threadIdx.x; e < kQ4Rows * cols; e += blockDim.x) {
    const int r = e / kQ4Rows, o = e % kQ4Rows;
    float v = 0.0f;
    for (int p = 0; p < warps; ++p) v += s_sum[p][r][o];
    q4_store(a, row0 + r, tile * kQ4Rows + o, v);
  }
}

// The same for matrices with tiles enough: the warps of a CTA that have the same
// columns (a part; there are `KS` of them) go through these side by side, so that
// a turn's rows of x are brought to shared memory once for all of them, by the
// part's first warp; a tile a warp.  (Through L1, as above, 16 rows are 16 cache
// lines a load: its tags, not memory, bound them: 16 x 8,192 to 32,768 54 us.  Two
// tiles a warp, which have a row of x in registers for both but half the warps: 47.)
//
// A warp whose wait runs out frees no more slots, so that the part's first warp and then
// all others of the part run out as well, each once, unless they have all they need: the
// tiles of those that did are NaN.  (An injected stall: the first CTA's first part, its
// last warp at the first turn's codes, or all its warps at the second turn's rows.)
constexpr int kQ4XPitch = 576;  // bytes of a row of x in a slot: 512, and 64 so that eight rows' parts lie in other banks
constexpr int kQ4Parts = 2, kQ4Slots = 2;
// Most tiles of a CTA, and CTAs of an SM: with 32 rows the rings leave room for one.
constexpr int q4_same(int nt) { return nt <= 2 ? 7 : 14; }
constexpr int q4_ctas(int nt) { return nt <= 2 ? 2 : 1; }

template <int NT, int GN>
__global__ void __launch_bounds__(kQ4Parts * q4_same(NT) * 32, q4_ctas(NT)) q4_wide_kernel(const __grid_constant__ Q4Args a) {
  constexpr int KS = kQ4Parts, SLOTS = kQ4Slots, kCols = NT * 8, kPitch = kQ4Rows + 1;
  constexpr int kBytes = kQ4StepCodes + kQ4Rows * 2 * GN, kTurn = 2 * kBytes, kX = kCols * kQ4XPitch;
  extern __shared__ __align__(128) uint8_t s_ring[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, same = warps / KS;
  const int part = warp / same, own = warp - part * same;
  const int g = lane >> 2, t = lane & 3;
  const int tile = blockIdx.x * same + own, row0 = blockIdx.y * kCols;
  const int rows = min(kCols, a.rows - row0);
  const int t0 = a.turns * part / KS, turns = a.turns * (part + 1) / KS - t0;
  uint8_t* ring = s_ring + warp * (SLOTS * kTurn);
  uint8_t* s_x = s_ring + warps * SLOTS * kTurn + part * SLOTS * kX;
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_ring + warps * SLOTS * kTurn + KS * SLOTS * kX);
  uint64_t *full = bars + warp * SLOTS, *x_full = bars + (warps + part) * SLOTS, *x_free = bars + (warps + KS + part) * SLOTS;

  float total[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) total[n][i] = 0.0f;
  if (lane < SLOTS) {
    const int stall = blockIdx.x + blockIdx.y + part == 0 ? a.stall : 0;
    mbar_init(full + lane, stall == MSI_Q4_STALL_CODES && own + 1 == same && lane == 0 ? 2 : 1);
    if (own == 0) {
      mbar_init(x_full + lane, stall == MSI_Q4_STALL_ROWS && lane == min(turns, SLOTS) - 1 ? 2 : 1);
      mbar_init(x_free + lane, same);
    }
    mbar_fence_init();
  }
  __syncthreads();
  const size_t pitch = (size_t)a.tiles * kTurn;  // of a turn
  const uint8_t* w = a.packed + t0 * pitch + (size_t)min(tile, a.tiles - 1) * kTurn;  // past the last tile: the last one again, not stored
  const __nv_bfloat16* x = a.x + (size_t)(row0 + min(lane, rows - 1)) * a.x_stride;
  const auto fetch = [&](int turn, int slot) {
    if (own == 0) {
      const int col0 = (t0 + turn) * 2 * kQ4Step;
      const uint32_t bytes = (uint32_t)min(2 * kQ4Step, a.n_in - col0) * 2;
      if (lane == 0) mbar_arrive_expect_tx(x_full + slot, rows * bytes);
      __syncwarp();
      if (lane < rows) bulk_load(s_x + slot * kX + lane * kQ4XPitch, x + col0, bytes, x_full + slot);
    }
    if (lane == 0) {
      mbar_arrive_expect_tx(full + slot, kTurn);
      bulk_load(ring + slot * kTurn, w, kTurn, full + slot);
      w += pitch;
    }
  };
#pragma unroll
  for (int d = 0; d < SLOTS; ++d)
    if (d < turns) fetch(d, d);
  int slot = 0, phase = 0, late = 0;
  for (int i = 0; i < turns; ++i) {
    if (!mbar_wait_warp(x_full + slot, phase, &late, a.wait_limit) || !mbar_wait_warp(full + slot, phase, &late, a.wait_limit)) break;
    const uint8_t* at = ring + slot * kTurn;
    const uint8_t* xs = s_x + slot * kX + g * kQ4XPitch + t * 16;
    const int live = (a.n_in - (t0 + i) * 2 * kQ4Step) >> 5;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto b = [&](int j, int n) { return *reinterpret_cast<const uint4*>(xs + n * 8 * kQ4XPitch + (4 * h + j) * 64); };
      if (live >= 8) q4_step<NT, GN, true>(total, at + h * kBytes, b, 4, lane);
      else q4_step<NT, GN, false>(total, at + h * kBytes, b, live - 4 * h, lane);
    }
    __syncwarp();  // the slots are read by all lanes
    if (lane == 0) mbar_arrive(x_free + slot);
    if (i + SLOTS < turns) {
      if (own == 0 && !mbar_wait_warp(x_free + slot, phase, &late, a.wait_limit)) break;
      fetch(i + SLOTS, slot);
    }
    if (++slot == SLOTS) slot = 0, phase ^= 1;
  }
  if (__any_sync(0xffffffffu, late)) {  // copies in flight still land in the rings
    for (int d = 0; d < SLOTS; ++d) {
      int again = 0;
      mbar_wait_warp(x_full + slot, phase, &again, kDrainCycles);
      again = 0;
      mbar_wait_warp(full + slot, phase, &again, kDrainCycles);
      if (++slot == SLOTS) slot = 0, phase ^= 1;
    }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) total[n][i] = __int_as_float(0x7fc00000);
  }
  __syncthreads();  // the rings are free: the totals go there, for stores of neighbours
  float(*s_sum)[kCols][kPitch] = reinterpret_cast<float(*)[kCols][kPitch]>(s_ring);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float(*o)[kPitch] = &s_sum[warp][n * 8 + 2 * t];
      o[0][g] = total[n][0];
      o[1][g] = total[n][1];
      o[0][g + 8] = total[n][2];
      o[1][g + 8] = total[n][3];
    }
  __syncthreads();
  const int all = same * kQ4Rows;
  for (int e = threadIdx.x; e < all * rows; e += blockDim.x) {
    const int r = e / all, o = e - r * all;
    float v = 0.0f;
#pragma unroll
    for (int p = 0; p < KS; ++p) v += s_sum[p * same + o / kQ4Rows][r][o % kQ4Rows];
    q4_store(a, row0 + r, blockIdx.x * all + o, v);
  }
}

// One word of eight codes (or one of two scales) a thread.
__global__ void q4_pack_kernel(const uint8_t* codes, const __half* scales, int n_out, int n_in, int group, int tiles,
                               long long words, uint32_t* out) {
  const int gn = kQ4Step / group, step_words = q4_step_bytes(group) / 4;
  for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < words; e += (long long)gridDim.x * blockDim.x) {
    const long long at = e / step_words;
    const int i = (int)(e - at * step_words), step = (int)(at / (2 * tiles) * 2 + (at & 1));
    const long long o0 = at / 2 % tiles * kQ4Rows;
    uint32_t v;
    if (i < kQ4StepCodes / 4) {
      const int lane = (i >> 2) & 31, j = i & 3;
      const long long o = o0 + (lane >> 2) + 8 * (j & 1);
      const int c = step * kQ4Step + 64 * (i >> 7) + 32 * (j >> 1) + 8 * (lane & 3);
      v = 0x88888888u;
      if (o < n_out && c < n_in) {
        const uint32_t u = *reinterpret_cast<const uint32_t*>(codes + (size_t)o * (n_in / 2) + c / 2);
        v = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) v |= ((u >> (4 * k)) & 15u) << (4 * ((k >> 1) + 4 * (k & 1)));
      }
    } else {
      const int k = i - kQ4StepCodes / 4;  // [g][group] pairs
      const int c = step * kQ4Step + k % gn * group;
      v = 0;
      for (int half = 0; half < 2; ++half) {
        const long long o = o0 + k / gn + 8 * half;
        if (o < n_out && c < n_in) v |= (uint32_t)__half_as_ushort(scales[(size_t)o * (n_in / group) + c / group]) << (16 * half);
      }
    }
    out[e] = v;
  }
}

template <int NT, int GN, int STAGES>
cudaError_t q4_launch(const Q4Args& a, dim3 grid, int warps, cudaStream_t s) {
  constexpr int kRing = STAGES * (2 * (kQ4StepCodes + kQ4Rows * 2 * GN) + 8);
  constexpr int kSums = NT * 8 * (kQ4Rows + 1) * 4, kSmem = kRing > kSums ? kRing : kSums;  // of a warp
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = smem_attr_once(q4_linear_kernel<NT, GN, STAGES>, kQ4Warps * kSmem, done);
  if (e != cudaSuccess) return e;
  q4_linear_kernel<NT, GN, STAGES><<<grid, warps * 32, warps * kSmem, s>>>(a);
  return cudaGetLastError();
}

template <int NT, int GN>
cudaError_t q4_launch_wide(const Q4Args& a, int sms, cudaStream_t s) {
  constexpr int kRing = kQ4Slots * (2 * (kQ4StepCodes + kQ4Rows * 2 * GN) + 8);  // of a warp
  constexpr int kX = kQ4Parts * kQ4Slots * (NT * 8 * kQ4XPitch + 16);
  static_assert(kRing > NT * 8 * (kQ4Rows + 1) * 4, "the totals fit in the rings");
  const auto smem = [](int warps) { return warps * kRing + kX; };
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = smem_attr_once(q4_wide_kernel<NT, GN>, smem(kQ4Parts * q4_same(NT)), done);
  if (e != cudaSuccess) return e;
  // CTAs of as few tiles as make no more waves, so that all SMs have work alike: 16 x
  // 4,096 to 24,000 by CTAs of 5 tiles 20 us, of 8 27
  const int wave = sms * q4_ctas(NT), waves = (a.tiles + wave * q4_same(NT) - 1) / (wave * q4_same(NT));
  const int same = (a.tiles + wave * waves - 1) / (wave * waves), warps = kQ4Parts * same;
  const dim3 grid((a.tiles + same - 1) / same, (a.rows + NT * 8 - 1) / (NT * 8));
  q4_wide_kernel<NT, GN><<<grid, warps * 32, smem(warps), s>>>(a);
  return cudaGetLastError();
}

template <int NT, int STAGES>
cudaError_t q4_as(const Q4Args& a, int group, int sms, cudaStream_t s) {
  // Up to 8 rows the loads of x are few, and the tiles by themselves are faster (one
  // row, 8,192 to 32,768: 33 us, with shared rows 35).  From 9 on, by themselves / with
  // shared rows, weights from memory, us:
  //             2,048 columns to 600, 912, 2,048 tiles    8,192 columns
  //   9 rows    8.0/7.4   11.6/9.2   18.9/15.4            18.1/21.1  25.2/24.3  49.7/40.5
  //   17        15.8/11.4 22.7/12.7  34.5/23.6            32.5/38.5  46.6/41.3  87.0/67.2
  //   512       236/125   356/216    547/361              465/419    736/754    1344/1154
  // and with 300 tiles 4.8/6.6 (9 rows, 2,048 columns), 10.4/18.7 (8,192).
  if constexpr (NT > 1) {
    if (a.tiles >= sms * 6) {
      if (group == 32) return q4_launch_wide<NT, 4>(a, sms, s);
      if (group == 64) return q4_launch_wide<NT, 2>(a, sms, s);
      return q4_launch_wide<NT, 1>(a, sms, s);
    }
  }
  // Warps enough to cover the latency of a step's chain: 16,384 to 1,000 by 2, 4, 8
  // warps a tile 19, 13, 8.6 us.  The limit at 12, 24, 48, 96 warps an SM (one row): 2,048
  // to 14,400 6.3, 8.0, 8.0, 8.0; to 40,000 13.6, 13.2, 14.0, 18.1; to 100,003 24.8, 24.9,
  // 25.3, 28.8; 8,192 to 32,768 41.3, 38.9, 33.0, 35.0 (8 rows 52, 49, 38.5, 37.9).  Groups
  // of rows beyond the first do not count.
  int warps = 1;
  while (warps < kQ4Warps && warps < a.turns && (long long)a.tiles * warps < (long long)sms * 48) warps *= 2;
  const dim3 grid(a.tiles, (a.rows + NT * 8 - 1) / (NT * 8));
  if (group == 32) return q4_launch<NT, 4, STAGES>(a, grid, warps, s);
  if (group == 64) return q4_launch<NT, 2, STAGES>(a, grid, warps, s);
  return q4_launch<NT, 1, STAGES>(a, grid, warps, s);
}

msi_status q4_shape(int n_out, int n_in, int group) {
  if (n_out < 1 || n_in < 1) return MSI_ERR_INVALID_ARG;
  if ((group != 32 && group != 64 && group != 128) || n_in % group != 0 || n_in > 1 << 20 || n_out > 1 << 24)
    return MSI_ERR_UNSUPPORTED;
  return MSI_OK;
}

std::atomic<long long> q4_wait_limit{kQ4WaitCycles};
std::atomic<int> q4_stall{0};

bool aligned(const void* p, unsigned bytes) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace
}  // namespace msi

using namespace msi;

extern "C" {

uint64_t msi_q4_packed_bytes(int n_out, int n_in, int group) {
  if (q4_shape(n_out, n_in, group) != MSI_OK) return 0;
  return (uint64_t)((n_out + kQ4Rows - 1) / kQ4Rows) * ((n_in + 2 * kQ4Step - 1) / (2 * kQ4Step)) * 2 * q4_step_bytes(group);
}

msi_status msi_q4_pack(const void* codes, const void* scales, int n_out, int n_in, int group, void* packed,
                       uint64_t packed_bytes, msi_stream stream) {
  const msi_status st = q4_shape(n_out, n_in, group);
  if (st != MSI_OK) return st;
  if (!aligned(codes, 4) || !aligned(scales, 2) || !aligned(packed, 16)) return MSI_ERR_INVALID_ARG;
  const uint64_t need = msi_q4_packed_bytes(n_out, n_in, group);
  if (packed_bytes < need) return MSI_ERR_WORKSPACE;
  const long long words = (long long)(need / 4), ctas = (words + 255) / 256;
  q4_pack_kernel<<<(unsigned)(ctas < 65536 ? ctas : 65536), 256, 0, stream>>>(
      static_cast<const uint8_t*>(codes), static_cast<const __half*>(scales), n_out, n_in, group,
      (n_out + kQ4Rows - 1) / kQ4Rows, words, static_cast<uint32_t*>(packed));
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? MSI_OK : note_cuda_error(e, "msi_q4_pack");
}

msi_status msi_q4_linear(const msi_q4_linear_args* g, msi_stream stream) {
  if (g == nullptr) return MSI_ERR_INVALID_ARG;
  const msi_status st = q4_shape(g->n_out, g->n_in, g->group);
  if (st != MSI_OK) return st;
  if (g->rows < 0 || (g->out_type != MSI_BF16 && g->out_type != MSI_F32)) return MSI_ERR_INVALID_ARG;
  if (g->rows > 1 << 20) return MSI_ERR_UNSUPPORTED;
  if (g->rows == 0) return MSI_OK;
  if (!aligned(g->packed, 16) || !aligned(g->x, 16) || g->x_stride < 0 || g->x_stride % 8 != 0 ||
      !aligned(g->out, g->out_type == MSI_F32 ? 4 : 2) || g->out_stride < g->n_out ||
      (g->add != nullptr && (!aligned(g->add, 2) || g->add_stride < 0)))
    return MSI_ERR_INVALID_ARG;
  Q4Args a = {};
  a.packed = static_cast<const uint8_t*>(g->packed);
  a.n_in = g->n_in;
  a.n_out = g->n_out;
  a.turns = (g->n_in + 2 * kQ4Step - 1) / (2 * kQ4Step);
  a.tiles = (g->n_out + kQ4Rows - 1) / kQ4Rows;
  a.rows = g->rows;
  a.x = static_cast<const __nv_bfloat16*>(g->x);
  a.x_stride = g->x_stride;
  a.add = static_cast<const __nv_bfloat16*>(g->add);
  a.add_stride = g->add_stride;
  a.out = g->out;
  a.out_stride = g->out_stride;
  a.out_f32 = g->out_type == MSI_F32;
  a.wait_limit = q4_wait_limit.load(std::memory_order_relaxed);
  if (q4_stall.load(std::memory_order_relaxed) != 0) a.stall = q4_stall.exchange(0);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) {
    if (a.rows <= 8) e = q4_as<1, 2>(a, g->group, sms, stream);
    else if (a.rows <= 16) e = q4_as<2, 2>(a, g->group, sms, stream);
    else e = q4_as<4, 2>(a, g->group, sms, stream);
  }
  return e == cudaSuccess ? MSI_OK : note_cuda_error(e, "msi_q4_linear");
}

msi_status msi_q4_set_wait_cycles(int64_t cycles) {
  q4_wait_limit = cycles > 0 ? (long long)cycles : kQ4WaitCycles;
  return MSI_OK;
}

msi_status msi_q4_inject_stall(int where) {
  if (where < 0 || where > MSI_Q4_STALL_ROWS) return MSI_ERR_INVALID_ARG;
  q4_stall = where;
  return MSI_OK;
}

}  // extern "C"
