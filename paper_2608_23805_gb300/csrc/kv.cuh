// Key-value cache in 8 bits (include/msi.h, msi_kv_*): what its kernels share.
#pragma once

#include <cuda_fp16.h>

#include "kernels.cuh"

namespace msi {

constexpr int kKvMaxSeqs = 1024;
constexpr int kKvMaxHeads = 64;
constexpr long long kKvWaitCycles = 4000000000LL;  // default limit of a device wait
constexpr int kKvStallSoftmax = MSI_KV_STALL_SOFTMAX, kKvStallMma = MSI_KV_STALL_MMA, kKvStallConversion = MSI_KV_STALL_CONVERSION;
constexpr float kKvTiny = 1e-20f;  // least absolute maximum of a block: its scale stays a normal number

// The cache as the kernels see it (msi_kv_desc).
struct KvCache {
  int n_seqs, max_blocks, n_blocks, K, D, P, logP, fmt;
  uint8_t* codes[2];
  float* scale[2];
  __nv_bfloat16* recent;
  int* table;
  int4* seq;     // {held, position, first position in `recent`, 0}
  int* free_ids;
  int* control;  // [0] free blocks, [1] status, [2] append ticket, [3] evict ticket
  float* weight;
};

struct KvAppendArgs {
  KvCache c;
  int n, n_rows;
  const int* seqs;
  const int* cu;
  const int* start;
  const __nv_bfloat16* x[2];
  long long stride;
  int sms;
};

struct KvEvictArgs {
  KvCache c;
  int n;
  const int* seqs;
  int keep, sinks, recent;
  int release;
};

struct KvReadArgs {
  KvCache c;
  int n, n_rows;
  const int* seqs;
  const int* first;
  const int* cu;
  __nv_bfloat16* out[2];
  int sms;
};

struct KvAttnArgs {
  KvCache c;
  int n, n_rows, max_rows, H, G;
  const int* seqs;
  const int* cu;
  const __nv_bfloat16* q;
  long long q_stride;
  __nv_bfloat16* out;
  long long out_stride;
  float* lse;
  float scale, softcap;
  int window, observe;
  int stall;             // chunk form: the kind of warp that waits in vain (msi_kv_inject_stall), 0: none
  long long wait_limit;  // chunk form: clock64 cycles of a wait
  int ctas;            // CTAs that share the work
  int groups;          // decode form: most groups of rows of a sequence and head
  // workspace
  float* part_o;       // [2 ctas][rows][D] unnormalised outputs of the parts of split items
  float* part_ml;      // [2 ctas][2][rows] their reference exponents and sums
  int4* split;         // decode form: [ctas] the pair that begins in a CTA's run and goes on past it
  float* lse2;         // [n_rows, H] log2 of the sums (observe)
  float* step_lse;     // [steps][rows] log2 of each 16-token step's sum (observe)
  long long max_steps;
  // chunk form: the items (sequence, key-value head, row tile) and the prefix of their token tiles
  int4* items;            // [2 max_items] {sequence, first row, rows, held}, {head, row tile, first token tile, 0}
  long long* item_pre;    // [max_items + 1]; decode form: [n + 1] steps before each sequence's (observe)
  int* plan;              // [4 + ctas] items, whether every sequence is in range, CTAs, whether the call failed; then each CTA's first item
  int max_items;
};

cudaError_t launch_kv_append(const KvAppendArgs& a, cudaStream_t s);
cudaError_t launch_kv_evict(const KvEvictArgs& a, cudaStream_t s);
cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s);
cudaError_t launch_kv_init(const KvCache& c, cudaStream_t s);
// Decode form: rows of one sequence and key-value head (its part of the query
// heads) as columns of the MMA.
int kv_decode_pair_cost();               // units of work that a pair is counted beside its steps
int kv_decode_tiles(int rows, int D);  // n8 tiles (1, 2 or 4) of a group of rows, 0: not in decode form
cudaError_t launch_kv_decode(const KvAttnArgs& a, int* launches, cudaStream_t s);
// Chunk form: rows of one sequence and key-value head in tiles of the MMA's rows.
int kv_chunk_rows(int D);  // rows of an item
cudaError_t launch_kv_chunk(const KvAttnArgs& a, int* launches, cudaStream_t s);

#if defined(__CUDACC__)

__device__ __forceinline__ void kv_raise(const KvCache& c, int status) { atomicCAS(c.control + 1, 0, status); }

__device__ __forceinline__ float kv_nan() { return __int_as_float(0x7fc00000); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// `total` units in `ctas` runs of nearly equal length, the longer ones spread
// evenly (so that equal items, cut by a multiple of their number, are cut alike).
struct KvRuns {
  long long total;
  int ctas;
  // where run i begins
  __device__ __forceinline__ long long begin(int i) const { return total * i / ctas; }
  // the run that holds unit u: the last i with total i < (u + 1) ctas
  __device__ __forceinline__ int owner(long long u) const { return (int)(((u + 1) * ctas - 1) / total); }
};
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ int kv_seq(const int* seqs, int b) { return seqs == nullptr ? b : seqs[b]; }

// One sequence of the call.
struct KvWork {
  int seq, row0, rows, held;
  int step0, steps;  // 16-token steps that some row sees
  bool ok;
};

__device__ __forceinline__ KvWork kv_work(const KvAttnArgs& a, int b) {
  const KvCache& c = a.c;
  KvWork w;
  w.seq = kv_seq(a.seqs, b);
  w.row0 = a.cu[b];
  w.rows = a.cu[b + 1] - w.row0;
  w.ok = w.seq >= 0 && w.seq < c.n_seqs && w.row0 >= 0 && w.rows >= 0 && w.rows <= a.max_rows &&
         w.row0 <= a.n_rows - w.rows;
  w.held = w.ok ? c.seq[w.seq].x : 0;
  w.ok = w.ok && w.held >= 0 && w.held <= c.max_blocks << c.logP;
  w.step0 = w.steps = 0;
  if (!w.ok || w.rows == 0) return w;
  const int lo = a.window > 0 ? max(0, w.held - w.rows - a.window + 1) : 0;
  w.step0 = lo >> 4;
  w.steps = ((w.held + 15) >> 4) - w.step0;
  return w;
}

// Inclusive sums of `v` over the block's threads (a multiple of 32, at most
// 1,024); `warp_sums` holds 32 ints.  Ends with the block in step.
__device__ __forceinline__ int block_scan(int v, int* warp_sums) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 31) warp_sums[w] = v;
  __syncthreads();
  if (w == 0) {
    int s = lane < nw ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += u;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  return v + (w > 0 ? warp_sums[w - 1] : 0);
}

// Two e4m3 numbers (low byte first) as fp16: exact.
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t v) {
  uint32_t r;
  asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(v));
  return r;
}

// Codes to fp16, exactly: byte 0 and 1 (HI: 2 and 3) of z.
//   Q8: byte q under the high byte 0x64 is the fp16 number 1024 + q; less 1152
//   it is q - 128.
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t kv_f16x2(uint32_t z) {
  if (FMT == MSI_KV_Q8) {
    const uint32_t v = __byte_perm(z, 0x64646464u, HI ? 0x4342 : 0x4140);
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&v), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  return e4m3x2_f16x2(HI ? z >> 16 : z);
}

// What a query row is multiplied with to lie in fp16's range: the power of two
// that takes its largest element to [1, 2) (bits of 2^-e; 2^e comes back into
// the score's scale).  bf16 has 8 significant bits, fp16 11 and 14 exponents
// below 1: products with codes stay exact but for elements under 2^-14 of the
// row's largest, which are rounded to 2^-24 of it.  amax: bits of the row's
// largest absolute value.
__device__ __forceinline__ uint32_t kv_row_exp(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;
  return e < 1 ? 1 : e > 253 ? 253 : e;
}

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// of the normal numbers
__device__ __forceinline__ float lg2(float x) {
  float r;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// and of the denormal ones too: sums beside the largest value scales
__device__ __forceinline__ float lg2_any(float x) {
  float r;
  asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// How far value scales may lie apart.  A weight for the sum is taken from the MMA's
// operand, 2^(s + log2 sv - M) / sv, and ex2 gives 0 below 2^-126.  The token that
// set M has the operand 1, so a row's sum is at least 1 / sv of that token: of a
// token whose sv is 2^90 times smaller less than 2^-36 of the sum can be lost.  The
// kernels look at the scales of the blocks that share a reference, and beyond that
// the call fails closed.  (The sum apart from the operand, a second exponential a
// score in its own loop, cost 2 to 10 % of every call.)
constexpr float kScaleRange = 1.2379400392853803e27f;  // 2^90

// l 2^d where 2^d by itself may be out of fp32's range: parts with references of
// their own may have any scales.
__device__ __forceinline__ float kv_scaled(float l, float d) {
  const float h = ex2(0.5f * d);
  return l * h * h;
}

// softcap * tanh(x / softcap) = softcap (1 - 2 / (e^(2 x / softcap) + 1)); the
// quotient's limits are those of the formula.  two_log2e_cap = 2 log2(e) / cap.
// The difference leaves an error of 2^-23 of the cap, whatever the score: up to
// caps of 64 that is no more than the scores' own roundings.  WIDE: any cap, with
// tanh's series (up to z^9) where the score is under a quarter of it.
constexpr float kSmallCap = 64.0f;
template <bool WIDE>
__device__ __forceinline__ float kv_softcap(float x, float cap, float two_log2e_cap) {
  const float y = x * two_log2e_cap;
  const float far = cap * (1.0f - __fdividef(2.0f, ex2(y > 80.0f ? 80.0f : y) + 1.0f));  // a NaN stays one
  if (!WIDE) return far;
  const float z = y * (0.5f * kLn2), z2 = z * z;
  const float near = fmaf(z2, fmaf(z2, fmaf(z2, fmaf(z2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  return fabsf(z) < 0.25f ? x * near : far;
}

#endif  // __CUDACC__

}  // namespace msi
