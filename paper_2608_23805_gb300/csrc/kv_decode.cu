// Attention over the 8-bit key-value cache in decode form: the rows of one
// sequence and key-value head (its query heads times a few tokens, in groups of
// R <= 32) against everything that the sequence holds.
//
// Mathematics.  With codes c and scales sk, sv of a token's block and head, a
// row's score is s = scale * sk * (q . ck), its weight p = 2^(s log2 e - M), and
//   out = sum p sv cv / sum p.
// Codes are exact in fp16; q is brought to fp16's range by a power of two per
// row (kv_row_exp), so the products are exact and the tensor core adds them up
// in fp32.  sk multiplies the fp32 score.  sv goes into the exponent: the MMA's
// operand is P = 2^(s log2 e + log2 sv - M) <= 2^8, rounded once to fp16 (the
// choice that costs precision here: 2^-12 a weight, an eighth of bf16's), and
// the sum takes P / sv in fp32.  M is a running reference, moved only when a P
// would pass 2^8, so most steps rescale nothing.
//
// Layout.  A warp takes 16 tokens a step.  S^T = K Q^T and O^T = V^T P^T have
// the tokens and the head's columns as the MMA's 16 rows and the query rows as
// its 8 columns: with 8 rows no lane of the MMA is idle (queries as rows would
// waste half of one).  The contraction's order is free, so a lane's operands
// are 16 consecutive bytes of a code row, and V^T needs only byte interleaving
// of two tokens' words.  Codes go to a ring of shared memory per warp by
// 16-byte asynchronous copies, chunks XOR-swizzled by row.  The legacy MMA is
// enough at 8 and 16 rows: 2 R flops a byte (110 TFLOP/s at 8 rows and 6.8 TB/s);
// with more, each group of a head converts the codes again.
//
// Split.  The work is the list of all 16-token steps of all (sequence, head)
// pairs; each CTA takes an equal run of it, whatever the lengths.  A pair that
// lies in one CTA is finished there; parts of split ones are joined by
// kv_finish_kernel in the CTAs' order, so results do not depend on timing.
//
// Measured: 64 sequences of up to 8,192, 2 heads of 128 with 8 query heads each,
// block weights added up: 45 us, 3.6 TB/s of codes and scales; one of 32,768: 15 us.
// Bound: the latency of a step's dependent instructions (about 500, half of them
// conversions and byte interleaving) at 16 warps an SM, 8 at D = 256: issue slots
// are 41 and 29 % busy, DRAM 54 and 47 %; without the copies it takes 0.86 of the time.
#include "kv.cuh"

namespace msi {
namespace {

constexpr float kLazy = 8.0f;  // P may reach 2^8

// Warps of a CTA, by the registers that a warp's outputs and queries take
// (D x 8 NT of each): the more the better hidden are a step's latencies (D = 128,
// 8 rows, 64 sequences of 8,192: 45.6 us with 8 warps, 46.9 with 4).  Two
// CTAs share an SM, so that one reads while the other begins or ends a pair.
__host__ __device__ constexpr int dec_warps(int D, int NT) { return D * NT <= 128 ? 8 : 4; }
// What a pair costs a CTA beside its steps (queries, first loads, the warps'
// sums), in steps; us at 16, 32, 48, 64, 96: 64 sequences of up to 8,192, D = 64
// 22.6, 22.0, 21.6, 22.1, 22.9, D = 128 38.8, 38.8, 37.3, 37.3, 37.9, 64 of 4,096 at
// D = 256 39.9, 38.7, 39.1, 40.0, 42.4; 12 of 20,000, 4 tokens, D = 128 39.4, 37.2,
// 37.0, 37.5, 38.5, D = 256 71.2, 68.2, 68.2, 69.9, 71.6; one of 32,768 within 0.5.
constexpr int kPairCost = 48;
__host__ __device__ constexpr int dec_stage_bytes(int D) { return 16 * 2 * D; }
// Stages of a warp's ring: 96 KB a CTA, at most 8.
__host__ __device__ constexpr int dec_stages(int D, int NT) {
  const int s = 96 * 1024 / dec_warps(D, NT) / dec_stage_bytes(D);
  return s > 8 ? 8 : s;
}

// A pair's units of work: its fixed cost, then its steps.
__device__ __forceinline__ int kv_units(const KvWork& w) { return w.steps > 0 ? w.steps + kPairCost : 0; }
// Pairs of a sequence and head: groups of R rows.
__device__ __forceinline__ int kv_groups(const KvAttnArgs& a, const KvWork& w, int R) { return (w.rows * a.G + R - 1) / R; }

// The batch's work: s_pre[b] = units of the pairs before sequence b, over all
// heads.  Returns whether every sequence is in range and, with s_seen (a bit for
// each sequence of the cache), named once: two entries would add to the weights of
// the same blocks.  s_pre holds n + 1 words.
__device__ __forceinline__ bool kv_share(const KvAttnArgs& a, int R, long long* s_pre, long long* s_sum, int* s_bad,
                                         unsigned* s_seen) {
  const int tid = threadIdx.x, T = blockDim.x, lane = tid & 31, wid = tid >> 5;
  const int per = (a.n + T - 1) / T, b0 = min(a.n, tid * per), b1 = min(a.n, b0 + per);
  if (tid == 0) *s_bad = 0;
  if (s_seen != nullptr && tid < kKvMaxSeqs / 32) s_seen[tid] = 0;
  __syncthreads();
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    const KvWork w = kv_work(a, b);
    if (!w.ok || (s_seen != nullptr && (atomicOr(&s_seen[w.seq >> 5], 1u << (w.seq & 31)) >> (w.seq & 31) & 1) != 0))
      *s_bad = 1;
    mine += (long long)kv_units(w) * a.c.K * (w.ok ? kv_groups(a, w, R) : 0);
  }
  long long v = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  if (lane == 31) s_sum[wid] = v;
  __syncthreads();
  long long before = v - mine;
  for (int i = 0; i < wid; ++i) before += s_sum[i];
  for (int b = b0; b < b1; ++b) {
    s_pre[b] = before;
    const KvWork w = kv_work(a, b);
    before += (long long)kv_units(w) * a.c.K * (w.ok ? kv_groups(a, w, R) : 0);
  }
  if (b0 < a.n && b1 == a.n) s_pre[a.n] = before;
  __syncthreads();
  return *s_bad == 0;
}

// CTAs that take part.
__device__ __forceinline__ int kv_ctas(long long total, int ctas, int warps) {
  // a step a warp at least
  return total >= (long long)ctas * warps ? ctas : max(1, ((int)total + warps - 1) / warps);
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Byte offset of 16-byte chunk `ch` of token row r in a stage's [16][D] codes.
template <int D>
__device__ __forceinline__ int dec_chunk(int r, int ch) {
  if (D == 64) return r * 64 + ((ch ^ ((r >> 1) & 3)) << 4);
  return r * D + ((ch ^ (r & 7)) << 4);
}
// The chunk that lane t of a quad reads as its j-th: the contraction's order.
template <int D>
__device__ __forceinline__ int dec_kchunk(int t, int j) {
  return D == 64 ? t : D == 128 ? 2 * t + j : 2 * t + (j & 1) + 8 * (j >> 1);
}

// A lane's view of the steps of a run: block and scales of step base + lane.
struct StepInfo {
  int blk;
  float ks, lv, iv;  // key scale, log2 of the value scale and its inverse
};

template <int D, int NT, int FMT, bool OBS>
__global__ void __launch_bounds__(32 * dec_warps(D, NT), 2) kv_decode_kernel(KvAttnArgs a) {
  constexpr int kDecWarps = dec_warps(D, NT), kDecThreads = 32 * kDecWarps;
  constexpr int KS = D / 16;          // MMAs along a row, and column tiles of the output
  constexpr int CH = D / 64;          // 16-byte chunks of a key row a lane takes
  constexpr int R = 8 * NT;
  constexpr int S = dec_stages(D, NT), SB = dec_stage_bytes(D), RING = S * SB;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long s_sum[kDecWarps];
  __shared__ int s_bad;
  __shared__ unsigned s_seen[OBS ? kKvMaxSeqs / 32 : 1];
  __shared__ float s_m[kDecWarps][R], s_l[kDecWarps][R];
  long long* s_pre = reinterpret_cast<long long*>(smem + kDecWarps * RING);
  const KvCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
  grid_release();

  const int status = c.control[1];
  const bool ok = kv_share(a, R, s_pre, s_sum, &s_bad, OBS ? s_seen : nullptr);
  const long long total = s_pre[a.n];
  if (tid == 0) a.split[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (OBS && blockIdx.x == 0)
    for (int i = tid; i <= a.n; i += kDecThreads) a.item_pre[i] = s_pre[i];
  if (!ok || status != 0 || (OBS && total > a.max_steps)) {
    if (status == 0 && tid == 0 && blockIdx.x == 0) kv_raise(c, MSI_ERR_INVALID_ARG);
    // fail closed: no row of the call can be read as an answer.  If the word was
    // raised by this call, other CTAs are at work: this one covers its rows itself.
    const int from = ok ? 0 : blockIdx.x, step = ok ? 1 : gridDim.x;
    const long long vecs = (long long)a.n_rows * a.H * (D / 8);
    for (long long i = (long long)from * kDecThreads + tid; i < vecs; i += (long long)step * kDecThreads) {
      const long long row = i / (a.H * (D / 8));
      *reinterpret_cast<uint4*>(a.out + row * a.out_stride + (i - row * a.H * (D / 8)) * 8) =
          make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    }
    for (long long i = (long long)from * kDecThreads + tid; i < (long long)a.n_rows * a.H; i += (long long)step * kDecThreads)
      if (a.lse != nullptr) a.lse[i] = kv_nan();
    return;
  }
  const int ctas = kv_ctas(total, a.ctas, kDecWarps);
  const KvRuns runs = {total, ctas};

  // sequences that hold nothing
  for (int b = blockIdx.x; b < a.n; b += gridDim.x) {
    if (s_pre[b + 1] != s_pre[b]) continue;
    const KvWork w = kv_work(a, b);
    for (int i = tid; i < w.rows * a.H * (D / 8); i += kDecThreads) {
      const int row = i / (a.H * (D / 8));
      *reinterpret_cast<uint4*>(a.out + (long long)(w.row0 + row) * a.out_stride + (i - row * a.H * (D / 8)) * 8) =
          make_uint4(0, 0, 0, 0);
    }
    for (int i = tid; i < w.rows * a.H; i += kDecThreads) {
      if (a.lse != nullptr) a.lse[(long long)w.row0 * a.H + i] = -INFINITY;
      if (OBS) a.lse2[(long long)w.row0 * a.H + i] = -INFINITY;
    }
  }
  if ((int)blockIdx.x >= ctas) return;

  uint8_t* ring = smem + wid * RING;
  const uint32_t ring_u = smem_u32(ring);
  long long u = runs.begin(blockIdx.x);
  const long long u_end = runs.begin(blockIdx.x + 1);
  int b = 0;
  {
    int hi = a.n;
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (s_pre[mid] <= u) b = mid; else hi = mid;
    }
  }

  while (u < u_end) {
    while (s_pre[b + 1] <= u) ++b;
    const KvWork w = kv_work(a, b);
    const int units = kv_units(w), groups = kv_groups(a, w, R), pair = (int)((u - s_pre[b]) / units);
    const int h = pair / groups, r0 = (pair - h * groups) * R;  // head, the pair's first row of it
    const long long item0 = s_pre[b] + (long long)pair * units + kPairCost;  // the first step
    const int first = (int)max(u - item0, 0LL);
    const int last = (int)(min(item0 + w.steps, u_end) - item0);  // steps [first, last) of the pair are this CTA's
    u = item0 + last;
    if (last <= first) {  // the run ends within the pair's fixed cost
      u = u_end;
      break;
    }
    const int n_rows = min(R, w.rows * a.G - r0);
    const bool cap = a.softcap > 0.0f;
    const int* table = c.table + (size_t)w.seq * c.max_blocks;

    // the query rows as the MMA's columns
    uint32_t qf[NT][KS][2];
    float cs[NT][2];  // scale * 2^e (log2 e) of rows 2t and 2t + 1 of a tile
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = 8 * nt + g;
      uint4 v[CH][2];
      uint32_t amax = 0;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        v[j][0] = v[j][1] = make_uint4(0, 0, 0, 0);
        if (r < n_rows) {
          const __nv_bfloat16* p = a.q + (long long)(w.row0 + (r0 + r) / a.G) * a.q_stride +
                                   (size_t)(h * a.G + (r0 + r) % a.G) * D + dec_kchunk<D>(t, j) * 16;
          v[j][0] = *reinterpret_cast<const uint4*>(p);
          v[j][1] = *reinterpret_cast<const uint4*>(p + 8);
        }
        const uint32_t* x = reinterpret_cast<const uint32_t*>(v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max(amax, max((x[i] << 16) & 0x7fffffffu, x[i] & 0x7fff0000u));
      }
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      const uint32_t e = kv_row_exp(amax);
      const float down = __uint_as_float((254 - e) << 23);
      const float up = amax < 0x7f800000u ? __uint_as_float(e << 23) * (cap ? a.scale : a.scale * kLog2e) : kv_nan();
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const uint32_t* x = reinterpret_cast<const uint32_t*>(v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t f = amax < 0x7f800000u ? pack_f16x2(bf16_lo(x[i]) * down, bf16_hi(x[i]) * down) : 0u;
          qf[nt][4 * j + (i >> 1)][i & 1] = f;
        }
      }
      cs[nt][0] = __shfl_sync(0xffffffffu, up, 8 * t);
      cs[nt][1] = __shfl_sync(0xffffffffu, up, 8 * t + 4);
    }

    float o[KS][NT][4], m[NT][2], l[NT][2];
    float mu[NT][2];  // m, or 0 where no token has been seen: masked exponents are -inf either way
    float lim[NT][2];  // exponents above it move m
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < KS; ++k) o[k][nt][0] = o[k][nt][1] = o[k][nt][2] = o[k][nt][3] = 0.0f;
      m[nt][0] = m[nt][1] = -INFINITY;
      mu[nt][0] = mu[nt][1] = 0.0f;
      lim[nt][0] = lim[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.0f;
    }
    const float two_cap = cap ? 2.0f * kLog2e / a.softcap : 0.0f;

    float lo = INFINITY, hi = 0.0f;  // value scales of the steps that this lane has looked up
    // this warp's steps: first + wid, + kDecWarps, ..
    const int mine = last - first > wid ? (last - first - wid + kDecWarps - 1) / kDecWarps : 0;
    auto info = [&](int i) {  // of the warp's step i
      StepInfo s = {0, 0.0f, 0.0f, 1.0f};
      if (i < mine) {
        const int tok = (w.step0 + first + wid + i * kDecWarps) << 4;
        s.blk = table[tok >> c.logP];
        if (s.blk >= 0 && s.blk < c.n_blocks) {
          s.ks = c.scale[0][(size_t)s.blk * c.K + h];
          const float vs = c.scale[1][(size_t)s.blk * c.K + h];
          s.lv = log2f(vs);
          lo = fminf(lo, vs);  // of the numbers
          hi = fmaxf(hi, vs);
          // a NaN comes in through the exponents of the tokens that a row sees;
          // rows that see none have weights 0 and must not meet it here
          s.iv = vs > 0.0f ? 1.0f / vs : 1.0f;
        } else {
          kv_raise(c, MSI_ERR_INVALID_ARG);
          s.blk = 0;
          s.ks = s.lv = kv_nan();
        }
      }
      return s;
    };
    StepInfo use = info(lane), ahead = use;  // steps 32 q + lane: those in use, those being fetched
    // a lane's copies: 16 bytes of row r0 + 512 / D per copy
    constexpr int CPR = D / 16, RPC = 32 / CPR;
    const uint32_t in_dst = ring_u + dec_chunk<D>(lane / CPR, lane % CPR);
    int st_in = 0;  // the stage that the next fetch fills
    auto fetch = [&](int i) {
      if ((i & 31) == 0 && i > 0) ahead = info(i + lane);
      const int blk = __shfl_sync(0xffffffffu, ahead.blk, i & 31);
      if (i < mine) {
        const int tok = (w.step0 + first + wid + i * kDecWarps) << 4;
        const size_t at = (((size_t)blk * c.K + h) * c.P + (tok & (c.P - 1))) * D + lane * 16;
        const uint8_t* kp = c.codes[0] + at;
        const uint8_t* vp = c.codes[1] + at;
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
          // rows n RPC on: the swizzle, row & 7, changes by n RPC & 7 (D = 64: by nothing)
          const uint32_t dst = ((in_dst + st_in * SB) ^ (D == 64 ? 0 : (n * RPC & 7) << 4)) + n * RPC * D;
          copy16(dst, kp + n * 512);
          copy16(dst + 16 * D, vp + n * 512);
        }
      }
      cp_async_commit();
      st_in = st_in + 1 == S ? 0 : st_in + 1;
    };
    int st = 0;  // the stage in use
    const uint32_t k_at = dec_chunk<D>(g, dec_kchunk<D>(t, 0));
    const uint32_t v_at = D == 64 ? dec_chunk<D>(2 * t, g >> 1) + (g & 1) * 8 : dec_chunk<D>(2 * t, g);
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) fetch(i);

#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
      if ((i & 31) == 0 && i > 0) use = ahead;
      cp_async_wait<S - 2>();
      __syncwarp();
      fetch(i + S - 1);
      const int idx = first + wid + i * kDecWarps;
      const int tok0 = (w.step0 + idx) << 4;
      const float ks = __shfl_sync(0xffffffffu, use.ks, i & 31);
      const float lv = __shfl_sync(0xffffffffu, use.lv, i & 31);
      const float iv = __shfl_sync(0xffffffffu, use.iv, i & 31);
      const uint32_t kb = ring_u + st * SB, vb = kb + 16 * D;
      st = st + 1 == S ? 0 : st + 1;

      float sc[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.0f;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        // chunk dec_kchunk(t, j): one more flips the lowest bit, eight more are the next 128 bytes
        const uint32_t kj = ((kb + k_at) ^ ((j & 1) << 4)) + (j >> 1) * 128;
        const uint4 x = ld_shared_v4(kj);
        const uint4 y = ld_shared_v4(kj + 8 * D);  // row g + 8: the same swizzle
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t a0 = kv_f16x2<FMT, false>(xs[q]), a2 = kv_f16x2<FMT, true>(xs[q]);
          const uint32_t a1 = kv_f16x2<FMT, false>(ys[q]), a3 = kv_f16x2<FMT, true>(ys[q]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_f16(sc[nt], a0, a1, a2, a3, qf[nt][4 * j + q][0], qf[nt][4 * j + q][1]);
        }
      }

      // exponents: [0], [1] token g, [2], [3] token g + 8; rows 2t, 2t + 1
      const bool whole = tok0 + 16 <= w.held - w.rows + 1 &&
                         (a.window == 0 || tok0 > w.held - 1 - a.window);
      if (cap && a.softcap <= kSmallCap) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            sc[nt][q] = fmaf(kv_softcap<false>(sc[nt][q] * (cs[nt][q & 1] * ks), a.softcap, two_cap), kLog2e, lv);
      } else if (cap) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            sc[nt][q] = fmaf(kv_softcap<true>(sc[nt][q] * (cs[nt][q & 1] * ks), a.softcap, two_cap), kLog2e, lv);
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 4; ++q) sc[nt][q] = fmaf(sc[nt][q], cs[nt][q & 1] * ks, lv);
      }
      if (!whole) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int tok = tok0 + g + (q >> 1) * 8;
            // the last token that the row sees
            const int see = w.held - w.rows + (r0 + 8 * nt + 2 * t + (q & 1)) / a.G;
            if (tok > see || (a.window > 0 && tok <= see - a.window)) sc[nt][q] = -INFINITY;
          }
      }
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int q = 0; q < 4; ++q) over |= sc[nt][q] > lim[nt][q & 1];
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float v = fmaxf(sc[nt][q], sc[nt][q + 2]);
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            v = fmaxf(v, m[nt][q]);
            const float f = v == -INFINITY ? 1.0f : ex2(m[nt][q] - v);
            m[nt][q] = v;
            mu[nt][q] = v == -INFINITY ? 0.0f : v;
            lim[nt][q] = v + kLazy;
            l[nt][q] *= f;
#pragma unroll
            for (int k = 0; k < KS; ++k) o[k][nt][q] *= f, o[k][nt][q + 2] *= f;
          }
      }
      uint32_t pf[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float p[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = ex2(sc[nt][q] - mu[nt][q & 1]);
        const float s0 = (p[0] + p[2]) * iv, s1 = (p[1] + p[3]) * iv;
        l[nt][0] += s0;
        l[nt][1] += s1;
        if (OBS) {
          float v0 = s0, v1 = s1;
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) {
            v0 += __shfl_xor_sync(0xffffffffu, v0, x);
            v1 += __shfl_xor_sync(0xffffffffu, v1, x);
          }
          if (g == 0)
            *reinterpret_cast<float2*>(a.step_lse + (item0 + idx) * R + 8 * nt + 2 * t) =
                make_float2(mu[nt][0] + lg2_any(v0), mu[nt][1] + lg2_any(v1));
        }
        pf[nt][0] = transpose8x8(pack_f16x2(p[0], p[1]));
        pf[nt][1] = transpose8x8(pack_f16x2(p[2], p[3]));
      }

      // O^T += V^T P^T: rows d0 and d0 + 1 of a column tile, tokens 2t, 2t + 1, 2t + 8, 2t + 9
      auto values = [&](const uint32_t* x, const uint32_t* y, const uint32_t* z, const uint32_t* v, int words, int k0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (q >= words) break;
          const uint32_t lo0 = __byte_perm(x[q], y[q], 0x5140), lo1 = __byte_perm(x[q], y[q], 0x7362);
          const uint32_t hi0 = __byte_perm(z[q], v[q], 0x5140), hi1 = __byte_perm(z[q], v[q], 0x7362);
          const uint32_t a0 = kv_f16x2<FMT, false>(lo0), a1 = kv_f16x2<FMT, true>(lo0);
          const uint32_t a2 = kv_f16x2<FMT, false>(hi0), a3 = kv_f16x2<FMT, true>(hi0);
          const uint32_t b0 = kv_f16x2<FMT, false>(lo1), b1 = kv_f16x2<FMT, true>(lo1);
          const uint32_t b2 = kv_f16x2<FMT, false>(hi1), b3 = kv_f16x2<FMT, true>(hi1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_f16(o[k0 + 2 * q][nt], a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
            mma_f16(o[k0 + 2 * q + 1][nt], b0, b1, b2, b3, pf[nt][0], pf[nt][1]);
          }
        }
      };
      // tokens 2t, 2t + 1 (the next row: D = 64 has its swizzle in pairs of rows), 2t + 8, 2t + 9
      if constexpr (D == 64) {
        const uint32_t va = vb + v_at;
        const uint2 x = ld_shared_v2(va), y = ld_shared_v2(va + D), z = ld_shared_v2(va + 8 * D), v = ld_shared_v2(va + 9 * D);
        const uint32_t xs[4] = {x.x, x.y, 0, 0}, ys[4] = {y.x, y.y, 0, 0}, zs[4] = {z.x, z.y, 0, 0}, vs4[4] = {v.x, v.y, 0, 0};
        values(xs, ys, zs, vs4, 2, 0);
      } else {
#pragma unroll
        for (int j = 0; j < D / 128; ++j) {
          const uint32_t va = vb + v_at + j * 128, vo = ((vb + v_at) ^ 16) + j * 128 + D;
          const uint4 x = ld_shared_v4(va), y = ld_shared_v4(vo), z = ld_shared_v4(va + 8 * D), v = ld_shared_v4(vo + 8 * D);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
          const uint32_t zs[4] = {z.x, z.y, z.z, z.w}, vs4[4] = {v.x, v.y, v.z, v.w};
          values(xs, ys, zs, vs4, 4, 8 * j);
        }
      }
      __syncwarp();  // the stage is read: the next turn's fetch writes it
    }
    cp_async_wait<0>();
    // positive numbers are ordered as their bits are
    lo = __uint_as_float(__reduce_min_sync(0xffffffffu, __float_as_uint(lo)));
    hi = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(hi)));
    if (hi > lo * kScaleRange) {
      if (lane == 0) kv_raise(c, MSI_ERR_UNSUPPORTED);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) l[nt][0] = l[nt][1] = kv_nan();
    }

    // the warps' parts: reference and sum per row, then the outputs
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float v = l[nt][q];
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v += __shfl_xor_sync(0xffffffffu, v, 8);
        v += __shfl_xor_sync(0xffffffffu, v, 16);
        if (g == 0) s_m[wid][8 * nt + 2 * t + q] = m[nt][q], s_l[wid][8 * nt + 2 * t + q] = v;
      }
    __syncthreads();  // also: every warp is done with its ring
    // [row][column tile][g]: the lanes' pairs of columns side by side, rows two
    // pairs further apart than their length, so that no two lanes share a bank
    constexpr int RS = D / 2 + 2;
    float2* part = reinterpret_cast<float2*>(smem) + (size_t)wid * R * RS;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int r = 8 * nt + 2 * t + q;
        float top = s_m[0][r];
#pragma unroll
        for (int i = 1; i < kDecWarps; ++i) top = fmaxf(top, s_m[i][r]);
        const float f = m[nt][q] == -INFINITY ? (l[nt][q] == 0.0f ? 0.0f : l[nt][q]) : ex2(m[nt][q] - top);
#pragma unroll
        for (int k = 0; k < KS; ++k) part[r * RS + 8 * k + g] = make_float2(o[k][nt][q] * f, o[k][nt][q + 2] * f);
      }
    __syncthreads();
    const bool split = first > 0 || last < w.steps;
    const int slot = 2 * blockIdx.x + (first > 0 ? 0 : 1);
    for (int e = tid; e < n_rows * (D / 2); e += kDecThreads) {
      const int r = e / (D / 2), p = e % (D / 2), k = p >> 3, pg = p & 7;
      const int d = D == 64 ? 8 * pg + 2 * k : 128 * (k >> 3) + 16 * pg + 2 * (k & 7);
      float top = s_m[0][r];
#pragma unroll
      for (int i = 1; i < kDecWarps; ++i) top = fmaxf(top, s_m[i][r]);
      float sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
      for (int i = 0; i < kDecWarps; ++i) {
        sum += s_m[i][r] == -INFINITY ? s_l[i][r] : kv_scaled(s_l[i][r], s_m[i][r] - top);
        const float2 v = reinterpret_cast<const float2*>(smem)[((size_t)i * R + r) * RS + p];
        x += v.x;
        y += v.y;
      }
      if (split) {
        *reinterpret_cast<float2*>(a.part_o + ((size_t)slot * R + r) * D + d) = make_float2(x, y);
        if (d == 0) a.part_ml[(size_t)slot * 2 * R + r] = top, a.part_ml[(size_t)slot * 2 * R + R + r] = sum;
        if (e == 0 && first == 0)
          a.split[blockIdx.x] = make_int4(w.row0, n_rows | r0 << 8, h, runs.owner(item0 + w.steps - 1) - blockIdx.x + 1);
      } else {
        const long long row = w.row0 + (r0 + r) / a.G;
        const int head = h * a.G + (r0 + r) % a.G;
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<uint32_t*>(a.out + row * a.out_stride + (size_t)head * D + d) = pack_bf16x2(x * f, y * f);
        if (d == 0) {
          const float l2 = sum == 0.0f ? -INFINITY : top + log2f(sum);
          if (a.lse != nullptr) a.lse[row * a.H + head] = l2 * kLn2;
          if (OBS) a.lse2[row * a.H + head] = l2;
        }
      }
    }
    __syncthreads();  // the parts are read: the ring may be written
  }
}

// Joins the parts of the pair that begins in run x and goes on past it: weights
// 2^(M_i - M) over the parts, in the CTAs' order.  Bound: latency (with the kernel
// before, 64 sequences of 8,192 take 45.6 us by warps and 49.8 by CTAs, one of
// 1,000 8.8 and 13.5; a warp has one lane a part, so more than 32 go to a CTA).
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinFew = 32;

// Up to 32 parts: a warp a row, no barriers.
template <int D>
__device__ __forceinline__ void kv_join_few(const KvAttnArgs& a, int R, int x, int r) {
  constexpr int V = D / 32, B = 8;  // a lane's columns, parts loaded at a time
  const int lane = threadIdx.x & 31;
  const int4 at = a.split[x];  // first row, rows and the first of them, head, parts
  const int parts = at.w;
  if (r >= (at.y & 255) || parts == 0 || parts > kJoinFew) return;
  const int hr = (at.y >> 8) + r;  // row of the head
  const long long row = at.x + hr / a.G;
  const int head = at.z * a.G + hr % a.G;
  const bool failed = a.c.control[1] != 0;  // within the call
  auto slot_of = [&](int i) { return (size_t)(2 * (x + i) + (i == 0 ? 1 : 0)); };
  const float pm = lane < parts ? a.part_ml[slot_of(lane) * 2 * R + r] : -INFINITY;
  const float pl = lane < parts ? a.part_ml[slot_of(lane) * 2 * R + R + r] : 0.0f;
  float acc[V], part[B][V];
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) part[i][v] = i0 + i < parts ? a.part_o[(slot_of(i0 + i) * R + r) * D + v * 32 + lane] : 0.0f;
  };
  load(0);  // on its way while the weights are worked out
  float top = pm;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float f = pm == -INFINITY ? (pl == 0.0f ? 0.0f : pl) : ex2(pm - top);
  float sum = pm == -INFINITY ? pl : kv_scaled(pl, pm - top);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.0f;
  for (int i0 = 0; i0 < parts; i0 += B) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const float w = __shfl_sync(0xffffffffu, f, i0 + i);  // 0 past the last part
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] = fmaf(w, part[i][v], acc[v]);
    }
  }
  const float inv = failed ? kv_nan() : sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int v = 0; v < V; ++v) a.out[row * a.out_stride + (size_t)head * D + v * 32 + lane] = __float2bfloat16_rn(acc[v] * inv);
  if (lane == 0 && a.lse != nullptr)
    a.lse[row * a.H + head] = failed ? kv_nan() : sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// More: the n-th such pair, a CTA a row.
template <int D>
__device__ __forceinline__ void kv_join_many(const KvAttnArgs& a, int R, int n, int r) {
  constexpr int W = kJoinWarps, V = D / 32;  // V: a lane's columns
  __shared__ float s_f[1024], s_part[W][D], s_red[W];
  __shared__ int s_scan[32], s_x;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  if (tid == 0) s_x = -1;
  int base = 0;  // such pairs before these runs
  for (int i0 = 0; i0 < a.ctas; i0 += kJoinThreads) {
    const int many = i0 + tid < a.ctas && a.split[i0 + tid].w > kJoinFew;
    const int in = block_scan(many, s_scan);
    if (many && base + in - 1 == n) s_x = i0 + tid;
    __syncthreads();
    base += s_scan[31];  // the last warp's running total
    __syncthreads();
  }
  const int x = s_x;
  if (x < 0) return;
  const int4 at = a.split[x];  // first row, rows and the first of them, head, parts
  const int parts = at.w;
  if (r >= (at.y & 255)) return;
  const int hr = (at.y >> 8) + r;  // row of the head
  const long long row = at.x + hr / a.G;
  const int head = at.z * a.G + hr % a.G;
  const bool failed = a.c.control[1] != 0;  // within the call
  auto slot_of = [&](int i) { return (size_t)(2 * (x + i) + (i == 0 ? 1 : 0)); };
  float mi[4], li[4];  // this thread's parts: 1,024 CTAs at most
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = k * kJoinThreads + tid;
    mi[k] = -INFINITY;
    li[k] = 0.0f;
    if (i < parts) {
      mi[k] = a.part_ml[slot_of(i) * 2 * R + r];
      li[k] = a.part_ml[slot_of(i) * 2 * R + R + r];
    }
    top = fmaxf(top, mi[k]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s_red[wid] = top;
  __syncthreads();
  top = s_red[0];
#pragma unroll
  for (int i = 1; i < W; ++i) top = fmaxf(top, s_red[i]);
  __syncthreads();
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = k * kJoinThreads + tid;
    const float f = mi[k] == -INFINITY ? (li[k] == 0.0f ? 0.0f : li[k]) : ex2(mi[k] - top);
    if (i < parts) s_f[i] = f;
    sum += mi[k] == -INFINITY ? li[k] : kv_scaled(li[k], mi[k] - top);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_red[wid] = sum;
  __syncthreads();
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < W; ++i) sum += s_red[i];
  float acc[V];
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.0f;
#pragma unroll 8
  for (int i = wid; i < parts; i += W) {
    const float* p = a.part_o + (slot_of(i) * R + r) * D;
    const float f = s_f[i];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = fmaf(f, p[v * 32 + lane], acc[v]);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) s_part[wid][v * 32 + lane] = acc[v];
  __syncthreads();
  const float f = failed ? kv_nan() : sum == 0.0f ? 0.0f : 1.0f / sum;
  for (int d = tid; d < D; d += kJoinThreads) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += s_part[i][d];
    a.out[row * a.out_stride + (size_t)head * D + d] = __float2bfloat16_rn(v * f);
  }
  if (tid == 0 && a.lse != nullptr)
    a.lse[row * a.H + head] = failed ? kv_nan() : sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// Attention weight of each block: over the heads, its 16-token granules and the
// rows, 2^(granule's log2 sum - row's log2 sum).  The granules of neighbouring
// blocks lie together, so a lane takes four rows of one granule for every head,
// and a warp the blocks that 128 of these sums hold (or one block, in passes).
// Lanes are added in one order.  `warps` warps, of which this is the wid-th.
// s_top: [pairs][R] log2 of the rows' sums; -inf: a row that is none.
__device__ __forceinline__ void kv_weights(const KvAttnArgs& a, const KvWork& w, long long pre, int R, const float* s_top, int wid,
                                           int warps) {
  const KvCache& c = a.c;
  const int lane = threadIdx.x & 31, pairs = c.K * kv_groups(a, w, R);
  const int per = c.P / 16, sums = per * R;                // of a block and head: 8 .. 256, a power of two
  const int nb = sums >= 128 ? 1 : 128 / sums;             // blocks of a warp's turn
  const int lanes = sums >= 128 ? 32 : sums / 4;           // lanes of a block
  const int j0 = w.step0 / per, j1 = (w.held + c.P - 1) >> c.logP;
  for (int j = j0 + wid * nb; j < j1; j += warps * nb) {
    const int mine = j + lane / lanes;
    const bool writes = (lane & (lanes - 1)) == 0 && mine < j1;
    const int id = writes ? c.table[(size_t)w.seq * c.max_blocks + mine] : -1;
    const bool there = id >= 0 && id < c.n_blocks;
    const float had = there ? c.weight[id] : 0.0f;
    float v = 0.0f;
    for (int f = lane * 4; f < nb * sums; f += 128) {
      const int step = j * per + f / R - w.step0, r = f & (R - 1);  // R is a power of two
      if (step < 0 || step >= w.steps) continue;
      const float* p = a.step_lse + (pre + kPairCost + step) * R + r;
#pragma unroll 4
      for (int h = 0; h < pairs; ++h) {
        const float4 x = *reinterpret_cast<const float4*>(p + (long long)h * kv_units(w) * R);
        const float4 t = *reinterpret_cast<const float4*>(s_top + h * R + r);
        if (t.x != -INFINITY) v += ex2(x.x - t.x);
        if (t.y != -INFINITY) v += ex2(x.y - t.y);
        if (t.z != -INFINITY) v += ex2(x.z - t.z);
        if (t.w != -INFINITY) v += ex2(x.w - t.w);
      }
    }
    __syncwarp();
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (there) c.weight[id] = had + v;
  }
}

// The block weights (`ny` CTAs a sequence), which put the sums of a split pair's
// rows together from its parts, and the joins (`joins` CTAs: runs by 8 rows for
// pairs of few parts, then the pairs of many by rows).
template <int D>
__global__ void __launch_bounds__(kJoinThreads) kv_finish_kernel(KvAttnArgs a, int R, int warps, int joins, int ny) {
  extern __shared__ __align__(16) float s_top[];
  grid_wait();
  grid_release();
  const int obs = gridDim.x - joins;  // first: they take longer
  if ((int)blockIdx.x >= obs) {
    const int i = blockIdx.x - obs, few = a.ctas * (R / kJoinWarps);
    if (i < few) kv_join_few<D>(a, R, i % a.ctas, i / a.ctas * kJoinWarps + (threadIdx.x >> 5));
    else kv_join_many<D>(a, R, (i - few) / R, (i - few) % R);
    return;
  }
  const KvCache& c = a.c;
  const int b = blockIdx.x / ny, y = blockIdx.x % ny;
  const KvWork w = kv_work(a, b);
  const long long pre = a.item_pre[b], total = a.item_pre[a.n];
  if (c.control[1] != 0 || w.steps == 0) return;
  const int n = w.rows * a.G, groups = kv_groups(a, w, R);
  const KvRuns runs = {total, kv_ctas(total, a.ctas, warps)};
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  for (int i = wid; i < c.K * groups * R; i += kJoinThreads / 32) {  // a warp a row
    const int pair = i / R, r = i - pair * R, h = pair / groups, hr = (pair - h * groups) * R + r;
    float l2 = -INFINITY;
    if (hr < n) {
      const long long u0 = pre + (long long)pair * kv_units(w) + kPairCost;
      const int c0 = runs.owner(u0), c1 = runs.owner(u0 + w.steps - 1);
      if (c0 == c1) {
        l2 = a.lse2[(long long)(w.row0 + hr / a.G) * a.H + h * a.G + hr % a.G];
      } else {
        float top = -INFINITY, sum = 0.0f;
        for (int x = c0 + lane; x <= c1; x += 32) {
          const float* ml = a.part_ml + (size_t)(2 * x + (x == c0 ? 1 : 0)) * 2 * R + r;
          const float m = ml[0], l = ml[R];
          if (m > top) sum = top == -INFINITY ? sum : kv_scaled(sum, top - m), top = m;
          sum += m == -INFINITY ? l : kv_scaled(l, m - top);
        }
        float all = top;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
        if (top != -INFINITY) sum = kv_scaled(sum, top - all);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        l2 = sum == 0.0f ? -INFINITY : all + log2f(sum);
      }
    }
    if (lane == 0) s_top[i] = l2;
  }
  __syncthreads();
  kv_weights(a, w, pre, R, s_top, y * (kJoinThreads / 32) + wid, ny * (kJoinThreads / 32));
}

template <int D, int NT, int FMT, bool OBS>
cudaError_t decode_as(const KvAttnArgs& a, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  constexpr int W = dec_warps(D, NT), ring = W * dec_stages(D, NT) * dec_stage_bytes(D);
  static_assert(W * 8 * NT * (D + 4) * 4 <= ring, "the parts fit the rings");
  cudaError_t e = smem_attr_once(kv_decode_kernel<D, NT, FMT, OBS>, ring + (kKvMaxSeqs + 1) * (int)sizeof(long long), done);
  if (e != cudaSuccess) return e;
  e = launch_after(false, kv_decode_kernel<D, NT, FMT, OBS>, dim3(a.ctas), dim3(32 * W),
                   ring + (a.n + 1) * sizeof(long long), s, a);
  if (e != cudaSuccess) return e;
  const int joins = a.ctas * NT + a.ctas / kJoinFew * 8 * NT;  // no more than that have more than 32 parts
  // a turn of every warp of a CTA; longer tables take several
  const int sums = a.c.P / 16 * 8 * NT, per = kJoinThreads / 32 * (sums >= 128 ? 1 : 128 / sums);
  const int ny = min((min(a.c.max_blocks, a.c.n_blocks) + per - 1) / per, 64);
  return launch_after(true, kv_finish_kernel<D>, dim3(joins + (OBS ? a.n * ny : 0)), dim3(kJoinThreads),
                      OBS ? a.c.K * a.groups * 8 * NT * sizeof(float) : 0, s, a, 8 * NT, W, joins, ny);
}

template <int D, int NT, int FMT>
cudaError_t decode_opt(const KvAttnArgs& a, cudaStream_t s) {
  return a.observe ? decode_as<D, NT, FMT, true>(a, s) : decode_as<D, NT, FMT, false>(a, s);
}

template <int D, int NT>
cudaError_t decode_fmt(const KvAttnArgs& a, cudaStream_t s) {
  return a.c.fmt == MSI_KV_Q8 ? decode_opt<D, NT, MSI_KV_Q8>(a, s) : decode_opt<D, NT, MSI_KV_E4M3>(a, s);
}

}  // namespace

int kv_decode_pair_cost() { return kPairCost; }

// More rows than a group holds are several pairs: each reads the codes again, but
// mostly from L2 (64 sequences of 8,192, D = 128: 59 us for 16 rows, 97 for 32 in
// two groups, against 157 in one group of 32, whose registers spill; D = 64: 56
// for 32 in one).  Chunk form takes over about where it is as fast for many
// sequences and the gap for one is small (decode form at its most rows, chunk form
// with 8 more; 64 sequences of 8,192 / one of 32,768): D = 64 97 and 160 / 19 and
// 31 us, D = 128 184 and 182 / 24 and 36, D = 256 272 and 288 / 33 and 46.
int kv_decode_tiles(int rows, int D) {
  return rows > (D == 256 ? 48 : 64) ? 0 : rows <= 8 ? 1 : rows <= 16 || D > 64 ? 2 : 4;
}

cudaError_t launch_kv_decode(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  const int nt = kv_decode_tiles(a.max_rows * a.G, a.c.D);
  *launches = 2;
  if (a.c.D == 64) return nt == 1 ? decode_fmt<64, 1>(a, s) : nt == 2 ? decode_fmt<64, 2>(a, s) : decode_fmt<64, 4>(a, s);
  if (a.c.D == 128) return nt == 1 ? decode_fmt<128, 1>(a, s) : decode_fmt<128, 2>(a, s);
  return nt == 1 ? decode_fmt<256, 1>(a, s) : decode_fmt<256, 2>(a, s);
}

}  // namespace msi
