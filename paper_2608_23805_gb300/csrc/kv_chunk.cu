// Attention over the 8-bit key-value cache in chunk form: many query rows of a
// sequence (a chunk of a prompt) against everything that it holds, on the
// tcgen05 tensor cores.  The mathematics is kv_decode.cu's: exact fp16 codes
// and queries, fp32 scores, the value's scale in the exponent, weights rounded
// once to fp16.
//
// An item is one sequence, key-value head and tile of 256 or 512 rows (query
// tokens times the head's query heads, so a tile reads the shared keys once).  Two
// CTAs share an item: each has half of the rows and of the outputs, and converts
// and holds half of the keys (tokens) and values (columns) for both (cta_group::2).
// Tiles of NT tokens go through
//   conversion warps: 16 tokens of keys or values at a time, from global memory
//     to registers two turns ahead, to fp16 (two instructions a pair), to
//     swizzled shared memory;
//   MMA warps, one a row tile, of the first CTA: S = Q K^T (both from shared
//     memory), O += P V (P from TMEM, V with the columns contiguous).  Two S of
//     each row tile, so that the next scores are ready when softmax is;
//   softmax warps, a row a thread (D = 256: two, each half of the columns): S
//     from TMEM, P = 2^(c s + log2 sv - M) to TMEM over S.  M is a running
//     reference: a tile is done in one pass with the old M unless some sum of 16
//     weights passes 2^11 (a bound on each of them, so no maximum is taken); only
//     then is M moved and O rescaled.
// Two row tiles of 128 rows a CTA, and at D = 256, whose O takes half of TMEM, one.
//
// The work is the list of all token tiles of all items; each pair takes an
// equal run, parts of split items are joined by kv_chunk_join_kernel in order.
//
// Measured: 4,096 rows on 32,768 tokens, 16 heads of 128 over 2: 697 us,
// 1,480 TFLOP/s, 0.76 of a large library product; four chunks of 3,000 on
// themselves, D = 256, capped: 343 us.  Single CTAs with one S a row tile had 790
// and 457 us (conversion and operand reads filled shared memory), pairs with one S
// 770 and 364 (a row tile's softmax, its products and the signals between them
// follow one another).  Bound: the softmax warps (without their arithmetic 566 and
// 271 us) and, for short items at D = 256, the items' fixed cost: O and two S fill
// TMEM, so that a product waits for the output before it.  Few rows: a tile's chain
// through the pair (72 rows of 64 sequences of 8,192, D = 128: 182 us).
//
// Every wait is bounded: on expiry the CTA gives up, drains its MMAs, frees
// TMEM and raises MSI_ERR_TIMEOUT; the join then makes every row of the call NaN.
#include "kv.cuh"

namespace msi {
namespace {

constexpr float kChunkTop = 2048.0f;            // sums of 16 weights above it move the reference

template <int D>
struct Chunk {
  static constexpr int NQ = D == 256 ? 1 : 2;     // row tiles
  static constexpr int NT = D == 256 ? 128 : 64;  // tokens of a tile: two S of each row tile and O fill TMEM
  static constexpr int ST = D == 256 ? 2 : 4;     // stages of keys and values
  static constexpr int TROWS = 256;               // rows of a row tile, 128 a CTA
  static constexpr int ROWS = TROWS * NQ;
  static constexpr int NG = NT / 16;              // 16-token granules
  static constexpr int COLS = 64;                 // S columns a softmax thread takes
  static constexpr int KROWS = NT / 2;            // a CTA's tokens of the keys,
  static constexpr int VCOLS = D / 2;             // and columns of the values
  static constexpr int QBYTES = 128 * D * 2;      // a CTA's part of a row tile
  static constexpr int KBYTES = KROWS * D * 2;    // and of a tile's keys, or values
  static constexpr int SMEM = NQ * QBYTES + 2 * ST * KBYTES + 1024;
  // conversion tasks: 16 tokens of keys, up to 128 columns; 16 tokens of values, or 32 of 64 columns or fewer
  static constexpr int KC = D < 128 ? D : 128;
  static constexpr int SUB = D / KC;              // tasks of 16 tokens' keys
  static constexpr int VT = D == 256 ? 16 : 32;
  // values: rows of one panel's columns, 128 bytes of 64 or (D = 64) 64 bytes of 32, swizzled by as many
  static constexpr int VROW = VCOLS < 64 ? 64 : 128;
  static constexpr int KTASKS = KROWS / 16 * SUB, VTASKS = NT / VT;
  static constexpr int LOADS = KC / 32;           // 16-byte loads a lane
  static_assert(VT * VCOLS == 16 * KC, "all tasks of one size");
  static constexpr int TO = 256;                  // first column of O in TMEM
  // 8 softmax warps, then conversion warps, then an MMA warp a row tile
  static constexpr int SOFT = 8, MMA = 16 - NQ, CONV = MMA - SOFT;
};
// 16 warps; the groups share 512 x 128 registers out: 2 x 144 + 2 x 112 a thread.
constexpr int kChunkThreads = 512;
constexpr int kSoftRegs = 144, kConvRegs = 112;
static_assert(2 * kSoftRegs + 2 * kConvRegs <= 512, "registers of the launch");
// What an item costs beside its tiles (queries, first scores, output), in tiles; us
// at 2, 3, 4, 5, 6: four chunks of 3,000 at D = 64 132, 127, 121, 119, 119, D = 128
// 185, 180, 168, 165, 157, D = 256 355, 326, 303, 307, 313; 8 of 500 at D = 64 26.0,
// 25.9, 25.8, 27.5, 27.7, D = 128 37.1, 36.4, 36.2, 36.3, 35.4, D = 256 53.2, 49.9, 47.7,
// 48.6, 49.8; long items within 1 %.
constexpr int kItemCost = 4;

__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
}
// D[tmem] (+)= A[tmem] * B[smem], fp16, both CTAs of a pair: each has its rows of A
// and its columns of B
__device__ __forceinline__ void umma_f16_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                                 uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// kind::f16 with fp16 operands and fp32 sums; mn: B's columns are contiguous
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, int mn) {
  return (1u << 4) | ((uint32_t)mn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// 32 lanes x 32 consecutive 32-bit columns, registers to TMEM
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
      "%13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
      "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
      "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int N, bool INC>
__device__ __forceinline__ void set_regs() {
  if (INC) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// ---------------------------------------------------------------------------
// The plan of a call: items and the prefix of their token tiles
// ---------------------------------------------------------------------------
// T threads: at least as many as sequences.
template <int T>
__global__ void __launch_bounds__(T) kv_plan_kernel(KvAttnArgs a, int rows_tile, int nt) {
  __shared__ int s_scan[32], s_base[kKvMaxSeqs + 1], s_bad;
  __shared__ int4 s_work[kKvMaxSeqs];  // seq, first row, rows, tokens held
  __shared__ long long s_sum[32], s_pre[T + 1], s_total;
  const KvCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  grid_release();
  if (tid == 0) s_bad = 0, s_total = 0;
  __syncthreads();
  int tiles = 0;
  if (tid < a.n) {
    const KvWork w = kv_work(a, tid);
    s_work[tid] = make_int4(w.seq, w.row0, w.rows, w.held);
    if (!w.ok) s_bad = 1;
    else tiles = (w.rows * a.G + rows_tile - 1) / rows_tile * c.K;
  }
  const int in = block_scan(tiles, s_scan);
  s_base[tid] = in - tiles;
  if (tid == T - 1) s_base[T] = in;
  __syncthreads();
  // one CTA reads the status word for all: it may change while the others start
  const int status = c.control[1];
  const bool ok = s_bad == 0 && s_base[T] <= a.max_items && status == 0;
  if (!ok && status == 0 && tid == 0) kv_raise(c, MSI_ERR_INVALID_ARG);
  const int items = ok ? s_base[T] : 0;
  for (int i0 = 0; i0 < items; i0 += T) {
    const int i = i0 + tid;
    long long n = 0;
    if (i < items) {
      int lo = 0, hi = a.n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_base[mid] <= i) lo = mid; else hi = mid;
      }
      const int4 w = s_work[lo];
      const int per = (w.z * a.G + rows_tile - 1) / rows_tile;
      const int h = (i - s_base[lo]) / per, rt = (i - s_base[lo]) % per;
      const int r1 = min(w.z * a.G, (rt + 1) * rows_tile) - 1;
      const int see0 = w.w - w.z + rt * rows_tile / a.G, see1 = w.w - w.z + r1 / a.G;
      const int t0 = a.window > 0 ? max(0, see0 - a.window + 1) / nt : 0;
      n = max(1, see1 < 0 ? 0 : see1 / nt + 1 - t0) + kItemCost;  // an item that sees nothing has a tile too
      a.items[2 * i] = w;
      a.items[2 * i + 1] = make_int4(h, rt, t0, 0);
    }
    long long v = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    if (lane == 31) s_sum[wid] = v;
    __syncthreads();
    long long before = s_total + v - n;
    for (int k = 0; k < wid; ++k) before += s_sum[k];
    if (i < items) a.item_pre[i] = before;
    s_pre[tid] = before;  // read below where one pass has all items
    __syncthreads();
    if (tid == T - 1) s_total = before + n;
    __syncthreads();
  }
  const long long total = s_total;
  const int ctas = (int)min((long long)a.ctas, max(1LL, total / 2));
  // where each CTA's run begins
  const KvRuns runs = {total, ctas};
  for (int x = tid; x < ctas && items > 0; x += T) {
    const long long u = runs.begin(x);
    int lo = 0, hi = items;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((items <= T ? s_pre[mid] : a.item_pre[mid]) <= u) lo = mid; else hi = mid;
    }
    a.plan[4 + x] = lo;
  }
  if (tid == 0) {
    a.item_pre[items] = total;
    a.plan[0] = items;
    a.plan[1] = ok;
    a.plan[2] = ctas;
    a.plan[3] = 0;  // a wait ran out, or value scales lie too far apart
  }
}

// ---------------------------------------------------------------------------
// A CTA's parts: runs of token tiles of successive items
// ---------------------------------------------------------------------------
struct Part {
  int seq, row0, rows, held;   // of the sequence
  int h, row_tile, tile0;      // of the item; tile0: its first token tile
  int first, last, tiles;      // token tiles [first, last) of the item's `tiles` are this CTA's
};

struct PartWalk {
  long long u, end;
  int item;

  __device__ __forceinline__ void init(const KvAttnArgs& a, int cta) {
    const int items = a.plan[0], ctas = a.plan[2];
    item = a.plan[4 + cta];
    const long long total = a.item_pre[items];
    const KvRuns runs = {total, ctas};
    u = runs.begin(cta);
    end = runs.begin(cta + 1);
  }
  __device__ __forceinline__ bool next(const KvAttnArgs& a, Part& p) {
    while (u < end) {
      const long long p0 = a.item_pre[item] + kItemCost, p1 = a.item_pre[item + 1];
      const int4 w = a.items[2 * item], it = a.items[2 * item + 1];
      p.first = (int)max(u - p0, 0LL);
      p.last = (int)(min(p1, end) - p0);
      p.tiles = (int)(p1 - p0);
      u = min(p1, end);
      ++item;
      if (p.last <= p.first) continue;  // the run ends within the item's fixed cost
      p.seq = w.x;
      p.row0 = w.y;
      p.rows = w.z;
      p.held = w.w;
      p.h = it.x;
      p.row_tile = it.y;
      p.tile0 = it.z;
      return true;
    }
    return false;
  }
};

// log2 weights of 16 scores: c s + ad, or its capped form (CAP 1: caps up to
// kSmallCap, 2: any), masked beyond `lim` and at or before `low` (columns of the granule)
template <int CAP, bool MASK>
__device__ __forceinline__ float chunk_exp(float s, float c, float ad, float cap, float two_cap, int col, int lim, int low) {
  float e = CAP != 0 ? fmaf(kv_softcap<CAP == 2>(s * c, cap, two_cap), kLog2e, ad) : fmaf(s, c, ad);
  if (MASK) e = col > lim || col <= low ? -INFINITY : e;
  return e;
}

struct Granule {
  // the key scale, log2 of the value scale and its inverse (1 for a NaN, which
  // comes in through the exponents of the tokens that a row sees)
  float ks, lv, iv, pad;
};

template <int D, int CAP, bool MASK>
__device__ __forceinline__ float chunk_max(uint32_t ts, const Granule* info, float crow, float cap, float two_cap, int lim, int low) {
  float m = -INFINITY;
#pragma unroll 1
  for (int ch = 0; ch < Chunk<D>::COLS / 32; ++ch) {
    uint32_t s[32];
    tmem_ld32(ts + 32 * ch, s);
    tmem_wait_regs(s);
#pragma unroll
    for (int gr = 0; gr < 2; ++gr) {
      const Granule g = info[2 * ch + gr];
      const float c = crow * g.ks;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        m = fmaxf(m, chunk_exp<CAP, MASK>(__uint_as_float(s[16 * gr + i]), c, g.lv, cap, two_cap, 32 * ch + 16 * gr + i, lim, low));
    }
  }
  return m;
}

// two fp32 at once
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// P of a tile in registers (two a word) and the row's sum; over: some sum of 16
// is above kChunkTop.  The next 16 scores are on their way while 16 are worked
// on; products and sums go two at a time.
template <int D, int CAP, bool MASK>
__device__ __forceinline__ float chunk_weights(uint32_t ts, const Granule* info, float crow, float m, float cap, float two_cap,
                                               int lim, int low, uint32_t (&p)[Chunk<D>::COLS / 2], bool& over) {
  constexpr int N = Chunk<D>::COLS / 16;
  float sum = 0.0f;
  over = m == -INFINITY;
  const float mu = over ? 0.0f : m;
  uint32_t s[2][32];
  tmem_ld32(ts, s[0]);
  tmem_wait_regs(s[0]);
  tmem_ld32(ts + 32, s[1]);
  Granule all_g[N];
#pragma unroll
  for (int gr = 0; gr < N; ++gr) all_g[gr] = info[gr];
#pragma unroll
  for (int gr = 0; gr < N; ++gr) {
    if (gr == 2) tmem_wait_regs(s[1]);
    const uint32_t* x = s[gr >> 1] + 16 * (gr & 1);
    const Granule g = all_g[gr];
    const float c = crow * g.ks, ad = g.lv - mu;
    uint64_t part[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const int col = 16 * gr + i;
      const float s0 = __uint_as_float(x[i]), s1 = __uint_as_float(x[i + 1]);
      float e0, e1;
      if (CAP || MASK) {
        e0 = chunk_exp<CAP, MASK>(s0, c, ad, cap, two_cap, col, lim, low);
        e1 = chunk_exp<CAP, MASK>(s1, c, ad, cap, two_cap, col + 1, lim, low);
      } else {
        unpack2(fma2(pack2(s0, s1), pack2(c, c), pack2(ad, ad)), e0, e1);
      }
      e0 = ex2(e0);
      e1 = ex2(e1);
      part[(i >> 1) & 1] = add2(part[(i >> 1) & 1], pack2(e0, e1));
      p[col / 2] = pack_f16x2(e0, e1);
    }
    float lo, hi;
    unpack2(add2(part[0], part[1]), lo, hi);
    const float all = lo + hi;
    over |= all > kChunkTop;
    sum = fmaf(all, g.iv, sum);
  }
  return sum;
}

// A vote of the two warps that share rows (D = 256): how many of their lanes say
// so.  The barrier is met by both or by none: a warp whose wait for a tile runs
// out comes to the vote that would have been its next one with all lanes, the
// others never have more than one, and both stop after it.  (After each of those
// waits there is another vote, and both warps have the same votes in the same order.)
constexpr uint32_t kPairLeave = 32;
__device__ __forceinline__ uint32_t pair_vote(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %2, 0;\n\t"
      "barrier.cta.red.popc.u32 %0, %1, 64, p;\n\t}"
      : "=r"(r)
      : "r"(id), "r"((uint32_t)v)
      : "memory");
  return r;
}

// 16 query elements a step to fp16, in the row's power of two, to swizzled shared memory
__device__ __forceinline__ void store_query(uint32_t sq, int row, int c8, const uint4& v, float down) {
  st_shared_v4(sq + (c8 >> 3) * 128 * 128 + (((c8 & 7) ^ (row & 7)) << 4),
               make_uint4(pack_f16x2(bf16_lo(v.x) * down, bf16_hi(v.x) * down), pack_f16x2(bf16_lo(v.y) * down, bf16_hi(v.y) * down),
                          pack_f16x2(bf16_lo(v.z) * down, bf16_hi(v.z) * down), pack_f16x2(bf16_lo(v.w) * down, bf16_hi(v.w) * down)));
}

// Fail closed: no row of the call can be read as an answer.  Threads i0, i0 + step, ..
template <int D>
__device__ __forceinline__ void chunk_fail(const KvAttnArgs& a, long long i0, long long step) {
  const long long vecs = (long long)a.n_rows * a.H * (D / 8);
  for (long long i = i0; i < vecs; i += step) {
    const long long row = i / (a.H * (D / 8));
    *reinterpret_cast<uint4*>(a.out + row * a.out_stride + (i - row * a.H * (D / 8)) * 8) =
        make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
  }
  if (a.lse != nullptr)
    for (long long i = i0; i < (long long)a.n_rows * a.H; i += step) a.lse[i] = kv_nan();
}

template <int D, int FMT, int CAP>
__global__ void __launch_bounds__(kChunkThreads, 1) kv_chunk_kernel(KvAttnArgs a) {
  using C = Chunk<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bar[40];  // the last: nobody arrives there (KvAttnArgs::stall)
  __shared__ __align__(16) Granule s_info[2 * C::ST][C::NG];
  __shared__ float s_pair[C::NQ == 1 ? 3 : 1][2][128];  // of two warps that share rows: query maximum, reference, sum
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ unsigned s_lo, s_hi;  // bits of the least and the greatest value scale of the CTA's tiles
  uint8_t* sQ = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* sK = sQ + C::NQ * C::QBYTES;
  uint8_t* sV = sK + C::ST * C::KBYTES;
  const int rank = cluster_ctarank(), run = blockIdx.x >> 1;
  // of each stage: keys full and empty, values full and empty
  uint64_t *kfull = s_bar, *kempty = s_bar + C::ST, *vfull = s_bar + 2 * C::ST, *vempty = s_bar + 3 * C::ST;
  // of each row tile and S: scores, weights and product done; of each row tile:
  // queries there, O free, a part's last product done
  uint64_t *sfull = s_bar + 16, *pfull = s_bar + 20, *ofull = s_bar + 24;
  uint64_t *qfull = s_bar + 28, *ofree = s_bar + 30, *olast = s_bar + 32, *drain = s_bar + 34, *never = s_bar + 39;
  // What the MMA warps wait for (kfull, vfull, qfull, pfull, ofree) is counted at
  // the first CTA of a pair, for both; what they signal arrives at both.  Weights
  // and outputs are in TMEM: tcgen05 fences order them.  Queries, keys and values
  // are ordinary stores to a CTA's own memory.  Those of the second CTA are counted
  // there, and its MMA warps, which issue nothing, pass the count on with a release
  // for the cluster: one fence a stage by a warp with nothing else under way.  (A
  // release by each storing warp waits for its loads ahead: 987 us for 4,096 rows on
  // 32,768 tokens.)
  const uint32_t lead_pfull = mapa_shared(smem_u32(pfull), 0), lead_ofree = lead_pfull + 10 * 8;
  volatile int* abort_flag = &s_abort;
  const KvCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    const int soft = C::NQ == 2 ? 8 : 16;  // warps of a row tile
    for (int i = 0; i < C::ST; ++i) {
      mbar_init(kfull + i, C::KTASKS + (rank == 0));
      mbar_init(kempty + i, C::NQ);
      mbar_init(vfull + i, C::VTASKS + (rank == 0));
      mbar_init(vempty + i, C::NQ);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(sfull + i, 1);
      mbar_init(pfull + i, soft);
      mbar_init(ofull + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(qfull + i, soft / 2 + (rank == 0));
      mbar_init(ofree + i, soft);
      mbar_init(olast + i, 1);
      mbar_init(drain + i, 1);
    }
    mbar_init(never, 1);
    mbar_fence_init();
    s_abort = 0;
    s_lo = 0x7f800000u;
    s_hi = 0;
  }
  if (warp == C::MMA) {
    tmem_alloc_pair(&s_tmem, 512);
    tmem_relinquish_pair();
  }
  grid_wait();
  grid_release();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // also: both CTAs' barriers are there before any arrival from the other
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const bool ok = a.plan[1] != 0;
  if (!ok) chunk_fail<D>(a, (long long)blockIdx.x * kChunkThreads + tid, (long long)gridDim.x * kChunkThreads);
  __syncthreads();  // every warp whole again before the register split
  PartWalk walk;
  walk.u = walk.end = 0;
  if (ok && a.plan[0] > 0 && run < a.plan[2]) walk.init(a, run);
  Part part;

  if (warp < C::SOFT) {
    // ------------------------------------------------------------------ softmax
    set_regs<kSoftRegs, true>();
    // a row a thread; D = 256: two threads, each half of the columns
    const int q = C::NQ == 2 ? warp >> 2 : 0, half = C::NQ == 2 ? 0 : warp >> 2;
    const int tr = tid & 127;  // row in the row tile
    const int pair = 1 + (warp & 3);
    const int lr = q * C::TROWS + rank * 128;  // the CTA's first row of the row tile, in the item's
    constexpr int kTopAt = C::NQ == 1 ? 1 : 0, kSumAt = C::NQ == 1 ? 2 : 0;
    // a vote (D = 256): whether any lane says so, or kPairLeave
    auto vote = [&](bool v) { return pair_vote(pair, __any_sync(0xffffffffu, v) && lane == 0); };
    // a wait that runs out comes to the next vote with all lanes
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      const bool there = mbar_wait_warp(bar, parity & 1, abort_flag, a.wait_limit);
      if (C::NQ == 1 && !there) pair_vote(pair, true);
      return there;
    };
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float two_cap = CAP ? 2.0f * kLog2e / a.softcap : 0.0f;
    uint32_t kv = 0, ns = 0, parts = 0;  // token tiles before the part's; S tiles and parts of this row tile
    bool go = true, pending = false;  // pending: a part whose output is still in TMEM
    const uint32_t to = tmem + C::TO + q * D + lanes;
    // of the part in work, kept beyond the next one's queries
    int n = 0, slot = 0, qh = 0;
    long long row = 0;
    bool valid = false, split = false;
    float crow = 0.0f, m = -INFINITY, l = 0.0f;
#pragma unroll 1
    while (true) {
      bool have = false;
      while (walk.next(a, part)) {
        if (q > 0 && part.rows * a.G - part.row_tile * C::ROWS <= C::TROWS) {  // no second row tile
          kv += part.last - part.first;
          continue;
        }
        have = true;
        break;
      }
      const int rows = part.rows * a.G, r = part.row_tile * C::ROWS + lr + tr;
      const bool nvalid = have && r < rows;
      const int qi = nvalid ? r / a.G : part.rows - 1, nqh = part.h * a.G + (nvalid ? r - qi * a.G : 0);
      const long long nrow = part.row0 + qi;
      float ncrow = 0.0f;
      if (have) {
        // the query row (its half) in fp16's range.  The scores of the part before
        // have all been computed: its output is read after this, while the tensor
        // core begins with the new rows.
        constexpr int QV = D / 8 / (C::NQ == 2 ? 1 : 2);
        const uint4* src = reinterpret_cast<const uint4*>(a.q + nrow * a.q_stride + (size_t)nqh * D) + half * QV;
        uint4 v[QV];
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < QV; ++i) v[i] = nvalid ? src[i] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < QV; ++i) {
          const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) amax = max(amax, max((x[k] << 16) & 0x7fffffffu, x[k] & 0x7fff0000u));
        }
        if (C::NQ == 1) {
          s_pair[0][half][tr] = __uint_as_float(amax);
          if (vote(false) >= kPairLeave) break;
          amax = max(amax, __float_as_uint(s_pair[0][half ^ 1][tr]));
        }
        const uint32_t e = kv_row_exp(amax);
        const bool finite = amax < 0x7f800000u;
        const float down = __uint_as_float((254 - e) << 23);
        ncrow = (finite ? __uint_as_float(e << 23) * a.scale : kv_nan()) * (CAP ? 1.0f : kLog2e);
        const uint32_t sq = smem_u32(sQ) + q * C::QBYTES + tr * 128;
#pragma unroll
        for (int i = 0; i < QV; ++i) store_query(sq, tr, half * QV + i, finite ? v[i] : make_uint4(0, 0, 0, 0), down);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(qfull + q);
        __syncwarp();
      }
      if (pending) {
        if (!wait(&olast[q], parts - 1)) break;
        tc_fence_after();
        if (C::NQ == 1) {
          s_pair[kSumAt][half][tr] = l;
          if (vote(false) >= kPairLeave) break;
          l = s_pair[kSumAt][0][tr] + s_pair[kSumAt][1][tr];
        }
        const float f = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
        __nv_bfloat16* dst = a.out + row * a.out_stride + (size_t)qh * D;
        float4* po = reinterpret_cast<float4*>(a.part_o) + (size_t)slot * (D / 4) * C::ROWS + lr + tr;
        constexpr int W = C::NQ == 2 ? D : D / 2;
#pragma unroll 1
        for (int d = half * W; d < (half + 1) * W; d += 32) {
          uint32_t o[32];
          tmem_ld32(to + d, o);
          tmem_wait_regs(o);
          if (valid && split) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              po[(size_t)(d / 4 + i) * C::ROWS] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                              __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
          } else if (valid) {
            uint32_t v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = pack_bf16x2(__uint_as_float(o[2 * i]) * f, __uint_as_float(o[2 * i + 1]) * f);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<uint4*>(dst + d + 8 * i) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
          __syncwarp();  // whole again before the next load from TMEM
        }
        __syncwarp();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed(lead_ofree + 8 * q);
        __syncwarp();
        if (valid && half == 0) {
          if (split) {
            a.part_ml[(size_t)slot * 2 * C::ROWS + lr + tr] = m;
            a.part_ml[(size_t)slot * 2 * C::ROWS + C::ROWS + lr + tr] = l;
          } else if (a.lse != nullptr) {
            a.lse[row * a.H + qh] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
          }
        }
        __syncwarp();
      }
      if (!have) break;
      pending = true;
      ++parts;
      n = part.last - part.first;
      row = nrow;
      qh = nqh;
      valid = nvalid;
      crow = ncrow;
      split = part.first > 0 || part.last < part.tiles;
      slot = 2 * run + (part.first > 0 ? 0 : 1);
      m = -INFINITY;
      l = 0.0f;
      if (a.stall == kKvStallSoftmax && blockIdx.x == 0 && warp == 0 && !wait(never, 0)) break;
      const int see = part.held - part.rows + qi;
      // tiles that every row of this row tile sees whole
      const int r_end = min(rows, part.row_tile * C::ROWS + lr + 128) - 1;
      const int see_lo = part.held - part.rows + (part.row_tile * C::ROWS + lr) / a.G;
      const int see_hi = part.held - part.rows + r_end / a.G;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const uint32_t mine = ns++;
        const int buf = 2 * q + (mine & 1);
        go = wait(&sfull[buf], mine >> 1);
        if (!go) break;
        tc_fence_after();
        const Granule* info = s_info[(kv + j) & (2 * C::ST - 1)] + half * (C::COLS / 16);
        const int tok0 = (part.tile0 + part.first + j) * C::NT + half * C::COLS;
        const uint32_t ts = tmem + buf * C::NT + lanes;
        const bool mask = tok0 + C::COLS - 1 > see_lo || (a.window > 0 && tok0 <= see_hi - a.window);
        const int lim = see - tok0, low = a.window > 0 ? lim - a.window : -1;
        uint32_t p[C::COLS / 2];
        float sum;
#pragma unroll 1
        for (int pass = j == 0;; ++pass) {
          if (pass == 1) {  // move the reference
            float top = fmaxf(m, chunk_max<D, CAP, true>(ts + half * C::COLS, info, crow, a.softcap, two_cap, lim, low));
            if (C::NQ == 1) {
              s_pair[kTopAt][half][tr] = top;
              go = vote(false) < kPairLeave;
              if (!go) break;
              top = fmaxf(top, s_pair[kTopAt][half ^ 1][tr]);
            }
            if (j > 0) {
              // the output so far, once the last product is in it
              const uint32_t last = mine - 1;
              go = wait(&ofull[2 * q + (last & 1)], last >> 1);
              if (!go) break;
              tc_fence_after();
              const float f = top == -INFINITY ? 1.0f : ex2(m - top);
              l *= f;
              constexpr int W = C::NQ == 2 ? D : D / 2;
#pragma unroll 1
              for (int d = half * W; d < (half + 1) * W; d += 32) {
                uint32_t o[32];
                tmem_ld32(to + d, o);
                tmem_wait_regs(o);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tmem_st32(to + d, o);
              }
              tmem_st_wait();
            }
            m = top;
          }
          bool over;
          // caps above kSmallCap are rare: one form of the loop (their kernel of both crashed ptxas on an Arm host)
          sum = CAP == 2 || mask
                    ? chunk_weights<D, CAP, true>(ts + half * C::COLS, info, crow, m, a.softcap, two_cap, lim, low, p, over)
                    : chunk_weights<D, CAP, false>(ts + half * C::COLS, info, crow, m, a.softcap, two_cap, lim, low, p, over);
          over = over && pass == 0;
          // both warps of a pair are through with S here: P goes over it
          const uint32_t again = C::NQ == 1 ? vote(over) : __any_sync(0xffffffffu, over);
          go = C::NQ == 2 || again < kPairLeave;
          if (!go || again == 0) break;
        }
        if (!go) break;
        l += sum;
        tmem_st32(ts + half * (C::COLS / 2), p);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed(lead_pfull + 8 * buf);
        __syncwarp();
      }
      kv += n;
      if (!go) break;
    }
  } else {
  set_regs<kConvRegs, false>();  // one instruction for the whole warpgroup
  if (warp >= C::MMA) {
    // -------------------------------------------- MMA issuers, one of each row tile
    // Issue runs only three or four products ahead of the tensor core, so what a
    // warp does between them (waits, addresses) shows unless the other's fill it.
    // A tile's scores are issued before the weights of the one before are waited for.
    const int q = warp - C::MMA;
    const uint32_t desc_hi = (uint32_t)(sw128_desc(0) >> 32);
    const uint32_t q_lo = uniform((uint32_t)sw128_desc(smem_u32(sQ)) + q * (C::QBYTES >> 4));
    const uint32_t k_lo = uniform((uint32_t)sw128_desc(smem_u32(sK)));
    // columns contiguous: a panel's rows, panels NT rows apart; groups of 8 rows;
    // descriptor version 1, swizzle mode 2 (128 bytes) or 4 (64)
    const uint32_t v_lo = uniform((smem_u32(sV) >> 4) | ((uint32_t)(C::NT * C::VROW) >> 4 << 16));
    constexpr uint32_t v_hi = 8 * C::VROW >> 4 | 1u << 14 | (C::VROW == 128 ? 2u : 4u) << 29;
    const uint32_t tm = uniform(tmem + q * 2 * C::NT), to = uniform(tmem + C::TO + q * D);
    constexpr uint32_t id_s = idesc_f16(C::TROWS, C::NT, 0), id_o = idesc_f16(C::TROWS, D, 1);
    uint32_t kv = 0;            // token tiles before the part's
    uint32_t parts = 0, ns = 0;  // parts begun, and S tiles begun before the part's, of this row tile
    bool go = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait_warp<true>(bar, parity & 1, abort_flag, a.wait_limit); };
    auto stage = [](uint32_t t) { return t & (C::ST - 1); };
    auto phase = [](uint32_t t) { return t / C::ST; };
    if (rank != 0) {
      // Pass the second CTA's queries (of row tile q), keys and values on.  A part's
      // first keys come before its queries; the next keys are asked for before a
      // tile's values, as the issuers do.
      auto pass = [&](uint64_t* bar, uint32_t parity) {
        go = go && mbar_wait_warp(bar, parity & 1, abort_flag, a.wait_limit);  // arrivals of this CTA
        if (go && lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(bar), 0));
        __syncwarp();
      };
      while (go && walk.next(a, part)) {
        const uint32_t n = part.last - part.first;
        if (q == 0) pass(&kfull[stage(kv)], phase(kv));
        if (q == 0 || part.rows * a.G - part.row_tile * C::ROWS > C::TROWS) pass(&qfull[q], parts++);
        for (uint32_t t = kv; go && t < kv + n; ++t) {
          if (q == 0 && t + 1 < kv + n) pass(&kfull[stage(t + 1)], phase(t + 1));
          if (q == C::NQ - 1) pass(&vfull[stage(t)], phase(t));
        }
        kv += n;
      }
    }
    Part ahead;  // read a part early: its loads take as long as a tile
    bool more = rank == 0 && walk.next(a, ahead);  // the first CTA of a pair issues for both
    while (go && __any_sync(0xffffffffu, more)) {
      part = ahead;
      more = walk.next(a, ahead);
      if (a.stall == kKvStallMma && blockIdx.x == 0 && q == 0) {
        go = wait(never, 0);
        if (!go) break;
      }
      const uint32_t n = uniform(part.last - part.first), t0 = uniform(kv), n0 = uniform(ns);
      kv += n;
      if (q > 0 && (int)uniform(part.rows * a.G - part.row_tile * C::ROWS) <= C::TROWS) {  // no second row tile
        for (uint32_t t = t0; go && t < t0 + n; ++t) {
          go = wait(&kfull[stage(t)], phase(t));
          if (go && elect_one()) umma_commit_pair(&kempty[stage(t)]);
          __syncwarp();
          go = go && wait(&vfull[stage(t)], phase(t));
          if (go && elect_one()) umma_commit_pair(&vempty[stage(t)]);
          __syncwarp();
        }
        continue;
      }
      auto scores = [&](uint32_t j) {
        const uint32_t st = uniform(stage(t0 + j)), buf = uniform((n0 + j) & 1);
        go = go && wait(&kfull[st], phase(t0 + j));
        if (!go) return;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            umma_bf16_pair(
                tm + buf * C::NT, desc64(q_lo + (((k >> 2) * 128 * 128 + (k & 3) * 32) >> 4), desc_hi),
                desc64(k_lo + ((st * C::KBYTES + (k >> 2) * C::KROWS * 128 + (k & 3) * 32) >> 4), desc_hi), id_s, k != 0);
          umma_commit_pair(&sfull[2 * q + buf]);
          umma_commit_pair(&kempty[st]);
        }
        __syncwarp();
      };
      go = wait(&qfull[q], parts);
      scores(0);
      go = go && wait(&ofree[q], parts ^ 1);
      for (uint32_t j = 0; go && j < n; ++j) {
        if (j + 1 < n) scores(j + 1);
        const uint32_t st = uniform(stage(t0 + j)), buf = uniform((n0 + j) & 1);
        go = go && wait(&vfull[st], phase(t0 + j)) && wait(&pfull[2 * q + buf], (n0 + j) >> 1);
        if (!go) break;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < C::NT / 16; ++k)
            umma_f16_ts_pair(
                to, tm + buf * C::NT + 8 * k, desc64(v_lo + ((st * C::KBYTES + k * 16 * C::VROW) >> 4), v_hi), id_o, (j | k) != 0);
          umma_commit_pair(&ofull[2 * q + buf]);
          if (j + 1 == n) umma_commit_pair(&olast[q]);
          umma_commit_pair(&vempty[st]);
        }
        __syncwarp();
      }
      ++parts;
      ns += n;
    }
    // every MMA this warp issued has completed before TMEM is released
    __syncwarp();
    if (rank == 0 && elect_one()) {
      umma_commit_pair(drain + q);
      const long long since = clock64();
      while (!mbar_try_wait(drain + q, 0) && clock64() - since < kDrainCycles) {
      }
    }
  } else {
    // --------------------------------------------------------------- conversion
    // The tasks of all token tiles in order, a tile's keys and then its values;
    // this warp takes every CONV-th.  Its waits cannot miss a phase: the task before
    // has waited for a product of at most ST + 2 tiles back, and that one came after
    // the product that freed this task's stage the time before.  A task's block is
    // looked up three turns ahead, its scales and codes are loaded two turns ahead.
    // Lanes 16 and up look up the second 16 tokens of a task of 32, and of a pair's
    // keys the 16 tokens that the other CTA converts at the same time: each CTA
    // needs the scales of all.
    struct Task {
      int n;    // in order; -1: none
      int id;   // block; -2: past the tokens held
      int off;  // the lane's first code in the block
    };
    constexpr int TASKS = C::KTASKS + C::VTASKS;
    // `width` columns a row: a lane's 16 codes of the row, and its first row
    auto col_of = [&](int width) { return width == 32 ? lane & 1 : (lane & 3) + (width == 64 ? 0 : (lane >> 4) << 2); };
    auto row_of = [&](int width) { return width == 32 ? lane >> 1 : (lane >> 2) & (width == 64 ? 7 : 3); };
    // where they go: eight lanes write two rows of one 64-column panel, no bank
    // conflicts; rows 4 apart: chunk ^ 4.  32 columns: rows of 64 bytes, swizzled in pairs
    auto to_of = [&](uint8_t* base, int width, int rows) {
      const int col = col_of(width), row = row_of(width);
      if (width == 32) return smem_u32(base) + row * 64 + ((col * 2 ^ ((row >> 1) & 3)) << 4);
      return smem_u32(base) + (col >> 2) * rows * 128 + row * 128 + (((col & 3) * 2 ^ row) << 4);
    };
    const uint32_t to_k = to_of(sK, C::KC, C::KROWS), to_v = to_of(sV, C::VCOLS, C::NT);
    const int at_k = row_of(C::KC) * D + col_of(C::KC) * 16, at_v = row_of(C::VCOLS) * D + col_of(C::VCOLS) * 16 + rank * C::VCOLS;
    const long long block_bytes = (long long)c.K * c.P * D;
    const int log_row = c.logP + (D == 64 ? 6 : D == 128 ? 7 : 8);  // codes of a block and head
    int n = 0, base = 0;                   // the walk's part: its tiles, the CTA's tiles before it
    int at = warp - C::SOFT;            // the next task to look up
    bool more = true;
    // of the part
    const int* table = nullptr;
    int tok_part = 0;                      // first token of its first tile, less the tiles before it
    auto look_up = [&]() {
      Task k = {-1, -2, 0};
      const int t = at / TASKS, idx = at % TASKS;
      while (more && t >= base + n) {
        base += n;
        n = 0;
        more = walk.next(a, part);
        if (more) {
          n = part.last - part.first;
          table = c.table + (size_t)part.seq * c.max_blocks;
          tok_part = (part.tile0 + part.first - base) * C::NT;
        }
      }
      if (!more) return k;
      const bool v = idx >= C::KTASKS;
      const int i = v ? idx - C::KTASKS : idx;
      const int tok = tok_part + t * C::NT + (v ? i * C::VT : rank * C::KROWS + i / C::SUB * 16);
      const int mine = tok + (lane < 16 ? 0 : v ? C::VT - 16 : rank == 0 ? C::KROWS : -C::KROWS);
      k.n = at;
      k.off = (part.h << log_row) + (tok & (c.P - 1)) * D + (v ? at_v : at_k + i % C::SUB * C::KC);
      // looked at when the codes are loaded: a wait for it here would cost a latency a task
      if (mine < part.held) k.id = table[mine >> c.logP];
      at += C::CONV;
      return k;
    };
    auto load = [&](const Task& k, uint4 (&x)[C::LOADS], float& ks, float& vs) {
      const int idx = k.n % TASKS;
      const bool v = idx >= C::KTASKS;
      const int id0 = __shfl_sync(0xffffffffu, k.id, 0), id1 = C::VT == 32 && v ? __shfl_sync(0xffffffffu, k.id, 16) : id0;
      const bool fine = (unsigned)k.id < (unsigned)c.n_blocks;
      ks = k.id == -2 ? 0.0f : kv_nan();  // past the tokens held: no row sees it
      vs = k.id == -2 ? 1.0f : kv_nan();
      if (!fine && k.id != -2) kv_raise(c, MSI_ERR_INVALID_ARG);
      const uint32_t z = FMT == MSI_KV_Q8 ? 0x80808080u : 0u;
      const uint8_t* codes = c.codes[v] + k.off;
      const int step = 512 / (v ? C::VCOLS : C::KC) * D;  // codes of the rows a load of the warp covers
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) {
        const bool up = C::VT == 32 && v && i >= C::LOADS / 2;
        const int id = up ? id1 : id0;
        // the second 16 tokens of a task of 32: the next rows, or those of the next block
        const uint8_t* src = codes + id * block_bytes + (up && c.P == 16 ? (i - C::LOADS / 2) * step : i * step);
        x[i] = make_uint4(z, z, z, z);
        if ((unsigned)id < (unsigned)c.n_blocks) x[i] = *reinterpret_cast<const uint4*>(src);
      }
      if (!v && idx % C::SUB == 0 && fine) {
        const size_t at = (size_t)k.id * c.K + (k.off >> log_row);
        ks = c.scale[0][at];
        vs = c.scale[1][at];
      }
    };
    Task k0 = look_up(), k1 = look_up(), k2 = look_up();
    uint4 x0[C::LOADS], x1[C::LOADS];
    float ks0, vs0, ks1, vs1;
    float lo = INFINITY, hi = 0.0f;  // value scales met
    load(k0, x0, ks0, vs0);
    load(k1, x1, ks1, vs1);
    auto turn = [&](const Task& k, uint4 (&x)[C::LOADS], float ks, float vs) {
      const uint32_t t = k.n / TASKS, idx = k.n % TASKS, st = t & (C::ST - 1), ph = ((t / C::ST) & 1) ^ 1, v = idx >= C::KTASKS;
      const int i = v ? idx - C::KTASKS : idx;
      // s_bar: full and empty barriers of keys, then of values
      if (!mbar_wait_warp(kempty + v * 2 * C::ST + st, ph, abort_flag, a.wait_limit)) return false;
      const uint32_t tile = st * C::KBYTES + (v ? to_v + i * C::VT * C::VROW : to_k + i / C::SUB * 16 * 128 + i % C::SUB * (C::KC / 64) * C::KROWS * 128);
      // the swizzle: chunk ^ (row & 7), the row being its first + a multiple of 4, of
      // 8, or (32 columns, where it has a period of 8) of 16
      const bool four = (v ? C::VCOLS : C::KC) == 128;
      const uint32_t step = four ? 512 : 1024, flip = four ? 64 : 0;
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) {
        const uint32_t to = (i & 1 ? tile ^ flip : tile) + i * step;
        st_shared_v4(to, make_uint4(kv_f16x2<FMT, false>(x[i].x), kv_f16x2<FMT, true>(x[i].x), kv_f16x2<FMT, false>(x[i].y), kv_f16x2<FMT, true>(x[i].y)));
        st_shared_v4(to ^ 16, make_uint4(kv_f16x2<FMT, false>(x[i].z), kv_f16x2<FMT, true>(x[i].z), kv_f16x2<FMT, false>(x[i].w), kv_f16x2<FMT, true>(x[i].w)));
      }
      if (!v && i % C::SUB == 0 && ks != 0.0f) lo = fminf(lo, vs), hi = fmaxf(hi, vs);  // of the numbers
      // the granules' scales: read by softmax after the scores, which follow kfull
      if (!v && i % C::SUB == 0 && (lane & 15) == 0) {
        const int g = i / C::SUB + (rank ^ (lane >> 4)) * (C::KROWS / 16);
        s_info[t & (2 * C::ST - 1)][g] = Granule{ks, lg2(vs), vs > 0.0f ? __fdividef(1.0f, vs) : 1.0f, 0.0f};
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(kfull + v * 2 * C::ST + st);
      return true;
    };
    const bool stall = a.stall == kKvStallConversion && blockIdx.x == 0 && warp == C::SOFT;
    while (k0.n >= 0) {
      if (stall && !mbar_wait_warp(never, 0, abort_flag, a.wait_limit)) break;
      if (!turn(k0, x0, ks0, vs0)) break;
      k0 = k2;
      load(k0, x0, ks0, vs0);
      k2 = look_up();
      if (k1.n < 0 || !turn(k1, x1, ks1, vs1)) break;
      k1 = k2;
      load(k1, x1, ks1, vs1);
      k2 = look_up();
    }
    __syncwarp();
    // positive numbers are ordered as their bits are
    atomicMin(&s_lo, __float_as_uint(lo));
    atomicMax(&s_hi, __float_as_uint(hi));
  }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA leaves while the other may still reach it
  tc_fence_after();
  if (warp == C::MMA) tmem_dealloc_pair(tmem, 512);
  const bool apart = __uint_as_float(s_hi) > __uint_as_float(s_lo) * kScaleRange;
  if (tid == 0 && (s_abort != 0 || apart)) {
    kv_raise(c, s_abort != 0 ? MSI_ERR_TIMEOUT : MSI_ERR_UNSUPPORTED);
    a.plan[3] = 1;
  }
}

// Joins the parts of each split item: CTA x takes the item that begins in run x
// and goes on past it, CTA y 32 of its rows.
constexpr int kChunkJoinThreads = 256, kChunkJoinRows = 32;

template <int D>
__global__ void __launch_bounds__(kChunkJoinThreads) kv_chunk_join_kernel(KvAttnArgs a) {
  using C = Chunk<D>;
  grid_wait();
  grid_release();
  const KvCache& c = a.c;
  const int4 plan = *reinterpret_cast<const int4*>(a.plan);  // items, in range, CTAs, failed
  if (plan.y == 0 || plan.x == 0) return;  // every row is NaN already, or there is none
  if (plan.w != 0) {  // rows that are not split among them
    chunk_fail<D>(a, ((long long)blockIdx.y * gridDim.x + blockIdx.x) * kChunkJoinThreads + threadIdx.x,
                  (long long)gridDim.x * gridDim.y * kChunkJoinThreads);
    return;
  }
  const int ctas = plan.z;
  if ((int)blockIdx.x + 1 >= ctas) return;
  const long long total = a.item_pre[plan.x];
  const KvRuns runs = {total, ctas};
  const long long begin = runs.begin(blockIdx.x), end = runs.begin(blockIdx.x + 1);
  // the item that the next run begins with, if it has tiles in this one
  const int item = a.plan[4 + blockIdx.x + 1];
  const long long p0 = a.item_pre[item] + kItemCost, p1 = a.item_pre[item + 1];
  if (p0 < begin || p0 >= end) return;
  const int parts = runs.owner(p1 - 1) - blockIdx.x + 1;
  const int4 w = a.items[2 * item], it = a.items[2 * item + 1];
  const int tr = blockIdx.y * kChunkJoinRows + (threadIdx.x & 31), r = it.y * C::ROWS + tr;
  if (r >= w.z * a.G) return;
  const int qi = r / a.G, qh = it.x * a.G + r % a.G;
  const long long row = w.y + qi;
  const int dw = threadIdx.x >> 5;  // this warp's columns: 4 dw, + 32, ..
  const bool failed = c.control[1] != 0;
  auto slot_of = [&](int i) { return (size_t)(2 * (blockIdx.x + i) + (i == 0 ? 1 : 0)); };
  // several parts' loads on their way at once: an item of few rows and many
  // tokens has up to a part a CTA
  float top = -INFINITY, sum = 0.0f;
#pragma unroll 8
  for (int i = 0; i < parts; ++i) top = fmaxf(top, a.part_ml[slot_of(i) * 2 * C::ROWS + tr]);
  float4 acc[D / 32];
#pragma unroll
  for (int k = 0; k < D / 32; ++k) acc[k] = make_float4(0, 0, 0, 0);
  constexpr int B = D == 256 ? 2 : 4;
  for (int i0 = 0; i0 < parts; i0 += B) {
    float4 v[B][D / 32];
    float mi[B], li[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const bool there = i0 + b < parts;
      const size_t slot = slot_of(there ? i0 + b : 0);
      mi[b] = there ? a.part_ml[slot * 2 * C::ROWS + tr] : -INFINITY;
      li[b] = there ? a.part_ml[slot * 2 * C::ROWS + C::ROWS + tr] : 0.0f;
      const float4* po = reinterpret_cast<const float4*>(a.part_o) + slot * (D / 4) * C::ROWS + tr;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) v[b][k] = there ? po[(size_t)(dw + 8 * k) * C::ROWS] : make_float4(0, 0, 0, 0);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const float f = mi[b] == -INFINITY ? (li[b] == 0.0f ? 0.0f : li[b]) : ex2(mi[b] - top);
      sum += mi[b] == -INFINITY ? li[b] : kv_scaled(li[b], mi[b] - top);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        acc[k].x = fmaf(f, v[b][k].x, acc[k].x);
        acc[k].y = fmaf(f, v[b][k].y, acc[k].y);
        acc[k].z = fmaf(f, v[b][k].z, acc[k].z);
        acc[k].w = fmaf(f, v[b][k].w, acc[k].w);
      }
    }
  }
  const float f = failed ? kv_nan() : sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
    *reinterpret_cast<uint2*>(a.out + row * a.out_stride + (size_t)qh * D + 4 * (dw + 8 * k)) =
        make_uint2(pack_bf16x2(acc[k].x * f, acc[k].y * f), pack_bf16x2(acc[k].z * f, acc[k].w * f));
  if (dw == 0 && a.lse != nullptr) a.lse[row * a.H + qh] = failed ? kv_nan() : sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

template <int D, int FMT, int CAP>
cudaError_t chunk_as(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  using C = Chunk<D>;
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = smem_attr_once(kv_chunk_kernel<D, FMT, CAP>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  // few warps scan sooner: 8 sequences of 500 take 25.7 us in all, 26.6 with 1,024 threads
  const bool few = a.n <= 256 && a.max_items <= 512;
  e = launch_after(false, few ? kv_plan_kernel<256> : kv_plan_kernel<1024>, dim3(1), dim3(few ? 256 : 1024), 0, s, a, C::ROWS, C::NT);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(2 * a.ctas);
  cfg.blockDim = dim3(kChunkThreads);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kv_chunk_kernel<D, FMT, CAP>, a);
  if (e != cudaSuccess) return e;
  e = launch_after(true, kv_chunk_join_kernel<D>, dim3(a.ctas, C::ROWS / kChunkJoinRows), dim3(kChunkJoinThreads), 0, s, a);
  *launches = 3;
  return e;
}

template <int D, int FMT>
cudaError_t chunk_fmt(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  return a.softcap == 0.0f         ? chunk_as<D, FMT, 0>(a, launches, s)
         : a.softcap <= kSmallCap ? chunk_as<D, FMT, 1>(a, launches, s)
                                  : chunk_as<D, FMT, 2>(a, launches, s);
}

template <int D>
cudaError_t chunk_d(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  return a.c.fmt == MSI_KV_Q8 ? chunk_fmt<D, MSI_KV_Q8>(a, launches, s) : chunk_fmt<D, MSI_KV_E4M3>(a, launches, s);
}

}  // namespace

int kv_chunk_rows(int D) { return D == 64 ? Chunk<64>::ROWS : D == 128 ? Chunk<128>::ROWS : Chunk<256>::ROWS; }

cudaError_t launch_kv_chunk(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  return a.c.D == 64 ? chunk_d<64>(a, launches, s) : a.c.D == 128 ? chunk_d<128>(a, launches, s) : chunk_d<256>(a, launches, s);
}

}  // namespace msi
