// Attention over the 8-bit key-value cache in chunk form: many query rows of a
// sequence (a chunk of a prompt) against everything that it holds, on the
// tcgen05 tensor cores.  The mathematics is kv_decode.cu's: exact fp16 codes
// and queries, fp32 scores, the value's scale in the exponent, weights rounded
// once to fp16.
//
// An item is one sequence, key-value head and tile of 128 or 256 rows (query
// tokens times the head's query heads, so a tile reads the shared keys once).
// A CTA works on one item at a time, in tiles of NT tokens:
//   conversion warps: codes from global memory to registers a tile ahead, to
//     fp16 (two instructions a pair), to swizzled shared memory;
//   MMA warp: S = Q K^T (both from shared memory), O += P V (P from TMEM, V with
//     the columns contiguous);
//   softmax warps, a row a thread: S from TMEM, P = 2^(c s + log2 sv - M) to
//     TMEM over S.  M is a running reference: a tile is done in one pass with
//     the old M unless some sum of 16 weights passes 2^11 (a bound on each of
//     them, so no maximum is taken); only then is M moved and O rescaled.
// With two row tiles the tensor core works on one while softmax works on the
// other; D = 256 leaves TMEM for one row tile, with two S buffers.
//
// The work is the list of all token tiles of all items; each CTA takes an equal
// run, parts of split items are joined by kv_chunk_join_kernel in order.
// Every wait is bounded: on expiry the CTA gives up, drains its MMAs, frees
// TMEM and raises MSI_ERR_TIMEOUT.
#include "kv.cuh"

namespace msi {
namespace {

constexpr long long kChunkWait = 4000000000LL;  // clock64 cycles of a wait
constexpr float kChunkTop = 2048.0f;            // sums of 16 weights above it move the reference

template <int D>
struct Chunk {
  static constexpr int NQ = D == 256 ? 1 : 2;   // row tiles of 128
  static constexpr int NT = D == 256 ? 64 : 128;  // tokens of a tile
  static constexpr int ROWS = 128 * NQ;
  static constexpr int NG = NT / 16;            // 16-token granules
  static constexpr int QBYTES = 128 * D * 2;    // one row tile
  static constexpr int KBYTES = NT * D * 2;
  static constexpr int SMEM = NQ * QBYTES + 4 * KBYTES + 1024;
  static constexpr int SW = 4 * NQ, CW = 4;     // softmax and conversion warps
  static constexpr int THREADS = 32 * (SW + CW + 1);
  static constexpr int IT = NT * D / 16 / 128;  // 16-code chunks of an operand a conversion thread takes
  static constexpr int TO = 256;                // first column of O in TMEM
};

__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
}
// D[tmem] (+)= A[tmem] * B[smem], fp16
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
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

// ---------------------------------------------------------------------------
// The plan of a call: items and the prefix of their token tiles
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(KvAttnArgs a, int rows_tile, int nt) {
  __shared__ int s_scan[32], s_base[kKvMaxSeqs + 1], s_bad;
  __shared__ long long s_sum[32], s_total;
  const KvCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  grid_release();
  if (tid == 0) s_bad = 0, s_total = 0;
  __syncthreads();
  int tiles = 0;
  if (tid < a.n) {
    const KvWork w = kv_work(a, tid);
    if (!w.ok) s_bad = 1;
    else tiles = (w.rows * a.G + rows_tile - 1) / rows_tile * c.K;
  }
  const int in = block_scan(tiles, s_scan);
  s_base[tid] = in - tiles;
  if (tid == kPlanThreads - 1) s_base[kPlanThreads] = in;
  __syncthreads();
  const bool ok = s_bad == 0 && s_base[kPlanThreads] <= a.max_items;
  const int items = ok ? s_base[kPlanThreads] : 0;
  for (int i0 = 0; i0 < items; i0 += kPlanThreads) {
    const int i = i0 + tid;
    long long n = 0;
    if (i < items) {
      int lo = 0, hi = a.n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_base[mid] <= i) lo = mid; else hi = mid;
      }
      const KvWork w = kv_work(a, lo);
      const int per = (w.rows * a.G + rows_tile - 1) / rows_tile;
      const int h = (i - s_base[lo]) / per, rt = (i - s_base[lo]) % per;
      const int r1 = min(w.rows * a.G, (rt + 1) * rows_tile) - 1;
      const int see0 = w.held - w.rows + rt * rows_tile / a.G, see1 = w.held - w.rows + r1 / a.G;
      const int t0 = a.window > 0 ? max(0, see0 - a.window + 1) / nt : 0;
      n = max(1, see1 < 0 ? 0 : see1 / nt + 1 - t0);  // an item that sees nothing has a tile too
      a.items[i] = make_int4(lo, h, rt, t0);
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
    __syncthreads();
    if (tid == kPlanThreads - 1) s_total = before + n;
    __syncthreads();
  }
  if (tid == 0) {
    a.item_pre[items] = s_total;
    a.plan[0] = items;
    a.plan[1] = ok;
  }
}

// ---------------------------------------------------------------------------
// A CTA's parts: runs of token tiles of successive items
// ---------------------------------------------------------------------------
struct Part {
  int b, h, row_tile, tile0;   // of the item; tile0: its first token tile
  int first, last, tiles;      // token tiles [first, last) of the item's `tiles` are this CTA's
  KvWork w;
};

struct PartWalk {
  long long u, end;
  int item;

  __device__ __forceinline__ void init(const KvAttnArgs& a, int cta, int ctas) {
    const int items = a.plan[0];
    const long long total = a.item_pre[items];
    u = kv_begin(total, ctas, cta);
    end = kv_begin(total, ctas, cta + 1);
    int hi = items;
    item = 0;
    while (hi - item > 1) {
      const int mid = (item + hi) >> 1;
      if (a.item_pre[mid] <= u) item = mid; else hi = mid;
    }
  }
  __device__ __forceinline__ bool next(const KvAttnArgs& a, Part& p) {
    if (u >= end) return false;
    const int4 it = a.items[item];
    const long long p0 = a.item_pre[item], p1 = a.item_pre[item + 1];
    p.b = it.x;
    p.h = it.y;
    p.row_tile = it.z;
    p.tile0 = it.w;
    p.tiles = (int)(p1 - p0);
    p.first = (int)(u - p0);
    p.last = (int)(min(p1, end) - p0);
    p.w = kv_work(a, it.x);
    u = min(p1, end);
    ++item;
    return true;
  }
};

__device__ __forceinline__ int chunk_ctas(const KvAttnArgs& a) {
  return (int)min((long long)a.ctas, max(1LL, a.item_pre[a.plan[0]]));
}

// log2 weights of 16 scores: c s + ad, or its capped form, masked beyond `lim`
// and at or before `low` (columns of the granule)
template <bool CAP, bool MASK>
__device__ __forceinline__ float chunk_exp(float s, float c, float ad, float cap, float two_cap, int col, int lim, int low) {
  float e = CAP ? fmaf(kv_softcap(s * c, cap, two_cap), kLog2e, ad) : fmaf(s, c, ad);
  if (MASK) e = col > lim || col <= low ? -INFINITY : e;
  return e;
}

struct Granule {
  float ks, lv, iv, pad;  // the key scale, log2 of the value scale and its inverse
};

template <int D, bool CAP, bool MASK>
__device__ __forceinline__ float chunk_max(uint32_t ts, const Granule* info, float crow, float cap, float two_cap, int lim, int low) {
  float m = -INFINITY;
#pragma unroll 1
  for (int ch = 0; ch < Chunk<D>::NT / 32; ++ch) {
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

// P of a tile in registers (two a word) and the row's sum; over: some sum of 16
// is above kChunkTop.
template <int D, bool CAP, bool MASK>
__device__ __forceinline__ float chunk_weights(uint32_t ts, const Granule* info, float crow, float m, float cap, float two_cap,
                                               int lim, int low, uint32_t (&p)[Chunk<D>::NT / 2], bool& over) {
  float sum = 0.0f;
  over = m == -INFINITY;
  const float mu = over ? 0.0f : m;
#pragma unroll
  for (int ch = 0; ch < Chunk<D>::NT / 32; ++ch) {
    uint32_t s[32];
    tmem_ld32(ts + 32 * ch, s);
    tmem_wait_regs(s);
#pragma unroll
    for (int gr = 0; gr < 2; ++gr) {
      const Granule g = info[2 * ch + gr];
      const float c = crow * g.ks, ad = g.lv - mu;
      float part = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const int col = 32 * ch + 16 * gr + i;
        const float x = ex2(chunk_exp<CAP, MASK>(__uint_as_float(s[16 * gr + i]), c, ad, cap, two_cap, col, lim, low));
        const float y = ex2(chunk_exp<CAP, MASK>(__uint_as_float(s[16 * gr + i + 1]), c, ad, cap, two_cap, col + 1, lim, low));
        part += x;
        part += y;
        p[col / 2] = pack_f16x2(x, y);
      }
      over |= part > kChunkTop;
      // a row that sees none of a block's tokens takes nothing from its scale, a NaN least of all
      sum += part == 0.0f ? 0.0f : part * g.iv;
    }
  }
  return sum;
}

template <int D, int FMT, bool CAP>
__global__ void __launch_bounds__(Chunk<D>::THREADS, 1) kv_chunk_kernel(KvAttnArgs a) {
  using C = Chunk<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bar[32];
  __shared__ __align__(16) Granule s_info[4][C::NG];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  uint8_t* sQ = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* sK = sQ + C::NQ * C::QBYTES;
  uint8_t* sV = sK + 2 * C::KBYTES;
  uint64_t *kfull = s_bar, *kempty = s_bar + 2, *vfull = s_bar + 4, *vempty = s_bar + 6;
  uint64_t *qfull = s_bar + 8, *sfull = s_bar + 10, *pfull = s_bar + 12, *ofull = s_bar + 14, *ofree = s_bar + 16;
  uint64_t* drain = s_bar + 18;
  volatile int* abort_flag = &s_abort;
  const KvCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(kfull + i, C::CW);
      mbar_init(kempty + i, 1);
      mbar_init(vfull + i, C::CW);
      mbar_init(vempty + i, 1);
      mbar_init(qfull + i, 128);
      mbar_init(sfull + i, 1);
      mbar_init(pfull + i, 128);
      mbar_init(ofull + i, 1);
      mbar_init(ofree + i, 128);
    }
    mbar_init(drain, 1);
    mbar_fence_init();
    s_abort = 0;
  }
  if (warp == C::SW + C::CW) {
    tmem_alloc(&s_tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  grid_wait();
  grid_release();

  const int status = c.control[1];
  const bool ok = a.plan[1] != 0 && status == 0;
  if (!ok) {
    if (status == 0 && tid == 0 && blockIdx.x == 0) kv_raise(c, MSI_ERR_INVALID_ARG);
    // fail closed: no row of the call can be read as an answer
    const long long vecs = (long long)a.n_rows * a.H * (D / 8);
    for (long long i = (long long)blockIdx.x * C::THREADS + tid; i < vecs; i += (long long)gridDim.x * C::THREADS) {
      const long long row = i / (a.H * (D / 8));
      *reinterpret_cast<uint4*>(a.out + row * a.out_stride + (i - row * a.H * (D / 8)) * 8) =
          make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    }
    for (long long i = (long long)blockIdx.x * C::THREADS + tid; i < (long long)a.n_rows * a.H;
         i += (long long)gridDim.x * C::THREADS)
      if (a.lse != nullptr) a.lse[i] = kv_nan();
  }
  const int ctas = ok ? chunk_ctas(a) : 0;
  PartWalk walk;
  walk.u = walk.end = 0;
  if (ok && a.plan[0] > 0 && (int)blockIdx.x < ctas) walk.init(a, blockIdx.x, ctas);
  Part part;

  if (warp == C::SW + C::CW) {
    // --------------------------------------------------------------- MMA issuer
    const uint32_t desc_hi = (uint32_t)(sw128_desc(0) >> 32);
    const uint32_t q_lo = uniform((uint32_t)sw128_desc(smem_u32(sQ)));
    const uint32_t k_lo = uniform((uint32_t)sw128_desc(smem_u32(sK)));
    // columns contiguous: 64 of them a panel, panels NT rows of 128 bytes apart
    const uint32_t v_lo = uniform((smem_u32(sV) >> 4) | ((uint32_t)(C::NT * 128) >> 4 << 16));
    const uint32_t tm = uniform(tmem);
    constexpr uint32_t id_s = idesc_f16(128, C::NT, 0), id_o = idesc_f16(128, D, 1);
    uint32_t kv = 0;                  // token tiles before the part's
    uint32_t np[2] = {0, 0};          // P tiles waited for, per S buffer
    uint32_t parts[2] = {0, 0};       // parts begun, per row tile
    bool go = true;
    while (go && __any_sync(0xffffffffu, walk.next(a, part))) {
      const int n = (int)uniform(part.last - part.first);
      const int nq = C::NQ == 2 && (int)uniform(part.w.rows * a.G - part.row_tile * C::ROWS) > 128 ? 2 : 1;
      auto scores = [&](int q, int buf, int j, bool first_q, bool last_q) {  // S[buf] = Q[q] K(tile j)^T
        const uint32_t t = kv + j, st = t & 1;
        if (first_q && !mbar_wait_warp(&kfull[st], (t >> 1) & 1, abort_flag, kChunkWait)) return false;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t qa = q_lo + ((q * C::QBYTES + (k >> 2) * 128 * 128 + (k & 3) * 32) >> 4);
            const uint32_t kb = k_lo + ((st * C::KBYTES + (k >> 2) * C::NT * 128 + (k & 3) * 32) >> 4);
            umma_bf16(tm + buf * C::NT, desc64(qa, desc_hi), desc64(kb, desc_hi), id_s, k != 0);
          }
          umma_commit(&sfull[buf]);
          if (last_q) umma_commit(&kempty[st]);
        }
        __syncwarp();
        return true;
      };
      auto outputs = [&](int q, int buf, int j, bool first_q, bool last_q) {  // O[q] += P[buf] V(tile j)
        const uint32_t t = kv + j, st = t & 1;
        if (!mbar_wait_warp(&pfull[buf], np[buf] & 1, abort_flag, kChunkWait)) return false;
        ++np[buf];
        if (first_q && !mbar_wait_warp(&vfull[st], (t >> 1) & 1, abort_flag, kChunkWait)) return false;
        if (j == 0) {
          if (!mbar_wait_warp(&ofree[q], (parts[q] & 1) ^ 1, abort_flag, kChunkWait)) return false;
          ++parts[q];
        }
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < C::NT / 16; ++k)
            umma_f16_ts(tm + C::TO + q * D, tm + buf * C::NT + 8 * k,
                        desc64(v_lo + ((st * C::KBYTES + k * 2048) >> 4), desc_hi), id_o, (j | k) != 0);
          umma_commit(&ofull[q]);
          if (last_q) umma_commit(&vempty[st]);
        }
        __syncwarp();
        return true;
      };
      for (int q = 0; go && q < nq; ++q) {
        go = mbar_wait_warp(&qfull[q], parts[q] & 1, abort_flag, kChunkWait);
        if (C::NQ == 2) go = go && scores(q, q, 0, q == 0, q == nq - 1);
        else go = go && scores(0, kv & 1, 0, true, true);
      }
      for (int j = 0; go && j < n; ++j) {
        if (C::NQ == 2) {
          for (int q = 0; go && q < nq; ++q) {
            go = outputs(q, q, j, q == 0, q == nq - 1);
            if (go && j + 1 < n) go = scores(q, q, j + 1, q == 0, q == nq - 1);
          }
        } else {
          if (j + 1 < n) go = scores(0, (kv + j + 1) & 1, j + 1, true, true);
          go = go && outputs(0, (kv + j) & 1, j, true, true);
        }
      }
      kv += n;
    }
    // every MMA this warp issued has completed before TMEM is released
    __syncwarp();
    if (elect_one()) {
      umma_commit(drain);
      const long long t0 = clock64();
      while (!mbar_try_wait(drain, 0) && clock64() - t0 < kDrainCycles) {
      }
    }
  } else if (warp >= C::SW) {
    // --------------------------------------------------------------- conversion
    const int ct = tid - 32 * C::SW;
    constexpr int CPR = D / 16;  // 16-code chunks of a row
    const int col = ct % CPR, row0 = ct / CPR;
    constexpr int RSTEP = 128 / CPR;
    const uint32_t flip = (col >> 2) & 1;  // neighbouring panels start with different halves: no bank conflicts
    uint4 kr[C::IT], vr[C::IT];
    // lane g of a warp: block and scales of the tile's granule g
    struct Tile {
      int seq, h, tok0, held;
    };
    int n = 0, j = 0;
    Tile next_tile = {0, 0, 0, 0};
    auto advance = [&]() {  // to the next token tile; false at the end
      if (j == n) {
        if (!walk.next(a, part)) return false;
        n = part.last - part.first;
        j = 0;
        next_tile.seq = part.w.seq;
        next_tile.h = part.h;
        next_tile.held = part.w.held;
        next_tile.tok0 = (part.tile0 + part.first) * C::NT;
      } else {
        next_tile.tok0 += C::NT;
      }
      ++j;
      return true;
    };
    auto block_of = [&](const Tile& t) {
      const int tok = t.tok0 + 16 * lane;
      if (lane >= C::NG || tok >= t.held) return -1;
      const int id = c.table[(size_t)t.seq * c.max_blocks + (tok >> c.logP)];
      if (id >= 0 && id < c.n_blocks) return id;
      kv_raise(c, MSI_ERR_INVALID_ARG);
      return -2;
    };
    auto load = [&](const Tile& t, int id, int w, uint4 (&x)[C::IT]) {
      const uint4 zero = FMT == MSI_KV_Q8 ? make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < C::IT; ++i) {
        const int row = i * RSTEP + row0;
        const int blk = __shfl_sync(0xffffffffu, id, row >> 4);
        x[i] = zero;
        if (blk >= 0)
          x[i] = *reinterpret_cast<const uint4*>(c.codes[w] + (((size_t)blk * c.K + t.h) * c.P + ((t.tok0 + row) & (c.P - 1))) * D + col * 16);
      }
    };
    auto store = [&](uint32_t base, const uint4 (&x)[C::IT]) {
#pragma unroll
      for (int i = 0; i < C::IT; ++i) {
        const int row = i * RSTEP + row0;
        const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint4 o[2];
        o[0] = make_uint4(kv_f16x2<FMT, false>(u[0]), kv_f16x2<FMT, true>(u[0]), kv_f16x2<FMT, false>(u[1]), kv_f16x2<FMT, true>(u[1]));
        o[1] = make_uint4(kv_f16x2<FMT, false>(u[2]), kv_f16x2<FMT, true>(u[2]), kv_f16x2<FMT, false>(u[3]), kv_f16x2<FMT, true>(u[3]));
        const uint32_t at = base + (col >> 2) * C::NT * 128 + row * 128;
        const uint32_t ch = (col & 3) * 2, x7 = row & 7;
        st_shared_v4(at + (((ch + flip) ^ x7) << 4), flip ? o[1] : o[0]);
        st_shared_v4(at + (((ch + (flip ^ 1)) ^ x7) << 4), flip ? o[0] : o[1]);
      }
    };
    auto scale_of = [&](const Tile& t, int id, int w) {
      return id >= 0 ? c.scale[w][(size_t)id * c.K + t.h] : id == -1 ? 1.0f : kv_nan();
    };
    uint32_t t = 0;
    bool more = advance();
    Tile cur = next_tile;
    int id = more ? block_of(cur) : -1;
    float ks = 1.0f, vs = 1.0f;
    if (more) {
      ks = scale_of(cur, id, 0);
      vs = scale_of(cur, id, 1);
      load(cur, id, 0, kr);
      load(cur, id, 1, vr);
    }
    while (more) {
      const uint32_t st = t & 1, ph = ((t >> 1) & 1) ^ 1;
      const bool again = advance();
      const Tile nxt = next_tile;
      const int nid = again ? block_of(nxt) : -1;
      if (!mbar_wait_warp(&kempty[st], ph, abort_flag, kChunkWait)) break;
      store(smem_u32(sK) + st * C::KBYTES, kr);
      if (ct < C::NG) s_info[t & 3][ct] = Granule{ks, log2f(vs), 1.0f / vs, 0.0f};
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&kfull[st]);
      if (again) {
        ks = scale_of(nxt, nid, 0);
        vs = scale_of(nxt, nid, 1);
        load(nxt, nid, 0, kr);
      }
      if (!mbar_wait_warp(&vempty[st], ph, abort_flag, kChunkWait)) break;
      store(smem_u32(sV) + st * C::KBYTES, vr);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&vfull[st]);
      if (again) load(nxt, nid, 1, vr);
      more = again;
      ++t;
    }
  } else {
    // ------------------------------------------------------------------ softmax
    const int q = warp >> 2, tr = tid & 127;  // row tile, row in it
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float two_cap = CAP ? 2.0f * kLog2e / a.softcap : 0.0f;
    uint32_t kv = 0, ns[2] = {0, 0}, no = 0;  // token tiles before the part's; S waited for; PVs of this row tile
    bool go = true;
    while (go && walk.next(a, part)) {
      const int n = part.last - part.first;
      const int rows = part.w.rows * a.G;
      if (q > 0 && rows - part.row_tile * C::ROWS <= 128) {  // no second row tile
        kv += n;
        continue;
      }
      const int r = part.row_tile * C::ROWS + q * 128 + tr;
      const bool valid = r < rows;
      const int qi = valid ? r / a.G : part.w.rows - 1, qh = part.h * a.G + (valid ? r - qi * a.G : 0);
      const int see = part.w.held - part.w.rows + qi;
      const long long row = part.w.row0 + qi;
      // the query row in fp16's range (the scores of the part before have all been computed)
      const uint4* src = reinterpret_cast<const uint4*>(a.q + row * a.q_stride + (size_t)qh * D);
      uint32_t amax = 0;
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        const uint4 v = valid ? src[i] : make_uint4(0, 0, 0, 0);
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) amax = max(amax, max((x[k] << 16) & 0x7fffffffu, x[k] & 0x7fff0000u));
      }
      const uint32_t e = kv_row_exp(amax);
      const bool finite = amax < 0x7f800000u;
      const float down = __uint_as_float((254 - e) << 23);
      const float crow = (finite ? __uint_as_float(e << 23) * a.scale : kv_nan()) * (CAP ? 1.0f : kLog2e);
      const uint32_t sq = smem_u32(sQ) + q * C::QBYTES + tr * 128;
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        const uint4 v = valid && finite ? src[i] : make_uint4(0, 0, 0, 0);
        st_shared_v4(sq + (i >> 3) * 128 * 128 + (((i & 7) ^ (tr & 7)) << 4),
                     make_uint4(pack_f16x2(bf16_lo(v.x) * down, bf16_hi(v.x) * down), pack_f16x2(bf16_lo(v.y) * down, bf16_hi(v.y) * down),
                                pack_f16x2(bf16_lo(v.z) * down, bf16_hi(v.z) * down), pack_f16x2(bf16_lo(v.w) * down, bf16_hi(v.w) * down)));
      }
      fence_proxy_async_smem();
      mbar_arrive(&qfull[q]);

      const uint32_t to = tmem + C::TO + q * D + lanes;
      float m = -INFINITY, l = 0.0f;
      // tiles that every row of this row tile sees whole
      const int r_end = min(rows, part.row_tile * C::ROWS + q * 128 + 128) - 1;
      const int see_lo = part.w.held - part.w.rows + (part.row_tile * C::ROWS + q * 128) / a.G;
      const int see_hi = part.w.held - part.w.rows + r_end / a.G;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int buf = C::NQ == 2 ? q : (kv + j) & 1;
        go = mbar_wait_warp(&sfull[buf], ns[buf] & 1, abort_flag, kChunkWait);
        if (!go) break;
        ++ns[buf];
        tc_fence_after();
        const Granule* info = s_info[(kv + j) & 3];
        const int tok0 = (part.tile0 + part.first + j) * C::NT;
        const uint32_t ts = tmem + buf * C::NT + lanes;
        const bool mask = tok0 + C::NT - 1 > see_lo || (a.window > 0 && tok0 <= see_hi - a.window);
        const int lim = see - tok0, low = a.window > 0 ? lim - a.window : -1;
        uint32_t p[C::NT / 2];
        float sum = 0.0f;
        bool over = true;
        if (j > 0) {
          sum = mask ? chunk_weights<D, CAP, true>(ts, info, crow, m, a.softcap, two_cap, lim, low, p, over)
                     : chunk_weights<D, CAP, false>(ts, info, crow, m, a.softcap, two_cap, lim, low, p, over);
        }
        if (__any_sync(0xffffffffu, over)) {
          const float top = fmaxf(m, chunk_max<D, CAP, true>(ts, info, crow, a.softcap, two_cap, lim, low));
          if (j > 0) {
            // the output so far, once the last product is in it (with two row
            // tiles the scores of this tile came after it)
            if (C::NQ == 1) {
              go = mbar_wait_warp(&ofull[0], (no - 1) & 1, abort_flag, kChunkWait);
              if (!go) break;
              tc_fence_after();
            }
            const float f = top == -INFINITY ? 1.0f : ex2(m - top);
            l *= f;
#pragma unroll 1
            for (int d = 0; d < D; d += 32) {
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
          sum = chunk_weights<D, CAP, true>(ts, info, crow, m, a.softcap, two_cap, lim, low, p, over);
        }
        l += sum;
#pragma unroll
        for (int i = 0; i < C::NT / 2; i += 32) tmem_st32(ts + i, p + i);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&pfull[buf]);
        ++no;
      }
      kv += n;
      if (!go) break;
      go = mbar_wait_warp(&ofull[q], (no - 1) & 1, abort_flag, kChunkWait);
      if (!go) break;
      tc_fence_after();
      const bool split = part.first > 0 || part.last < part.tiles;
      const float f = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
      const int slot = 2 * blockIdx.x + (part.first > 0 ? 0 : 1);
      __nv_bfloat16* dst = a.out + row * a.out_stride + (size_t)qh * D;
      float4* po = reinterpret_cast<float4*>(a.part_o) + (size_t)slot * (D / 4) * C::ROWS + q * 128 + tr;
#pragma unroll 1
      for (int d = 0; d < D; d += 32) {
        uint32_t o[32];
        tmem_ld32(to + d, o);
        tmem_wait_regs(o);
        if (!valid) continue;
        if (split) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            po[(size_t)(d / 4 + i) * C::ROWS] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                            __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
        } else {
          uint32_t v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = pack_bf16x2(__uint_as_float(o[2 * i]) * f, __uint_as_float(o[2 * i + 1]) * f);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(dst + d + 8 * i) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
      }
      tc_fence_before();
      mbar_arrive(&ofree[q]);
      if (valid) {
        if (split) {
          a.part_ml[(size_t)slot * 2 * C::ROWS + q * 128 + tr] = m;
          a.part_ml[(size_t)slot * 2 * C::ROWS + C::ROWS + q * 128 + tr] = l;
        } else if (a.lse != nullptr) {
          a.lse[row * a.H + qh] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
        }
      }
      __syncwarp();
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == C::SW + C::CW) tmem_dealloc(tmem, 512);
  if (tid == 0 && s_abort != 0) kv_raise(c, MSI_ERR_TIMEOUT);
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
  if (a.plan[1] == 0 || a.plan[0] == 0) return;  // every row is NaN already, or there is none
  const int ctas = chunk_ctas(a);
  if ((int)blockIdx.x >= ctas) return;
  const long long total = a.item_pre[a.plan[0]];
  const long long begin = kv_begin(total, ctas, blockIdx.x), end = kv_begin(total, ctas, blockIdx.x + 1);
  int item = 0, hi = a.plan[0];
  while (hi - item > 1) {
    const int mid = (item + hi) >> 1;
    if (a.item_pre[mid] <= end - 1) item = mid; else hi = mid;
  }
  const long long p0 = a.item_pre[item], p1 = a.item_pre[item + 1];
  if (p0 < begin || p1 <= end) return;
  const int parts = kv_owner(total, ctas, p1 - 1) - blockIdx.x + 1;
  const int4 it = a.items[item];
  const KvWork w = kv_work(a, it.x);
  const int tr = blockIdx.y * kChunkJoinRows + (threadIdx.x & 31), r = it.z * C::ROWS + tr;
  if (r >= w.rows * a.G) return;
  const int qi = r / a.G, qh = it.y * a.G + r % a.G;
  const long long row = w.row0 + qi;
  const int dw = threadIdx.x >> 5;  // this warp's columns: 4 dw, + 32, ..
  const bool failed = c.control[1] != 0;
  auto slot_of = [&](int i) { return (size_t)(2 * (blockIdx.x + i) + (i == 0 ? 1 : 0)); };
  float top = -INFINITY, sum = 0.0f;
  for (int i = 0; i < parts; ++i) top = fmaxf(top, a.part_ml[slot_of(i) * 2 * C::ROWS + tr]);
  float4 acc[D / 32];
#pragma unroll
  for (int k = 0; k < D / 32; ++k) acc[k] = make_float4(0, 0, 0, 0);
  for (int i = 0; i < parts; ++i) {
    const float mi = a.part_ml[slot_of(i) * 2 * C::ROWS + tr], li = a.part_ml[slot_of(i) * 2 * C::ROWS + C::ROWS + tr];
    const float f = mi == -INFINITY ? (li == 0.0f ? 0.0f : li) : ex2(mi - top);
    sum += mi == -INFINITY ? li : li * f;
    const float4* po = reinterpret_cast<const float4*>(a.part_o) + slot_of(i) * (D / 4) * C::ROWS + tr;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const float4 v = po[(size_t)(dw + 8 * k) * C::ROWS];
      acc[k].x = fmaf(f, v.x, acc[k].x);
      acc[k].y = fmaf(f, v.y, acc[k].y);
      acc[k].z = fmaf(f, v.z, acc[k].z);
      acc[k].w = fmaf(f, v.w, acc[k].w);
    }
  }
  const float f = failed ? kv_nan() : sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
    *reinterpret_cast<uint2*>(a.out + row * a.out_stride + (size_t)qh * D + 4 * (dw + 8 * k)) =
        make_uint2(pack_bf16x2(acc[k].x * f, acc[k].y * f), pack_bf16x2(acc[k].z * f, acc[k].w * f));
  if (dw == 0 && a.lse != nullptr) a.lse[row * a.H + qh] = failed ? kv_nan() : sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

template <int D, int FMT, bool CAP>
cudaError_t chunk_as(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  using C = Chunk<D>;
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = smem_attr_once(kv_chunk_kernel<D, FMT, CAP>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  e = launch_after(false, kv_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a, C::ROWS, C::NT);
  if (e != cudaSuccess) return e;
  e = launch_after(true, kv_chunk_kernel<D, FMT, CAP>, dim3(a.ctas), dim3(C::THREADS), C::SMEM, s, a);
  if (e != cudaSuccess) return e;
  e = launch_after(true, kv_chunk_join_kernel<D>, dim3(a.ctas, C::ROWS / kChunkJoinRows), dim3(kChunkJoinThreads), 0, s, a);
  *launches = 3;
  return e;
}

template <int D>
cudaError_t chunk_d(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  if (a.c.fmt == MSI_KV_Q8)
    return a.softcap > 0.0f ? chunk_as<D, MSI_KV_Q8, true>(a, launches, s) : chunk_as<D, MSI_KV_Q8, false>(a, launches, s);
  return a.softcap > 0.0f ? chunk_as<D, MSI_KV_E4M3, true>(a, launches, s) : chunk_as<D, MSI_KV_E4M3, false>(a, launches, s);
}

}  // namespace

int kv_chunk_rows(int D) { return D == 256 ? 128 : 256; }

cudaError_t launch_kv_chunk(const KvAttnArgs& a, int* launches, cudaStream_t s) {
  return a.c.D == 64 ? chunk_d<64>(a, launches, s) : a.c.D == 128 ? chunk_d<128>(a, launches, s) : chunk_d<256>(a, launches, s);
}

}  // namespace msi
