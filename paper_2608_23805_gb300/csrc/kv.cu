// Key-value cache in 8 bits: append (rows rounded into their blocks), eviction
// by the attention weight received, release, read back, and the host side of
// every msi_kv_* call.  The attention itself: kv_decode.cu, kv_chunk.cu.
//
// The cache's state is on the device and changes there, so every CTA of an
// append or an eviction works out the whole batch's bookkeeping for itself (a
// scan over at most 1,024 sequences), does its part, and the last CTA to finish
// (a ticket) writes the new state: nobody reads it any more then.
#include <math.h>

#include <new>

#include "kv.cuh"

namespace msi {
namespace {

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

// One sequence's part of an append: tokens start .. end - 1 are new.
struct KvSpan {
  int seq, row0, start, end;
  int held, shift;           // tokens held before; position minus token index
  int from;                  // first position with a row in `recent`
  int had, have;             // blocks before and after
  int blocks;                // blocks that change
  bool ok, full;             // in range; more tokens than the table has place for
};

__device__ __forceinline__ KvSpan kv_span(const KvAppendArgs& a, int b) {
  const KvCache& c = a.c;
  KvSpan s;
  s.seq = kv_seq(a.seqs, b);
  s.row0 = a.cu[b];
  const int n = a.cu[b + 1] - s.row0;
  s.ok = s.seq >= 0 && s.seq < c.n_seqs && s.row0 >= 0 && n >= 0 && s.row0 <= a.n_rows - n;
  const int4 st = s.ok ? c.seq[s.seq] : make_int4(0, 0, 0, 0);
  const int cap = c.max_blocks << c.logP;
  s.held = st.x;
  s.shift = st.y - st.x;
  s.from = st.z;
  s.start = a.start == nullptr ? st.x : a.start[b];
  s.ok = s.ok && st.x >= 0 && st.x <= cap && s.start >= 0 && s.start <= st.x;
  s.full = false;
  s.end = s.start;
  s.had = s.have = s.blocks = 0;
  if (!s.ok) return s;
  s.had = (s.held + c.P - 1) >> c.logP;
  s.ok = s.had <= c.n_blocks;
  s.full = n > cap - s.start;
  if (!s.ok || s.full) return s;
  s.end = s.start + n;
  s.have = (s.end + c.P - 1) >> c.logP;
  const bool ragged = (s.start & (c.P - 1)) != 0;
  const int j0 = s.start >> c.logP;
  s.blocks = n > 0 ? ((s.end - 1) >> c.logP) - j0 + 1 : (ragged && s.start < s.held) ? 1 : 0;
  // the first block's earlier rows come from `recent`
  if (ragged && s.blocks > 0 && (j0 << c.logP) + s.shift < s.from) s.ok = false;
  return s;
}

__device__ __forceinline__ unsigned max_u16x2(unsigned x, unsigned y) {
  unsigned r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}

// Four bf16 times inv, rounded to whole numbers (ties to even) plus 128, as
// bytes: the sum with 1.5 2^23 + 128 has a spacing of 1, its low byte is the code.
__device__ __forceinline__ uint32_t round_q8(uint32_t a, uint32_t b, float inv) {
  constexpr float kMagic = 12583040.0f;
  const uint32_t r0 = __float_as_uint(__fadd_rn(__fmul_rn(bf16_lo(a), inv), kMagic));
  const uint32_t r1 = __float_as_uint(__fadd_rn(__fmul_rn(bf16_hi(a), inv), kMagic));
  const uint32_t r2 = __float_as_uint(__fadd_rn(__fmul_rn(bf16_lo(b), inv), kMagic));
  const uint32_t r3 = __float_as_uint(__fadd_rn(__fmul_rn(bf16_hi(b), inv), kMagic));
  return __byte_perm(__byte_perm(r0, r1, 0x0040), __byte_perm(r2, r3, 0x0040), 0x5410);
}

// Four bf16 times inv as e4m3 bytes.
__device__ __forceinline__ uint32_t round_e4m3(uint32_t a, uint32_t b, float inv) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__fmul_rn(bf16_hi(a), inv)), "f"(__fmul_rn(bf16_lo(a), inv)));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__fmul_rn(bf16_hi(b), inv)), "f"(__fmul_rn(bf16_lo(b), inv)));
  return (uint32_t)lo | (uint32_t)hi << 16;
}

// A block of one head, keys or values, is a task: rounded in one pass over its
// rows, which stay in registers between the maximum and the rounding.  A CTA
// takes every gridDim-th task, so that the bookkeeping is paid for once in
// several blocks.  Bound: for prompts the chain of a task (look-up, rows, maximum,
// codes, with barriers between them) beside memory (32,768 tokens of 2 heads of
// 128: 16 us, 3.2 TB/s of rows in and codes out), latency for single tokens (64
// sequences: 8 us).
constexpr int kWrongBlock = 1 << 16;  // in the ticket: CTAs that met a wrong block number, above those that are done
constexpr int append_threads(int vpt) { return vpt <= 4 ? 1024 : 512; }  // of an SM, by the registers a thread takes

template <int THREADS, int VPT>
__global__ void __launch_bounds__(THREADS, append_threads(VPT) / THREADS) kv_append_kernel(KvAppendArgs a) {
  const KvCache& c = a.c;
  __shared__ int s_scan[32];
  __shared__ unsigned s_seen[kKvMaxSeqs / 32];
  __shared__ int s_blocks[kKvMaxSeqs + 1], s_add[kKvMaxSeqs];  // changing and new blocks before each entry's
  __shared__ int s_bad, s_tot[3], s_at[2];  // s_at: the task's block in the table and in the pool
  __shared__ KvSpan s_span;
  __shared__ unsigned s_max[THREADS / 32];
  __shared__ unsigned s_last;
  const int tid = threadIdx.x;

  for (int i = tid; i < kKvMaxSeqs / 32; i += THREADS) s_seen[i] = 0;
  if (tid == 0) s_bad = 0;
  const int n_free = c.control[0];
  const int status = c.control[1];
  __syncthreads();

  // the batch's bookkeeping: a run of entries a thread
  const int per = (a.n + THREADS - 1) / THREADS;
  const int b0 = min(a.n, tid * per), b1 = min(a.n, b0 + per);
  int blocks = 0, add = 0, drop = 0;
  for (int b = b0; b < b1; ++b) {
    const KvSpan s = kv_span(a, b);
    if (!s.ok || (atomicOr(&s_seen[s.seq >> 5], 1u << (s.seq & 31)) & (1u << (s.seq & 31))) != 0) {
      atomicOr(&s_bad, 1);
      continue;
    }
    if (s.full) {
      atomicOr(&s_bad, 2);
      continue;
    }
    blocks += s.blocks;
    add += max(0, s.have - s.had);  // in all at most a block for P rows and two for a sequence
    drop += max(0, s.had - s.have);
  }
  const int blocks_in = block_scan(blocks, s_scan);
  const int add_in = block_scan(add, s_scan);
  const int drop_in = block_scan(drop, s_scan);
  if (tid == THREADS - 1) s_tot[0] = blocks_in, s_tot[1] = add_in, s_tot[2] = drop_in;
  {
    int p = blocks_in - blocks, q = add_in - add;
    for (int b = b0; b < b1; ++b) {
      const KvSpan s = kv_span(a, b);
      s_blocks[b] = p;
      s_add[b] = q;
      p += s.blocks;
      q += max(0, s.have - s.had);
    }
    if (b0 < a.n && b1 == a.n) s_blocks[a.n] = p;
  }
  __syncthreads();
  const int bad = (s_bad & 1) != 0 || n_free < 0 || n_free > c.n_blocks || s_tot[2] > c.n_blocks - n_free
                      ? (int)MSI_ERR_INVALID_ARG
                  : s_bad != 0 || s_tot[1] > n_free ? (int)MSI_ERR_NOT_RESIDENT
                                                    : 0;
  const bool go = bad == 0 && status == 0;

  // A block number out of range is told to the last CTA with the ticket: the status
  // word stays as it is until every CTA has looked at it.
  int wrong = 0;
  const int tasks = go ? s_tot[0] * 2 * c.K : 0;
  for (int task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int block = task / (2 * c.K), h = (task - block * 2 * c.K) >> 1, w = task & 1;
    if (tid == 0) {
      int b = 0, hi = a.n;  // the entry whose blocks hold it
      while (hi - b > 1) {
        const int mid = (b + hi) >> 1;
        if (s_blocks[mid] <= block) b = mid; else hi = mid;
      }
      s_span = kv_span(a, b);
      const int j = (s_span.start >> c.logP) + block - s_blocks[b];
      s_at[0] = j;
      s_at[1] = j < s_span.had ? c.table[(size_t)s_span.seq * c.max_blocks + j]
                               : c.free_ids[n_free - 1 - s_add[b] - (j - s_span.had)];
    }
    __syncthreads();
    const KvSpan s = s_span;
    const int j = s_at[0], id = s_at[1];
    const bool id_ok = id >= 0 && id < c.n_blocks;
    const __nv_bfloat16* x = a.x[w] + (size_t)h * c.D;
    __nv_bfloat16* ring = c.recent + (((size_t)s.seq * 2 + w) * c.K + h) * (size_t)(2 * c.P) * c.D;
    const int log_vpr = c.D == 64 ? 3 : c.D == 128 ? 4 : 5, vpr = 1 << log_vpr;  // 16-byte vectors a row
    const int mask2 = 2 * c.P - 1;
    uint4 v[VPT];
    const int dc0 = (tid & (vpr - 1)) * 8, o0 = tid >> log_vpr, ostep = THREADS >> log_vpr;  // a thread keeps its columns
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int tok = (j << c.logP) + o0 + i * ostep;
      v[i] = make_uint4(0, 0, 0, 0);
      if (tok < s.start)
        v[i] = *reinterpret_cast<const uint4*>(ring + (size_t)((tok + s.shift) & mask2) * c.D + dc0);
      else if (tok < s.end)
        v[i] = *reinterpret_cast<const uint4*>(x + (size_t)(s.row0 + tok - s.start) * a.stride + dc0);
    }
    unsigned both = 0;  // as whole numbers, two at a time: an infinity or NaN is above every number
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      both = max_u16x2(both, max_u16x2(v[i].x & 0x7fff7fffu, v[i].y & 0x7fff7fffu));
      both = max_u16x2(both, max_u16x2(v[i].z & 0x7fff7fffu, v[i].w & 0x7fff7fffu));
    }
    unsigned amax = __reduce_max_sync(0xffffffffu, max(both << 16, both & 0xffff0000u));
    if ((tid & 31) == 0) s_max[tid >> 5] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) amax = max(amax, s_max[i]);
    const bool finite = amax < 0x7f800000u;
    const float top = c.fmt == MSI_KV_Q8 ? 127.0f : 448.0f;
    const float am = fmaxf(__uint_as_float(amax), kKvTiny);
    const float inv = __fdiv_rn(top, am);
    const float scale = __fmul_rn(am, c.fmt == MSI_KV_Q8 ? 1.0f / 127.0f : 1.0f / 448.0f);
    if (id_ok) {
      uint8_t* dst = c.codes[w] + ((size_t)id * c.K + h) * (size_t)c.P * c.D + o0 * c.D + dc0;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const uint4 q = finite ? v[i] : make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint2*>(dst + (size_t)i * ostep * c.D) =
            c.fmt == MSI_KV_Q8 ? make_uint2(round_q8(q.x, q.y, inv), round_q8(q.z, q.w, inv))
                               : make_uint2(round_e4m3(q.x, q.y, inv), round_e4m3(q.z, q.w, inv));
      }
      if (tid == 0) c.scale[w][(size_t)id * c.K + h] = finite ? scale : kv_nan();
    } else {
      wrong = kWrongBlock;
    }
    if (tid == 0 && j >= s.had && h == 0 && w == 0) {
      c.table[(size_t)s.seq * c.max_blocks + j] = id;  // a wrong one too: what reads it finds it so
      if (id_ok) c.weight[id] = 0.0f;
    }

    // the last two blocks' new rows into `recent`.  The ring has two blocks: a
    // later block of the first block's parity lands where that one's earlier
    // rows are, so the first block's CTA, which has read them, writes it too.
    const int j0 = s.start >> c.logP, jl = (s.end - 1) >> c.logP;
    const bool rides = (s.start & (c.P - 1)) != 0;
    if (s.end > s.start) {
      if (j >= jl - 1 && !(rides && j > j0 && ((j - j0) & 1) == 0)) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          const int tok = (j << c.logP) + o0 + i * ostep;
          if (tok >= s.start && tok < s.end)
            *reinterpret_cast<uint4*>(ring + (size_t)((tok + s.shift) & mask2) * c.D + dc0) = v[i];
        }
      }
      const int jm = ((jl - j0) & 1) == 0 ? jl : jl - 1;
      if (rides && j == j0 && jm > j0) {  // the barrier after the maximum is behind the reads of `recent`
        const int rows = min(c.P, s.end - (jm << c.logP));
        for (int e = tid; e < rows * vpr; e += THREADS) {
          const int o = e >> log_vpr, dc = (e & (vpr - 1)) * 8, tok = (jm << c.logP) + o;
          *reinterpret_cast<uint4*>(ring + (size_t)((tok + s.shift) & mask2) * c.D + dc) =
              *reinterpret_cast<const uint4*>(x + (size_t)(s.row0 + tok - s.start) * a.stride + dc);
        }
      }
    }
    __syncthreads();  // s_max is read: the next task may write it
  }

  __syncthreads();
  if (tid == 0) {
    __threadfence();
    const unsigned before = atomicAdd(reinterpret_cast<unsigned*>(c.control + 2), 1u + wrong);
    s_last = before % kWrongBlock == gridDim.x - 1 ? 1 + (before + wrong) / kWrongBlock : 0;
  }
  __syncthreads();
  if (s_last == 0) return;
  __threadfence();
  if (go) {
    int q = n_free - s_tot[1] + drop_in - drop;
    for (int b = b0; b < b1; ++b) {
      const KvSpan s = kv_span(a, b);
      for (int j = s.have; j < s.had; ++j) c.free_ids[q++] = c.table[(size_t)s.seq * c.max_blocks + j];
      const int pos = s.end + s.shift;
      // `recent` reaches back to the block before the last one, and no further than it did
      const int lo = (((pos - 1) >> c.logP) - 1) * c.P;
      c.seq[s.seq] = make_int4(s.end, pos, max(min(s.from, s.start + s.shift), lo), 0);
    }
  }
  if (tid == 0) {
    if (bad != 0 || s_last > 1) kv_raise(c, bad != 0 ? bad : (int)MSI_ERR_INVALID_ARG);
    c.control[2] = 0;
    if (go) c.control[0] = n_free - s_tot[1] + s_tot[2];
  }
}

template <int THREADS, int VPT>
cudaError_t append_as(const KvAppendArgs& a, cudaStream_t s) {
  // each sequence changes at most (rows - 1) / P + 2 blocks
  const long long tasks = ((long long)a.n_rows / a.c.P + 2LL * a.n) * 2 * a.c.K;
  const long long most = (long long)a.sms * (append_threads(VPT) / THREADS);  // all resident
  kv_append_kernel<THREADS, VPT><<<(unsigned)(tasks < most ? tasks : most), THREADS, 0, s>>>(a);
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// Eviction and release
// ---------------------------------------------------------------------------
constexpr int kEvictThreads = 1024;
constexpr int kEvictFew = 4, kEvictMine = 4;  // evictions found one by one, and candidates a thread then holds
constexpr int kEvictKeys = 24576;  // candidates held in shared memory; longer tables are read again each pass

// Ordering of fp32 weights as whole numbers (a NaN with a clear sign is above
// infinity: what cannot be ranked is not evicted).
__device__ __forceinline__ unsigned kv_key(float w) {
  const unsigned u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA a sequence.  A cache that stays at its budget gives up a block or
// two at a time: up to four are found one by one as the block-wide least (weight,
// then the later block), which takes two barriers each, and the entries after
// them move down.  More: the threshold weight by a radix selection (four passes
// over 8 bits, whole-number histograms, so the result does not depend on any
// order), then one pass over the table in order that keeps or frees.  With the
// append before, us one by one / by radix selection: 64 sequences of 256 blocks
// that give up one 11.8 / 15.4, four 13.9 / 15.9, six 16.4 / 16.9, eight 18.5 / 17.4;
// three of 4,000 that give up one 11.7 / 19.0, four 13.8 / 19.0, eight 17.5 / 19.1,
// twelve 21.5 / 20.0; one of 100, four 13.3 / 15.4, eight 16.2 / 14.9.  (The two meet
// at six to ten; beyond 4,096 candidates a thread would hold more than four: two
// sequences of 8,000, eight candidates a thread, one 12.3 / 23.1.)  Bound: latency
// (dependent passes over a few KB).
__global__ void __launch_bounds__(kEvictThreads) kv_evict_kernel(KvEvictArgs a) {
  extern __shared__ unsigned s_key[];
  __shared__ int s_scan[32], s_hist[8][256], s_pick[2];
  __shared__ unsigned s_least[32];
  __shared__ int s_where[32], s_gone[kEvictFew + 1];
  __shared__ unsigned s_seen[kKvMaxSeqs / 32];
  __shared__ int s_bad, s_mine[3];  // s_mine: sequence, held, freed blocks before its own
  __shared__ int s_total;
  __shared__ unsigned s_last;
  const KvCache& c = a.c;
  const int tid = threadIdx.x;
  const int keep = a.release ? 0 : a.keep;
  if (tid < kKvMaxSeqs / 32) s_seen[tid] = 0;
  if (tid == 0) s_bad = 0, s_mine[0] = -1;
  const int n_free = c.control[0];
  const int status = c.control[1];
  __syncthreads();

  // the batch's bookkeeping: an entry a thread
  int seq = -1, freed = 0;
  int4 st = make_int4(0, 0, 0, 0);
  if (tid < a.n) {
    seq = kv_seq(a.seqs, tid);
    if (seq < 0 || seq >= c.n_seqs ||
        (atomicOr(&s_seen[seq >> 5], 1u << (seq & 31)) & (1u << (seq & 31))) != 0) {
      s_bad = 1;
    } else {
      st = c.seq[seq];
      const int had = st.x < 0 || st.x > c.max_blocks << c.logP ? c.n_blocks + 1 : (st.x + c.P - 1) >> c.logP;
      if (had > c.n_blocks) s_bad = 1;
      else freed = max(0, had - keep);
    }
  }
  const int freed_in = block_scan(freed, s_scan);
  if (tid == kEvictThreads - 1) s_total = freed_in;
  if (tid == blockIdx.x) s_mine[0] = seq, s_mine[1] = st.x, s_mine[2] = freed_in - freed;
  __syncthreads();
  // more blocks than the pool has: the tables cannot be right
  const bool bad = s_bad != 0 || n_free < 0 || n_free > c.n_blocks || s_total > c.n_blocks - n_free;
  const bool go = !bad && status == 0;
  const int n = go ? (s_mine[1] + c.P - 1) >> c.logP : 0;

  if (go && n > keep && !a.release && n - keep <= kEvictFew && n - a.sinks - a.recent <= kEvictMine * kEvictThreads) {
    int* table = c.table + (size_t)s_mine[0] * c.max_blocks;
    const int m = n - a.sinks - a.recent, out = n - keep;
    const int lane = tid & 31, wid = tid >> 5;
    unsigned key[kEvictMine];
    int left[kEvictMine];  // table index; -1: none, or found already
#pragma unroll
    for (int k = 0; k < kEvictMine; ++k) {
      const int i = k * kEvictThreads + tid;
      left[k] = i < m ? a.sinks + i : -1;
      key[k] = 0xffffffffu;
      if (i < m) {
        const int id = table[a.sinks + i];
        key[k] = id >= 0 && id < c.n_blocks ? kv_key(c.weight[id]) : 0u;
      }
    }
    for (int e = 0; e < out; ++e) {
      unsigned low = 0xffffffffu;
      int at = -1;
#pragma unroll
      for (int k = 0; k < kEvictMine; ++k)  // the later of equals
        if (left[k] >= 0 && key[k] <= low) low = key[k], at = left[k];
      const unsigned wl = __reduce_min_sync(0xffffffffu, at >= 0 ? low : 0xffffffffu);
      const int wa = __reduce_max_sync(0xffffffffu, at >= 0 && low == wl ? at : -1);
      if (lane == 0) s_least[wid] = wl, s_where[wid] = wa;
      __syncthreads();
      const unsigned bl = __reduce_min_sync(0xffffffffu, s_where[lane] >= 0 ? s_least[lane] : 0xffffffffu);
      const int ba = __reduce_max_sync(0xffffffffu, s_where[lane] >= 0 && s_least[lane] == bl ? s_where[lane] : -1);
#pragma unroll
      for (int k = 0; k < kEvictMine; ++k)
        if (left[k] == ba) left[k] = -1;
      if (tid == 0) {  // in table order
        int p = e;
        for (; p > 0 && s_gone[p - 1] > ba; --p) s_gone[p] = s_gone[p - 1];
        s_gone[p] = ba;
      }
      __syncthreads();
    }
    if (tid < out) c.free_ids[n_free + s_mine[2] + tid] = table[s_gone[tid]];
    for (int t0 = s_gone[0] / kEvictThreads * kEvictThreads; t0 < n; t0 += kEvictThreads) {
      const int j = t0 + tid;
      const int id = j < n ? table[j] : -1;
      int down = 0;
      bool gone = false;
      for (int e = 0; e < out; ++e) down += s_gone[e] < j, gone |= s_gone[e] == j;
      __syncthreads();  // the tile is read; what it writes lies in it or before
      if (j < n && !gone && down > 0) table[j - down] = id;
    }
  } else if (go && n > keep) {
    int* table = c.table + (size_t)s_mine[0] * c.max_blocks;
    const int sinks = a.release ? 0 : a.sinks;
    const int m = n - sinks - a.recent;        // candidates
    const int need = keep - sinks - a.recent;  // of which this many stay
    const bool cached = m <= kEvictKeys;
    auto key_of = [&](int i) {
      const int id = table[sinks + i];
      return id >= 0 && id < c.n_blocks ? kv_key(c.weight[id]) : 0u;
    };
    unsigned thr = 0xffffffffu;
    int need_eq = 0;
    if (!a.release && need > 0) {
      if (cached)
        for (int i = tid; i < m; i += kEvictThreads) s_key[i] = key_of(i);
      unsigned prefix = 0;
      int left = need;
      for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 8 * 256; i += kEvictThreads) (&s_hist[0][0])[i] = 0;
        __syncthreads();
        for (int i = tid; i < m; i += kEvictThreads) {
          const unsigned k = cached ? s_key[i] : key_of(i);
          if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
            atomicAdd(&s_hist[(tid >> 5) & 7][(k >> shift) & 255], 1);
        }
        __syncthreads();
        // thread t: digit 255 - t, so that inclusive sums count from the greatest
        int v = 0;
        if (tid < 256)
#pragma unroll
          for (int i = 0; i < 8; ++i) v += s_hist[i][255 - tid];
        const int upto = block_scan(v, s_scan);
        if (tid < 256 && upto >= left && upto - v < left) s_pick[0] = 255 - tid, s_pick[1] = left - (upto - v);
        __syncthreads();
        prefix |= (unsigned)s_pick[0] << shift;
        left = s_pick[1];
      }
      thr = prefix;
      need_eq = left;
    }
    // keep or free, in table order
    int kept = 0, gone = 0, eq = 0;
    int* free_to = c.free_ids + n_free + s_mine[2];
    for (int t0 = 0; t0 < n; t0 += kEvictThreads) {
      const int j = t0 + tid, i = j - sinks;
      const int id = j < n ? table[j] : -1;
      bool stay = false, is_eq = false;
      if (j < n && !a.release) {
        if (j < sinks || j >= n - a.recent) stay = true;
        else if (need > 0) {
          const unsigned k = cached ? s_key[i] : key_of(i);
          stay = k > thr;
          is_eq = k == thr;
        }
      }
      const int e_in = block_scan(is_eq, s_scan);
      if (is_eq && eq + e_in <= need_eq) stay = true;
      const int k_in = block_scan(stay, s_scan);
      if (j < n) {
        if (stay) table[kept + k_in - 1] = id;  // at or before j: read above, in this pass or an earlier one
        else free_to[gone + (tid + 1 - k_in) - 1] = id;
      }
      if (tid == kEvictThreads - 1) s_pick[0] = k_in, s_pick[1] = e_in;
      __syncthreads();
      kept += s_pick[0];
      eq += s_pick[1];
      gone += min(kEvictThreads, n - t0) - s_pick[0];
    }
  }

  __syncthreads();
  if (tid == 0) {
    __threadfence();
    s_last = atomicAdd(reinterpret_cast<unsigned*>(c.control + 3), 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (s_last == 0) return;
  __threadfence();
  if (go && tid < a.n) {
    if (a.release) {
      c.seq[seq] = make_int4(0, 0, 0, 0);
    } else if (freed > 0) {
      // with one recent block, the one before it in the table is no longer the one before it in the text
      const int from = a.recent == 1 ? max(st.z, ((st.y - 1) >> c.logP) << c.logP) : st.z;
      c.seq[seq] = make_int4(st.x - (freed << c.logP), st.y, from, 0);
    }
  }
  if (tid == 0) {
    if (bad) kv_raise(c, MSI_ERR_INVALID_ARG);
    if (go) c.control[0] = n_free + s_total;
    c.control[3] = 0;
  }
}

// ---------------------------------------------------------------------------
// Read back and init
// ---------------------------------------------------------------------------
constexpr int kReadThreads = 256, kReadRows = 64;

// `per` (at most 64) rows a CTA: their blocks looked up by a thread each, then 16
// codes a thread and step to two 16-byte stores.  16 rows where that leaves an
// SM no more than four CTAs, so that short calls fill the GPU (us with 16 / 64 rows:
// the last blocks of 64 sequences 4.1 / 7.2, 8,741 rows of 2 x 256 7.7 / 10.3), 64 for
// the rest (32,768 rows of 2 x 128 11.4 / 11.6).  Bound: memory (codes in, twice as
// many bytes out: 4.4 TB/s at 32,768 rows) and the CTAs' two dependent loads.
__global__ void __launch_bounds__(kReadThreads) kv_read_kernel(KvReadArgs a, int per) {
  const KvCache& c = a.c;
  __shared__ long long s_at[kReadRows];  // element of the row in a head-0 block, or -1
  __shared__ int s_id[kReadRows];
  const int tid = threadIdx.x;
  const int row0 = blockIdx.x * per;
  if (tid < per) {
    const int row = row0 + tid;
    s_at[tid] = -1;
    s_id[tid] = 0;
    if (row < a.n_rows) {
      int lo = 0, hi = a.n;  // the last entry with cu <= row
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid] <= row) lo = mid; else hi = mid;
      }
      const int seq = kv_seq(a.seqs, lo);
      const int i = row - a.cu[lo];
      if (a.cu[lo] >= 0 && i >= 0 && row < a.cu[lo + 1] && seq >= 0 && seq < c.n_seqs) {
        const long long tok = (long long)(a.first == nullptr ? 0 : a.first[lo]) + i;
        const int held = min(c.seq[seq].x, c.max_blocks << c.logP);
        if (tok >= 0 && tok < held) {
          const int id = c.table[(size_t)seq * c.max_blocks + (tok >> c.logP)];
          if (id >= 0 && id < c.n_blocks) {
            s_id[tid] = id;
            s_at[tid] = (long long)id * c.K * c.P * c.D + (tok & (c.P - 1)) * c.D;
          }
        }
      }
      if (s_at[tid] < 0) kv_raise(c, MSI_ERR_INVALID_ARG);
    }
  }
  __syncthreads();
  // `group` lanes a row (a power of two), 16 codes a lane and turn
  const int log_ph = c.D == 64 ? 2 : c.D == 128 ? 3 : 4, per_row = c.K << log_ph, both = 2 * per_row;
  const int rows = min(per, a.n_rows - row0);
  const int group = both >= 32 ? 32 : 1 << (31 - __clz(both));
  const int lane = tid & (group - 1);
#pragma unroll 4
  for (int r = tid / group; r < rows; r += kReadThreads / group) {
    const long long at = s_at[r];
    for (int e = lane; e < both; e += group) {
      const int w = e >= per_row, f = e - w * per_row, h = f >> log_ph, dc = (f - (h << log_ph)) * 16;
      uint32_t o[8];
      if (at < 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = 0x7fc07fc0u;
      } else {
        const uint4 v = *reinterpret_cast<const uint4*>(c.codes[w] + at + (size_t)h * c.P * c.D + dc);
        const float s = c.scale[w][(size_t)s_id[r] * c.K + h];
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t p, q;
          if (c.fmt == MSI_KV_Q8) p = kv_f16x2<MSI_KV_Q8, false>(u[i]), q = kv_f16x2<MSI_KV_Q8, true>(u[i]);
          else p = kv_f16x2<MSI_KV_E4M3, false>(u[i]), q = kv_f16x2<MSI_KV_E4M3, true>(u[i]);
          const float2 x = __half22float2(*reinterpret_cast<__half2*>(&p));
          const float2 y = __half22float2(*reinterpret_cast<__half2*>(&q));
          o[2 * i] = pack_bf16x2(x.x * s, x.y * s);
          o[2 * i + 1] = pack_bf16x2(y.x * s, y.y * s);
        }
      }
      uint4* dst = reinterpret_cast<uint4*>(a.out[w] + ((size_t)(row0 + r) * c.K + h) * c.D + dc);
      dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
      dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
  }
}

__global__ void kv_init_kernel(KvCache c) {
  const int i0 = blockIdx.x * blockDim.x + threadIdx.x, step = gridDim.x * blockDim.x;
  for (int i = i0; i < c.n_blocks; i += step) {
    c.free_ids[i] = c.n_blocks - 1 - i;
    c.weight[i] = 0.0f;
  }
  for (int i = i0; i < c.n_seqs; i += step) c.seq[i] = make_int4(0, 0, 0, 0);
  if (i0 < 8) c.control[i0] = i0 == 0 ? c.n_blocks : 0;
}

}  // namespace

cudaError_t launch_kv_append(const KvAppendArgs& a, cudaStream_t s) {
  switch (a.c.P * a.c.D) {  // elements of a block: 8 a thread and pass, at most 16 passes
    case 1024: return append_as<128, 1>(a, s);
    case 2048: return append_as<128, 2>(a, s);
    case 4096: return append_as<128, 4>(a, s);
    case 8192: return append_as<256, 4>(a, s);
    case 16384: return append_as<256, 8>(a, s);
    default: return append_as<256, 16>(a, s);
  }
}

cudaError_t launch_kv_evict(const KvEvictArgs& a, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const int smem = a.release ? 0 : min(kEvictKeys, a.c.max_blocks) * 4;
  cudaError_t e = smem_attr_once(kv_evict_kernel, kEvictKeys * 4, done);
  if (e != cudaSuccess) return e;
  kv_evict_kernel<<<a.n, kEvictThreads, smem, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_kv_read(const KvReadArgs& a, cudaStream_t s) {
  const int per = a.n_rows <= a.sms * 4 * 16 ? 16 : kReadRows;
  kv_read_kernel<<<(a.n_rows + per - 1) / per, kReadThreads, 0, s>>>(a, per);
  return cudaGetLastError();
}

cudaError_t launch_kv_init(const KvCache& c, cudaStream_t s) {
  const int most = c.n_blocks > c.n_seqs ? c.n_blocks : c.n_seqs;
  kv_init_kernel<<<min(1024, (most + 255) / 256), 256, 0, s>>>(c);
  return cudaGetLastError();
}

}  // namespace msi

// ===========================================================================
// C ABI
// ===========================================================================
using namespace msi;

struct msi_kv {
  KvCache c;
  int dev, sms;
  std::atomic<unsigned long long> launches;
  std::atomic<long long> wait_cycles{kKvWaitCycles};
  std::atomic<int> stall{0};  // of the next call in chunk form
};

namespace {

bool aligned16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

msi_status enter(const msi_kv* kv, int n) {
  if (kv == nullptr || n < 0) return MSI_ERR_INVALID_ARG;
  if (n > kv->c.n_seqs) return MSI_ERR_INVALID_ARG;
  int cur = -1;
  const cudaError_t e = cudaGetDevice(&cur);
  if (e != cudaSuccess) return note_cuda_error(e, "cudaGetDevice");
  return cur == kv->dev ? MSI_OK : MSI_ERR_INVALID_ARG;
}

msi_status launched(msi_kv* kv, cudaError_t e, const char* what, int kernels = 1) {
  if (e != cudaSuccess) return note_cuda_error(e, what);
  kv->launches += kernels;
  return MSI_OK;
}

size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// A call's arguments checked and laid out over `ws` (null: sizes only).
msi_status attention_args(const msi_kv* kv, const msi_kv_attention_args* g, char* ws, KvAttnArgs* out, size_t* bytes) {
  const KvCache& c = kv->c;
  if (g->n < 0 || g->n > c.n_seqs || g->n_rows < 0 || g->max_rows < 0 || g->max_rows > g->n_rows || g->n_heads < 1 ||
      g->n_heads % c.K != 0)
    return MSI_ERR_INVALID_ARG;
  if ((g->flags & ~(unsigned)MSI_KV_OBSERVE) != 0) return MSI_ERR_INVALID_ARG;
  if (g->n_heads / c.K > 128 || (long long)g->n_rows * (g->n_heads / c.K) > (1 << 30)) return MSI_ERR_UNSUPPORTED;
  KvAttnArgs a = {};
  a.c = c;
  a.n = g->n;
  a.n_rows = g->n_rows;
  a.max_rows = g->max_rows;
  a.H = g->n_heads;
  a.G = g->n_heads / c.K;
  a.seqs = g->seqs;
  a.cu = g->cu;
  a.q = static_cast<const __nv_bfloat16*>(g->q);
  a.q_stride = g->q_stride;
  a.out = static_cast<__nv_bfloat16*>(g->out);
  a.out_stride = g->out_stride;
  a.lse = g->lse;
  a.scale = g->scale;
  a.softcap = g->softcap > 0.0f && g->softcap < 1e-30f ? 1e-30f : g->softcap;  // scores of 0 all the same; 1 / cap stays finite
  // as long as a sequence can be, or longer: none (and the kernels' sums with it stay within 32 bits)
  a.window = g->window >= c.max_blocks << c.logP ? 0 : g->window;
  a.observe = (g->flags & MSI_KV_OBSERVE) != 0;
  const int tiles = kv_decode_tiles(a.max_rows * a.G, c.D);
  if (tiles == 0 && a.observe) return MSI_ERR_UNSUPPORTED;
  if (tiles != 0) a.groups = (a.max_rows * a.G + 8 * tiles - 1) / (8 * tiles);
  a.ctas = kv->sms < 512 ? kv->sms : 512;
  a.ctas = tiles != 0 ? 2 * a.ctas : a.ctas / 2;  // two of the decode form's share an SM, two of the chunk form's an item
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at = round256(at + n);
    return ws == nullptr ? nullptr : ws + here;
  };
  const size_t rows = tiles != 0 ? 8 * (size_t)tiles : kv_chunk_rows(c.D);
  a.part_o = reinterpret_cast<float*>(take(2 * (size_t)a.ctas * rows * c.D * 4));
  a.part_ml = reinterpret_cast<float*>(take(2 * (size_t)a.ctas * rows * 2 * 4));
  if (tiles == 0) {
    // each sequence has at most (rows - 1) / tile + 1 row tiles
    a.max_items = (int)(((long long)a.n_rows * a.G / (long long)rows + a.n) * c.K);
    a.items = reinterpret_cast<int4*>(take(2 * (size_t)a.max_items * sizeof(int4)));
    a.item_pre = reinterpret_cast<long long*>(take(((size_t)a.max_items + 1) * sizeof(long long)));
    a.plan = reinterpret_cast<int*>(take((4 + (size_t)a.ctas) * sizeof(int)));
  }
  if (tiles != 0) a.split = reinterpret_cast<int4*>(take((size_t)a.ctas * sizeof(int4)));
  if (a.observe) {
    a.item_pre = reinterpret_cast<long long*>(take(((size_t)a.n + 1) * sizeof(long long)));
    a.lse2 = reinterpret_cast<float*>(take((size_t)a.n_rows * a.H * 4));
    // no block belongs to two sequences: the pool bounds the steps
    a.max_steps = ((long long)c.n_blocks * (c.P / 16) + (long long)a.n * kv_decode_pair_cost()) * c.K * a.groups;
    a.step_lse = reinterpret_cast<float*>(take((size_t)a.max_steps * rows * 4));
  }
  *bytes = at;
  *out = a;
  return MSI_OK;
}

}  // namespace

extern "C" {

msi_status msi_kv_create(const msi_kv_desc* desc, msi_kv** out) {
  if (desc == nullptr || out == nullptr) return MSI_ERR_INVALID_ARG;
  *out = nullptr;
  const msi_kv_desc& d = *desc;
  if (d.n_seqs < 1 || d.max_blocks < 1 || d.n_blocks < 1 || d.n_kv_heads < 1 ||
      (d.format != MSI_KV_Q8 && d.format != MSI_KV_E4M3))
    return MSI_ERR_INVALID_ARG;
  const int P = d.block_tokens, D = d.head_dim;
  if (d.n_seqs > kKvMaxSeqs || d.n_kv_heads > kKvMaxHeads || (D != 64 && D != 128 && D != 256) ||
      (P != 16 && P != 32 && P != 64 && P != 128) || (long long)d.max_blocks * P > (1LL << 28) ||
      d.n_blocks >= 1 << 21)
    return MSI_ERR_UNSUPPORTED;
  for (const void* p : {(const void*)d.k_codes, (const void*)d.v_codes, (const void*)d.recent, (const void*)d.seq_state})
    if (!aligned16(p)) return MSI_ERR_INVALID_ARG;
  for (const void* p : {(const void*)d.k_scale, (const void*)d.v_scale, (const void*)d.table, (const void*)d.free_ids,
                        (const void*)d.control, (const void*)d.weight})
    if (p == nullptr || (reinterpret_cast<uintptr_t>(p) & 3) != 0) return MSI_ERR_INVALID_ARG;
  msi_kv* kv = new (std::nothrow) msi_kv();
  if (kv == nullptr) return MSI_ERR_CUDA;
  cudaError_t e = cudaGetDevice(&kv->dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, kv->dev);
  if (e != cudaSuccess) {
    delete kv;
    return note_cuda_error(e, "msi_kv_create");
  }
  KvCache& c = kv->c;
  c.n_seqs = d.n_seqs;
  c.max_blocks = d.max_blocks;
  c.n_blocks = d.n_blocks;
  c.K = d.n_kv_heads;
  c.D = D;
  c.P = P;
  c.logP = P == 16 ? 4 : P == 32 ? 5 : P == 64 ? 6 : 7;
  c.fmt = d.format;
  c.codes[0] = static_cast<uint8_t*>(d.k_codes);
  c.codes[1] = static_cast<uint8_t*>(d.v_codes);
  c.scale[0] = d.k_scale;
  c.scale[1] = d.v_scale;
  c.recent = static_cast<__nv_bfloat16*>(d.recent);
  c.table = d.table;
  c.seq = reinterpret_cast<int4*>(d.seq_state);
  c.free_ids = d.free_ids;
  c.control = d.control;
  c.weight = d.weight;
  kv->launches = 0;
  *out = kv;
  return MSI_OK;
}

msi_status msi_kv_destroy(msi_kv* kv) {
  if (kv == nullptr) return MSI_ERR_INVALID_ARG;
  delete kv;
  return MSI_OK;
}

msi_status msi_kv_init(msi_kv* kv, msi_stream stream) {
  msi_status st = enter(kv, 0);
  if (st != MSI_OK) return st;
  return launched(kv, launch_kv_init(kv->c, stream), "msi_kv_init");
}

msi_status msi_kv_append(msi_kv* kv, int n, const int32_t* seqs, const int32_t* cu, const int32_t* start,
                         const void* k, const void* v, int64_t row_stride, int n_rows, msi_stream stream) {
  msi_status st = enter(kv, n);
  if (st != MSI_OK) return st;
  if (n_rows < 0 || (n > 0 && cu == nullptr) || (n_rows > 0 && n == 0)) return MSI_ERR_INVALID_ARG;
  if (n_rows > 1 << 27) return MSI_ERR_UNSUPPORTED;
  if (n == 0) return MSI_OK;
  if (n_rows > 0 && (!aligned16(k) || !aligned16(v) || row_stride < 0 || row_stride % 8 != 0)) return MSI_ERR_INVALID_ARG;
  KvAppendArgs a = {kv->c, n, n_rows, seqs, cu, start,
                    {static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v)}, row_stride, kv->sms};
  return launched(kv, launch_kv_append(a, stream), "msi_kv_append");
}

msi_status msi_kv_workspace_size(const msi_kv* kv, const msi_kv_attention_args* args, size_t* bytes,
                                 int* decode_form) {
  if (kv == nullptr || args == nullptr || bytes == nullptr) return MSI_ERR_INVALID_ARG;
  KvAttnArgs a;
  msi_status st = attention_args(kv, args, nullptr, &a, bytes);
  if (st != MSI_OK) return st;
  if (decode_form != nullptr) *decode_form = kv_decode_tiles(a.max_rows * a.G, a.c.D) != 0;
  return MSI_OK;
}

msi_status msi_kv_attention(msi_kv* kv, const msi_kv_attention_args* args, void* workspace, size_t workspace_bytes,
                            msi_stream stream) {
  msi_status st = enter(kv, 0);
  if (st != MSI_OK) return st;
  if (args == nullptr) return MSI_ERR_INVALID_ARG;
  if (!(args->scale > 0.0f) || !isfinite(args->scale) || !(args->softcap >= 0.0f) || !isfinite(args->softcap) ||
      args->window < 0)
    return MSI_ERR_INVALID_ARG;
  KvAttnArgs a;
  size_t need = 0;
  st = attention_args(kv, args, static_cast<char*>(workspace), &a, &need);
  if (st != MSI_OK) return st;
  if (a.n == 0 || a.n_rows == 0) return MSI_OK;
  if (a.max_rows == 0 || a.cu == nullptr || !aligned16(a.q) || !aligned16(a.out) || a.q_stride < 0 ||
      a.q_stride % 8 != 0 || a.out_stride < (long long)a.H * a.c.D || a.out_stride % 8 != 0)
    return MSI_ERR_INVALID_ARG;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < need)
    return MSI_ERR_WORKSPACE;
  int kernels = 0;
  cudaError_t e;
  if (kv_decode_tiles(a.max_rows * a.G, a.c.D) != 0) {
    e = launch_kv_decode(a, &kernels, stream);
  } else {
    a.wait_limit = kv->wait_cycles.load();
    a.stall = kv->stall.exchange(0);
    e = launch_kv_chunk(a, &kernels, stream);
  }
  return launched(kv, e, "msi_kv_attention", kernels);
}

msi_status msi_kv_evict(msi_kv* kv, int n, const int32_t* seqs, int keep, int sinks, int recent, msi_stream stream) {
  msi_status st = enter(kv, n);
  if (st != MSI_OK) return st;
  if (sinks < 0 || recent < 1 || keep < 1 || sinks > keep - recent) return MSI_ERR_INVALID_ARG;
  if (n == 0) return MSI_OK;
  KvEvictArgs a = {kv->c, n, seqs, keep, sinks, recent, 0};
  return launched(kv, launch_kv_evict(a, stream), "msi_kv_evict");
}

msi_status msi_kv_release(msi_kv* kv, int n, const int32_t* seqs, msi_stream stream) {
  msi_status st = enter(kv, n);
  if (st != MSI_OK) return st;
  if (n == 0) return MSI_OK;
  KvEvictArgs a = {kv->c, n, seqs, 0, 0, 0, 1};
  return launched(kv, launch_kv_evict(a, stream), "msi_kv_release");
}

msi_status msi_kv_read(msi_kv* kv, int n, const int32_t* seqs, const int32_t* first, const int32_t* cu, int n_rows,
                       void* k_out, void* v_out, msi_stream stream) {
  msi_status st = enter(kv, n);
  if (st != MSI_OK) return st;
  if (n_rows < 0 || (n_rows > 0 && (n == 0 || cu == nullptr || !aligned16(k_out) || !aligned16(v_out))))
    return MSI_ERR_INVALID_ARG;
  if (n_rows == 0) return MSI_OK;
  KvReadArgs a = {kv->c, n, n_rows, seqs, first, cu,
                  {static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out)}, kv->sms};
  return launched(kv, launch_kv_read(a, stream), "msi_kv_read");
}

msi_status msi_kv_status(msi_kv* kv, msi_stream stream, int* device_status) {
  msi_status st = enter(kv, 0);
  if (st != MSI_OK) return st;
  if (device_status == nullptr) return MSI_ERR_INVALID_ARG;
  int word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, kv->c.control + 1, sizeof(int), cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  if (e == cudaSuccess && word != 0) e = cudaMemsetAsync(kv->c.control + 1, 0, sizeof(int), stream);
  if (e != cudaSuccess) return note_cuda_error(e, "msi_kv_status");
  *device_status = word;
  return MSI_OK;
}

msi_status msi_kv_set_wait_cycles(msi_kv* kv, int64_t cycles) {
  if (kv == nullptr) return MSI_ERR_INVALID_ARG;
  kv->wait_cycles = cycles > 0 ? (long long)cycles : kKvWaitCycles;
  return MSI_OK;
}

msi_status msi_kv_inject_stall(msi_kv* kv, int where) {
  if (kv == nullptr || where < 0 || where > MSI_KV_STALL_CONVERSION) return MSI_ERR_INVALID_ARG;
  kv->stall = where;
  return MSI_OK;
}

uint64_t msi_kv_kernel_launches(const msi_kv* kv) { return kv == nullptr ? 0 : (uint64_t)kv->launches.load(); }

}  // extern "C"
