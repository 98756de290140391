// A token for each row of logits (include/msi.h, msi_sample): temperature,
// top-k, top-p, min-p, and the draw by a given random number.
//
// Arithmetic.  A token's weight is exp((l - max) / T) = 2^a, a <= 0.  a is worked
// out as the sum of two fp32 numbers, 2^a from a table of 2^(j / 32) and a
// polynomial, and rounded once, to a code of 32 bits: 6 bits of the whole part of
// a, 26 of the mantissa.  Codes order tokens as their logits do; from there on
// everything is whole numbers: a code stands for 2^44 2^a, rounded down below
// 2^-18 of the greatest, and sums of those are exact in 64 bits.  So nothing
// depends on the order of a sum or on how a row is split, and a border (the
// k-th token, the share top_p, the drawn token) lies where 2^-26 of each weight
// and 2^-44 of the greatest say it does.
//
// A row belongs to a cluster of CTAs, its codes stay in their shared memory.  A
// border among sorted tokens is found without sorting: histograms of the codes'
// upper 11, middle 11 and lower 10 bits, in shared memory, added up over the
// cluster.  Before a top-k of up to 32 tokens a warp, logits under a bound that
// more than k reach (the least, over the warps, of the r-th greatest of their
// lanes' greatest) get no code at all.
//
// Floor: the logits, read once.  Bound: for many long rows the instructions that make
// a code (about 45 a token, a third of them on the half-rate integer pipe) and two
// waves of clusters, since a GPU's shared memory holds the codes of 36 rows of
// 131,072 (64 rows, top-p: 54 us, a wave 27); for a few the chain of barriers and
// scans (one row of 32,000: 10 us with top-k, 13 with top-p alone, 7.5 without).
#include <math.h>

#include <type_traits>

#include "kernels.cuh"
#include "per_device.h"

namespace msi {
namespace {

typedef unsigned long long u64;

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kSampleMaxVocab = 1 << 18;
constexpr int kBins = 2048, kCoarse = 64, kFine = 32;  // a coarse bin is 32 bins: codes with the same upper 6 bits, at first
constexpr int kFew = 256;                    // codes that are compared with each other
constexpr int kListed = 256, kPicked = 1400;  // codes that are picked out: of a CTA at most, of all as expected
// Groups of 128 codes of a warp: what fits an SM beside the rest (8 CTAs hold 2^18
// and a vector more with 18), and where two CTAs fit one.
constexpr int kSampleMaxGroups = 22, kSampleTwoGroups = 8;

struct SampleArgs {
  const void* logits;
  long long stride;
  int rows, vocab;
  const float* u;
  const float* temperature;
  const int* top_k;
  const float* top_p;
  const float* min_p;
  float temperature0, top_p0, min_p0;
  int top_k0;
  int* ids;
  float* logprobs;
};

constexpr float kMostFloat = 3.4028234e38f;
constexpr float kRoundMagic = 12582912.0f;  // 1.5 2^23: a sum with it is rounded to a whole number
constexpr uint32_t kRoundBits = 0x4B400000u;
constexpr float kLeast = -42.9f;  // log2 of the least weight, beside the greatest, that has a code: its share is 1 or more

// How a row's logits become codes: ch + cl = log2(e) / (before after T); y = top ch of
// the greatest logit, top: times `before`.
struct RowScale {
  float top, ch, cl, y;
  float before, after;  // powers of two, 1 but for the least and greatest temperatures
  uint32_t whole;  // (44 - the whole part of y) << 26
};

// 2^(j / 32) in units of 2^-27
__constant__ uint32_t kPow32[32] = {
    134217728u, 137156714u, 140160054u, 143229160u, 146365470u, 149570457u, 152845623u, 156192507u, 159612677u, 163107740u, 166679334u,
    170329136u, 174058859u, 177870251u, 181765103u, 185745240u, 189812531u, 193968884u, 198216250u, 202556621u, 206992033u, 211524568u,
    216156353u, 220889561u, 225726413u, 230669177u, 235720175u, 240881774u, 246156398u, 251546522u, 257054673u, 262683438u};

// 2^(a + e) as a code, |a| up to 4,096 and |e| up to 2^-11; whole: (44 - what a's
// whole part counts from) << 26.  a's nearest 32nd is split off, the rest goes
// through the series of 2^r - 1 (the next term is under 2^-39); off by 2^-27 before
// the rounding to 26 bits, whose leading one stands for 2^25: 2^25 2^(-1 / 64) to 2^25
// 2^(63 / 64), past either end by what e adds.
__device__ __forceinline__ uint32_t power_code(float a, float e, uint32_t whole, const uint2* tab) {
  const float n = fmaf(a, 32.0f, kRoundMagic);
  const float r = fmaf(__fadd_rn(n, -kRoundMagic), -1.0f / 32.0f, a) + e;  // exact but for e; about 1/64 at most
  const float p = r * fmaf(r, fmaf(r, fmaf(r, 0.00961812911f, 0.0555041087f), 0.240226507f), 0.693147181f);
  const uint32_t k = __float_as_uint(n) - kRoundBits;
  const uint2 w = tab[k & 31u];
  const uint32_t mant = (w.x + __float_as_uint(fmaf(p, __uint_as_float(w.y), kRoundMagic))) >> 2;  // under 2^22 of 2^-27
  return whole + (k * (1u << 21) & 0xfc000000u) + mant;
}
__device__ __forceinline__ uint2 power_entry(int j) {
  return make_uint2(kPow32[j] + 2u - kRoundBits, __float_as_uint((float)kPow32[j]));
}

// The code of logit x.  0: a weight under 2^kLeast of the greatest, or none.
// Codes ascend with x.  NEAR (top ch is 4,096 at most, T within 2^-96 .. 2^96): x ch is
// split as it stands; else x - top first, as the sum of two numbers (any logits).  At
// temperatures beyond, log2(e) / T is no normal fp32 number, or leaves no room for cl:
// the least ones are scaled up after that difference, which is exact at any size, the
// greatest ones down before it, where it could overflow.
template <bool NEAR>
__device__ __forceinline__ uint32_t weight_code(float x, const RowScale& s, const uint2* tab) {
  if (NEAR) {
    const float y = __fmul_rn(x, s.ch);
    const float e = fmaf(x, s.cl, fmaf(x, s.ch, -y));
    return y > s.y + kLeast ? power_code(y, e, s.whole, tab) : 0u;
  }
  x *= s.before;
  float d = __fadd_rn(x, -s.top);
  const float b = __fadd_rn(d, -x);
  const float t = __fadd_rn(__fadd_rn(x, -__fadd_rn(d, -b)), -__fadd_rn(s.top, b)) * s.after;
  d *= s.after;
  const float a = __fmul_rn(d, s.ch);
  const float e = fmaf(t, s.ch, fmaf(d, s.cl, fmaf(d, s.ch, -a)));
  return a > kLeast ? power_code(a, e, 44u << 26, tab) : 0u;  // no number (an infinity times 0): 0
}

// A NaN if either is one.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ u64 code_weight(uint32_t code) {
  return ((u64)(code & 0x3ffffffu) << 19) >> (44 - (code >> 26));  // of code 0: 0
}

// What the weight is proportional to, of codes with the same upper 6 bits.
__device__ __forceinline__ u64 mass(uint32_t code) { return code & 0x3ffffffu; }

// floor(m f) for f in [0, 1), and whether something was cut off
__device__ __forceinline__ u64 share(u64 m, float f, bool* cut) {
  const u64 g = (u64)(f * 18446744073709551616.0f);  // exact from 2^-40 on
  *cut = m * g != 0;
  return __umul64hi(m, g);
}

template <typename U>
__device__ __forceinline__ U sum_warp(U v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename U>
__device__ __forceinline__ U scan_warp(U v) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const U w = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += w;
  }
  return v;
}

__device__ __forceinline__ u64 ld_cluster64(const void* p, uint32_t rank) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];"
               : "=l"(v)
               : "r"(mapa_shared((uint32_t)__cvta_generic_to_shared(p), rank))
               : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_cluster32(const void* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];"
               : "=r"(v)
               : "r"(mapa_shared((uint32_t)__cvta_generic_to_shared(p), rank))
               : "memory");
  return v;
}

// Its instructions want a warp's threads together.
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  cluster_sync_all();
}
__device__ __forceinline__ void st_cluster64(const void* p, uint32_t rank, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(mapa_shared((uint32_t)__cvta_generic_to_shared(p), rank)), "l"(v)
               : "memory");
}

__device__ __forceinline__ void st_cluster32(const void* p, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_shared((uint32_t)__cvta_generic_to_shared(p), rank)), "r"(v)
               : "memory");
}

// Sums that all CTAs of the cluster need are written into each CTA's copy, then
// comes a barrier of the cluster.  What another CTA writes or reads here is there
// twice, used in turn (buf): its next use but one is behind another barrier.
struct SampleShared {
  u64 bins[2][kBins];               // histogram (of counts: as 32-bit words); or, by CTA, codes picked out with their places
  u64 coarse[2][8][kCoarse];        // by CTA
  u64 cta[2][8];
  u64 total[kCoarse], fine[kFine];  // own: sums over the cluster
  int listed[2][8], mine, few;
  u64 key[kFew], share[kFew];       // own: a few codes with their places, and their weights
  u64 warp[kSampleWarps];
  float scale[4];
  int found, ties, tied[8];
  uint32_t lowest, highest;         // code that was picked
  uint2 pow[32];
};

// A code with its place: greater is earlier in descending order.
__device__ __forceinline__ u64 order_key(uint32_t code, int index) { return (u64)code << 32 | (uint32_t)~index; }
__device__ __forceinline__ uint32_t key_code(u64 key) { return (uint32_t)(key >> 32); }
__device__ __forceinline__ int key_index(u64 key) { return (int)~(uint32_t)key; }

// Where the search for a border stands.
struct Border {
  uint32_t prefix;  // the upper bits of its code
  u64 left;         // what of the target lies in the codes with that prefix
  u64 bin;          // their sum
  u64 all;          // the sum over all codes
};

// What a thread sees of a row: groups of 128 codes of its warp, four a lane.
struct Row {
  SampleShared& sh;
  uint4* codes;    // the warp's
  int groups, first;
  int ctas, rank;
  int buf, hist;   // the copies in use: of the sums, of the histogram
  uint32_t least;  // codes under it are dropped

  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    const uint4* mine = codes + (threadIdx.x & 31);
#pragma unroll 4
    for (int g = 0; g < groups; ++g) {
      const uint4 c = mine[g * 32];
      f(c.x), f(c.y), f(c.z), f(c.w);
    }
  }

  // The first index, from the top of N sums (32 or 64), at which they reach
  // `target` together; -1 if they do not.  Each warp works it out.
  template <int N, typename U>
  __device__ __forceinline__ int reach(const U* v, U target, U* above) const {
    const int lane = threadIdx.x & 31;
    const U a = N == 64 ? v[63 - 2 * lane] : (U)0, b = N == 64 ? v[62 - 2 * lane] : v[31 - lane];
    const U incl = scan_warp(a + b);
    const unsigned hit = __ballot_sync(0xffffffffu, incl >= target);
    if (hit == 0) return -1;
    const int l = __ffs(hit) - 1;
    const U before = __shfl_sync(0xffffffffu, incl - a - b, l);
    if (N != 64) {
      *above = before;
      return 31 - l;
    }
    const U first = __shfl_sync(0xffffffffu, a, l);
    const bool at_first = before + first >= target;
    *above = at_first ? before : before + first;
    return at_first ? 63 - 2 * l : 62 - 2 * l;
  }

  __device__ __forceinline__ void clear(u64* bins) const {
    static_assert(kBins * 8 == 2 * 16 * kSampleThreads, "two vectors a thread");
    reinterpret_cast<uint4*>(bins)[threadIdx.x] = make_uint4(0, 0, 0, 0);
    reinterpret_cast<uint4*>(bins)[kSampleThreads + threadIdx.x] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }

  // A bin of masses: the sums of their lower 16 and of their upper 10 bits.
  static __device__ __forceinline__ u64 mass_of(u64 bin) { return (uint32_t)bin + (u64)(uint32_t)(bin >> 32) * 65536u; }

  // The 8 threads of a coarse bin add up its sums; all of them get it.
  template <typename U>
  __device__ __forceinline__ U coarse_sum(const u64* bins) const {
    static_assert(kBins / kSampleThreads == 4 && kFine == 32, "four bins a thread, 8 threads a coarse bin");
    U s;
    if constexpr (sizeof(U) == 8) {
      const ulonglong2 l = reinterpret_cast<const ulonglong2*>(bins)[2 * threadIdx.x];
      const ulonglong2 h = reinterpret_cast<const ulonglong2*>(bins)[2 * threadIdx.x + 1];
      s = mass_of(l.x) + mass_of(l.y) + mass_of(h.x) + mass_of(h.y);
    } else {
      const uint4 l = reinterpret_cast<const uint4*>(bins)[threadIdx.x];
      s = l.x + l.y + l.z + l.w;
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
  }

  // Masses: codes in a bin have the same upper 6 bits, so their weights are as the
  // lower 26, and those are what is added up, in two halves that do not overflow (a
  // CTA has under 2^16 codes).  (Sums of the weights in 64 bits, by halves with a
  // carry, take 2 us more of 31 for a wave of 16,384 codes a CTA; a 64-bit atomic is
  // a loop here: 98 us for 64 rows of 131,072.)
  template <bool MASS>
  __device__ __forceinline__ void count(u64* bins, uint32_t bin, uint32_t code) const {
    if (MASS) {
      uint32_t* at = reinterpret_cast<uint32_t*>(bins + bin);
      atomicAdd(at, code & 0xffffu);
      atomicAdd(at + 1, code >> 16 & 0x3ffu);
    } else {
      atomicAdd(reinterpret_cast<uint32_t*>(bins) + bin, 1u);
    }
  }

  // A step toward the border among the codes in descending order: the greatest
  // code at which the number of codes (MASS: the sum of their weights) at or above
  // it reaches the target, which is target(sum of all).  Step 0 finds its upper 11
  // bits, step 1 the next 11, step 2 the rest.  False: the target is never reached
  // (step 0 only).  `counted`: the histogram is made.  MASS: from the upper 6 bits on
  // all that is left has one exponent, and b->left and b->bin are in units of the
  // lower 26.
  template <bool MASS, typename F>
  __device__ __forceinline__ bool step(int pass, bool counted, F target_of, Border* b) {
    using U = typename std::conditional<MASS, u64, uint32_t>::type;
    const int tid = threadIdx.x, lane = tid & 31;
    if (!counted) {
      clear(sh.bins[hist]);
      if (pass == 0) {
        each([&](uint32_t c) {
          if (c >= least) count<MASS>(sh.bins[hist], c >> 21, c);
        });
      } else {
        const int shift = pass == 1 ? 21 : 10, low = pass == 1 ? 10 : 0;
        const uint32_t mask = pass == 1 ? 2047u : 1023u, prefix = b->prefix;
        each([&](uint32_t c) {
          if (c >> shift == prefix && c >= least) count<MASS>(sh.bins[hist], (c >> low) & mask, c);
        });
      }
    }
    __syncthreads();
    const u64* bins = sh.bins[hist];
    {
      const U s = coarse_sum<U>(bins);
      if ((tid & 7) < ctas) st_cluster64(&sh.coarse[buf][rank][tid >> 3], tid & 7, s);
    }
    cluster_barrier();
    {
      U s = (tid & 7) < ctas ? (U)sh.coarse[buf][tid & 7][tid >> 3] : (U)0;
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      // as weights: rounded down once for all of an exponent
      if (MASS && pass == 0) s = (tid >> 3) <= 44 ? (U)(((u64)s << 19) >> (44 - (tid >> 3))) : (U)0;
      if ((tid & 7) == 0) reinterpret_cast<U*>(sh.total)[tid >> 3] = s;
    }
    buf ^= 1;
    __syncthreads();
    U target = (U)b->left;
    if (pass == 0) {
      b->all = sum_warp((U)(reinterpret_cast<const U*>(sh.total)[lane] + reinterpret_cast<const U*>(sh.total)[lane + 32]));
      target = (U)target_of(b->all);
    }
    U above = 0;
    const int coarse = reach<kCoarse, U>(reinterpret_cast<const U*>(sh.total), target, &above);
    if (coarse < 0) {  // in all CTAs alike
      hist ^= 1;
      __syncthreads();
      return false;
    }
    target -= above;
    if (MASS && pass == 0) {  // the least sum of lower bits that weighs as much
      const int up = coarse - 25;
      target = up <= 0 ? (U)((u64)target << -up) : (U)(((u64)target + (1ull << up) - 1) >> up);
    }
    if (tid < 8 * kFine) {
      const int bin = coarse * kFine + (tid >> 3);
      U s = 0;
      if ((tid & 7) < ctas) {
        if constexpr (MASS) s = mass_of(ld_cluster64(bins + bin, tid & 7));
        else s = ld_cluster32(reinterpret_cast<const uint32_t*>(bins) + bin, tid & 7);
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if ((tid & 7) == 0) reinterpret_cast<U*>(sh.fine)[tid >> 3] = s;
    }
    __syncthreads();
    const int fine = reach<kFine, U>(reinterpret_cast<const U*>(sh.fine), target, &above);
    b->left = target - above;
    b->bin = reinterpret_cast<const U*>(sh.fine)[fine];
    b->prefix = (pass == 0 ? 0u : b->prefix << (pass == 2 ? 10 : 11)) | (uint32_t)(coarse * kFine + fine);
    hist ^= 1;
    return true;
  }

  // The codes that want(code) picks, of all CTAs, into each CTA's list: each CTA's
  // own part of it, sh.listed (of before buf turned) long.  False: one has too many.
  template <typename F>
  __device__ __forceinline__ bool gather(F want) {
    const int tid = threadIdx.x, lane = tid & 31;
    const uint4* mine = codes + lane;
    static_assert(kFew >= kListed, "sh.key holds them");
    u64* own = sh.key;  // this CTA's, before they go to all
    for (int g = 0; g < groups; ++g) {
      const uint4 v = mine[g * 32];
      const uint32_t c[4] = {v.x, v.y, v.z, v.w};
      bool any = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) any = any || (c[k] >= least && want(c[k]));
      if (!any) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c[k] >= least && want(c[k])) {
          const int at = atomicAdd(&sh.mine, 1);
          if (at < kListed) own[at] = order_key(c[k], first + g * 128 + lane * 4 + k);
        }
    }
    __syncthreads();
    for (int i = tid; i < min(sh.mine, kListed) * ctas; i += kSampleThreads) {
      const int r = i % ctas, at = i / ctas;
      st_cluster64(sh.bins[hist] + rank * kListed + at, r, own[at]);
    }
    if (tid < ctas) st_cluster32(&sh.listed[buf][rank], tid, (uint32_t)sh.mine);
    cluster_barrier();
    if (tid == 0) sh.mine = sh.few = 0, sh.lowest = 0xffffffffu, sh.highest = 0u;
    if (tid < 8) sh.tied[tid] = 0;
    const bool over = __any_sync(0xffffffffu, lane < ctas && sh.listed[buf][lane] > kListed);
    buf ^= 1;
    __syncthreads();
    return !over;
  }

  template <typename F>
  __device__ __forceinline__ void each_listed(F f) const {
    static_assert(8 * 64 == kSampleThreads && kListed % 64 == 0, "64 threads a CTA's part");
    const int r = threadIdx.x >> 6;
    const u64* list = sh.bins[hist] + r * kListed;
    if (r < ctas)
      for (int i = threadIdx.x & 63; i < sh.listed[buf ^ 1][r]; i += 64) f(list[i]);
  }

  // Those of the list that want(code) picks into sh.key and sh.share, in any order;
  // their number, which may be above kFew; the least and greatest of them.
  template <typename F>
  __device__ __forceinline__ int pick(F want) const {
    each_listed([&](u64 key) {
      if (want(key_code(key))) {
        const int at = atomicAdd(&sh.few, 1);
        if (at < kFew) sh.key[at] = key, sh.share[at] = code_weight(key_code(key));
        atomicMin(&sh.lowest, key_code(key));
        atomicMax(&sh.highest, key_code(key));
      }
    });
    __syncthreads();
    return sh.few;
  }

  // The border, once its upper bits are known: `least` becomes its code, and codes
  // equal to it that come after it in the row are dropped.  Where the codes with
  // its upper bits are not too many, each CTA gets them all and goes on by itself:
  // a histogram of the next bits, and the few of its bin compared with each other.
  template <bool MASS>
  __device__ __forceinline__ void settle(Border b) {
    using U = typename std::conditional<MASS, u64, uint32_t>::type;
    const int tid = threadIdx.x;
#pragma unroll 1
    for (int pass = 1; pass <= 2; ++pass) {
      const int shift = pass == 1 ? 21 : 10, low = pass == 1 ? 10 : 0;
      const uint32_t prefix = b.prefix, mask = pass == 1 ? 2047u : 1023u;
      const u64 w = MASS ? mass(prefix << shift) : 1ull;  // no code with the prefix has less
      if (w > 0 && b.bin <= w * kPicked && gather([&](uint32_t c) { return c >> shift == prefix; })) {
        U left = (U)b.left;
        uint32_t bin = 0xffffffffu;  // all
        if (b.bin > w * 16) {
          u64* bins = sh.bins[hist ^ 1];  // read by nobody since the barrier of gather
          clear(bins);
          each_listed([&](u64 key) {
            const uint32_t c = key_code(key);
            count<MASS>(bins, (c >> low) & mask, c);
          });
          __syncthreads();
          const U s = coarse_sum<U>(bins);
          if ((tid & 7) == 0) reinterpret_cast<U*>(sh.total)[tid >> 3] = s;
          __syncthreads();
          U above = 0;
          const int coarse = reach<kCoarse, U>(reinterpret_cast<const U*>(sh.total), left, &above);
          left -= above;
          if (tid < kFine) {
            if constexpr (MASS) reinterpret_cast<U*>(sh.fine)[tid] = mass_of(bins[coarse * kFine + tid]);
            else reinterpret_cast<U*>(sh.fine)[tid] = reinterpret_cast<const uint32_t*>(bins)[coarse * kFine + tid];
          }
          __syncthreads();
          const int fine = reach<kFine, U>(reinterpret_cast<const U*>(sh.fine), left, &above);
          left -= above;
          bin = (uint32_t)(coarse * kFine + fine);
        }
        const int n = pick([&](uint32_t c) { return bin == 0xffffffffu || ((c >> low) & mask) == bin; });
        // (160 equal ones 0.6 us so, 9 compared with each other)
        if (n > 8 && sh.lowest == sh.highest) {  // one code many times (logits of 16 bits): the first few in the row stay
          const uint32_t code = sh.lowest;
          const U w = MASS ? (U)mass(code) : (U)1;
          const int keep = (int)((left + w - 1) / w);
          least = code;
          if (keep >= n) return;
          each_listed([&](u64 key) {
            if (key_code(key) == code) atomicAdd(sh.tied + (tid >> 6), 1);
          });
          __syncthreads();
          int r = 0, before = 0;  // the CTA whose part has it; CTAs are in the row's order
          while (before + sh.tied[r] < keep) before += sh.tied[r++];
          const u64* list = sh.bins[hist] + r * kListed;
          const int listed = sh.listed[buf ^ 1][r];
          if (tid < listed && key_code(list[tid]) == code) {
            int ahead = before;
            for (int i = 0; i < listed; ++i) ahead += key_code(list[i]) == code && list[i] > list[tid];
            if (ahead == keep - 1) sh.found = key_index(list[tid]);
          }
          __syncthreads();
          const int last = sh.found;
          __syncthreads();
          drop(last);
          return;
        }
        if (n <= kFew / 2) {
          if (tid < n) {
            const u64 key = sh.key[tid], own = MASS ? mass(key_code(key)) : 1ull;
            u64 before = 0;
            bool ties = false;
            for (int i = 0; i < n; ++i) {
              const u64 k = sh.key[i];
              if (k > key) before += MASS ? mass(key_code(k)) : 1ull;
              ties = ties || (k < key && key_code(k) == key_code(key));
            }
            if (before < left && before + own >= left) {
              sh.warp[0] = key;
              sh.ties = ties;
            }
          }
          __syncthreads();
          const u64 key = sh.warp[0];
          const bool ties = sh.ties != 0;
          __syncthreads();
          least = key_code(key);
          if (ties) drop(key_index(key));
          return;
        }
        __syncthreads();
      }
      step<MASS>(pass, false, [](u64) { return 0ull; }, &b);
    }
    // one code: the first few in the row stay
    const u64 w = MASS ? mass(b.prefix) : 1ull, keep = (b.left + w - 1) / w;
    least = b.prefix;
    if (keep >= b.bin / w) return;
    const uint32_t at = least;
    const auto is = [&](uint32_t v) { return (u64)(v == at); };
    u64 n = 0, before, own;
    each([&](uint32_t v) { n += v == at; });
    sums(n, &before, &own);
    const u64 want = keep - 1;
    if (want >= before && want < before + own) {
      int place;
      uint32_t code;
      if (locate(is, want - before, &place, &code))
        for (int k = 0; k < ctas; ++k) st_cluster32(&sh.found, k, (uint32_t)(first + place));
    }
    cluster_barrier();
    const int last = *reinterpret_cast<volatile int*>(&sh.found);
    cluster_barrier();  // read before another border writes it
    drop(last);
  }

  // Codes equal to `least` after index `last` are dropped.
  __device__ __forceinline__ void drop(int last) {
    const int lane = threadIdx.x & 31;
    uint4* mine = codes + lane;
    for (int g = 0; g < groups; ++g) {
      uint4 v = mine[g * 32];
      const int p = first + g * 128 + lane * 4;
      if (v.x == least && p > last) v.x = 0u;
      if (v.y == least && p + 1 > last) v.y = 0u;
      if (v.z == least && p + 2 > last) v.z = 0u;
      if (v.w == least && p + 3 > last) v.w = 0u;
      mine[g * 32] = v;
    }
    __syncwarp();
  }

  // Sum over the row of the threads' s, and what lies in the CTAs and warps before
  // this one.
  __device__ __forceinline__ u64 sums(u64 s, u64* before_warp, u64* own_warp) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    s = sum_warp(s);
    if (lane == 0) sh.warp[warp] = s;
    __syncthreads();
    const u64 mine = lane < kSampleWarps ? sh.warp[lane] : 0ull;
    const u64 cta = sum_warp(mine), before = sum_warp(lane < warp ? mine : 0ull);
    if (tid < ctas) st_cluster64(&sh.cta[buf][rank], tid, cta);
    cluster_barrier();  // and sh.warp is free
    const u64 theirs = lane < ctas ? sh.cta[buf][lane] : 0ull;
    buf ^= 1;
    *before_warp = sum_warp(lane < rank ? theirs : 0ull) + before;
    *own_warp = s;
    return sum_warp(theirs);
  }

  // In the warp that holds it: the element, in index order, at which the sum of
  // value(code) goes past `target` (counted from this warp's first), in the lane
  // that finds it; its place among the warp's elements, and its code.  A lane adds
  // up its share of neighbours first, then the warp looks into one share.
  template <typename F>
  __device__ __forceinline__ bool locate(F value, u64 target, int* place, uint32_t* at_code) const {
    const int lane = threadIdx.x & 31;
    u64 s = 0;
    int i = lane % groups;
    for (int n = 0; n < groups; ++n) {  // lanes begin at different places: fewer of them at one bank
      const uint4 v = codes[lane * groups + i];
      i = i + 1 < groups ? i + 1 : 0;
      s += value(v.x) + value(v.y) + value(v.z) + value(v.w);
    }
    const u64 incl = scan_warp(s);
    const int l = __ffs(__ballot_sync(0xffffffffu, target < incl)) - 1;
    target -= __shfl_sync(0xffffffffu, incl - s, l);
    const uint32_t* share = reinterpret_cast<const uint32_t*>(codes + l * groups);
    for (int i0 = 0; i0 < 4 * groups; i0 += 32) {
      const int i = i0 + lane;
      const uint32_t c = i < 4 * groups ? share[i] : 0u;
      const u64 v = value(c), sum = scan_warp(v);
      const u64 all = __shfl_sync(0xffffffffu, sum, 31);  // before any lane leaves
      if (target < all) {
        *place = l * 4 * groups + i;
        *at_code = c;
        return target < sum && target >= sum - v;
      }
      target -= all;
    }
    return false;
  }
};

template <typename T>
struct Logits;
template <>
struct Logits<float> {
  static constexpr int VEC = 4;
  static __device__ __forceinline__ void load(const float* p, float* x) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p));
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  }
  static __device__ __forceinline__ float one(const float* p) { return __ldg(p); }
};
template <>
struct Logits<__nv_bfloat16> {
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* x) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};

// The filters and the draw among n tokens (sh.key, sh.share) that hold the row's
// top_k: one a thread, each compared with all.
template <typename S, typename W>
__device__ __forceinline__ void sample_few(SampleShared& sh, int n, int top_k, float top_p, u64 least, float u, S share_up, W write) {
  const int tid = threadIdx.x;
  const auto total = [&](u64 v) {  // over the block
    v = sum_warp(v);
    __syncthreads();
    if ((tid & 31) == 0) sh.warp[tid >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < kFew / 32; ++i) v += sh.warp[i];
    return v;
  };
  u64 key = 0, w = 0, before = 0;
  int ahead = 0;
  if (tid < n) {
    key = sh.key[tid];
    w = sh.share[tid];
    for (int i = 0; i < n; ++i) {
      if (sh.key[i] > key) {
        before += sh.share[i];
        ++ahead;
      }
    }
  }
  if (ahead >= top_k) w = 0;
  if (top_p < 1.0f) {
    const u64 all = total(w), t = share_up(all, top_p);
    if (before >= (t == 0 ? 1ull : t)) w = 0;
  }
  if (w < least) w = 0;
  const u64 all = total(w);
  if (tid < n) sh.share[tid] = w;
  __syncthreads();
  bool more;
  const u64 target = u < 1.0f ? share(all, u, &more) : all - 1;
  if (w == 0) return;
  before = 0;
  for (int i = 0; i < n; ++i)
    if (key_index(sh.key[i]) < key_index(key)) before += sh.share[i];
  if (target >= before && target < before + w) write(key_index(key), w, all);
}

// A warp holds 128 `groups` neighbours (a multiple of 32 VEC), so that (CTA, warp,
// place) is the vocabulary's order.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a, int ctas, int groups) {
  constexpr int VEC = Logits<T>::VEC;
  extern __shared__ uint4 s_codes[];
  __shared__ __align__(16) SampleShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / ctas, rank = blockIdx.x - row * ctas;

  // no CTA's shared memory is written by another before that one has started
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");

  // A row begins anywhere: its first vector is the aligned one that holds its
  // first element, and elements before it are none.
  const T* base = static_cast<const T*>(a.logits) + (long long)row * a.stride;
  const int skip = (int)((reinterpret_cast<uintptr_t>(base) & 15) / sizeof(T));
  const int per = 128 * groups, first = (rank * kSampleWarps + warp) * per - skip;  // the warp's first element
  uint4* codes = s_codes + warp * (32 * groups);
  float top = -INFINITY;
#pragma unroll 4
  for (int g = 0; g < per / (32 * VEC); ++g) {
    const int i = first + (g * 32 + lane) * VEC;
    float x[VEC];
    if (i >= 0 && i + VEC <= a.vocab) {
      Logits<T>::load(base + i, x);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[k] = i + k >= 0 && i + k < a.vocab ? Logits<T>::one(base + i + k) : -INFINITY;
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      top = max_nan(top, x[k]);
    }
#pragma unroll
    for (int k = 0; k < VEC; k += 4)
      codes[(g * 32 + lane) * (VEC / 4) + k / 4] =
          make_uint4(__float_as_uint(x[k]), __float_as_uint(x[k + 1]), __float_as_uint(x[k + 2]), __float_as_uint(x[k + 3]));
  }
  for (int i = tid; i < kBins; i += kSampleThreads) sh.bins[0][i] = 0;
  if (tid < 32) sh.pow[tid] = power_entry(tid);
  if (tid == 0) sh.mine = sh.few = 0;

  const float temperature = a.temperature == nullptr ? a.temperature0 : a.temperature[row];
  const float top_p = a.top_p == nullptr ? a.top_p0 : a.top_p[row];
  const float min_p = a.min_p == nullptr ? a.min_p0 : a.min_p[row];
  const float u = a.u[row];
  int top_k = a.top_k == nullptr ? a.top_k0 : a.top_k[row];
  if (temperature == 0.0f) top_k = 1;
  if (tid == kSampleThreads - 1) {  // double precision is slow: by one thread, beside the others' loads
    const float before = temperature > 0x1p96f ? 0x1p-64f : 1.0f, after = temperature < 0x1p-96f ? 0x1p64f : 1.0f;
    const double c = 1.4426950408889634 / (double)(temperature * before * after);  // exact; T = 0: not used
    sh.scale[0] = (float)c;
    sh.scale[1] = (float)(c - (double)sh.scale[0]);
    sh.scale[2] = before;
    sh.scale[3] = after;
  }
  if (top_k >= a.vocab || top_k < 0) top_k = 0;
  if (a.vocab == 1) top_k = 1;

  // Logits under the `bound` do not belong to the top_k: of the warps that are
  // filled, each has r lanes with a logit at or above it, and r times their number
  // is top_k or more.
  float bound = -INFINITY;
  if (top_k > 1) {
    const int full = max(0, (a.vocab + skip) / per - (skip > 0 ? 1 : 0));
    const int r = full == 0 ? 33 : (top_k + full - 1) / full;
    if (r <= 32 && first >= 0 && first + per <= a.vocab) {
      int above = 0;
#pragma unroll 8
      for (int l = 0; l < 32; ++l) {
        const float v = __shfl_sync(0xffffffffu, top, l);
        above += v > top || (v == top && l < lane);
      }
      const unsigned at = __ballot_sync(0xffffffffu, above == r - 1);
      bound = __shfl_sync(0xffffffffu, top, at == 0 ? 0 : __ffs(at) - 1);
    } else if (r <= 32) {
      bound = INFINITY;  // says nothing
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) sh.warp[warp] = (u64)__float_as_uint(top) << 32 | __float_as_uint(bound);
  __syncthreads();
  __syncwarp();
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (warp == 0) {
    const u64 v = sh.warp[lane & (kSampleWarps - 1)];
    top = __uint_as_float((uint32_t)(v >> 32));
    bound = __uint_as_float((uint32_t)v);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
      bound = fminf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
    }
    if (lane < ctas) st_cluster64(&sh.cta[0][rank], lane, (u64)__float_as_uint(top) << 32 | __float_as_uint(bound));
  }
  cluster_barrier();
  {
    const u64 v = sh.cta[0][lane < ctas ? lane : 0];
    top = __uint_as_float((uint32_t)(v >> 32));
    bound = __uint_as_float((uint32_t)v);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
      bound = fminf(bound, __shfl_xor_sync(0xffffffffu, bound, o));
    }
    top = __shfl_sync(0xffffffffu, top, 0);
    bound = __shfl_sync(0xffffffffu, bound, 0);
  }
  const bool sound = temperature >= 0.0f && temperature <= kMostFloat && top_p >= 0.0f && min_p >= 0.0f && min_p <= 1.0f &&
                     u >= 0.0f && u <= 1.0f && fabsf(top) <= kMostFloat;
  if (!sound) {  // the cluster's CTAs alike; nothing of theirs is read from here on
    if (rank == 0 && tid == 0) {
      a.ids[row] = -1;
      if (a.logprobs != nullptr) a.logprobs[row] = __int_as_float(0x7fc00000);
    }
    return;
  }

  Row r{sh, codes, groups, first, ctas, rank, 1, 0, 1u};
  uint4* mine = codes + lane;
  u64 before, own, sum = 0;
  const auto kept = [&](uint32_t v) { return v >= r.least ? code_weight(v) : 0ull; };
  const auto share_up = [](u64 all, float f) {  // of `all`, rounded up
    if (f >= 1.0f) return all;
    bool more;
    const u64 t = share(all, f, &more);
    return t + (more ? 1ull : 0ull);
  };
  const auto logprob = [](u64 w, u64 all) {  // fp32: the quotient, and its distance from 1 where that is small
    return w > all / 2 ? log1pf(-((float)(all - w) / (float)all)) : logf((float)w / (float)all);
  };
  if (top_k == 1) {  // the greatest alone
    constexpr uint32_t kOne = (44u << 26) + (1u << 25);
    for (int g = 0; g < groups; ++g) {
      uint4 c = mine[g * 32];
      c.x = __uint_as_float(c.x) == top ? kOne : 0u;
      c.y = __uint_as_float(c.y) == top ? kOne : 0u;
      c.z = __uint_as_float(c.z) == top ? kOne : 0u;
      c.w = __uint_as_float(c.w) == top ? kOne : 0u;
      mine[g * 32] = c;
      sum += code_weight(c.x) + code_weight(c.y) + code_weight(c.z) + code_weight(c.w);
    }
  } else {
    RowScale s;
    s.before = sh.scale[2];
    s.after = sh.scale[3];
    s.top = top * s.before;
    s.ch = sh.scale[0];
    s.cl = sh.scale[1];
    s.y = __fmul_rn(top, s.ch);
    s.whole = (44u << 26) - ((__float_as_uint(fmaf(s.y, 32.0f, kRoundMagic)) - kRoundBits) * (1u << 21) & 0xfc000000u);
    const bool mass = top_k == 0 && top_p < 1.0f, plain = top_k == 0 && !mass, bounded = bound > -INFINITY;
    const bool near = fabsf(s.y) <= 4096.0f && temperature >= 0x1p-96f && temperature <= 0x1p96f;
    const auto each_code = [&](auto is_near, auto is_bounded, auto take) {
      constexpr bool NEAR = decltype(is_near)::value, BOUNDED = decltype(is_bounded)::value;
#pragma unroll 2
      for (int g = 0; g < groups; ++g) {
        const uint4 v = mine[g * 32];
        const float x[4] = {__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
        uint32_t o[4] = {0u, 0u, 0u, 0u};
        if (!BOUNDED || __any_sync(0xffffffffu, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= bound)) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            o[k] = !BOUNDED || x[k] >= bound ? weight_code<NEAR>(x[k], s, sh.pow) : 0u;
            if (o[k] != 0u) take(o[k]);
          }
        }
        mine[g * 32] = make_uint4(o[0], o[1], o[2], o[3]);
      }
    };
    const auto codes_of = [&](auto take) {  // the greatest's as well
      uint32_t greatest;
      if (near) {
        if (bounded) each_code(std::true_type(), std::true_type(), take);
        else each_code(std::true_type(), std::false_type(), take);
        greatest = weight_code<true>(top, s, sh.pow);
      } else {
        each_code(std::false_type(), std::true_type(), take);
        greatest = weight_code<false>(top, s, sh.pow);
      }
      return greatest;
    };
    uint32_t greatest;
    if (mass) greatest = codes_of([&](uint32_t v) { r.count<true>(sh.bins[0], v >> 21, v); });
    else if (!plain) greatest = codes_of([&](uint32_t v) { r.count<false>(sh.bins[0], v >> 21, v); });
    else greatest = codes_of([&](uint32_t v) { sum += code_weight(v); });
    const u64 light = min_p > 0.0f ? share_up(code_weight(greatest), min_p) : 0ull;  // lighter ones are dropped at the end

    Border b;
    if (top_k > 1) {
      const bool found = r.step<false>(0, true, [&](u64) { return (u64)top_k; }, &b);
      const u64 most = found ? (u64)top_k - b.left + b.bin : b.all;
      if (most <= kFew) {
        // few enough that they are all looked at one by one, by the first CTA alone
        const uint32_t from = found ? b.prefix << 21 : 1u;
        if (r.gather([&](uint32_t v) { return v >= from; })) {
          if (rank == 0) sample_few(sh, r.pick([](uint32_t) { return true; }), top_k, top_p, light, u, share_up, [&](int id, u64 w, u64 all) {
            a.ids[row] = id;
            if (a.logprobs != nullptr) a.logprobs[row] = logprob(w, all);
          });
          return;
        }
      }
      if (found) r.settle<false>(b);
    }
    if (top_p < 1.0f) {
      const auto target = [&](u64 all) {
        const u64 t = share_up(all, top_p);
        return t == 0 ? 1ull : t;
      };
      if (r.step<true>(0, mass, target, &b)) r.settle<true>(b);
    }
    if (light > 0) {
      // Weights are compared, not codes: next to a power of two a code of one exponent
      // may stand for as much as the next one's codes, or more (power_code).
      const auto heavy = [&](uint32_t v) { return v >= r.least && code_weight(v) >= light ? v : 0u; };
      sum = 0;
      for (int g = 0; g < groups; ++g) {
        uint4 c = mine[g * 32];
        c.x = heavy(c.x), c.y = heavy(c.y), c.z = heavy(c.z), c.w = heavy(c.w);
        mine[g * 32] = c;
        sum += code_weight(c.x) + code_weight(c.y) + code_weight(c.z) + code_weight(c.w);
      }
    } else if (!plain) {
      sum = 0;
      r.each([&](uint32_t v) { sum += kept(v); });
    }
  }
  const u64 all = r.sums(sum, &before, &own);
  bool more;
  const u64 target = top_k == 1 ? 0ull : u < 1.0f ? share(all, u, &more) : all - 1;
  if (target >= before && target < before + own) {
    int place;
    uint32_t got;
    if (r.locate(kept, target - before, &place, &got)) {
      a.ids[row] = first + place;
      if (a.logprobs != nullptr) a.logprobs[row] = top_k == 1 ? 0.0f : logprob(code_weight(got), all);
    }
  }
}

template <typename T>
cudaError_t sample_config(int rows, int ctas, int groups, cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attr) {
  static std::atomic<unsigned long long> done{0};
  *cfg = {};
  attr->id = cudaLaunchAttributeClusterDimension;
  attr->val.clusterDim.x = ctas;
  attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
  cfg->gridDim = dim3((unsigned)rows * ctas);
  cfg->blockDim = dim3(kSampleThreads);
  cfg->dynamicSmemBytes = kSampleWarps * 512 * groups;
  cfg->attrs = attr;
  cfg->numAttrs = 1;
  return smem_attr_once(sample_kernel<T>, kSampleWarps * 512 * kSampleMaxGroups, done);
}

template <typename T>
cudaError_t sample_at_once(int ctas, int groups, int* clusters) {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  const cudaError_t e = sample_config<T>(1, ctas, groups, &cfg, attr);
  return e != cudaSuccess ? e : cudaOccupancyMaxActiveClusters(clusters, sample_kernel<T>, &cfg);
}

template <typename T>
cudaError_t sample_as(const SampleArgs& a, int ctas, int groups, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[1];
  const cudaError_t e = sample_config<T>(a.rows, ctas, groups, &cfg, attr);
  if (e != cudaSuccess) return e;
  cfg.stream = s;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a, ctas, groups);
}

template <typename T>
cudaError_t sample_any(const SampleArgs& a, cudaStream_t s) {
  constexpr int kVec = 16 / (int)sizeof(T);
  const bool even = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && (a.rows == 1 || a.stride % kVec == 0);
  // The CTAs of a row, by what a wave of them costs (us, measured with top-p): 10,
  // and 1.4 for each group of a warp, 2.2 where two CTAs share an SM.  Rows differ,
  // so the next wave begins before one ends: a third whole waves, two thirds parts
  // of them.  250 rows of 32,000 by 1, 2, 3, 4, 8 CTAs: 81, 64, 79, 81, 129 us; one
  // row by 2, 4, 8: 14.1, 12.1, 11.3.
  static PerDevice<2 * 9> at_once;  // clusters of so many CTAs, one or two an SM, that run together
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const auto ask = [&](int two, int ctas, int* clusters) {
    return at_once.get(dev, two * 9 + ctas, clusters, [&](int* n) {
      const cudaError_t e = sample_at_once<T>(ctas, two ? kSampleTwoGroups : kSampleMaxGroups, n);
      if (*n < 1) *n = 1;
      return e;
    });
  };
  e = ask(0, 1, &sms);
  if (e != cudaSuccess) return e;
  const int most = a.vocab + (even ? 0 : kVec - 1);  // with what a row's first vector skips
  const int unit = 32 * kVec;                        // of a warp
  int best = 0, best_groups = 0;
  float least = 0.0f;
  for (int ctas = 1; ctas <= 8; ++ctas) {
    const int per = ctas * kSampleWarps * unit, groups = (most + per - 1) / per * (unit / 128);
    if (groups > kSampleMaxGroups) continue;
    const int two = groups <= kSampleTwoGroups;
    int fit = 0;
    e = ask(two, ctas, &fit);
    if (e != cudaSuccess) return e;
    const float waves = a.rows <= fit ? 1.0f : ((a.rows + fit - 1) / fit + 2.0f * a.rows / fit) / 3.0f;
    const float cost = waves * (10.0f + (two && (long long)a.rows * ctas > sms ? 2.2f : 1.4f) * groups);
    if (best == 0 || cost < least) best = ctas, best_groups = groups, least = cost;
  }
  return sample_as<T>(a, best, best_groups, s);
}

}  // namespace
}  // namespace msi

using namespace msi;

extern "C" msi_status msi_sample(const msi_sample_args* g, msi_stream stream) {
  if (g == nullptr || g->rows < 0 || g->vocab < 1 || (g->type != MSI_BF16 && g->type != MSI_F32)) return MSI_ERR_INVALID_ARG;
  if (g->vocab > kSampleMaxVocab || g->rows > 1 << 24) return MSI_ERR_UNSUPPORTED;
  if ((g->temperatures == nullptr && !(g->temperature >= 0.0f && isfinite(g->temperature))) ||
      (g->top_ps == nullptr && !(g->top_p >= 0.0f)) ||
      (g->min_ps == nullptr && !(g->min_p >= 0.0f && g->min_p <= 1.0f)))
    return MSI_ERR_INVALID_ARG;
  if (g->rows == 0) return MSI_OK;
  const uintptr_t size = g->type == MSI_F32 ? 4 : 2;
  if (g->logits == nullptr || (reinterpret_cast<uintptr_t>(g->logits) & (size - 1)) != 0 || g->stride < 0 ||
      g->u == nullptr || g->ids == nullptr)
    return MSI_ERR_INVALID_ARG;
  SampleArgs a = {};
  a.logits = g->logits;
  a.stride = g->stride;
  a.rows = g->rows;
  a.vocab = g->vocab;
  a.u = g->u;
  a.temperature = g->temperatures;
  a.top_k = g->top_ks;
  a.top_p = g->top_ps;
  a.min_p = g->min_ps;
  a.temperature0 = g->temperature;
  a.top_k0 = g->top_k;
  a.top_p0 = g->top_p;
  a.min_p0 = g->min_p;
  a.ids = g->ids;
  a.logprobs = g->logprobs;
  const cudaError_t e = g->type == MSI_F32 ? sample_any<float>(a, stream) : sample_any<__nv_bfloat16>(a, stream);
  return e == cudaSuccess ? MSI_OK : note_cuda_error(e, "msi_sample");
}
