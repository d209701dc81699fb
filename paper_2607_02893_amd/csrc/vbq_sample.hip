// The choice of a token on gfx950 (MI355X) from a row of logits: temperature, top-k,
// top-p and min-p, with the random number given.
//
// With z_max the row's largest logit, w_i = exp((z_i - z_max) / T).  Every limit keeps
// a prefix of the tokens in descending order (the lower index first among equals):
// the first k; of those the shortest prefix whose w sum to p times their sum; those
// with w >= min_p.  The token is the first, in index order, at which the running sum of
// the kept w exceeds u times their total.
//
// Which token a number lands on depends on sums over the whole vocabulary, so the w are
// held as whole multiples of 2^-43 (64-bit integers): their sums are exact in any
// order, and a result does not depend on how a row was spread over lanes.
//
// A row is 32 to 512 KB and its steps depend on each other (largest logit, weights,
// where the limits cut, their total, the token), so the latency of that chain bounds
// the call, not its bytes.  Rows up to kCap logits: one workgroup holds the row in LDS.
// Longer ones: four launches, three of them with each row spread over up to kMaxChunks
// workgroups:
//   most    the largest logit of each chunk;
//   bins    (top-k or top-p) counts and sums of the weights by x = (z - z_max) / T in bins
//           of 1/16: they say in which bins the limits cut;
//   gather  sums of what is before those bins, and a list of what is in them;
//   token   one workgroup a row orders the list, finds the chunk that u falls into and the
//           token in it.
// In a graph 16 rows of 128256 fp32 logits with every kind of limit take 51 us (4.6 + 9.9 + 13 +
// 24), one of 32000 28 (3.8 + 6.6 + 8.4 + 10.7); one workgroup a row took 551 and 201.
// Launches rather than a row's last workgroup to arrive: that one needs the others' caches
// written back, which took 30 us with 32 workgroups and 75 with 256, a launch takes 2.
// Rows of 4096 logits take 9.6 us without a limit, 18 with top-k, 24 with top-p and 32 with both.
// Below x = -30.5 a weight is 0, so the bins end there.  A list that does not fit (more than kCap
// logits within 1/16 of T, equal or not: 262144 of standard deviation T, cut by top-p near
// their peak) sends its row through the row kernel's steps, over global memory, instead: 1.1 ms, where
// the same row with a standard deviation of 3 T takes 49 us.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/vbq.h"

vbq_status vbq_detail_hip_status(hipError_t e);

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024;
constexpr int kWavesRow = kThreads / 64;  // 16: a value a wave is a row of lanes
constexpr double kOne = 0x1p43;  // the weight of the largest logit; 2^20 of them are at most 2^63
constexpr double kLeast = -30.5; // below ln 2^-44 = -30.498 a weight rounds to 0
constexpr double kNone = -1e300;
constexpr int kBinsPerUnit = 16, kBins = 489;  // (the last holds x = kLeast alone)
constexpr int kDigitBits = 10, kDigits = 1 << kDigitBits;  // of a key, at a time
constexpr int kCap = 4096;       // entries of a list; rows up to this length take one workgroup
constexpr int kRanked = kThreads / 4;  // entries of a list that is ordered pair by pair
constexpr int kMaxChunks = 32;
constexpr int64_t kRowsAtOnce = 64;   // rows of a set of launches: bounds the workspace

struct SampleArgs {
  const void* z;
  int64_t ld;
  int32_t V, type;
  const float* temperature;  // each may be null
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* token;
  float* prob;               // may be null
};

// Logits as whole numbers in the same order; 0 for what is no candidate (NaN, -inf).
__device__ __forceinline__ uint32_t key_of(float z) {
  if (!(z > -__builtin_inff())) return 0;
  const uint32_t b = __float_as_uint(z + 0.0f);  // -0 is 0
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }

__device__ __forceinline__ uint32_t key_at(const SampleArgs& a, int64_t row, int i) {
  const int64_t at = row * a.ld + i;
  if (a.type == VBQ_F32) return key_of(((const float*)a.z)[at]);
  const uint16_t b = ((const uint16_t*)a.z)[at];
  return key_of(a.type == VBQ_F16 ? (float)__builtin_bit_cast(_Float16, b) : __uint_as_float((uint32_t)b << 16));
}

// e^x for x <= 0, within 2^-50: x = n ln 2 + r, |r| <= ln(2) / 2, and the series of e^r up to
// r^13 (the next term is below 2^-57).
__device__ __forceinline__ double exp_below(double x) {
  const double n = __builtin_rint(x * 1.4426950408889634074);
  const double r = __builtin_fma(n, -2.3190468138462996e-17, __builtin_fma(n, -0.69314718055994530942, x));
  double p = 1.0 / 6227020800.0;
  p = __builtin_fma(p, r, 1.0 / 479001600.0);
  p = __builtin_fma(p, r, 1.0 / 39916800.0);
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_ldexp(p, (int)n);
}

struct Weight {
  double top, per;  // z_max, 1 / T
  bool inf;         // z_max is +inf: its equals weigh 1, the others nothing
  __device__ __forceinline__ void set(uint32_t top_key, float t) {
    top = (double)logit_of(top_key);
    per = 1.0 / (double)t;
    inf = top == (double)__builtin_inff();
  }
  // (z - z_max) / T, kNone where the weight is 0
  __device__ __forceinline__ double x(uint32_t key) const {
    if (key == 0) return kNone;
    const double z = (double)logit_of(key);
    if (inf) return z == top ? 0.0 : kNone;
    const double v = (z - top) * per;
    return v >= kLeast ? v : kNone;
  }
  __device__ __forceinline__ double real(uint32_t key) const {
    const double v = x(key);
    return v == kNone ? 0.0 : exp_below(v);
  }
  // as whole(), 0 below min-p
  __device__ __forceinline__ uint64_t kept(uint32_t key, double least) const {
    const double v = real(key);
    return v >= least ? (uint64_t)__builtin_rint(v * kOne) : 0;
  }
  __device__ __forceinline__ uint64_t whole(uint32_t key) const { return (uint64_t)__builtin_rint(real(key) * kOne); }
  // the bin of a candidate with weight; kBins for others
  __device__ __forceinline__ int bin(uint32_t key) const {
    const double v = x(key);
    return v == kNone ? kBins : (int)(v * -(double)kBinsPerUnit);
  }
};

// Scans of a wave in registers: each step takes the value of the lane 1, 2, 4, 8 before within
// a row of 16, then the last of the row before, then of the first half (lanes without one: 0).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t from_lane(uint64_t v) {
  return ((uint64_t)from_lane<CTRL, ROWS>((uint32_t)(v >> 32)) << 32) | from_lane<CTRL, ROWS>((uint32_t)v);
}
template <typename T, typename Op>
__device__ __forceinline__ T row_scan(T v, Op op) {
  v = op(v, from_lane<0x111, 0xf>(v));
  v = op(v, from_lane<0x112, 0xf>(v));
  v = op(v, from_lane<0x114, 0xf>(v));
  return op(v, from_lane<0x118, 0xf>(v));
}
template <typename T, typename Op>
__device__ __forceinline__ T wave_scan(T v, Op op) {
  v = row_scan(v, op);
  v = op(v, from_lane<0x142, 0xa>(v));
  return op(v, from_lane<0x143, 0xc>(v));
}
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane) {
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return ((uint64_t)hi << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
struct Add {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Most {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; }
};

// What the limits keep of the descending order: the keys above `key` and the first `take`
// (by index) of those equal to it.
struct Cut {
  uint32_t key;
  uint64_t take;
  bool all;  // that is all of them
};

struct Limits {
  float t;
  int k;          // 0: none
  float p;        // 1: none
  double least;   // the smallest weight kept by min-p
  double u;
};

__device__ __forceinline__ Limits limits_of(const SampleArgs& a, int64_t row) {
  Limits l;
  l.t = a.temperature ? a.temperature[row] : 1.0f;
  l.k = a.top_k && a.top_k[row] > 0 && a.top_k[row] < a.V ? a.top_k[row] : 0;
  l.p = a.top_p && a.top_p[row] < 1.0f ? a.top_p[row] : 1.0f;
  l.p = l.p > 0.0f ? l.p : 0.0f;
  const float m = a.min_p && a.min_p[row] > 0.0f ? a.min_p[row] : 0.0f;
  l.least = m < 1.0f ? (double)m : 1.0;
  const float u = a.u[row];
  l.u = u > 0.0f ? (double)u : 0.0;
  return l;
}

// What a workgroup's steps share.
struct Shared {
  uint64_t weights[kDigits];
  uint32_t counts[kDigits];
  // one pair a wave, in turns: a value is read after one barrier and written again two calls later
  uint64_t wave[2][kWavesRow], wave2[2][kWavesRow];
  uint64_t above_w, above_c;
  uint32_t digit;
};

// A workgroup's sums and scans.
struct Block {
  Shared& sh;
  int turn = 0;
  __device__ explicit Block(Shared& s) : sh(s) {}

  template <typename Op>
  __device__ __forceinline__ void fold(uint64_t& a, uint64_t& b, Op op) {
    turn ^= 1;
    a = wave_scan(a, op);
    b = wave_scan(b, op);
    if ((threadIdx.x & 63) == 63) {
      sh.wave[turn][threadIdx.x >> 6] = a;
      sh.wave2[turn][threadIdx.x >> 6] = b;
    }
    __syncthreads();
    a = of_lane(row_scan(sh.wave[turn][threadIdx.x & 15], op), 15);
    b = of_lane(row_scan(sh.wave2[turn][threadIdx.x & 15], op), 15);
  }
  __device__ __forceinline__ uint64_t sum(uint64_t v) {
    uint64_t none = 0;
    fold(v, none, Add());
    return v;
  }
  __device__ __forceinline__ uint64_t most(uint64_t v) {
    uint64_t none = 0;
    fold(v, none, Most());
    return v;
  }
  // Sums of v and n over the threads before this one.
  __device__ __forceinline__ void before(uint64_t v, uint32_t n, uint64_t& v_before, uint64_t& n_before) {
    turn ^= 1;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint64_t s = wave_scan(v, Add());
    const uint32_t c = wave_scan(n, Add());
    if ((threadIdx.x & 63) == 63) {
      sh.wave[turn][wave] = s;
      sh.wave2[turn][wave] = c;
    }
    __syncthreads();
    const uint64_t vs = row_scan(sh.wave[turn][threadIdx.x & 15], Add()), ns = row_scan(sh.wave2[turn][threadIdx.x & 15], Add());
    v_before = s - v + (wave ? of_lane(vs, wave - 1) : 0);
    n_before = c - n + (wave ? of_lane(ns, wave - 1) : 0);
  }
  __device__ __forceinline__ uint64_t before(uint64_t v) {
    uint64_t b, none;
    before(v, 0, b, none);
    return b;
  }
};

// A running sum reaches its target: where it is at least `target`, a share of sums in double.
// A target is at least a half (the first weight that counts) and at most what there is.
__device__ __forceinline__ double target_within(double target, uint64_t all) {
  const double most = (double)all;
  return target < 0.5 ? 0.5 : target < most ? target : most;
}

// Where a limit cuts the keys key_at(0 .. n - 1) (0: none) of weights whole_at: k of them, or as many as
// sum to the target, `above_*` being what lies above all of them.  Ten bits of the key at a time, from the
// first bit in which the keys differ: a histogram, its running sums, the digit that reaches.
template <typename K, typename W>
__device__ __forceinline__ Cut cut_keys(Block& bl, int n, K key_at, W whole_at, const Weight& weight, bool by_count, uint64_t k,
                                        double target, uint64_t above_w, uint64_t above_c) {
  Shared& sh = bl.sh;
  uint64_t hi = 0, lo = 0;
#pragma unroll 1
  for (int i = (int)threadIdx.x; i < n; i += kThreads) {
    const uint32_t key = key_at(i);
    if (key) {
      hi = key > hi ? key : hi;
      lo = (uint32_t)~key > lo ? (uint32_t)~key : lo;
    }
  }
  bl.fold(hi, lo, Most());
  const uint32_t differ = (uint32_t)hi ^ ~(uint32_t)lo;
  const int bits = differ ? 32 - __builtin_clz(differ) : 1, digits = (bits + kDigitBits - 1) / kDigitBits;
  uint64_t prefix = hi >> (digits * kDigitBits);
#pragma unroll 1
  for (int shift = (digits - 1) * kDigitBits; shift >= 0; shift -= kDigitBits) {
    sh.weights[threadIdx.x] = 0;
    sh.counts[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = (int)threadIdx.x; i < n; i += kThreads) {
      const uint64_t key = key_at(i);
      if (key && (key >> (shift + kDigitBits)) == prefix) {
        const int at = (kDigits - 1) - (int)((key >> shift) & (kDigits - 1));
        atomicAdd(&sh.counts[at], 1u);
        if (!by_count) atomicAdd((unsigned long long*)&sh.weights[at], (unsigned long long)whole_at(i));
      }
    }
    __syncthreads();
    const uint64_t w = sh.weights[threadIdx.x];
    const uint32_t c = sh.counts[threadIdx.x];
    uint64_t wb, cb;
    bl.before(w, c, wb, cb);
    if (c && (by_count ? above_c + cb < k && above_c + cb + c >= k
                       : (double)(above_w + wb) < target && (double)(above_w + wb + w) >= target)) {
      sh.digit = (uint32_t)threadIdx.x;
      sh.above_w = above_w + wb;
      sh.above_c = above_c + cb;
    }
    __syncthreads();
    prefix = (prefix << kDigitBits) | ((kDigits - 1) - sh.digit);
    above_w = sh.above_w;
    above_c = sh.above_c;
  }
  // the equals of the cut's key weigh the same: as many as the limit takes, one at least
  const uint64_t ties = sh.counts[sh.digit];
  uint64_t take = ties;
  if (by_count) {
    take = k - above_c < ties ? k - above_c : ties;
  } else if (const uint64_t each = weight.whole((uint32_t)prefix)) {
    const double left = (target - (double)above_w) / (double)each;
    take = left >= (double)ties ? ties : left > 1.0 ? (uint64_t)__builtin_ceil(left) : 1;
  }
  return Cut{(uint32_t)prefix, take, take == ties};
}

__device__ __forceinline__ Cut shorter(const Cut& a, const Cut& b) {
  if (a.key != b.key) return a.key > b.key ? a : b;
  return a.take < b.take ? a : b;
}

// u times the total, below the total.
__device__ __forceinline__ double wanted(double u, uint64_t total) {
  const double below = (double)total * (1.0 - 0x1p-53), v = u * (double)total;
  return v <= below ? v : below;
}

__device__ __forceinline__ void write_token(const SampleArgs& a, int64_t row, int32_t token, float prob) {
  a.token[row] = token;
  if (a.prob) a.prob[row] = prob;
}

// Rows without candidates and greedy rows end here.
__device__ __forceinline__ bool ends_early(const SampleArgs& a, int64_t row, uint64_t best, float t) {
  if (best && t > 0.0f) return false;
  if (threadIdx.x == 0) write_token(a, row, best ? (int32_t)~(uint32_t)best : -1, best ? 1.0f : 0.0f);
  return true;
}

// A whole row by one workgroup, key_at(i) its keys in index order and whole_at(i) their weights.
template <typename K, typename W>
__device__ void choose(const SampleArgs& a, Block& bl, int64_t row, int n, K key_at, W whole_at, const Weight& w, const Limits& l) {
  Cut cut = {0, 0, true};
  uint64_t candidates = 0;
#pragma unroll 1
  for (int i = (int)threadIdx.x; i < n; i += kThreads) candidates += key_at(i) != 0;
  candidates = bl.sum(candidates);
#pragma unroll 1  // one copy of the steps' code: a workgroup alone waits for its instructions too
  for (int by_p = 0; by_p < 2; ++by_p) {
    if (by_p ? !(l.p < 1.0f) : !(l.k && (uint64_t)l.k < candidates)) continue;
    double target = 0.0;
    if (by_p) {
      uint64_t all = 0;
#pragma unroll 1
      for (int i = (int)threadIdx.x; i < n; i += kThreads) all += key_at(i) > cut.key ? whole_at(i) : 0;
      all = bl.sum(all) + cut.take * w.whole(cut.key);
      target = target_within((double)l.p * (double)all, all);
    }
    cut = shorter(cut_keys(bl, n, key_at, whole_at, w, !by_p, (uint64_t)l.k, target, 0, 0), cut);
  }
  // each thread sums a run of the row; the equals of the cut are kept in index order
  auto weigh = [&](uint32_t key) -> uint64_t { return key == 0 || key < cut.key ? 0 : w.kept(key, l.least); };
  const int per = (n + kThreads - 1) / kThreads;
  const int from = (int)threadIdx.x * per, to = from + per < n ? from + per : n;
  uint64_t sum = 0, ties = 0;
#pragma unroll 1
  for (int i = from; i < to; ++i) {
    const uint32_t key = key_at(i);
    if (cut.take && key == cut.key) ++ties;
    else sum += weigh(key);
  }
  const uint64_t ties_before = cut.take ? bl.before(ties) : 0;
  uint64_t left = cut.take > ties_before ? cut.take - ties_before : 0;
  const uint64_t tie_w = cut.take ? weigh(cut.key) : 0;
  sum += (ties < left ? ties : left) * tie_w;
  uint64_t run = bl.before(sum);
  const uint64_t total = bl.sum(sum);
  const double want = wanted(l.u, total);
  if (sum == 0 || (double)run > want || !((double)(run + sum) > want)) return;
#pragma unroll 1
  for (int i = from; i < to; ++i) {
    const uint32_t key = key_at(i);
    uint64_t own;
    if (cut.take && key == cut.key) {
      own = left ? tie_w : 0;
      left -= left ? 1 : 0;
    } else {
      own = weigh(key);
    }
    run += own;
    if (own && (double)run > want) {
      write_token(a, row, i, (float)((double)own / (double)total));
      return;
    }
  }
}

// Rows of up to kCap logits, held in LDS.
__global__ __launch_bounds__(kThreads) void vbq_sample_row_kernel(SampleArgs a) {
  __shared__ Shared sh;
  Block bl(sh);
  __shared__ uint32_t keys[kCap];
  __shared__ uint64_t whole[kCap];
  const int64_t row = blockIdx.x;
  uint64_t best = 0;
#pragma unroll 1
  for (int i = (int)threadIdx.x; i < a.V; i += kThreads) {
    const uint32_t key = key_at(a, row, i);
    keys[i] = key;
    const uint64_t v = key ? ((uint64_t)key << 32) | (uint32_t)~i : 0;
    best = v > best ? v : best;
  }
  best = bl.most(best);
  const Limits l = limits_of(a, row);
  if (ends_early(a, row, best, l.t)) return;
  Weight w;
  w.set((uint32_t)(best >> 32), l.t);
  if (l.p < 1.0f) {  // (each thread's own, as in every loop over all of them)
#pragma unroll 1
    for (int i = (int)threadIdx.x; i < a.V; i += kThreads) whole[i] = w.whole(keys[i]);
  }
  choose(a, bl, row, a.V, [&](int i) { return keys[i]; }, [&](int i) { return whole[i]; }, w, l);
}

// ------------------------------------------------------------------ long rows

// What a row's steps leave each other.
struct RowState {
  uint64_t best[kMaxChunks];    // per chunk: largest key and, inverted, its first index
  uint64_t sum[kMaxChunks];     // per chunk: kept weight before the bins in which the limits cut
  uint64_t bin_w[kBins];
  uint32_t bin_c[kBins];
  uint32_t listed;
  uint64_t list[kCap];          // key, index
};

struct LongArgs {
  SampleArgs s;
  RowState* state;
  int64_t row0;
  int32_t chunks, per;  // of a row; elements of a chunk
};

// The keys of elements i, i + kThreads, .. below `to`, all loads before the first use.
constexpr int kAhead = 4;
__device__ __forceinline__ void load_keys(const SampleArgs& a, int64_t row, int i, int to, uint32_t (&key)[kAhead]) {
#pragma unroll
  for (int j = 0; j < kAhead; ++j) key[j] = i + j * kThreads < to ? key_at(a, row, i + j * kThreads) : 0;
}

__global__ __launch_bounds__(kThreads) void vbq_sample_most_kernel(LongArgs a) {
  __shared__ Shared sh;
  Block bl(sh);
  const int chunk = (int)(blockIdx.x % a.chunks);
  const int64_t r = blockIdx.x / a.chunks;
  const int from = chunk * a.per, to = from + a.per < a.s.V ? from + a.per : a.s.V;
  uint64_t best = 0;
#pragma unroll 4
  for (int i = from + (int)threadIdx.x; i < to; i += kThreads) {
    const uint32_t key = key_at(a.s, a.row0 + r, i);
    const uint64_t v = key ? ((uint64_t)key << 32) | (uint32_t)~i : 0;
    best = v > best ? v : best;
  }
  best = bl.most(best);
  RowState& st = a.state[r];
  if (threadIdx.x == 0) st.best[chunk] = best;
  if (chunk == 0) {
#pragma unroll 1
    for (int i = (int)threadIdx.x; i < kBins; i += kThreads) {
      st.bin_w[i] = 0;
      st.bin_c[i] = 0;
    }
    if (threadIdx.x == 0) st.listed = 0;
  }
}

__device__ __forceinline__ uint64_t row_best(const RowState& st, int chunks) {
  uint64_t best = 0;
  for (int j = 0; j < chunks; ++j) best = st.best[j] > best ? st.best[j] : best;
  return best;
}

// Counts and sums of the weights by bin, in LDS, then added to the row's.  A row that has only one
// of the limits needs only the one (top-p takes a sum for a count: nothing there or something).
__global__ __launch_bounds__(kThreads) void vbq_sample_bins_kernel(LongArgs a) {
  __shared__ uint64_t bin_w[kBins];
  __shared__ uint32_t bin_c[kBins];
  const int chunk = (int)(blockIdx.x % a.chunks), tid = (int)threadIdx.x;
  const int64_t r = blockIdx.x / a.chunks, row = a.row0 + r;
  RowState& st = a.state[r];
  const uint64_t best = row_best(st, a.chunks);
  const Limits l = limits_of(a.s, row);
  const bool by_w = l.p < 1.0f;
  if (best == 0 || !(l.t > 0.0f) || (l.k == 0 && !by_w)) return;
  Weight w;
  w.set((uint32_t)(best >> 32), l.t);
#pragma unroll 1
  for (int i = tid; i < kBins; i += kThreads) {
    bin_w[i] = 0;
    bin_c[i] = 0;
  }
  __syncthreads();
  const int from = chunk * a.per, to = from + a.per < a.s.V ? from + a.per : a.s.V;
  for (int i0 = from; i0 < to; i0 += kAhead * kThreads) {
    uint32_t key[kAhead];
    load_keys(a.s, row, i0 + tid, to, key);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int b = w.bin(key[j]);
      if (b < kBins) {
        if (l.k) atomicAdd(&bin_c[b], 1u);
        if (by_w) atomicAdd((unsigned long long*)&bin_w[b], (unsigned long long)w.whole(key[j]));
      }
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < kBins; i += kThreads) {
    if (bin_w[i]) atomicAdd((unsigned long long*)&st.bin_w[i], (unsigned long long)bin_w[i]);
    if (bin_c[i]) atomicAdd(&st.bin_c[i], bin_c[i]);
  }
}

// The bins in which the limits cut, from the row's bins.
struct Cuts {
  int k_bin;       // top-k cuts in this one (-1: nowhere)
  int p_lo, p_hi;  // top-p in one of these (-1: nowhere); which, depends on where in k_bin top-k cuts
  int definite;    // bins before this one are kept
  uint64_t k_above_c, k_above_w, p_above_w, all_w;
};

__device__ __forceinline__ Cuts find_cuts(Block& bl, const RowState& st, const Limits& l, Cuts* out) {
  const int i = (int)threadIdx.x;
  const bool by_w = l.p < 1.0f;
  const uint64_t w = by_w && i < kBins ? st.bin_w[i] : 0;
  const uint32_t c = l.k && i < kBins ? st.bin_c[i] : 0;
  uint64_t wb, cb;
  bl.before(w, c, wb, cb);
  Shared& sh = bl.sh;
  if (i == kThreads - 1) *out = Cuts{-1, -1, -1, kBins, 0, 0, 0, wb};  // (no bin is this thread's: all sums are before it)
  __syncthreads();
  if (c && cb < (uint64_t)l.k && cb + c >= (uint64_t)l.k) {  // (nowhere if there are fewer than k)
    out->k_bin = out->definite = i;
    out->k_above_c = cb;
    out->k_above_w = wb;
    sh.above_w = wb + w;
  }
  __syncthreads();
  if (by_w) {
    const uint64_t lo = out->k_bin < 0 ? out->all_w : out->k_above_w, hi = out->k_bin < 0 ? out->all_w : sh.above_w;
    const double t_lo = target_within((double)l.p * (double)lo, lo), t_hi = target_within((double)l.p * (double)hi, hi);
    if ((double)wb < t_hi && (double)(wb + w) >= t_hi) out->p_hi = i;
    if ((double)wb < t_lo && (double)(wb + w) >= t_lo) {
      out->p_lo = out->definite = i;
      out->p_above_w = wb;
    }
  }
  __syncthreads();
  return *out;
}

// Each chunk's sum of what is certainly kept, and the row's list of what lies in the cuts' bins.
__global__ __launch_bounds__(kThreads) void vbq_sample_gather_kernel(LongArgs a) {
  __shared__ Shared sh;
  Block bl(sh);
  __shared__ Cuts cuts;
  __shared__ uint64_t own[kCap];  // this chunk's entries of the list
  __shared__ uint32_t own_n, own_at;
  const int chunk = (int)(blockIdx.x % a.chunks), tid = (int)threadIdx.x, lane = tid & 63;
  const int64_t r = blockIdx.x / a.chunks, row = a.row0 + r;
  RowState& st = a.state[r];
  const uint64_t best = row_best(st, a.chunks);
  const Limits l = limits_of(a.s, row);
  if (!best || !(l.t > 0.0f)) return;
  if (tid == 0) own_n = 0;
  __syncthreads();
  Weight w;
  w.set((uint32_t)(best >> 32), l.t);
  Cuts c = {-1, -1, -1, kBins, 0, 0, 0, 0};
  if (l.k || l.p < 1.0f) c = find_cuts(bl, st, l, &cuts);
  const int from = chunk * a.per, to = from + a.per < a.s.V ? from + a.per : a.s.V;
  uint64_t sum = 0;
  for (int i0 = from; i0 < to; i0 += kAhead * kThreads) {
    uint32_t key[kAhead];
    load_keys(a.s, row, i0 + tid, to, key);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int b = w.bin(key[j]);
      if (b < c.definite) sum += w.kept(key[j], l.least);
      const uint64_t mask = __builtin_amdgcn_ballot_w64(b < kBins && (b == c.k_bin || (b >= c.p_lo && b <= c.p_hi)));
      if (mask) {
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&own_n, (uint32_t)__builtin_popcountll(mask));
        at = __shfl(at, 0, 64) + (uint32_t)__builtin_popcountll(mask & ((1ull << lane) - 1));
        if (((mask >> lane) & 1) && at < (uint32_t)kCap) own[at] = ((uint64_t)key[j] << 32) | (uint32_t)(i0 + tid + j * kThreads);
      }
    }
  }
  sum = bl.sum(sum);
  if (tid == 0) {
    st.sum[chunk] = sum;
    // one addition a chunk: one a wave took 10 us of 20 with 16 rows
    own_at = own_n ? atomicAdd(&st.listed, own_n) : 0;
  }
  __syncthreads();
  const uint32_t n = own_n < (uint32_t)kCap ? own_n : (uint32_t)kCap;
  for (uint32_t i = (uint32_t)tid; i < n; i += kThreads) {
    if (own_at + i < (uint32_t)kCap) st.list[own_at + i] = own[i];
  }
}

__global__ __launch_bounds__(kThreads) void vbq_sample_token_kernel(LongArgs a) {
  __shared__ Shared sh;
  Block bl(sh);
  __shared__ Cuts cuts;
  __shared__ uint32_t keys[kCap], index[kCap];
  __shared__ uint16_t bins[kCap];
  __shared__ __attribute__((aligned(16))) u32x4 entries[kRanked];  // key, bin and index, weight
  __shared__ uint64_t whole[kCap];
  __shared__ uint64_t chunk_w[kMaxChunks];
  __shared__ uint64_t before_chunk, the_total;
  __shared__ int the_chunk;
  const int tid = (int)threadIdx.x;
  const int64_t r = blockIdx.x, row = a.row0 + r;
  const RowState& st = a.state[r];
  const uint64_t best = row_best(st, a.chunks);
  const Limits l = limits_of(a.s, row);
  if (ends_early(a.s, row, best, l.t)) return;
  Weight w;
  w.set((uint32_t)(best >> 32), l.t);
  Cuts c = {-1, -1, -1, kBins, 0, 0, 0, 0};
  if (l.k || l.p < 1.0f) c = find_cuts(bl, st, l, &cuts);
  const uint32_t listed = st.listed;
  if (listed > (uint32_t)kCap) {
    auto key = [&](int i) { return key_at(a.s, row, i); };
    choose(a.s, bl, row, a.s.V, key, [&](int i) { return w.whole(key(i)); }, w, l);
    return;
  }
  const int n = (int)listed;
#pragma unroll 1
  for (int i = tid; i < n; i += kThreads) {
    const uint64_t v = st.list[i];
    keys[i] = (uint32_t)(v >> 32);
    index[i] = (uint32_t)v;
    bins[i] = (uint16_t)w.bin(keys[i]);
    whole[i] = w.whole(keys[i]);
    if (i < kRanked)
      entries[i] = u32x4{keys[i], ((uint32_t)bins[i] << 20) | index[i], (uint32_t)whole[i], (uint32_t)(whole[i] >> 32)};
  }
  if (tid < kMaxChunks) chunk_w[tid] = tid < a.chunks ? st.sum[tid] : 0;
  __syncthreads();

  Cut cut = {0, 0, true};
  uint64_t kept = c.all_w;
  uint32_t last_tie = 0xffffffffu;  // of the cut's equals those up to this index are kept
  if (n > 0 && n <= kRanked) {
    // A short list is ordered by comparing every entry with every other, four threads an
    // entry: two barriers, where the digits take nine a limit.  The last entry kept is the cut.
    const int i = tid >> 2;
    const uint32_t key = i < n ? keys[i] : 0, at = i < n ? index[i] : 0;
    const int bin = i < n ? bins[i] : kBins;
    uint32_t rank = 0;
    uint64_t before = 0;
    if (i < n) {
#pragma unroll 4
      for (int j = tid & 3; j < n; j += 4) {
        const u32x4 e = entries[j];
        const int other = (int)(e.y >> 20);
        const bool first = e.x > key || (e.x == key && (e.y & 0xfffffu) < at);
        rank += first && other == c.k_bin;
        before += first && other >= c.p_lo && other <= c.p_hi ? ((uint64_t)e.w << 32) | e.z : 0;
      }
    }
    rank += from_lane<0xB1, 0xf>(rank);  // (the four threads' sums: from the neighbour, then from the other pair)
    rank += from_lane<0x4E, 0xf>(rank);
    before += from_lane<0xB1, 0xf>(before);
    before += from_lane<0x4E, 0xf>(before);
    const bool by_k = c.k_bin < 0 || bin < c.k_bin || (bin == c.k_bin && c.k_above_c + rank < (uint64_t)l.k);
    if (c.k_bin >= 0 && c.p_lo >= 0)
      kept = c.k_above_w + bl.sum((tid & 3) == 0 && bin == c.k_bin && by_k ? whole[i] : 0);
    const double target = target_within((double)l.p * (double)kept, kept);
    const bool by_p = c.p_lo < 0 || bin < c.p_lo || (bin <= c.p_hi && (double)(c.p_above_w + before) < target);
    const uint64_t last = bl.most(i < n && by_k && by_p ? ((uint64_t)~key << 32) | at : 0);
    cut.key = ~(uint32_t)(last >> 32);
    last_tie = (uint32_t)last;
  } else {
#pragma unroll 1  // one copy of the steps' code: a workgroup alone waits for its instructions too
    for (int step = 0; step < 3; ++step) {  // top-k, top-p, which of the cut's equals
      if (step == 0 ? c.k_bin < 0 : step == 1 ? c.p_lo < 0 : cut.all) continue;
      const int lo = step == 0 ? c.k_bin : c.p_lo, hi = step == 0 ? c.k_bin : c.p_hi;
      const Cut got = cut_keys(
          bl, n,
          [&](int i) {
            if (step == 2) return keys[i] == cut.key ? ~index[i] : 0u;
            return bins[i] >= lo && bins[i] <= hi ? keys[i] : 0u;
          },
          [&](int i) { return whole[i]; }, w, step != 1, step == 0 ? (uint64_t)l.k : cut.take,
          target_within((double)l.p * (double)kept, kept), step == 1 ? c.p_above_w : 0, step == 0 ? c.k_above_c : 0);
      if (step == 2) {
        last_tie = ~got.key;
        break;
      }
      cut = shorter(got, cut);
      if (step == 0 && c.p_lo >= 0) {
        uint64_t above = 0;
#pragma unroll 1
        for (int i = tid; i < n; i += kThreads) above += bins[i] == c.k_bin && keys[i] > cut.key ? whole[i] : 0;
        kept = c.k_above_w + bl.sum(above) + cut.take * w.whole(cut.key);
      }
    }
  }
#pragma unroll 1
  for (int i = tid; i < n; i += kThreads) {
    const uint32_t key = keys[i];
    if (bins[i] < c.definite || key < cut.key) continue;
    if (key == cut.key && index[i] > last_tie) continue;
    const uint64_t v = w.kept(key, l.least);
    if (v) atomicAdd((unsigned long long*)&chunk_w[index[i] / (uint32_t)a.per], (unsigned long long)v);
  }
  __syncthreads();
  if (tid < 64) {  // the chunk in which the running sum passes u times the total
    const uint64_t own = tid < kMaxChunks ? chunk_w[tid] : 0;
    const uint64_t run = wave_scan(own, Add());
    const uint64_t all = __shfl((unsigned long long)run, 63, 64);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64((double)run > wanted(l.u, all)));
    if (tid == at) {
      the_chunk = at;
      before_chunk = run - own;
      the_total = all;
    }
  }
  __syncthreads();
  const uint64_t total = the_total;
  const double want = wanted(l.u, total);
  // the chunk's elements again, each thread a run of them, kAhead loads at a time
  const int first = the_chunk * a.per, end = first + a.per < a.s.V ? first + a.per : a.s.V;
  const int each = (a.per + kThreads - 1) / kThreads, lo = first + tid * each, hi = lo + each < end ? lo + each : end;
  auto own_of = [&](int i, uint32_t key) -> uint64_t {
    return key == 0 || key < cut.key || (key == cut.key && (uint32_t)i > last_tie) ? 0 : w.kept(key, l.least);
  };
  auto load_run = [&](int i, uint32_t (&key)[kAhead]) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) key[j] = i + j < hi ? key_at(a.s, row, i + j) : 0;
  };
  uint64_t part = 0;
#pragma unroll 1
  for (int i = lo; i < hi; i += kAhead) {
    uint32_t key[kAhead];
    load_run(i, key);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) part += own_of(i + j, key[j]);
  }
  uint64_t run = before_chunk + bl.before(part);
  if (part == 0 || (double)run > want || !((double)(run + part) > want)) return;
#pragma unroll 1
  for (int i = lo; i < hi; i += kAhead) {
    uint32_t key[kAhead];
    load_run(i, key);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint64_t own = own_of(i + j, key[j]);
      if (own && !((double)run > want) && (double)(run + own) > want)
        write_token(a.s, row, i + j, (float)((double)own / (double)total));
      run += own;
    }
  }
}

// Chunks of a long row: a workgroup a CU over all rows (two took 57 us for 16 rows of 128256, one 49:
// each finds the cuts for itself), none below 1024 logits.
void split_row(int64_t M, int64_t V, int32_t* chunks, int32_t* per) {
  const int64_t rows = M < kRowsAtOnce ? M : kRowsAtOnce;
  int64_t c = (256 + rows - 1) / rows;
  c = c < kMaxChunks ? c : kMaxChunks;
  const int64_t each = ((V + c - 1) / c + kThreads - 1) / kThreads * kThreads;
  *per = (int32_t)each;
  *chunks = (int32_t)((V + each - 1) / each);
}

bool known(int32_t type) { return type == VBQ_F32 || type == VBQ_F16 || type == VBQ_BF16; }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace

extern "C" {

vbq_status vbq_sample_workspace_size(int64_t M, int64_t V, size_t* bytes) {
  if (!bytes) return VBQ_ERR_NULL;
  if (M < 0 || M > VBQ_SAMPLE_MAX_ROWS || V < 1 || V > VBQ_SAMPLE_MAX_V) return VBQ_ERR_SHAPE;
  *bytes = V <= kCap ? 0 : (size_t)(M < kRowsAtOnce ? M : kRowsAtOnce) * sizeof(RowState);
  return VBQ_OK;
}

vbq_status vbq_sample(int64_t M, int64_t V, int32_t type, const void* logits_dev, int64_t ld, const float* temperature_dev,
                      const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev, const float* u_dev,
                      int32_t* token_dev, float* prob_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const vbq_status st = vbq_sample_workspace_size(M, V, &need);
  if (st != VBQ_OK) return st;
  if (ld < V || ld > ((int64_t)1 << 40)) return VBQ_ERR_SHAPE;
  if (!known(type)) return VBQ_ERR_UNSUPPORTED;
  if (M == 0) return VBQ_OK;
  if (!logits_dev || !u_dev || !token_dev) return VBQ_ERR_NULL;
  const void* words[] = {temperature_dev, top_k_dev, top_p_dev, min_p_dev, u_dev, token_dev, prob_dev};
  for (const void* p : words)
    if (!aligned(p, 4)) return VBQ_ERR_BUFFER;
  if (!aligned(logits_dev, type == VBQ_F32 ? 4 : 2)) return VBQ_ERR_BUFFER;
  if (need && !workspace_dev) return VBQ_ERR_NULL;
  if (need && (!aligned(workspace_dev, 16) || workspace_bytes < need)) return VBQ_ERR_BUFFER;
  SampleArgs a{logits_dev, ld, (int32_t)V, type, temperature_dev, top_k_dev, top_p_dev, min_p_dev, u_dev, token_dev, prob_dev};
  if (V <= kCap) {
    void* args[] = {&a};
    return vbq_detail_hip_status(hipLaunchKernel((const void*)vbq_sample_row_kernel, dim3((unsigned)M), dim3(kThreads),
                                                 args, 0, (hipStream_t)stream));
  }
  LongArgs b{a, (RowState*)workspace_dev, 0, 0, 0};
  split_row(M, V, &b.chunks, &b.per);
  void* args[] = {&b};
  const void* steps[] = {(const void*)vbq_sample_most_kernel, top_k_dev || top_p_dev ? (const void*)vbq_sample_bins_kernel : nullptr,
                         (const void*)vbq_sample_gather_kernel, (const void*)vbq_sample_token_kernel};
  for (; b.row0 < M; b.row0 += kRowsAtOnce) {
    const int64_t rows = M - b.row0 < kRowsAtOnce ? M - b.row0 : kRowsAtOnce;
    for (const void* f : steps) {
      if (!f) continue;
      const dim3 grid((unsigned)(f == steps[3] ? rows : rows * b.chunks));
      const vbq_status e = vbq_detail_hip_status(hipLaunchKernel(f, grid, dim3(kThreads), args, 0, (hipStream_t)stream));
      if (e != VBQ_OK) return e;
    }
  }
  return VBQ_OK;
}

}  // extern "C"
