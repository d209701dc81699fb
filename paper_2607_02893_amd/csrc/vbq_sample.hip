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

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/vbq.h"

vbq_status vbq_detail_hip_status(hipError_t e);

namespace {

constexpr int kThreads = 1024;
constexpr int kWavesRow = kThreads / 64;
constexpr double kOne = 0x1p43;  // the weight of the largest logit; 2^20 of them stay below 2^63

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

struct Weight {
  double top, t;  // z_max, T
  bool inf;       // z_max is +inf: its equals weigh 1, the others nothing
  __device__ __forceinline__ double real(uint32_t key) const {
    if (key == 0) return 0.0;
    const double z = (double)logit_of(key);
    if (inf) return z == top ? 1.0 : 0.0;
    return exp((z - top) / t);
  }
  __device__ __forceinline__ uint64_t whole(uint32_t key) const { return (uint64_t)__builtin_rint(real(key) * kOne); }
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor((unsigned long long)v, d, 64);
  return v;
}

// A tail of the descending order that is cut away: kept are the keys above `key` and the
// first `ties` of the keys equal to it.
struct Cut {
  uint32_t key;
  uint64_t ties;
};

// One workgroup a row, the row read again for every step.
__global__ __launch_bounds__(kThreads) void vbq_sample_row_kernel(SampleArgs a) {
  __shared__ uint64_t weights[256];
  __shared__ uint32_t counts[256];
  __shared__ uint64_t wave_w[kWavesRow], wave_c[kWavesRow];
  __shared__ uint64_t found_above, found_count;
  __shared__ uint32_t found_digit;
  const int64_t row = blockIdx.x;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // ---- the first maximum
  uint64_t best = 0;
  for (int i = tid; i < a.V; i += kThreads) {
    const uint32_t key = key_at(a, row, i);
    const uint64_t v = ((uint64_t)key << 32) | (uint32_t)~i;
    if (key && v > best) best = v;
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)best, d, 64);
    best = o > best ? o : best;
  }
  if (lane == 0) wave_w[wave] = best;
  __syncthreads();
  for (int w = 0; w < kWavesRow; ++w) best = wave_w[w] > best ? wave_w[w] : best;
  __syncthreads();
  const float T = a.temperature ? a.temperature[row] : 1.0f;
  if (best == 0 || !(T > 0.0f)) {
    if (tid == 0) {
      a.token[row] = best ? (int32_t)~(uint32_t)best : -1;
      if (a.prob) a.prob[row] = best ? 1.0f : 0.0f;
    }
    return;
  }
  const uint32_t top_key = (uint32_t)(best >> 32);
  Weight w;
  w.top = (double)logit_of(top_key);
  w.t = (double)T;
  w.inf = w.top == (double)__builtin_inff();

  // ---- top-k, then top-p: the cut's key digit by digit, from the sums above it
  const int k = a.top_k && a.top_k[row] > 0 && a.top_k[row] < a.V ? a.top_k[row] : 0;
  const float p = a.top_p && a.top_p[row] < 1.0f ? a.top_p[row] : 1.0f;
  Cut cut = {0, 0};
  uint64_t kept_sum = 0;
  bool have_sum = false;
  for (int pass = 0; pass < 2; ++pass) {
    const bool by_count = pass == 0;
    if (by_count ? k == 0 : !(p < 1.0f)) continue;
    double target = 0.0;
    if (!by_count) {
      if (!have_sum) {
        uint64_t s = 0;
        for (int i = tid; i < a.V; i += kThreads) s += w.whole(key_at(a, row, i));
        s = wave_sum(s);
        if (lane == 0) wave_w[wave] = s;
        __syncthreads();
        kept_sum = 0;
        for (int j = 0; j < kWavesRow; ++j) kept_sum += wave_w[j];
        __syncthreads();
      }
      target = (p > 0.0f ? (double)p : 0.0) * (double)kept_sum;
    }
    uint32_t prefix = 0;
    uint64_t above_w = 0, above_c = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) {
        weights[tid] = 0;
        counts[tid] = 0;
      }
      __syncthreads();
      for (int i = tid; i < a.V; i += kThreads) {
        const uint32_t key = key_at(a, row, i);
        if (key && (shift == 24 || (key >> (shift + 8)) == prefix)) {
          atomicAdd(&counts[(key >> shift) & 255], 1u);
          atomicAdd((unsigned long long*)&weights[(key >> shift) & 255], (unsigned long long)w.whole(key));
        }
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t cw = above_w, cc = above_c;
        int digit = 255, last = -1;
        for (; digit >= 0; --digit) {
          if (counts[digit] == 0) continue;
          last = digit;
          const bool here = by_count ? cc + counts[digit] >= (uint64_t)k : (double)(cw + weights[digit]) >= target;
          if (here) break;
          cw += weights[digit];
          cc += counts[digit];
        }
        if (digit < 0) {  // fewer candidates than k, or a target that rounding put past the sum: keep all of the last
          digit = last;
          cw -= weights[digit];
          cc -= counts[digit];
        }
        found_digit = (uint32_t)digit;
        found_above = cw;
        found_count = cc;
      }
      __syncthreads();
      prefix = (prefix << 8) | found_digit;
      above_w = found_above;
      above_c = found_count;
      __syncthreads();
    }
    // the ties of the cut's key weigh the same: as many as the limit takes, one at least
    const uint64_t ties = counts[prefix & 255], each = w.whole(prefix);
    uint64_t take = ties;
    if (by_count) {
      take = (uint64_t)k - above_c < ties ? (uint64_t)k - above_c : ties;
    } else if (each) {
      const double left = (target - (double)above_w) / (double)each;
      take = left >= (double)ties ? ties : left > 1.0 ? (uint64_t)__builtin_ceil(left) : 1;
    }
    if (!by_count && prefix == cut.key && cut.ties < take) take = cut.ties;
    if (by_count || prefix > cut.key || (prefix == cut.key && take <= cut.ties)) cut = Cut{prefix, take};
    kept_sum = above_w + take * each;
    have_sum = true;
    __syncthreads();
  }

  // ---- sums of what is kept, each wave a run of the row
  float least = a.min_p && a.min_p[row] > 0.0f ? a.min_p[row] : 0.0f;
  least = least < 1.0f ? least : 1.0f;
  auto weigh = [&](uint32_t key) -> uint64_t {  // (ties of the cut apart)
    if (key == 0 || key < cut.key) return 0;
    const double r = w.real(key);
    return r >= (double)least ? (uint64_t)__builtin_rint(r * kOne) : 0;
  };
  const uint64_t tie_w = cut.ties ? weigh(cut.key) : 0;
  const int per = ((a.V + kWavesRow - 1) / kWavesRow + 63) / 64 * 64;
  const int from = wave * per, to = from + per < a.V ? from + per : a.V;
  uint64_t sum = 0, n_ties = 0;
  for (int i = from + lane; i < to; i += 64) {
    const uint32_t key = key_at(a, row, i);
    if (cut.ties && key == cut.key) ++n_ties;
    else sum += weigh(key);
  }
  sum = wave_sum(sum);
  n_ties = wave_sum(n_ties);
  if (lane == 0) {
    wave_w[wave] = sum;
    wave_c[wave] = n_ties;
  }
  __syncthreads();
  uint64_t total = 0, left = cut.ties;
  uint64_t run_w[kWavesRow];
  for (int j = 0; j < kWavesRow; ++j) {
    const uint64_t t = wave_c[j] < left ? wave_c[j] : left;
    left -= t;
    run_w[j] = wave_w[j] + t * tie_w;
    total += run_w[j];
  }
  // ---- the run, then the element, whose running sum passes u times the total
  float u = a.u[row];
  u = u > 0.0f ? u : 0.0f;
  double want = (double)u * (double)total;
  const double below = (double)total * (1.0 - 0x1p-53);
  if (!(want <= below)) want = below;
  uint64_t before = 0, ties_left = cut.ties;
  int run = -1;
  for (int j = 0; j < kWavesRow; ++j) {
    if (run_w[j] && (double)(before + run_w[j]) > want) {
      run = j;
      break;
    }
    before += run_w[j];
    ties_left -= wave_c[j] < ties_left ? wave_c[j] : ties_left;
  }
  if (wave != run) return;
  for (int i0 = from; i0 < to; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t key = i < to ? key_at(a, row, i) : 0;
    const bool tie = cut.ties && key == cut.key;
    const uint64_t tie_mask = __builtin_amdgcn_ballot_w64(tie);
    const uint64_t rank = __builtin_popcountll(tie_mask & ((1ull << lane) - 1));
    const uint64_t own = tie ? (rank < ties_left ? tie_w : 0) : weigh(key);
    uint64_t run_sum = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t o = __shfl_up((unsigned long long)run_sum, d, 64);
      if (lane >= d) run_sum += o;
    }
    const uint64_t hit = __builtin_amdgcn_ballot_w64(own && (double)(before + run_sum) > want);
    if (hit) {
      if (lane == __builtin_ctzll(hit)) {
        a.token[row] = i;
        if (a.prob) a.prob[row] = (float)((double)own / (double)total);
      }
      return;
    }
    before += __shfl((unsigned long long)run_sum, 63, 64);
    const uint64_t n = __builtin_popcountll(tie_mask);
    ties_left -= n < ties_left ? n : ties_left;
  }
}

bool known(int32_t type) { return type == VBQ_F32 || type == VBQ_F16 || type == VBQ_BF16; }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace

extern "C" {

vbq_status vbq_sample_workspace_size(int64_t M, int64_t V, size_t* bytes) {
  if (!bytes) return VBQ_ERR_NULL;
  if (M < 0 || M > VBQ_SAMPLE_MAX_ROWS || V < 1 || V > VBQ_SAMPLE_MAX_V) return VBQ_ERR_SHAPE;
  *bytes = 0;
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
  void* args[] = {&a};
  return vbq_detail_hip_status(hipLaunchKernel((const void*)vbq_sample_row_kernel, dim3((unsigned)M), dim3(kThreads), args, 0, (hipStream_t)stream));
}

}  // extern "C"
