// Attention over a cache held in 4 bits on gfx950 (MI355X): rows of keys and
// values quantized into pages (vbq_kv_append), attention of query rows over the
// pages (vbq_kv_attention), and the pages' rows as the values they stand for
// (vbq_kv_dequant).  include/vbq.h gives the layout and the definitions.
//
// The attention of a query row over positions p with keys k_p and values v_p:
//   o = sum_p w_p v_p / sum_p w_p,   w_p = exp(scale q.k_p - max).
// A key's element is s (u - 8) with the group's scale s and the 4-bit code u, so
//   q.k_p = sum_groups s (sum_i q_i u_i - 8 sum_i q_i),
// and the keys' codes themselves are the matrix operand: four bits u in an otherwise
// zero fp16 are the subnormal u 2^-24 (bits 0-3) or 16 u 2^-24 (bits 4-7), which
// the matrix cores multiply exactly.  One AND makes two operand elements; nothing
// is converted.  The 2^-24 joins the softmax scale, the 16 is taken out of the query,
// the 8's are the accumulator's start.  The values' codes take one more operation a
// pair, to u - 8: sums of w u and of 8 w are nearly equal over many positions, and the
// matrix cores cut the small bits of 32 products off downwards, which does not cancel
// (measured over 131073 positions: 5.7e-4 of the result, 2.0e-4 with u - 8).
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T, on 16x16x32 tiles:
// a lane then holds one query row's weights of the positions 4 g .. 4 g + 3 of two
// 16-position tiles (g = lane / 16), which are the eight k-elements of its B
// operand of the second product once a 32-position block is taken in the order
//   slot(p) = 8 ((p % 16) / 4) + 4 ((p % 32) / 16) + p % 4.
// The pages hold values and scales in that order, so the weights never leave
// their lane, and every code load is 16 bytes a lane, 1 KiB a wave.
//
// One token over long sequences is bound by the pages' reads and, nearly as much, by vector issue
// (131073 positions of 8 heads of 128: 33 us and 4.7 for the join, 3.8 TB/s; the reads alone 25, the issue
// alone 15), prompts most by vector issue (2048 and 1371 rows over 6144 and 4099 positions, 32 heads: 527 us,
// 470 TFLOP/s; 353 instructions a block of 32 positions and 32 rows, 112 of them converting codes; vector
// units are active for 302 of the 527 us, matrix cores for 99, and of the waves' cycles 22 % wait for memory
// and 24 % for issue).

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/vbq.h"
#include "vbq_cache.hpp"
#include "vbq_quant.hpp"

vbq_status vbq_detail_hip_status(hipError_t e);

namespace {

using vbq::Batch;
using vbq::blocks_of;
using vbq::code_bit;
using vbq::exact_rne;
using vbq::fp16_from_double;
using vbq::key_word;
using vbq::kPage;
using vbq::page_id;
using vbq::PageOf;
using vbq::Seq;
using vbq::seq_of;
using vbq::slot_of;
using vbq::value_word;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;           // waves of a workgroup
constexpr int kMaxSplits = 64;      // parts of a sequence's positions: a lane each in the join
constexpr int kNowhere = 0x7fffff00; // a position that no row sees
constexpr float kLog2e = 1.44269504088896340736f;

// ------------------------------------------------------------------ element types

__device__ __forceinline__ float bf16_float(uint32_t bits) { return __uint_as_float(bits << 16); }

// Eight consecutive elements (16-byte aligned) as floats.
__device__ __forceinline__ void load8(const void* base, int64_t index, int type, float (&f)[8]) {
  if (type == VBQ_F32) {
    const f32x4* p = (const f32x4*)((const float*)base + index);
    const f32x4 a = p[0], b = p[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else if (type == VBQ_F16) {
    const f16x8 v = *(const f16x8*)((const uint16_t*)base + index);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
  } else {
    const u32x4 v = *(const u32x4*)((const uint16_t*)base + index);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_float(w[i] & 0xffffu);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ uint32_t pair16(float lo, float hi, int type) {
  if (type == VBQ_F16) {
    const f16x2 v = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, v);
  }
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}
// Four consecutive elements, each rounded once to nearest even.
__device__ __forceinline__ void store4(void* base, int64_t index, int type, const f32x4& v) {
  if (type == VBQ_F32) {
    *(f32x4*)((float*)base + index) = v;
  } else {
    *(u32x2*)((uint16_t*)base + index) = u32x2{pair16(v.x, v.y, type), pair16(v.z, v.w, type)};
  }
}

// ------------------------------------------------------------------ append

struct AppendArgs {
  Batch batch;
  uint8_t* cache;
  int64_t n_pages;
  int32_t heads;
  int32_t type;
  const void* k;
  const void* v;
  int64_t ldk, hsk, ldv, hsv;  // row and head strides in elements
};

__device__ __forceinline__ float level4(float x, float s, float r) {
  const float t = x * r;
  float q = __builtin_rintf(t);
  // rint(x * rcp(s)) is exact unless within 2^-12 of a half-integer (|x/s| < 16, rcp to 1 ulp)
  if (__builtin_amdgcn_ballot_w64(__builtin_fabsf(t - q) > 0.5f - 1.0f / 4096.0f)) q = exact_rne(x, q, s);
  return __builtin_amdgcn_fmed3f(q, -7.0f, 7.0f);
}

// One group of 64 spread over 8 lanes, 8 elements each: its scale and its codes q + 8.
__device__ __forceinline__ float quantize8(const float (&f)[8], int (&code)[8]) {
  float amax = 0.0f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    amax = __builtin_fmaxf(amax, __builtin_fabsf(f[i]));
    nan |= !(f[i] == f[i]);
  }
  if (nan) amax = __builtin_nanf("");
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) {
    const float o = __shfl_xor(amax, d, 64);
    amax = !(o == o) || o > amax ? o : amax;  // a NaN stays
  }
  // what fp16 cannot scale becomes NaN: an infinite scale times a sum that rounding left
  // below zero would be a score of -inf, a position quietly left out
  float s = amax == amax ? fp16_from_double((double)amax / 7.0) : amax;
  s = s < __builtin_inff() ? s : __builtin_nanf("");
  // with s = 0 every level is 0: r is, and a NaN keeps exact_rne, which a neighbour may call for, from stepping
  const float r = s > 0.0f ? __builtin_amdgcn_rcpf(s) : 0.0f, by = s > 0.0f ? s : __builtin_nanf("");
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    code[i] = (int)(level4(f[i], by, r) + 8.0f);  // (some code where the scale is NaN)
  }
  return s;
}

// A workgroup takes the rows of a call that fall into one 32-position block of one
// head: it owns the block's value words, whose eight codes belong to eight
// positions, so no other workgroup of the call touches them; positions outside
// the call keep their codes.  Eight lanes a position, eight elements a lane.
template <int D>
__global__ __launch_bounds__(256) void vbq_kv_append_kernel(AppendArgs a) {
  using P = PageOf<D>;
  constexpr int kLine = 36;  // bytes of an element's 32 slots: with 32 eight lanes would write one bank
  __shared__ __attribute__((aligned(4))) uint8_t codes[D * kLine];  // [element][slot]
  const int tid = (int)threadIdx.x, t = tid >> 3, sub = tid & 7;
  const int h = (int)blockIdx.y, b = (int)blockIdx.z;
  const Seq s = seq_of(a.batch, b);
  const int64_t first = s.pos0 > 0 ? s.pos0 : 0;
  for (int64_t block = (first >> 5) + blockIdx.x; block * 32 < s.end; block += gridDim.x) {
    const int64_t id = page_id(a.batch, a.n_pages, b, block >> 1);
    if (id < 0) continue;
    uint8_t* page = a.cache + (id * a.heads + h) * (int64_t)P::kBytes;
    const int half = (int)(block & 1);
    const int64_t pos = block * 32 + t;
    const bool on = pos >= first && pos < s.end;
    const int64_t row = s.row0 + (on ? pos - s.pos0 : 0);
    // every load goes out before the first is used: a token's append is a chain of latencies
    float fk[P::kGroups][8], fv[P::kGroups][8];
#pragma unroll
    for (int grp = 0; grp < P::kGroups; ++grp) {
#pragma unroll
      for (int i = 0; i < 8; ++i) fk[grp][i] = fv[grp][i] = 0.0f;
    }
    if (on) {
#pragma unroll
      for (int grp = 0; grp < P::kGroups; ++grp) {
        load8(a.k, row * a.ldk + h * a.hsk + 64 * grp + 8 * sub, a.type, fk[grp]);
        load8(a.v, row * a.ldv + h * a.hsv + 64 * grp + 8 * sub, a.type, fv[grp]);
      }
    }
    constexpr int kWords = D * 4 / 256;  // value words of a thread
    uint32_t mask[kWords], old[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int at = tid + 256 * i, d = at >> 2, g = at & 3;
      mask[i] = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t p = block * 32 + 4 * g + (k & 3) + 16 * (k >> 2);
        if (p >= first && p < s.end) mask[i] |= 15u << code_bit(k);
      }
      old[i] = 0;
      if (mask[i] && ~mask[i]) old[i] = *(const uint32_t*)(page + value_word<D>(half, d, g));
    }
    const int slot = slot_of(t);
#pragma unroll
    for (int grp = 0; grp < P::kGroups; ++grp) {
      const int d = 64 * grp + 8 * sub;
      int c[8];
      const float ks = quantize8(fk[grp], c);
      if (on) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= (uint32_t)c[i] << code_bit(i);
        *(uint32_t*)(page + key_word<D>(32 * half + t, d >> 5, (d >> 3) & 3)) = w;
        if (sub == 0) *(_Float16*)(page + P::kKeyScales + 128 * grp + 2 * (32 * half + slot)) = (_Float16)ks;
      }
      const float vs = quantize8(fv[grp], c);
      if (on && sub == 0) *(_Float16*)(page + P::kValueScales + 128 * grp + 2 * (32 * half + slot)) = (_Float16)vs;
#pragma unroll
      for (int i = 0; i < 8; ++i) codes[(d + i) * kLine + slot] = (uint8_t)c[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int at = tid + 256 * i, d = at >> 2, g = at & 3;
      const uint32_t* bytes = (const uint32_t*)(codes + d * kLine + 8 * g);
      const uint32_t lo = bytes[0], hi = bytes[1];
      uint32_t w = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) w |= (((k < 4 ? lo : hi) >> (8 * (k & 3))) & 15u) << code_bit(k);
      if (mask[i]) *(uint32_t*)(page + value_word<D>(half, d, g)) = (w & mask[i]) | (old[i] & ~mask[i]);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ dequant

struct DequantArgs {
  Batch batch;
  const uint8_t* cache;
  int64_t n_pages;
  int32_t heads;
  float* k;
  float* v;
};

// A workgroup takes the rows of a call that fall into one 32-position block of one head, as
// the append does: value words are read in their order in memory and turned from
// eight positions of an element into elements of a position in LDS (each row gathering its eight words for
// itself: 29 us for 13193 rows of 8 heads).  s (u - 8) is exact in fp32.
template <int D>
__global__ __launch_bounds__(256) void vbq_kv_dequant_kernel(DequantArgs a) {
  using P = PageOf<D>;
  constexpr int kLine = 36;
  __shared__ __attribute__((aligned(4))) uint8_t codes[D * kLine];  // [element][slot]
  const int tid = (int)threadIdx.x, t = tid >> 3, sub = tid & 7;
  const int h = (int)blockIdx.y, b = (int)blockIdx.z;
  const Seq s = seq_of(a.batch, b);
  const int64_t first = s.pos0 > 0 ? s.pos0 : 0;
  for (int64_t block = (first >> 5) + blockIdx.x; block * 32 < s.end; block += gridDim.x) {
    const int64_t id = page_id(a.batch, a.n_pages, b, block >> 1);
    if (id < 0) continue;
    const uint8_t* page = a.cache + (id * a.heads + h) * (int64_t)P::kBytes;
    const int half = (int)(block & 1), slot = slot_of(t);
    const int64_t pos = block * 32 + t;
    const bool on = pos >= first && pos < s.end;
#pragma unroll
    for (int i = 0; i < D * 4 / 256; ++i) {
      const int at = tid + 256 * i, g = (at >> 6) & 3, d = 64 * i + 16 * (at & 3) + ((at >> 2) & 15);
      const uint32_t w = *(const uint32_t*)(page + value_word<D>(half, d, g));
      uint32_t lo = 0, hi = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        lo |= ((w >> code_bit(k)) & 15u) << (8 * k);
        hi |= ((w >> code_bit(k + 4)) & 15u) << (8 * k);
      }
      uint32_t* bytes = (uint32_t*)(codes + d * kLine + 8 * g);
      bytes[0] = lo;
      bytes[1] = hi;
    }
    __syncthreads();
    if (on) {
      const int64_t row = ((s.row0 + pos - s.pos0) * a.heads + h) * D;
#pragma unroll
      for (int grp = 0; grp < P::kGroups; ++grp) {
        const int d = 64 * grp + 8 * sub, at = 128 * grp + 2 * (32 * half + slot);
        const float ks = (float)*(const _Float16*)(page + P::kKeyScales + at);
        const float vs = (float)*(const _Float16*)(page + P::kValueScales + at);
        const uint32_t kw = *(const uint32_t*)(page + key_word<D>(32 * half + t, d >> 5, (d >> 3) & 3));
        float kf[8], vf[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          kf[i] = ks * (float)((int)((kw >> code_bit(i)) & 15u) - 8);
          vf[i] = vs * (float)((int)codes[(d + i) * kLine + slot] - 8);
        }
        *(f32x4*)(a.k + row + d) = f32x4{kf[0], kf[1], kf[2], kf[3]};
        *(f32x4*)(a.k + row + d + 4) = f32x4{kf[4], kf[5], kf[6], kf[7]};
        *(f32x4*)(a.v + row + d) = f32x4{vf[0], vf[1], vf[2], vf[3]};
        *(f32x4*)(a.v + row + d + 4) = f32x4{vf[4], vf[5], vf[6], vf[7]};
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ attention

struct AttnArgs {
  Batch batch;
  const uint8_t* cache;
  int64_t n_pages;
  int32_t heads, group;  // kv heads, query heads of each
  int32_t q_type, out_type;
  const void* q;
  void* out;
  int64_t ldq, hsq, ldo, hso;
  float scale;
  int32_t splits;         // parts of the positions
  int32_t split_pages;    // pages of a part
  float* part;            // [row * query heads + head][split][D], then as many pairs (bias, sum)
};

// v of the lanes 16 and 32 apart joined with op: all four lanes of a query row get the result.
template <typename Op>
__device__ __forceinline__ float across_groups(float v, Op op) {
  const uint32_t a = __float_as_uint(v);
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a, a, false, false));
  const float m = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const uint32_t c = __float_as_uint(m);
  const u32x2 t = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(c, c, false, false));
  return op(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
// (fmaxf's operands would each be made quiet first)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}
__device__ __forceinline__ float group_max(float v) {
  return across_groups(v, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ float group_sum(float v) {
  return across_groups(v, [](float a, float b) { return a + b; });
}

// Eight codes as a matrix operand: elements (0,1) and (4,5) stand for u 2^-24,
// (2,3) and (6,7) for 16 u 2^-24.
__device__ __forceinline__ f16x8 code_operand(uint32_t w) {
  const uint32_t w8 = w >> 8;
  return __builtin_bit_cast(f16x8, u32x4{w & 0x000f000fu, w & 0x00f000f0u, w8 & 0x000f000fu, w8 & 0x00f000f0u});
}

// Eight codes as the levels u - 8 in fp16: u or 16 u placed in the mantissa of 1024, then one packed
// operation, all exact.  `one` is 0x64006400 in a vector register: the AND and the OR are one
// operation then (of two constants it takes only one from elsewhere).
__device__ __forceinline__ f16x8 level_operand(uint32_t w, uint32_t one) {
  const uint32_t w8 = w >> 8;
  const f16x2 unit = {(_Float16)-1032.0f, (_Float16)-1032.0f}, sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  const f16x2 minus = {(_Float16)-72.0f, (_Float16)-72.0f};
  const f16x2 a = __builtin_bit_cast(f16x2, (w & 0x000f000fu) | one) + unit;
  const f16x2 b = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (w & 0x00f000f0u) | one), sixteenth, minus);
  const f16x2 c = __builtin_bit_cast(f16x2, (w8 & 0x000f000fu) | one) + unit;
  const f16x2 d = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (w8 & 0x00f000f0u) | one), sixteenth, minus);
  return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// The larger of two pairs of whole numbers (scales are not negative: their bits order as they do).  The
// words come as arguments: __builtin_bit_cast of a vector's component takes another component
// with this compiler.
__device__ __forceinline__ uint32_t larger16(uint32_t a, uint32_t b) {
  const u16x2 m = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b));
  return __builtin_bit_cast(uint32_t, m);
}

__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// A lane's share of a 32-position block.
template <int D>
struct Block {
  uint32_t kw[2][PageOf<D>::kKeyWords];
  uint32_t vw[D / 16];
  u32x4 ks[PageOf<D>::kGroups], vs[PageOf<D>::kGroups];  // eight scales, by slot
};

template <int D>
__device__ __forceinline__ void load_block(Block<D>& k, const uint8_t* page, int half, int lane) {
  using P = PageOf<D>;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint8_t* at = page + (2 * half + t) * (256 * P::kKeyWords);
    if constexpr (D == 64) {
      const u32x2 w = *(const u32x2*)(at + lane * 8);
      k.kw[t][0] = w.x;
      k.kw[t][1] = w.y;
    } else {
#pragma unroll
      for (int j = 0; j < P::kKeyWords; j += 4) {
        const u32x4 w = *(const u32x4*)(at + j * 256 + lane * 16);
        k.kw[t][j] = w.x;
        k.kw[t][j + 1] = w.y;
        k.kw[t][j + 2] = w.z;
        k.kw[t][j + 3] = w.w;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < P::kGroups; ++j) {
    const u32x4 w = *(const u32x4*)(page + P::kValues + half * 16 * D + j * 1024 + lane * 16);
    k.vw[4 * j] = w.x;
    k.vw[4 * j + 1] = w.y;
    k.vw[4 * j + 2] = w.z;
    k.vw[4 * j + 3] = w.w;
    k.ks[j] = *(const u32x4*)(page + P::kKeyScales + 128 * j + 64 * half + (lane >> 4) * 16);
    k.vs[j] = *(const u32x4*)(page + P::kValueScales + 128 * j + 64 * half + (lane >> 4) * 16);
  }
}

// Query rows of one wave and what it has summed of them.  Lane l holds of row
// l % 16 of each tile: every quantity here, and o[d block] elements 4 (l / 16) + i.
// Weights are held as 2^(score - mu - E): mu is within 8 of the row's largest score
// so far (in powers of two; a sum is rescaled only where a score passes that), and
// 2^E brings the largest value scale that the row has seen so far into [2^6, 2^7), so
// that weight times scale is an fp16 below 2^15 with 21 powers of two to its smallest
// normal.  The product's rounding to fp16 (2^-11 of a term, or 2^-31 of the largest weight
// times the largest scale where that is more) is the only one below 32 bits.  E is a
// row's own: with one of a tile's, a later token's scale took the bits of earlier rows.
template <int D, int NT, bool kTwoTerms>
struct Rows {
  static constexpr int kGroups = D / 64;
  f16x8 q[NT][D / 32], q_low[kTwoTerms ? NT : 1][D / 32];
  float start[NT][kGroups];  // -8 2^-24 sum of q over a group
  f32x4 c;                   // (by tile) what a raw score is multiplied with to be a power of two
  f32x4 mu, sum;
  f32x4 e;                   // E + 21, the fp16 exponent field of the largest value scale
  // (vectors: as arrays these four are kept in LDS, an access each a block)
  int visible[NT];
  f32x4 o[NT][D / 16];
  uint32_t one;              // 0x64006400

  // The row's elements times a power of two that puts the largest into [2^14, 2^15);
  // fp32 rows are split into two fp16 terms, the others are exact in one (unless
  // smaller than 2^-34 of the row's largest).
  __device__ __forceinline__ void load(const AttnArgs& a, int nt, int64_t row, uint32_t head, int g) {
    float f[D / 32][8];
    float amax = 0.0f;
    const int64_t at = row * a.ldq + (int64_t)head * a.hsq + 8 * g;
    // (rows that are none take the call's first: any will do, they are not stored)
    if constexpr (kTwoTerms) {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) load8(a.q, at + 32 * j, VBQ_F32, f[j]);
    } else if (a.q_type == VBQ_F16) {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) load8(a.q, at + 32 * j, VBQ_F16, f[j]);
    } else {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) load8(a.q, at + 32 * j, VBQ_BF16, f[j]);
    }
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = __builtin_fmaxf(amax, __builtin_fabsf(f[j][i]));
    }
    amax = group_max(amax);
    const int ex = (int)(__float_as_uint(amax) >> 23);
    int up = ex == 0 || ex == 255 ? 0 : 141 - ex;
    up = up > 80 ? 80 : up;  // (c stays a normal number, so hidden scores stay -inf)
    c[nt] = __builtin_ldexpf(a.scale * kLog2e, 24 - up);
#pragma unroll
    for (int grp = 0; grp < kGroups; ++grp) {
      float total = 0.0f;
#pragma unroll
      for (int j = 2 * grp; j < 2 * grp + 2; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool sixteen = (i & 2) != 0;  // its code stands for 16 u
          const float x = __builtin_ldexpf(f[j][i], sixteen ? up - 4 : up);
          const _Float16 hi = (_Float16)x;
          q[nt][j][i] = hi;
          float both = (float)hi;
          if constexpr (kTwoTerms) {
            const _Float16 lo = (_Float16)(x - (float)hi);
            q_low[nt][j][i] = lo;
            both += (float)lo;
          }
          total += sixteen ? 16.0f * both : both;
        }
      }
      start[nt][grp] = -8.0f * 0x1p-24f * group_sum(total);
    }
    mu[nt] = -__builtin_inff();
    sum[nt] = e[nt] = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[nt][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  __device__ __forceinline__ float bias(int nt) const {
    return (mu[nt] == -__builtin_inff() ? 0.0f : mu[nt]) + (e[nt] - 21.0f);
  }

  // The exponent field of the largest of a lane's value scales (by slot), without those that `seen` clears.
  __device__ __forceinline__ float largest(const Block<D>& k, const u32x4& seen) const {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4 * kGroups; ++i) top = larger16(top, k.vs[i / 4][i % 4] & seen[i % 4]);
    top = ((top & 0xffffu) > (top >> 16) ? top & 0xffffu : top >> 16) >> 10;
    if (top >= 31) {  // a NaN among them: the others set the range
      top = 0;
#pragma unroll
      for (int i = 0; i < 4 * kGroups; ++i) {
        const uint32_t w = k.vs[i / 4][i % 4] & seen[i % 4], lo = (w >> 10) & 31u, hi = (w >> 26) & 31u;
        top = lo < 31 && lo > top ? lo : top;
        top = hi < 31 && hi > top ? hi : top;
      }
    }
    return (float)top;
  }

  // One block of 32 positions from `pos` on; edge: some of them are hidden from some row.
  // Hidden positions get the score -inf, their product with the value scale is 0 and
  // the scale does not count for E, whatever their memory holds.
  __device__ __forceinline__ void block(Block<D>& k, int pos, int g, bool edge) {
    float x[NT][8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 acc[NT][kGroups];
#pragma unroll
      for (int grp = 0; grp < kGroups; ++grp) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt][grp] = f32x4{start[nt][grp], start[nt][grp], start[nt][grp], start[nt][grp]};
#pragma unroll
        for (int j = 2 * grp; j < 2 * grp + 2; ++j) {
          const f16x8 kf = code_operand(k.kw[t][j]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            acc[nt][grp] = mfma(kf, q[nt][j], acc[nt][grp]);
            if constexpr (kTwoTerms) acc[nt][grp] = mfma(kf, q_low[nt][j], acc[nt][grp]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float s = 0.0f;
#pragma unroll
          for (int grp = 0; grp < kGroups; ++grp)
            s = __builtin_fmaf((float)__builtin_bit_cast(f16x8, k.ks[grp])[4 * t + i], acc[nt][grp][i], s);
          x[nt][4 * t + i] = s;
        }
      }
    }

    if (edge) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (pos + 16 * (i >> 2) + 4 * g + (i & 3) >= visible[nt]) {
            x[nt][i] = -__builtin_inff();
            if constexpr (NT == 1) {
#pragma unroll
              for (int grp = 0; grp < kGroups; ++grp) k.vs[grp][i >> 1] &= i & 1 ? 0x0000ffffu : 0xffff0000u;
            }
          }
        }
      }
    }

    // ---- the bias moves where a score passes it by 2^8, or a value scale the largest so far
    float top[NT];
    if (NT > 1 && edge) {  // (two rows of a lane: what the one sees the other may not)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        u32x4 seen = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (pos + 16 * (i >> 2) + 4 * g + (i & 3) >= visible[nt]) seen[i >> 1] &= i & 1 ? 0x0000ffffu : 0xffff0000u;
        }
        top[nt] = largest(k, seen);
      }
    } else {
      top[0] = largest(k, u32x4{0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu});
#pragma unroll
      for (int nt = 1; nt < NT; ++nt) top[nt] = top[0];
    }
    bool grow = false;
    float most[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float low = max3(max3(x[nt][0], x[nt][1], x[nt][2]), x[nt][3], x[nt][4]);
      most[nt] = max3(low, max3(x[nt][5], x[nt][6], x[nt][7]), x[nt][7]) * c[nt];
      grow |= most[nt] > mu[nt] + 8.0f || top[nt] > e[nt];
    }
    if (__builtin_amdgcn_ballot_w64(grow)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float en = group_max(top[nt] > e[nt] ? top[nt] : e[nt]);
        const float m = group_max(most[nt]), now = m > mu[nt] + 8.0f ? m : mu[nt];
        const float alpha = mu[nt] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((mu[nt] - now) + (e[nt] - en));
        mu[nt] = now;
        e[nt] = en;
        sum[nt] *= alpha;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[nt][d] *= alpha;
      }
    }

    // ---- weights, and their products with the value scales as the second product's operand
    f16x8 w[NT][kGroups];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float b = bias(nt);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[nt][i], c[nt], -b));
        sum[nt] += p;
#pragma unroll
        for (int grp = 0; grp < kGroups; ++grp)
          w[nt][grp][i] = (_Float16)__builtin_fmaf(p, (float)__builtin_bit_cast(f16x8, k.vs[grp])[i], 0.0f);
      }
    }
    if (NT > 1 && edge) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (pos + 16 * (i >> 2) + 4 * g + (i & 3) >= visible[nt]) {
#pragma unroll
            for (int grp = 0; grp < kGroups; ++grp) w[nt][grp][i] = (_Float16)0.0f;
          }
        }
      }
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      const f16x8 vf = level_operand(k.vw[d], one);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[nt][d] = mfma(vf, w[nt][d / 4], o[nt][d]);
    }
  }
};

// What the join needs of a row's part beside its D sums: their bias and the sum of weights (0: it saw nothing).
template <int D>
__device__ __forceinline__ void store_bias(const AttnArgs& a, int64_t row_head, int split, float bias, float sum) {
  float* at = a.part + a.batch.n_rows * a.heads * a.group * (int64_t)a.splits * D + 2 * (row_head * a.splits + split);
  at[0] = bias;
  at[1] = sum;
}

constexpr int waves_per_simd(int D, int NT) { return NT > 1 || D > 128 ? 2 : D > 64 ? 3 : 4; }

// A workgroup takes a tile of 16 NT rows (query heads of one kv head, row by row) and a part of
// the positions; its waves take every fourth page each and join at the end, a lane's sums through LDS.
// Rows of their own for the waves (no join, each page read by all four) came to much the same on grids
// that fill the chip (the two prompts above 505 us, so 524 at the time) and to four to five times as long
// on smaller ones (64 rows of 32 heads over 16384 positions: 284 us, so 54), where a wave walks all positions.
// fp32 queries keep twice the registers: with 64 and 128 elements 2 to 8 values wait in scratch memory
// outside the loop over pages, with 256 elements 24, four of them read back within it (sixteen sequences:
// 36.7 us, 30.2 with 16-bit queries; the prompts 589 and 527).
template <int D, int NT, bool kTwoTerms>
__global__ __launch_bounds__(kWaves * 64, waves_per_simd(D, NT)) void vbq_kv_attention_kernel(AttnArgs a) {
  using P = PageOf<D>;
  constexpr int kRows = 16 * NT;
  __shared__ __attribute__((aligned(16))) float o_lds[kWaves][kRows][D + 4];
  __shared__ float bias_lds[kWaves][kRows], sum_lds[kWaves][kRows];
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)threadIdx.x & 63, g = lane >> 4;
  const uint32_t h = blockIdx.x % (uint32_t)a.heads, split = blockIdx.x / (uint32_t)a.heads, group = (uint32_t)a.group;
  const int b = (int)blockIdx.y;
  const Seq s = seq_of(a.batch, b);
  const uint32_t n_rows = (uint32_t)s.n * group;  // (below 2^31)
  const uint32_t hq0 = h * group;

  // the last tiles see the most positions: they start first
  for (uint32_t tile = gridDim.z - 1 - blockIdx.z; tile * kRows < n_rows; tile += gridDim.z) {
    const uint32_t base = tile * kRows;
    Rows<D, NT, kTwoTerms> r;
    asm("v_mov_b32 %0, 0x64006400" : "=v"(r.one));
    const uint32_t last = base + 16 * NT < n_rows ? base + 16 * NT : n_rows;
    auto seen = [&](uint32_t row) {
      const int64_t v = s.pos0 + row + 1;
      return (int)(v < 0 ? 0 : v < s.end ? v : s.end);
    };
    const int least = seen(base / group), most = seen((last - 1) / group);
    const int pages = (most + kPage - 1) / kPage, least_per = (pages + a.splits - 1) / a.splits;
    const int per = a.split_pages > least_per ? a.split_pages : least_per;
    const int64_t first = (int64_t)split * per + wave;
    const int stop = (int)(split + 1) * (int64_t)per < pages ? (int)(split + 1) * per : pages;
    const int64_t heads = (int64_t)a.heads * a.group;
    if (split && split * (int64_t)per >= pages) {  // nothing to see in this part: the join reads no more of it than that
      const uint32_t i = base + threadIdx.x;
      if (threadIdx.x < kRows && i < n_rows)
        store_bias<D>(a, (s.row0 + i / group) * heads + hq0 + i % group, (int)split, 0.0f, 0.0f);
      continue;
    }
    // What is no page of the cache is read as page 0 and hidden.  Ids are read a page ahead, the
    // first block before the queries.
    auto id_of = [&](int64_t page) { return page < stop ? page_id(a.batch, a.n_pages, b, page) : -1; };
    auto load = [&](Block<D>& k, int64_t id, int half) {
      load_block<D>(k, a.cache + ((id < 0 ? 0 : id) * a.heads + h) * (int64_t)P::kBytes, half, lane);
    };
    Block<D> k;
    int page = (int)(first < stop ? first : stop), half = 0;
    int64_t id = id_of(first), next = id_of(first + kWaves);
    if (page < stop) load(k, id, 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint32_t i = base + 16 * nt + (lane & 15), row = i / group;
      const bool on = i < n_rows;
      r.visible[nt] = on ? seen(row) : 0;
      r.load(a, nt, s.row0 + (on ? row : 0), hq0 + (on ? i - row * group : 0), g);
    }
#pragma unroll 1
    while (page < stop) {
      const int pos = id < 0 ? kNowhere : page * kPage + 32 * half;
      if (half || page * kPage + 32 >= most) {  // the next block is another page's first
        page += kWaves;
        id = next;
        half = 0;
        next = id_of((int64_t)page + kWaves);
      } else {
        half = 1;
      }
      r.block(k, pos, g, pos + 32 > least);
      if (page < stop) load(k, id, half);
    }

#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float sum = group_sum(r.sum[nt]);
      const int i = 16 * nt + (lane & 15);
      if (g == 0) {
        bias_lds[wave][i] = r.bias(nt);
        sum_lds[wave][i] = sum;
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) *(f32x4*)&o_lds[wave][i][16 * d + 4 * g] = r.o[nt][d];
    }
    __syncthreads();
    constexpr int kLanes = 256 / kRows, kEach = D / kLanes;  // lanes of a row, elements of a lane
    const int i = (int)threadIdx.x / kLanes, sub = (int)threadIdx.x % kLanes;
    const uint32_t ri = base + i;
    if (ri < n_rows) {
      float top = -__builtin_inff(), f[kWaves], sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        f[w] = sum_lds[w][i] == 0.0f ? -__builtin_inff() : bias_lds[w][i];
        top = __builtin_fmaxf(top, f[w]);
      }
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        // -1: a wave that saw nothing of the row.  One that weighs nothing still adds its sums: 0 times NaN is NaN.
        f[w] = f[w] == -__builtin_inff() ? -1.0f : __builtin_amdgcn_exp2f(f[w] - top);
        sum += f[w] < 0.0f ? 0.0f : sum_lds[w][i] * f[w];
      }
      const int64_t row = s.row0 + ri / group;
      const int64_t hq = hq0 + ri % group;
      const int64_t rh = row * heads + hq;
      const float scale = a.splits > 1 ? 1.0f : 1.0f / sum;
      if (a.splits > 1 && sub == 0) store_bias<D>(a, rh, split, top == -__builtin_inff() ? 0.0f : top, sum);
#pragma unroll
      for (int d = 0; d < kEach; d += 4) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          if (f[w] >= 0.0f) v += *(const f32x4*)&o_lds[w][i][4 * (sub + kLanes * (d / 4))] * f[w];
        }
        const int el = 4 * (sub + kLanes * (d / 4));
        if (a.splits > 1) *(f32x4*)(a.part + (rh * a.splits + split) * D + el) = v;
        else store4(a.out, row * a.ldo + hq * a.hso + el, a.out_type, sum == 0.0f ? v : v * scale);
      }
    }
    __syncthreads();
  }
}

// A row's parts joined: one workgroup a row and head, a wave's lanes over the parts' biases, then
// 16 bytes a lane of several parts side by side, all loads before the first use.
template <int D>
__global__ __launch_bounds__(kWaves * 64) void vbq_kv_join_kernel(AttnArgs a) {
  constexpr int kLanes = D / 4;                   // lanes of a part, four elements each
  constexpr int kSide = 256 / kLanes;             // parts side by side
  constexpr int kTurns = kMaxSplits / kSide;
  __shared__ __attribute__((aligned(16))) float o_lds[kSide][D];
  __shared__ float f_lds[kMaxSplits];
  const int heads = a.heads * a.group;
  const int hq = (int)blockIdx.x, b = (int)blockIdx.y;
  const Seq s = seq_of(a.batch, b);
  const int tid = (int)threadIdx.x, side = tid / kLanes, el = 4 * (tid % kLanes);
  for (int64_t i = blockIdx.z; i < s.n; i += gridDim.z) {
    const int64_t rh = (s.row0 + i) * heads + hq;
    float sum = 0.0f;
    if (tid < kMaxSplits) {  // (the first wave)
      const float* pair = a.part + a.batch.n_rows * heads * a.splits * (int64_t)D + 2 * rh * a.splits;
      const bool on = tid < a.splits;
      const float n = on ? pair[2 * tid + 1] : 0.0f, bias = on && n != 0.0f ? pair[2 * tid] : -__builtin_inff();
      float top = bias;
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, d, 64));
      const float f = n == 0.0f ? -1.0f : __builtin_amdgcn_exp2f(bias - top);  // -1: it saw nothing of the row
      f_lds[tid] = f;
      sum = n == 0.0f ? 0.0f : n * f;
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    }
    __syncthreads();
    // a part that saw nothing was not written: the first is read in its place and not added (one that
    // weighs nothing is: 0 times NaN is NaN)
    f32x4 part[kTurns];
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
      const int p = side + j * kSide;
      part[j] = *(const f32x4*)(a.part + (rh * a.splits + (f_lds[p] >= 0.0f ? p : 0)) * D + el);
    }
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
      const float f = f_lds[side + j * kSide];
      if (f >= 0.0f) v += part[j] * f;
    }
    *(f32x4*)&o_lds[side][el] = v;
    __syncthreads();
    if (tid < kLanes) {
      v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kSide; ++j) v += *(const f32x4*)&o_lds[j][el];
      const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
      store4(a.out, (s.row0 + i) * a.ldo + hq * a.hso + el, a.out_type, sum == 0.0f ? none : v * (1.0f / sum));
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ host side

constexpr int64_t kMaxGrid = (int64_t)1 << 30;

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }
bool known(int32_t type) { return type == VBQ_F32 || type == VBQ_F16 || type == VBQ_BF16; }

vbq_status check_desc(const vbq_kv_desc* d) {
  if (!d) return VBQ_ERR_NULL;
  vbq_kv_desc want;
  if (d->magic != VBQ_KV_MAGIC || d->version != VBQ_KV_VERSION) return VBQ_ERR_DESC;
  if (vbq_kv_layout(d->n_pages, d->n_heads, d->head_dim, &want) != VBQ_OK) return VBQ_ERR_DESC;
  return d->page_bytes == want.page_bytes && d->total_bytes == want.total_bytes ? VBQ_OK : VBQ_ERR_DESC;
}

vbq_status check_batch(const vbq_kv_batch* b) {
  if (!b) return VBQ_ERR_NULL;
  if (b->n_seqs < 0 || b->n_seqs > VBQ_KV_MAX_SEQS || b->n_rows < 0 || b->n_rows > VBQ_KV_MAX_ROWS)
    return VBQ_ERR_SHAPE;
  if (b->max_rows < 1 || b->max_len < 0 || b->table_stride < 1 || b->table_stride > VBQ_KV_MAX_TABLE)
    return VBQ_ERR_SHAPE;
  if (!b->row_start && b->n_rows != (int64_t)b->n_seqs * b->max_rows) return VBQ_ERR_SHAPE;
  if (b->n_seqs == 0 || b->n_rows == 0) return VBQ_OK;
  if (!b->page_table || !b->seq_len) return VBQ_ERR_NULL;
  return aligned(b->page_table, 4) && aligned(b->seq_len, 4) && aligned(b->row_start, 4) ? VBQ_OK : VBQ_ERR_BUFFER;
}

// Rows of 16-byte aligned runs of elements: both strides multiples of 8, within 2^40 elements.
bool strides_fit(int64_t ld, int64_t hs, int64_t least) {
  const int64_t most = (int64_t)1 << 40;
  return ld >= least && hs >= least && ld <= most && hs <= most && ld % 8 == 0 && hs % 8 == 0;
}

Batch batch_of(const vbq_kv_batch* b) {
  return Batch{b->page_table, b->row_start, b->seq_len, b->n_seqs, b->table_stride, b->n_rows, b->max_rows};
}

struct Plan {
  int nt;  // 16-row tiles of a workgroup
  int tiles, splits, split_pages;
};

Plan plan_of(const vbq_kv_desc* d, const vbq_kv_batch* b, int group) {
  Plan p;
  const int64_t rows = (b->max_rows < b->n_rows ? b->max_rows : b->n_rows) * (int64_t)group;
  const int64_t units = (int64_t)b->n_seqs * d->n_heads, most = kMaxGrid / kMaxSplits / units;  // (the kernel's loop takes the rest)
  // 32 rows share a page's loads and conversions where workgroups of them are many (us, 16 / 32 rows,
  // 128 elements, 4096 positions: 128 of them 38.6 / 35.6, 512 138 / 115; 64 16.1 / 28.4); with 256
  // elements their sums do not fit the registers.
  p.nt = d->head_dim <= 128 && units * ((rows + 31) / 32) >= 128 ? 2 : 1;
  const int64_t per = 16 * p.nt, tiles = (rows + per - 1) / per;
  p.tiles = (int)(tiles < 16384 ? tiles : 16384);
  if (p.tiles > most) p.tiles = most > 1 ? (int)most : 1;
  // Parts of equal size whatever a sequence's length, so that long sequences of a ragged batch get
  // more workgroups: at 64 and 128 elements twice as many as the chip holds at a time if all were
  // max_len long (once / twice, a ragged batch of eight: 22.7 / 21.6 us), at 256 as many (sixteen
  // sequences 34.7 / 39.1); no part below a page a wave, nor so small that its sums
  // (4 D bytes a row, written and read) cost a tenth of its pages.
  const int64_t base = units * p.tiles, pages = ((int64_t)b->max_len + kPage - 1) / kPage;
  const int64_t want = (p.nt > 1 || d->head_dim == 256 ? 512 : 1536) / base;
  int64_t part = want > 1 ? (pages + want - 1) / want : pages;
  const int64_t most_parts = (pages + kMaxSplits - 1) / kMaxSplits, tile_rows = rows < 16 ? rows : 16;
  part = part < kWaves ? kWaves : part;
  part = part < tile_rows ? tile_rows : part;
  part = part < most_parts ? most_parts : part;
  p.split_pages = (int)part;
  p.splits = pages > part ? (int)((pages + part - 1) / part) : 1;
  // A max_rows that is right (and no rows but the sequences') keeps n_rows * query heads * splits below
  // 16 * 1536.  Where it is far too small, the parts' sums would fill the memory (8192 rows of 32 heads
  // said to be one a sequence: 8.7 GB): fewer parts then, and tiles for what the rows are on average.
  const int64_t row_heads = b->n_rows * d->n_heads * (int64_t)group;
  if (p.splits > 1 && row_heads * p.splits > VBQ_KV_MAX_PARTS) {
    const int64_t fewer = VBQ_KV_MAX_PARTS / row_heads, mean = (b->n_rows * group / b->n_seqs + per) / per;
    p.splits = fewer > 1 ? (int)fewer : 1;
    if (p.tiles < mean) p.tiles = (int)(mean < 16384 ? mean : 16384);
    if (p.tiles > most) p.tiles = most > 1 ? (int)most : 1;
  }
  return p;
}

template <int D>
const void* attention_kernel(const Plan& p, bool two_terms) {
  if constexpr (D <= 128) {
    if (p.nt == 2)
      return two_terms ? (const void*)vbq_kv_attention_kernel<D, 2, true>
                       : (const void*)vbq_kv_attention_kernel<D, 2, false>;
  }
  return two_terms ? (const void*)vbq_kv_attention_kernel<D, 1, true>
                   : (const void*)vbq_kv_attention_kernel<D, 1, false>;
}

vbq_status launch(const void* f, dim3 grid, int threads, void** args, void* stream) {
  return vbq_detail_hip_status(hipLaunchKernel(f, grid, dim3((unsigned)threads), args, 0, (hipStream_t)stream));
}

}  // namespace

extern "C" {

vbq_status vbq_kv_layout(int64_t n_pages, int32_t n_heads, int32_t head_dim, vbq_kv_desc* desc_out) {
  if (!desc_out) return VBQ_ERR_NULL;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return head_dim < 1 ? VBQ_ERR_SHAPE : VBQ_ERR_UNSUPPORTED;
  if (n_pages < 1 || n_pages > INT32_MAX || n_heads < 1 || n_heads > VBQ_KV_MAX_HEADS) return VBQ_ERR_SHAPE;
  vbq_kv_desc d = {};
  d.magic = VBQ_KV_MAGIC;
  d.version = VBQ_KV_VERSION;
  d.n_pages = n_pages;
  d.n_heads = n_heads;
  d.head_dim = head_dim;
  d.page_bytes = (uint64_t)n_heads * 68u * (uint64_t)head_dim;
  d.total_bytes = d.page_bytes * (uint64_t)n_pages;
  *desc_out = d;
  return VBQ_OK;
}

vbq_status vbq_kv_append(const vbq_kv_desc* desc, void* cache_dev, const vbq_kv_batch* batch, int32_t type,
                         const void* k_dev, int64_t ldk, int64_t hsk, const void* v_dev, int64_t ldv, int64_t hsv,
                         void* stream) {
  vbq_status st = check_desc(desc);
  if (st != VBQ_OK) return st;
  if ((st = check_batch(batch)) != VBQ_OK) return st;
  if (!known(type)) return VBQ_ERR_UNSUPPORTED;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return VBQ_OK;
  if (!cache_dev || !k_dev || !v_dev) return VBQ_ERR_NULL;
  if (!strides_fit(ldk, hsk, 0) || !strides_fit(ldv, hsv, 0)) return VBQ_ERR_SHAPE;
  if (!aligned(cache_dev, 256) || !aligned(k_dev, 16) || !aligned(v_dev, 16)) return VBQ_ERR_BUFFER;
  AppendArgs a{batch_of(batch), (uint8_t*)cache_dev, desc->n_pages, desc->n_heads, type, k_dev, v_dev, ldk, hsk, ldv, hsv};
  void* args[] = {&a};
  const dim3 grid((unsigned)blocks_of(batch->max_rows, batch->n_rows, desc->n_heads, batch->n_seqs), (unsigned)desc->n_heads,
                  (unsigned)batch->n_seqs);
  const void* f = desc->head_dim == 64    ? (const void*)vbq_kv_append_kernel<64>
                  : desc->head_dim == 128 ? (const void*)vbq_kv_append_kernel<128>
                                          : (const void*)vbq_kv_append_kernel<256>;
  return launch(f, grid, 256, args, stream);
}

vbq_status vbq_kv_dequant(const vbq_kv_desc* desc, const void* cache_dev, const vbq_kv_batch* batch, float* k_dev,
                          float* v_dev, void* stream) {
  vbq_status st = check_desc(desc);
  if (st != VBQ_OK) return st;
  if ((st = check_batch(batch)) != VBQ_OK) return st;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return VBQ_OK;
  if (!cache_dev || !k_dev || !v_dev) return VBQ_ERR_NULL;
  if (!aligned(cache_dev, 256) || !aligned(k_dev, 16) || !aligned(v_dev, 16)) return VBQ_ERR_BUFFER;
  DequantArgs a{batch_of(batch), (const uint8_t*)cache_dev, desc->n_pages, desc->n_heads, k_dev, v_dev};
  void* args[] = {&a};
  const dim3 grid((unsigned)blocks_of(batch->max_rows, batch->n_rows, desc->n_heads, batch->n_seqs), (unsigned)desc->n_heads,
                  (unsigned)batch->n_seqs);
  const void* f = desc->head_dim == 64    ? (const void*)vbq_kv_dequant_kernel<64>
                  : desc->head_dim == 128 ? (const void*)vbq_kv_dequant_kernel<128>
                                          : (const void*)vbq_kv_dequant_kernel<256>;
  return launch(f, grid, 256, args, stream);
}

vbq_status vbq_kv_attention_workspace_size(const vbq_kv_desc* desc, const vbq_kv_batch* batch, int32_t n_q_heads,
                                           size_t* bytes) {
  if (!bytes) return VBQ_ERR_NULL;
  vbq_status st = check_desc(desc);
  if (st != VBQ_OK) return st;
  if ((st = check_batch(batch)) != VBQ_OK) return st;
  if (n_q_heads < 1 || n_q_heads % desc->n_heads || n_q_heads / desc->n_heads > VBQ_KV_MAX_GROUP)
    return VBQ_ERR_SHAPE;
  if (batch->n_rows * (n_q_heads / desc->n_heads) > (int64_t)1 << 30) return VBQ_ERR_SHAPE;
  *bytes = 0;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return VBQ_OK;
  const Plan p = plan_of(desc, batch, n_q_heads / desc->n_heads);
  const size_t row = (size_t)(desc->head_dim + 2) * sizeof(float);
  if (p.splits > 1) *bytes = (size_t)batch->n_rows * (size_t)n_q_heads * (size_t)p.splits * row;
  return VBQ_OK;
}

vbq_status vbq_kv_attention(const vbq_kv_desc* desc, const void* cache_dev, const vbq_kv_batch* batch, int32_t n_q_heads,
                            float scale, int32_t q_type, const void* q_dev, int64_t ldq, int64_t hsq, int32_t out_type,
                            void* out_dev, int64_t ldo, int64_t hso, void* workspace_dev, size_t workspace_bytes,
                            void* stream) {
  size_t need = 0;
  vbq_status st = vbq_kv_attention_workspace_size(desc, batch, n_q_heads, &need);
  if (st != VBQ_OK) return st;
  if (!known(q_type) || !known(out_type)) return VBQ_ERR_UNSUPPORTED;
  if (!(scale == scale) || scale == __builtin_inff() || scale == -__builtin_inff()) return VBQ_ERR_NONFINITE;
  if (!(scale >= 0x1p-60f && scale <= 0x1p30f)) return VBQ_ERR_UNSUPPORTED;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return VBQ_OK;
  if (!cache_dev || !q_dev || !out_dev) return VBQ_ERR_NULL;
  if (!strides_fit(ldq, hsq, 0) || !strides_fit(ldo, hso, desc->head_dim)) return VBQ_ERR_SHAPE;
  if (!aligned(cache_dev, 256) || !aligned(q_dev, 16) || !aligned(out_dev, 16)) return VBQ_ERR_BUFFER;
  if (need) {
    if (!workspace_dev) return VBQ_ERR_NULL;
    if (!aligned(workspace_dev, 16) || workspace_bytes < need) return VBQ_ERR_BUFFER;
  }
  const int group = n_q_heads / desc->n_heads;
  const Plan p = plan_of(desc, batch, group);
  AttnArgs a{batch_of(batch), (const uint8_t*)cache_dev, desc->n_pages, desc->n_heads, group, q_type, out_type, q_dev, out_dev,
             ldq, hsq, ldo, hso, scale, p.splits, p.split_pages, (float*)workspace_dev};
  void* args[] = {&a};
  const int D = desc->head_dim;
  const bool two = q_type == VBQ_F32;
  const void* f = D == 64 ? attention_kernel<64>(p, two) : D == 128 ? attention_kernel<128>(p, two) : attention_kernel<256>(p, two);
  const dim3 grid((unsigned)(p.splits * desc->n_heads), (unsigned)batch->n_seqs, (unsigned)p.tiles);
  if ((st = launch(f, grid, kWaves * 64, args, stream)) != VBQ_OK || p.splits == 1) return st;
  const void* j = D == 64    ? (const void*)vbq_kv_join_kernel<64>
                  : D == 128 ? (const void*)vbq_kv_join_kernel<128>
                             : (const void*)vbq_kv_join_kernel<256>;
  const int64_t rows = batch->max_rows < batch->n_rows ? batch->max_rows : batch->n_rows;
  const dim3 joins((unsigned)n_q_heads, (unsigned)batch->n_seqs, (unsigned)(rows < 1024 ? rows : 1024));
  return launch(j, joins, kWaves * 64, args, stream);
}

}  // extern "C"
