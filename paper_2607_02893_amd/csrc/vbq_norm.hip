// Residual sum and root-mean-square norm on gfx950 (MI355X): what stands between
// one product's y and the next product's x in a decoder layer.
//
//   h = round(residual + y),  x = h / sqrt(mean(h^2) + eps) * weight.
//
// One pass: a workgroup takes a row and keeps h in registers from the sum to the
// scaling, so each input is read once and each output written once; HBM traffic
// bounds many rows, the latency of one chain (load, add up, scale) bounds few
// (4096 elements, in a graph: 8191 bf16 rows 44 us, 6.1 TB/s; one row 3.6 us).

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/vbq.h"

vbq_status vbq_detail_hip_status(hipError_t e);

namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Up to this many rows a workgroup has 512 threads, half the elements a thread (us at 4096 elements,
// 512 / 256 threads: one row 3.6 / 4.3, 16 rows 3.8 / 5.8, 256 rows 4.3 / 5.0, 4096 rows 27.7 / 27.3).
constexpr int64_t kFewRows = 256;

// Rows of a launch, a workgroup each: a grid holds fewer than 2^32 threads along a dimension.
constexpr int64_t kRowsAtOnce = (int64_t)1 << 22;

struct NormArgs {
  const void* residual;
  const void* y;       // may be null
  const void* weight;  // may be null: ones
  void* h;             // may be null, may be residual
  void* x;
  int64_t ldr, ldy, ldh, ldx;
  int32_t K;
  int32_t res_type, y_type, w_type, x_type;
  int32_t vec;         // rows begin at 16 bytes and hold whole runs of 8
  float eps;
};

__device__ __forceinline__ float half_bits(uint16_t v, int type) {
  return type == VBQ_F16 ? (float)__builtin_bit_cast(_Float16, v) : __uint_as_float((uint32_t)v << 16);
}
__device__ __forceinline__ uint16_t to_half_bits(float f, int type) {
  if (type == VBQ_F16) return __builtin_bit_cast(uint16_t, (_Float16)f);
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ float rounded(float f, int type) {
  return type == VBQ_F32 ? f : half_bits(to_half_bits(f, type), type);
}

// Elements i .. i + 7 of a row (zeros from K on).
__device__ __forceinline__ void load8(const void* base, int64_t row, int i, const NormArgs& a, int type, float (&f)[8]) {
  if (a.vec) {
    if (type == VBQ_F32) {
      const f32x4* p = (const f32x4*)((const float*)base + row + i);
      const f32x4 u = p[0], v = p[1];
      f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w;
      f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
    } else {
      const u16x8 v = *(const u16x8*)((const uint16_t*)base + row + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = half_bits(v[e], type);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = 0.0f;
      if (i + e < a.K)
        f[e] = type == VBQ_F32 ? ((const float*)base)[row + i + e] : half_bits(((const uint16_t*)base)[row + i + e], type);
    }
  }
}
__device__ __forceinline__ void store8(void* base, int64_t row, int i, const NormArgs& a, int type, const float (&f)[8]) {
  if (a.vec) {
    if (type == VBQ_F32) {
      f32x4* p = (f32x4*)((float*)base + row + i);
      p[0] = f32x4{f[0], f[1], f[2], f[3]};
      p[1] = f32x4{f[4], f[5], f[6], f[7]};
    } else {
      u16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_half_bits(f[e], type);
      *(u16x8*)((uint16_t*)base + row + i) = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (i + e < a.K) {
        if (type == VBQ_F32) ((float*)base)[row + i + e] = f[e];
        else ((uint16_t*)base)[row + i + e] = to_half_bits(f[e], type);
      }
    }
  }
}

// h of elements i .. i + 7, as the residual's type holds it.
__device__ __forceinline__ void sum8(const NormArgs& a, int64_t row, int i, float (&h)[8]) {
  load8(a.residual, row * a.ldr, i, a, a.res_type, h);
  if (a.y) {
    float y[8];
    load8(a.y, row * a.ldy, i, a, a.y_type, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = rounded(h[e] + y[e], a.res_type);
  }
}
__device__ __forceinline__ void scale8(const NormArgs& a, int64_t row, int i, float r, float (&h)[8]) {
  float w[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
  if (a.weight) load8(a.weight, 0, i, a, a.w_type, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = h[e] * r * w[e];
  store8(a.x, row * a.ldx, i, a, a.x_type, h);
}

// kHeld: the runs of 8 elements that a thread keeps.
template <int kThreads, int kHeld>
__global__ __launch_bounds__(kThreads) void vbq_add_norm_kernel(NormArgs a) {
  constexpr int kWaves = kThreads / 64, kStep = 8 * kThreads;
  __shared__ float part[kWaves];
  const int64_t row = blockIdx.x;
  const int first = 8 * (int)threadIdx.x;
  // (all loads before the first use)
  float h[kHeld][8], y[kHeld][8], total = 0.0f;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = first + j * kStep;
    if (i < a.K) {
      load8(a.residual, row * a.ldr, i, a, a.res_type, h[j]);
      if (a.y) load8(a.y, row * a.ldy, i, a, a.y_type, y[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = first + j * kStep;
    if (i < a.K) {
      if (a.y) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[j][e] = rounded(h[j][e] + y[j][e], a.res_type);
      }
      if (a.h) store8(a.h, row * a.ldh, i, a, a.res_type, h[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) total = __builtin_fmaf(h[j][e], h[j][e], total);
    }
  }
  // longer rows: the rest is read again for the scaling (from h where it was stored: the residual may be h)
  for (int i = first + kHeld * kStep; i < a.K; i += kStep) {
    float t[8];
    sum8(a, row, i, t);
    if (a.h) store8(a.h, row * a.ldh, i, a, a.res_type, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) total = __builtin_fmaf(t[e], t[e], total);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = total;
  __syncthreads();
  total = 0.0f;
#pragma unroll
  for (int j = 0; j < kWaves; ++j) total += part[j];
  const float r = 1.0f / __builtin_sqrtf(total / (float)a.K + a.eps);
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = first + j * kStep;
    if (i < a.K) scale8(a, row, i, r, h[j]);
  }
  for (int i = first + kHeld * kStep; i < a.K; i += kStep) {
    float t[8];
    if (a.h) load8(a.h, row * a.ldh, i, a, a.res_type, t);
    else sum8(a, row, i, t);
    scale8(a, row, i, r, t);
  }
}

bool known(int32_t type) { return type == VBQ_F32 || type == VBQ_F16 || type == VBQ_BF16; }
uintptr_t size_of(int32_t type) { return type == VBQ_F32 ? 4 : 2; }

}  // namespace

extern "C" {

vbq_status vbq_add_norm(int64_t n_rows, int64_t K, int32_t res_type, const void* residual_dev, int64_t ldr, int32_t y_type,
                        const void* y_dev, int64_t ldy, int32_t weight_type, const void* weight_dev, float eps, void* h_dev,
                        int64_t ldh, int32_t x_type, void* x_dev, int64_t ldx, void* stream) {
  const int64_t most = (int64_t)1 << 40;
  if (n_rows < 0 || n_rows > INT32_MAX || K < 1 || K > VBQ_NORM_MAX_K) return VBQ_ERR_SHAPE;
  if (!known(res_type) || !known(x_type) || (y_dev && !known(y_type)) || (weight_dev && !known(weight_type)))
    return VBQ_ERR_UNSUPPORTED;
  if (!(eps == eps) || eps == __builtin_inff() || eps == -__builtin_inff()) return VBQ_ERR_NONFINITE;
  if (eps < 0.0f) return VBQ_ERR_UNSUPPORTED;
  if (n_rows == 0) return VBQ_OK;
  if (!residual_dev || !x_dev) return VBQ_ERR_NULL;
  if (ldr < K || ldx < K || ldr > most || ldx > most || (y_dev && (ldy < K || ldy > most)) || (h_dev && (ldh < K || ldh > most)))
    return VBQ_ERR_SHAPE;
  struct Row { const void* p; int64_t ld; int32_t type; };
  const Row rows[] = {{residual_dev, ldr, res_type}, {x_dev, ldx, x_type}, {y_dev, ldy, y_type}, {h_dev, ldh, res_type},
                      {weight_dev, 0, weight_type}};
  bool vec = K % 8 == 0;
  for (const Row& r : rows) {
    if (!r.p) continue;
    if ((uintptr_t)r.p % size_of(r.type)) return VBQ_ERR_BUFFER;
    vec = vec && (uintptr_t)r.p % 16 == 0 && r.ld % 8 == 0;
  }
  const int threads = n_rows <= kFewRows ? 512 : 256;
  const bool shorter = K <= 16 * threads;
  const void* f = threads == 512 ? (shorter ? (const void*)vbq_add_norm_kernel<512, 2> : (const void*)vbq_add_norm_kernel<512, 4>)
                                 : (shorter ? (const void*)vbq_add_norm_kernel<256, 2> : (const void*)vbq_add_norm_kernel<256, 4>);
  for (int64_t row = 0; row < n_rows; row += kRowsAtOnce) {
    const int64_t n = n_rows - row < kRowsAtOnce ? n_rows - row : kRowsAtOnce;
    auto from = [&](const void* p, int64_t ld, int32_t type) {
      return p ? (uint8_t*)p + (size_t)row * (size_t)ld * size_of(type) : nullptr;
    };
    NormArgs a{from(residual_dev, ldr, res_type), from(y_dev, ldy, y_type), weight_dev, from(h_dev, ldh, res_type),
               from(x_dev, ldx, x_type), ldr, ldy, ldh, ldx, (int32_t)K, res_type, y_type, weight_type, x_type, vec ? 1 : 0, eps};
    void* args[] = {&a};
    const vbq_status st =
        vbq_detail_hip_status(hipLaunchKernel(f, dim3((unsigned)n), dim3((unsigned)threads), args, 0, (hipStream_t)stream));
    if (st != VBQ_OK) return st;
  }
  return VBQ_OK;
}

}  // extern "C"
