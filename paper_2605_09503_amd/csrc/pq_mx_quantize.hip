// MXFP4: quantizers into the stored and the operand layout, packing of stored rows, and reading back (all formats).
#include "pq_host.h"
#include "pq_mx.h"

namespace pq {

namespace {

constexpr int kThreads = 256;

// eight bf16 of a row, in order or gathered
template <bool GATHER>
__device__ __forceinline__ uint4 load8(const uint16_t* row, const int32_t* perm, int64_t k) {
  if constexpr (!GATHER) {
    return *reinterpret_cast<const uint4*>(row + k);
  } else {
    const int4 a = *reinterpret_cast<const int4*>(perm + k), b = *reinterpret_cast<const int4*>(perm + k + 4);
    return make_uint4(row[a.x] | (uint32_t)row[a.y] << 16, row[a.z] | (uint32_t)row[a.w] << 16, row[b.x] | (uint32_t)row[b.y] << 16,
                      row[b.z] | (uint32_t)row[b.w] << 16);
  }
}

// Stored layout: four lanes a group, eight channels a lane.
template <bool GATHER>
__global__ __launch_bounds__(kThreads) void mx_quantize_rows_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t K, int64_t ld,
                                                                    const int32_t* __restrict__ perm, uint8_t* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales) {
  const int64_t per_row = K / 8, n = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / per_row, c = i - r * per_row;
    uint32_t byte;
    const uint32_t q = mx_quantize8(load8<GATHER>(x + r * ld, perm, c * 8), byte);
    reinterpret_cast<uint32_t*>(codes)[i] = q;
    if ((i & 3) == 0) scales[i >> 2] = (uint8_t)byte;
  }
}

// Operand layout: 16 lanes a row's piece of a panel.
__global__ __launch_bounds__(kThreads) void mx_quantize_operand_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t K, int64_t ld,
                                                                       uint8_t* __restrict__ operand, size_t scales_at,
                                                                       uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t n = mx_panels(K) * rows * 16;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t piece = i >> 4, p = piece / rows, r = piece - p * rows, k = p * kMxPanel + (i & 15) * 8;
    uint32_t byte = 0, q = 0;
    if (k < K) {                                             // K is a multiple of 32: the four lanes of a group together
      q = mx_quantize8(*reinterpret_cast<const uint4*>(x + r * ld + k), byte);
      if (codes) {
        reinterpret_cast<uint32_t*>(codes)[(r * K + k) >> 3] = q;
        if ((i & 3) == 0) scales[(r * K + k) >> 5] = (uint8_t)byte;
      }
    }
    reinterpret_cast<uint32_t*>(operand)[i] = q;
    if ((i & 3) == 0) operand[scales_at + (i >> 2)] = (uint8_t)byte;
  }
}

// Stored rows into the operand layout, a group a thread.
__global__ __launch_bounds__(kThreads) void mx_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows,
                                                           int64_t K, uint8_t* __restrict__ operand, size_t scales_at) {
  const int64_t n = mx_panels(K) * rows * kMxRowScales, groups = K / kMxBlock;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t piece = i / kMxRowScales, p = piece / rows, r = piece - p * rows, g = p * kMxRowScales + i % kMxRowScales;
    const bool there = g < groups;
    reinterpret_cast<uint4*>(operand)[i] = there ? reinterpret_cast<const uint4*>(codes)[r * groups + g] : make_uint4(0, 0, 0, 0);
    operand[scales_at + i] = there ? scales[r * groups + g] : 0;
  }
}

// ---------------------------------------------------------------- reading back
// E2M1 magnitudes times two are whole numbers: 0 1 2 3 4 6 8 12
__device__ __forceinline__ float e2m1_value(uint32_t code) {
  const float v = 0.5f * (float)((0xC8643210u >> (4 * (code & 7u))) & 15u);
  return code & 8u ? -v : v;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}
// the stored value by binary32 operations, rounded once more to bf16 (nearest even); eight codes a thread
template <int FMT>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const uint8_t* __restrict__ codes, const void* __restrict__ scales,
                                                              const float* __restrict__ tensor_scale, int64_t rows, int64_t K, int group,
                                                              uint16_t* __restrict__ y, int64_t ldy) {
  const int64_t per_row = K / 8, n = rows * per_row;
  const float T = FMT == PQ_FMT_NVFP4 ? tensor_scale[0] : 1.0f;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / per_row, c = i - r * per_row, g = r * (K / group) + c * 8 / group;
    const uint32_t q = reinterpret_cast<const uint32_t*>(codes)[i];
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t code = q >> (4 * j) & 15u;
      if constexpr (FMT == PQ_FMT_MXFP4) {
        v[j] = e2m1_value(code) * mx_scale_value(((const uint8_t*)scales)[g]);
      } else if constexpr (FMT == PQ_FMT_NVFP4) {
        v[j] = e2m1_value(code) * e4m3_decode(((const uint8_t*)scales)[g]) * T;      // the first product is exact
      } else {
        v[j] = (float)((int)(code << 28) >> 28) * ((const float*)scales)[g];
      }
    }
    *reinterpret_cast<uint4*>(y + r * ldy + c * 8) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                                                pack_bf16(v[6], v[7]));
  }
}

int blocks_for(int64_t threads) {
  const int64_t b = (threads + kThreads - 1) / kThreads;
  return (int)(b < 65536 ? b : 65536);
}

}  // namespace

size_t mx_operand_bytes(int64_t rows, int64_t K) {
  return mx_scales_at(rows, K) + align_up((size_t)mx_panels(K) * rows * kMxRowScales, 256);
}

int launch_mx_quantize_rows(const void* x, int64_t rows, int64_t K, int64_t ld, const int32_t* perm, uint8_t* codes, void* scales,
                            hipStream_t st) {
  const int n = blocks_for(rows * (K / 8));
  if (perm)
    mx_quantize_rows_kernel<true><<<n, kThreads, 0, st>>>((const uint16_t*)x, rows, K, ld, perm, codes, (uint8_t*)scales);
  else
    mx_quantize_rows_kernel<false><<<n, kThreads, 0, st>>>((const uint16_t*)x, rows, K, ld, perm, codes, (uint8_t*)scales);
  return check_hip(hipGetLastError(), "mx_quantize_rows_kernel");
}

int launch_mx_quantize_operand(const void* x, int64_t rows, int64_t K, int64_t ld, void* operand, uint8_t* codes, void* scales,
                               hipStream_t st) {
  mx_quantize_operand_kernel<<<blocks_for(mx_panels(K) * rows * 16), kThreads, 0, st>>>((const uint16_t*)x, rows, K, ld, (uint8_t*)operand,
                                                                                        mx_scales_at(rows, K), codes, (uint8_t*)scales);
  return check_hip(hipGetLastError(), "mx_quantize_operand_kernel");
}

int launch_mx_pack(const uint8_t* codes, const void* scales, int64_t rows, int64_t K, void* operand, hipStream_t st) {
  mx_pack_kernel<<<blocks_for(mx_panels(K) * rows * kMxRowScales), kThreads, 0, st>>>(codes, (const uint8_t*)scales, rows, K, (uint8_t*)operand,
                                                                                      mx_scales_at(rows, K));
  return check_hip(hipGetLastError(), "mx_pack_kernel");
}

int launch_dequantize(pq_format fmt, int group, const uint8_t* codes, const void* scales, const float* tensor_scale, int64_t rows, int64_t K,
                      void* y, int64_t ldy, hipStream_t st) {
  const int n = blocks_for(rows * (K / 8));
  switch (fmt) {
    case PQ_FMT_MXFP4:
      dequantize_kernel<PQ_FMT_MXFP4><<<n, kThreads, 0, st>>>(codes, scales, tensor_scale, rows, K, group, (uint16_t*)y, ldy);
      break;
    case PQ_FMT_NVFP4:
      dequantize_kernel<PQ_FMT_NVFP4><<<n, kThreads, 0, st>>>(codes, scales, tensor_scale, rows, K, group, (uint16_t*)y, ldy);
      break;
    default:
      dequantize_kernel<PQ_FMT_INT4><<<n, kThreads, 0, st>>>(codes, scales, tensor_scale, rows, K, group, (uint16_t*)y, ldy);
  }
  return check_hip(hipGetLastError(), "dequantize_kernel");
}

}  // namespace pq
