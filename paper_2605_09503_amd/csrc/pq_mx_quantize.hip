// MXFP4: quantizers into the stored and the operand layout, packing of stored rows, and reading back (all formats).
#include "pq_host.h"
#include "pq_mx.h"

#include <type_traits>

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

// A wave takes kRows rows by 512 channels, eight channels a lane and row: every row's load is under way before the first is waited for,
// and a row's 1 KB is read in one piece.  The waves of a workgroup take the next rows.  Stored 8211 x 5120: 21.4 us with an item a
// thread and its division, now 18.9 (5.6 TB/s); into the operand, 8192 x 8192, panel by panel 43, now 37; read back 26.8, now 18.2.
constexpr int kRows = 4, kChunk = 512;
struct Place {
  int64_t row;                                                 // first of kRows
  int64_t k;                                                   // first channel of this lane
};
__device__ __forceinline__ Place place_of(int64_t K) {
  const uint32_t chunks = (uint32_t)((K + kChunk - 1) / kChunk), b = blockIdx.x / chunks, c = blockIdx.x - b * chunks;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  return Place{((int64_t)b * (kThreads / 64) + wave) * kRows, (int64_t)c * kChunk + (threadIdx.x & 63) * 8};
}
int64_t blocks_of(int64_t rows, int64_t K) {
  return (rows + kRows * (kThreads / 64) - 1) / (kRows * (kThreads / 64)) * ((K + kChunk - 1) / kChunk);
}
// a grid has fewer than 2^32 threads (2^24 workgroups: 2^37 elements)
bool too_many(int64_t rows, int64_t K) {
  constexpr int64_t most = (int64_t)1 << 37;                   // the product below does not overflow
  return rows > most || K > most || blocks_of(rows, K) >= (int64_t)1 << 24;
}

// Stored layout: four lanes a group.
template <bool GATHER>
__global__ __launch_bounds__(kThreads) void mx_quantize_rows_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t K, int64_t ld,
                                                                    const int32_t* __restrict__ perm, uint8_t* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales) {
  const Place at = place_of(K);
  if (at.k >= K) return;                                       // K is a multiple of 32: the four lanes of a group together
  uint4 v[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (at.row + i < rows) v[i] = load8<GATHER>(x + (at.row + i) * ld, perm, at.k);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (at.row + i >= rows) break;
    uint32_t byte;
    const uint32_t q = mx_quantize8(v[i], byte);
    const int64_t e = (at.row + i) * K + at.k;
    *reinterpret_cast<uint32_t*>(codes + e / 2) = q;
    if ((threadIdx.x & 3) == 0) scales[e / kMxBlock] = (uint8_t)byte;
  }
}

// Operand layout: 16 lanes a row's piece of a panel; the channels from K on are zeros.
__global__ __launch_bounds__(kThreads) void mx_quantize_operand_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t K, int64_t ld,
                                                                       uint8_t* __restrict__ operand, size_t scales_at,
                                                                       uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const Place at = place_of(K);
  const int64_t p = at.k / kMxPanel;
  if (p >= mx_panels(K)) return;
  uint4 v[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    v[i] = make_uint4(0, 0, 0, 0);
    if (at.row + i < rows && at.k < K) v[i] = *reinterpret_cast<const uint4*>(x + (at.row + i) * ld + at.k);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (at.row + i >= rows) break;
    uint32_t byte;
    const uint32_t q = mx_quantize8(v[i], byte);               // zeros have byte 0 and codes 0
    const int64_t piece = p * rows + at.row + i;
    *reinterpret_cast<uint32_t*>(operand + piece * kMxRowBytes + (threadIdx.x & 15) * 4) = q;
    // four groups a piece: their bytes together in the piece's first lane
    uint32_t word = byte | dpp_u32<0x104>(byte) << 8 | dpp_u32<0x108>(byte) << 16 | dpp_u32<0x10C>(byte) << 24;      // row_shl 4, 8, 12
    if ((threadIdx.x & 15) == 0) *reinterpret_cast<uint32_t*>(operand + scales_at + piece * kMxRowScales) = word;
    if (codes && at.k < K) {
      const int64_t e = (at.row + i) * K + at.k;
      *reinterpret_cast<uint32_t*>(codes + e / 2) = q;
      if ((threadIdx.x & 3) == 0) scales[e / kMxBlock] = (uint8_t)byte;
    }
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
template <int FMT>
__device__ __forceinline__ uint4 dequantize8(uint32_t q, float scale, float T) {
  if constexpr (FMT == PQ_FMT_MXFP4) {
    // the conversion unit: exact below 2^128
    const auto two = [&](auto sel) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, sel)); };
    return make_uint4(two(std::integral_constant<int, 0>()), two(std::integral_constant<int, 1>()), two(std::integral_constant<int, 2>()),
                      two(std::integral_constant<int, 3>()));
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t code = q >> (4 * j) & 15u;
      if constexpr (FMT == PQ_FMT_NVFP4)
        v[j] = e2m1_value(code) * scale * T;                     // the first product is exact
      else
        v[j] = (float)((int)(code << 28) >> 28) * scale;
    }
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
}
// the stored value by binary32 operations, rounded once more to bf16 (nearest even)
template <int FMT>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const uint8_t* __restrict__ codes, const void* __restrict__ scales,
                                                              const float* __restrict__ tensor_scale, int64_t rows, int64_t K, int group_log2,
                                                              uint16_t* __restrict__ y, int64_t ldy) {
  const Place at = place_of(K);
  if (at.k >= K) return;
  const float T = FMT == PQ_FMT_NVFP4 ? tensor_scale[0] : 1.0f;
  uint32_t q[kRows];
  float scale[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (at.row + i >= rows) break;
    const int64_t e = (at.row + i) * K + at.k, g = e >> group_log2;
    q[i] = *reinterpret_cast<const uint32_t*>(codes + e / 2);
    scale[i] = FMT == PQ_FMT_MXFP4    ? mx_scale_value(((const uint8_t*)scales)[g])
               : FMT == PQ_FMT_NVFP4 ? e4m3_decode(((const uint8_t*)scales)[g])
                                     : ((const float*)scales)[g];
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (at.row + i >= rows) break;
    *reinterpret_cast<uint4*>(y + (at.row + i) * ldy + at.k) = dequantize8<FMT>(q[i], scale[i], T);
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
  if (too_many(rows, K)) return fail(PQ_ERR_SHAPE, "MXFP4 quantizer: rows=%lld K=%lld are too many for one call", (long long)rows, (long long)K);
  const int n = (int)blocks_of(rows, K);
  if (perm)
    mx_quantize_rows_kernel<true><<<n, kThreads, 0, st>>>((const uint16_t*)x, rows, K, ld, perm, codes, (uint8_t*)scales);
  else
    mx_quantize_rows_kernel<false><<<n, kThreads, 0, st>>>((const uint16_t*)x, rows, K, ld, perm, codes, (uint8_t*)scales);
  return check_hip(hipGetLastError(), "mx_quantize_rows_kernel");
}

int launch_mx_quantize_operand(const void* x, int64_t rows, int64_t K, int64_t ld, void* operand, uint8_t* codes, void* scales,
                               hipStream_t st) {
  if (too_many(rows, K)) return fail(PQ_ERR_SHAPE, "MXFP4 quantizer: rows=%lld K=%lld are too many for one call", (long long)rows, (long long)K);
  mx_quantize_operand_kernel<<<(int)blocks_of(rows, K), kThreads, 0, st>>>((const uint16_t*)x, rows, K, ld, (uint8_t*)operand,
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
  if (too_many(rows, K)) return fail(PQ_ERR_SHAPE, "pq_dequantize: rows=%lld K=%lld are too many for one call", (long long)rows, (long long)K);
  const int n = (int)blocks_of(rows, K), group_log2 = __builtin_ctz(group);
  switch (fmt) {
    case PQ_FMT_MXFP4:
      dequantize_kernel<PQ_FMT_MXFP4><<<n, kThreads, 0, st>>>(codes, scales, tensor_scale, rows, K, group_log2, (uint16_t*)y, ldy);
      break;
    case PQ_FMT_NVFP4:
      dequantize_kernel<PQ_FMT_NVFP4><<<n, kThreads, 0, st>>>(codes, scales, tensor_scale, rows, K, group_log2, (uint16_t*)y, ldy);
      break;
    default:
      dequantize_kernel<PQ_FMT_INT4><<<n, kThreads, 0, st>>>(codes, scales, tensor_scale, rows, K, group_log2, (uint16_t*)y, ldy);
  }
  return check_hip(hipGetLastError(), "dequantize_kernel");
}

}  // namespace pq
