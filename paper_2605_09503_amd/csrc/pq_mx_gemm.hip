// MXFP4 products, dense and grouped by expert, on the scaled matrix instruction: v_mfma_scale_f32_32x32x64_f8f6f4 multiplies
// E2M1 codes as they are and applies both operands' power-of-two scales inside, a 32-channel block a lane.
#include "pq_host.h"
#include "pq_mx.h"

namespace pq {

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

// The rows of the product that a workgroup's tile holds: `first` .. `end` of y, of expert `expert`.
struct Rows {
  int64_t first, end;
  int expert;
};

// Tile `tile` of `bm` rows, counted through the experts in turn (each expert's rows start a tile); end <= first where there is none.
__device__ __forceinline__ Rows find_rows(const MxCall& c, int64_t tile, int bm) {
  if (!c.offsets) return Rows{tile * bm, min((tile + 1) * bm, c.M), 0};
  const auto cut = [&](int e) { return min(max((int64_t)c.offsets[e], (int64_t)0), c.M); };
  for (int e = 0; e < c.experts; ++e) {
    const int64_t from = cut(e), to = cut(e + 1), tiles = to > from ? (to - from + bm - 1) / bm : 0;
    if (tile < tiles) return Rows{from + tile * bm, min(from + (tile + 1) * bm, to), e};
    tile -= tiles;
  }
  return Rows{0, 0, 0};
}

// One wave computes 32 x 32 outputs, operands straight from memory.
__global__ __launch_bounds__(64) void mx_gemm_simple_kernel(const MxCall c) {
  const int64_t across = (c.N + 31) / 32;
  const Rows rows = find_rows(c, blockIdx.x / across, 32);
  if (rows.end <= rows.first) return;
  const int lane = threadIdx.x, l = lane & 31, half = lane >> 5;
  const int64_t n0 = blockIdx.x % across * 32, panels = mx_panels(c.K);
  const uint8_t* w = c.w + (size_t)rows.expert * c.w_next;
  const int64_t wr = min(n0 + l, c.N - 1), m = rows.first + l;
  int64_t ar = min(m, rows.end - 1);
  if (c.rows) ar = c.rows[ar];
  const bool known = ar >= 0 && ar < c.a_rows;
  if (!known) ar = 0;
  const size_t a_scales = mx_scales_at(c.a_rows, c.K), w_scales = mx_scales_at(c.N, c.K);
  float16v acc = {};
  for (int64_t p = 0; p < panels; ++p) {
    const uint8_t *ap = c.a + (p * c.a_rows + ar) * kMxRowBytes, *wp = w + (p * c.N + wr) * kMxRowBytes;
    const uint8_t *as = c.a + a_scales + (p * c.a_rows + ar) * kMxRowScales, *ws = w + w_scales + (p * c.N + wr) * kMxRowScales;
    for (int s = 0; s < 4; ++s) {
      const int4v a = *reinterpret_cast<const int4v*>(ap + 16 * (2 * s + half)), b = *reinterpret_cast<const int4v*>(wp + 16 * (2 * s + half));
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(int8v{b[0], b[1], b[2], b[3], 0, 0, 0, 0}, int8v{a[0], a[1], a[2], a[3], 0, 0, 0, 0},
                                                            acc, 4, 4, 0, ws[2 * s + half], 0, as[2 * s + half]);
    }
  }
  if (m >= rows.end || !known) return;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t n = n0 + 8 * (i / 4) + 4 * half + i % 4;
    if (n >= c.N) continue;
    float v = acc[i];
    if (c.bias) v += bf16_to_f32(c.bias[rows.expert * c.N + n]);
    if (c.out_f32)
      ((float*)c.y)[m * c.ldy + n] = v;
    else
      ((uint16_t*)c.y)[m * c.ldy + n] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
}

}  // namespace

int run_mx_gemm(const MxCall& c, hipStream_t st) {
  if (c.M == 0) return PQ_OK;
  const int64_t tiles = (c.M + 31) / 32 + (c.offsets ? (c.experts < c.M ? c.experts : c.M) : 0);
  // a grid has fewer than 2^32 threads
  if (tiles * ((c.N + 31) / 32) >= (int64_t)1 << 26)
    return fail(PQ_ERR_SHAPE, "MXFP4 product: M=%lld N=%lld are too many tiles for one call", (long long)c.M, (long long)c.N);
  mx_gemm_simple_kernel<<<(unsigned)(tiles * ((c.N + 31) / 32)), 64, 0, st>>>(c);
  return check_hip(hipGetLastError(), "mx_gemm_kernel");
}

}  // namespace pq
