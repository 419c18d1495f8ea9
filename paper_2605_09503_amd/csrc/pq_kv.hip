// Keys and values quantized into a cache's pages as they are produced, and read back (layout: pq_kv.h; the arithmetic is the
// pinned quantizer's of pq_quantize.hip, so a cache holds what pq_quantize_act would).  Bound by HBM: 2 bytes an element on
// one side, 0.5 and the scales on the other.
#include "pq_kv.h"
#include "pq_qgemm_common.h"

namespace pq {

namespace {

struct KvRows {                          // rows of [token][head][D] bf16; strides in elements
  uint16_t* p;
  int64_t ld, head;
};

// A workgroup: 32 tokens of one head, keys (z = 0) or values (z = 1).  Neighbouring lanes hold neighbouring channels of a token,
// so a wave reads whole rows, and the codes of neighbouring tokens meet in the L2.
template <class L>
__global__ __launch_bounds__(256) void kv_write_kernel(KvView cache, KvRows k, KvRows v, const int64_t* __restrict__ slots,
                                                       int64_t n) {
  constexpr int D = L::D;
  const int head = blockIdx.y;
  const int64_t t0 = (int64_t)blockIdx.x * kKvBlock;
  const bool values = blockIdx.z != 0;
  float T = 0.0f, encT = 0.0f;
  if constexpr (L::FMT == kNvfp4) {
    T = values ? *cache.v_ts : *cache.k_ts;
    encT = nv4_enc_scale(T);
  }
  const int64_t n_slots = cache.slots();
  if (!values) {
    constexpr int LPR = D / 8;                                 // lanes of a row, 8 channels each
    for (int u = threadIdx.x; u < kKvBlock * LPR; u += 256) {
      const int64_t row = t0 + u / LPR;
      const int c = u % LPR;
      const int64_t slot = row < n ? slots[row] : -1;
      const bool ok = slot >= 0 && slot < n_slots;             // other slots keep nothing
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (ok) x = *reinterpret_cast<const uint4*>(k.p + row * k.ld + head * k.head + c * 8);
      uint8_t* block = kv_block<L>(cache, ok ? slot : 0, head);
      const int t = (int)(slot & (kKvBlock - 1));
      if constexpr (L::FMT == kBf16) {
        if (ok) *reinterpret_cast<uint4*>(block + L::k_chunk(t, c)) = x;
      } else {
        const float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y),
                            bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w)};
        float a = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) a = fmaxf(a, fabsf(f[j]));
        constexpr int LPG = L::G / 8;                          // lanes of a group
        a = group_max<LPG>(a);
        uint32_t codes;
        if constexpr (L::FMT == kNvfp4) {
          const Nv4Scale sc = nv4_scale(a, T, encT);
          codes = 0;
          codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0] * sc.inv, f[1] * sc.inv, 1.0f, 0);
          codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2] * sc.inv, f[3] * sc.inv, 1.0f, 1);
          codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4] * sc.inv, f[5] * sc.inv, 1.0f, 2);
          codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6] * sc.inv, f[7] * sc.inv, 1.0f, 3);
          if (ok && c % LPG == 0) block[L::k_byte_at(t, c / LPG)] = (uint8_t)sc.byte;
        } else {
          const float inv = int_scale<kInt4>(a).inv;
          codes = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) codes |= int_encode(f[j], inv, j & 3) << (j & 4) * 4;
          if (ok && c % LPG == 0) *reinterpret_cast<uint16_t*>(block + L::int_scale_at(t, c / LPG)) = (uint16_t)(as_u32(a) >> 16);
        }
        if (ok) *reinterpret_cast<uint32_t*>(block + L::k_chunk(t, c)) = codes;
      }
    }
  } else {
    constexpr int PER = L::PER, RUNS = L::NJ / PER, PAIRS = PER / 2;       // runs of PER adjacent channels of a lane
    for (int u = threadIdx.x; u < kKvBlock * 16; u += 256) {
      const int64_t row = t0 + u / 16;
      const int lane = u % 16;
      const int64_t slot = row < n ? slots[row] : -1;
      const bool ok = slot >= 0 && slot < n_slots;
      uint32_t x[L::NJ / 2] = {};                              // pairs of channels
      if (ok) {
        const uint16_t* src = v.p + row * v.ld + head * v.head + lane * PER;
#pragma unroll
        for (int g = 0; g < RUNS; ++g) __builtin_memcpy(&x[g * PAIRS], __builtin_assume_aligned(src + g * L::GV, PER >= 8 ? 16 : PER * 2), PER * 2);
      }
      uint8_t* block = kv_block<L>(cache, ok ? slot : 0, head);
      const int t = (int)(slot & (kKvBlock - 1));
      if constexpr (L::FMT == kBf16) {
        if (ok)
#pragma unroll
          for (int w = 0; w < L::NJ / 2; ++w) *reinterpret_cast<uint32_t*>(block + L::v_pair(t, lane, w)) = x[w];
      } else {
        uint32_t codes[(L::NJ + 7) / 8] = {};
#pragma unroll
        for (int g = 0; g < RUNS; ++g) {
          float a = 0.0f;
#pragma unroll
          for (int j = 0; j < PAIRS; ++j) a = fmaxf(a, fmaxf(fabsf(bf16_lo(x[g * PAIRS + j])), fabsf(bf16_hi(x[g * PAIRS + j]))));
          constexpr int LPG = L::G / PER;                      // lanes of a group
          a = group_max<LPG>(a);
          float inv;
          if constexpr (L::FMT == kNvfp4) {
            const Nv4Scale sc = nv4_scale(a, T, encT);
            inv = sc.inv;
            if (ok && lane % LPG == 0) block[L::v_byte_at(t, lane / LPG)] = (uint8_t)sc.byte;
          } else {
            inv = int_scale<kInt4>(a).inv;
            if (ok && lane == 0) *reinterpret_cast<uint16_t*>(block + L::v_at + L::int_scale_at(t, g)) = (uint16_t)(as_u32(a) >> 16);
          }
#pragma unroll
          for (int j = 0; j < PAIRS; ++j) {
            const int at = g * PER + 2 * j;                    // nibble of the first of two
            const float lo = bf16_lo(x[g * PAIRS + j]), hi = bf16_hi(x[g * PAIRS + j]);
            if constexpr (L::FMT == kNvfp4) codes[at / 8] |= nv4_code_pair(lo, hi, inv) << (at % 8 * 4);
            else codes[at / 8] |= (int_encode(lo, inv, at & 3) | int_encode(hi, inv, (at + 1) & 3)) << (at & 4) * 4;
          }
        }
        if (ok)
#pragma unroll
          for (int jq = 0; jq < L::NQ; ++jq)
            *reinterpret_cast<uint16_t*>(block + L::v_quad(t, lane, jq)) = (uint16_t)(codes[jq / 2] >> (jq % 2 * 16));
      }
    }
  }
}

// values: INT4 z * s, NVFP4 value * s_b * T, every step one binary32 operation
template <class L>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView cache, const int64_t* __restrict__ slots, int64_t n, KvRows k, KvRows v) {
  constexpr int D = L::D;
  const int head = blockIdx.y;
  const int64_t t0 = (int64_t)blockIdx.x * kKvBlock;
  const bool values = blockIdx.z != 0;
  float T = 0.0f;
  if constexpr (L::FMT == kNvfp4) T = values ? *cache.v_ts : *cache.k_ts;
  const int64_t n_slots = cache.slots();
  const int64_t rows = min((int64_t)kKvBlock, n - t0);
  if (!values) {
    constexpr int LPR = D / 8;
    for (int u = threadIdx.x; u < rows * LPR; u += 256) {
      const int64_t row = t0 + u / LPR;
      const int c = u % LPR;
      const int64_t slot = slots[row];
      const bool ok = slot >= 0 && slot < n_slots;
      uint4 y = make_uint4(0u, 0u, 0u, 0u);                    // what another slot reads as
      if (ok) {
        const uint8_t* block = kv_block<L>(cache, slot, head);
        const int t = (int)(slot & (kKvBlock - 1));
        if constexpr (L::FMT == kBf16) {
          y = *reinterpret_cast<const uint4*>(block + L::k_chunk(t, c));
        } else {
          const uint32_t codes = *reinterpret_cast<const uint32_t*>(block + L::k_chunk(t, c));
          float f[8];
          if constexpr (L::FMT == kNvfp4) {
            const float s = e4m3_decode(block[L::k_byte_at(t, c / 2)]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes >> (8 * j), 1.0f, 0);
              f[2 * j] = two[0] * s * T;
              f[2 * j + 1] = two[1] * s * T;
            }
          } else {
            const float a = as_f32((uint32_t)*reinterpret_cast<const uint16_t*>(block + L::int_scale_at(t, c / (L::G / 8))) << 16);
            const float s = div_const(a, 7.0f, 1.0f / 7.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = int_decode(codes >> (j & 4) * 4, j & 3) * s;
          }
          y = make_uint4(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]), cvt_pk_bf16(f[6], f[7]));
        }
      }
      *reinterpret_cast<uint4*>(k.p + row * k.ld + head * k.head + c * 8) = y;
    }
  } else {
    constexpr int PER = L::PER, RUNS = L::NJ / PER, PAIRS = PER / 2;
    for (int u = threadIdx.x; u < rows * 16; u += 256) {
      const int64_t row = t0 + u / 16;
      const int lane = u % 16;
      const int64_t slot = slots[row];
      const bool ok = slot >= 0 && slot < n_slots;
      uint32_t y[L::NJ / 2] = {};
      if (ok) {
        const uint8_t* block = kv_block<L>(cache, slot, head);
        const int t = (int)(slot & (kKvBlock - 1));
        if constexpr (L::FMT == kBf16) {
#pragma unroll
          for (int w = 0; w < L::NJ / 2; ++w) y[w] = *reinterpret_cast<const uint32_t*>(block + L::v_pair(t, lane, w));
        } else {
          uint32_t quad[L::NQ];
#pragma unroll
          for (int jq = 0; jq < L::NQ; ++jq) quad[jq] = *reinterpret_cast<const uint16_t*>(block + L::v_quad(t, lane, jq));
#pragma unroll
          for (int g = 0; g < RUNS; ++g) {
            float s;
            if constexpr (L::FMT == kNvfp4) s = e4m3_decode(block[L::v_byte_at(t, lane / (L::G / PER))]);
            else s = div_const(as_f32((uint32_t)*reinterpret_cast<const uint16_t*>(block + L::v_at + L::int_scale_at(t, g)) << 16), 7.0f,
                               1.0f / 7.0f);
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) {
              const int at = g * PER + 2 * j;
              if constexpr (L::FMT == kNvfp4) {
                const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(quad[at / 4] >> (at % 4 * 4), 1.0f, 0);
                y[g * PAIRS + j] = cvt_pk_bf16(f[0] * s * T, f[1] * s * T);
              } else {
                y[g * PAIRS + j] = cvt_pk_bf16(int_decode(quad[at / 4], at & 3) * s, int_decode(quad[at / 4], (at + 1) & 3) * s);
              }
            }
          }
        }
      }
      uint16_t* dst = v.p + row * v.ld + head * v.head + lane * PER;
#pragma unroll
      for (int g = 0; g < RUNS; ++g) __builtin_memcpy(__builtin_assume_aligned(dst + g * L::GV, PER >= 8 ? 16 : PER * 2), &y[g * PAIRS], PER * 2);
    }
  }
}

}  // namespace

size_t kv_cache_bytes(pq_format fmt, int group, int kv_heads, int head_dim, int page, int64_t pages) {
  size_t bytes = 0;
  (void)kv_dispatch(fmt, group, head_dim, [&](auto l) {
    bytes = (size_t)pages * kv_heads * (page / kKvBlock) * decltype(l)::bytes;
    return PQ_OK;
  });
  return bytes;
}

KvView kv_view(const pq_kv_cache& c) {
  KvView v{(uint8_t*)c.data, c.pages, c.kv_heads, 0, c.k_tensor_scale, c.v_tensor_scale};
  while ((1 << v.page_log2) < c.page) ++v.page_log2;
  return v;
}

int run_kv_write(const pq_kv_cache& c, const void* k, int64_t k_ld, int64_t k_head, const void* v, int64_t v_ld, int64_t v_head,
                 const int64_t* slots, int64_t n, hipStream_t st) {
  return kv_dispatch(c.fmt, c.group, c.head_dim, [&](auto l) {
    const dim3 grid((unsigned)((n + kKvBlock - 1) / kKvBlock), c.kv_heads, 2);
    kv_write_kernel<decltype(l)><<<grid, 256, 0, st>>>(kv_view(c), KvRows{(uint16_t*)k, k_ld, k_head}, KvRows{(uint16_t*)v, v_ld, v_head},
                                                      slots, n);
    return check_hip(hipGetLastError(), "pq_kv_write");
  });
}

int run_kv_read(const pq_kv_cache& c, const int64_t* slots, int64_t n, void* k, int64_t k_ld, int64_t k_head, void* v, int64_t v_ld,
                int64_t v_head, hipStream_t st) {
  return kv_dispatch(c.fmt, c.group, c.head_dim, [&](auto l) {
    const dim3 grid((unsigned)((n + kKvBlock - 1) / kKvBlock), c.kv_heads, 2);
    kv_read_kernel<decltype(l)><<<grid, 256, 0, st>>>(kv_view(c), slots, n, KvRows{(uint16_t*)k, k_ld, k_head},
                                                     KvRows{(uint16_t*)v, v_ld, v_head});
    return check_hip(hipGetLastError(), "pq_kv_read");
  });
}

}  // namespace pq
