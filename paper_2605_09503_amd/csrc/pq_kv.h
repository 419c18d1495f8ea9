// Layout of the key-value cache and what its kernels share.
//
// A cache is pages x heads x (page / 32) blocks.  A block holds 32 consecutive tokens of one head: the keys' codes, their
// scales, the values' codes, their scales, each part in the order in which the lanes of a wave hold the operands of
// v_mfma_f32_16x16x32 in the attention of pq_attn_decode: one contiguous 16-byte load a lane, no exchange between lanes, and
// one base address a block.
//
//   keys    a block is two tiles (s) of 16 tokens (i).  As the product's first operand, lane 16 q + i holds token i's channels
//           32 kk + 8 q .. + 7 for the kk-th instruction: the dword of that chunk (4-bit codes) or its 16 bytes (bf16).
//   values  the product with the weights runs over tokens, so a lane needs one channel of eight tokens: lane 16 q + n holds
//           tokens 4 q + r (r < 4) of both tiles and D / 16 channels, one for each instruction.  16 channels of an instruction lie
//           in one group, so that the group's scale can go to the weights: lane n's channels are n PER .. n PER + PER - 1 of every
//           group, PER = group / 16 (NVFP4 and bf16: of the whole head).  Codes lie in quads of 16 bits (four channels of a
//           token); a dword holds the quads of tokens 2 p and 2 p + 1, which unpacks to pairs of tokens without a permute.
//   scales  INT4: the group's largest magnitude as bf16 (exact for bf16 input; the stored scale is fl32(max / 7)), the four tokens
//           of a lane adjacent.  NVFP4: E4M3 bytes, a lane's adjacent.
//
// INT4 codes lie as sign and magnitude, spread over their quad so that a mask, after a shift by one for the odd ones and a swap of
// bytes for the upper two, leaves an fp16 subnormal: the magnitude in low mantissa bits, z 2^-24 (odd ones z 2^-20), the sign on
// top.  (A nibble z + 8 takes 5 instructions for eight codes where this takes 7, but the sums over tokens then hold 8 times the
// weights, which leaves errors of 2^-24 of the largest weight where the codes themselves are zero.)
#pragma once
#include "pq_device.h"
#include "pq_host.h"

namespace pq {

constexpr int kBf16 = 3;                 // PQ_FMT_BF16; extends Fmt
constexpr int kKvBlock = 32;             // tokens of a block

template <int FMT_, int G_, int D_>
struct KvLayout {
  static constexpr int FMT = FMT_, G = G_, D = D_;
  static constexpr int NK = D / 32;                                  // instructions of a tile's scores
  static constexpr int NJ = D / 16;                                  // channels of a lane's values
  static constexpr int NQ = D / 64;                                  // quads of them
  static constexpr int NG = FMT == kBf16 ? 1 : D / G;                // groups of a head
  static constexpr int GV = FMT == kInt4 ? G : D;                    // run of channels that the lanes share
  static constexpr int PER = GV / 16;                                // of it, adjacent channels of a lane
  static constexpr int code_bytes = FMT == kBf16 ? 64 * D : 16 * D;
  static constexpr int scale_bytes = FMT == kBf16 ? 0 : FMT == kNvfp4 ? 2 * D : 64 * NG;
  static constexpr int v_at = code_bytes + scale_bytes;              // the values' part of a block
  static constexpr int bytes = 2 * v_at;

  // chunk c (8 channels) of key t
  static __host__ __device__ constexpr int k_chunk(int t, int c) {
    const int s = t >> 4, i = t & 15, kk = c >> 2, q = c & 3, e = s * NK + kk;
    return FMT == kBf16 ? (e * 64 + q * 16 + i) * 16 : ((e >> 2) * 64 + q * 16 + i) * 16 + (e & 3) * 4;
  }
  // channel of nibble / element j of lane n's values
  static __host__ __device__ constexpr int v_channel(int n, int j) { return j / PER * GV + n * PER + j % PER; }
  // 4-bit codes: quad jq (elements 4 jq .. + 3) of lane n of value t
  static __host__ __device__ constexpr int v_quad(int t, int n, int jq) {
    const int s = t >> 4, q = (t & 15) >> 2, r = t & 3, f = (s * 2 + (r >> 1)) * NQ + jq;
    return v_at + ((f >> 2) * 64 + q * 16 + n) * 16 + (f & 3) * 4 + (r & 1) * 2;
  }
  // bf16: elements 2 w, 2 w + 1 of lane n of value t
  static __host__ __device__ constexpr int v_pair(int t, int n, int w) {
    const int s = t >> 4, q = (t & 15) >> 2, r = t & 3, f = (s * 4 + r) * (D / 32) + w;
    return v_at + ((f >> 2) * 64 + q * 16 + n) * 16 + (f & 3) * 4;
  }
  // INT4: scale of group g of token t, the same for keys and values (relative to the part's scales)
  static __host__ __device__ constexpr int int_scale_at(int t, int g) {
    const int s = t >> 4, q = (t & 15) >> 2, r = t & 3;
    return code_bytes + (((q * 2 + s) * 4 + r) * NG + g) * 2;
  }
  // NVFP4: scale byte of group g of key t; of value t
  static __host__ __device__ constexpr int k_byte_at(int t, int g) {
    const int s = t >> 4, i = t & 15, kk = g >> 1, half = g & 1;
    return code_bytes + ((s * 2 + half) * 16 + i) * NK + kk;
  }
  static __host__ __device__ constexpr int v_byte_at(int t, int g) {
    const int s = t >> 4, q = (t & 15) >> 2, r = t & 3;
    return v_at + code_bytes + (g * 4 + q) * 8 + s * 4 + (r & 1) * 2 + (r >> 1);
  }
};

// INT4: code c (0 .. 3) of a quad
__device__ __forceinline__ constexpr int int_mag_at(int c) { return (c & 2) * 4 + (c & 1) * 3; }       // 0, 3, 8, 11
__device__ __forceinline__ constexpr int int_sign_at(int c) { return 15 - (c & 2) * 4 - (c & 1); }     // 15, 14, 7, 6
// Two quads side by side, from eight values (pairs of bf16, values 2 i and 2 i + 1 in x[i]; quads of values 0 .. 3 and 4 .. 7):
// x * inv (an inverse a pair) rounded to the nearest integer (ties to even), below 7.5 in magnitude.  Adding 2^23 leaves the integer in
// the low bits under a constant; the words are summed at the codes' places, the constants taken off once.  Signs go two at a time.
__device__ __forceinline__ uint32_t int_encode8(const uint32_t (&x)[4], const float (&inv)[4]) {
  constexpr uint32_t kBase = 0x4B000000u;                              // bits of 2^23
  uint32_t mags = 0, bases = 0, signs = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const float v = c & 1 ? bf16_hi(x[c / 2]) : bf16_lo(x[c / 2]);
    const int at = int_mag_at(c & 3) + (c & 4) * 4;
    mags += as_u32(fabsf(v * inv[c / 2]) + 8388608.0f) << at;
    bases += kBase << at;
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {                                        // values c and c + 4: signs at bits 15 and 31
    const uint32_t two = __builtin_amdgcn_perm(x[c / 2 + 2], x[c / 2], c & 1 ? 0x07060302u : 0x05040100u);
    signs |= (two >> (15 - int_sign_at(c))) & (0x00010001u << int_sign_at(c));
  }
  return (mags - bases) | signs;
}

// Two quads side by side: codes a of both as a pair of fp16 subnormals, the odd ones 16 times as large.
struct IntCodes {
  uint32_t d, swapped;
  __device__ __forceinline__ explicit IntCodes(uint32_t x) : d(x), swapped(__builtin_amdgcn_perm(0u, x, 0x02030001u)) {}
  __device__ __forceinline__ uint32_t pair(int a) const {
    const uint32_t x = a & 2 ? swapped : d;
    return a & 1 ? (x << 1) & 0x80708070u : x & 0x80078007u;
  }
  // the integers
  __device__ __forceinline__ void values(int a, float& lo, float& hi) const {
    typedef _Float16 half2 __attribute__((ext_vector_type(2)));
    const half2 h = __builtin_bit_cast(half2, pair(a));
    const float unit = a & 1 ? 1048576.0f : 16777216.0f;
    lo = __builtin_fmaf((float)h.x, unit, 0.0f);
    hi = __builtin_fmaf((float)h.y, unit, 0.0f);
  }
};

// what the kernels need of a pq_kv_cache
struct KvView {
  uint8_t* data;
  int64_t pages;
  int heads;
  int page_log2;
  const float *k_ts, *v_ts;
  __host__ __device__ int64_t slots() const { return pages << page_log2; }
};

// the block of a slot and the token's place in it
template <class L>
__device__ __forceinline__ uint8_t* kv_block(const KvView& c, int64_t slot, int head) {
  const uint32_t page = (uint32_t)(slot >> c.page_log2), in_page = (uint32_t)slot & ((1u << c.page_log2) - 1);
  const uint32_t block = ((page * c.heads + head) << (c.page_log2 - 5)) + (in_page >> 5);      // fewer than 2^31 in a cache
  return c.data + (uint64_t)block * L::bytes;
}

// f(KvLayout) for a format, group and head size that check_kv_cache let through
template <int FMT, int G, class F>
static inline int kv_by_dim(int D, F&& f) {
  switch (D) {
    case 64:
      if constexpr (G <= 64) return f(KvLayout<FMT, G, 64>{});
      break;
    case 128:
      if constexpr (G <= 128) return f(KvLayout<FMT, G, 128>{});
      break;
    case 256: return f(KvLayout<FMT, G, 256>{});
  }
  return fail(PQ_ERR_FORMAT, "no cache of groups of %d in heads of %d", G, D);
}
template <class F>
static inline int kv_dispatch(int fmt, int group, int D, F&& f) {
  if (fmt == kNvfp4) return kv_by_dim<kNvfp4, 16>(D, f);
  if (fmt == kBf16) return kv_by_dim<kBf16, 0>(D, f);
  if (group == 32) return kv_by_dim<kInt4, 32>(D, f);
  if (group == 64) return kv_by_dim<kInt4, 64>(D, f);
  if (group == 128) return kv_by_dim<kInt4, 128>(D, f);
  return kv_by_dim<kInt4, 256>(D, f);
}

}  // namespace pq
