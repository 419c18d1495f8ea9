// Attention of one new token a sequence over the paged cache (layout: pq_kv.h).
//
//   out = sum_t p_t v_t / sum_t p_t,   p_t = 2^(c s_t - M),   s_t = q . k_t,   c = scale log2 e,   M any reference
//
// The queries that share a key head are the columns of both products, so the cache is read once for all of them:
//   scores   S[token, head]  = K Q      v_mfma_f32_16x16x32, 16 tokens x 32 channels of keys, codes straight from memory
//   outputs  O[channel, head] += V' P   the same instruction, 16 channels x 32 tokens; the scores' result layout (lane 16 q + h
//                                       holds tokens 4 q .. 4 q + 3 of head h) is the operand layout of the weights
// Nothing goes through LDS or between lanes in the loop.
//
// Bound by the reading of the cache where it is long: two flops a stored number and query are far below what the matrix unit gives, and
// a block's vector work (unpacking, eight exponentials a lane) fits beside its loads.  Measured (MI355X, a copy runs at 4.9 TB/s):
//   64 sequences up to 24 000 tokens, 8 heads of 128, INT4/64: 1.05 GB in 192 us, 5.5 TB/s
//   one of 131 000 tokens, 8 heads of 128, INT4/128:         138 MB in 35 us, 3.9 TB/s
//   8 up to 4600 tokens, 24 heads of 128, bf16:          304 MB in 62 us, 4.9 TB/s
// Short work is bound by the chain of what waits for one another, by clock stamps of every workgroup: lengths and plan 1.4 to 2.2 us,
// pages 1.2, first block 0.7 to 2.4, the waves' join 0.6 to 1.8, a part's store and counter 1.1, fetch and sum of parts 1.1 to 2 a
// level.  A call over 19 tokens takes 6 us.
//
// Each wave keeps one block ahead in registers.  Two ahead (4-bit formats, heads up to 128) cost 10 to 30 % in short sequences and
// gave nothing in long ones; eight waves a workgroup, three or four a SIMD gave less than they cost elsewhere.
#include "pq_kv.h"
#include "pq_qgemm_common.h"

namespace pq {

KvView kv_view(const pq_kv_cache& c);

namespace {

typedef float float4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

constexpr int kAttnWaves = 4;            // of a workgroup; they take a segment's blocks in turn
constexpr int kUnits = 256;              // compute units
constexpr int kMaxSplits = 1024;         // workgroups that may hold a part of a pair: counters in the workspace
// The limits of the plan below (what they say and what they are worth is told there).
constexpr int kLeastBlocks = 4, kWholeBlocks = 20, kMostParts = 64, kSoloBlocks = 8, kExtraBlocks = 64, kPartBlocks = 32;

constexpr float kNoReference = -1e38f;   // M before the first token
// A weight with its value's scale stays below 2^15 (fp16); M follows when it would not, to 2^7 and less: seldom, so that neither the
// maximum over the lanes nor the rescaling is part of an ordinary block.
constexpr float kHeadroom = 15.0f, kStart = 7.0f;

__device__ __forceinline__ float4_t mfma(const uint4_t& a, const uint4_t& b, const float4_t& c, IntC<0>) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ float4_t mfma(const uint4_t& a, const uint4_t& b, const float4_t& c, IntC<1>) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// two fp32 to fp16, nearest even, packed
__device__ __forceinline__ uint32_t cvt_pk_f16(float lo, float hi) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){lo, hi}, half2_t));
}

// a value that the compiler takes for new: what follows from it is not kept in registers across the loops before
__device__ __forceinline__ int renewed(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// over the four lanes of a column (16 apart)
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// What a lane holds of a block, codes (or bf16 values) and scales.
template <class L>
struct Part {
  static constexpr int NP = L::code_bytes / 1024;            // 16-byte pieces of the codes
  static constexpr int NS = L::FMT == kInt4 ? L::NG : 1;
  static constexpr int registers = 4 * NP + (L::FMT == kInt4 ? 4 * NS : L::FMT == kNvfp4 ? 2 : 0);
  uint4_t c[NP], sc[NS];

  __device__ __forceinline__ void load_codes(const uint8_t* __restrict__ p, uint32_t lane) {
#pragma unroll
    for (int i = 0; i < NP; ++i) c[i] = *reinterpret_cast<const uint4_t*>(p + (lane * 16 + i * 1024));
  }
  // INT4: 16-byte pieces of the four tokens 4 q .. of both tiles
  __device__ __forceinline__ void load_int_scales(const uint8_t* __restrict__ p, uint32_t lane) {
#pragma unroll
    for (int i = 0; i < NS; ++i) sc[i] = *reinterpret_cast<const uint4_t*>(p + ((lane >> 4) * (16 * NS) + L::code_bytes + i * 16));
  }
  // INT4: the scale of group g of token (s, r) of the lane
  __device__ __forceinline__ float h(int s, int r, int g) const {
    const int x = (s * 4 + r) * L::NG + g;
    const uint32_t two = sc[x >> 3][(x >> 1) & 3];
    return x & 1 ? bf16_hi(two) : bf16_lo(two);
  }
};

template <class L>
struct Keys : Part<L> {
  __device__ __forceinline__ void load(const uint8_t* __restrict__ p, uint32_t lane) {
    this->load_codes(p, lane);
    if constexpr (L::FMT == kInt4) this->load_int_scales(p, lane);
    if constexpr (L::FMT == kNvfp4) {                        // the bytes of tile s in sc[s] (16 channels' tiles: two words each)
      constexpr int NK = L::NK;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint8_t* at = p + (((lane >> 5) * 16 + (lane & 15)) * NK + (L::code_bytes + s * 32 * NK));
        if constexpr (NK == 2) this->sc[0][s] = *reinterpret_cast<const uint16_t*>(at);
        else if constexpr (NK == 4) this->sc[0][s] = *reinterpret_cast<const uint32_t*>(at);
        else {
          const uint2 two = *reinterpret_cast<const uint2*>(at);
          this->sc[0][2 * s] = two.x;
          this->sc[0][2 * s + 1] = two.y;
        }
      }
    }
  }
};

template <class L>
struct Values : Part<L> {
  __device__ __forceinline__ void load(const uint8_t* __restrict__ block, uint32_t lane) {
    const uint8_t* p = block + L::v_at;
    this->load_codes(p, lane);
    if constexpr (L::FMT == kInt4) this->load_int_scales(p, lane);
    if constexpr (L::FMT == kNvfp4) {
      const uint2 two = *reinterpret_cast<const uint2*>(p + (((lane & 15) / (256 / L::D) * 4 + (lane >> 4)) * 8 + L::code_bytes));
      this->sc[0][0] = two.x;
      this->sc[0][1] = two.y;
    }
  }
  // tokens outside [lo, hi) of the block become zeros: their weights are, and what lies there may be NaN
  __device__ __forceinline__ void clear(int lane, int lo, int hi) {
    const int q = lane >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = s * 16 + q * 4 + r;
        const bool keep = (t >= lo) & (t < hi);
        if constexpr (L::FMT == kBf16) {
#pragma unroll
          for (int w = 0; w < L::D / 32; ++w) {
            const int f = (s * 4 + r) * (L::D / 32) + w;
            this->c[f >> 2][f & 3] = keep ? this->c[f >> 2][f & 3] : 0u;
          }
        } else if constexpr (L::FMT == kNvfp4) {
          this->sc[0][s] &= keep ? ~0u : ~(0xFFu << (8 * ((r & 1) * 2 + (r >> 1))));
        } else {
#pragma unroll
          for (int g = 0; g < L::NG; ++g) {
            const int x = (s * 4 + r) * L::NG + g;
            this->sc[x >> 3][(x >> 1) & 3] &= keep ? ~0u : ~(0xFFFFu << (16 * (x & 1)));
          }
        }
      }
  }
};

// The queries as the second operand, and what else the loop keeps of a pair.
template <class L>
struct Query {
  uint4_t q[L::NK];
  float c;                         // scores to powers of two

  // count queries of the key head; columns past them are zeros
  __device__ __forceinline__ void fetch(const AttnCall& a, const uint16_t* __restrict__ src, int count, int lane) {
    const int kq = lane >> 4, n = lane & 15;
#pragma unroll
    for (int kk = 0; kk < L::NK; ++kk) {
      q[kk] = (uint4_t){0u, 0u, 0u, 0u};
      if (n < count) q[kk] = *reinterpret_cast<const uint4_t*>(src + n * a.q_head + kk * 32 + kq * 8);
    }
  }
  __device__ __forceinline__ void convert(const AttnCall& a, float key_unit) {
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;           // c is positive: the sign goes to the query
    const float scale = fabsf(a.scale) * 1.4426950408889634f * key_unit;
    uint4_t x[L::NK];
    float top = 0.0f;
#pragma unroll
    for (int kk = 0; kk < L::NK; ++kk) x[kk] = q[kk] ^ flip;
    if constexpr (L::FMT == kBf16) {
      c = scale;
#pragma unroll
      for (int kk = 0; kk < L::NK; ++kk) q[kk] = x[kk];
    } else {
      // fp16, the head's largest in [2^13, 2^14): bf16's eight bits stay exact down to 2^-27 of it
#pragma unroll
      for (int kk = 0; kk < L::NK; ++kk)
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, fmaxf(fabsf(bf16_lo(x[kk][w])), fabsf(bf16_hi(x[kk][w]))));
      const int e = max((int)(as_u32(column_max(top)) >> 23) - 127, -100);
      const float down = as_f32((uint32_t)(127 + 13 - e) << 23);
      c = ldexpf(scale, e - 13);
#pragma unroll
      for (int kk = 0; kk < L::NK; ++kk) {
        float f[8];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          f[2 * w] = bf16_lo(x[kk][w]) * down;
          f[2 * w + 1] = bf16_hi(x[kk][w]) * down;
        }
        if constexpr (L::FMT == kNvfp4) {
#pragma unroll
          for (int w = 0; w < 4; ++w) q[kk][w] = cvt_pk_f16(f[2 * w], f[2 * w + 1]);
        } else {
#pragma unroll
          for (int w = 0; w < 4; ++w) {                              // the order of IntCodes, and its factor
            const float m = w & 1 ? 0.0625f : 1.0f;
            q[kk][w] = cvt_pk_f16(f[w] * m, f[w + 4] * m);
          }
        }
      }
    }
  }
};

// The running result of a wave: O[channel n = 4 q + r of instruction j, head] and the sums of the weights, both times 2^M.
template <class L>
struct Result {
  float4_t acc[L::NJ];
  float m, l;

  __device__ __forceinline__ void clear() {
    m = kNoReference;
    l = 0.0f;
#pragma unroll
    for (int j = 0; j < L::NJ; ++j) acc[j] = (float4_t){0.0f, 0.0f, 0.0f, 0.0f};
  }
};

// scores of a block's tokens, 16 s + 4 q + r in s_[.][s][r]
template <class L>
__device__ __forceinline__ void block_scores(const Keys<L>& x, const Query<L>& query, float4_t (&s_)[2]) {
  constexpr IntC<L::FMT == kBf16> kType{};
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float4_t sum;
#pragma unroll
    for (int kk = 0; kk < L::NK; ++kk) {
      const int e = s * L::NK + kk;
      uint4_t a;
      if constexpr (L::FMT == kBf16) {
        a = x.c[e];
      } else {
        const uint32_t d = x.c[e >> 2][e & 3];
        if constexpr (L::FMT == kInt4) {
#pragma unroll
          for (int w = 0; w < 4; ++w) a[w] = IntCodes(d).pair(w);
        } else {
          // the bytes of chunks kk and kk ^ 1 convert together
          const uint32_t bytes = L::NK == 8 ? x.sc[0][2 * s + (kk >> 2)] : x.sc[0][s];
          const half2_t two = kk & 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)bytes, 1.0f, 1)
                                     : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)bytes, 1.0f, 0);
          const half2_t sc = kk & 1 ? (half2_t){two.y, two.y} : (half2_t){two.x, two.x};
          a[0] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 0) * sc);
          a[1] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 1) * sc);
          a[2] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 2) * sc);
          a[3] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 3) * sc);
        }
      }
      // INT4: a group's sum is scaled as soon as it is there
      constexpr int KG = L::FMT == kInt4 ? L::G / 32 : L::NK;
      sum = mfma(a, query.q[kk], kk % KG ? sum : (float4_t){0.0f, 0.0f, 0.0f, 0.0f}, kType);
      if (kk % KG != KG - 1) continue;
      if constexpr (L::FMT == kInt4) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s_[s][r] = kk / KG ? __builtin_fmaf(x.h(s, r, kk / KG), sum[r], s_[s][r]) : x.h(s, r, 0) * sum[r];
      } else {
        s_[s] = sum;
      }
    }
  }
}

// their weights, and the values' sums; tokens outside [lo, hi) are left out
template <class L>
__device__ __forceinline__ void block_outputs(Values<L>& x, float4_t (&s_)[2], const Query<L>& query, Result<L>& out, int lane,
                                              int lo, int hi) {
  constexpr IntC<L::FMT == kBf16> kType{};
  const int kq = lane >> 4;
  const bool part = lo > 0 || hi < kKvBlock;                           // wave-uniform
  if (__builtin_expect(part, 0)) x.clear(lane, lo, hi);
  // INT4: 2^eb bounds the lane's scales; kept from going where the sum of the weights would overflow
  float eb = 0.0f;
  if constexpr (L::FMT == kInt4) {
    ushort2_t top = {0, 0};
#pragma unroll
    for (int w = 0; w < 4 * L::NG; ++w) {
      const uint32_t two = x.sc[w >> 2][w & 3];        // by value: a bit cast of a vector's element takes its first
      top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort2_t, two));
    }
    eb = (float)(max((int)max(top.x, top.y) >> 7, 127 - 80) - 126);
  }
  // weights
  float p[2][4];
  if (__builtin_expect(part, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = (i >> 2) * 16 + kq * 4 + (i & 3);
      s_[i >> 2][i & 3] = ((t < lo) | (t >= hi)) ? -1e38f : s_[i >> 2][i & 3];
    }
  }
  float top = fmaxf(s_[0][0], s_[0][1]);
#pragma unroll
  for (int i = 2; i < 8; ++i) top = fmaxf(top, s_[i >> 2][i & 3]);
  const float bound = top * query.c + eb;
  if (__builtin_expect(__any(bound > out.m + kHeadroom), 0)) {
    const float b = column_max(bound);
    const float m = b > out.m + kHeadroom ? b - kStart : out.m;
    const float f = __builtin_amdgcn_exp2f(out.m - m);
    out.m = m;
    out.l *= f;
#pragma unroll
    for (int j = 0; j < L::NJ; ++j) out.acc[j] *= f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s_[i >> 2][i & 3], query.c, -out.m));
    if (__builtin_expect(part, 0)) {
      const int t = (i >> 2) * 16 + kq * 4 + (i & 3);
      w = ((t < lo) | (t >= hi)) ? 0.0f : w;
    }
    p[i >> 2][i & 3] = w;
    out.l += w;
  }
  // Outputs.  The 4-bit formats take a weight (INT4: times its value's scale) in fp16: an error of at most 2^-11 of a token's share,
  // an eighth of what rounding the output to bf16 may add.  A second fp16 for the rest costs 3 to 6 % (64 sequences up to 24 000 tokens
  // 192 -> 201 us, 32 up to 4099 27.0 -> 28.4, one of 131 000 35.4 -> 36.4).  Where weight and scale fall below 2^-20 of the largest,
  // fp16's subnormals take further bits.
  if constexpr (L::FMT == kInt4) {
#pragma unroll
    for (int g = 0; g < L::NG; ++g) {
      uint4_t w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = i >> 1, r = (i & 1) * 2;
        w[i] = cvt_pk_f16(p[s][r] * x.h(s, r, g), p[s][r + 1] * x.h(s, r + 1, g));
      }
#pragma unroll
      for (int j = g * L::PER; j < (g + 1) * L::PER; ++j) {
        uint4_t a;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int f = i * L::NQ + j / 4;
          a[i] = IntCodes(x.c[f >> 2][f & 3]).pair(j & 3);
        }
        out.acc[j] = mfma(a, w, out.acc[j], kType);
      }
    }
  } else if constexpr (L::FMT == kNvfp4) {
    uint4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = cvt_pk_f16(p[i >> 1][i & 1], p[i >> 1][(i & 1) + 2]);
    half2_t sc[4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      sc[2 * s] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x.sc[0][s], 1.0f, 0);
      sc[2 * s + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x.sc[0][s], 1.0f, 1);
    }
#pragma unroll
    for (int jq = 0; jq < L::NQ; ++jq) {
      uint32_t even[2], odd[2];                    // bytes: channels 0 and 2 (1 and 3) of tokens 0 | 2, then of tokens 1 | 3
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int f0 = (s * 2) * L::NQ + jq, f1 = (s * 2 + 1) * L::NQ + jq;
        const uint32_t x0 = x.c[f0 >> 2][f0 & 3], x1 = x.c[f1 >> 2][f1 & 3];
        even[s] = (x0 & 0x0F0F0F0Fu) | ((x1 << 4) & 0xF0F0F0F0u);
        odd[s] = ((x0 >> 4) & 0x0F0F0F0Fu) | (x1 & 0xF0F0F0F0u);
      }
      auto channel = [&](const uint32_t (&d)[2], auto byte, int j) {
        constexpr int B = decltype(byte)::value;
        uint4_t a;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          a[2 * s] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d[s], 1.0f, B) * sc[2 * s]);
          a[2 * s + 1] = h2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d[s], 1.0f, B + 2) * sc[2 * s + 1]);
        }
        out.acc[j] = mfma(a, w, out.acc[j], kType);
      };
      channel(even, IntC<0>{}, jq * 4);
      channel(odd, IntC<0>{}, jq * 4 + 1);
      channel(even, IntC<1>{}, jq * 4 + 2);
      channel(odd, IntC<1>{}, jq * 4 + 3);
    }
  } else {
    // the weights as two bf16 each, 16 bits: one would add as much error as the output's own rounding
    uint4_t w[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = p[i >> 1][(i & 1) * 2], p1 = p[i >> 1][(i & 1) * 2 + 1];
      const uint32_t two = cvt_pk_bf16(p0, p1);
      w[0][i] = two;
      w[1][i] = cvt_pk_bf16(p0 - bf16_lo(two), p1 - bf16_hi(two));
    }
#pragma unroll
    for (int j = 0; j < L::NJ; ++j) {
      uint4_t a;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int f0 = (i * 2) * (L::D / 32) + j / 2, f1 = f0 + L::D / 32;
        a[i] = __builtin_amdgcn_perm(x.c[f1 >> 2][f1 & 3], x.c[f0 >> 2][f0 & 3], j & 1 ? 0x07060302u : 0x05040100u);
      }
      out.acc[j] = mfma(a, w[0], out.acc[j], kType);
      out.acc[j] = mfma(a, w[1], out.acc[j], kType);
    }
  }
}

// ------------------------------------------------------------------------ which blocks are whose
// A pair is a sequence and up to sixteen queries of one key head; workers (workgroups, or waves) share the blocks of all pairs.  Every
// wave works the plan out from the lengths, so that it holds for the lengths of this call, whatever the grid was sized for (one
// sequence of 2000 tokens where max_len is 131 072: 9.4 us; sized by max_len 18.0).  With `even` = all blocks / resident workers:
//
//   parts    where pairs are few: every pair in equal parts of up to `per` blocks, per = even to 1.5 even, the least with which each
//            part finds a resident worker: no worker then holds two pairs.  (48 sequences up to 5000 tokens, 2 heads: 14.5 us; per =
//            even only 18.3.)  A pair up to kWholeBlocks stays whole (128 pairs up to 300 tokens: 8.7 us, parted 10.0; but 64 pairs up
//            to 2000 with 40: 13.9, 12.2 with 20), a part is at least kLeastBlocks (8 pairs of 1500 tokens: 9.3 us; of 2 blocks 11.4, of
//            8 9.8), and a pair has at most kMostParts (4 pairs of 60 000 tokens, 8 queries each: 17.7 us; 32 parts 21.6, 128 20.0).
//   solo     a wave a pair, nothing to join, where pairs fill the workers and are short for their number: blocks of the longest <=
//            kSoloBlocks pairs / workers (2160 pairs up to 40 tokens: 10.8 us, a workgroup each 20.7; 2400 up to 1200 with a limit of
//            12: 105, 90 with 8).
//   whole    a worker a pair, where the longest has at most kExtraBlocks more than `even`: 600 pairs up to 800 tokens 18.9 us, in a row
//            26.9; 480 up to 3000 37.7, with 32 more 41.8; 400 up to 5000 with 128 more 33.6, 32.0 with 64.
//   parts    again, up to kMaxSplits of them, more than are resident, where `even` is below kPartBlocks: 800 pairs up to 300 tokens
//            but 8 of 3000 20.5 us, in a row 25.2; a bound of 64: 55.6 against 52.9 with 2400 pairs, 8 of them of 10 000 tokens.
//   in a row blocks numbered sequence by sequence, pair by pair, `even` of them a worker: the same work whatever the lengths, at up to
//            two joins a worker (512 pairs up to 24 000 tokens: 197 us, whole 232).
//
// Equal parts of long and short pairs leave an imbalance: 256 pairs up to 4099 tokens get up to 57 blocks a worker over a mean of 41
// (27 us, and half of the workers have ended their blocks by 18).
// Every wave goes through all lengths, so many sequences cost their number squared: 100 tokens, 8 heads, 32 queries, INT4: 256
// sequences 17 us, 1024 131, 4096 1580, 16 384 27 000, 65 535 433 000.  Past some 300 sequences, calls of 256 each are quicker.
struct Lengths {           // of a sequence: first attended token and end, first block, blocks (at least one)
  int first_token, end, first, n;
};
__device__ __forceinline__ Lengths lengths_of(const AttnCall& a, int length) {
  Lengths r;
  r.end = min(max(length, 0), a.max_len);
  r.first_token = a.window ? max(0, r.end - a.window) : 0;
  r.first = r.first_token / kKvBlock;
  r.n = max(1, (r.end + kKvBlock - 1) / kKvBlock - r.first);
  return r;
}
// sums over the lanes up to each, by exchanges inside rows of 16 lanes and broadcasts of a row's last lane: no LDS round trips
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);      // row_bcast 15 into rows 1 and 3
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast 31 into rows 2 and 3
}
// the largest of all lanes (none is negative)
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));
  return __builtin_amdgcn_readlane(max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false)), 63);
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

// a part's outputs, then (M, l) of its queries
template <class L>
constexpr uint32_t part_bytes_of() { return L::NJ * 1024 + 256; }

// the part of a pair that worker w holds, first the one that began it
__device__ __forceinline__ int part_slot(int w, int w_first) { return w == w_first ? 2 * w + 1 : 2 * w; }

// Waves a SIMD, and with them the registers of a wave: one where a block and the results pass 256 (16 sequences up to 8000 tokens,
// 4 heads of 256, INT4/32: 36.5 us, with two and what that spills 76.5).
template <class L>
constexpr int waves_of() { return L::D == 256 && (L::FMT == kBf16 || L::G == 32) ? 1 : 2; }
// the part buffer is written and read by workgroups of different chiplets in one launch: past the caches that they do not share
constexpr int kAgent = 16;               // sc1 of a buffer instruction
__device__ __forceinline__ void put_part(__amdgpu_buffer_rsrc_t buf, uint32_t at, uint32_t uniform, const float4_t& v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4_t, v), buf, at, uniform, kAgent);
}
__device__ __forceinline__ float4_t get_part(__amdgpu_buffer_rsrc_t buf, uint32_t at, uint32_t uniform) {
  return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(buf, at, uniform, kAgent));
}

template <class L>
__global__ __launch_bounds__((64 * kAttnWaves), (waves_of<L>())) void attn_decode_kernel(KvView cache, AttnCall a, int chunks,
                                                                                          uint32_t part_bytes) {
  constexpr int NJ = L::NJ, NW = kAttnWaves;
  constexpr int kWorkers = kUnits * waves_of<L>();                     // what is resident
  constexpr int JW = NJ / NW;                                          // instructions' outputs that a wave joins
  __shared__ float4_t shared_acc[NW][NJ][64];
  __shared__ float2 shared_ml[NW][16];
  __shared__ int last_one;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per_head = a.q_heads / cache.heads, pairs = cache.heads * chunks;      // pairs of a sequence
  const int width = (per_head + chunks - 1) / chunks;                  // queries of a pair
  int* counters = static_cast<int*>(a.ws);
  const auto parts = __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t*>(a.ws) + PQ_ATTN_DECODE_ZERO_BYTES, 0, part_bytes, 0x00027000);
  const float key_unit = L::FMT == kNvfp4 ? *cache.k_ts : L::FMT == kInt4 ? 16777216.0f / 7.0f : 1.0f;
  const float value_unit = L::FMT == kNvfp4 ? *cache.v_ts : L::FMT == kInt4 ? 16777216.0f / 7.0f : 1.0f;

  // the plan
  const int length0 = lane < a.seqs ? a.lengths[lane] : 0;             // of the first 64 sequences: often of all
  auto length_at = [&](int b0) { return b0 == 0 ? length0 : b0 + lane < a.seqs ? a.lengths[b0 + lane] : 0; };
  auto blocks_at = [&](int b0) { return b0 + lane < a.seqs ? lengths_of(a, length_at(b0)).n : 0; };
  int blocks = 0, longest = 0;                                         // of a pair of each sequence
  for (int b0 = 0; b0 < a.seqs; b0 += 64) {
    blocks += last_lane(wave_scan(blocks_at(b0)));
    longest = max(longest, wave_max(blocks_at(b0)));
  }
  auto parts_of = [&](int n, int per) { return n <= kWholeBlocks ? 1 : (n + per - 1) / per; };
  auto items_of = [&](int per) {                                       // workers of padded pairs
    int items = 0;
    for (int b0 = 0; b0 < a.seqs; b0 += 64) items += last_lane(wave_scan(b0 + lane < a.seqs ? parts_of(blocks_at(b0), per) : 0));
    return items * pairs;
  };
  const int even = max(max((blocks * pairs + kWorkers - 1) / kWorkers, kLeastBlocks), (longest + kMostParts - 1) / kMostParts);
  int per = even;
  bool padded = false, solo = false;
  if (a.seqs * pairs <= kWorkers) {
#pragma unroll 1
    for (int more = 0; more <= 4 && !padded; ++more) {
      per = even + even * more / 8;
      padded = items_of(per) <= min(kWorkers, (int)gridDim.x);
    }
  }
  if (!padded) {
    per = even;
    solo = a.seqs * pairs >= kWorkers && (int64_t)longest * kWorkers <= (int64_t)kSoloBlocks * a.seqs * pairs;
    if (solo || longest <= even + kExtraBlocks) {
      per = longest;
      padded = true;
    } else if (even < kPartBlocks) {
      padded = items_of(per) <= min(kMaxSplits, (int)gridDim.x);
    }
  }
  const int worker = solo ? blockIdx.x * NW + wave : blockIdx.x;
  // blocks of a pair in the numbering: padded to whole workers
  auto counted = [&](int n) { return padded ? (per == longest ? per : parts_of(n, per) * per) : n; };

  // All blocks and the last worker's share fit 31 bits (the host's limit is 2^30 before padding); idle workers' numbers may not.
  if ((int64_t)worker * per > INT32_MAX - per) return;
  const int u_begin = worker * per, u_end = u_begin + per;
  int u = u_begin, base = 0, b = 0;                                    // the sequence that holds block u, its first block `base`
  for (int b0 = 0;; b0 += 64) {
    if (b0 >= a.seqs) return;                                          // workers past the last block
    const int n = b0 + lane < a.seqs ? counted(blocks_at(b0)) * pairs : 0, incl = wave_scan(n);
    const uint64_t past = __ballot(base + incl > u);
    if (past) {
      const int at = __builtin_ctzll(past);
      base += __builtin_amdgcn_readlane(incl - n, at);
      b = b0 + at;
      break;
    }
    base += last_lane(incl);
  }

  while (u < u_end && b < a.seqs) {
    const Lengths len = lengths_of(a, b < 64 ? __builtin_amdgcn_readlane(length0, b) : __builtin_amdgcn_readfirstlane(a.lengths[b]));
    const int seq = b, np = __builtin_amdgcn_readfirstlane(counted(len.n));
    const int pair = __builtin_amdgcn_readfirstlane((u - base) / np), pair_base = base + pair * np, t_at = u - pair_base;
    int t0 = t_at, t1 = min(np, t_at + u_end - u);
    int w_first = __builtin_amdgcn_readfirstlane(pair_base / per), w_last = __builtin_amdgcn_readfirstlane((pair_base + np - 1) / per);
    if (padded) {                                                      // even parts
      const int k = worker - w_first, of = w_last - w_first + 1, each = __builtin_amdgcn_readfirstlane(len.n / of), more = len.n - each * of;
      t0 = k * each + min(k, more);
      t1 = t0 + each + (k < more);
    }
    u = padded ? u_end : pair_base + np;
    if (pair + 1 == pairs) {
      base += np * pairs;
      ++b;
    }

    const int head = __builtin_amdgcn_readfirstlane(pair / chunks), h0 = (pair - head * chunks) * width;
    const int count = min(per_head - h0, width);
    const int32_t* table = a.table + seq * a.table_ld;
    // this wave's blocks: all in solo, else every NW-th
    const int stride = solo ? 1 : NW, block0 = len.first + t0 + (solo ? 0 : wave);
    const int n_mine = solo ? t1 - t0 : (t1 - t0 - wave + NW - 1) / NW;
    // pages of this wave's blocks, a lane each, 64 blocks in a register: of even and odd runs of 64
    int pages[2];
    auto fetch_pages = [&](int run) {
      const int token = (block0 + (run * 64 + lane) * stride) * kKvBlock;
      int p = -1;
      if (run * 64 + lane < n_mine && token < len.end) p = table[token >> cache.page_log2];
      return p < cache.pages ? p : -1;
    };
    auto page_of = [&](int i) {
      const int even = __builtin_amdgcn_readlane(pages[0], i & 63), odd = __builtin_amdgcn_readlane(pages[1], i & 63);
      return i & 64 ? odd : even;
    };
    auto address = [&](int i) {
      const int page = max(page_of(i), 0), in_page = (block0 + i * stride) & ((1 << (cache.page_log2 - 5)) - 1);
      return cache.data + ((((int64_t)page * cache.heads + head) << (cache.page_log2 - 5)) + in_page) * L::bytes;
    };
    Query<L> query;
    query.fetch(a, a.q + seq * a.q_ld + (int64_t)(head * per_head + h0) * a.q_head, count, lane);
    Result<L> res;
    res.clear();
    if (n_mine > 0) {
      Keys<L> keys;
      Values<L> values;
      pages[0] = fetch_pages(0);
      pages[1] = fetch_pages(1);
      const uint8_t* block = address(0);
      keys.load(block, lane);
      values.load(block, lane);
      query.convert(a, key_unit);
      for (int i = 0; i < n_mine; ++i) {
        if (i && (i & 63) == 0) pages[((i >> 6) + 1) & 1] = fetch_pages((i >> 6) + 1);
        // the next block's keys replace this one's as soon as the scores are there, its values the same; past the end the last
        // block once more, so that the loads in flight are always as many
        block = address(min(i + 1, n_mine - 1));
        float4_t s[2];
        block_scores<L>(keys, query, s);
        keys.load(block, lane);
        __builtin_amdgcn_sched_barrier(0);                             // loads stay where they are: early
        const int token = (block0 + i * stride) * kKvBlock;
        const int lo = page_of(i) >= 0 ? max(0, len.first_token - token) : kKvBlock, hi = min(kKvBlock, len.end - token);
        block_outputs<L>(values, s, query, res, lane, lo, hi);
        values.load(block, lane);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (L::FMT == kInt4)                                     // the odd codes came 16 times as large
#pragma unroll
      for (int j = 1; j < NJ; j += 2) res.acc[j] *= 0.0625f;
    res.l = column_sum(res.l);

    const int lane_now = renewed(lane), kq = lane_now >> 4, col = lane_now & 15;
    float m, l;
    float4_t acc[JW];                                                  // JW instructions' outputs at a time
    auto add = [&](float om, float ol, auto&& other) {
      const float top = fmaxf(m, om), f = __builtin_amdgcn_exp2f(m - top), g = __builtin_amdgcn_exp2f(om - top);
      m = top;
      l = l * f + ol * g;
#pragma unroll
      for (int j = 0; j < JW; ++j) acc[j] = acc[j] * f + other(j) * g;
    };
    auto clear = [&] {
      m = kNoReference;
      l = 0.0f;
#pragma unroll
      for (int j = 0; j < JW; ++j) acc[j] = (float4_t){0.0f, 0.0f, 0.0f, 0.0f};
    };
    auto put_wave = [&] {
      if (col >= count) return;
#pragma unroll
      for (int j = 0; j < NJ; ++j) shared_acc[wave][j][lane_now] = res.acc[j];
      if (kq == 0) shared_ml[wave][col] = make_float2(res.m, res.l);
    };
    auto add_wave = [&](int w, int j0) {                               // columns past the queries: whatever lies there, not used
      const float2 ml = shared_ml[w][col];
      add(ml.x, ml.y, [&](int j) { return shared_acc[w][j0 + j][lane_now]; });
    };
    auto emit = [&](int j0) {
      if (col >= count) return;
      const int64_t q_head = head * per_head + h0 + col;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;                   // NaN stays
      uint16_t* o = a.out + seq * a.out_ld + q_head * a.out_head;
      constexpr int RUN = L::PER < JW ? L::PER : JW;                   // adjacent channels of a lane
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int g = 0; g < JW; g += RUN) {
          uint16_t v[RUN];
#pragma unroll
          for (int j = 0; j < RUN; ++j) v[j] = (uint16_t)cvt_pk_bf16(acc[g + j][r] * inv * value_unit, 0.0f);
          __builtin_memcpy(__builtin_assume_aligned(o + L::v_channel(kq * 4 + r, j0 + g), RUN * 2), v, RUN * 2);
        }
      if (a.lse && kq == 0 && j0 == 0)
        a.lse[(int64_t)seq * a.q_heads + q_head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    };

    if (solo) {                                                        // nothing to join; through LDS for one way of storing
      put_wave();
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
      for (int j0 = 0; j0 < NJ; j0 += JW) {
        clear();
        add_wave(wave, j0);
        emit(j0);
      }
      continue;                                                        // one pair a wave: the loop ends
    }

    // Join the waves: every wave takes JW instructions' outputs of all of them, and keeps them to the end.
    const int held = min(t1 - t0, NW), j0 = wave * JW;                 // waves that hold anything
    __syncthreads();                                                   // reads of the last join are over
    if (wave < held) put_wave();
    __syncthreads();
    clear();
    for (int w = 0; w < held; ++w) add_wave(w, j0);

    // A part of a pair: groups of `fan` parts, then of their sums, are joined by the one of their workers that is last to come.
    int entry = worker - w_first, entries = w_last - w_first + 1, step = 1, level = 0;
    bool done = true;
    // Parts that a workgroup joins at a time: a level costs 2 to 3 us, but so do more loads than a wave has in flight (8 pairs of
    // 1500 tokens, 4 queries each: 9.3 us, with 8 at a time 11.2; 4 pairs of 30 000, 16 queries: 16.8 us, with 16 at a time 18.1).
    const int fan = count > 4 ? 8 : 16;
    while (entries > 1) {
      constexpr uint32_t kPart = part_bytes_of<L>();
      const int first = entry / fan * fan, n = min(fan, entries - first);     // of the group
      auto slot = [&](int e) { return (uint32_t)part_slot(w_first + e * step, w_first) * kPart; };
      if (n > 1) {
        // A sum goes to its first part's slot.  Every wave has read that part's (M, l) at the level below before wave 0 stores the sum's;
        // outputs are read and stored by the same wave.
        if (level > 0) {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          __syncthreads();
        }
        if (col < count) {
          const uint32_t at = slot(entry);
#pragma unroll
          for (int j = 0; j < JW; ++j) put_part(parts, (kq * count + col) * 16, at + (j0 + j) * count * 64, acc[j]);
          if (wave == 0 && kq == 0) put_part(parts, col * 16, at + NJ * 1024, (float4_t){m, l, 0.0f, 0.0f});
        }
        // Every wave's stores have reached memory before the counter says so.  Counters of different groups and levels differ: a group
        // of two and more at a level reaches past the worker `level` behind its first.
        int* counter = counters + w_first + first * step + level;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
          last_one = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
          if (last_one) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next call
        }
        __syncthreads();
        done = __builtin_amdgcn_readfirstlane(last_one);
        if (!done) break;
        // Where a part has fewer than sixteen heads, the lanes that would hold the others take further parts.  The order is the
        // workers': the same bits whoever comes last.
        constexpr int B = JW <= 2 ? 4 : 2;
        clear();
        const int run_log2 = count > 8 ? 4 : count > 4 ? 3 : count > 2 ? 2 : count > 1 ? 1 : 0, runs = 16 >> run_log2;
        const int mine = col & ((1 << run_log2) - 1), run = col >> run_log2;
        struct Loaded {
          float4_t ml[B], acc[B][JW];
        };
        auto fetch = [&](Loaded& x, int e0) {
#pragma unroll
          for (int b = 0; b < B; ++b) {
            const int e = e0 + b * runs + run;
            const bool ok = e < n && mine < count;                     // others read past the buffer: zeros
            const uint32_t at = ok ? slot(first + e) : 0x80000000u;
            x.ml[b] = get_part(parts, at + mine * 16, NJ * 1024);
#pragma unroll
            for (int j = 0; j < JW; ++j) x.acc[b][j] = get_part(parts, at + (kq * count + mine) * 16, (j0 + j) * count * 64);
            if (!ok) x.ml[b][0] = kNoReference;
          }
          __builtin_amdgcn_sched_barrier(0);                           // the loads stay in front of what follows
        };
        auto add_all = [&](const Loaded& x) {
#pragma unroll
          for (int b = 0; b < B; ++b) add(x.ml[b][0], x.ml[b][1], [&](int j) { return x.acc[b][j]; });
        };
#pragma unroll 1
        for (int e = 0; e < n; e += B * runs) {                        // uniform
          Loaded x;
          fetch(x, e);
          add_all(x);
        }
#pragma unroll 1
        for (int off = 1 << run_log2; off < 16; off <<= 1)
          add(__shfl_xor(m, off), __shfl_xor(l, off), [&](int j) {
            const float4_t v = acc[j];
            return (float4_t){__shfl_xor(v[0], off), __shfl_xor(v[1], off), __shfl_xor(v[2], off), __shfl_xor(v[3], off)};
          });
      }
      entry /= fan;
      entries = (entries + fan - 1) / fan;
      step *= fan;
      ++level;
    }
    if (done) emit(j0);
  }
}

// Queries of a key head that share a pass: sixteen columns of the products; more take as many passes, of about as many queries each.
// (Two tiles of columns a pass read the cache once for up to 32, but leave a wave too few registers: 20 queries a key head, 16
// sequences up to 8000 tokens, INT4 in heads of 128: 24.6 us against 20.8, of 256: 46 against 29.)
int chunks_of(const pq_kv_cache& c, int q_heads) { return (q_heads / c.kv_heads + 15) / 16; }
int64_t longest_of(int64_t max_len, int64_t window) {                  // blocks of the longest sequence
  int64_t n = (max_len + kKvBlock - 1) / kKvBlock;
  if (window && n > window / kKvBlock + 2) n = window / kKvBlock + 2;
  return n < 1 ? 1 : n;
}
int64_t grid_of(const pq_kv_cache& c, int64_t seqs, int q_heads, int64_t max_len, int64_t window) {
  const int64_t pairs = seqs * c.kv_heads * chunks_of(c, q_heads);
  const int64_t parts = pairs * ((longest_of(max_len, window) + kLeastBlocks - 1) / kLeastBlocks);
  const int64_t most = pairs > kMaxSplits ? pairs : kMaxSplits;
  return parts < most ? parts : most;
}

}  // namespace

size_t attn_decode_workspace_bytes(const pq_kv_cache& c, int64_t seqs, int q_heads, int64_t max_len, int64_t window) {
  int64_t workers = grid_of(c, seqs, q_heads, max_len, window);
  if (workers > kMaxSplits) workers = kMaxSplits;
  return PQ_ATTN_DECODE_ZERO_BYTES + (size_t)workers * 2 * (size_t)(c.head_dim / 16 * 1024 + 256);
}

int run_attn_decode(const pq_kv_cache& c, const AttnCall& a, hipStream_t st) {
  const int grid = (int)grid_of(c, a.seqs, a.q_heads, a.max_len, a.window), chunks = chunks_of(c, a.q_heads);
  const uint32_t part_bytes = (uint32_t)(attn_decode_workspace_bytes(c, a.seqs, a.q_heads, a.max_len, a.window) - PQ_ATTN_DECODE_ZERO_BYTES);
  return kv_dispatch(c.fmt, c.group, c.head_dim, [&](auto l) {
    attn_decode_kernel<decltype(l)><<<grid, 64 * kAttnWaves, 0, st>>>(kv_view(c), a, chunks, part_bytes);
    return check_hip(hipGetLastError(), "pq_attn_decode");
  });
}

}  // namespace pq
