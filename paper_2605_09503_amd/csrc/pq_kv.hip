// Keys and values quantized into a cache's pages as they are produced, and read back (layout: pq_kv.h; the arithmetic is the
// pinned quantizer's of pq_quantize.hip, so a cache holds what pq_quantize_act would).  Bound by HBM: 2 bytes an element on
// one side, 0.5 and the scales on the other.  Measured (MI355X; a copy of 4 GiB runs at 4.9 TB/s):
//   65 000 tokens, 8 heads of 128, NVFP4, 341 MB each way: written in 70 us (4.9 TB/s), read back in 53 (6.4)
//   14 400 tokens, 8 heads of 128, INT4/32, 75 MB:         written in 19 us (4.0 TB/s), read back in 17 (4.4)
//   65 000 tokens, 8 heads of 128, bf16, 532 MB:           written in 109 us (4.9 TB/s), read back in 101 (5.3)
//   30 000 tokens, 4 heads of 256, bf16, 246 MB:           written in 63 us (3.9 TB/s), read back in 56 (4.4)
// One token of 16 sequences takes 3.3 us, 650 tokens read back 4.2: a launch and three loads in a row (slot, row, scale).
#include "pq_kv.h"
#include "pq_qgemm_common.h"

namespace pq {

namespace {

struct KvRows {                          // rows of [token][head][D] bf16; strides in elements
  uint16_t* p;
  int64_t ld, head;
};

// A workgroup takes 32 tokens of one head, keys and values; workgroups next to each other take the heads of the same tokens, whose
// rows lie next to each other.  Neighbouring lanes hold neighbouring channels of a token, so a wave reads (or writes) whole rows, and
// the codes of neighbouring tokens meet in the L2 (65 000 tokens: HBM reads 271 MB for 266 and 79 for 75, the slots by eight chiplets
// included, and writes what there is); all of a thread's loads are in flight together.  With a head after the other and a load at a
// time the 65 000 tokens took 195 us for both ways.
constexpr int kKvThreads = 256;
template <class L>
constexpr int key_items() { return kKvBlock * L::D / 8 / kKvThreads; }   // of a thread: a row's 8 channels each
constexpr int kValueItems = kKvBlock * 16 / kKvThreads;                   // a row's lane each

// The 32 tokens of a workgroup often lie in two blocks, and the next workgroup of the head has the rest of the second: both
// belong on one chiplet, whose L2 then reads (fills) the block once.  Workgroups go round the eight chiplets, so with a multiple of
// eight heads they do by themselves (and runs of tiles a chiplet are 1 to 3 % slower: 127.0 -> 128.8 us for 65 000 tokens both ways);
// else chiplets take runs: 4 heads of 64, INT4/32, 71 000 tokens read back 21.1 -> 20.1 us, 2 of 64 written and read 20.4 -> 19.1, 20
// 37.1 -> 36.3 (5 heads of 256 46.5 -> 47.2).  The grid's size follows from arguments that are there: read from gridDim, a pass of two
// small calls took 9.8 us in place of 8.0.
__device__ __forceinline__ uint32_t tile_of_workgroup(int heads, int64_t n) {
  return heads & 7 ? (uint32_t)block_by_chiplet(blockIdx.x, (int)((n + kKvBlock - 1) / kKvBlock) * heads) : blockIdx.x;
}

// eight channels of keys, a lane each
template <class L>
__device__ __forceinline__ void write_key(uint8_t* block, int t, int c, bool ok, const uint4& x, float T, float encT) {
  if constexpr (L::FMT == kBf16) {
    if (ok) *reinterpret_cast<uint4*>(block + L::k_chunk(t, c)) = x;
  } else {
    const float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y), bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w)};
    float a = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) a = fmaxf(a, fabsf(f[j]));
    constexpr int LPG = L::G / 8;                              // lanes of a group
    a = group_max<LPG>(a);
    uint32_t codes = 0;
    if constexpr (L::FMT == kNvfp4) {
      const Nv4Scale sc = nv4_scale(a, T, encT);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0] * sc.inv, f[1] * sc.inv, 1.0f, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2] * sc.inv, f[3] * sc.inv, 1.0f, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4] * sc.inv, f[5] * sc.inv, 1.0f, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6] * sc.inv, f[7] * sc.inv, 1.0f, 3);
      if (ok && c % LPG == 0) block[L::k_byte_at(t, c / LPG)] = (uint8_t)sc.byte;
    } else {
      const float inv = int_scale<kInt4>(a).inv;
      codes = int_encode8({x.x, x.y, x.z, x.w}, {inv, inv, inv, inv});
      if (ok && c % LPG == 0) *reinterpret_cast<uint16_t*>(block + L::int_scale_at(t, c / LPG)) = (uint16_t)(as_u32(a) >> 16);
    }
    if (ok) *reinterpret_cast<uint32_t*>(block + L::k_chunk(t, c)) = codes;
  }
}

// A lane's runs are PER channels, 4 bytes with groups of 32.  Rows are read and written in pieces of up to 16 bytes instead: TS
// neighbouring lanes hold, before (after) an exchange, one run's channels of all of them each.  4-byte stores against this: reading
// back 12 sequences up to 9001 tokens, INT4 groups of 32 in heads of 64, 24.6 against 23.2 us.
template <class L>
struct Pieces {
  static constexpr int RUNS = L::NJ / L::PER, TS = L::PER >= 8 ? 1 : 8 / L::PER < RUNS ? 8 / L::PER : RUNS;
  static constexpr int N = RUNS / TS, WORDS = L::PER * TS / 2, UNIT = L::PER / 2;
  // channel of piece p of a lane
  static __device__ __forceinline__ int channel(int p, int lane) { return (p * TS + (lane & (TS - 1))) * L::GV + (lane & ~(TS - 1)) * L::PER; }
  static __device__ __forceinline__ void exchange(uint32_t (&x)[L::NJ / 2], int lane) {
    if constexpr (TS > 1) swap<1, 0xB1>(x, lane);              // quad_perm [1,0,3,2]
    if constexpr (TS > 2) swap<2, 0x4E>(x, lane);              // quad_perm [2,3,0,1]
  }

  // INT4: the largest magnitude of the group of piece p (before the exchange), in every lane that holds some of it
  static __device__ __forceinline__ float group_maximum(const uint32_t (&x)[L::NJ / 2], int p) {
    float a = 0.0f;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) a = fmaxf(a, fmaxf(fabsf(bf16_lo(x[p * WORDS + w])), fabsf(bf16_hi(x[p * WORDS + w]))));
    uint32_t u = as_u32(a);                                    // magnitudes order like their bits
    u = max(u, dpp_u32<0x128>(u));                             // row_ror 8, 4, 2, 1: lanes TS apart
    u = max(u, dpp_u32<0x124>(u));
    if constexpr (TS <= 2) u = max(u, dpp_u32<0x122>(u));
    if constexpr (TS == 1) u = max(u, dpp_u32<0x121>(u));
    return as_f32(u);
  }
  // a piece's value in lane k of every TS
  template <int K>
  static __device__ __forceinline__ float of_lane(float v) {
    if constexpr (TS == 4) return dpp_f32<K * 0x55>(v);        // quad_perm [k,k,k,k]
    else if constexpr (TS == 2) return dpp_f32<K ? 0xF5 : 0xA0>(v);   // [0,0,2,2], [1,1,3,3]
    else return v;
  }

 private:
  template <int S, int CTRL>
  static __device__ __forceinline__ void swap(uint32_t (&x)[L::NJ / 2], int lane) {
    const bool upper = lane & S;
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
      if (r & S) continue;
#pragma unroll
      for (int d = 0; d < UNIT; ++d) {
        uint32_t &a = x[r * UNIT + d], &b = x[(r + S) * UNIT + d];
        const uint32_t got = dpp_u32<CTRL>(upper ? a : b);
        if (upper) a = got;
        else b = got;
      }
    }
  }
};

// a lane's pieces of a value
template <class L>
__device__ __forceinline__ void write_value(uint8_t* block, int t, int lane, bool ok, uint32_t (&x)[L::NJ / 2], float T, float encT) {
  typedef Pieces<L> P;
  constexpr int PER = L::PER, RUNS = P::RUNS, PAIRS = PER / 2;
  if constexpr (L::FMT == kBf16) {
    if (ok)
#pragma unroll
      for (int w = 0; w < L::NJ / 2; ++w) *reinterpret_cast<uint32_t*>(block + L::v_pair(t, lane, w)) = x[w];
  } else {
    float invs[RUNS];
    if constexpr (L::FMT == kNvfp4) {
      float a = 0.0f;
#pragma unroll
      for (int j = 0; j < PAIRS; ++j) a = fmaxf(a, fmaxf(fabsf(bf16_lo(x[j])), fabsf(bf16_hi(x[j]))));
      constexpr int LPG = L::G / PER;                          // lanes of a group
      const Nv4Scale sc = nv4_scale(group_max<LPG>(a), T, encT);
      invs[0] = sc.inv;
      if (ok && lane % LPG == 0) block[L::v_byte_at(t, lane / LPG)] = (uint8_t)sc.byte;
    } else {
#pragma unroll
      for (int p = 0; p < P::N; ++p) {
        const float a = P::group_maximum(x, p), inv = int_scale<kInt4>(a).inv;
        if (ok && lane < P::TS)
          *reinterpret_cast<uint16_t*>(block + L::v_at + L::int_scale_at(t, p * P::TS + lane)) = (uint16_t)(as_u32(a) >> 16);
        invs[p * P::TS] = P::template of_lane<0>(inv);
        if constexpr (P::TS > 1) invs[p * P::TS + 1] = P::template of_lane<1>(inv);
        if constexpr (P::TS > 2) {
          invs[p * P::TS + 2] = P::template of_lane<2>(inv);
          invs[p * P::TS + 3] = P::template of_lane<3>(inv);
        }
      }
      P::exchange(x, lane);
    }
    uint32_t codes[(L::NJ + 7) / 8] = {};
#pragma unroll
    for (int w = 0; w < L::NJ / 2; w += 4) {                   // eight channels (of heads of 64: four)
      uint32_t four[4] = {};
      float inv[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        four[j] = w + j < L::NJ / 2 ? x[w + j] : 0u;
        inv[j] = invs[w + j < L::NJ / 2 ? (w + j) / PAIRS : 0];
      }
      if constexpr (L::FMT == kNvfp4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[w / 4] |= nv4_code_pair(bf16_lo(four[j]), bf16_hi(four[j]), inv[j]) << (8 * j);
      } else {
        codes[w / 4] = int_encode8(four, inv);
      }
    }
    if (ok)
#pragma unroll
      for (int jq = 0; jq < L::NQ; ++jq)
        *reinterpret_cast<uint16_t*>(block + L::v_quad(t, lane, jq)) = (uint16_t)(codes[jq / 2] >> (jq % 2 * 16));
  }
}

typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
template <int N>
struct Words;
template <>
struct Words<2> { typedef words2 type; };
template <>
struct Words<4> { typedef words4 type; };
template <>
struct Words<8> { typedef words4 type; };

// Pieces of a row, past the caches: these are read (written) once, the codes' lines come from several stores.  65 000 tokens NVFP4
// written and read back 167 us without, 144 with.
template <class L>
__device__ __forceinline__ void load_pieces(uint32_t (&x)[L::NJ / 2], const uint16_t* row, int lane) {
  typedef Pieces<L> P;
  typedef typename Words<P::WORDS>::type W;
#pragma unroll
  for (int p = 0; p < P::N; ++p)
#pragma unroll
    for (int d = 0; d < P::WORDS; d += sizeof(W) / 4) {
      const W w = __builtin_nontemporal_load(reinterpret_cast<const W*>(row + P::channel(p, lane) + 2 * d));
      __builtin_memcpy(&x[p * P::WORDS + d], &w, sizeof(W));
    }
}
template <class L>
__device__ __forceinline__ void store_pieces(const uint32_t (&x)[L::NJ / 2], uint16_t* row, int lane) {
  typedef Pieces<L> P;
  typedef typename Words<P::WORDS>::type W;
#pragma unroll
  for (int p = 0; p < P::N; ++p)
#pragma unroll
    for (int d = 0; d < P::WORDS; d += sizeof(W) / 4) {
      W w;
      __builtin_memcpy(&w, &x[p * P::WORDS + d], sizeof(W));
      __builtin_nontemporal_store(w, reinterpret_cast<W*>(row + P::channel(p, lane) + 2 * d));
    }
}

template <class L>
__global__ __launch_bounds__(kKvThreads) void kv_write_kernel(KvView cache, KvRows k, KvRows v, const int64_t* __restrict__ slots,
                                                              int64_t n) {
  constexpr int LPR = L::D / 8, KI = key_items<L>(), VI = kValueItems;
  const uint32_t tile = tile_of_workgroup(cache.heads, n);
  const int head = tile % cache.heads;
  const int64_t t0 = (int64_t)(tile / cache.heads) * kKvBlock, n_slots = cache.slots();
  int64_t k_slot[KI], v_slot[VI];
  uint4 kx[KI];
  uint32_t vx[VI][L::NJ / 2];
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int u = threadIdx.x + i * kKvThreads;
    const int64_t row = t0 + u / LPR;
    k_slot[i] = row < n ? slots[row] : -1;
    kx[i] = make_uint4(0u, 0u, 0u, 0u);
    if (row < n) {
      const words4 w = __builtin_nontemporal_load(reinterpret_cast<const words4*>(k.p + row * k.ld + head * k.head + u % LPR * 8));
      kx[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const int u = threadIdx.x + i * kKvThreads;
    const int64_t row = t0 + u / 16;
    v_slot[i] = row < n ? slots[row] : -1;
#pragma unroll
    for (int j = 0; j < L::NJ / 2; ++j) vx[i][j] = 0u;
    if (row < n) load_pieces<L>(vx[i], v.p + row * v.ld + head * v.head, u % 16);
  }
  float kT = 0.0f, vT = 0.0f, kE = 0.0f, vE = 0.0f;
  if constexpr (L::FMT == kNvfp4) {
    kT = *cache.k_ts;
    vT = *cache.v_ts;
    kE = nv4_enc_scale(kT);
    vE = nv4_enc_scale(vT);
  }
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const bool ok = k_slot[i] >= 0 && k_slot[i] < n_slots;     // other slots keep nothing
    write_key<L>(kv_block<L>(cache, ok ? k_slot[i] : 0, head), (int)k_slot[i] & (kKvBlock - 1),
                 (threadIdx.x + i * kKvThreads) % LPR, ok, kx[i], kT, kE);
  }
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const bool ok = v_slot[i] >= 0 && v_slot[i] < n_slots;
    write_value<L>(kv_block<L>(cache, ok ? v_slot[i] : 0, head), (int)v_slot[i] & (kKvBlock - 1),
                   (threadIdx.x + i * kKvThreads) % 16, ok, vx[i], vT, vE);
  }
}

// values: INT4 z * s, NVFP4 value * s_b * T, every step one binary32 operation
template <class L>
__global__ __launch_bounds__(kKvThreads) void kv_read_kernel(KvView cache, const int64_t* __restrict__ slots, int64_t n, KvRows k,
                                                             KvRows v) {
  constexpr int LPR = L::D / 8, KI = key_items<L>(), VI = kValueItems, PER = L::PER, RUNS = L::NJ / PER, PAIRS = PER / 2;
  const uint32_t tile = tile_of_workgroup(cache.heads, n);
  const int head = tile % cache.heads;
  const int64_t t0 = (int64_t)(tile / cache.heads) * kKvBlock, n_slots = cache.slots();
  int64_t k_slot[KI], v_slot[VI];
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int64_t row = t0 + (threadIdx.x + i * kKvThreads) / LPR;
    k_slot[i] = row < n ? slots[row] : -1;
  }
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const int64_t row = t0 + (threadIdx.x + i * kKvThreads) / 16;
    v_slot[i] = row < n ? slots[row] : -1;
  }
  // all loads, then all stores; a slot outside the cache reads as zeros
  uint4 kc[KI];                                                // 4-bit codes in x
  uint32_t ks[KI], vc[VI][L::FMT == kBf16 ? L::NJ / 2 : L::NQ], vs[VI][RUNS];
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    kc[i] = make_uint4(0u, 0u, 0u, 0u);
    ks[i] = 0u;
    if (k_slot[i] < 0 || k_slot[i] >= n_slots) continue;
    const uint8_t* block = kv_block<L>(cache, k_slot[i], head);
    const int t = (int)k_slot[i] & (kKvBlock - 1), c = (threadIdx.x + i * kKvThreads) % LPR;
    if constexpr (L::FMT == kBf16) kc[i] = *reinterpret_cast<const uint4*>(block + L::k_chunk(t, c));
    else kc[i].x = *reinterpret_cast<const uint32_t*>(block + L::k_chunk(t, c));
    if constexpr (L::FMT == kNvfp4) ks[i] = block[L::k_byte_at(t, c / 2)];
    if constexpr (L::FMT == kInt4) ks[i] = *reinterpret_cast<const uint16_t*>(block + L::int_scale_at(t, c / (L::G / 8)));
  }
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const bool ok = v_slot[i] >= 0 && v_slot[i] < n_slots;
    const uint8_t* block = kv_block<L>(cache, ok ? v_slot[i] : 0, head);
    const int t = (int)v_slot[i] & (kKvBlock - 1), lane = (threadIdx.x + i * kKvThreads) % 16;
    if constexpr (L::FMT == kBf16) {
#pragma unroll
      for (int w = 0; w < L::NJ / 2; ++w) vc[i][w] = ok ? *reinterpret_cast<const uint32_t*>(block + L::v_pair(t, lane, w)) : 0u;
    } else {
#pragma unroll
      for (int jq = 0; jq < L::NQ; ++jq) vc[i][jq] = ok ? *reinterpret_cast<const uint16_t*>(block + L::v_quad(t, lane, jq)) : 0u;
#pragma unroll
      for (int g = 0; g < RUNS; ++g) {
        if constexpr (L::FMT == kNvfp4) vs[i][g] = ok ? block[L::v_byte_at(t, lane / (L::G / PER))] : 0u;
        else vs[i][g] = ok ? *reinterpret_cast<const uint16_t*>(block + L::v_at + L::int_scale_at(t, g)) : 0u;
      }
    }
  }
  float kT = 0.0f, vT = 0.0f;
  if constexpr (L::FMT == kNvfp4) {
    kT = *cache.k_ts;
    vT = *cache.v_ts;
  }
  auto scale_of = [](uint32_t bits) {
    return L::FMT == kNvfp4 ? e4m3_decode(bits) : div_const(as_f32(bits << 16), 7.0f, 1.0f / 7.0f);
  };
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int u = threadIdx.x + i * kKvThreads;
    const int64_t row = t0 + u / LPR;
    uint4 y = kc[i];
    if constexpr (L::FMT != kBf16) {
      float f[8];
      const float s = scale_of(ks[i]);
      if constexpr (L::FMT == kNvfp4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(kc[i].x >> (8 * j), 1.0f, 0);
          f[2 * j] = two[0] * s * kT;
          f[2 * j + 1] = two[1] * s * kT;
        }
      } else {
        const IntCodes codes(kc[i].x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          codes.values(j, f[j], f[j + 4]);
          f[j] *= s;
          f[j + 4] *= s;
        }
      }
      y = make_uint4(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]), cvt_pk_bf16(f[6], f[7]));
    }
    if (row < n)
      __builtin_nontemporal_store((words4){y.x, y.y, y.z, y.w}, reinterpret_cast<words4*>(k.p + row * k.ld + head * k.head + u % LPR * 8));
  }
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const int u = threadIdx.x + i * kKvThreads;
    const int64_t row = t0 + u / 16;
    uint32_t y[L::NJ / 2];
    if constexpr (L::FMT == kBf16) {
#pragma unroll
      for (int w = 0; w < L::NJ / 2; ++w) y[w] = vc[i][w];
    } else {
      float s[RUNS], f[L::NJ < 8 ? 8 : L::NJ];
#pragma unroll
      for (int g = 0; g < RUNS; ++g) s[g] = scale_of(vs[i][g]);
#pragma unroll
      for (int jq = 0; jq < L::NQ; jq += 2) {                  // two quads (of heads of 64: one)
        const uint32_t quads = vc[i][jq] | (jq + 1 < L::NQ ? vc[i][jq + 1] << 16 : 0u);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          if constexpr (L::FMT == kNvfp4) {
            const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(quads >> (8 * a), 1.0f, 0);
            f[jq * 4 + 2 * a] = two[0];
            f[jq * 4 + 2 * a + 1] = two[1];
          } else {
            IntCodes(quads).values(a, f[jq * 4 + a], f[jq * 4 + a + 4]);
          }
        }
      }
#pragma unroll
      for (int w = 0; w < L::NJ / 2; ++w) {
        const float m = s[w / PAIRS];
        if constexpr (L::FMT == kNvfp4) y[w] = cvt_pk_bf16(f[2 * w] * m * vT, f[2 * w + 1] * m * vT);
        else y[w] = cvt_pk_bf16(f[2 * w] * m, f[2 * w + 1] * m);
      }
    }
    Pieces<L>::exchange(y, u % 16);
    if (row < n) store_pieces<L>(y, v.p + row * v.ld + head * v.head, u % 16);
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
    const unsigned grid = (unsigned)((n + kKvBlock - 1) / kKvBlock * c.kv_heads);
    kv_write_kernel<decltype(l)><<<grid, kKvThreads, 0, st>>>(kv_view(c), KvRows{(uint16_t*)k, k_ld, k_head},
                                                              KvRows{(uint16_t*)v, v_ld, v_head}, slots, n);
    return check_hip(hipGetLastError(), "pq_kv_write");
  });
}

int run_kv_read(const pq_kv_cache& c, const int64_t* slots, int64_t n, void* k, int64_t k_ld, int64_t k_head, void* v, int64_t v_ld,
                int64_t v_head, hipStream_t st) {
  return kv_dispatch(c.fmt, c.group, c.head_dim, [&](auto l) {
    const unsigned grid = (unsigned)((n + kKvBlock - 1) / kKvBlock * c.kv_heads);
    kv_read_kernel<decltype(l)><<<grid, kKvThreads, 0, st>>>(kv_view(c), slots, n, KvRows{(uint16_t*)k, k_ld, k_head},
                                                             KvRows{(uint16_t*)v, v_ld, v_head});
    return check_hip(hipGetLastError(), "pq_kv_read");
  });
}

}  // namespace pq
