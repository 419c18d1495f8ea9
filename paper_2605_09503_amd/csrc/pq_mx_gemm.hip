// MXFP4 products, dense and grouped by expert, on the scaled matrix instruction: v_mfma_scale_f32_32x32x64_f8f6f4 multiplies
// E2M1 codes as they are and applies both operands' power-of-two scales inside, a 32-channel block a lane.
#include "pq_host.h"
#include "pq_mx.h"

namespace pq {

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------- which tile a workgroup computes
// Rows first .. end - 1 of y, of expert `expert`, and columns from n0 on.
struct Tile {
  int64_t first, end, n0;
  int expert;
};

// inclusive sum over the lanes up to this one
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);       // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);       // row_bcast 15, 31
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// Tiles of `bm` rows are counted through the experts in turn, each expert's rows start one.  Workgroups go round the eight
// chiplets in turn; each chiplet takes a contiguous eighth of the tiles that there are (the launch has as many workgroups as there
// could be), in blocks of eight tiles of rows, so that what its workgroups read at a time meets in its L2.
// False where the workgroup has no tile.  Uniform; every wave does it for itself.
__device__ __forceinline__ bool locate(const MxCall& c, int bm, int bn, Tile& t) {
  const int lane = threadIdx.x & 63, M = (int)c.M, across = (int)((c.N + bn - 1) / bn);
  const auto tiles_of = [&](int e, int& from, int& to) {
    from = to = 0;
    if (e < c.experts) {
      from = min(max(c.offsets[e], 0), M);
      to = min(max(c.offsets[e + 1], 0), M);
    }
    return to > from ? (to - from + bm - 1) / bm : 0;
  };
  int from, to, total = (M + bm - 1) / bm;
  if (c.offsets) {
    total = 0;
    for (int e = 0; e < c.experts; e += 64) total += __builtin_amdgcn_readlane(wave_scan(tiles_of(e + lane, from, to)), 63);
  }
  const int64_t all = (int64_t)total * across;
  const int64_t per = all >> 3, extra = all & 7, chiplet = blockIdx.x & 7, at = blockIdx.x >> 3;
  if (at >= per + (chiplet < extra ? 1 : 0)) return false;
  const int64_t flat = chiplet * per + min(chiplet, extra) + at;
  const int64_t block = (int64_t)8 * across, b = flat / block, in = flat - b * block;
  const int high = min(8, total - (int)b * 8);
  int mt = (int)(b * 8 + in % high);
  t.n0 = in / high * bn;
  if (!c.offsets) {
    t.first = (int64_t)mt * bm;
    t.end = min(t.first + bm, c.M);
    t.expert = 0;
    return true;
  }
  for (int e = 0; e < c.experts; e += 64) {
    const int n = tiles_of(e + lane, from, to), upto = wave_scan(n);
    const uint64_t past = __ballot(upto > mt);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int start = __builtin_amdgcn_readlane(from, l) + (mt - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l))) * bm;
      t.first = start;
      t.end = min(start + bm, __builtin_amdgcn_readlane(to, l));
      t.expert = e + l;
      return true;
    }
    mt -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// the row of A that row m of y is made from, -1 where the index is none of A's
__device__ __forceinline__ int a_row_of(const MxCall& c, int64_t m) {
  if (!c.rows) return (int)m;
  const int r = c.rows[m];
  return (uint32_t)r < (uint32_t)c.a_rows ? r : -1;
}

// ---------------------------------------------------------------- loads into LDS
// 16 or 4 bytes a lane from memory into LDS, from byte `to` on, without a register in between.  m0, an operand, holds `to`.
__device__ __forceinline__ void load16_to_lds(uint32_t to, const uint8_t* base, uint32_t offset) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void load4_to_lds(uint32_t to, const uint8_t* base, uint32_t offset) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, %2" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
}
// all but the last N loads of this wave have arrived and its LDS reads are done
template <int N>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

// A row's piece of a panel is 128 bytes of LDS, its 16-byte blocks permuted by (row / 2) % 8: the 16 rows that a read takes at a
// time then have a block in every bank.
__device__ __forceinline__ int block_at(int row, int block) { return (block ^ ((row >> 1) & 7)) * 16; }

template <int SEL>
__device__ __forceinline__ float16v mfma(const int4v& w, const int4v& a, const float16v& acc, int w_scale, int a_scale) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(int8v{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, int8v{a[0], a[1], a[2], a[3], 0, 0, 0, 0},
                                                         acc, 4, 4, SEL, w_scale, SEL, a_scale);
}

// ---------------------------------------------------------------- outputs
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}
// outputs n .. n + 7 of row m, n a multiple of 8
__device__ __forceinline__ void store8(const MxCall& c, int64_t m, int64_t n, const float (&v)[8]) {
  if (c.out_f32) {
    float* y = (float*)c.y + m * c.ldy + n;
    for (int e = 0; e < 8; ++e)
      if (n + e < c.N) y[e] = v[e];
    return;
  }
  uint16_t* y = (uint16_t*)c.y + m * c.ldy + n;
  const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  if (n + 7 < c.N) {
    *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (n + e < c.N) y[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
  }
}

// ---------------------------------------------------------------- tiles whose waves share both operands through LDS
template <int BM, int BN, int WM, int WN>
struct Shared {
  static constexpr int waves = WM * WN, fm = BM / WM / 32, fn = BN / WN / 32;       // fragments of 32 a wave
  static constexpr int a_scales = (BM + BN) * kMxRowBytes, w_scales = a_scales + BM * kMxRowScales;
  static constexpr int stage = (BM + BN) * (kMxRowBytes + kMxRowScales), lds = 2 * stage;
  static constexpr int a_loads = BM / 8 / waves, w_loads = BN / 8 / waves;           // of 8 rows
  static constexpr int as_loads = BM / 32, ws_loads = BN / 32;                        // of 32 rows' scales, over all waves
  static constexpr int pitch = fn * 32 + 4;                                           // floats a row of outputs
  static_assert(waves * 32 * pitch * 4 <= lds, "32 rows of every wave's outputs");
  static_assert((as_loads + ws_loads) % waves == 0, "every wave issues as many loads");
};

template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 2) void mx_gemm_shared_kernel(const MxCall c) {
  using S = Shared<BM, BN, WM, WN>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  Tile t;
  if (!locate(c, BM, BN, t)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave % WM, wave_n = wave / WM;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;

  // loader: a load takes 8 rows' pieces of a panel, lane l the block that belongs at place l % 8 of row l / 8; rows past the
  // tile's last re-read it (their outputs are not stored)
  const int a_last = (int)(t.end - t.first) - 1, w_last = (int)min((int64_t)BN, c.N - t.n0) - 1;
  const uint8_t *a = c.a, *w = c.w + (size_t)t.expert * c.w_next + t.n0 * kMxRowBytes;
  const uint8_t *as = c.a + mx_scales_at(c.a_rows, c.K), *ws = c.w + (size_t)t.expert * c.w_next + mx_scales_at(c.N, c.K) + t.n0 * kMxRowScales;
  const size_t a_next = (size_t)c.a_rows, w_next = (size_t)c.N;
  const auto a_row = [&](int row) { return (uint32_t)max(a_row_of(c, t.first + min(row, a_last)), 0); };
  uint32_t a_at[S::a_loads], w_at[S::w_loads], s_at[(S::as_loads + S::ws_loads) / S::waves];
#pragma unroll
  for (int i = 0; i < S::a_loads; ++i) {
    const int row = 8 * (S::waves * i + wave) + (lane >> 3);
    a_at[i] = a_row(row) * kMxRowBytes + block_at(row, lane & 7);
  }
#pragma unroll
  for (int i = 0; i < S::w_loads; ++i) {
    const int row = 8 * (S::waves * i + wave) + (lane >> 3);
    w_at[i] = (uint32_t)min(row, w_last) * kMxRowBytes + block_at(row, lane & 7);
  }
#pragma unroll
  for (int i = 0; i < (S::as_loads + S::ws_loads) / S::waves; ++i) {
    const int j = S::waves * i + wave, row = (j < S::as_loads ? j : j - S::as_loads) * 32 + (lane >> 1);
    s_at[i] = (j < S::as_loads ? a_row(row) : (uint32_t)min(row, w_last)) * kMxRowScales + (lane & 1) * 4;
  }
  const int panels = (int)mx_panels(c.K);
  const auto load = [&](int p, int stage) {
    const uint32_t to = lds0 + stage * S::stage;
#pragma unroll
    for (int i = 0; i < S::a_loads; ++i) load16_to_lds(to + (S::waves * i + wave) * 1024, a + p * a_next * kMxRowBytes, a_at[i]);
#pragma unroll
    for (int i = 0; i < S::w_loads; ++i) load16_to_lds(to + BM * kMxRowBytes + (S::waves * i + wave) * 1024, w + p * w_next * kMxRowBytes, w_at[i]);
#pragma unroll
    for (int i = 0; i < (S::as_loads + S::ws_loads) / S::waves; ++i) {
      const int j = S::waves * i + wave;
      load4_to_lds(to + S::a_scales + j * 256, j < S::as_loads ? as + p * a_next * kMxRowScales : ws + p * w_next * kMxRowScales, s_at[i]);
    }
  };

  // lane l multiplies row l % 32 of a fragment, channels 32 (l / 32) .. of every 64
  const int row = lane & 31, half = lane >> 5;
  int block[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) block[s] = block_at(row, 2 * s + half);
  const int a_base = (wave_m * S::fm * 32 + row) * kMxRowBytes, w_base = (BM + wave_n * S::fn * 32 + row) * kMxRowBytes;
  const int as_base = S::a_scales + (wave_m * S::fm * 32 + row) * kMxRowScales, ws_base = S::w_scales + (wave_n * S::fn * 32 + row) * kMxRowScales;

  float16v acc[S::fn][S::fm];
#pragma unroll
  for (int i = 0; i < S::fn; ++i)
#pragma unroll
    for (int j = 0; j < S::fm; ++j) acc[i][j] = float16v{};

  int4v af[2][S::fm], wf[2][S::fn];
  int asc[S::fm][2], wsc[S::fn][2];            // a row's scale bytes of 128 channels a word, this lane's blocks in bytes 0 and 2
  const auto read = [&](int set, int stage, int s) {
    const unsigned char* at = lds + stage * S::stage + block[s];
#pragma unroll
    for (int i = 0; i < S::fn; ++i) wf[set][i] = *reinterpret_cast<const int4v*>(at + w_base + i * 32 * kMxRowBytes);
#pragma unroll
    for (int j = 0; j < S::fm; ++j) af[set][j] = *reinterpret_cast<const int4v*>(at + a_base + j * 32 * kMxRowBytes);
  };
  const auto read_scales = [&](int stage, int (&sa)[S::fm][2], int (&sw)[S::fn][2]) {
    const unsigned char* at = lds + stage * S::stage;
#pragma unroll
    for (int i = 0; i < S::fn; ++i) {
      const uint2 v = *reinterpret_cast<const uint2*>(at + ws_base + i * 32 * kMxRowScales);
      sw[i][0] = (int)(v.x >> (8 * half)), sw[i][1] = (int)(v.y >> (8 * half));
    }
#pragma unroll
    for (int j = 0; j < S::fm; ++j) {
      const uint2 v = *reinterpret_cast<const uint2*>(at + as_base + j * 32 * kMxRowScales);
      sa[j][0] = (int)(v.x >> (8 * half)), sa[j][1] = (int)(v.y >> (8 * half));
    }
  };
#define PQ_MULTIPLY(set, s)                                                                                             \
  _Pragma("unroll") for (int i = 0; i < S::fn; ++i) _Pragma("unroll") for (int j = 0; j < S::fm; ++j) acc[i][j] =       \
      mfma<2 * ((s) & 1)>(wf[set][i], af[set][j], acc[i][j], wsc[i][(s) >> 1], asc[j][(s) >> 1])

  // The fragments of 64 channels are read while those before them are multiplied; the barrier stands before the last of a panel:
  // behind it the next panel has arrived in the other stage, and this one's is free for the panel after that.
  load(0, 0);
  arrived<0>();
  meet();
  if (panels > 1) load(1, 1);
  read_scales(0, asc, wsc);
  read(0, 0, 0);
  for (int p = 0; p < panels; ++p) {
    const int stage = p & 1;
    read(1, stage, 1);
    PQ_MULTIPLY(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    read(0, stage, 2);
    PQ_MULTIPLY(1, 1);
    __builtin_amdgcn_sched_barrier(0);
    read(1, stage, 3);
    PQ_MULTIPLY(0, 2);
    if (p + 1 < panels) {
      arrived<0>();
      meet();
      if (p + 2 < panels) load(p + 2, stage);
      read(0, stage ^ 1, 0);
      int na[S::fm][2], nw[S::fn][2];
      read_scales(stage ^ 1, na, nw);
      PQ_MULTIPLY(1, 3);
#pragma unroll
      for (int j = 0; j < S::fm; ++j) asc[j][0] = na[j][0], asc[j][1] = na[j][1];
#pragma unroll
      for (int i = 0; i < S::fn; ++i) wsc[i][0] = nw[i][0], wsc[i][1] = nw[i][1];
    } else {
      PQ_MULTIPLY(1, 3);
    }
  }
#undef PQ_MULTIPLY

  // A lane has row l % 32 of a fragment and columns 8 q + 4 (l / 32) + 0 .. 3.  Through LDS, 32 rows at a time in a part of the wave's
  // own, a row's columns come together: whole lines are stored, eight columns a lane.
  arrived<0>();
  meet();
  float* part = reinterpret_cast<float*>(lds) + wave * 32 * S::pitch;
  constexpr int lanes = S::fn * 4, at_once = 64 / lanes;                // lanes a row, rows a store
  const int64_t n = t.n0 + wave_n * S::fn * 32 + lane % lanes * 8;
  float bias[8] = {};
  if (c.bias) {
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = bf16_to_f32(c.bias[t.expert * c.N + min(n + e, c.N - 1)]);
  }
#pragma unroll
  for (int j = 0; j < S::fm; ++j) {
#pragma unroll
    for (int i = 0; i < S::fn; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(part + row * S::pitch + 32 * i + 8 * q + 4 * half) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int r = lane / lanes; r < 32; r += at_once) {
      const float* from = part + r * S::pitch + lane % lanes * 8;
      const float4 x = *reinterpret_cast<const float4*>(from), z = *reinterpret_cast<const float4*>(from + 4);
      const int64_t m = t.first + (wave_m * S::fm + j) * 32 + r;
      if (m >= t.end || n >= c.N || a_row_of(c, m) < 0) continue;
      store8(c, m, n, {x.x + bias[0], x.y + bias[1], x.z + bias[2], x.w + bias[3], z.x + bias[4], z.y + bias[5], z.z + bias[6], z.w + bias[7]});
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// ---------------------------------------------------------------- small tiles whose waves share K
// Each of KW waves multiplies the whole tile of 32 FM x 32 over every KW-th panel, its panels in a part of LDS of its own (no
// barrier while it runs), then the waves' sums are added up in their order.
template <int FM, int KW>
struct Split {
  static constexpr int bm = 32 * FM, bn = 32;
  static constexpr int a_scales = (bm + bn) * kMxRowBytes, w_scales = a_scales + bm * kMxRowScales;
  static constexpr int stage = (bm + bn) * (kMxRowBytes + kMxRowScales), own = 2 * stage, lds = KW * own;
  static constexpr int loads = (bm + bn) / 8 + (bm + bn) / 32;
  static constexpr int pitch = 36;                                     // floats a row of sums: rows start four banks apart
  static_assert(bm * pitch * 4 <= own, "the sums take a wave's own part");
};

template <int FM, int KW>
__global__ __launch_bounds__(KW * 64) void mx_gemm_split_kernel(const MxCall c) {
  using S = Split<FM, KW>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  Tile t;
  if (!locate(c, S::bm, S::bn, t)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  unsigned char* own = lds + wave * S::own;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)own;

  const int a_last = (int)(t.end - t.first) - 1, w_last = (int)min((int64_t)S::bn, c.N - t.n0) - 1;
  const uint8_t *a = c.a, *w = c.w + (size_t)t.expert * c.w_next + t.n0 * kMxRowBytes;
  const uint8_t *as = c.a + mx_scales_at(c.a_rows, c.K), *ws = c.w + (size_t)t.expert * c.w_next + mx_scales_at(c.N, c.K) + t.n0 * kMxRowScales;
  const size_t a_next = (size_t)c.a_rows, w_next = (size_t)c.N;
  const auto a_row = [&](int row) { return (uint32_t)max(a_row_of(c, t.first + min(row, a_last)), 0); };
  uint32_t a_at[4 * FM], w_at[4], as_at[FM], ws_at;
#pragma unroll
  for (int i = 0; i < 4 * FM; ++i) {
    const int row = 8 * i + (lane >> 3);
    a_at[i] = a_row(row) * kMxRowBytes + block_at(row, lane & 7);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 8 * i + (lane >> 3);
    w_at[i] = (uint32_t)min(row, w_last) * kMxRowBytes + block_at(row, lane & 7);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) as_at[i] = a_row(32 * i + (lane >> 1)) * kMxRowScales + (lane & 1) * 4;
  ws_at = (uint32_t)min(lane >> 1, w_last) * kMxRowScales + (lane & 1) * 4;
  const int panels = (int)mx_panels(c.K);
  const auto load = [&](int p, int stage) {
    const uint32_t to = lds0 + stage * S::stage;
#pragma unroll
    for (int i = 0; i < 4; ++i) load16_to_lds(to + S::bm * kMxRowBytes + i * 1024, w + p * w_next * kMxRowBytes, w_at[i]);
    load4_to_lds(to + S::w_scales, ws + p * w_next * kMxRowScales, ws_at);
#pragma unroll
    for (int i = 0; i < 4 * FM; ++i) load16_to_lds(to + i * 1024, a + p * a_next * kMxRowBytes, a_at[i]);
#pragma unroll
    for (int i = 0; i < FM; ++i) load4_to_lds(to + S::a_scales + i * 256, as + p * a_next * kMxRowScales, as_at[i]);
  };

  const int row = lane & 31, half = lane >> 5;
  float16v acc[FM];
#pragma unroll
  for (int j = 0; j < FM; ++j) acc[j] = float16v{};
  const auto multiply = [&](int stage) {
    const unsigned char* at = own + stage * S::stage;
    int4v wf[4], af[4][FM];
    uint2 sw = *reinterpret_cast<const uint2*>(at + S::w_scales + row * kMxRowScales), sa[FM];
    const int wl = (int)(sw.x >> (8 * half)), wh = (int)(sw.y >> (8 * half));
#pragma unroll
    for (int j = 0; j < FM; ++j) sa[j] = *reinterpret_cast<const uint2*>(at + S::a_scales + (32 * j + row) * kMxRowScales);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      wf[s] = *reinterpret_cast<const int4v*>(at + (S::bm + row) * kMxRowBytes + block_at(row, 2 * s + half));
#pragma unroll
      for (int j = 0; j < FM; ++j) af[s][j] = *reinterpret_cast<const int4v*>(at + (32 * j + row) * kMxRowBytes + block_at(row, 2 * s + half));
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
      const int al = (int)(sa[j].x >> (8 * half)), ah = (int)(sa[j].y >> (8 * half));
      acc[j] = mfma<0>(wf[0], af[0][j], acc[j], wl, al);
      acc[j] = mfma<2>(wf[1], af[1][j], acc[j], wl, al);
      acc[j] = mfma<0>(wf[2], af[2][j], acc[j], wh, ah);
      acc[j] = mfma<2>(wf[3], af[3][j], acc[j], wh, ah);
    }
  };
  if (wave < panels) load(wave, 0);
  if (wave + KW < panels) load(wave + KW, 1);
  int stage = 0;
  for (int p = wave; p < panels; p += KW, stage ^= 1) {
    if (p + KW < panels)
      arrived<S::loads>();
    else
      arrived<0>();
    multiply(stage);
    if (p + 2 * KW < panels) {
      arrived<S::loads>();                               // this stage's reads are done
      load(p + 2 * KW, stage);
    }
  }
  // sums: row m = l % 32, columns 8 q + 4 (l / 32) .. of this wave's part
  arrived<0>();
  float* part = reinterpret_cast<float*>(own);
#pragma unroll
  for (int j = 0; j < FM; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<float4*>(part + (32 * j + row) * S::pitch + 8 * q + 4 * half) = make_float4(acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2], acc[j][4 * q + 3]);
  __syncthreads();
  const float* parts = reinterpret_cast<const float*>(lds);
  for (int i = tid; i < S::bm * 4; i += KW * 64) {
    const int r = i >> 2, col = (i & 3) * 8;
    const int64_t m = t.first + r, n = t.n0 + col;
    if (m >= t.end || n >= c.N || a_row_of(c, m) < 0) continue;
    float v[8] = {};
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const float* from = parts + k * (S::own / 4) + r * S::pitch + col;
      const float4 x = *reinterpret_cast<const float4*>(from), z = *reinterpret_cast<const float4*>(from + 4);
      v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w, v[4] += z.x, v[5] += z.y, v[6] += z.z, v[7] += z.w;
    }
    if (c.bias) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bf16_to_f32(c.bias[t.expert * c.N + min(n + e, c.N - 1)]);
    }
    store8(c, m, n, v);
  }
}

template <class K>
int launch(K kernel, const char* name, const MxCall& c, int bm, int bn, int waves, int lds, std::atomic<uint64_t>& allowed, hipStream_t st) {
  const int64_t tiles_m = (c.M + bm - 1) / bm + (c.offsets ? (c.experts < c.M ? c.experts : c.M) : 0), across = (c.N + bn - 1) / bn;
  // a grid has fewer than 2^32 threads; workgroups beyond the tiles that there are end at once
  if (tiles_m * across + 8 >= ((int64_t)1 << 26) / waves)
    return fail(PQ_ERR_SHAPE, "MXFP4 product: M=%lld N=%lld are too many tiles for one call", (long long)c.M, (long long)c.N);
  int rc = allow_lds((const void*)kernel, (size_t)lds, allowed, name);
  if (rc) return rc;
  kernel<<<(unsigned)((tiles_m * across + 7) / 8 * 8), waves * 64, lds, st>>>(c);
  return check_hip(hipGetLastError(), name);
}

template <int BM, int BN, int WM, int WN>
int launch_shared(const MxCall& c, hipStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  return launch(mx_gemm_shared_kernel<BM, BN, WM, WN>, "mx_gemm_shared_kernel", c, BM, BN, WM * WN, Shared<BM, BN, WM, WN>::lds, allowed, st);
}
template <int FM, int KW>
int launch_split(const MxCall& c, hipStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  return launch(mx_gemm_split_kernel<FM, KW>, "mx_gemm_split_kernel", c, 32 * FM, 32, KW, Split<FM, KW>::lds, allowed, st);
}

}  // namespace

int run_mx_gemm(const MxCall& c, hipStream_t st) {
  if (c.M == 0) return PQ_OK;
  const int64_t each = c.offsets ? (c.M + c.experts - 1) / c.experts : c.M;
  if (each <= 32) return launch_split<1, 4>(c, st);
  if (each <= 64) return launch_split<2, 4>(c, st);
  if (((each + 255) / 256) * ((c.N + 255) / 256) * (c.offsets ? c.experts : 1) < 200) return launch_shared<128, 128, 2, 2>(c, st);
  return launch_shared<256, 256, 2, 4>(c, st);
}

}  // namespace pq
