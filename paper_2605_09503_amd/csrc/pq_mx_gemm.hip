// MXFP4 products, dense and grouped by expert, on the scaled matrix instruction: v_mfma_scale_f32_32x32x64_f8f6f4 multiplies
// E2M1 codes as they are and applies both operands' power-of-two scales inside, a 32-channel block a lane.
#include "pq_host.h"
#include "pq_mx.h"

namespace pq {

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
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

// rows from .. to - 1 of expert e, and how many tiles of bm they take: each expert's rows start one
__device__ __forceinline__ int tiles_of(const MxCall& c, int bm, int e, int& from, int& to) {
  from = to = 0;
  if (e < c.experts) {
    from = min(max(c.offsets[e], 0), (int)c.M);
    to = min(max(c.offsets[e + 1], 0), (int)c.M);
  }
  return to > from ? (to - from + bm - 1) / bm : 0;
}
// The tiles a workgroup computes.  Workgroups go round the eight chiplets in turn; each chiplet takes a contiguous eighth of the
// tiles, in blocks of four tiles of rows, and its workgroups go through it side by side: what they read at a time meets in its L2
// (blocks of eight: 8192 x 12288 x 8192 takes 407 us, not 388, 16384 x 8192 x 1024 112, not 102, 65536 gathered rows by 64 experts,
// 2816 x 2048, 333, not 320; two to six are alike, sixteen and more slower still).
template <bool GROUPED>
struct Tiles {
  // A table in LDS for up to kTable experts: tiles of the experts up to each one, and their offsets cut to 0 .. M.  What a search
  // in memory waits for would hold up the loads that are on their way.
  static constexpr int kTable = GROUPED ? 1024 : 0, kTableBytes = GROUPED ? (2 * kTable + 4) * 4 : 0;
  int total, across, next, step, end;         // tiles of rows and of columns; numbers of this workgroup's tiles
  const int32_t* table;                       // or null
  __device__ __forceinline__ Tiles(const MxCall& c, int bm, int bn, int32_t* lds) {
    table = nullptr;
    if constexpr (GROUPED) {
      const int lane = threadIdx.x & 63;
      table = lds && c.experts <= kTable ? lds : nullptr;
      total = 0;
      for (int e = 0; e < c.experts; e += 64) {
        int from, to;
        const int upto = total + wave_scan(tiles_of(c, bm, e + lane, from, to));
        if (table && e + lane < c.experts) {                     // every wave writes the same, each word once
          lds[e + lane] = upto;
          lds[kTable + e + lane] = from;
          if (e + lane == c.experts - 1) lds[kTable + e + lane + 1] = to;
        }
        total = min(__builtin_amdgcn_readlane(upto, 63), 1 << 26);
      }
      // offsets that do not decrease make no more tiles than this; with others there may be more than can be counted: none is computed
      if (total > (int)((c.M + bm - 1) / bm + min((int64_t)c.experts, c.M))) total = 0;
      if (table) __syncthreads();
    } else {
      total = (int)((c.M + bm - 1) / bm);
    }
    across = (int)((c.N + bn - 1) / bn);
    const int all = total * across, per = all >> 3, extra = all & 7, chiplet = blockIdx.x & 7;
    const int start = chiplet * per + min(chiplet, extra);
    next = start + (int)(blockIdx.x >> 3);
    step = (int)((gridDim.x + 7 - chiplet) >> 3);
    end = start + per + (chiplet < extra ? 1 : 0);
  }
  // tile number `flat` (uniform)
  __device__ __forceinline__ Tile at(const MxCall& c, int bm, int bn, int flat) const {
    Tile t;
    const int block = 4 * across, b = flat / block, in = flat - b * block, high = min(4, total - b * 4);
    const int mt = b * 4 + in % high;
    t.n0 = (int64_t)(in / high) * bn;
    t.first = (int64_t)mt * bm;
    t.end = min(t.first + bm, c.M);
    t.expert = 0;
    if constexpr (!GROUPED) return t;
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int e = 0; e < c.experts; e += 64) {
      int from = 0, to = 0, upto;
      if (table)
        upto = e + lane < c.experts ? table[e + lane] : total;
      else
        upto = before + wave_scan(tiles_of(c, bm, e + lane, from, to));
      const uint64_t past = __ballot(upto > mt);
      if (past) {
        const int l = __builtin_ctzll(past);
        if (table) {
          from = table[kTable + e + l];
          to = table[kTable + e + l + 1];
          before = e + l ? table[e + l - 1] : 0;
          from = __builtin_amdgcn_readfirstlane(from);
          to = __builtin_amdgcn_readfirstlane(to);
          before = __builtin_amdgcn_readfirstlane(before);
        } else {
          if (l) before = __builtin_amdgcn_readlane(upto, l - 1);
          from = __builtin_amdgcn_readlane(from, l);
          to = __builtin_amdgcn_readlane(to, l);
        }
        t.first = from + (int64_t)(mt - before) * bm;
        t.end = min(t.first + bm, (int64_t)to);
        t.expert = e + l;
        break;
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
    return t;
  }
};

// a value that the compiler computes anew from here on: what is derived from it does not stay in registers across a loop
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// a pointer that is the same in all lanes, where the compiler does not see that it is
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return (const uint8_t*)((uint64_t)hi << 32 | lo);
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
__device__ __forceinline__ void load4_to_lds(uint32_t to, const uint8_t* from) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(to), "v"(from) : "memory");
}
// two bytes a lane, which take four in LDS
__device__ __forceinline__ void load2_to_lds(uint32_t to, const uint8_t* base, uint32_t offset) {
  asm volatile("s_nop 0\n\tglobal_load_lds_ushort %1, %2" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
}
// all but the last N loads of this wave have arrived and its LDS reads are done
template <int N>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

// A row's piece of a panel is 64 bytes of LDS, its 16-byte blocks permuted by (row / 4) % 4: the 16 rows that a read takes at a
// time then have a block in every bank.
__device__ __forceinline__ int block_at(int row, int block) { return (block ^ ((row >> 2) & 3)) * 16; }

template <int SEL>
__device__ __forceinline__ float16v mfma(const int4v& w, const int4v& a, const float16v& acc, int w_scale, int a_scale) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(int8v{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, int8v{a[0], a[1], a[2], a[3], 0, 0, 0, 0},
                                                         acc, 4, 4, SEL, w_scale, SEL, a_scale);
}

// ---------------------------------------------------------------- outputs
// outputs n .. n + 7 of row m, n a multiple of 8
__device__ __forceinline__ void store8(const MxCall& c, int64_t m, int64_t n, const uint4& v) {
  uint16_t* y = (uint16_t*)c.y + m * c.ldy + n;
  if (n + 7 < c.N) {
    *reinterpret_cast<uint4*>(y) = v;
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
  static constexpr int stages = 4, stage = (BM + BN) * (kMxRowBytes + kMxRowScales);
  static constexpr int a_loads = BM / 16 / waves, w_loads = BN / 16 / waves;         // of 16 rows
  static constexpr int as_loads = BM / 64, ws_loads = BN / 64;                        // of 64 rows' scales, over all waves
  static constexpr int s_loads = (as_loads + ws_loads) / waves, loads = a_loads + w_loads + s_loads;
  static constexpr int stores = fm * fn * 2;                                          // of a wave, a tile
  // behind the stages, for this tile and the next: bias of its columns, a word each, and (grouped) the index of its rows; the table
  static constexpr int bias = stages * stage, index = bias + 2 * BN * 4, table = index + 2 * BM * 4;
  static constexpr int lds(bool grouped) { return grouped ? table + Tiles<true>::kTableBytes : index; }
  static constexpr int few = 5;            // panels: with fewer (FEW) the loads reach past the next tile, bias and index are read as they are needed
  static_assert(fn * 32 <= 64, "a lane a column");
  static_assert((as_loads + ws_loads) % waves == 0 && as_loads % s_loads == 0, "every wave issues as many loads");
};

// A workgroup goes through its tiles, and through the panels of each, without a stop: three panels are on their way while one is
// multiplied, also where they are the next tile's.
// Bound by the matrix unit under the chip's power limit: 8192 x 12288 x 8192 takes 384 to 413 us = 4.0 to 4.3 PFLOP/s, on operands of zeros, by the
// same instructions, 281 to 305; without the loads behind the first four panels 359 to 368, without the stores 367 to 372.  A wave of a 256 x 256 tile has 4 x 2
// fragments and reads 3/4 KB of LDS a matrix instruction, one of a 128 x 128 tile 2 x 2 and 1 KB; from memory the larger tile takes half
// as much.  Four waves of 128 x 128 each, 256 x 128 tiles, and eight stages of 128 x 128 were slower.  128 x 128 tiles, two workgroups a
// unit, for outputs that make too few large ones: 1777 x 4008 x 2016 15.0 us.
template <int BM, int BN, int WM, int WN, bool GROUPED, bool FEW>
__global__ __launch_bounds__(WM* WN * 64, 2) void mx_gemm_shared_kernel(const MxCall c) {
  using S = Shared<BM, BN, WM, WN>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Tiles<GROUPED> tiles(c, BM, BN, reinterpret_cast<int32_t*>(lds + S::table));
  if (tiles.next >= tiles.end) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave / WN, wave_n = wave % WN;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  const int panels = (int)mx_panels(c.K);
  constexpr bool ahead = !FEW;
  const bool index_ahead = GROUPED && ahead && c.rows;
  const size_t as_at = mx_scales_at(c.a_rows, c.K), ws_at = mx_scales_at(c.N, c.K);

  // Loader: a load takes 16 rows' pieces of a panel, lane l the block that belongs at place l % 4 of row l / 4 (the same for all of a
  // wave's loads); rows past the tile's last re-read it (their outputs are not stored).  The scale loads of the first waves are of A's
  // rows, of those behind of W's.
  const bool s_of_a = wave * S::s_loads < S::as_loads;
  const int s_first = (wave * S::s_loads - (s_of_a ? 0 : S::as_loads)) * 64;
  // Few instructions a panel: the matrix unit takes 32 cycles an instruction, and whatever else a wave issues between two costs 4.
  int load_tile = tiles.next, load_panel = 0;
  bool more = true, drain = false;                             // the last load() was of a panel; it was a tile's last
  int load_slot = 0;
  Tile lt;
  const uint8_t *a_from, *w_from, *s_from;                     // of the next panel
  const size_t a_step = (size_t)c.a_rows * kMxRowBytes, w_step = (size_t)c.N * kMxRowBytes;
  const size_t s_step = (size_t)(s_of_a ? c.a_rows : c.N) * kMxRowScales;
  uint32_t a_off[S::a_loads], w_off[S::w_loads], s_off[S::s_loads];
  const uint32_t blk = block_at(16 * wave + (lane >> 2), lane & 3);
  const auto aim = [&] {                                       // at tile load_tile
    lt = tiles.at(c, BM, BN, load_tile);
    const int l = opaque(lane), first = 16 * wave + (l >> 2);
    const int a_last = (int)(lt.end - lt.first) - 1, w_last = (int)min((int64_t)BN, c.N - lt.n0) - 1;
    a_from = c.a + (GROUPED ? 0 : lt.first * kMxRowBytes);
    w_from = c.w + (size_t)lt.expert * c.w_next;
    s_from = s_of_a ? c.a + as_at + (GROUPED ? 0 : lt.first * kMxRowScales) : w_from + ws_at + lt.n0 * kMxRowScales;
    w_from += lt.n0 * kMxRowBytes;
    load_slot ^= 1;
    if (c.bias && ahead && wave * 64 < BN)
      load2_to_lds(lds0 + S::bias + (load_slot * BN + wave * 64) * 4, (const uint8_t*)(c.bias + lt.expert * c.N + lt.n0), (uint32_t)min(wave * 64 + l, w_last) * 2);
    if (index_ahead && wave * 64 < BM)
      load4_to_lds(lds0 + S::index + (load_slot * BM + wave * 64) * 4, (const uint8_t*)(c.rows + lt.first), (uint32_t)min(wave * 64 + l, a_last) * 4);
    // grouped: the rows as the index gives them, which load() makes offsets of before it first uses them
    const auto a_row = [&](int row) {
      row = min(row, a_last);
      if (GROUPED && FEW && c.rows) return (uint32_t)c.rows[lt.first + row];
      return GROUPED ? (uint32_t)lt.first + row : (uint32_t)row;      // with an index ahead load() puts its rows in their place
    };
#pragma unroll
    for (int i = 0; i < S::a_loads; ++i) {
      a_off[i] = a_row(first + 16 * S::waves * i);
      if constexpr (!GROUPED) a_off[i] = a_off[i] * kMxRowBytes + blk;
    }
#pragma unroll
    for (int i = 0; i < S::w_loads; ++i) w_off[i] = (uint32_t)min(first + 16 * S::waves * i, w_last) * kMxRowBytes + blk;
#pragma unroll
    for (int i = 0; i < S::s_loads; ++i) {
      const int row = s_first + 64 * i + l;
      s_off[i] = s_of_a ? a_row(row) : (uint32_t)min(row, w_last);
      if constexpr (!GROUPED) s_off[i] *= kMxRowScales;
    }
  };
  const auto load = [&](int stage) {
    more = load_tile < tiles.end;
    if (!more) return;
    drain = false;
    if (GROUPED && load_panel == 0) {
      if (index_ahead) {
        const uint32_t* rows = reinterpret_cast<const uint32_t*>(lds + S::index) + load_slot * BM;
        const int l = opaque(lane);
#pragma unroll
        for (int i = 0; i < S::a_loads; ++i) a_off[i] = rows[16 * (S::waves * i + wave) + (l >> 2)];
        if (s_of_a) {
#pragma unroll
          for (int i = 0; i < S::s_loads; ++i) s_off[i] = rows[s_first + 64 * i + l];
        }
      }
      const auto known = [&](uint32_t r) { return r < (uint32_t)c.a_rows ? r : 0u; };
#pragma unroll
      for (int i = 0; i < S::a_loads; ++i) a_off[i] = known(a_off[i]) * kMxRowBytes + blk;
#pragma unroll
      for (int i = 0; i < S::s_loads; ++i) s_off[i] = (s_of_a ? known(s_off[i]) : s_off[i]) * kMxRowScales;
    }
    const uint32_t to = lds0 + stage * S::stage + wave * 1024;
#pragma unroll
    for (int i = 0; i < S::a_loads; ++i) load16_to_lds(to + S::waves * i * 1024, a_from, a_off[i]);
#pragma unroll
    for (int i = 0; i < S::w_loads; ++i) load16_to_lds(to + BM * kMxRowBytes + S::waves * i * 1024, w_from, w_off[i]);
#pragma unroll
    for (int i = 0; i < S::s_loads; ++i) load4_to_lds(lds0 + stage * S::stage + S::a_scales + (wave * S::s_loads + i) * 256, s_from, s_off[i]);
    a_from += a_step;
    w_from += w_step;
    s_from += s_step;
    if (++load_panel == panels) {
      load_panel = 0;
      load_tile += tiles.step;
      if (load_tile < tiles.end) {
        aim();
        drain = index_ahead;
      }
    }
  };

  // lane l multiplies row l % 32 of a fragment, channels 32 (l / 32) .. of every 64
  const int row = lane & 31, half = lane >> 5;
  // block 2 s + half of the row: its place is that of block `half` with a bit flipped
  const int a_base = (wave_m * S::fm * 32 + row) * kMxRowBytes + block_at(row, half);
  const int w_base = (BM + wave_n * S::fn * 32 + row) * kMxRowBytes + block_at(row, half);
  static_assert(S::stage % kMxRowBytes == 0, "rows of a stage are aligned to their size");
  const int as_base = S::a_scales + (wave_m * S::fm * 32 + row) * kMxRowScales, ws_base = S::w_scales + (wave_n * S::fn * 32 + row) * kMxRowScales;

  float16v acc[S::fn][S::fm];
  int4v af[2][S::fm], wf[2][S::fn];
  int asc[S::fm], wsc[S::fn];                  // scale bytes of this lane's two blocks of a panel: 0 and 2
  const auto read = [&](int set, int stage, int s) {
    const unsigned char *wp = lds + ((stage * S::stage + w_base) ^ (32 * s)), *ap = lds + ((stage * S::stage + a_base) ^ (32 * s));
#pragma unroll
    for (int i = 0; i < S::fn; ++i) wf[set][i] = *reinterpret_cast<const int4v*>(wp + i * 32 * kMxRowBytes);
#pragma unroll
    for (int j = 0; j < S::fm; ++j) af[set][j] = *reinterpret_cast<const int4v*>(ap + j * 32 * kMxRowBytes);
  };
  const auto read_scales = [&](int stage, int (&sa)[S::fm], int (&sw)[S::fn]) {
    const unsigned char* at = lds + stage * S::stage;
#pragma unroll
    for (int i = 0; i < S::fn; ++i) sw[i] = *reinterpret_cast<const int*>(at + ws_base + i * 32 * kMxRowScales);
#pragma unroll
    for (int j = 0; j < S::fm; ++j) sa[j] = *reinterpret_cast<const int*>(at + as_base + j * 32 * kMxRowScales);
  };
  const auto take_scales = [&](const int (&sa)[S::fm], const int (&sw)[S::fn]) {
#pragma unroll
    for (int i = 0; i < S::fn; ++i) wsc[i] = (int)((uint32_t)sw[i] >> (8 * half));
#pragma unroll
    for (int j = 0; j < S::fm; ++j) asc[j] = (int)((uint32_t)sa[j] >> (8 * half));
  };
#define PQ_MULTIPLY(s)                                                                                                  \
  _Pragma("unroll") for (int i = 0; i < S::fn; ++i) _Pragma("unroll") for (int j = 0; j < S::fm; ++j) acc[i][j] =       \
      mfma<2 * (s)>(wf[s][i], af[s][j], acc[i][j], wsc[i], asc[j]);                                                     \
  pin()

  // the products stay in front of what follows: moved behind the barrier they would hold the fragments of a whole panel
  const auto pin = [&] {
#pragma unroll
    for (int i = 0; i < S::fn; ++i)
#pragma unroll
      for (int j = 0; j < S::fm; ++j) asm volatile("" : "+v"(acc[i][j]));
  };

  // the sums begin with the bias of their columns, zeros in LDS where there is none
  const auto begin = [&](const Tile& t, int slot) {
    const int l = opaque(lane), h = l >> 5, n0 = wave_n * S::fn * 32;
    if (FEW && c.bias) {                                       // this wave's columns, as the loader would have left them
      if (l < S::fn * 32)
        reinterpret_cast<uint32_t*>(lds + S::bias)[slot * BN + n0 + l] = c.bias[t.expert * c.N + min(t.n0 + n0 + l, c.N - 1)];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < S::fn; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4v b = *reinterpret_cast<const uint4v*>(lds + S::bias + (slot * BN + n0 + 32 * i + 8 * q + 4 * h) * 4);
#pragma unroll
        for (int j = 0; j < S::fm; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = as_f32(b[e] << 16);
      }
  };

  // A lane has row l % 32 of a fragment and columns 8 q + 4 (l / 32) + 0 .. 3.  The stores are S::stores of a wave whatever they
  // keep (what has no place goes past the buffer's end and is dropped), so that waits can count past them.
  const auto store = [&](const Tile& t, int slot) {
    if (!GROUPED && c.out_f32) {                               // for checks of the sums: no care taken of its speed
      const int l = opaque(lane);
#pragma unroll
      for (int i = 0; i < S::fn; ++i)
#pragma unroll
        for (int j = 0; j < S::fm; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int64_t m = t.first + (wave_m * S::fm + j) * 32 + (l & 31), n = t.n0 + (wave_n * S::fn + i) * 32 + 8 * (e >> 2) + 4 * (l >> 5) + (e & 3);
            if (m < t.end && n < c.N) ((float*)c.y)[m * c.ldy + n] = acc[i][j][e];
          }
      return;
    }
    const int l = opaque(lane), h = l >> 5;
    const int64_t n0 = t.n0 + wave_n * S::fn * 32;
    const int cols = (int)min(c.N - n0, (int64_t)S::fn * 32);  // of this wave; may be none
    uint64_t kept[(S::fm + 1) / 2];                            // rows of this wave that have one of A's
    if (GROUPED && c.rows) {
#pragma unroll
      for (int j = 0; j < (S::fm + 1) / 2; ++j) {
        const int r = wave_m * S::fm * 32 + 64 * j + l;
        const int64_t m = min(t.first + r, t.end - 1);
        const uint32_t from = ahead ? reinterpret_cast<const uint32_t*>(lds + S::index)[slot * BM + min(r, BM - 1)] : (uint32_t)c.rows[m];
        kept[j] = __ballot(from < (uint32_t)c.a_rows);
      }
    }
    constexpr int kNowhere = 0x7FFFFFF0;
#pragma unroll
    for (int j = 0; j < S::fm; ++j) {
      const int64_t m0 = t.first + (wave_m * S::fm + j) * 32;
      const int rows = (int)min(t.end - m0, (int64_t)32), r = l & 15, piece = 16 * (l >> 4 & 1) + 8 * h;      // first column in a fragment
      uint16_t* y = (uint16_t*)c.y + m0 * c.ldy + n0;
      const auto buf = __builtin_amdgcn_make_buffer_rsrc(y, 0, 0x7FFFFFF0, 0x00027000);
      bool ok[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        ok[s] = r + 16 * s < rows;
        if (GROUPED && c.rows) ok[s] = ok[s] && (kept[j / 2] >> (32 * (j & 1) + 16 * s + r) & 1);
      }
#pragma unroll
      for (int i = 0; i < S::fn; ++i) {
        // halves of the wave: eight columns of a row a lane, columns 16 q + 8 (l / 32); then rows of sixteen lanes: q = 0 and 1 of a row
        // side by side, 64 bytes of it in one store (with 32 bytes 16384 x 8192 x 1024 takes 107 us, not 102, 65536 rows x 2816 x
        // 2048 of 64 experts 254, not 250)
        uint4v half_row[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const auto pack = [&](int g, int e) { return pack_bf16(acc[i][j][4 * g + e], acc[i][j][4 * g + e + 1]); };
          const auto x = __builtin_amdgcn_permlane32_swap(pack(2 * q, 0), pack(2 * q + 1, 0), false, false);
          const auto z = __builtin_amdgcn_permlane32_swap(pack(2 * q, 2), pack(2 * q + 1, 2), false, false);
          half_row[q] = uint4v{x[0], z[0], x[1], z[1]};
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const auto x = __builtin_amdgcn_permlane16_swap(half_row[0][e], half_row[1][e], false, false);
          half_row[0][e] = x[0];
          half_row[1][e] = x[1];
        }
        const int col = 32 * i + piece;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int at = (r + 16 * s) * (int)c.ldy * 2 + 2 * col;
          __builtin_amdgcn_raw_buffer_store_b128(half_row[s], buf, ok[s] && col + 8 <= cols ? at : kNowhere, 0, 0);
          if (c.N & 7) {                                       // uniform; the last columns of rows that end inside eight
#pragma unroll
            for (int e = 0; e < 7; ++e)
              __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(half_row[s][e >> 1] >> (16 * (e & 1))), buf,
                                                    ok[s] && col + 8 > cols && col + e < cols ? at + 2 * e : kNowhere, 0, 0);
          }
        }
      }
    }
  };

  // The fragments of 64 channels are read while those before them are multiplied; the barrier stands before the last of a panel:
  // behind it the next panel has arrived, and the stage of the one before this one is free for the panel three on.
  if (!c.bias)
    for (int i = tid; i < 2 * BN; i += S::waves * 64) reinterpret_cast<uint32_t*>(lds + S::bias)[i] = 0;
  aim();
  Tile t = lt;
  int stage = 0, slot = load_slot;
  if (index_ahead) {
    arrived<0>();
    meet();
  }
#pragma unroll
  for (int p = 0; p < S::stages - 1; ++p) load(p);
  if (more && !drain)
    arrived<(S::stages - 2) * S::loads>();
  else
    arrived<0>();
  meet();
  read_scales(0, asc, wsc);
  take_scales(asc, wsc);
  read(0, 0, 0);
  bool stored = false;                                         // the tile before this one issued S::stores stores, and they may be under way
  for (int tile = tiles.next; tile < tiles.end; tile += tiles.step) {
    const auto fetch = [&] { load((stage + S::stages - 1) & (S::stages - 1)); };
    // What is waited for is the next panel.  Behind its loads come those of two more, and in a tile's first two panels the
    // stores of the tile before.
    const auto turn = [&](int p) {
      if (!more || drain)
        arrived<0>();
      else if (stored && p < 2)
        arrived<(S::stages - 2) * S::loads + S::stores>();
      else
        arrived<(S::stages - 2) * S::loads>();
      meet();
      stage = (stage + 1) & (S::stages - 1);
    };
    int na[S::fm], nw[S::fn];
    if (t.first + wave_m * S::fm * 32 < t.end) {
      begin(t, slot);
      for (int p = 0; p < panels; ++p) {
        fetch();
        read(1, stage, 1);
        PQ_MULTIPLY(0);
        __builtin_amdgcn_sched_barrier(0);
        turn(p);
        read(0, stage, 0);                                     // of no use behind the last panel of all
        read_scales(stage, na, nw);
        PQ_MULTIPLY(1);
        __builtin_amdgcn_sched_barrier(0);
        take_scales(na, nw);
      }
      store(t, slot);
      stored = panels >= 2 && (GROUPED || !c.out_f32) && (c.N & 7) == 0;
    } else {                                                   // none of this wave's rows are in the tile: the others have the matrix units
      for (int p = 0; p < panels; ++p) {
        fetch();
        turn(p);
      }
      stored = false;
      read(0, stage, 0);
      read_scales(stage, na, nw);
      take_scales(na, nw);
    }
    slot ^= 1;
    // the loads are three panels ahead, in the next tile where a tile has more than three
    if (tile + tiles.step < tiles.end) t = !FEW ? lt : tiles.at(c, BM, BN, tile + tiles.step);
  }
#undef PQ_MULTIPLY
}

// ---------------------------------------------------------------- small tiles whose waves share K
// Each of KW waves multiplies the whole tile of 32 FM x 32 FN over every KW-th panel, its panels in a part of LDS of its own (no
// barrier while it runs), then the waves' sums are added up in their order.
// Few rows: bound by the weights' bytes, 1 x 6144 x 4096 4.6 us (13 MB: 2.9 TB/s with the start and the end of the launch, 2.7 us at the
// rate of a large copy; 56 x 12288 x 4096 9.1 us), and from some 32 rows on by what the units take from the caches, since every tile of rows reads the weights and
// every tile of columns the rows.  32 x 32 where there are few of them, 32 x 64 and 64 x 64 for more, us at N 12288:
//   K 8192, M 16   12.6  11.1  11.7     M 56  17.8  17.5  14.5     K 512, M 56   4.9  3.9  4.3     M 128  7.3  5.7  7.2
// (64 x 32 tiles take 13.1, 17.5, 4.0, 6.0: never less than both of the others by 4 %.)  Four waves and four stages (three for 32 x 64), two
// workgroups a unit, one of 64 x 64, have 48 to 64 KB of weights a unit under way beside the panel that each wave multiplies; eight waves, and tiles
// of 128 x 32, were no faster.
template <int FM, int FN, int KW>
struct Split {
  static constexpr int bm = 32 * FM, bn = 32 * FN;
  static constexpr int scales = (bm + bn) * kMxRowBytes, s_loads = FN == 1 ? FM : 2;
  static constexpr int stages = FM * FN == 2 ? 3 : 4;                  // two workgroups of four waves a compute unit, or one of the largest tiles
  static constexpr int stage = (bm + bn) * kMxRowBytes + s_loads * 256, own = stages * stage, lds = KW * own;
  static constexpr int least = 2 * FN + 1 + s_loads;                   // loads of a panel: W's, one of A's at least, scales
  static constexpr int pitch = bn + 4;                                     // floats a row of sums: rows start four banks apart
  static_assert(bm * pitch * 4 <= own, "the sums take a wave's own part");
};

template <int FM, int FN, int KW, bool GROUPED>
__global__ __launch_bounds__(KW * 64) void mx_gemm_split_kernel(const MxCall c) {
  using S = Split<FM, FN, KW>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Tiles<GROUPED> tiles(c, S::bm, S::bn, nullptr);
  if (tiles.next >= tiles.end) return;
  const Tile t = tiles.at(c, S::bm, S::bn, tiles.next);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  unsigned char* own = lds + wave * S::own;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)own;

  const int a_last = (int)(t.end - t.first) - 1, w_last = (int)min((int64_t)S::bn, c.N - t.n0) - 1;
  const uint8_t *a = c.a, *w = c.w + (size_t)t.expert * c.w_next + t.n0 * kMxRowBytes;
  const uint8_t *as = c.a + mx_scales_at(c.a_rows, c.K), *ws = c.w + (size_t)t.expert * c.w_next + mx_scales_at(c.N, c.K) + t.n0 * kMxRowScales;
  const size_t a_next = (size_t)c.a_rows, w_next = (size_t)c.N;
  const auto a_row = [&](int row) { return (uint32_t)max(a_row_of(c, t.first + min(row, a_last)), 0); };
  uint32_t a_at[2 * FM], w_at[2 * FN], s_at[S::s_loads];
#pragma unroll
  for (int i = 0; i < 2 * FM; ++i) {
    const int row = 16 * i + (lane >> 2);
    a_at[i] = a_row(row) * kMxRowBytes + block_at(row, lane & 3);
  }
#pragma unroll
  for (int i = 0; i < 2 * FN; ++i) {
    const int row = 16 * i + (lane >> 2);
    w_at[i] = (uint32_t)min(row, w_last) * kMxRowBytes + block_at(row, lane & 3);
  }
  // scales: W's 32 rows and A's first 32 in one load, A's other 32 (and W's again) in the next; of 64 rows of W in a load of their own
  const bool of_w = lane < 32;
#pragma unroll
  for (int i = 0; i < S::s_loads; ++i) {
    if constexpr (FN == 1)
      s_at[i] = (of_w ? (uint32_t)min(lane, w_last) : a_row(32 * i + lane - 32)) * kMxRowScales;
    else
      s_at[i] = (i == 0 ? (uint32_t)min(lane, w_last) : a_row(min(lane, S::bm - 1))) * kMxRowScales;
  }
  const auto s_base = [&](int i, int p) {
    const bool w_rows = FN == 1 ? of_w : i == 0;
    return (w_rows ? ws : as) + p * ((w_rows ? w_next : a_next) * kMxRowScales);
  };
  constexpr int sw_at = S::scales, sa_at = S::scales + (FN == 1 ? 128 : 256), sa_step = FN == 1 ? 256 : 128;
  const int panels = (int)mx_panels(c.K);
  const auto load = [&](int p, int stage) {
    const uint32_t to = lds0 + stage * S::stage;
#pragma unroll
    for (int i = 0; i < 2 * FN; ++i) load16_to_lds(to + S::bm * kMxRowBytes + i * 1024, w + p * w_next * kMxRowBytes, w_at[i]);
    // rows that the tile has not are left out: what LDS holds instead makes sums that are not stored
#pragma unroll
    for (int i = 0; i < 2 * FM; ++i)
      if (16 * i + (lane >> 2) <= a_last) load16_to_lds(to + i * 1024, a + p * a_next * kMxRowBytes, a_at[i]);
#pragma unroll
    for (int i = 0; i < S::s_loads; ++i) load4_to_lds(to + S::scales + i * 256, s_base(i, p) + s_at[i]);
  };

  const int row = lane & 31, half = lane >> 5;
  float16v acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = float16v{};
  const auto multiply = [&](int stage) {
    const unsigned char* at = own + stage * S::stage;
    int4v wf[2][FN], af[2][FM];
    int sw[FN], sa[FM];
#pragma unroll
    for (int i = 0; i < FN; ++i) sw[i] = (int)(*reinterpret_cast<const uint32_t*>(at + sw_at + i * 128 + row * 4) >> (8 * half));
#pragma unroll
    for (int j = 0; j < FM; ++j) sa[j] = (int)(*reinterpret_cast<const uint32_t*>(at + sa_at + j * sa_step + row * 4) >> (8 * half));
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < FN; ++i) wf[s][i] = *reinterpret_cast<const int4v*>(at + (S::bm + 32 * i + row) * kMxRowBytes + block_at(row, 2 * s + half));
#pragma unroll
      for (int j = 0; j < FM; ++j) af[s][j] = *reinterpret_cast<const int4v*>(at + (32 * j + row) * kMxRowBytes + block_at(row, 2 * s + half));
    }
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        acc[i][j] = mfma<0>(wf[0][i], af[0][j], acc[i][j], sw[i], sa[j]);
        acc[i][j] = mfma<2>(wf[1][i], af[1][j], acc[i][j], sw[i], sa[j]);
      }
  };
#pragma unroll
  for (int i = 0; i < S::stages; ++i)
    if (wave + i * KW < panels) load(wave + i * KW, i);
  int stage = 0;
  for (int p = wave; p < panels; p += KW) {
    // behind the panel that is waited for come the loads of stages - 1 others, each of `least` at least, or fewer at the end
    if (p + (S::stages - 1) * KW < panels)
      arrived<(S::stages - 1) * S::least>();
    else
      arrived<0>();
    multiply(stage);
    if (p + S::stages * KW < panels) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // this stage's reads are done
      load(p + S::stages * KW, stage);
    }
    stage = (stage + 1) % S::stages;
  }
  // sums: row m = l % 32, columns 8 q + 4 (l / 32) .. of this wave's part
  arrived<0>();
  float* part = reinterpret_cast<float*>(own);
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(part + (32 * j + row) * S::pitch + 32 * i + 8 * q + 4 * half) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
  __syncthreads();
  const float* parts = reinterpret_cast<const float*>(lds);
  for (int i = tid; i < S::bm * 4 * FN; i += KW * 64) {
    const int r = i / (4 * FN), col = i % (4 * FN) * 8;
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
    if (!GROUPED && c.out_f32) {
      for (int e = 0; e < 8; ++e)
        if (n + e < c.N) ((float*)c.y)[m * c.ldy + n + e] = v[e];
    } else {
      store8(c, m, n, make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])));
    }
  }
}

// ---------------------------------------------------------------- small tiles, a wave each
// Where there are enough of them, every wave computes tiles of 32 FM x 32 by itself, one after another, three panels ahead also across
// tiles: nothing to meet for and nothing to add up.  The waves of a workgroup take neighbouring columns of the same rows.
// Bound by the weights' bytes: 1536 rows of 128 experts, 1536 x 2560, in 50 to 52 us (267 MB of weights: 5.2 TB/s, a large copy's rate),
// with the quantizer in front 59; with waves that share K, which start and end with every tile, 80.
template <int FM>
struct Alone {
  static constexpr int bm = 32 * FM, bn = 32, waves = 4;
  static constexpr int scales = (bm + bn) * kMxRowBytes;
  static constexpr int stages = FM == 1 ? 4 : 2, stage = (bm + bn) * kMxRowBytes + FM * 256, own = stages * stage;
  static constexpr int table = waves * own, lds = table + Tiles<true>::kTableBytes;
  static constexpr int least = 2 + 1 + FM;                             // loads of a panel: W's, one of A's at least, scales
};

template <int FM>
__global__ __launch_bounds__(256) void mx_gemm_alone_kernel(const MxCall c) {
  using S = Alone<FM>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Tiles<true> tiles(c, S::bm, S::bn * S::waves, reinterpret_cast<int32_t*>(lds + S::table));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  unsigned char* own = lds + wave * S::own;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)own;
  const int panels = (int)mx_panels(c.K);
  const size_t as_at = mx_scales_at(c.a_rows, c.K), ws_at = mx_scales_at(c.N, c.K);

  // loader, at tile load_tile; a tile of columns from N on is none of this wave's
  int load_tile = tiles.next, load_panel = 0, a_last = 0;
  Tile lt;
  const uint8_t *a_from, *w_from, *s_from;                             // s_from: a lane's own, of W's rows below lane 32, of A's above
  const size_t a_step = (size_t)c.a_rows * kMxRowBytes, w_step = (size_t)c.N * kMxRowBytes;
  const bool of_w = lane < 32;
  const size_t s_step = (size_t)(of_w ? c.N : c.a_rows) * kMxRowScales;
  uint32_t a_off[2 * FM], w_off[2], s_off[FM];
  const auto find = [&](int tile, Tile& t) {
    t = tiles.at(c, S::bm, S::bn * S::waves, tile);
    t.n0 += S::bn * wave;
    return (bool)__builtin_amdgcn_readfirstlane(t.n0 < c.N);
  };
  const auto aim = [&] {                                               // load_tile moves past tiles that are none of this wave's
    while (load_tile < tiles.end && !find(load_tile, lt)) load_tile += tiles.step;
    if (load_tile >= tiles.end) return;
    a_last = (int)(lt.end - lt.first) - 1;
    const int w_last = (int)min((int64_t)S::bn, c.N - lt.n0) - 1;
    const auto a_row = [&](int row) { return (uint32_t)max(a_row_of(c, lt.first + min(row, a_last)), 0); };
    a_from = uniform(c.a);
    const uint8_t* w = c.w + (size_t)lt.expert * c.w_next;
    w_from = uniform(w + lt.n0 * kMxRowBytes);
    s_from = of_w ? w + ws_at + lt.n0 * kMxRowScales : c.a + as_at;
#pragma unroll
    for (int i = 0; i < 2 * FM; ++i) {
      const int row = 16 * i + (lane >> 2);
      a_off[i] = a_row(row) * kMxRowBytes + block_at(row, lane & 3);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 16 * i + (lane >> 2);
      w_off[i] = (uint32_t)min(row, w_last) * kMxRowBytes + block_at(row, lane & 3);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) s_off[i] = (of_w ? (uint32_t)min(lane, w_last) : a_row(32 * i + lane - 32)) * kMxRowScales;
  };
  // rows that the tile has not are left out: what LDS holds instead makes sums that are not stored
  const auto load = [&](int stage) {
    if (load_tile >= tiles.end) return;
    const uint32_t to = lds0 + stage * S::stage;
#pragma unroll
    for (int i = 0; i < 2; ++i) load16_to_lds(to + S::bm * kMxRowBytes + i * 1024, w_from, w_off[i]);
#pragma unroll
    for (int i = 0; i < 2 * FM; ++i)
      if (16 * i + (lane >> 2) <= a_last) load16_to_lds(to + i * 1024, a_from, a_off[i]);
#pragma unroll
    for (int i = 0; i < FM; ++i) load4_to_lds(to + S::scales + i * 256, s_from + s_off[i]);
    a_from += a_step;
    w_from += w_step;
    s_from += s_step;
    if (++load_panel == panels) {
      load_panel = 0;
      load_tile += tiles.step;
      aim();
    }
  };

  const int row = lane & 31, half = lane >> 5;
  float16v acc[FM];
  const auto multiply = [&](int stage) {
    const unsigned char* at = own + stage * S::stage;
    int4v wf[2], af[2][FM];
    const int sw = (int)(*reinterpret_cast<const uint32_t*>(at + S::scales + row * 4) >> (8 * half));
    int sa[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) sa[j] = (int)(*reinterpret_cast<const uint32_t*>(at + S::scales + j * 256 + 128 + row * 4) >> (8 * half));
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      wf[s] = *reinterpret_cast<const int4v*>(at + (S::bm + row) * kMxRowBytes + block_at(row, 2 * s + half));
#pragma unroll
      for (int j = 0; j < FM; ++j) af[s][j] = *reinterpret_cast<const int4v*>(at + (32 * j + row) * kMxRowBytes + block_at(row, 2 * s + half));
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
      acc[j] = mfma<0>(wf[0], af[0][j], acc[j], sw, sa[j]);
      acc[j] = mfma<2>(wf[1], af[1][j], acc[j], sw, sa[j]);
    }
  };

  aim();
  int tile = load_tile;
#pragma unroll
  for (int i = 0; i < S::stages; ++i) load(i);
  int stage = 0;
  for (; tile < tiles.end; tile += tiles.step) {
    Tile t;
    if (!find(tile, t)) continue;
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[j] = float16v{};
    for (int p = 0; p < panels; ++p) {
      // behind the panel that is waited for come the loads of stages - 1 others, each of `least` at least, or none at the end
      if (load_tile < tiles.end)
        arrived<(S::stages - 1) * S::least>();
      else
        arrived<0>();
      multiply(stage);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");               // this stage's reads are done
      load(stage);
      stage = (stage + 1) & (S::stages - 1);
    }
    // a lane has row l % 32 and columns 8 q + 4 (l / 32) .. + 3; the halves of the wave exchange what makes eight columns
    const int cols = (int)min(c.N - t.n0, (int64_t)S::bn);
    float bias[16] = {};
    if (c.bias) {
#pragma unroll
      for (int e = 0; e < 16; ++e) bias[e] = bf16_to_f32(c.bias[t.expert * c.N + t.n0 + min(8 * (e >> 2) + 4 * half + (e & 3), cols - 1)]);
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
      const int64_t m = t.first + 32 * j + row;
      const bool ok = m < t.end && a_row_of(c, min(m, t.end - 1)) >= 0;
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        const auto pack = [&](int g, int e) { return pack_bf16(acc[j][4 * g + e] + bias[4 * g + e], acc[j][4 * g + e + 1] + bias[4 * g + e + 1]); };
        const auto x = __builtin_amdgcn_permlane32_swap(pack(q, 0), pack(q + 1, 0), false, false);
        const auto z = __builtin_amdgcn_permlane32_swap(pack(q, 2), pack(q + 1, 2), false, false);
        const int64_t n = t.n0 + 8 * (q + half);
        if (ok && n < c.N) store8(c, m, n, make_uint4(x[0], z[0], x[1], z[1]));
      }
    }
  }
  arrived<0>();                                                        // loads into this wave's LDS
}

// `most`: workgroups that run at a time and go through all tiles, or 0: one for every tile that there could be (those beyond the
// tiles that there are end at once)
template <class K>
int launch(K kernel, const char* name, const MxCall& c, int bm, int bn, int waves, int lds, int most, std::atomic<uint64_t>& allowed,
           hipStream_t st) {
  const int64_t tiles_m = (c.M + bm - 1) / bm + (c.offsets ? (c.experts < c.M ? c.experts : c.M) : 0), across = (c.N + bn - 1) / bn;
  // a grid has fewer than 2^32 threads
  if (tiles_m * across + 8 >= ((int64_t)1 << 26) / waves)
    return fail(PQ_ERR_SHAPE, "MXFP4 product: M=%lld N=%lld are too many tiles for one call", (long long)c.M, (long long)c.N);
  int rc = allow_lds((const void*)kernel, (size_t)lds, allowed, name);
  if (rc) return rc;
  const int64_t n = (tiles_m * across + 7) / 8 * 8;
  kernel<<<(unsigned)(most && most < n ? most : n), waves * 64, lds, st>>>(c);
  return check_hip(hipGetLastError(), name);
}

constexpr int kUnits = 256;                  // compute units

template <int BM, int BN, int WM, int WN, bool GROUPED>
int launch_shared(const MxCall& c, hipStream_t st) {
  using S = Shared<BM, BN, WM, WN>;
  static std::atomic<uint64_t> allowed{0}, allowed_few{0};
  constexpr int lds = S::lds(GROUPED), most = kUnits * (160 * 1024 / lds);
  if (mx_panels(c.K) < S::few)
    return launch(mx_gemm_shared_kernel<BM, BN, WM, WN, GROUPED, true>, "mx_gemm_shared_kernel", c, BM, BN, S::waves, lds, most, allowed_few, st);
  return launch(mx_gemm_shared_kernel<BM, BN, WM, WN, GROUPED, false>, "mx_gemm_shared_kernel", c, BM, BN, S::waves, lds, most, allowed, st);
}
template <int FM, int FN, int KW, bool GROUPED>
int launch_split(const MxCall& c, hipStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  return launch(mx_gemm_split_kernel<FM, FN, KW, GROUPED>, "mx_gemm_split_kernel", c, 32 * FM, 32 * FN, KW, Split<FM, FN, KW>::lds, 0, allowed, st);
}

template <int FM>
int launch_alone(const MxCall& c, hipStream_t st) {
  using S = Alone<FM>;
  static std::atomic<uint64_t> allowed{0};
  return launch(mx_gemm_alone_kernel<FM>, "mx_gemm_alone_kernel", c, S::bm, S::bn * S::waves, S::waves, S::lds, kUnits * (160 * 1024 / S::lds), allowed, st);
}

// Which kernel: the one that takes the shortest time by a model of each in us.  Small tiles read more than they multiply and are bound by what
// the units take from the caches: a start, some us and a time a panel for every round of 256 tiles, and the weights' bytes.  Large ones
// take some us a turn and a time a panel, and only pay where there are enough of them.  Fitted to the dense kernels timed at M 16 .. 768, N 1024 ..
// 16384 and K 512 .. 8192 (200 shapes: the choice is within 7 % of the best for 191, within 13 % for all), the two largest tiles at M up to
// 8192 as well.  us, 32 x 32, 32 x 64, 64 x 64, 128 x 128:
//   M 32, N 4096, K 2048    3.9   4.4   5.1   8.1        M 256, N 4096, K 8192   15.4  12.4  10.3  25.1
//   M 512, N 12288, K 512  23.5  15.6  19.0   7.9        M 256, N 12288, K 8192  48.5  38.2  35.5  25.8
// and 128 x 128 and 256 x 256 at M 1024, N 12288, K 8192  62  55.
// By expert the same constants stand, and the kernels of a wave a tile take the weights' bytes or what the units take from the caches: not fitted.  Against
// all kernels at 8, 64 and 256 experts, 16 to 1000 rows of each, N 1024 and 4096, K 128 to 4096, rows spread evenly and not (288 shapes) the choice is
// within 7 % of the best for 146 and within 30 % for 239.  The worst are those of few panels and many rows, where a wave a tile is taken and what its
// outputs, its start and its end cost is left out: 200000 rows and more, K 128, take 1.9 to 2.1 times as long as with 256 x 256 tiles.
// enough tiles of 32 columns for every wave of the chip: no need to share K
bool enough_alone(const MxCall& c) {
  const int64_t whole = (c.M + 31) / 32, rows = whole > c.experts ? whole : c.experts < c.M ? c.experts : c.M;
  return rows * ((c.N + 31) / 32) >= 2048;
}
enum class Kernel { split32x32, split32x64, split64x64, alone32, alone64, shared128, shared256 };
Kernel choose(const MxCall& c, bool grouped) {
  const double panels = (double)mx_panels(c.K), groups = grouped ? (double)(c.experts < c.M ? c.experts : c.M) : 1.0;
  // tiles of rows: a group's last is half full on average
  const auto tiles = [&](int bm, int bn) {
    const double whole = (double)c.M / bm, rows = grouped ? (whole + 0.5 * groups > groups ? whole + 0.5 * groups : groups) : (double)((c.M + bm - 1) / bm);
    return rows * (double)((c.N + bn - 1) / bn);
  };
  const double mb = groups * (double)c.N * panels * (kMxRowBytes + kMxRowScales) / 1e6, weights = mb / 5.2;      // at 5.2 TB/s
  const auto split = [&](int fm, int fn) {
    const double rounds = (double)(int64_t)((tiles(32 * fm, 32 * fn) + kUnits - 1) / kUnits);
    return fm == 2   ? 0.56 + rounds * (3.07 + 0.0913 * panels) + 0.063 * mb
           : fn == 2 ? 2.26 + rounds * (0.73 + 0.0619 * panels) + 0.075 * mb
                     : 2.20 + rounds * (0.59 + 0.0418 * panels) + 0.063 * mb;
  };
  const auto alone = [&](int fm) {
    const double traffic = tiles(32 * fm, 32) * panels * (fm == 1 ? 4.35e-3 : 6.65e-3) / 24.0;           // MB at 24 TB/s
    return 2.8 + (traffic > weights ? traffic : weights);
  };
  const auto shared = [&](int bm) {
    const double n = tiles(bm, bm), turns = (double)(int64_t)((n + kUnits - 1) / kUnits);
    const double full = n < kUnits ? n / kUnits : 1.0;                   // how much of the chip works
    const double panel = bm == 128 ? (turns <= 1 ? 0.33 : 0.29 * turns) : turns * (0.62 + 0.35 * full), t = panels * panel;
    return (bm == 128 ? 2.8 + turns : 2.6 + turns * (1.5 + 3.0 * full)) + (t > weights ? t : weights);
  };
  const bool many = grouped && enough_alone(c);
  Kernel best = many ? Kernel::alone32 : Kernel::split32x32;
  double least = many ? alone(1) : split(1, 1);
  const auto consider = [&](Kernel k, double t) {
    if (t < least) best = k, least = t;
  };
  if (many) {
    consider(Kernel::alone64, alone(2));
  } else {
    consider(Kernel::split32x64, split(1, 2));
    consider(Kernel::split64x64, split(2, 2));
  }
  consider(Kernel::shared128, shared(128));
  consider(Kernel::shared256, shared(256));
  return best;
}

template <bool GROUPED>
int run(const MxCall& c, hipStream_t st) {
  const Kernel k = choose(c, GROUPED);
  if constexpr (GROUPED) {
    if (k == Kernel::alone32) return launch_alone<1>(c, st);
    if (k == Kernel::alone64) return launch_alone<2>(c, st);
  }
  switch (k) {
    case Kernel::split32x32: return launch_split<1, 1, 4, GROUPED>(c, st);
    case Kernel::split32x64: return launch_split<1, 2, 4, GROUPED>(c, st);
    case Kernel::split64x64: return launch_split<2, 2, 4, GROUPED>(c, st);
    case Kernel::shared128: return launch_shared<128, 128, 2, 2, GROUPED>(c, st);
    default: return launch_shared<256, 256, 2, 4, GROUPED>(c, st);
  }
}

}  // namespace

void mx_gemm_tile(int experts, int64_t M, int64_t N, int64_t K, int* bm, int* bn) {
  MxCall c{};
  c.M = M, c.N = N, c.K = K, c.experts = experts ? experts : 1;
  switch (choose(c, experts > 0)) {
    case Kernel::split32x32: *bm = *bn = 32; break;
    case Kernel::split32x64: *bm = 32, *bn = 64; break;
    case Kernel::split64x64: *bm = *bn = 64; break;
    case Kernel::alone32: *bm = Alone<1>::bm, *bn = Alone<1>::bn * Alone<1>::waves; break;
    case Kernel::alone64: *bm = Alone<2>::bm, *bn = Alone<2>::bn * Alone<2>::waves; break;
    case Kernel::shared128: *bm = *bn = 128; break;
    case Kernel::shared256: *bm = *bn = 256; break;
  }
}

int run_mx_gemm(const MxCall& c, hipStream_t st) {
  if (c.M == 0) return PQ_OK;
  return c.offsets ? run<true>(c, st) : run<false>(c, st);
}

}  // namespace pq
