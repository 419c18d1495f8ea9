// What stands around the experts' products: routing (the largest of the router's logits, their softmax weights, and the order of
// the rows by expert) and the weighted sum of the rows that the experts made.
#include "pq_host.h"
#include "pq_mx.h"

namespace pq {

namespace {

constexpr int kTile = 64;                                     // tokens a pass of a workgroup: a bit each of a 64-bit mask
constexpr int kRouteWaves = 16, kRouteThreads = kRouteWaves * kWave;
constexpr int kMaxBlocks = 512;                               // workgroups; more tokens mean more passes of each

// ---------------------------------------------------------------- the k largest of a token's logits
// A logit as an unsigned key that orders alike, 0 where the expert cannot be chosen (-inf, NaN); -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = as_u32(v + 0.0f);
  return v > -INFINITY ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return as_f32(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

// largest and sum, in a fixed order, over the LANES lanes of a token, in each of them: inside a row of sixteen lanes by DPP exchanges, then (a wave
// a token) the four rows on the scalar unit
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  v = max(v, dpp_u32<0xB1>(v));                               // quad_perm [1,0,3,2]
  v = max(v, dpp_u32<0x4E>(v));                               // quad_perm [2,3,0,1]
  v = max(v, dpp_u32<0x141>(v));                              // row_half_mirror
  v = max(v, dpp_u32<0x140>(v));                              // row_mirror
  if constexpr (LANES == 16) return v;
  const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16), c = __builtin_amdgcn_readlane(v, 32),
                 d = __builtin_amdgcn_readlane(v, 48);
  return max(max(a, b), max(c, d));
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp_f32<0xB1>(v);
  v += dpp_f32<0x4E>(v);
  v += dpp_f32<0x141>(v);
  v += dpp_f32<0x140>(v);
  if constexpr (LANES == 16) return v;
  const float a = as_f32(__builtin_amdgcn_readlane(as_u32(v), 0)), b = as_f32(__builtin_amdgcn_readlane(as_u32(v), 16)),
              c = as_f32(__builtin_amdgcn_readlane(as_u32(v), 32)), d = as_f32(__builtin_amdgcn_readlane(as_u32(v), 48));
  return (a + b) + (c + d);
}

// A lane's PER experts, PER lane + i, largest first: a token's largest is then one of its lanes' first, and the lane that has it moves
// on to its next.  A bf16 logit and its expert fit one word (the expert's complement below, so that equal logits order by
// expert); binary32 logits keep the expert beside the key.
template <int PER, bool BF16, int LANES>
struct Sorted {
  uint32_t key[PER], low[BF16 ? 1 : PER];                     // low: complement of the expert
  __device__ __forceinline__ void order(int i, int j) {       // the larger of two to place i
    if constexpr (BF16) {
      const uint32_t a = max(key[i], key[j]), b = min(key[i], key[j]);
      key[i] = a, key[j] = b;
    } else {
      const uint64_t a = (uint64_t)key[i] << 32 | low[i], b = (uint64_t)key[j] << 32 | low[j];
      const bool swap = b > a;
      const uint32_t k = key[i], l = low[i];
      key[i] = swap ? key[j] : k, low[i] = swap ? low[j] : l;
      key[j] = swap ? k : key[j], low[j] = swap ? l : low[j];
    }
  }
  __device__ __forceinline__ void sort() {                    // odd-even merges
#pragma unroll
    for (int p = 1; p < PER; p *= 2)
#pragma unroll
      for (int k = p; k >= 1; k /= 2)
#pragma unroll
        for (int j = k % p; j + k < PER; j += 2 * k)
#pragma unroll
          for (int i = 0; i < k; ++i)
            if (i + j + k < PER && (i + j) / (2 * p) == (i + j + k) / (2 * p)) order(i + j, i + j + k);
  }
  // the token's largest: its key and expert (0 and -1: none is left); it is taken out
  __device__ __forceinline__ uint32_t pop(int& expert) {
    uint32_t best = lanes_max<LANES>(key[0]);
    bool mine = key[0] == best;
    if constexpr (BF16) {
      expert = best ? 0xFFFF - (int)(best & 0xFFFFu) : -1;
    } else {
      const uint32_t l = lanes_max<LANES>(mine ? low[0] : 0u);
      mine = mine && low[0] == l;
      expert = best ? (int)~l : -1;
    }
#pragma unroll
    for (int i = 0; i + 1 < PER; ++i) {
      key[i] = mine ? key[i + 1] : key[i];
      if constexpr (!BF16) low[i] = mine ? low[i + 1] : low[i];
    }
    key[PER - 1] = mine ? 0u : key[PER - 1];
    return BF16 ? best & 0xFFFF0000u : best;
  }
};

// e^x, x <= 0, for a sum whose largest term is 1, by the unit's power of two.  The product with log2 e is rounded (2^-24 of it) and so is the constant
// (0.22 2^-24), which together change the term by 1.23 |x| 2^-24 of itself, at most 0.45 2^-24 of the largest; the unit adds a last place,
// 2^-23 of the term.  Weights over all of 256 normal logits of deviation 2, 8192 tokens: off by 6.6 10^-8 of themselves in the root mean square,
// those of a plain binary32 softmax by 5.7 10^-8.
__device__ __forceinline__ float exp_in_sum(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// A token's logits, expert PER sub + i at place i of lane `sub` of its LANES: up to 16 bytes a load where the rows allow it, else one
// logit (16381 tokens of bf16, 256 experts, k 8: the first launch takes 8.4 us, with one logit a load 10.1).
template <int PER, bool BF16>
__device__ __forceinline__ void load_logits(const RouteCall& c, int64_t t, int sub, float (&v)[PER]) {
  const int first = PER * sub;
  if (c.wide) {                                               // uniform
    constexpr int per = BF16 ? (PER < 8 ? PER : 8) : 4;       // logits a load
#pragma unroll
    for (int i = 0; i < PER; i += per) {
      uint32_t w[4] = {};
      const bool there = first + i < c.experts;               // the experts are a multiple of what a load takes
      if constexpr (BF16 && per == 4) {
        const uint2 x = there ? *reinterpret_cast<const uint2*>((const uint16_t*)c.logits + t * c.ld + first + i) : make_uint2(0, 0);
        w[0] = x.x, w[1] = x.y;
      } else if (there) {
        const uint4 x = BF16 ? *reinterpret_cast<const uint4*>((const uint16_t*)c.logits + t * c.ld + first + i)
                             : *reinterpret_cast<const uint4*>((const float*)c.logits + t * c.ld + first + i);
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
      }
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float x = BF16 ? (j & 1 ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1])) : as_f32(w[j & 3]);
        v[i + j] = there ? x : -INFINITY;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = first + i;
    if constexpr (BF16)
      v[i] = e < c.experts ? bf16_to_f32(((const uint16_t*)c.logits)[t * c.ld + e]) : -INFINITY;
    else
      v[i] = e < c.experts ? ((const float*)c.logits)[t * c.ld + e] : -INFINITY;
  }
}
// LANES lanes a token: ids and weights written (where `there`), lane j < k has the j-th expert (-1: none).
template <int PER, bool BF16, int LANES>
__device__ __forceinline__ int route_token(const RouteCall& c, int64_t t, bool there, int sub, const float (&v)[PER]) {
  Sorted<PER, BF16, LANES> s;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = (uint32_t)(PER * sub + i), key = key_of(v[i]);
    if constexpr (BF16) {
      s.key[i] = key ? (key & 0xFFFF0000u) | (0xFFFFu - e) : 0u;      // a bf16 value says nothing in the low half
    } else {
      s.key[i] = key;
      s.low[i] = ~e;
    }
  }
  s.sort();
  uint32_t kept = 0, first = 0;
  int id = -1;
  for (int j = 0; j < c.k; ++j) {
    int e;
    const uint32_t key = s.pop(e);
    if (j == 0) first = key;
    if (sub == j) kept = key, id = e;
  }
  const auto value = [](uint32_t key) { return BF16 && !(key & 0x80000000u) ? as_f32(~key & 0xFFFF0000u) : value_of(key); };
  const float top = value(first), p = id >= 0 ? expf(value(kept) - top) : 0.0f;
  float sum = p;
  if (!c.renormalize) {
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += v[i] > -INFINITY ? exp_in_sum(v[i] - top) : 0.0f;
  }
  sum = lanes_sum<LANES>(sum);
  if (there && sub < c.k) {
    c.ids[t * c.k + sub] = id;
    c.weights[t * c.k + sub] = id >= 0 ? p / sum : 0.0f;
  }
  return there ? id : -1;
}

// counts that a workgroup of the first launch leaves: of four experts together
__host__ __device__ constexpr int counts_of(int experts) { return (experts + 3) / 4 * 4; }

// exclusive sums of counts[0 .. n), n <= kRouteThreads, by the whole workgroup; returns this thread's and leaves the total
__device__ __forceinline__ int block_scan(int v, int* wave_sums, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int o = __shfl_up(upto, d, kWave);
    if (lane >= d) upto += o;
  }
  if (lane == 63) wave_sums[wave] = upto;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kRouteWaves; ++w) {
    const int n = wave_sums[w];
    if (w < wave) before += n;
    total += n;
  }
  return before + upto - v;
}

// The experts of the pairs (token, j) of one pass, at most 64 x 32: thread e has those of pairs e and e + 1024
constexpr int kPairs = kTile * 32 / kRouteThreads;
__device__ __forceinline__ void load_ids(const RouteCall& c, int64_t t0, int n, int (&id)[kPairs]) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const int pair = i * kRouteThreads + threadIdx.x;
    id[i] = pair < n ? c.ids[t0 * c.k + pair] : -1;
  }
}
// positions and rows of the tokens of one pass, from a mask of tokens and the next place of every expert
__device__ __forceinline__ void place_pass(const RouteCall& c, int64_t t0, int n, const int (&id)[kPairs], const uint64_t* mask, const int32_t* base) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const int pair = i * kRouteThreads + threadIdx.x, t = pair / c.k;
    if (pair >= n) break;
    int place = -1;
    if (id[i] >= 0) {
      place = base[id[i]] + __popcll(mask[id[i]] & ((1ull << t) - 1));
      c.rows[place] = (int32_t)(t0 + t);
    }
    c.positions[t0 * c.k + pair] = place;
  }
}

// Few tokens, one for every LANES threads at most, one launch: a mask of tokens for every expert says all of it.
template <int PER, bool BF16, int LANES>
__global__ __launch_bounds__(kRouteThreads) void route_few_kernel(const RouteCall c) {
  __shared__ uint64_t mask[LANES * PER];
  __shared__ int32_t base[LANES * PER];
  __shared__ int wave_sums[kRouteWaves];
  const int sub = threadIdx.x % LANES, t = threadIdx.x / LANES, e = threadIdx.x, tokens = (int)c.tokens;
  const bool any = (int)(threadIdx.x / kWave) * (kWave / LANES) < tokens;      // waves without a token read nothing and leave the unit to the others
  float v[PER];
  if (any) load_logits<PER, BF16>(c, min(t, tokens - 1), sub, v);
  if (e < c.experts) mask[e] = 0;
  __syncthreads();
  if (any) {
    const int id = route_token<PER, BF16, LANES>(c, t, t < tokens, sub, v);
    if (sub < c.k && id >= 0) atomicOr((unsigned long long*)&mask[id], 1ull << t);
  }
  __syncthreads();
  int total;
  const int at = block_scan(e < c.experts ? __popcll(mask[e]) : 0, wave_sums, total);
  if (e < c.experts) base[e] = c.offsets[e] = at;
  if (e == 0) c.offsets[c.experts] = total;
  __threadfence_block();
  __syncthreads();
  const int pairs = tokens * c.k;
  for (int i = total + threadIdx.x; i < pairs; i += kRouteThreads) c.rows[i] = -1;
  int id[kPairs];
  load_ids(c, 0, pairs, id);
  place_pass(c, 0, pairs, id, mask, base);
}

// Many tokens, first launch: experts and weights, and how many rows of each expert a workgroup's tokens make.
template <int PER, bool BF16, int LANES>
__global__ __launch_bounds__(kRouteThreads) void route_topk_kernel(const RouteCall c, int per_block, uint16_t* __restrict__ hist) {
  __shared__ uint32_t count[LANES * PER];
  const int sub = threadIdx.x % LANES, group = threadIdx.x / LANES;
  constexpr int groups = kRouteThreads / LANES;
  const int wave_first = threadIdx.x / kWave * (kWave / LANES);
  const int64_t first = (int64_t)blockIdx.x * per_block, end = min(first + per_block, c.tokens);
  float v[PER];
  if (first + wave_first < end) load_logits<PER, BF16>(c, min(first + group, end - 1), sub, v);
  for (int e = threadIdx.x; e < c.experts; e += kRouteThreads) count[e] = 0;
  __syncthreads();
  for (int64_t t0 = first; t0 + wave_first < end; t0 += groups) {
    const int64_t t = t0 + group;
    float next[PER] = {};
    if (t0 + groups < end) load_logits<PER, BF16>(c, min(t + groups, end - 1), sub, next);
    const int id = route_token<PER, BF16, LANES>(c, t, t < end, sub, v);
    if (sub < c.k && id >= 0) atomicAdd(&count[id], 1u);
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = next[i];
  }
  __syncthreads();
  const int width = counts_of(c.experts);
  for (int e = threadIdx.x; e < width; e += kRouteThreads) hist[(int64_t)blockIdx.x * width + e] = e < c.experts ? (uint16_t)count[e] : 0;
}

// Second launch, places of the rows: the experts' offsets, then the rows of earlier workgroups, then the earlier tokens of this one.
// Every workgroup sums up all counts itself: at most 512 x 1024 of two bytes, out of the caches, four experts a load (one: 8.6 us for
// 16381 tokens and 256 experts, now 6.8).
__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(const RouteCall c, int per_block, const uint16_t* __restrict__ hist) {
  __shared__ uint64_t mask[1024];                             // tokens of the pass that chose the expert
  __shared__ int32_t base[1024];                              // place of its next row
  __shared__ int32_t part[2][kRouteThreads * 4];
  __shared__ int wave_sums[kRouteWaves];
  const int e = threadIdx.x, blocks = (int)gridDim.x;
  const int64_t first = (int64_t)blockIdx.x * per_block, end = min(first + per_block, c.tokens);
  const auto pairs_at = [&](int64_t t0) { return (int)min((int64_t)kTile, end - t0) * c.k; };
  int id[kPairs];
  load_ids(c, first, pairs_at(first), id);                    // on their way while the counts are summed up
  // thread (four experts, share): shares of the workgroups' counts, as many as there are threads for
  const int width = counts_of(c.experts), quads = width / 4, shares = min(kRouteThreads / quads, 32), mine = e % quads, share = e / quads;
  int before[4] = {}, all[4] = {};
  if (share < shares) {
    const uint2* h = reinterpret_cast<const uint2*>(hist) + mine;
    // two counts a word while their sums fit sixteen bits: runs of `run` workgroups
    const int run = 65535 / per_block * shares;
    for (int b0 = share; b0 < blocks; b0 += run) {
      uint2 p = make_uint2(0, 0), q = make_uint2(0, 0);
#pragma unroll 8
      for (int b = b0; b < min(b0 + run, blocks); b += shares) {
        const uint2 n = h[(int64_t)b * quads];
        const bool earlier = b < (int)blockIdx.x;
        q.x += n.x, q.y += n.y;
        p.x += earlier ? n.x : 0u, p.y += earlier ? n.y : 0u;
      }
      before[0] += p.x & 0xFFFFu, before[1] += p.x >> 16, before[2] += p.y & 0xFFFFu, before[3] += p.y >> 16;
      all[0] += q.x & 0xFFFFu, all[1] += q.x >> 16, all[2] += q.y & 0xFFFFu, all[3] += q.y >> 16;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[0][share * width + mine * 4 + i] = before[i], part[1][share * width + mine * 4 + i] = all[i];
  }
  __syncthreads();
  int earlier = 0, rows = 0;
  if (e < c.experts)
    for (int s = 0; s < shares; ++s) earlier += part[0][s * width + e], rows += part[1][s * width + e];
  int total;
  const int at = block_scan(rows, wave_sums, total);
  if (e < c.experts) {
    base[e] = at + earlier;
    mask[e] = 0;
    if (blockIdx.x == 0) c.offsets[e] = at;
  }
  if (e == 0 && blockIdx.x == 0) c.offsets[c.experts] = total;
  const int64_t pairs = c.tokens * c.k;
  for (int64_t i = total + (int64_t)blockIdx.x * kRouteThreads + e; i < pairs; i += (int64_t)blocks * kRouteThreads) c.rows[i] = -1;
  for (int64_t t0 = first; t0 < end; t0 += kTile) {
    const int n = pairs_at(t0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPairs; ++i)
      if (id[i] >= 0) atomicOr((unsigned long long*)&mask[id[i]], 1ull << ((i * kRouteThreads + e) / c.k));
    __syncthreads();
    place_pass(c, t0, n, id, mask, base);
    if (t0 + kTile < end) load_ids(c, t0 + kTile, pairs_at(t0 + kTile), id);
    __syncthreads();
    if (e < c.experts) base[e] += __popcll(mask[e]), mask[e] = 0;
  }
}

// ---------------------------------------------------------------- the weighted sum
// out[t] = addend[t] + sum_j weights[t, j] * y[positions[t, j]], j ascending, in binary32, rounded once to bf16.  Eight columns a
// thread, a token a workgroup: its rows and weights are uniform, and the loads of kAhead rows are under way at a time.  Memory bound:
// 8191 tokens, k 8, 5120 columns, an addend: 839 MB in 157 to 160 us, 5.3 TB/s (a large copy: 5.1); with a row after the other 179.
constexpr int kAhead = 8, kCombineThreads = 128;
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(const CombineCall c, int chunks) {
  const int64_t t = blockIdx.x / (uint32_t)chunks;
  const int64_t col = ((int64_t)(blockIdx.x % (uint32_t)chunks) * kCombineThreads + threadIdx.x) * 8;
  if (col >= c.N) return;
  const int width = (int)min((int64_t)8, c.N - col);
  const auto load = [&](const uint16_t* from) {
    uint4 v;
    if (width == 8) {
      v = *reinterpret_cast<const uint4*>(from);
    } else {                                                  // a row may end with its last column
      uint32_t w[4] = {};
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < width) w[j >> 1] |= (uint32_t)from[j] << (16 * (j & 1));
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
  };
  float acc[8] = {};
  if (c.addend) {
    const uint4 v = load(c.addend + t * c.addend_ld + col);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = j & 1 ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]);
  }
  for (int j0 = 0; j0 < c.k; j0 += kAhead) {
    uint4 v[kAhead];
    bool there[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      there[j] = false;
      if (j0 + j < c.k) {
        const int p = c.positions[t * c.k + j0 + j];
        there[j] = p >= 0 && p < c.rows;
        if (there[j]) v[j] = load(c.y + (int64_t)p * c.y_ld + col);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (!there[j]) continue;
      const float weight = c.weights[t * c.k + j0 + j];
      const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = fmaf(weight, i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]), acc[i]);
    }
  }
  uint32_t o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = pack_bf16(acc[2 * j], acc[2 * j + 1]);
  uint16_t* to = c.out + t * c.out_ld + col;
  if (width == 8) {
    *reinterpret_cast<uint4*>(to) = make_uint4(o[0], o[1], o[2], o[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < width) to[j] = (uint16_t)(o[j >> 1] >> (16 * (j & 1)));
  }
}

// Workgroups of the two launches: every one of the second sums up what all of the first counted, so few where few tokens make the first
// short.  256 experts, k 8, binary32, us with at most 64, 128 and 256: 1024 tokens 12.5 12.6 12.5, 4096 18.6 13.6 14.1, 8192 19.1 19.2 15.4;
// 1024 experts 21.3 17.9 20.1, 45.4 32.1 28.6, 50.0 50.2 38.0.
int64_t most_blocks(int64_t tokens) {
  const int64_t some = (tokens + 15) / 16, passes = (tokens + kTile - 1) / kTile, few = some < 64 ? 64 : some < 256 ? some : 256;
  return passes <= few ? few : passes < kMaxBlocks ? passes : kMaxBlocks;
}
// Tokens a workgroup takes: a wave of them on every SIMD (`unit`) at least, so that their steps do not wait for each other's, or whole passes
// (256 tokens, 1024 experts, k 8, binary32: 14 us, 42 with 64 tokens a workgroup).
int tokens_per_block(int64_t tokens, int unit) {
  const int64_t most = most_blocks(tokens), least = (tokens + most - 1) / most;
  const int by = least < kTile ? unit : kTile;
  return (int)((least + by - 1) / by) * by;
}

}  // namespace

size_t moe_route_workspace_bytes(int64_t tokens, int experts) {
  // no less for more tokens: a workspace serves every smaller call
  return align_up((size_t)most_blocks(tokens) * counts_of(experts) * 2, 256) + 256;
}

template <int PER, int LANES>
static int route(const RouteCall& c, uint16_t* hist, hipStream_t st) {
  // One launch for one pass of a workgroup, half of it where a step is long: us with one and two launches, 64 experts, k 8, 64 tokens 5.2 7.1;
  // 256 experts, 32 tokens 8.4 10.1, 64 tokens 12.0 10.2 (bf16 8.0 8.4); 1024 experts, 4 tokens 7.1 10.1, 16 tokens 12.8 11.4
  if (c.tokens <= kRouteThreads / LANES / (PER == 16 && !c.bf16 ? 2 : 1)) {
    if (c.bf16)
      route_few_kernel<PER, true, LANES><<<1, kRouteThreads, 0, st>>>(c);
    else
      route_few_kernel<PER, false, LANES><<<1, kRouteThreads, 0, st>>>(c);
    return check_hip(hipGetLastError(), "route_few_kernel");
  }
  const int per = tokens_per_block(c.tokens, 4 * kWave / LANES), blocks = (int)((c.tokens + per - 1) / per);
  if (c.bf16)
    route_topk_kernel<PER, true, LANES><<<blocks, kRouteThreads, 0, st>>>(c, per, hist);
  else
    route_topk_kernel<PER, false, LANES><<<blocks, kRouteThreads, 0, st>>>(c, per, hist);
  const int rc = check_hip(hipGetLastError(), "route_topk_kernel");
  if (rc) return rc;
  route_place_kernel<<<blocks, kRouteThreads, 0, st>>>(c, per, hist);
  return check_hip(hipGetLastError(), "route_place_kernel");
}

int run_moe_route(RouteCall c, void* ws, hipStream_t st) {
  const int each_load = c.bf16 ? 8 : 4;                       // logits of 16 bytes
  c.wide = c.experts % each_load == 0 && c.ld % each_load == 0 && ((uintptr_t)c.logits & 15) == 0;
  uint16_t* hist = (uint16_t*)ws;
  // Sixteen lanes a token where its experts fit their registers and its k experts the lanes: what a step of the selection costs is shared
  // by four tokens (16381 tokens, 256 experts, k 8: the first launch 10.1 us with one logit a load, with a wave a token 15.8).
  if (c.experts <= 256 && c.k <= 16) {
    return c.experts <= 64 ? route<4, 16>(c, hist, st) : c.experts <= 128 ? route<8, 16>(c, hist, st) : route<16, 16>(c, hist, st);
  }
  const int each = (c.experts + 63) / 64;                     // experts a lane
  return each <= 4 ? route<4, 64>(c, hist, st) : each <= 8 ? route<8, 64>(c, hist, st) : route<16, 64>(c, hist, st);
}

int run_moe_combine(const CombineCall& c, hipStream_t st) {
  if (c.tokens == 0) return PQ_OK;
  const int64_t chunks = ((c.N + 7) / 8 + kCombineThreads - 1) / kCombineThreads;
  // a grid has fewer than 2^32 threads
  if (c.tokens * chunks >= (int64_t)1 << 25)
    return fail(PQ_ERR_SHAPE, "pq_moe_combine: tokens=%lld N=%lld are too many for one call", (long long)c.tokens, (long long)c.N);
  combine_kernel<<<(unsigned)(c.tokens * chunks), kCombineThreads, 0, st>>>(c, (int)chunks);
  return check_hip(hipGetLastError(), "combine_kernel");
}

}  // namespace pq
