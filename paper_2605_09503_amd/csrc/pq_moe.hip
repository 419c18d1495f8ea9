// What stands around the experts' products: routing (the largest of the router's logits, their softmax weights, and the order of
// the rows by expert) and the weighted sum of the rows that the experts made.
#include "pq_host.h"
#include "pq_mx.h"

namespace pq {

namespace {

constexpr int kTile = 64;                                     // tokens a pass of a workgroup: a bit each of a 64-bit mask
constexpr int kRouteWaves = 16;
constexpr int kMaxBlocks = 512;                               // workgroups; more tokens mean more passes of each

__device__ __forceinline__ float logit_at(const RouteCall& c, int64_t t, int e) {
  return c.bf16 ? bf16_to_f32(((const uint16_t*)c.logits)[t * c.ld + e]) : ((const float*)c.logits)[t * c.ld + e];
}

template <class Op>
__device__ __forceinline__ float wave_reduce(float v, Op op) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v = op(v, __shfl_xor(v, d, kWave));
  return v;
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v = min(v, __shfl_xor(v, d, kWave));
  return v;
}

// A wave a token.  The k largest one after another: the largest value over the wave, then the lowest index that holds it.
// PER: experts a lane, lane + 64 i.
template <int PER>
__global__ __launch_bounds__(kRouteWaves* kWave) void route_topk_kernel(const RouteCall c, int per_block, uint16_t* __restrict__ hist) {
  extern __shared__ uint32_t count[];                         // [experts]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < c.experts; e += blockDim.x) count[e] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * per_block, end = min(first + per_block, c.tokens);
  for (int64_t t = first + wave; t < end; t += kRouteWaves) {
    float v[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane + 64 * i;
      v[i] = e < c.experts ? logit_at(c, t, e) : -INFINITY;
      if (!(v[i] > -INFINITY)) v[i] = -INFINITY;              // NaN too: never chosen
    }
    float top = -INFINITY, total = 0.0f;
    float kept = -INFINITY;                                   // lane j: the j-th largest
    int kept_id = -1;
    for (int j = 0; j < c.k; ++j) {
      float best = v[0];
#pragma unroll
      for (int i = 1; i < PER; ++i) best = fmaxf(best, v[i]);
      const float max = wave_reduce(best, [](float a, float b) { return fmaxf(a, b); });
      if (j == 0) {
        top = max;
        if (!c.renormalize) {
          float part = 0.0f;
#pragma unroll
          for (int i = 0; i < PER; ++i) part += v[i] > -INFINITY ? expf(v[i] - top) : 0.0f;
          total = wave_reduce(part, [](float a, float b) { return a + b; });
        }
      }
      if (max == -INFINITY) break;                            // uniform: none left
      int at = 0x7FFFFFFF;
#pragma unroll
      for (int i = PER - 1; i >= 0; --i)
        if (v[i] == max) at = lane + 64 * i;
      const int id = wave_min(at);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane + 64 * i == id) v[i] = -INFINITY;
      if (lane == j) kept = max, kept_id = id;
    }
    const float p = kept_id >= 0 ? expf(kept - top) : 0.0f;
    if (c.renormalize) total = wave_reduce(p, [](float a, float b) { return a + b; });
    if (lane < c.k) {
      c.ids[t * c.k + lane] = kept_id;
      c.weights[t * c.k + lane] = kept_id >= 0 ? p / total : 0.0f;
      if (kept_id >= 0) atomicAdd(&count[kept_id], 1u);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < c.experts; e += blockDim.x) hist[(int64_t)blockIdx.x * c.experts + e] = (uint16_t)count[e];
}

// Places of the rows: the experts' offsets, then the rows of earlier workgroups, then the earlier tokens of this one.
__global__ __launch_bounds__(kRouteWaves* kWave) void route_place_kernel(const RouteCall c, int per_block, const uint16_t* __restrict__ hist) {
  extern __shared__ uint64_t lds[];
  uint64_t* mask = lds;                                       // [experts]: tokens of the pass that chose it
  int32_t* base = (int32_t*)(lds + c.experts);                // [experts]: place of the next row
  int32_t* total = base + c.experts;                          // [experts]
  for (int e = threadIdx.x; e < c.experts; e += blockDim.x) {
    int before = 0, all = 0;
    for (int b = 0; b < (int)gridDim.x; ++b) {
      const int n = hist[(int64_t)b * c.experts + e];
      if (b < (int)blockIdx.x) before += n;
      all += n;
    }
    base[e] = before;
    total[e] = all;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int at = 0;
    for (int e = 0; e < c.experts; ++e) {
      base[e] += at;
      if (blockIdx.x == 0) c.offsets[e] = at;
      at += total[e];
    }
    total[0] = at;
    if (blockIdx.x == 0) c.offsets[c.experts] = at;
  }
  __syncthreads();
  const int64_t pairs = c.tokens * c.k;
  for (int64_t i = total[0] + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pairs; i += (int64_t)gridDim.x * blockDim.x) c.rows[i] = -1;
  const int64_t first = (int64_t)blockIdx.x * per_block, end = min(first + per_block, c.tokens);
  for (int64_t t0 = first; t0 < end; t0 += kTile) {
    const int n = (int)min((int64_t)kTile, end - t0) * c.k;
    for (int e = threadIdx.x; e < c.experts; e += blockDim.x) mask[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const int id = c.ids[t0 * c.k + i];
      if (id >= 0) atomicOr((unsigned long long*)&mask[id], 1ull << (i / c.k));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const int id = c.ids[t0 * c.k + i], t = i / c.k;
      int place = -1;
      if (id >= 0) {
        place = base[id] + __popcll(mask[id] & ((1ull << t) - 1));
        c.rows[place] = (int32_t)(t0 + t);
      }
      c.positions[t0 * c.k + i] = place;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < c.experts; e += blockDim.x) base[e] += __popcll(mask[e]);
    __syncthreads();
  }
}

// out[t] = addend[t] + sum_j weights[t, j] * y[positions[t, j]], j ascending, in binary32, rounded once to bf16.  Eight columns a thread.
__global__ __launch_bounds__(256) void combine_kernel(const CombineCall c) {
  const int64_t across = (c.N + 7) / 8, n = c.tokens * across;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / across, col = (i - t * across) * 8;
    const int width = (int)min((int64_t)8, c.N - col);
    float acc[8] = {};
    const auto add = [&](const uint16_t* from, float w, bool weighted) {
      uint16_t v[8] = {};
      if (width == 8)
        *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(from);
      else
        for (int j = 0; j < width; ++j) v[j] = from[j];
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = weighted ? fmaf(w, bf16_to_f32(v[j]), acc[j]) : bf16_to_f32(v[j]);
    };
    if (c.addend) add(c.addend + t * c.addend_ld + col, 1.0f, false);
    for (int j = 0; j < c.k; ++j) {
      const int64_t p = c.positions[t * c.k + j];
      if (p >= 0 && p < c.rows) add(c.y + p * c.y_ld + col, c.weights[t * c.k + j], true);
    }
    uint16_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = __builtin_bit_cast(uint16_t, (__bf16)acc[j]);
    uint16_t* to = c.out + t * c.out_ld + col;
    if (width == 8)
      *reinterpret_cast<uint4*>(to) = *reinterpret_cast<uint4*>(o);
    else
      for (int j = 0; j < width; ++j) to[j] = o[j];
  }
}

// tokens a workgroup takes: whole passes, so few workgroups that each can sum up what the others counted
int tokens_per_block(int64_t tokens) { return (int)((tokens + (int64_t)kTile * kMaxBlocks - 1) / ((int64_t)kTile * kMaxBlocks)) * kTile; }

}  // namespace

size_t moe_route_workspace_bytes(int64_t tokens, int experts) {
  const int64_t per = tokens ? tokens_per_block(tokens) : 1, blocks = (tokens + per - 1) / per;
  return align_up((size_t)blocks * experts * 2, 256) + 256;
}

int run_moe_route(const RouteCall& c, void* ws, hipStream_t st) {
  // without tokens one workgroup still writes the offsets
  const int per = c.tokens ? tokens_per_block(c.tokens) : kTile;
  const int blocks = c.tokens ? (int)((c.tokens + per - 1) / per) : 1;
  const size_t lds = (size_t)c.experts * 4;
  uint16_t* hist = (uint16_t*)ws;
  const int each = (c.experts + 63) / 64;
  const auto topk = each <= 1 ? route_topk_kernel<1> : each <= 2 ? route_topk_kernel<2> : each <= 4 ? route_topk_kernel<4> : each <= 8 ? route_topk_kernel<8> : route_topk_kernel<16>;
  topk<<<blocks, kRouteWaves * kWave, lds, st>>>(c, per, hist);
  int rc = check_hip(hipGetLastError(), "route_topk_kernel");
  if (rc) return rc;
  route_place_kernel<<<blocks, kRouteWaves * kWave, (size_t)c.experts * 16, st>>>(c, per, hist);
  return check_hip(hipGetLastError(), "route_place_kernel");
}

int run_moe_combine(const CombineCall& c, hipStream_t st) {
  if (c.tokens == 0) return PQ_OK;
  const int64_t blocks = (c.tokens * ((c.N + 7) / 8) + 255) / 256;
  combine_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(c);
  return check_hip(hipGetLastError(), "combine_kernel");
}

}  // namespace pq
