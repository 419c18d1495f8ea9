// Attention of one new token a sequence over the paged cache (layout: pq_kv.h), the plain way: a workgroup takes a query head of
// a sequence, its waves the tokens in turn, a lane D / 64 channels; running maximum and sum of the softmax in fp32.
#include "pq_kv.h"
#include "pq_qgemm_common.h"

namespace pq {

KvView kv_view(const pq_kv_cache& c);

namespace {

// the stored key / value of a channel without the tensor scale
template <class L>
__device__ __forceinline__ float kv_key(const uint8_t* block, int t, int ch) {
  const uint8_t* at = block + L::k_chunk(t, ch / 8);
  if constexpr (L::FMT == kBf16) return bf16_to_f32(reinterpret_cast<const uint16_t*>(at)[ch % 8]);
  else {
    const uint32_t code = *reinterpret_cast<const uint32_t*>(at) >> (ch % 8 * 4);
    if constexpr (L::FMT == kNvfp4)
      return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code & 15u, 1.0f, 0)[0] * e4m3_decode(block[L::k_byte_at(t, ch / 16)]);
    else
      return (float)((int)(code & 15u) - 8) *
             div_const(bf16_to_f32(*reinterpret_cast<const uint16_t*>(block + L::int_scale_at(t, ch / L::G))), 7.0f, 1.0f / 7.0f);
  }
}
template <class L>
__device__ __forceinline__ float kv_value(const uint8_t* block, int t, int ch) {
  const int n = ch % L::GV / L::PER, j = ch / L::GV * L::PER + ch % L::PER;
  if constexpr (L::FMT == kBf16) return bf16_to_f32(reinterpret_cast<const uint16_t*>(block + L::v_pair(t, n, j / 2))[j % 2]);
  else {
    const uint32_t code = *reinterpret_cast<const uint16_t*>(block + L::v_quad(t, n, j / 4)) >> (j % 4 * 4);
    if constexpr (L::FMT == kNvfp4)
      return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code & 15u, 1.0f, 0)[0] * e4m3_decode(block[L::v_byte_at(t, ch / 16)]);
    else
      return (float)((int)(code & 15u) - 8) *
             div_const(bf16_to_f32(*reinterpret_cast<const uint16_t*>(block + L::v_at + L::int_scale_at(t, ch / L::G))), 7.0f, 1.0f / 7.0f);
  }
}

constexpr float kNoScore = -1e38f;       // a running maximum before the first score

template <class L>
__global__ __launch_bounds__(256) void attn_decode_kernel(KvView cache, AttnCall a) {
  constexpr int D = L::D, C = D / 64;
  __shared__ float part[4][D + 2];
  const int h = blockIdx.x, b = blockIdx.y, head = h / (a.q_heads / cache.heads);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = min(a.lengths[b], a.max_len), first = a.window ? max(0, len - a.window) : 0;
  float c = a.scale;
  if constexpr (L::FMT == kNvfp4) c *= *cache.k_ts;
  float q[C], acc[C] = {}, m = kNoScore, l = 0.0f;
#pragma unroll
  for (int j = 0; j < C; ++j) q[j] = bf16_to_f32(a.q[b * a.q_ld + h * a.q_head + lane * C + j]);
  for (int t = first + wave; t < len; t += 4) {
    const int64_t page = a.table[b * a.table_ld + (t >> cache.page_log2)];
    if (page < 0 || page >= cache.pages) continue;
    const uint8_t* block = kv_block<L>(cache, (page << cache.page_log2) + (t & ((1 << cache.page_log2) - 1)), head);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < C; ++j) s = __builtin_fmaf(q[j], kv_key<L>(block, t & 31, lane * C + j), s);
#pragma unroll
    for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off);
    s *= c;
    const float m2 = fmaxf(m, s), f = __expf(m - m2), p = __expf(s - m2);
    m = m2;
    l = l * f + p;
#pragma unroll
    for (int j = 0; j < C; ++j) acc[j] = acc[j] * f + p * kv_value<L>(block, t & 31, lane * C + j);
  }
#pragma unroll
  for (int j = 0; j < C; ++j) part[wave][lane * C + j] = acc[j];
  if (lane == 0) {
    part[wave][D] = m;
    part[wave][D + 1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float top = kNoScore, total = 0.0f, sum = 0.0f;
  for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w][D]);
  for (int w = 0; w < 4; ++w) {
    const float f = __expf(part[w][D] - top);
    total += part[w][D + 1] * f;
    sum += part[w][threadIdx.x] * f;
  }
  float o = total > 0.0f ? sum / total : 0.0f;
  if constexpr (L::FMT == kNvfp4) o *= *cache.v_ts;
  a.out[b * a.out_ld + h * a.out_head + threadIdx.x] = (uint16_t)cvt_pk_bf16(o, 0.0f);
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)b * a.q_heads + h] = total > 0.0f ? top + logf(total) : -INFINITY;
}

}  // namespace

size_t attn_decode_workspace_bytes(const pq_kv_cache&, int64_t, int, int64_t, int64_t) { return PQ_ATTN_DECODE_ZERO_BYTES; }

int run_attn_decode(const pq_kv_cache& c, const AttnCall& a, hipStream_t st) {
  return kv_dispatch(c.fmt, c.group, c.head_dim, [&](auto l) {
    attn_decode_kernel<decltype(l)><<<dim3(a.q_heads, a.seqs), 256, 0, st>>>(kv_view(c), a);
    return check_hip(hipGetLastError(), "pq_attn_decode");
  });
}

}  // namespace pq
