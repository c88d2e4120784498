// kvq_paged_attn: attention of new tokens over the pages of their sequences.
//
//   s_j = softmax_scale * rope(q) . k_j,  k_j = code * 2^e(page, head);  out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)
//
// One warp takes one query row: 32 keys at a time, a key a lane, then the weights' sum of values with four channels (two of heads of 64) a lane.
#include <cuda_fp16.h>

#include "paged.cuh"

namespace kvq {
namespace paged {

namespace {

struct AttnParams {
  Pool pool;
  Seqs seqs;
  Rope rope;
  const uint16_t* q; kvq_strides qs;
  uint16_t* out; kvq_strides os;
  int q_heads, group, m_tokens;
  float scale;
  bool causal;
  int window;
  float* lse;
  int32_t* status;
};

constexpr int kWarps = 8;

template <int D>
__global__ void __launch_bounds__(kWarps * 32) paged_attn_kernel(const AttnParams p) {
  __shared__ __align__(16) float s_q[kWarps][D];
  wait_for_previous_grid();
  allow_next_grid();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.z, h = blockIdx.y, t = blockIdx.x * kWarps + warp;
  if (t >= p.m_tokens) return;
  const int page = p.pool.page, kvh = h / p.group;
  const Extent ex = extent_of(p.seqs, page, b, p.m_tokens, p.status);
  constexpr int C = D / 32;                        // channels of a lane
  float o[C] = {};
  float m = -INFINITY, l = 0.f;
  if (t < ex.fresh) {
    {
      float x[8] = {};
      const int j = lane & (D / 8 - 1);
      bf16x8_to_f32(*reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.qs.b + (int64_t)h * p.qs.h + (int64_t)t * p.qs.t + 8 * j), x);
      if (p.rope.dim) {
        const int64_t at = (int64_t)rope_row(p.rope, b, t, ex.before, p.status) * (p.rope.dim >> 1);
        rotate8(x, p.rope.cos + at, p.rope.sin + at, p.rope, j);
      }
      if (lane < D / 8)
        for (int i = 0; i < 8; ++i) s_q[warp][8 * j + i] = x[i];
      __syncwarp();
    }
    const int total = ex.before + ex.fresh, pos = ex.before + t;
    const int end = p.causal ? min(pos + 1, total) : total;
    const int begin = p.window ? max(pos + 1 - p.window, 0) : 0;
    const int32_t* table = p.seqs.table + (int64_t)b * p.seqs.table_stride;
    for (int j0 = begin; j0 < end; j0 += 32) {
      const int j = j0 + lane;
      float s = -INFINITY;
      int64_t block = -1;
      if (j < end) {
        const int64_t id = load_coherent(table + j / page);
        if (id < 0 || id >= p.pool.pages) report(p.status, kBadPage);
        else block = id * p.pool.kv_heads + kvh;
      }
      if (block >= 0) {
        const uint4* k = reinterpret_cast<const uint4*>(p.pool.k_codes + (block * page + (j & (page - 1))) * D);
        float dot = 0.f;
        for (int c = 0; c < D / 16; ++c) {
          const uint4 w = k[c];
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
          for (int i = 0; i < 4; ++i) {
            const float2 a = e4m3x2_to_f32(u[i] & 0xFFFFu), g = e4m3x2_to_f32(u[i] >> 16);
            const float4 q = *reinterpret_cast<const float4*>(&s_q[warp][16 * c + 4 * i]);
            dot += a.x * q.x + a.y * q.y + g.x * q.z + g.y * q.w;
          }
        }
        s = dot * pow2(max((int)load_coherent(p.pool.k_scale + block) - kExpBias, -126)) * p.scale;
      }
      float mx = s;
      for (int i = 16; i; i >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, i));
      const float m_new = fmaxf(m, mx);
      if (m_new == -INFINITY && !__any_sync(0xFFFFFFFFu, s != s)) continue;
      const float f = expf(m - no_key_yet(m_new)), w = expf(s - no_key_yet(m_new));
      m = m_new;
      float sum = w;
      for (int i = 16; i; i >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, i);
      l = l * f + sum;
      for (int c = 0; c < C; ++c) o[c] *= f;
      const float vs = block >= 0 ? pow2(max((int)load_coherent(p.pool.v_scale + block) - kExpBias, -126)) : 0.f;
      for (int i = 0; i < 32; ++i) {
        const int64_t blk = __shfl_sync(0xFFFFFFFFu, block, i);
        const float wi = __shfl_sync(0xFFFFFFFFu, w, i) * __shfl_sync(0xFFFFFFFFu, vs, i);
        if (blk < 0) continue;
        const uint8_t* v = p.pool.v_codes + (blk * page + ((j0 + i) & (page - 1))) * D + C * lane;
        for (int c = 0; c < C; c += 2) {
          const float2 a = e4m3x2_to_f32(*reinterpret_cast<const uint16_t*>(v + c));
          o[c] += wi * a.x; o[c + 1] += wi * a.y;
        }
      }
    }
  }
  uint16_t* out = p.out + (int64_t)b * p.os.b + (int64_t)h * p.os.h + (int64_t)t * p.os.t + C * lane;
  for (int c = 0; c < C; ++c) out[c] = (uint16_t)f32_to_bf16_bits(l == 0.f ? 0.f : o[c] / l);
  if (p.lse && lane == 0) p.lse[((int64_t)b * p.q_heads + h) * p.m_tokens + t] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

int launch_attn(const AttnCall& c) {
  if (few_supports(c.head_dim, c.group, c.m_tokens)) return launch_attn_few(c);
  return launch_attn_chunk(c);
  AttnParams p;
  p.pool = c.pool; p.seqs = c.seqs; p.rope = c.rope;
  p.q = static_cast<const uint16_t*>(c.q); p.qs = c.qs;
  p.out = static_cast<uint16_t*>(c.out); p.os = c.os;
  p.q_heads = c.q_heads; p.group = c.group; p.m_tokens = (int)c.m_tokens;
  p.scale = c.softmax_scale; p.causal = c.causal; p.window = (int)c.window; p.lse = c.lse; p.status = c.status;
  const dim3 grid((unsigned)((c.m_tokens + kWarps - 1) / kWarps), (unsigned)c.q_heads, (unsigned)c.seqs.batch);
  if (c.head_dim == 64) return launch_after(true, 1, grid, dim3(kWarps * 32), 0, c.stream, paged_attn_kernel<64>, p);
  return launch_after(true, 1, grid, dim3(kWarps * 32), 0, c.stream, paged_attn_kernel<128>, p);
}

}  // namespace paged
}  // namespace kvq
