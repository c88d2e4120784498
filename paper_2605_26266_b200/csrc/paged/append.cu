// kvq_paged_append: rotates the keys of new tokens by their positions, quantizes keys and values to E4M3 under one power of two
// per block (the tokens of a page that a head has) and writes them into their pages.
//
//   y = rope(k) (values: y = v);  a = max |finite y| over the block's new tokens
//   e = the smallest exponent with a <= 448 2^e, not below -64; with earlier tokens in the page, not below theirs
//   code = E4M3(y 2^-e)
//
// The scale is a power of two because E4M3 is a floating format: its relative precision does not depend on where under 448 the
// largest number lies, products with the scale are exact, and where a later token raises a page's scale the codes that are there
// move by whole exponents, without a second rounding (but of those that leave the format's normal range).
//
// One CTA takes one page of one head, keys and values: all of it is read once; the rotated keys (in shared memory) and the values as they came (in registers)
// stay between the maximum and the codes.  So a page's scale needs no second pass, no atomics in global memory and no order among CTAs.
//
// Bound by bytes, 4 d read and 2 d written for a token of a head.  24 heads of 128 channels x 4 680 tokens in pages of 128: 25.9 us with its launch,
// 3.3 TB/s (89 MB at the rate of a plain copy are 13.5 us); 16 requests of up to 700 tokens, 4 heads of 64: 5.3 us; a token of 8 requests: 2.6 us, which
// is a launch and three loads that wait for one another (lengths, table, page).
#include <cuda_fp16.h>

#include "paged.cuh"

namespace kvq {
namespace paged {

namespace {

struct AppendParams {
  Pool pool;
  Seqs seqs;
  Rope rope;
  const uint16_t *k, *v;
  kvq_strides ks, vs;
  int n_tokens;
  int32_t* status;
};

// Exponent of a block whose largest magnitude has these FP32 bits (448 = 1.75 * 2^8).
__device__ __forceinline__ int exponent_of(uint32_t bits) {
  const int x = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
  return max(x, kExpMin);                          // 0 and subnormals: their exponent field is 0, far below
}

// Threads of a block: 64 keys and 64 values each, and a whole warp; 512 threads an SM, whose 128 registers hold a thread's numbers as they come.  24 heads x 4680
// tokens in pages of 128: 25.9 us; 32 numbers of each a thread 26.6 (1 024 threads an SM), 29.7 (512); rotated keys in registers instead of shared
// memory 29.3; 256 threads an SM 33.7.
__host__ __device__ constexpr int threads_of(int d, int page) { return page * d / 64 < 32 ? 32 : page * d / 64; }

template <bool INTERLEAVED>
__device__ __forceinline__ void pack(const float (&x)[16], float f, uint2& a, uint2& b) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 v = __fmul2_rn(INTERLEAVED ? make_float2(x[i], x[8 + i]) : make_float2(x[2 * i], x[2 * i + 1]), make_float2(f, f));
    w[i] = e4m3x2(v.x, v.y);
  }
  a = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
  b = make_uint2(w[4] | w[5] << 16, w[6] | w[7] << 16);
}
template <int D, int PAGE, bool INTERLEAVED>
__global__ void __launch_bounds__(threads_of(D, PAGE), 512 / threads_of(D, PAGE)) paged_append_kernel(const AppendParams p) {
  constexpr int kThreads = threads_of(D, PAGE), kLanes = D / 16, kRows = kThreads / kLanes, kPer = PAGE / kRows;      // lanes of a token; tokens at a time; passes
  extern __shared__ float4 s_key[];                // [pass][quarter][thread]: the rotated keys, each read back by the thread that wrote it
  __shared__ uint32_t s_max[2];
  __shared__ uint8_t s_nan[PAGE];                  // keys or values of this token hold a NaN
  wait_for_previous_grid();
  allow_next_grid();
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const Extent ex = extent_of(p.seqs, PAGE, b, p.n_tokens, p.status);
  const int first = ex.before / PAGE + blockIdx.x;                             // page of the sequence
  const int lo = max(ex.before - first * PAGE, 0), hi = min(ex.before + ex.fresh - first * PAGE, PAGE);      // its new slots
  if (hi <= lo) return;
  const int64_t page = load_coherent(p.seqs.table + (int64_t)b * p.seqs.table_stride + first);
  const int lane = tid % kLanes, r0 = tid / kLanes;
  const int64_t tok0 = (int64_t)first * PAGE - ex.before;                      // new token of slot 0
  // this lane's chunks of a key, and the column of the tables that their rotation begins with
  const bool turn = lane < p.rope.dim >> 4;
  const Chunks mine = chunks_of<INTERLEAVED>(lane, p.rope.dim);
  const int ca = mine.a, cb = mine.b;
  const uint16_t* kp = p.k + (int64_t)b * p.ks.b + (int64_t)h * p.ks.h;
  const uint16_t* vp = p.v + (int64_t)b * p.vs.b + (int64_t)h * p.vs.h + 8 * lane;      // of a value: chunks lane and lane + kLanes
  uint4 ka[kPer], kb[kPer], va[kPer], vb[kPer];
  int row[kPer];                                   // of the rotation's tables
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = r0 + i * kRows;
    ka[i] = kb[i] = va[i] = vb[i] = make_uint4(0, 0, 0, 0);
    row[i] = 0;
    if (slot >= lo && slot < hi) {
      const uint16_t *kt = kp + (tok0 + slot) * p.ks.t, *vt = vp + (tok0 + slot) * p.vs.t;
      ka[i] = *reinterpret_cast<const uint4*>(kt + 8 * ca);
      kb[i] = *reinterpret_cast<const uint4*>(kt + 8 * cb);
      va[i] = *reinterpret_cast<const uint4*>(vt);
      vb[i] = *reinterpret_cast<const uint4*>(vt + 8 * kLanes);
      const int t = (int)(tok0 + slot);
      if (turn) row[i] = p.rope.positions ? load_coherent(p.rope.positions + (int64_t)b * p.rope.positions_stride + t) : ex.before + t;
    }
  }
  if (page < 0 || page >= p.pool.pages) {
    if (tid == 0) report(p.status, kBadPage);
    return;
  }
  if (tid < 2) s_max[tid] = 0;
  bool far = false;                                // a position that the tables do not have
  auto key_at = [&](int i, float (&y)[16]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4 v = s_key[(i * 4 + c) * kThreads + tid];
      y[4 * c] = v.x; y[4 * c + 1] = v.y; y[4 * c + 2] = v.z; y[4 * c + 3] = v.w;
    }
  };
  float top_k = 0.f, top_v = 0.f;
  float2 odd = make_float2(0.f, 0.f);              // a NaN once a number is not finite
  const float2 zero = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    float y[16];
    unpack<INTERLEAVED>(ka[i], kb[i], y);
    const int slot = r0 + i * kRows;
    if (turn && slot >= lo && slot < hi) {
      const int in = min(max(row[i], 0), p.rope.rows - 1);
      far |= in != row[i];
      const int64_t at = (int64_t)in * (p.rope.dim >> 1) + 8 * lane;
      rotate16(y, p.rope.cos + at, p.rope.sin + at);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) s_key[(i * 4 + c) * kThreads + tid] = make_float4(y[4 * c], y[4 * c + 1], y[4 * c + 2], y[4 * c + 3]);
    float x[16];
    unpack<false>(va[i], vb[i], x);
#pragma unroll
    for (int c = 0; c < 16; c += 2) {
      top_k = fmaxf(top_k, fmaxf(fabsf(y[c]), fabsf(y[c + 1])));
      top_v = fmaxf(top_v, fmaxf(fabsf(x[c]), fabsf(x[c + 1])));
      odd = __ffma2_rn(make_float2(y[c], y[c + 1]), zero, odd);
      odd = __ffma2_rn(make_float2(x[c], x[c + 1]), zero, odd);
    }
  }
  if (far) report(p.status, kBadPosition);
  const bool strange = __syncthreads_or(!(odd.x + odd.y == 0.f));
  if (strange) {                                   // infinities do not count, NaN are found token by token
    for (int i = tid; i < PAGE; i += kThreads) s_nan[i] = 0;
    __syncthreads();
    top_k = top_v = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float x[16], y[16];
      unpack<false>(va[i], vb[i], x);
      key_at(i, y);
      bool nan = false;
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        const float a = fabsf(y[c]), w = fabsf(x[c]);
        if (a < INFINITY) top_k = fmaxf(top_k, a);
        if (w < INFINITY) top_v = fmaxf(top_v, w);
        nan |= a != a || w != w;
      }
      if (nan) s_nan[r0 + i * kRows] = 1;
    }
  }
  const uint32_t tk = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_k)), tv = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_v));
  if ((tid & 31) == 0) {
    atomicMax(&s_max[0], tk);
    atomicMax(&s_max[1], tv);
  }
  const int64_t block = page * p.pool.kv_heads + h;
  const int old_k = lo > 0 ? min((int)load_coherent(p.pool.k_scale + block) - kExpBias, 126) : kExpMin;      // 126: of a byte that no append wrote
  const int old_v = lo > 0 ? min((int)load_coherent(p.pool.v_scale + block) - kExpBias, 126) : kExpMin;
  __syncthreads();
  const int new_k = exponent_of(s_max[0]), new_v = exponent_of(s_max[1]);
  uint8_t *kc = p.pool.k_codes + block * (PAGE * D), *vc = p.pool.v_codes + block * (PAGE * D);
  if (lo > 0) {                                    // the page holds earlier tokens: they keep their scale or move to a larger one
    auto move = [&](uint8_t* codes, int by) {
      const float f = pow2(max(-by, -126));
      for (int i = tid; i < lo * (D / 8); i += kThreads) {
        uint2* at = reinterpret_cast<uint2*>(codes) + i;
        const uint2 w = *at;
        uint32_t o[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t u = c ? w.y : w.x;
          const float2 a = e4m3x2_to_f32(u & 0xFFFFu), q = e4m3x2_to_f32(u >> 16);
          o[c] = e4m3x2(a.x * f, a.y * f) | e4m3x2(q.x * f, q.y * f) << 16;
        }
        *at = make_uint2(o[0], o[1]);
      }
    };
    if (new_k > old_k) move(kc, new_k - old_k);
    if (new_v > old_v) move(vc, new_v - old_v);
  }
  const int e_k = max(new_k, old_k), e_v = max(new_v, old_v);
  if (tid == 0) { p.pool.k_scale[block] = (uint8_t)(e_k + kExpBias); p.pool.v_scale[block] = (uint8_t)(e_v + kExpBias); }
  const float f_k = pow2(-e_k), f_v = pow2(-e_v);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = r0 + i * kRows;
    if (slot < lo || slot >= hi) continue;
    float x[16];
    unpack<false>(va[i], vb[i], x);
    // A NaN in a token's keys or values becomes NaN keys and no NaN value: a weight of 0 times a NaN value would reach rows that do not see the token.
    const bool nan = strange && s_nan[slot];
    if (nan) {
#pragma unroll
      for (int c = 0; c < 16; ++c) x[c] = x[c] == x[c] ? x[c] : 0.f;
    }
    uint2 a, c;
    pack<false>(x, f_v, a, c);
    *reinterpret_cast<uint2*>(vc + slot * D + 8 * lane) = a;
    *reinterpret_cast<uint2*>(vc + slot * D + 8 * (lane + kLanes)) = c;
    float y[16];
    key_at(i, y);
    pack<INTERLEAVED>(y, f_k, a, c);
    if (nan) a = c = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
    *reinterpret_cast<uint2*>(kc + slot * D + 8 * ca) = a;
    *reinterpret_cast<uint2*>(kc + slot * D + 8 * cb) = c;
  }
}

template <int D, int PAGE>
int launch(const AppendCall& c, const AppendParams& p) {
  const int64_t blocks = (c.n_tokens + PAGE - 2) / PAGE + 1;       // pages that n_tokens can touch
  const dim3 grid((unsigned)blocks, (unsigned)c.pool.kv_heads, (unsigned)c.seqs.batch);
  const auto kernel = p.rope.interleaved ? paged_append_kernel<D, PAGE, true> : paged_append_kernel<D, PAGE, false>;
  constexpr size_t smem = (size_t)PAGE * D * sizeof(float);
  if (smem > 48 * 1024) {
    static PerDevice set[2];
    int dev = 0;
    const int r = current_device(&dev);
    if (r != KVQ_OK) return r;
    if (set[p.rope.interleaved].first(dev)) {
      KVQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
      set[p.rope.interleaved].done(dev);
    }
  }
  return launch_after(true, 1, grid, dim3(threads_of(D, PAGE)), smem, c.stream, kernel, p);
}

}  // namespace

int launch_append(const AppendCall& c) {
  AppendParams p;
  p.pool = c.pool; p.seqs = c.seqs; p.rope = c.rope;
  p.k = static_cast<const uint16_t*>(c.k); p.v = static_cast<const uint16_t*>(c.v);
  p.ks = c.ks; p.vs = c.vs; p.n_tokens = (int)c.n_tokens; p.status = c.status;
  if (c.head_dim == 64) {
    switch (c.pool.page) {
      case 16: return launch<64, 16>(c, p);
      case 32: return launch<64, 32>(c, p);
      case 64: return launch<64, 64>(c, p);
      default: return launch<64, 128>(c, p);
    }
  }
  switch (c.pool.page) {
    case 16: return launch<128, 16>(c, p);
    case 32: return launch<128, 32>(c, p);
    case 64: return launch<128, 64>(c, p);
    default: return launch<128, 128>(c, p);
  }
}

}  // namespace paged
}  // namespace kvq
