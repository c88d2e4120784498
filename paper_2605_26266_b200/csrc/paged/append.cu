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
// One CTA takes one page of one head: half of its threads the keys, half the values, 64 numbers a thread, read once and held in
// registers between the maximum and the codes.  So a page's scale needs no second pass, no atomics and no order among CTAs.
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

// Threads of the keys, and of the values, of a block: 64 numbers each, and whole warps.
__host__ __device__ constexpr int side_threads(int d, int page) { return page * d / 64 < 32 ? 32 : page * d / 64; }

template <int D, int PAGE>
__global__ void __launch_bounds__(2 * side_threads(D, PAGE)) paged_append_kernel(const AppendParams p) {
  constexpr int kSide = side_threads(D, PAGE);
  constexpr int kLanes = D / 8, kRows = kSide / kLanes, kPer = PAGE / kRows;      // lanes of a token; tokens at a time; passes
  __shared__ uint32_t s_max[2];
  __shared__ uint8_t s_nan[PAGE];                  // values of this token hold a NaN
  wait_for_previous_grid();
  allow_next_grid();
  const int b = blockIdx.z, h = blockIdx.y;
  const Extent ex = extent_of(p.seqs, PAGE, b, p.n_tokens, p.status);
  const int first = ex.before / PAGE + blockIdx.x;                             // page of the sequence
  const int lo = max(ex.before - first * PAGE, 0), hi = min(ex.before + ex.fresh - first * PAGE, PAGE);      // its new slots
  if (hi <= lo) return;
  const int64_t page = load_coherent(p.seqs.table + (int64_t)b * p.seqs.table_stride + first);
  if (page < 0 || page >= p.pool.pages) {
    if (threadIdx.x == 0) report(p.status, kBadPage);
    return;
  }
  const int side = threadIdx.x / kSide, t = threadIdx.x % kSide;               // 0: keys, 1: values
  const int j = t % kLanes, r0 = t / kLanes;
  const kvq_strides st = side ? p.vs : p.ks;
  const uint16_t* src = (side ? p.v : p.k) + (int64_t)b * st.b + (int64_t)h * st.h + 8 * j;
  const int64_t tok0 = (int64_t)first * PAGE - ex.before;                      // new token of slot 0
  uint4 raw[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = r0 + i * kRows;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (slot >= lo && slot < hi) raw[i] = *reinterpret_cast<const uint4*>(src + (tok0 + slot) * st.t);
  }
  if (threadIdx.x < 2) s_max[threadIdx.x] = 0;
  if (threadIdx.x < PAGE) s_nan[threadIdx.x] = 0;
  __syncthreads();

  const bool turn = side == 0 && p.rope.dim > 0;                               // the same for a whole warp
  auto numbers = [&](int i, float (&x)[8]) {
    bf16x8_to_f32(raw[i], x);
    if (turn) {
      const int slot = min(max(r0 + i * kRows, lo), hi - 1);
      const int64_t row = rope_row(p.rope, b, (int)(tok0 + slot), ex.before, p.status);
      const int64_t at = row * (p.rope.dim >> 1);
      rotate8(x, p.rope.cos + at, p.rope.sin + at, p.rope, j);
    }
  };
  uint32_t top = 0;                                // largest finite magnitude, as its bits
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = r0 + i * kRows;
    float x[8];
    numbers(i, x);
    bool nan = false;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t u = __float_as_uint(x[c]) & 0x7FFFFFFFu;
      if (u < 0x7F800000u && slot >= lo && slot < hi) top = max(top, u);
      nan |= u > 0x7F800000u;
    }
    if (nan && slot >= lo && slot < hi) s_nan[slot] = 1;
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if ((threadIdx.x & 31) == 0 && top) atomicMax(&s_max[side], top);
  __syncthreads();

  uint8_t* codes = (side ? p.pool.v_codes : p.pool.k_codes) + (page * p.pool.kv_heads + h) * (int64_t)(PAGE * D);
  uint8_t* scale = (side ? p.pool.v_scale : p.pool.k_scale) + page * p.pool.kv_heads + h;
  int e = exponent_of(s_max[side]);
  if (lo > 0) {                                    // the page holds earlier tokens: they keep their scale or move to a larger one
    const int old = min((int)load_coherent(scale) - kExpBias, 126);      // of a byte that no append wrote
    if (e > old) {
      const float f = pow2(max(old - e, -126));
      for (int i = t; i < lo * (D / 8); i += kSide) {
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
    }
    e = max(e, old);
  }
  __syncthreads();                                 // every thread has read the old scale
  if (t == 0) *scale = (uint8_t)(e + kExpBias);
  const float f = pow2(-e);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = r0 + i * kRows;
    float x[8];
    numbers(i, x);
    if (slot < lo || slot >= hi) continue;
    uint32_t w[2];
    // A NaN in a token's keys or values becomes NaN keys and no NaN value: a weight of 0 times a NaN value would reach rows that do not see the token.
    const bool nan = s_nan[slot];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (nan && side == 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[4 * c + k] = x[4 * c + k] == x[4 * c + k] ? x[4 * c + k] : 0.f;
      }
      w[c] = e4m3x2(x[4 * c] * f, x[4 * c + 1] * f) | e4m3x2(x[4 * c + 2] * f, x[4 * c + 3] * f) << 16;
    }
    if (nan && side == 0) w[0] = w[1] = 0x7F7F7F7Fu;
    *reinterpret_cast<uint2*>(codes + slot * D + 8 * j) = make_uint2(w[0], w[1]);
  }
}

template <int D, int PAGE>
int launch(const AppendCall& c, const AppendParams& p) {
  const int64_t blocks = (c.n_tokens + PAGE - 2) / PAGE + 1;       // pages that n_tokens can touch
  const dim3 grid((unsigned)blocks, (unsigned)c.pool.kv_heads, (unsigned)c.seqs.batch);
  return launch_after(true, 1, grid, dim3(2 * side_threads(D, PAGE)), 0, c.stream, paged_append_kernel<D, PAGE>, p);
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
