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
// A block is one page of one head, keys and values: all of it is read once; the rotated keys and the values as they came stay in shared memory
// between the maximum and the codes.  So a page's scale needs no second pass, no atomics in global memory and no order among CTAs.
//
// Few blocks have a CTA each, with its rows in registers.  Of many, a CTA takes a run, the heads of a page one after the other.  Their rotation is the same: its
// tables' rows, as many bytes of L2 as keys and values together, are read once a page and stay in registers; and the next block's rows are on their way to
// shared memory while one is worked on.
//
// Bound by bytes, 4 d read and 2 d written for a token of a head.  24 heads of 128 channels x 4 680 tokens in pages of 128: 23.6 us with its launch, 3.7 TB/s
// (89 MB at the rate of a plain copy are 13.5 us; a CTA has 6 or 7 blocks, so five in six wait at the end).  A CTA each: 25.7; blocks that stride over the grid,
// tables read for each: 29.9.  16 requests of up to 700 tokens, 4 heads of 64: 4.1 us; a token of 8 requests: 2.5 us, which is a launch and three loads that
// wait for one another (lengths, table, page).
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
  int blocks;                      // pages that a sequence's new tokens can touch
  int exact;                       // the cut goes by those that they do touch
  int32_t* status;
};

// Exponent of a block whose largest magnitude has these FP32 bits (448 = 1.75 * 2^8).
__device__ __forceinline__ int exponent_of(uint32_t bits) {
  const int x = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
  return max(x, kExpMin);                          // 0 and subnormals: their exponent field is 0, far below
}

// The largest magnitude of `top` and y; a NaN once there is one.
__device__ __forceinline__ float top_of(float top, const float (&y)[16]) {
#pragma unroll
  for (int c = 0; c < 16; c += 2) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(top) : "f"(top), "f"(y[c]), "f"(y[c + 1]));
  return top;
}
// The same of BF16 pairs, each half by itself; signs are left over, magnitude() takes them and the halves' larger one.
__device__ __forceinline__ uint32_t top_of(uint32_t top, const uint4& a, const uint4& b) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int c = 0; c < 8; ++c) asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(top) : "r"(top), "r"(w[c]));
  return top;
}
__device__ __forceinline__ uint32_t magnitude(uint32_t top) { return max(top << 16 & 0x7FFF0000u, top & 0x7FFF0000u); }

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
// The largest magnitudes of a block's keys and values, of those of its threads.  `place`: two words a warp.
template <int THREADS>
__device__ __forceinline__ void top_of_block(uint32_t k, uint32_t v, uint32_t (*place)[THREADS / 32], uint32_t (&top)[2]) {
  k = __reduce_max_sync(0xFFFFFFFFu, k);
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  if ((threadIdx.x & 31) == 0) { place[0][threadIdx.x >> 5] = k; place[1][threadIdx.x >> 5] = v; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    top[i] = place[i][0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) top[i] = max(top[i], place[i][w]);
  }
}

// What a thread has of a block: pass i is slot r0 + i * kRows, this lane's two chunks of its key and of its value.  key(i, y) and value(i, x) bring them back.
template <int D, int PAGE, int THREADS, bool INTERLEAVED>
struct Mine {
  static constexpr int kLanes = D / 16, kRows = THREADS / kLanes, kPer = PAGE / kRows;      // lanes of a token; tokens at a time; passes
  int lane, r0, ca, cb;            // ca, cb: chunks of a key
  bool turn;                       // the rotation has them
  __device__ __forceinline__ Mine(const Rope& rope) : lane(threadIdx.x % kLanes), r0(threadIdx.x / kLanes), turn(lane < rope.dim >> 4) {
    const Chunks c = chunks_of<INTERLEAVED>(lane, rope.dim);
    ca = c.a; cb = c.b;
  }
  __device__ __forceinline__ int slot(int i) const { return r0 + i * kRows; }

  // Scale, and codes of the slots [lo, hi).  Every thread's old_k and old_v were read before a barrier that lies before this.
  template <class KEY, class VALUE>
  __device__ __forceinline__ void write(const AppendParams& p, int64_t block, int lo, int hi, uint32_t (&top)[2], uint32_t (*place)[THREADS / 32], uint8_t* s_nan,
                                        int old_k, int old_v, KEY key, VALUE value) const {
    const bool strange = max(top[0], top[1]) >= 0x7F800000u;
    if (strange) {                                 // infinities do not count, NaN are found token by token
      for (int i = threadIdx.x; i < PAGE; i += THREADS) s_nan[i] = 0;
      __syncthreads();
      float top_k = 0.f, top_v = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (slot(i) < lo || slot(i) >= hi) continue;
        float x[16], y[16];
        value(i, x);
        key(i, y);
        bool nan = false;
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const float a = fabsf(y[c]), w = fabsf(x[c]);
          if (a < INFINITY) top_k = fmaxf(top_k, a);
          if (w < INFINITY) top_v = fmaxf(top_v, w);
          nan |= a != a || w != w;
        }
        if (nan) s_nan[slot(i)] = 1;
      }
      top_of_block<THREADS>(__float_as_uint(top_k), __float_as_uint(top_v), place, top);
    }
    const int new_k = exponent_of(top[0]), new_v = exponent_of(top[1]);
    uint8_t *kc = p.pool.k_codes + block * (PAGE * D), *vc = p.pool.v_codes + block * (PAGE * D);
    if (lo > 0) {                                  // the page holds earlier tokens: they keep their scale or move to a larger one
      auto move = [&](uint8_t* codes, int by) {
        const float f = pow2(max(-by, -126));
        for (int i = threadIdx.x; i < lo * (D / 8); i += THREADS) {
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
    if (threadIdx.x == 0) { p.pool.k_scale[block] = (uint8_t)(e_k + kExpBias); p.pool.v_scale[block] = (uint8_t)(e_v + kExpBias); }
    const float f_k = pow2(-e_k), f_v = pow2(-e_v);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (slot(i) < lo || slot(i) >= hi) continue;
      float x[16];
      value(i, x);
      // A NaN in a token's keys or values becomes NaN keys and no NaN value: a weight of 0 times a NaN value would reach rows that do not see the token.
      const bool nan = strange && s_nan[slot(i)];
      if (nan) {
#pragma unroll
        for (int c = 0; c < 16; ++c) x[c] = x[c] == x[c] ? x[c] : 0.f;
      }
      uint2 a, c;
      pack<false>(x, f_v, a, c);
      *reinterpret_cast<uint2*>(vc + slot(i) * D + 8 * lane) = a;
      *reinterpret_cast<uint2*>(vc + slot(i) * D + 8 * (lane + kLanes)) = c;
      float y[16];
      key(i, y);
      pack<INTERLEAVED>(y, f_k, a, c);
      if (nan) a = c = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
      *reinterpret_cast<uint2*>(kc + slot(i) * D + 8 * ca) = a;
      *reinterpret_cast<uint2*>(kc + slot(i) * D + 8 * cb) = c;
    }
  }
};

// The scales that a block's page has from earlier tokens.
__device__ __forceinline__ int2 old_scales(const AppendParams& p, int64_t block, int lo) {
  if (lo == 0) return make_int2(kExpMin, kExpMin);
  return make_int2(min((int)load_coherent(p.pool.k_scale + block) - kExpBias, 126), min((int)load_coherent(p.pool.v_scale + block) - kExpBias, 126));      // 126: of a byte that no append wrote
}
__device__ __forceinline__ float4 quarter(const float (&y)[16], int c) { return make_float4(y[4 * c], y[4 * c + 1], y[4 * c + 2], y[4 * c + 3]); }
template <int THREADS>
__device__ __forceinline__ void bring_back(const float4* s_key, int i, float (&y)[16]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float4 v = s_key[(i * 4 + c) * THREADS + threadIdx.x];
    y[4 * c] = v.x; y[4 * c + 1] = v.y; y[4 * c + 2] = v.z; y[4 * c + 3] = v.w;
  }
}

// ---- a CTA for each block ----
// Threads: 64 keys and 64 values each, and a whole warp; 512 an SM, whose 128 registers hold a thread's numbers as they come.
__host__ __device__ constexpr int threads_of(int d, int page) { return page * d / 64 < 32 ? 32 : page * d / 64; }
template <int D, int PAGE, bool INTERLEAVED>
__global__ void __launch_bounds__(threads_of(D, PAGE), 512 / threads_of(D, PAGE)) paged_append_kernel(const AppendParams p) {
  constexpr int kThreads = threads_of(D, PAGE);
  using M = Mine<D, PAGE, kThreads, INTERLEAVED>;
  constexpr int kPer = M::kPer;
  extern __shared__ float4 s_key[];                // [pass][quarter][thread]: the rotated keys, each read back by the thread that wrote it
  __shared__ uint32_t s_top[2][kThreads / 32];     // bits of the largest magnitude that a warp saw
  __shared__ uint8_t s_nan[PAGE];                  // keys or values of this token hold a NaN
  wait_for_previous_grid();
  allow_next_grid();
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const Extent ex = extent_of(p.seqs, PAGE, b, p.n_tokens, p.status);
  const int first = ex.before / PAGE + blockIdx.x;                             // page of the sequence
  const int lo = max(ex.before - first * PAGE, 0), hi = min(ex.before + ex.fresh - first * PAGE, PAGE);      // its new slots
  if (hi <= lo) return;
  const int64_t page = load_coherent(p.seqs.table + (int64_t)b * p.seqs.table_stride + first);
  const M my(p.rope);
  const int64_t tok0 = (int64_t)first * PAGE - ex.before;                      // new token of slot 0
  const uint16_t* kp = p.k + (int64_t)b * p.ks.b + (int64_t)h * p.ks.h;
  const uint16_t* vp = p.v + (int64_t)b * p.vs.b + (int64_t)h * p.vs.h + 8 * my.lane;      // of a value: chunks lane and lane + kLanes
  uint4 ka[kPer], kb[kPer], va[kPer], vb[kPer];
  int row[kPer];                                   // of the rotation's tables
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = my.slot(i);
    ka[i] = kb[i] = va[i] = vb[i] = make_uint4(0, 0, 0, 0);
    row[i] = 0;
    if (slot >= lo && slot < hi) {
      const uint16_t *kt = kp + (tok0 + slot) * p.ks.t, *vt = vp + (tok0 + slot) * p.vs.t;
      ka[i] = *reinterpret_cast<const uint4*>(kt + 8 * my.ca);
      kb[i] = *reinterpret_cast<const uint4*>(kt + 8 * my.cb);
      va[i] = *reinterpret_cast<const uint4*>(vt);
      vb[i] = *reinterpret_cast<const uint4*>(vt + 8 * M::kLanes);
      const int t = (int)(tok0 + slot);
      if (my.turn) row[i] = p.rope.positions ? load_coherent(p.rope.positions + (int64_t)b * p.rope.positions_stride + t) : ex.before + t;
    }
  }
  if (page < 0 || page >= p.pool.pages) {
    if (tid == 0) report(p.status, kBadPage);
    return;
  }
  bool far = false;                                // a position that the tables do not have
  float top_k = 0.f;
  uint32_t top_2 = 0;                              // of values
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    float y[16];
    unpack<INTERLEAVED>(ka[i], kb[i], y);
    const int slot = my.slot(i);
    if (my.turn && slot >= lo && slot < hi) {
      const int in = min(max(row[i], 0), p.rope.rows - 1);
      far |= in != row[i];
      const int64_t at = (int64_t)in * (p.rope.dim >> 1) + 8 * my.lane;
      rotate16(y, p.rope.cos + at, p.rope.sin + at);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) s_key[(i * 4 + c) * kThreads + tid] = quarter(y, c);
    top_k = top_of(top_k, y);
    top_2 = top_of(top_2, va[i], vb[i]);
  }
  if (far) report(p.status, kBadPosition);
  const int64_t block = page * p.pool.kv_heads + h;
  const int2 old = old_scales(p, block, lo);
  uint32_t top[2];
  top_of_block<kThreads>(__float_as_uint(top_k), magnitude(top_2), s_top, top);
  my.write(p, block, lo, hi, top, s_top, s_nan, old.x, old.y, [&](int i, float (&y)[16]) { bring_back<kThreads>(s_key, i, y); },
           [&](int i, float (&x)[16]) { unpack<false>(va[i], vb[i], x); });
}

// ---- a run of blocks for each CTA ----
// Threads: 32 keys and 32 values each; 512 an SM, whose shared memory holds the numbers of two blocks as they come and the rotated keys of one.
__host__ __device__ constexpr int run_threads_of(int d, int page) { return page * d / 32; }
template <int D, int PAGE, bool INTERLEAVED>
__global__ void __launch_bounds__(run_threads_of(D, PAGE), 512 / run_threads_of(D, PAGE)) paged_append_run_kernel(const AppendParams p) {
  constexpr int kThreads = run_threads_of(D, PAGE);
  using M = Mine<D, PAGE, kThreads, INTERLEAVED>;
  constexpr int kPer = M::kPer;
  static_assert(kPer == 2, "half a page at a time");
  // [buffer][pass][two chunks of the key, two of the value][thread], and the rotated keys, [pass][quarter][thread]: each read back by the thread that wrote it
  extern __shared__ uint4 s_raw[];
  float4* s_key = reinterpret_cast<float4*>(s_raw + 2 * kPer * 4 * kThreads);
  __shared__ uint32_t s_top[2][2][kThreads / 32];  // bits of the largest magnitude that a warp saw; every other block's
  __shared__ uint8_t s_nan[PAGE];                  // keys or values of this token hold a NaN
  const int tid = threadIdx.x;
  const M my(p.rope);

  // A block: one page of one head.  What is needed of it before its numbers are there.
  struct Block {
    int x, h, b;                                   // page of the sequence's new ones; head; sequence
    Extent ex;
    int first, lo, hi;                             // page of the sequence, its new slots
    int64_t page;
    int row[kPer];                                 // of the rotation's tables
  };
  // the extent is known; rows go to buffer `buf`
  auto fetch = [&](Block& n, int buf, bool again) {
    n.first = n.ex.before / PAGE + n.x;
    n.lo = max(n.ex.before - n.first * PAGE, 0);
    n.hi = min(n.ex.before + n.ex.fresh - n.first * PAGE, PAGE);
    n.page = -1;
    if (n.hi <= n.lo) return;
    n.page = load_coherent(p.seqs.table + (int64_t)n.b * p.seqs.table_stride + n.first);
    const int64_t tok0 = (int64_t)n.first * PAGE - n.ex.before;                // new token of slot 0
    const uint16_t* kp = p.k + (int64_t)n.b * p.ks.b + (int64_t)n.h * p.ks.h;
    const uint16_t* vp = p.v + (int64_t)n.b * p.vs.b + (int64_t)n.h * p.vs.h + 8 * my.lane;      // of a value: chunks lane and lane + kLanes
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(s_raw + buf * kPer * 4 * kThreads + tid);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = my.slot(i);
      if (!again) n.row[i] = 0;
      if (slot >= n.lo && slot < n.hi) {
        const int t = (int)(tok0 + slot);
        const uint16_t *kt = kp + (int64_t)t * p.ks.t, *vt = vp + (int64_t)t * p.vs.t;
        const uint32_t at = to + i * 4 * kThreads * 16;
        copy16(at, kt + 8 * my.ca);
        copy16(at + kThreads * 16, kt + 8 * my.cb);
        copy16(at + 2 * kThreads * 16, vt);
        copy16(at + 3 * kThreads * 16, vt + 8 * M::kLanes);
        if (my.turn && !again) n.row[i] = p.rope.positions ? load_coherent(p.rope.positions + (int64_t)n.b * p.rope.positions_stride + t) : n.ex.before + t;
      }
    }
  };
  bool far = false;                                // a position that the tables do not have
  float4 cs[kPer][4];                              // of the next block's keys: cosines, sines
  auto fetch_turn = [&](const Block& n) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = my.slot(i);
      if (!my.turn || slot < n.lo || slot >= n.hi) continue;
      const int in = min(max(n.row[i], 0), p.rope.rows - 1);
      far |= in != n.row[i];
      const int64_t at = (int64_t)in * (p.rope.dim >> 1) + 8 * my.lane;
      const float4 *c = reinterpret_cast<const float4*>(p.rope.cos + at), *s = reinterpret_cast<const float4*>(p.rope.sin + at);
      cs[i][0] = c[0]; cs[i][1] = c[1]; cs[i][2] = s[0]; cs[i][3] = s[1];
    }
  };
  wait_for_previous_grid();
  allow_next_grid();
  Block now, next;
  // This CTA's blocks: a piece of the line of all, heads first, then pages, then sequences.
  auto pages_of = [&](const Extent& ex) { return ex.fresh > 0 ? (ex.before + ex.fresh - 1) / PAGE - ex.before / PAGE + 1 : 0; };
  int left;
  if (!p.exact) {
    const long long total = (long long)p.blocks * p.pool.kv_heads * p.seqs.batch, from = total * blockIdx.x / gridDim.x;
    left = (int)(total * (blockIdx.x + 1) / gridDim.x - from);
    now.h = (int)(from % p.pool.kv_heads);
    now.x = (int)(from / p.pool.kv_heads % p.blocks);
    now.b = (int)(from / p.pool.kv_heads / p.blocks);
    now.ex = extent_of(p.seqs, PAGE, now.b, p.n_tokens, p.status);
  } else {
    const int at = tid & 31;
    auto pages_at = [&](int b) { return b < p.seqs.batch ? pages_of(extent_of(p.seqs, PAGE, b, p.n_tokens, p.status)) : 0; };
    long long all = 0;
    for (int b = at; b < p.seqs.batch; b += 32) all += pages_at(b);
    for (int i = 16; i; i >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, i);
    all *= p.pool.kv_heads;
    const long long from = all * blockIdx.x / gridDim.x;
    left = (int)(all * (blockIdx.x + 1) / gridDim.x - from);
    if (left == 0) return;
    long long before = from / p.pool.kv_heads;       // pages
    now.h = (int)(from - before * p.pool.kv_heads);
    now.b = -1;
    for (int b0 = 0; b0 < p.seqs.batch; b0 += 32) {
      const int mine = pages_at(b0 + at);
      long long upto = mine;
      for (int i = 1; i < 32; i <<= 1) {
        const long long o = __shfl_up_sync(0xFFFFFFFFu, upto, i);
        if (at >= i) upto += o;
      }
      const unsigned hit = __ballot_sync(0xFFFFFFFFu, upto > before);
      if (hit) {
        const int src = __ffs(hit) - 1;
        now.x = (int)(before - __shfl_sync(0xFFFFFFFFu, upto - mine, src));
        now.b = b0 + src;
        break;
      }
      before -= __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    if (now.b < 0) return;                           // cannot be: from < all
    now.ex = extent_of(p.seqs, PAGE, now.b, p.n_tokens, p.status);
  }
  fetch(now, 0, false);
  copies_sent();
  fetch_turn(now);
  int turn_of = 0;                                 // of s_top's two places
  for (int n = 0; left > 0; ++n, --left, now = next) {
    // The next block's rows are on their way while this one's are worked on.
    next = now;
    bool more = left > 1, again = true;
    if (++next.h == p.pool.kv_heads) {
      next.h = 0; again = false;
      if (++next.x == (p.exact ? pages_of(next.ex) : p.blocks)) {
        next.x = 0;
        do {                                       // there is another, with new tokens, where there is more
          if (++next.b == p.seqs.batch) { more = false; left = 1; }
          if (more) next.ex = extent_of(p.seqs, PAGE, next.b, p.n_tokens, p.status);
        } while (more && p.exact && next.ex.fresh == 0);
      }
    }
    if (more) fetch(next, (n & 1) ^ 1, again);
    copies_sent();
    copies_landed<1>();
    const int lo = now.lo, hi = now.hi, h = now.h;
    const int64_t page = now.page;
    const bool idle = hi <= lo, bad = !idle && (page < 0 || page >= p.pool.pages);
    if (bad && tid == 0) report(p.status, kBadPage);
    if (idle || bad) {                               // the same for all threads
      if (more && !again) fetch_turn(next);
      continue;
    }
    turn_of ^= 1;
    const uint4* raw = s_raw + (n & 1) * kPer * 4 * kThreads + tid;
    float top_k = 0.f;
    uint32_t top_2 = 0;                              // of values
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = my.slot(i);
      if (slot < lo || slot >= hi) continue;
      float y[16];
      unpack<INTERLEAVED>(raw[i * 4 * kThreads], raw[(i * 4 + 1) * kThreads], y);
      if (my.turn) rotate16(y, reinterpret_cast<const float*>(&cs[i][0]), reinterpret_cast<const float*>(&cs[i][2]));
#pragma unroll
      for (int c = 0; c < 4; ++c) s_key[(i * 4 + c) * kThreads + tid] = quarter(y, c);
      top_k = top_of(top_k, y);
      top_2 = top_of(top_2, raw[(i * 4 + 2) * kThreads], raw[(i * 4 + 3) * kThreads]);
    }
    const int64_t block = page * p.pool.kv_heads + h;
    const int2 old = old_scales(p, block, lo);
    if (more && !again) fetch_turn(next);
    uint32_t top[2];
    top_of_block<kThreads>(__float_as_uint(top_k), magnitude(top_2), s_top[turn_of], top);
    my.write(p, block, lo, hi, top, s_top[turn_of], s_nan, old.x, old.y, [&](int i, float (&y)[16]) { bring_back<kThreads>(s_key, i, y); },
             [&](int i, float (&x)[16]) { unpack<false>(raw[(i * 4 + 2) * kThreads], raw[(i * 4 + 3) * kThreads], x); });
  }
  if (far) report(p.status, kBadPosition);
}

// Runs, where blocks are at least five times as many as run at a time and sequences have new tokens for several pages; of fewer the start of a run and the place in
// the line are not paid for.  A CTA each against runs, us from a graph.  One sequence, 8 heads, blocks 2, 4, 6 and 10 times as many as run at a time: 128
// channels, pages of 128 6.6 / 9.7, 11.8 / 14.8, 20.7 / 20.0, 38.5 / 32.0; 64 channels, pages of 16 7.6 / 7.8, 12.8 / 12.1, 19.0 / 17.4, 32.2 / 30.4.  128
// sequences, 128 channels, pages of 64, each with new tokens of 2, 4 and 8 pages 26.5 / 25.2, 49.6 / 44.0, 89.0 / 75.0; of up to 2, 4 and 8 pages, which has to be
// looked up, 15.5 / 21.0, 28.3 / 30.2, 51.8 / 47.4.  2 048 sequences with a token each 55 / 64 and 56 / 107.
constexpr int kRunRounds = 5, kRunPages = 4, kRunPagesLookedUp = 8;
template <int D, int PAGE>
int launch(const AppendCall& c, const AppendParams& p) {
  AppendParams q = p;
  q.blocks = (int)((c.n_tokens + PAGE - 2) / PAGE + 1);            // pages that n_tokens can touch
  int sms = 0, dev = 0, r = device_sm_count(&sms);
  if (r != KVQ_OK || (r = current_device(&dev)) != KVQ_OK) return r;
  static PerDevice set[2][2];
  const int64_t total = (int64_t)q.blocks * c.pool.kv_heads * c.seqs.batch, at_a_time = (int64_t)sms * (512 / run_threads_of(D, PAGE));
  const bool runs = total >= kRunRounds * at_a_time && c.n_tokens >= (c.seqs.n_new ? kRunPagesLookedUp : kRunPages) * PAGE;
  const auto kernel = runs ? p.rope.interleaved ? paged_append_run_kernel<D, PAGE, true> : paged_append_run_kernel<D, PAGE, false>
                           : p.rope.interleaved ? paged_append_kernel<D, PAGE, true> : paged_append_kernel<D, PAGE, false>;
  // the rotated keys, and of a run the rows of two blocks
  const size_t smem = (size_t)PAGE * D * (runs ? 12 : 4);
  PerDevice& done = set[runs][p.rope.interleaved];
  if (smem > 32 * 1024 && done.first(dev)) {                       // 48 KB are to be had without, with what is static
    KVQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    done.done(dev);
  }
  if (!runs) return launch_after(true, 1, dim3((unsigned)q.blocks, (unsigned)c.pool.kv_heads, (unsigned)c.seqs.batch), dim3(threads_of(D, PAGE)), smem, c.stream, kernel, q);
  q.exact = c.seqs.n_new != nullptr;
  return launch_after(true, 1, dim3((unsigned)at_a_time), dim3(run_threads_of(D, PAGE)), smem, c.stream, kernel, q);
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
