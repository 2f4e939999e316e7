// What the two tensor-core kernels of attention share: their waits and products, the rows
// of a tile, and the way round a product where values are not finite.
#pragma once

#include "cache.cuh"
#include "tc.cuh"

namespace gmc {

constexpr int TM = 128;                 // rows of a tile
constexpr long long T_WAIT = 4000000000LL;
constexpr float GROWN = 8.f;            // powers of two the maximum may fall behind

// Bits 0 .. n - 1 of a word.
__device__ __forceinline__ uint32_t below(int n) {
  return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
}

__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  const long long end = clock64() + T_WAIT;
  while (!tc::mbar_try_wait(bar, parity)) {
    if (*abort || clock64() > end) {
      *abort = 1;
      return false;
    }
  }
  return true;
}

// The issuing warp runs as a whole, so that addresses and descriptors stay in uniform
// registers; the one thread whose `go` is set issues.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t p;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(p));
  return p;
}
// D[tmem] (+)= A[smem] * B[smem]^T, bf16 inputs, fp32 accumulate.
__device__ __forceinline__ void mma_ss(uint32_t go, uint32_t d, uint64_t adesc, uint64_t bdesc,
                                       uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(go)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem].
__device__ __forceinline__ void mma_ts(uint32_t go, uint32_t d, uint32_t a, uint64_t bdesc,
                                       uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(go)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t go, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
          tc::smem_u32(bar)),
      "r"(go)
      : "memory");
}

// MN-major operand stored as rows of 64 elements (128 bytes, 128-byte swizzle), one row
// a k: 8-row groups 1024 bytes apart along k, 64-element blocks `block` bytes apart.
__device__ __forceinline__ uint64_t desc_sw128_mnmajor(uint32_t addr, uint32_t block) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(block >> 4) << 16;   // leading byte offset: between 64-element blocks
  d |= (uint64_t)(1024 >> 4) << 32;    // stride byte offset: between groups of 8 k
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// 32 columns of 32 bits, without the wait.
__device__ __forceinline__ void tmem_st32_async(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// One row from the keys that it sees alone, a warp a row: the CTAs whose values hold
// infinities or NaN that some of their rows do not see.
template <typename T>
__device__ __noinline__ void row_alone(const AttnArgs& a, int b, int h, long long row, int hq,
                                       int place, int j0, int j1, float* m_, float* l_,
                                       float o[4]) {
  const int lane = threadIdx.x & 31, x = lane * 4;
  float q[4] = {0.f, 0.f, 0.f, 0.f};
  if (x < a.c.d) {
    const T* p = reinterpret_cast<const T*>(a.q) + row * a.q_row +
                             (long long)hq * a.q_head + x;
    for (int e = 0; e < 4; ++e) q[e] = to_f32(p[e]);
  }
  float m = *m_, l = *l_;
  for (int j = j0; j < j1; ++j) {
    if (!sees(place, j, a.window, a.sinks)) continue;
    const long long off = kv_row(a.c, b, h, j);
    if (off < 0) continue;
    float s = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
    if (x < a.c.d) {
      const T* kp = reinterpret_cast<const T*>(a.c.k) + off + x;
      const T* vp = reinterpret_cast<const T*>(a.c.v) + off + x;
      for (int e = 0; e < 4; ++e) {
        s = fmaf(q[e], to_f32(kp[e]), s);
        v[e] = to_f32(vp[e]);
      }
    }
    s = warp_sum(s) * a.scale2;
    const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn;
    const float f = exp2_fast(m - base), p = exp2_fast(s - base);
    l = l * f + p;
    for (int e = 0; e < 4; ++e) o[e] = o[e] * f + p * v[e];
    m = mn;
  }
  *m_ = m;
  *l_ = l;
}

// The sequence and the tile of it (`tokens` new tokens each) that is number c of all.
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int c, int tokens, const Div& by_tokens,
                                          int* b, int* tile, NewRows* nr, int* n) {
  auto tiles = [&](int T) { return by_tokens.of(T + tokens - 1); };
  if (!a.q_offsets) {
    const int each = tiles(a.T);
    *b = c / each;
    *tile = c - *b * each;
    if (*b >= a.c.B) return false;
    *nr = new_rows(a.q_offsets, *b, a.rows, a.T, a.c.status);
    *n = kv_len(a.c, *b);
    return true;
  }
  // each lane counts the tiles of some consecutive sequences
  const int lane = threadIdx.x & 31, cs = ceil_div(a.c.B, 32);
  const int b0 = min(a.c.B, lane * cs), b1 = min(a.c.B, b0 + cs);
  int mine = 0, len = 0;
  NewRows last = {0, 0};
#pragma unroll 4
  for (int x = b0; x < b1; ++x) {
    // all on their way before the first is looked at
    const int from = a.q_offsets[x], to = a.q_offsets[x + 1], raw = __ldcg(a.c.lens + x);
    last = new_rows(from, to, a.rows, a.T, a.c.status);
    len = kv_clamp(a.c, raw);
    mine += tiles(last.T);
  }
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(FULL, sum, o);
    if (lane >= o) sum += y;
  }
  if (c >= __shfl_sync(FULL, sum, 31)) return false;
  const int lo = __popc(__ballot_sync(FULL, sum - mine <= c)) - 1;
  int u = c - __shfl_sync(FULL, sum - mine, lo);
  last.off = __shfl_sync(FULL, last.off, lo);
  last.T = __shfl_sync(FULL, last.T, lo);
  len = __shfl_sync(FULL, len, lo);
  if (cs == 1) {
    *b = lo;
    *tile = u;
    *nr = last;
    *n = len;
    return true;
  }
  for (int x = lo * cs;; ++x) {
    *nr = new_rows(a.q_offsets, x, a.rows, a.T, a.c.status);
    const int here = tiles(nr->T);
    if (u < here) {
      *b = x;
      *tile = u;
      *n = kv_len(a.c, x);
      return true;
    }
    u -= here;
  }
}

// The number of parts, `most` at most, in which a key axis of so many turns takes the least
// time: a CTA's turns one after another (`turn` us each), and for more than one part the
// joining kernel (2.5 us) and the parts' rows (`floats` each), written and read again at
// about 5 TB/s.
inline int cheapest_parts(long long most, int turns, float turn, long long floats) {
  int best = 1;
  float least = turns * turn;
  for (int s = 2; s <= most; ++s) {
    const float t = ceil_div(turns, s) * turn + 2.5f + (float)s * floats * 8.f / 5e6f;
    if (t < least) {
      least = t;
      best = s;
    }
  }
  return best;
}

}  // namespace gmc
