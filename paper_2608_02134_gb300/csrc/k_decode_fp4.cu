// One new token's attention over a cache held in 4 bits (fp4.cuh); the outline, the parts
// and the scores are those of decode.cuh.
//
// Bound by memory, as with bf16, but with 72 bytes a key or value of 128 channels the copies
// leave a key 6 clocks of an SM, so instructions are the second bound: codes go from shared
// memory to the tensor cores' operands in registers, without a tile of values in between.
//
//   S = K q^T: the rows of mma m16n8k16 are 16 keys, its columns up to 8 query heads (of 9 to 16
//   with d <= 128 a second product takes the same fragments).  A
//   product sums over channels in any order, so a thread takes the fragments of a row from
//   d / 4 consecutive channels: two bytes a step, one conversion a pair, one product a pair
//   with the block's scale.  Values and q are exact in half precision: the row of q is
//   multiplied by a power of two that puts its largest value into [2^14, 2^15), and what that
//   makes too small for a half is 2^-39 of the largest.
//   O^T = V^T P^T: the rows are 16 channels, a thread's are consecutive again.  Here pairs are
//   two keys' values of one channel, so the codes of two keys are interleaved first (4
//   instructions for 16 codes).  P^T comes from S by a transposition in registers.  Weights
//   are rounded to half (relative 2^-11, an eighth of the output's own rounding; below 2^-21 of
//   the largest 2^-32 of it, FP4_UP), their sum is the unrounded ones'.
//
// A turn is 32 keys from a multiple of 32 on.  Where they are all seen a warp copies their codes
// and scales in straight runs, else row by row.
#include <cuda_fp16.h>

#include "decode.cuh"
#include "fp4.cuh"
#include "tc.cuh"

namespace gmc {

namespace {

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values over the warp, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Words of shared memory.
template <int BYTES> __device__ __forceinline__ void lds(uint32_t at, uint32_t* w) {
  if constexpr (BYTES == 16)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(at));
  else if constexpr (BYTES == 8)
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
  else if constexpr (BYTES == 4)
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
  else if constexpr (BYTES == 2)
    asm volatile("ld.shared.u16 %0, [%1];" : "=r"(w[0]) : "r"(at));
  else
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(w[0]) : "r"(at));
}
template <int BYTES>
__device__ __forceinline__ void cp_async_small(void* smem, const void* src, bool pred) {
  const unsigned sa = (unsigned)__cvta_generic_to_shared(smem);
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(sa), "l"(src), "n"(BYTES),
               "r"(pred ? BYTES : 0)
               : "memory");
}

// The key of row r (0 .. 7) of an mma.  Four lanes read a key's codes, and lanes 2t (and 2t + 1)
// of the rows the values' that they are multiplied with: in this order neither meets a bank
// twice with 64 channels, values twice with 128.
template <int DP> __device__ __forceinline__ int key_of_row(int r) {
  return DP == 64 ? (r & 4) | (((r & 1) << 1 | (r >> 1 & 1)) ^ (r >> 1 & 2)) : r ^ (r >> 1 & 1);
}

// A stage: 32 keys' codes, 32 values', 32 keys' scales, 32 values'.
template <int DP> struct Fp4Stage {
  static constexpr int CB = DP / 2, SB = DP / 16, P = CB / 16;  // bytes of a row, pieces of codes
  static constexpr int VC = 32 * CB, KS = 64 * CB, VS = KS + 32 * SB, BYTES = VS + 32 * SB;
};

// A turn's copies.  Turns whose keys are all seen and cached, in runs of 32 or 16 of one page
// each, are copied straight through, their page numbers read a turn ahead; any other goes row by
// row.  Where pages hold whole turns the next turn of the same page is just further on.
struct Fp4Turn {
  bool whole, found;        // found: codes and scales are this turn's
  int page[2], slot, more;  // more: turns of the same page from here on
  long long codes, scales;  // offsets of the lane's first pieces
};
__device__ __forceinline__ int page_of(const DecodeArgs& a, const Walk<32>& w, int j, int* slot) {
  const int p = a.by_ps.of(j);
  *slot = j - p * a.c.ps;
  return a.c.table[(long long)w.b * a.c.max_pages + p];
}
__device__ __forceinline__ void look_up(const DecodeArgs& a, const Walk<32>& w, Fp4Turn* x) {
  x->more = 0;
  x->found = false;
  x->whole = (a.c.ps & 15) == 0 && w.t >= w.lo && w.t < w.hi;
  if (!x->whole) return;
  const int j = w.t * 32 + w.off;
  x->page[0] = x->page[1] = page_of(a, w, j, &x->slot);
  int other;
  if (a.c.ps & 31)
    x->page[1] = page_of(a, w, j + 16, &other);
  else
    x->more = min((a.c.ps - x->slot) >> 5, w.hi - w.t);
}

// A key a lane; rows that are not seen become zeros, the appended one is packed here, from the
// caller's.
template <int DP>
__device__ __forceinline__ void fill_rows(const DecodeArgs& a, const Walk<32>& w, int lane,
                                          char* base) {
  typedef Fp4Stage<DP> S;
  const int x = w.t * 32 + lane, j = w.seen.place(x);
  const bool in = x < w.nv && sees(w.n - 1, j, a.window, a.sinks);
  const bool fixed = in && a.k_new && j == w.n - 1;
  int slot = 0, page = -1;
  if (in && !fixed) page = page_of(a, w, j, &slot);
  const bool there = in && !fixed && (unsigned)page < (unsigned)a.c.num_pages;
  if (in && !fixed && !there) set_status(a.c.status, CACHE_BAD);
  if (!fixed) {
    const long long part = there ? page * a.c.page_stride + w.h * a.c.head_stride : 0;
    const long long codes = there ? part + (long long)slot * S::CB : 0;
#pragma unroll
    for (int pc = 0; pc < S::P; ++pc) {
      cp_async16(base + lane * S::CB + pc * 16, a.c.k + codes + pc * 16, there);
      cp_async16(base + S::VC + lane * S::CB + pc * 16, a.c.v + codes + pc * 16, there);
    }
    const long long from = there ? part + fp4_scale_at(a.c, slot) : 0;
    cp_async_small<S::SB>(base + S::KS + lane * S::SB, a.c.k + from, there);
    cp_async_small<S::SB>(base + S::VS + lane * S::SB, a.c.v + from, there);
  }
  const unsigned who = __ballot_sync(FULL, fixed);
  if (who && lane < 2 * S::SB) {
    const int y = __ffs(who) - 1, blk = lane % S::SB;
    const bool key = lane < S::SB;
    const uint4* src = reinterpret_cast<const uint4*>(
        (key ? a.k_new : a.v_new) + (((long long)w.b * a.c.Hkv + w.h) * DP + blk * 16) * 2);
    uint32_t s;
    const uint2 block = fp4_block(src[0], src[1], &s);
    *reinterpret_cast<uint2*>(base + (key ? 0 : S::VC) + y * S::CB + blk * 8) = block;
    base[(key ? S::KS : S::VS) + y * S::SB + blk] = (char)s;
  }
}
// The stage at `base` takes the turn w, looked up before.  Behind it x is the next turn's, if
// x.more is not 0.
template <int DP>
__device__ __forceinline__ void fill(const DecodeArgs& a, const Walk<32>& w, Fp4Turn& x, int lane,
                                     char* base) {
  typedef Fp4Stage<DP> S;
  constexpr int STEPS = 16 * S::CB / 512;  // codes: two runs of 16 keys, 512 bytes a step
  constexpr int RP = 2 * S::SB;            // scales: of the keys, then of the values, 16 bytes each
  if (!x.whole || (unsigned)x.page[0] >= (unsigned)a.c.num_pages ||
      (unsigned)x.page[1] >= (unsigned)a.c.num_pages) {
    x.more = 0;
    fill_rows<DP>(a, w, lane, base);
    return;
  }
  const int l16 = lane * 16;
  if (a.c.ps & 31) {  // two runs of 16
    const long long head = w.h * a.c.head_stride;
    const long long p0 = head + x.page[0] * a.c.page_stride,
                    p1 = head + x.page[1] * a.c.page_stride;
    const int slot1 = x.slot + 16 < a.c.ps ? x.slot + 16 : 0;
    const long long o0 = p0 + (long long)x.slot * S::CB + l16,
                    o1 = p1 + (long long)slot1 * S::CB + l16;
#pragma unroll
    for (int y = 0; y < STEPS; ++y) {
      cp_async16(base + l16 + y * 512, a.c.k + o0 + y * 512);
      cp_async16(base + S::VC + l16 + y * 512, a.c.v + o0 + y * 512);
      cp_async16(base + l16 + (STEPS + y) * 512, a.c.k + o1 + y * 512);
      cp_async16(base + S::VC + l16 + (STEPS + y) * 512, a.c.v + o1 + y * 512);
    }
#pragma unroll
    for (int y = 0; y < 2 * RP; y += 32) {
      const int z = y + lane, run = z / S::SB, pc = z % S::SB;  // runs: keys' two, values' two
      const long long o = (run & 1 ? p1 : p0) +
                          fp4_scale_at(a.c, run & 1 ? slot1 : x.slot) + pc * 16;
      if (2 * RP >= 32 || z < 2 * RP)
        cp_async16(base + S::KS + z * 16, (run & 2 ? a.c.v : a.c.k) + o);
    }
    return;
  }
  if (!x.found) {
    const long long part = w.h * a.c.head_stride + x.page[0] * a.c.page_stride;
    x.codes = part + (long long)x.slot * S::CB + l16;
    x.scales = part + fp4_scale_at(a.c, x.slot) + (lane & (RP - 1)) * 16;
    x.found = true;
  }
  const char *k = a.c.k + x.codes, *v = a.c.v + x.codes;
#pragma unroll
  for (int y = 0; y < 2 * STEPS; ++y) {
    cp_async16(base + l16 + y * 512, k + y * 512);
    cp_async16(base + S::VC + l16 + y * 512, v + y * 512);
  }
  if constexpr (RP == 32) {
    cp_async16(base + S::KS + l16, a.c.k + x.scales);
    cp_async16(base + S::VS + l16, a.c.v + x.scales);
  } else if (2 * RP >= 32 || lane < 2 * RP) {
    cp_async16(base + S::KS + l16, (lane & RP ? a.c.v : a.c.k) + x.scales);
  }
  x.codes += 32 * S::CB;
  x.scales += 32 * S::SB;
  --x.more;
}

// NT x 8 query heads.
template <int DP, int NT> struct HeadsFp4 {
  static constexpr int HM = 8 * NT;
  typedef __nv_bfloat16 T;
  typedef Fp4Stage<DP> S;
  static constexpr int CT = DP / 4;  // channels of a thread in a key
  static constexpr int CV = DP / 8;  // and in a value
  // Lane (g, t) = (lane / 4, lane % 4).  Of eight heads qf: head g, channels t CT ..; o: heads 2t
  // and 2t + 1, channels g CV .. in pairs.
  uint32_t qf[NT][DP / 16][2];
  float o[NT][DP / 16][4], m[NT][2], l[NT][2], factor[NT][2], room[NT][2];
  __device__ __forceinline__ void begin(const DecodeArgs& a, const Walk<32>& w, int lane) {
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      const int g = (lane >> 2) + 8 * z, t = lane & 3;
      uint2 raw[DP / 16];
      const T* q = reinterpret_cast<const T*>(a.q) + w.b * a.q_row +
                   (long long)(w.h * a.G + a.h0 + min(g, a.heads - 1)) * a.q_head + t * CT;
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < DP / 16; s += 2) {
        const uint4 v = *reinterpret_cast<const uint4*>(q + s * 4);
        raw[s] = make_uint2(v.x, v.y);
        raw[s + 1] = make_uint2(v.z, v.w);
        const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          top = max(top, max(y[i] & 0x7fffu, (y[i] >> 16) & 0x7fffu));
      }
      top = max(top, __shfl_xor_sync(FULL, top, 1));
      top = max(top, __shfl_xor_sync(FULL, top, 2));
      // 2^k that puts the largest magnitude into [2^14, 2^15); none for zeros and what is not
      // finite
      const int e = (int)(top >> 7) - 127;
      const int k = top == 0 || top >= 0x7f80u ? 0 : min(14 - e, 126);
      const float up = __uint_as_float((uint32_t)(k + 127) << 23);
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        const uint32_t y[2] = {raw[s].x, raw[s].y};
#pragma unroll
        for (int i = 0; i < 2; ++i)
          qf[z][s][i] = g < a.heads ? pack_half(__uint_as_float(y[i] << 16) * up,
                                                __uint_as_float(y[i] & 0xffff0000u) * up)
                                    : 0u;
      }
      // logits are multiplied by the scale and 2^-k of their heads
      const float down = fmaxf(a.scale2 * __uint_as_float((uint32_t)(127 - k) << 23), 1e-37f);
      factor[z][0] = __shfl_sync(FULL, down, t * 8);
      factor[z][1] = __shfl_sync(FULL, down, t * 8 + 4);
#pragma unroll
      for (int x = 0; x < DP / 16; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) o[z][x][y] = 0.f;
      m[z][0] = m[z][1] = room[z][0] = room[z][1] = -INFINITY;
      l[z][0] = l[z][1] = 0.f;
    }
  }
  // The key's codes and scales of a thread: CT / 8 words, CT / 16 scales.
  static __device__ __forceinline__ void load_key(uint32_t stage, int row, int t, uint32_t* w,
                                                  uint32_t* s) {
    const uint32_t c = stage + row * S::CB + t * (CT / 2);
    if constexpr (DP == 256) {
      lds<16>(c, w);
      lds<16>(c + 16, w + 4);
    } else {
      lds<CT / 2>(c, w);
    }
    uint32_t z;
    lds<DP / 64>(stage + S::KS + row * S::SB + t * (DP / 64), &z);
#pragma unroll
    for (int i = 0; i < DP / 64; ++i)
      s[i] = fp4_scale2(DP == 64 ? z : (z >> (8 * i)) & 0xffu);
  }
  // The value's: CV / 8 words, and its blocks' scales, a byte each.
  static __device__ __forceinline__ void load_value(uint32_t stage, int row, int g, uint32_t* w,
                                                    uint32_t* s) {
    lds<CV / 2>(stage + S::VC + row * S::CB + g * (CV / 2), w);
    const uint32_t z = stage + S::VS + row * S::SB;
    if constexpr (DP == 256)
      lds<2>(z + 2 * g, s);
    else
      lds<1>(z + (DP == 64 ? g >> 1 : g), s);
  }
  __device__ __forceinline__ void turn(const DecodeArgs& a, const Walk<32>& w, const char* from,
                                       int lane) {
    const uint32_t stage = tc::smem_u32(from);
    const int g = lane >> 2, t = lane & 3;
    const int kg = key_of_row<DP>(g), k0 = key_of_row<DP>(2 * t), k1 = key_of_row<DP>(2 * t + 1);
    float s[NT][2][4];  // keys kg and kg + 8 of two groups of 16
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int z = 0; z < NT; ++z)
        s[z][n][0] = s[z][n][1] = s[z][n][2] = s[z][n][3] = 0.f;
      uint32_t w0[CT / 8], w1[CT / 8], s0[CT / 16], s1[CT / 16];
      load_key(stage, n * 16 + kg, t, w0, s0);
      load_key(stage, n * 16 + kg + 8, t, w1, s1);
#pragma unroll
      for (int i = 0; i < CT / 8; ++i) {
        uint32_t h0[4], h1[4];
        fp4_halves(w0[i], h0);
        fp4_halves(w1[i], h1);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t x[4] = {hmul2(h0[2 * j], s0[i / 2]), hmul2(h1[2 * j], s1[i / 2]),
                                 hmul2(h0[2 * j + 1], s0[i / 2]), hmul2(h1[2 * j + 1], s1[i / 2])};
#pragma unroll
          for (int z = 0; z < NT; ++z)
            mma_f16(s[z][n], x, qf[z][2 * i + j][0], qf[z][2 * i + j][1]);
        }
      }
    }
    if (w.t < w.lo || w.t >= w.hi) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int x = w.t * 32 + n * 16 + (y >> 1) * 8 + kg;
          if (x >= w.nv || !sees(w.n - 1, w.seen.place(x), a.window, a.sinks))
#pragma unroll
            for (int z = 0; z < NT; ++z) s[z][n][y] = -INFINITY;
        }
    }
    if (a.scores) {
#pragma unroll
      for (int z = 0; z < NT; ++z) {
        const int head = 8 * z + t * 2;
        float* lg = logits_of(a, w) + kg * a.hs + head;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float* to = lg + (n * 16 + y * 8) * a.hs;
            const float x0 = s[z][n][2 * y] * factor[z][0],
                        x1 = s[z][n][2 * y + 1] * factor[z][1];
            if (head + 1 < a.hs)
              *reinterpret_cast<float2*>(to) = make_float2(x0, x1);
            else if (head < a.hs)
              *to = x0;
          }
      }
    }
    // the base that weights are taken against (FP4_UP below a maximum) follows the running maximum
    // when that has grown by 2^8 (`room`: that much more as a sum of products): lanes only meet then
    float top[NT][2];
    bool grew = false;
#pragma unroll
    for (int z = 0; z < NT; ++z)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        top[z][r] = fmaxf(fmaxf(s[z][0][r], s[z][0][2 + r]), fmaxf(s[z][1][r], s[z][1][2 + r]));
        grew |= top[z][r] > room[z][r];
      }
    if (__any_sync(FULL, grew)) {
#pragma unroll
      for (int z = 0; z < NT; ++z)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float mn = fmaxf(__fmul_ru(top[z][r], factor[z][r]) - FP4_UP, m[z][r]);
          mn = fmaxf(mn, __shfl_xor_sync(FULL, mn, 4));
          mn = fmaxf(mn, __shfl_xor_sync(FULL, mn, 8));
          mn = fmaxf(mn, __shfl_xor_sync(FULL, mn, 16));
          const float f = exp2_fast(m[z][r] - (mn == -INFINITY ? 0.f : mn));
          l[z][r] *= f;
#pragma unroll
          for (int y = 0; y < DP / 16; ++y) {
            o[z][y][r] *= f;
            o[z][y][2 + r] *= f;
          }
          m[z][r] = mn;
          const float above = (mn + FP4_ROOM) / factor[z][r];
          room[z][r] = fmaf(fabsf(above), -0x1p-22f, above);  // not more by two roundings
        }
    }
    uint32_t p[NT][2][2];  // weights: of group n the first and the second eight keys'
#pragma unroll
    for (int z = 0; z < NT; ++z) {
      const f32x2 scale = pair(factor[z][0], factor[z][1]),
                  off = pair(m[z][0] == -INFINITY ? 0.f : -m[z][0],
                             m[z][1] == -INFINITY ? 0.f : -m[z][1]);
      f32x2 sum = pair(l[z][0], l[z][1]);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float2 x =
              unpair(fma2(pair(s[z][n][2 * y], s[z][n][2 * y + 1]), scale, off));
          const float p0 = exp2_fast(x.x), p1 = exp2_fast(x.y);
          sum = add2(sum, pair(p0, p1));
          p[z][n][y] = transpose8(pack_half(p0, p1));
        }
      const float2 all = unpair(sum);
      l[z][0] = all.x;
      l[z][1] = all.y;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      // values of keys k0, k1 (the k of p[.][n][0]) and k0 + 8, k1 + 8 (of p[.][n][1])
      uint32_t v[4][CV / 8], z4[4];
#pragma unroll
      for (int y = 0; y < 4; ++y)
        load_value(stage, n * 16 + (y >> 1) * 8 + (y & 1 ? k1 : k0), g, v[y], &z4[y]);
#pragma unroll
      for (int i = 0; i < CV / 8; ++i) {
        const int sh = DP == 256 ? (i >> 1) * 8 : 0;
        const uint32_t s0 = fp4_scales((z4[0] >> sh) & 0xffu, (z4[1] >> sh) & 0xffu),
                       s1 = fp4_scales((z4[2] >> sh) & 0xffu, (z4[3] >> sh) & 0xffu);
        constexpr uint32_t LO = 0x0f0f0f0fu;
        uint32_t h[4][4];  // even and odd channels of the first pair of keys, of the second
        fp4_halves((v[0][i] & LO) | ((v[1][i] << 4) & ~LO), h[0]);
        fp4_halves(((v[0][i] >> 4) & LO) | (v[1][i] & ~LO), h[1]);
        fp4_halves((v[2][i] & LO) | ((v[3][i] << 4) & ~LO), h[2]);
        fp4_halves(((v[2][i] >> 4) & LO) | (v[3][i] & ~LO), h[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x[4] = {hmul2(h[0][j], s0), hmul2(h[1][j], s0), hmul2(h[2][j], s1),
                                 hmul2(h[3][j], s1)};
#pragma unroll
          for (int z = 0; z < NT; ++z) mma_f16(o[z][i * 4 + j], x, p[z][n][0], p[z][n][1]);
        }
      }
    }
  }
  // Maxima and sums, and the unnormalised output rows [heads][DP].
  __device__ __forceinline__ void leave(const DecodeArgs& a, float2* ml, float* out, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int z = 0; z < NT; ++z)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l[z][r] += __shfl_xor_sync(FULL, l[z][r], 4);
        l[z][r] += __shfl_xor_sync(FULL, l[z][r], 8);
        l[z][r] += __shfl_xor_sync(FULL, l[z][r], 16);
        const int head = 8 * z + t * 2 + r;
        if (head < a.heads) {
          if (g == 0) ml[head] = make_float2(m[z][r], l[z][r]);
#pragma unroll
          for (int x = 0; x < DP / 16; ++x)
            *reinterpret_cast<float2*>(out + head * DP + g * CV + x * 2) =
                make_float2(o[z][x][r], o[z][x][2 + r]);
        }
      }
  }
  // The appended row goes to its page, as it was packed: the warp that has the pair's last turn.
  static __device__ __forceinline__ void append(const DecodeArgs& a, const Walk<32>& w,
                                                const char* stage, int lane) {
    const Slot at = kv_slot(a.c, w.b, w.n - 1);
    if ((unsigned)at.page >= (unsigned)a.c.num_pages) {
      set_status(a.c.status, CACHE_BAD);
      return;
    }
    const int x = w.nv - 1 - w.t * 32;
    const long long part = at.page * a.c.page_stride + w.h * a.c.head_stride;
    const long long codes = part + (long long)at.slot * S::CB,
                    scales = part + fp4_scale_at(a.c, at.slot);
    if (lane < S::P)
      *reinterpret_cast<uint4*>(a.c.k + codes + lane * 16) =
          *reinterpret_cast<const uint4*>(stage + x * S::CB + lane * 16);
    else if (lane < 2 * S::P)
      *reinterpret_cast<uint4*>(a.c.v + codes + (lane - S::P) * 16) =
          *reinterpret_cast<const uint4*>(stage + S::VC + x * S::CB + (lane - S::P) * 16);
    constexpr int SW = S::SB / 4;
    if (lane < SW)
      *reinterpret_cast<uint32_t*>(a.c.k + scales + lane * 4) =
          *reinterpret_cast<const uint32_t*>(stage + S::KS + x * S::SB + lane * 4);
    else if (lane < 2 * SW)
      *reinterpret_cast<uint32_t*>(a.c.v + scales + (lane - SW) * 4) =
          *reinterpret_cast<const uint32_t*>(stage + S::VS + x * S::SB + (lane - SW) * 4);
  }
};

// W warps, each with a ring of NST stages and a run of turns.  Where a CTA has three pairs at most
// it joins its warps' parts: they are balanced whatever the borders, and few are left.  (A pair's
// turns shared out among all warps, pair after pair, took 28.7 us for 8 x 16,005 keys: a border
// costs a barrier, and the parts' rounding up.)  OWN: a CTA takes a whole pair, and no other.
template <int DP, int NT, int W, int NST, bool OWN>
__global__ void __launch_bounds__(W * 32, 1) k_decode_fp4(DecodeArgs a) {
  typedef HeadsFp4<DP, NT> H;
  typedef typename H::T T;
  typedef Fp4Stage<DP> S;
  constexpr int HM = H::HM, ROWS = HM * DP * 4, SLOTS = W + 2;  // bytes of a part, parts
  extern __shared__ __align__(512) char smem[];
  __shared__ float2 fin[OWN ? HM : 1];
  char* rows = smem + W * NST * S::BYTES;                       // [SLOTS][HM][DP]
  float2* ml = reinterpret_cast<float2*>(rows + SLOTS * ROWS);  // [SLOTS][HM]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dep_wait();
  grid_dep_launch();  // not before: k_decode_join reads the lengths ahead of its own wait
  Stretch<32, W> s;
  int per;
  Walk<32> first;  // the CTA's first turn
  if constexpr (OWN) {
    s.own(a);
    if (s.count == 0) {
      write_nothing<T, DP>(a, s.w.b, s.w.h);
      return;
    }
    first = s.w;
    per = ceil_div(s.count, W);
    s.warp_of_own(warp);
  } else {
    const TurnRow<32> turns(a);
    if (!s.share(a, turns)) return;
    first = s.w;
    per = turns.per;
    s.warp_of_several(a, turns, warp);
  }
  const int pair0 = first.b * a.c.Hkv + first.h;
  int left = s.end - s.u;  // of the run
  if (left > 0) {
    char* const ring = smem + warp * NST * S::BYTES;
    int put = 0, got = 0, ahead = left;  // stages, turns to be copied
    Walk<32> f = s.w;
    Fp4Turn x;
    look_up(a, f, &x);
    auto copy = [&]() {
      if (ahead > 0) {
        fill<DP>(a, f, x, lane, ring + put * S::BYTES);
        put = put + 1 == NST ? 0 : put + 1;
        if (--ahead > 0) {
          if (++f.t >= f.turns) {
            f.next_pair(a);
            x.more = 0;
          }
          if (x.more == 0) look_up(a, f, &x);
        }
      }
      cp_async_commit();
    };
#pragma unroll 1
    for (int y = 0; y < NST - 1; ++y) copy();
    H heads;
    Walk<32> w = s.w;
    while (true) {  // pair after pair
      heads.begin(a, w, lane);
      const int limit = min(w.turns, w.t + left);
      left -= limit - w.t;
#pragma unroll 1
      for (; w.t < limit; ++w.t) {
        copy();  // into the stage that the turn before has left
        cp_async_wait<NST - 1>();
        __syncwarp();
        const char* here = ring + got * S::BYTES;
        got = got + 1 == NST ? 0 : got + 1;
        heads.turn(a, w, here, lane);
        if (w.t == w.turns - 1 && a.k_new) H::append(a, w, here, lane);
        __syncwarp();  // every lane has read the stage
      }
      const int pair = w.b * a.c.Hkv + w.h;
      if (s.few) {
        const int slot = warp + pair - pair0;
        heads.leave(a, ml + slot * HM, reinterpret_cast<float*>(rows + slot * ROWS), lane);
      } else {
        const long long part = (long long)blockIdx.x * W + warp + pair;
        heads.leave(a, a.ml + part * a.heads, a.part + part * a.heads * DP, lane);
      }
      if (left <= 0) break;
      w.next_pair(a);
    }
  }
  if (!s.few) return;
  __syncthreads();
  // the pairs' parts: of warps t0 / per to (t1 - 1) / per
  Walk<32>& w = first;
  for (int t0 = 0;;) {
    const int t1 = min(s.count, t0 + w.turns - w.t), p0 = t0 / per, p1 = (t1 - 1) / per;
    const int slot = p0 + w.b * a.c.Hkv + w.h - pair0;
    join_warps<T, HM, DP, W>(a, w.b, w.h, p1 - p0 + 1, t1 - t0 == w.turns, ml + slot * HM,
                             rows + slot * ROWS, ROWS, OWN ? fin : nullptr);
    if (t1 >= s.count) break;
    t0 = t1;
    w.next_pair(a);
  }
  if (OWN && a.scores) {
    __syncthreads();
    add_scores(a, w, fin, tid, W * 32);
  }
}

template <int DP, int NT, int W, int NST>
cudaError_t decode_fp4_go(const DecodeArgs& a, cudaStream_t st, int* launches) {
  static_assert(W <= 16, "the workspace holds a part a warp");
  constexpr size_t smem = (size_t)W * NST * Fp4Stage<DP>::BYTES +
                          (size_t)(W + 2) * 8 * NT * (DP * 4 + sizeof(float2));
  static_assert(smem <= 226 * 1024, "shared memory of a CTA");
  // own pairs, with 128 channels and 4 key heads: 32 sequences of 512 keys and scores 8.2 us, in
  // stretches 14.0; of up to 3,000 25.7 and 27.6; 20 of 4,000 21.7 and 21.2.  One of 322 keys 5.6
  // and 9.7, of 1,500 9.9 and 11.8; two of 3,000 15.5 and 14.7.
  return decode_launch<__nv_bfloat16, 32, DP, W>(a, k_decode_fp4<DP, NT, W, NST, true>,
                                                 k_decode_fp4<DP, NT, W, NST, false>,
                                                 OwnTurns{8 * 12 / W, 4 * 12 / W}, smem, st, launches);
}

}  // namespace

cudaError_t launch_decode_fp4(const DecodeArgs& a, cudaStream_t st, int* launches) {
  if (a.heads > 8)
    return a.c.d == 64 ? decode_fp4_go<64, 2, 12, 4>(a, st, launches)
                       : decode_fp4_go<128, 2, 8, 3>(a, st, launches);
  return a.c.d == 64    ? decode_fp4_go<64, 1, 12, 4>(a, st, launches)
         : a.c.d == 128 ? decode_fp4_go<128, 1, 12, 2>(a, st, launches)
                        : decode_fp4_go<256, 1, 6, 2>(a, st, launches);
}

}  // namespace gmc
