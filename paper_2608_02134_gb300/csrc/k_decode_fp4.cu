// One new token's attention over a cache held in 4 bits (fp4.cuh); the outline, the parts
// and the scores are those of decode.cuh.
//
// Bound by memory, as with bf16, but with 72 bytes a key or value of 128 channels the copies
// leave a key 6 clocks of an SM, so instructions are the second bound: codes go from shared
// memory to the tensor cores' operands in registers, without a tile of values in between.
//
//   S = K q^T: the rows of mma m16n8k16 are 16 keys, its columns up to 8 query heads.  A
//   product sums over channels in any order, so a thread takes the fragments of a row from
//   d / 4 consecutive channels: two bytes a step, one conversion a pair, one product a pair
//   with the block's scale.  Values and q are exact in half precision: the row of q is
//   multiplied by a power of two that puts its largest value into [2^14, 2^15), and what that
//   makes too small for a half is 2^-39 of the largest.
//   O^T = V^T P^T: the rows are 16 channels, a thread's are consecutive again.  Here pairs are
//   two keys' values of one channel, so the codes of two keys are interleaved first (4
//   instructions for 16 codes).  P^T comes from S by a transposition in registers.  Weights
//   are rounded to half (relative 2^-12, an eighth of the output's own rounding; below 2^-14 of
//   the largest 2^-25 of it), their sum is the unrounded ones'.
//
// A turn is 32 keys.  Key x of it lies in row slot(x) of the stage's keys and row x of its
// values, and 16-byte pieces are swizzled, so that neither read meets a bank twice.
#include <cuda_fp16.h>

#include "decode.cuh"
#include "fp4.cuh"

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
template <int BYTES>
__device__ __forceinline__ void cp_async_small(void* smem, const void* src, bool pred) {
  const unsigned sa = (unsigned)__cvta_generic_to_shared(smem);
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(sa), "l"(src), "n"(BYTES),
               "r"(pred ? BYTES : 0)
               : "memory");
}

// A lane's row of a turn: place `lane` of it.
struct Fp4Row {
  enum { NONE, PAGE, FIXED } kind;
  int slot, page;
  __device__ __forceinline__ void look_up(const DecodeArgs& a, const Walk<32>& w, int lane) {
    const int x = w.t * 32 + lane;
    kind = NONE;
    page = slot = 0;
    if (x >= w.nv) return;
    const int j = w.seen.place(x);
    if (a.k_new && j == w.n - 1) {
      kind = FIXED;
      return;
    }
    kind = PAGE;
    const Slot at = kv_slot(a.c, w.b, j);
    page = at.page;
    slot = at.slot;
  }
};

// Rows of a stage: the key of row r of an mma's 16 is t + 4 e + 8 h with r = 2 t + e + 8 h.
__device__ __forceinline__ int key_of_row(int r) { return (r & 24) | ((r & 7) >> 1) | ((r & 1) << 2); }
__device__ __forceinline__ int row_of_key(int x) { return (x & 24) | ((x & 3) << 1) | ((x & 4) >> 2); }

// A stage: 32 keys' codes, 32 values', 32 keys' scales, 32 values'.
template <int DP> struct Fp4Stage {
  static constexpr int CB = DP / 2, SB = DP / 16, P = CB / 16;  // bytes of a row, pieces of codes
  static constexpr int VC = 32 * CB, KS = 64 * CB, VS = KS + 32 * SB, BYTES = VS + 32 * SB;
  // where a 16-byte piece of a row lies in it
  static __device__ __forceinline__ int key_piece(int row, int p) {
    return DP == 256 ? p ^ (row & 1) : p;
  }
  static __device__ __forceinline__ int value_piece(int row, int p) {
    return DP == 256 ? p ^ ((row & 3) * 2) : DP == 128 ? p ^ (row & 2) : p;
  }
};

template <int DP, int NST> struct Fp4Ring {
  typedef Fp4Stage<DP> S;
  static constexpr int STAGE = S::BYTES;
  char* at;
  int put, got;
  // The next stage takes the turn that `row` was looked up for; rows past the end become
  // zeros.  The appended row is packed here, from the caller's.
  __device__ __forceinline__ void fill(const DecodeArgs& a, const Fp4Row& row, int b, int h,
                                       int lane) {
    char* base = at + put * STAGE;
    put = put + 1 == NST ? 0 : put + 1;
    const bool there = row.kind == Fp4Row::PAGE && (unsigned)row.page < (unsigned)a.c.num_pages;
    if (row.kind == Fp4Row::PAGE && !there) set_status(a.c.status, CACHE_BAD);
    const long long part = row.page * a.c.page_stride + h * a.c.head_stride;
    // -1: no row, zeros; -2: written below
    const long long codes = there ? part + row.slot * S::CB : row.kind == Fp4Row::FIXED ? -2 : -1;
    constexpr int P = S::P, RPI = 32 / P;
    const int sub = lane / P, pc = lane % P;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RPI) {
      const int x = r0 + sub, y = row_of_key(x);
      const long long o = __shfl_sync(FULL, codes, x);
      if (o == -2) continue;
      const long long from = (o >= 0 ? o : 0) + pc * 16;
      cp_async16(base + y * S::CB + S::key_piece(y, pc) * 16, a.c.k + from, o >= 0);
      cp_async16(base + S::VC + x * S::CB + S::value_piece(x, pc) * 16, a.c.v + from, o >= 0);
    }
    if (row.kind != Fp4Row::FIXED) {
      const long long from = there ? part + fp4_scale_at(a.c, row.slot) : 0;
      cp_async_small<S::SB>(base + S::KS + row_of_key(lane) * S::SB, a.c.k + from, there);
      cp_async_small<S::SB>(base + S::VS + lane * S::SB, a.c.v + from, there);
    }
    const unsigned fixed = __ballot_sync(FULL, row.kind == Fp4Row::FIXED);
    if (fixed) {
      const int x = __ffs(fixed) - 1, y = row_of_key(x), blk = lane % S::SB;
      if (lane < 2 * S::SB) {
        const bool key = lane < S::SB;
        const uint4* src = reinterpret_cast<const uint4*>(
            (key ? a.k_new : a.v_new) + (((long long)b * a.c.Hkv + h) * DP + blk * 16) * 2);
        float v[16];
        unpack_bf16(src[0], v);
        unpack_bf16(src[1], v + 8);
        uint32_t s;
        const uint2 codes16 = fp4_block(v, &s);
        char* c = key ? base + y * S::CB + S::key_piece(y, blk >> 1) * 16
                      : base + S::VC + x * S::CB + S::value_piece(x, blk >> 1) * 16;
        *reinterpret_cast<uint2*>(c + (blk & 1) * 8) = codes16;
        base[key ? S::KS + y * S::SB + blk : S::VS + x * S::SB + blk] = (char)s;
      }
    }
  }
  __device__ __forceinline__ const char* take() {
    const char* p = at + got * STAGE;
    got = got + 1 == NST ? 0 : got + 1;
    return p;
  }
};

template <int DP> struct HeadsFp4 {
  static constexpr int DT = 32, HM = 8, EXTRA = 0, CTAS = 1;
  typedef __nv_bfloat16 T;
  typedef Fp4Row Row;
  template <int NST> using Ring = Fp4Ring<DP, NST>;
  typedef Fp4Stage<DP> S;
  static constexpr int CT = DP / 4;  // channels of a thread in a key
  static constexpr int CV = DP / 8;  // and in a value
  // Lane (g, t) = (lane / 4, lane % 4).  qf: head g, channels t CT ..; o: heads 2t and 2t + 1,
  // channels g CV .. in pairs.
  uint32_t qf[DP / 16][2];
  float o[DP / 16][4], m[2], l[2], factor[2];
  __device__ __forceinline__ void begin(const DecodeArgs& a, const Walk<32>& w, char*, int lane) {
    const int g = lane >> 2, t = lane & 3;
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
        qf[s][i] = g < a.heads ? pack_half(__uint_as_float(y[i] << 16) * up,
                                           __uint_as_float(y[i] & 0xffff0000u) * up)
                               : 0u;
    }
    // logits are multiplied by the scale and 2^-k of their heads
    const float down = a.scale2 * __uint_as_float((uint32_t)(127 - k) << 23);
    factor[0] = __shfl_sync(FULL, down, t * 8);
    factor[1] = __shfl_sync(FULL, down, t * 8 + 4);
#pragma unroll
    for (int x = 0; x < DP / 16; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  // The key's codes and scales of a thread: CT / 8 words, CT / 16 scales.
  static __device__ __forceinline__ void load_key(const char* stage, int row, int t, uint32_t* w,
                                                  uint32_t* s) {
    const char* c = stage + row * S::CB;
    if constexpr (DP == 64) {
      const uint2 v = *reinterpret_cast<const uint2*>(c + t * 8);
      w[0] = v.x;
      w[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < DP / 128; ++i) {
        const int p = DP / 128 * t + i;
        const uint4 v = *reinterpret_cast<const uint4*>(c + S::key_piece(row, p) * 16);
        w[4 * i] = v.x;
        w[4 * i + 1] = v.y;
        w[4 * i + 2] = v.z;
        w[4 * i + 3] = v.w;
      }
    }
    const char* z = stage + S::KS + row * S::SB + t * (DP / 64);
    if constexpr (DP == 64) {
      s[0] = fp4_scale2((uint32_t)(uint8_t)*z);
    } else if constexpr (DP == 128) {
      const uint32_t v = *reinterpret_cast<const uint16_t*>(z);
      s[0] = fp4_scale2(v & 0xffu);
      s[1] = fp4_scale2(v >> 8);
    } else {
      const uint32_t v = *reinterpret_cast<const uint32_t*>(z);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = fp4_scale2((v >> (8 * i)) & 0xffu);
    }
  }
  // The value's: CV / 8 words, and its blocks' scales, a byte each.
  static __device__ __forceinline__ void load_value(const char* stage, int row, int g, uint32_t* w,
                                                    uint32_t* s) {
    const char* c = stage + S::VC + row * S::CB;
    const char* z = stage + S::VS + row * S::SB;
    if constexpr (DP == 64) {
      w[0] = *reinterpret_cast<const uint32_t*>(c + g * 4);
      *s = (uint8_t)z[g >> 1];
    } else if constexpr (DP == 128) {
      const uint2 v =
          *reinterpret_cast<const uint2*>(c + S::value_piece(row, g >> 1) * 16 + (g & 1) * 8);
      w[0] = v.x;
      w[1] = v.y;
      *s = (uint8_t)z[g];
    } else {
      const uint4 v = *reinterpret_cast<const uint4*>(c + S::value_piece(row, g) * 16);
      w[0] = v.x;
      w[1] = v.y;
      w[2] = v.z;
      w[3] = v.w;
      *s = *reinterpret_cast<const uint16_t*>(z + 2 * g);
    }
  }
  __device__ __forceinline__ void turn(const DecodeArgs& a, const Walk<32>& w, const char* stage,
                                       char*, int lane) {
    const int g = lane >> 2, t = lane & 3;
    float s[2][4];  // keys of rows g and g + 8 of two groups of 16
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};  // shorter chains
      uint32_t w0[CT / 8], w1[CT / 8], s0[CT / 16], s1[CT / 16];
      load_key(stage, n * 16 + g, t, w0, s0);
      load_key(stage, n * 16 + g + 8, t, w1, s1);
#pragma unroll
      for (int i = 0; i < CT / 8; ++i) {
        uint32_t h0[4], h1[4];
        fp4_halves(w0[i], h0);
        fp4_halves(w1[i], h1);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t x[4] = {hmul2(h0[2 * j], s0[i / 2]), hmul2(h1[2 * j], s1[i / 2]),
                                 hmul2(h0[2 * j + 1], s0[i / 2]), hmul2(h1[2 * j + 1], s1[i / 2])};
          mma_f16(d[j], x, qf[2 * i + j][0], qf[2 * i + j][1]);
        }
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) s[n][y] = (d[0][y] + d[1][y]) * factor[y & 1];
    }
    const int x0 = w.t * 32 + key_of_row(g);
    if (w.t == w.turns - 1) {  // places past the end leave
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (x0 + n * 16 + (y >> 1) * 8 >= w.nv) s[n][y] = -INFINITY;
    }
    if (a.scores) {
      float* lg = logits_of(a, w) + key_of_row(g) * a.hs + t * 2;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          float* z = lg + (n * 16 + y * 8) * a.hs;
          if (t * 2 + 1 < a.hs)
            *reinterpret_cast<float2*>(z) = make_float2(s[n][2 * y], s[n][2 * y + 1]);
          else if (t * 2 < a.hs)
            *z = s[n][2 * y];
        }
    }
    // the maximum that weights are taken against follows the running one when that has grown
    // by 2^8: lanes only meet then
    float top[2];
    bool grew = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = fmaxf(fmaxf(s[0][r], s[0][2 + r]), fmaxf(s[1][r], s[1][2 + r]));
      grew |= top[r] > m[r] + 8.f || (m[r] == -INFINITY && top[r] > m[r]);
    }
    if (__any_sync(FULL, grew)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float mn = fmaxf(top[r], m[r]);
        mn = fmaxf(mn, __shfl_xor_sync(FULL, mn, 4));
        mn = fmaxf(mn, __shfl_xor_sync(FULL, mn, 8));
        mn = fmaxf(mn, __shfl_xor_sync(FULL, mn, 16));
        const float f = exp2_fast(m[r] - (mn == -INFINITY ? 0.f : mn));
        l[r] *= f;
#pragma unroll
        for (int y = 0; y < DP / 16; ++y) {
          o[y][r] *= f;
          o[y][2 + r] *= f;
        }
        m[r] = mn;
      }
    }
    const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        s[n][y] = exp2_fast(s[n][y] - base[y & 1]);
        l[y & 1] += s[n][y];
      }
      const uint32_t p0 = transpose8(pack_half(s[n][0], s[n][1]));
      const uint32_t p1 = transpose8(pack_half(s[n][2], s[n][3]));
      // values of keys t, t + 4 (the k of p0) and t + 8, t + 12 (of p1)
      uint32_t v[4][CV / 8], z[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) load_value(stage, n * 16 + y * 4 + t, g, v[y], &z[y]);
#pragma unroll
      for (int i = 0; i < CV / 8; ++i) {
        const int sh = DP == 256 ? (i >> 1) * 8 : 0;
        const uint32_t s0 = fp4_scales((z[0] >> sh) & 0xffu, (z[1] >> sh) & 0xffu),
                       s1 = fp4_scales((z[2] >> sh) & 0xffu, (z[3] >> sh) & 0xffu);
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
          mma_f16(o[i * 4 + j], x, p0, p1);
        }
      }
    }
  }
  // Maxima and sums, and the unnormalised output rows [heads][DP].
  __device__ __forceinline__ void leave(const DecodeArgs& a, float2* ml, float* out, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(FULL, l[r], 4);
      l[r] += __shfl_xor_sync(FULL, l[r], 8);
      l[r] += __shfl_xor_sync(FULL, l[r], 16);
      const int head = t * 2 + r;
      if (head < a.heads) {
        if (g == 0) ml[head] = make_float2(m[r], l[r]);
#pragma unroll
        for (int x = 0; x < DP / 16; ++x)
          *reinterpret_cast<float2*>(out + head * DP + g * CV + x * 2) =
              make_float2(o[x][r], o[x][2 + r]);
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
    const int x = w.nv - 1 - w.t * 32, y = row_of_key(x);
    const long long part = at.page * a.c.page_stride + w.h * a.c.head_stride;
    const long long codes = part + (long long)at.slot * S::CB,
                    scales = part + fp4_scale_at(a.c, at.slot);
    if (lane < S::P)
      *reinterpret_cast<uint4*>(a.c.k + codes + lane * 16) =
          *reinterpret_cast<const uint4*>(stage + y * S::CB + S::key_piece(y, lane) * 16);
    else if (lane < 2 * S::P)
      *reinterpret_cast<uint4*>(a.c.v + codes + (lane - S::P) * 16) =
          *reinterpret_cast<const uint4*>(stage + S::VC + x * S::CB +
                                          S::value_piece(x, lane - S::P) * 16);
    constexpr int SW = S::SB / 4;
    if (lane < SW)
      *reinterpret_cast<uint32_t*>(a.c.k + scales + lane * 4) =
          *reinterpret_cast<const uint32_t*>(stage + S::KS + y * S::SB + lane * 4);
    else if (lane < 2 * SW)
      *reinterpret_cast<uint32_t*>(a.c.v + scales + (lane - SW) * 4) =
          *reinterpret_cast<const uint32_t*>(stage + S::VS + x * S::SB + (lane - SW) * 4);
  }
};

}  // namespace

cudaError_t launch_decode_fp4(const DecodeArgs& a, cudaStream_t st, int* launches) {
  return a.c.d == 64    ? decode_launch<HeadsFp4<64>, 64, 16, 4>(a, st, launches)
         : a.c.d == 128 ? decode_launch<HeadsFp4<128>, 128, 16, 3>(a, st, launches)
                        : decode_launch<HeadsFp4<256>, 256, 8, 3>(a, st, launches);
}

}  // namespace gmc
