// One new token's attention over a paged key-value cache: out = sum_j p_j v_j with
// p = softmax(scale q . k_j) over the seen keys, the new token's own key and value
// appended on the way, and optionally the weight that every key received added to
// its running score.
//
// Bound by memory: each key and value is read once for the G query heads that share
// it.  The seen keys of all sequences and key heads, 16 a turn, lie in one row, and
// every CTA of the GPU takes an equal stretch of it, whatever the sequences' lengths.
// Inside one pair (sequence, key head) the warps of a CTA take turns in turn, so that
// the CTA reads neighbouring rows at a time; a stretch over several pairs is cut into
// one run a warp.  A warp copies its keys and values ahead into its own ring in shared
// memory (cp.async, no barrier; the page numbers a turn earlier still) and keeps the
// running maxima and sums of its query heads and their output in registers.  8 sequences
// of 16,005 keys (28 heads, 4 key heads of 128, bf16): 49 us, 5.3 TB/s; 64 of 4,000: 96 us,
// 5.5 TB/s.
//
// What a CTA holds of a pair that others share is left as a part in the workspace, and a
// second kernel joins the parts of every query head in the order of the row and adds the
// scores.  Where the sequences are short a CTA takes a pair, whatever its length, and
// nothing is left to join.  (Joined by the CTA that is last instead, one launch took 18.4 us for one
// sequence of 322 keys where the two take 8.4: a count, a fence and the joining one after
// another on one SM.)
#include <algorithm>

#include "cache.cuh"

namespace gmc {

namespace {
constexpr int DT = 16;  // keys of a turn

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// ---- the row of turns ----------------------------------------------------------------
// A pair and a turn of it.
struct Walk {
  int b, h, t, turns, nv, n;
  Seen seen;
  __device__ __forceinline__ void load(const DecodeArgs& a) { load(a, kv_len(a.c, b)); }
  __device__ __forceinline__ void load(const DecodeArgs& a, int tokens) {
    n = tokens;
    seen = seen_keys(n - 1, n - 1, a.window, a.sinks);
    nv = seen.count();
    turns = ceil_div(nv, DT);
  }
  __device__ __forceinline__ void next_pair(const DecodeArgs& a) {
    t = 0;
    if (++h < a.c.Hkv) return;
    h = 0;
    do {
      if (++b >= a.c.B) return;
      load(a);
    } while (turns == 0);
  }
  __device__ __forceinline__ void next(const DecodeArgs& a, int step) {
    if ((t += step) >= turns) next_pair(a);
  }
};

// The row of turns as a warp sees it: each lane counts the turns of `cs` consecutive
// sequences, `before` lie before them.
struct TurnRow {
  int cs, before, all, per;  // per: turns of a warp's run
  int n;                     // tokens of the lane's last sequence
  __device__ __forceinline__ TurnRow(const DecodeArgs& a) {
    const int lane = threadIdx.x & 31;
    cs = ceil_div(a.c.B, 32);
    const int b0 = min(a.c.B, lane * cs), b1 = min(a.c.B, b0 + cs);
    int mine = 0;
    n = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) {
      n = kv_len(a.c, b);
      mine += ceil_div(seen_keys(n - 1, n - 1, a.window, a.sinks).count(), DT);
    }
    mine *= a.c.Hkv;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(FULL, sum, o);
      if (lane >= o) sum += y;
    }
    all = __shfl_sync(FULL, sum, 31);
    before = sum - mine;
    per = max(ceil_div(all, a.warps), 1);
  }
  __device__ __forceinline__ void find(const DecodeArgs& a, int at, Walk* w) const {
    const int lo = __popc(__ballot_sync(FULL, before <= at)) - 1;
    w->b = lo * cs;
    int u = at - __shfl_sync(FULL, before, lo);
    if (cs == 1) {
      w->load(a, __shfl_sync(FULL, n, lo));
    } else {
      for (;; ++w->b) {
        w->load(a);
        const int here = w->turns * a.c.Hkv;
        if (u < here) break;
        u -= here;
      }
    }
    w->h = u / w->turns;
    w->t = u - w->h * w->turns;
  }
  // The first turn of sequence b, and its walk.
  __device__ __forceinline__ int first(const DecodeArgs& a, int b, Walk* w) const {
    int u = __shfl_sync(FULL, before, b / cs);
    const int tokens = __shfl_sync(FULL, n, b / cs);
    if (cs == 1) {
      w->b = b;
      w->load(a, tokens);
      return u;
    }
    for (w->b = b / cs * cs; w->b < b; ++w->b) {
      w->load(a);
      u += w->turns * a.c.Hkv;
    }
    w->load(a);
    return u;
  }
};

// ---- copies ----------------------------------------------------------------------------
// A lane's row of a turn, the key's and the value's alike: lanes r and r + 16 hold place
// r of the turn.  The page number is only loaded here; Ring::fill looks at it a turn later.
struct Row {
  enum { NONE, PAGE, FIXED } kind;  // past the end; in the cache; the appended row, which
                                    // the caller has
  unsigned rest;                    // 16-byte pieces inside the page
  int page;
  __device__ __forceinline__ void look_up(const DecodeArgs& a, const Walk& w, int lane) {
    const int x = w.t * DT + (lane & 15);
    kind = NONE;
    page = 0;
    rest = 0;
    if (x >= w.nv) return;
    const int j = w.seen.place(x);
    if (a.k_new && j == w.n - 1) {
      kind = FIXED;
      return;
    }
    kind = PAGE;
    const unsigned p = (unsigned)j / (unsigned)a.c.ps, s = (unsigned)j - p * (unsigned)a.c.ps;
    rest = w.h * a.head16 + s * a.slot16;
    page = a.c.table[(long long)w.b * a.c.max_pages + p];
  }
};

// A warp's ring: stages of 16 keys' and 16 values' rows.  Piece p (16 bytes) of row r
// lies at p ^ (r & 7), so that reads down a column of rows meet no bank twice.
template <int ROWB, int NST> struct Ring {
  static constexpr int STAGE = 2 * DT * ROWB;
  static constexpr int P = ROWB / 16, RPI = P >= 32 ? 1 : 32 / P;  // pieces, rows a copy
  char* at;
  int put, got;  // stages filled and used, modulo NST
  // The next stage takes the turn that `row` was looked up for; rows past the end and
  // pieces past d become zeros.
  __device__ __forceinline__ void fill(const DecodeArgs& a, const Row& row, int b, int h, int lane,
                                       int rowbytes) {
    const int sub = P >= 32 ? 0 : lane / P, pc = P >= 32 ? lane : lane % P;
    char* base = at + put * STAGE + sub * ROWB;
    const int xp = (pc ^ sub) * 16;  // rows r0 + sub with r0 a multiple of RPI
    const bool there = row.kind == Row::PAGE && (unsigned)row.page < (unsigned)a.c.num_pages;
    if (row.kind == Row::PAGE && !there) set_status(a.c.status, CACHE_BAD);
    if (__all_sync(FULL, there) && a.page16 != 0) {  // offsets of 16-byte pieces fit 32 bits
      const unsigned off = row.page * a.page16 + row.rest;
#pragma unroll
      for (int r0 = 0; r0 < DT; r0 += RPI) {
        const unsigned o = __shfl_sync(FULL, off, r0 + sub);
        char* dst = base + r0 * ROWB + (xp ^ ((r0 & 7) * 16));
#pragma unroll
        for (int p0 = 0; p0 < P; p0 += 32) {
          const bool ok = (pc + p0) * 16 < rowbytes;
          const size_t x = (size_t)(o + (ok ? pc + p0 : 0)) * 16;
          cp_async16(dst + p0 * 16, a.c.k + x, ok);
          cp_async16(dst + DT * ROWB + p0 * 16, a.c.v + x, ok);
        }
      }
    } else {
      const int esize = rowbytes / a.c.d;
      const char *kp = nullptr, *vp = nullptr;
      if (row.kind == Row::FIXED) {
        const long long x = ((long long)b * a.c.Hkv + h) * rowbytes;
        kp = a.k_new + x;
        vp = a.v_new + x;
      } else if (there) {
        const long long x = row.page * a.c.page_stride * esize + (long long)row.rest * 16;
        kp = a.c.k + x;
        vp = a.c.v + x;
      }
#pragma unroll 1
      for (int r0 = 0; r0 < DT; r0 += RPI) {
        const char* k = (const char*)__shfl_sync(FULL, (unsigned long long)kp, r0 + sub);
        const char* v = (const char*)__shfl_sync(FULL, (unsigned long long)vp, r0 + sub);
        char* dst = base + r0 * ROWB + (xp ^ ((r0 & 7) * 16));
        for (int p0 = 0; p0 < P; p0 += 32) {
          const bool ok = k != nullptr && (pc + p0) * 16 < rowbytes;
          cp_async16(dst + p0 * 16, ok ? k + (pc + p0) * 16 : a.c.k, ok);
          cp_async16(dst + DT * ROWB + p0 * 16, ok ? v + (pc + p0) * 16 : a.c.v, ok);
        }
      }
    }
    put = put + 1 == NST ? 0 : put + 1;
  }
  __device__ __forceinline__ const char* take() {
    const char* p = at + got * STAGE;
    got = got + 1 == NST ? 0 : got + 1;
    return p;
  }
};

// The appended row goes to its page: the warp that has the pair's last turn.
__device__ __forceinline__ void append_new(const DecodeArgs& a, const Walk& w, int esize,
                                           int lane) {
  const long long o = kv_row(a.c, w.b, w.h, w.n - 1);
  if (o < 0) return;
  const long long src = ((long long)w.b * a.c.Hkv + w.h) * a.c.d;
  for (int x = lane; x < a.c.d * esize / 16; x += 32) {
    *(int4*)(a.c.k + o * esize + x * 16) = *(const int4*)(a.k_new + src * esize + x * 16);
    *(int4*)(a.c.v + o * esize + x * 16) = *(const int4*)(a.v_new + src * esize + x * 16);
  }
}

// Logits of a pair's turn, [key][heads of a launch].
__device__ __forceinline__ float* logits_of(const DecodeArgs& a, const Walk& w) {
  return a.logits + (((long long)w.b * a.c.Hkv + w.h) * a.places + w.t * DT) * a.hs;
}

// ---- the query heads of a warp -----------------------------------------------------------
// bf16: up to 16 query heads are the rows of mma m16n8k16 (fp32 accumulation); the
// keys' and values' fragments come from the ring by ldmatrix.  The products are far
// from the bound (48 instructions per 16 keys), so the rows that G leaves idle cost
// nothing that shows.
template <int DP> struct HeadsBf16 {
  static constexpr int HM = 16, EXTRA = 0;  // shared memory of its own, a warp
  static constexpr int CTAS = 0;  // an SM, for the registers: left to the compiler
  typedef __nv_bfloat16 T;
  uint32_t qf[DP / 16][4];
  float o[DP / 8][4], m[2], l[2];
  __device__ __forceinline__ void begin(const DecodeArgs& a, const Walk& w, char*, int lane) {
    // fragments: rows lane/4 and lane/4 + 8
    const int g0 = lane >> 2, c0 = (lane & 3) * 2;
    const T* q = reinterpret_cast<const T*>(a.q) + w.b * a.q_row +
                 (long long)(w.h * a.G + a.h0) * a.q_head;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int g = g0 + (x & 1) * 8, col = ks * 16 + c0 + (x >> 1) * 8;
        qf[ks][x] = g < a.heads && col < a.c.d
                        ? *reinterpret_cast<const uint32_t*>(q + g * a.q_head + col)
                        : 0u;
      }
#pragma unroll
    for (int x = 0; x < DP / 8; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  __device__ __forceinline__ void turn(const DecodeArgs& a, const Walk& w, const char* stage,
                                       char*, int lane) {
    constexpr int ROWB = DP * 2;
    const uint32_t kb = (uint32_t)__cvta_generic_to_shared(stage), vb = kb + DT * ROWB;
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    {
      float s2[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};  // shorter chains
      const int r = ((lane >> 4) << 3) + (lane & 7);
      const uint32_t at = kb + r * ROWB + ((((lane >> 3) & 1) ^ (lane & 7)) * 16);
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) {
        uint32_t x[4];
        ldsm4(x, at ^ (ks * 32));
        mma16816(ks & 1 ? s2[0] : s[0], qf[ks], x[0], x[1]);
        mma16816(ks & 1 ? s2[1] : s[1], qf[ks], x[2], x[3]);
      }
      // logits in powers of two; places past the end leave
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int y = 0; y < 4; ++y) s[nt][y] = (s[nt][y] + s2[nt][y]) * a.scale2;
      if (w.t == w.turns - 1) {
        const int x0 = w.t * DT + (lane & 3) * 2;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (x0 + nt * 8 + (y & 1) >= w.nv) s[nt][y] = -INFINITY;
      }
    }
    if (a.scores) {
      float* lg = logits_of(a, w) + (lane & 3) * 2 * a.hs + (lane >> 2);
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if ((lane >> 2) + (y >> 1) * 8 < a.hs)
            lg[(nt * 8 + (y & 1)) * a.hs + (y >> 1) * 8] = s[nt][y];
    }
    // the maximum that weights are taken against follows the running one when that has
    // grown by 2^8: the output is hardly ever rescaled, and weights up to 256 lose nothing
    float top[2];
    bool grew = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
      x = fmaxf(x, __shfl_xor_sync(FULL, x, 1));
      top[r] = fmaxf(x, __shfl_xor_sync(FULL, x, 2));
      grew |= top[r] > m[r] + 8.f || (m[r] == -INFINITY && top[r] > m[r]);
    }
    if (__any_sync(FULL, grew)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float mn = fmaxf(m[r], top[r]);
        const float x = exp2_fast(m[r] - (mn == -INFINITY ? 0.f : mn));
        l[r] *= x;
#pragma unroll
        for (int y = 0; y < DP / 8; ++y) {
          o[y][2 * r] *= x;
          o[y][2 * r + 1] *= x;
        }
        m[r] = mn;
      }
    }
    const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        s[nt][y] = exp2_fast(s[nt][y] - base[y >> 1]);
        l[y >> 1] += s[nt][y];
      }
    // the weights as two bf16 terms (relative error 2^-17), each multiplied with the
    // values: the second product hides behind the copies, and the output then carries its
    // own rounding only
    uint32_t pf[4], pl[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float p0 = s[x >> 1][(x & 1) * 2], p1 = s[x >> 1][(x & 1) * 2 + 1];
      pf[x] = pack_bf16(p0, p1);
      pl[x] = pack_bf16(p0 - __uint_as_float(pf[x] << 16),
                        p1 - __uint_as_float(pf[x] & 0xffff0000u));
    }
    const int r = (((lane >> 3) & 1) << 3) + (lane & 7);
    const uint32_t at = vb + r * ROWB + (((lane >> 4) ^ (lane & 7)) * 16);
#pragma unroll
    for (int c = 0; c < DP / 16; c += 2) {  // two pieces at a time: longer ways between sums
      uint32_t x[8];
      ldsm4t(x, at ^ (c * 32));
      ldsm4t(x + 4, at ^ (c * 32 + 32));
#pragma unroll
      for (int y = 0; y < 4; ++y) mma16816(o[2 * c + y], pf, x[2 * y], x[2 * y + 1]);
#pragma unroll
      for (int y = 0; y < 4; ++y) mma16816(o[2 * c + y], pl, x[2 * y], x[2 * y + 1]);
    }
  }
  // Maxima and sums, and the unnormalised output rows [heads][DP].
  __device__ __forceinline__ void leave(const DecodeArgs& a, float2* ml, float* out, int lane) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(FULL, l[r], 1);
      l[r] += __shfl_xor_sync(FULL, l[r], 2);
      const int g = (lane >> 2) + 8 * r;
      if (g < a.heads) {
        if ((lane & 3) == 0) ml[g] = make_float2(m[r], l[r]);
#pragma unroll
        for (int x = 0; x < DP / 8; ++x)
          *reinterpret_cast<float2*>(out + g * DP + (lane & 3) * 2 + x * 8) =
              make_float2(o[x][2 * r], o[x][2 * r + 1]);
      }
    }
  }
};

// fp32 on the CUDA cores, up to HM query heads a launch: a lane holds half a key's row
// for the products with q, and 4 columns of the output (or 2 x 4) for those with v.
template <int DP, int HM_> struct HeadsF32 {
  static constexpr int HM = HM_, EXTRA = (HM * DP + DT * HM) * 4;
  static constexpr int CTAS = 1;  // an SM: all registers (16 sequences of 4,000 keys, 7
                                  // heads a key head: 77 us, 93 with 168 a thread)
  typedef float T;
  static constexpr int ROWB = DP * 4, P = DP / 4;
  static constexpr int NC = P >= 32 ? P / 32 : 1;  // output pieces of a lane
  static constexpr int KS = P >= 32 ? 1 : 32 / P;  // lanes that share a piece, alternate keys
  f32x2 o[HM][NC * 2];  // columns in pairs
  float m[HM], l[HM];
  __device__ __forceinline__ void begin(const DecodeArgs& a, const Walk& w, char* extra,
                                        int lane) {
    float* qw = reinterpret_cast<float*>(extra);
    const float* q = reinterpret_cast<const float*>(a.q) + w.b * a.q_row +
                     (long long)(w.h * a.G + a.h0) * a.q_head;
    for (int x = lane; x < HM * DP; x += 32) {
      const int g = x / DP, y = x - g * DP;
      qw[x] = g < a.heads && y < a.c.d ? q[g * a.q_head + y] : 0.f;
    }
#pragma unroll
    for (int g = 0; g < HM; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int x = 0; x < NC * 2; ++x) o[g][x] = 0ull;
    }
    __syncwarp();
  }
  __device__ __forceinline__ void turn(const DecodeArgs& a, const Walk& w, const char* kb,
                                       char* extra, int lane) {
    const float* qw = reinterpret_cast<float*>(extra);
    float* pw = reinterpret_cast<float*>(extra) + HM * DP;
    const char* vb = kb + DT * ROWB;
    const int key = lane & 15, half = lane >> 4;
    float s[HM];
    {
      f32x2 z[HM];  // sums over even and odd columns
#pragma unroll
      for (int g = 0; g < HM; ++g) z[g] = 0ull;
#pragma unroll 4
      for (int c = 0; c < P / 2; ++c) {
        const int pc = half * (P / 2) + c;
        const ulonglong2 kv =
            *reinterpret_cast<const ulonglong2*>(kb + key * ROWB + ((pc ^ (key & 7)) * 16));
#pragma unroll
        for (int g = 0; g < HM; ++g) {
          const ulonglong2 qv = *reinterpret_cast<const ulonglong2*>(qw + g * DP + pc * 4);
          z[g] = fma2(qv.y, kv.y, fma2(qv.x, kv.x, z[g]));
        }
      }
#pragma unroll
      for (int g = 0; g < HM; ++g) {
        const float2 v = unpair(z[g]);
        s[g] = v.x + v.y;
      }
    }
    const bool in = w.t * DT + key < w.nv;
#pragma unroll
    for (int g = 0; g < HM; ++g) {
      s[g] += __shfl_xor_sync(FULL, s[g], 16);
      s[g] = in ? s[g] * a.scale2 : -INFINITY;
      if (a.scores && half == 0 && g < a.hs) logits_of(a, w)[key * a.hs + g] = s[g];
      float mx = s[g];
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, x));
      const float mn = fmaxf(m[g], mx), base = mn == -INFINITY ? 0.f : mn;
      if (mn > m[g]) {  // the same in every lane
        const float x = exp2_fast(m[g] - base);
        l[g] *= x;
#pragma unroll
        for (int y = 0; y < NC * 2; ++y) o[g][y] = mul2(o[g][y], pair(x, x));
        m[g] = mn;
      }
      const float p = exp2_fast(s[g] - base);
      l[g] += half == 0 ? p : 0.f;
      if (half == 0) pw[key * HM + g] = p;
    }
    __syncwarp();
    const int piece = P >= 32 ? lane : lane % P, sub = P >= 32 ? 0 : lane / P;
#pragma unroll 4
    for (int k = sub; k < DT; k += KS) {
      float p[HM];
      if constexpr (HM % 4 == 0) {
#pragma unroll
        for (int g = 0; g < HM; g += 4)
          *reinterpret_cast<float4*>(p + g) = *reinterpret_cast<const float4*>(pw + k * HM + g);
      } else {
#pragma unroll
        for (int g = 0; g < HM; ++g) p[g] = pw[k * HM + g];
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int pc = piece + c * 32;
        const ulonglong2 vv =
            *reinterpret_cast<const ulonglong2*>(vb + k * ROWB + ((pc ^ (k & 7)) * 16));
#pragma unroll
        for (int g = 0; g < HM; ++g) {
          const f32x2 pp = pair(p[g], p[g]);
          o[g][2 * c] = fma2(pp, vv.x, o[g][2 * c]);
          o[g][2 * c + 1] = fma2(pp, vv.y, o[g][2 * c + 1]);
        }
      }
    }
  }
  __device__ __forceinline__ void leave(const DecodeArgs& a, float2* ml, float* out, int lane) {
#pragma unroll
    for (int g = 0; g < HM; ++g) {
      const float L = warp_sum(l[g]);
      if (KS > 1) {
#pragma unroll
        for (int x = P; x < 32; x <<= 1)
#pragma unroll
          for (int y = 0; y < NC * 2; ++y)
            o[g][y] = add2(o[g][y], __shfl_xor_sync(FULL, o[g][y], x));
      }
      if (g < a.heads) {
        if (lane == 0) ml[g] = make_float2(m[g], L);
        if (P >= 32 || lane < P)
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const float2 lo = unpair(o[g][2 * c]), hi = unpair(o[g][2 * c + 1]);
            *reinterpret_cast<float4*>(out + g * DP + (lane + c * 32) * 4) =
                make_float4(lo.x, lo.y, hi.x, hi.y);
          }
      }
    }
  }
};

// ---- joining -------------------------------------------------------------------------------
// The parts of a pair whose turns are u0 .. u0 + turns - 1 of the row: one of every CTA
// that has nothing else, one of every warp's run in the others.  Runs and pairs both only
// grow along the row, so the sum of their numbers numbers the parts' places.
struct Parts {
  int run0, n0, run1, mid, run2, count, W;
  long long pair;
  bool whole;  // one CTA had it all: its output is written
  __device__ __forceinline__ Parts(const TurnRow& r, int W_, int u0, int turns, long long pair_) {
    W = W_;
    pair = pair_;
    const int cta = W * r.per, u1 = u0 + turns;
    const int c0 = u0 / cta, c1 = (u1 - 1) / cta;
    int n, first;
    auto of = [&](int c) {
      const int lo = c * cta, hi = r.all - lo < cta ? r.all : lo + cta;
      const bool one = lo >= u0 && hi <= u1;
      first = one ? 0 : (max(u0, lo) - lo) / r.per;
      n = one ? 1 : (min(u1, hi) - 1 - lo) / r.per - first + 1;
      return one;
    };
    const bool one = of(c0);
    run0 = c0 * W + first;
    n0 = n;
    whole = one && c0 == c1;
    run1 = (c0 + 1) * W;
    mid = max(0, c1 - c0 - 1);
    n = 0;
    if (c1 > c0) of(c1);
    run2 = c1 * W;
    count = n0 + mid + n;
  }
  __device__ __forceinline__ long long place(int x) const {
    return pair + (x < n0 ? run0 + x : x < n0 + mid ? run1 + (x - n0) * W : run2 + x - n0 - mid);
  }
};

__device__ __forceinline__ float2 final_ml(float M, float L) {
  return make_float2(M, L == 0.f ? 0.f : 1.f / L);
}
template <typename T>
__device__ __forceinline__ void write_head(const DecodeArgs& a, int b, int h, int g, int y, float4 s,
                                           float inv) {
  if (y >= a.c.d) return;
  T* out = reinterpret_cast<T*>(a.out) + b * a.o_row +
           (long long)(h * a.G + a.h0 + g) * a.o_head + y;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv);
  } else {
    *reinterpret_cast<uint2*>(out) =
        make_uint2(pack_bf16(s.x * inv, s.y * inv), pack_bf16(s.z * inv, s.w * inv));
  }
}
__device__ __forceinline__ void write_lse(const DecodeArgs& a, int b, int h, int g, float M,
                                          float L) {
  if (a.lse)
    a.lse[(long long)b * a.H + h * a.G + a.h0 + g] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
}

__device__ __forceinline__ void fetch_l1(const void* p) {
  asm volatile("prefetch.global.L1 [%0];" ::"l"(p));
}

// out_scores of a pair's places x0, x0 + step, .. from its logits and final maxima and sums.
__device__ __forceinline__ void add_scores(const DecodeArgs& a, const Walk& w, const float2* ml,
                                           int x0, int step) {
  const long long pair = (long long)w.b * a.c.Hkv + w.h;
  const float* in = a.scores + pair * a.score_stride;
  float* out = a.out_scores + pair * a.score_stride;
  const float* lg = a.logits + pair * a.places * a.hs;
#pragma unroll 4
  for (int x = x0; x < w.nv; x += step) {
    const int j = w.seen.place(x);
    float s = 0.f;
    if (a.hs >= 4) {
      for (int g = 0; g < a.heads; g += 4) {
        const float4 v = *reinterpret_cast<const float4*>(lg + (long long)x * a.hs + g);
        s += exp2_fast(v.x - ml[g].x) * ml[g].y;
        if (g + 1 < a.heads) s += exp2_fast(v.y - ml[g + 1].x) * ml[g + 1].y;
        if (g + 2 < a.heads) s += exp2_fast(v.z - ml[g + 2].x) * ml[g + 2].y;
        if (g + 3 < a.heads) s += exp2_fast(v.w - ml[g + 3].x) * ml[g + 3].y;
      }
    } else {
      for (int g = 0; g < a.heads; ++g)
        s += exp2_fast(lg[(long long)x * a.hs + g] - ml[g].x) * ml[g].y;
    }
    out[j] = (a.fresh && j == w.n - 1 ? 0.f : in[j]) + s;
  }
  if (in != out)  // unseen keys keep what they had
    for (int j = w.seen.a + x0; j < w.seen.b0; j += step) out[j] = in[j];
}

template <class H, int DP, int W, int NST> constexpr size_t decode_smem() {
  return (size_t)W * (NST * Ring<DP * sizeof(typename H::T), NST>::STAGE + H::EXTRA +
                      H::HM * sizeof(float2));
}

// OWN: a CTA takes a whole pair, and no other.
template <class H, int DP, int W, int NST, bool OWN>
__global__ void __launch_bounds__(W * 32, H::CTAS) k_decode(DecodeArgs a) {
  typedef typename H::T T;
  typedef Ring<DP * sizeof(T), NST> R;
  constexpr int HM = H::HM, ES = sizeof(T);
  static_assert(NST * R::STAGE >= HM * DP * 4, "a warp's ring holds its output rows");
  extern __shared__ __align__(512) char smem[];
  __shared__ float2 fin[OWN ? 16 : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  char* extra = smem + W * NST * R::STAGE + warp * H::EXTRA;
  float2* ml = reinterpret_cast<float2*>(smem + W * (NST * R::STAGE + H::EXTRA));  // [W][HM]
  grid_dep_wait();
  grid_dep_launch();  // not before: k_decode_join reads the lengths ahead of its own wait
  Walk w;
  int at, count, u, end, step = W;  // this warp's turns: u, u + step, .. below end
  bool one, whole;                  // all of the CTA's are of one pair; all the pair's
  if constexpr (OWN) {
    w.b = blockIdx.x / a.c.Hkv;
    w.h = blockIdx.x - w.b * a.c.Hkv;
    w.t = 0;
    w.load(a);
    at = 0;
    count = w.turns;
    one = whole = true;
    if (count == 0) {  // it sees nothing
      for (int x = tid; x < a.heads * (DP / 4); x += W * 32) {
        const int g = x / (DP / 4), y = (x - g * (DP / 4)) * 4;
        write_head<T>(a, w.b, w.h, g, y, make_float4(0.f, 0.f, 0.f, 0.f), 0.f);
        if (y == 0) write_lse(a, w.b, w.h, g, 0.f, 0.f);
      }
      return;
    }
    w.t = u = warp;
    end = count;
  } else {
    const TurnRow turns(a);
    const int cta = W * turns.per;
    at = turns.all / cta < (int)blockIdx.x ? turns.all : (int)blockIdx.x * cta;
    count = min(cta, turns.all - at);
    if (count <= 0) return;
    turns.find(a, at, &w);
    one = w.t + count <= w.turns;
    whole = one && count == w.turns;
    u = at + warp;
    end = at + count;
    if (one) {
      w.t += warp;
    } else {
      u = at + warp * turns.per;
      end = min(end, u + turns.per);
      step = 1;
      if (u < end) turns.find(a, u, &w);
    }
  }
  const int pair0 = w.b * a.c.Hkv + w.h;
  const int b0 = w.b, h0 = w.h;
  if (u < end) {
    H heads;
    R ring{smem + warp * NST * R::STAGE, 0, 0};
    const int rowbytes = a.c.d * ES, run = (int)blockIdx.x * W + warp;
    heads.begin(a, w, extra, lane);
    Walk f = w;  // the turn whose pages are looked up
    Row row;
    row.look_up(a, f, lane);
    int fu = u, ahead = 0;
#pragma unroll 1
    while (true) {
      if (fu < end) {  // into the stage that the turn before has left
        ring.fill(a, row, f.b, f.h, lane, rowbytes);
        if ((fu += step) < end) {
          f.next(a, step);
          row.look_up(a, f, lane);
        }
      }
      cp_async_commit();
      if (++ahead < NST) continue;
      cp_async_wait<NST - 1>();
      __syncwarp();
      heads.turn(a, w, ring.take(), extra, lane);
      __syncwarp();  // every lane has read the stage
      const bool last = w.t == w.turns - 1;
      if (last && a.k_new) append_new(a, w, ES, lane);
      u += step;
      if (u < end && !last) {
        w.t += step;
        continue;
      }
      // the run or the pair ends
      const long long part = (long long)run + w.b * a.c.Hkv + w.h;
      if (one)
        heads.leave(a, ml + warp * HM, reinterpret_cast<float*>(ring.at), lane);
      else
        heads.leave(a, a.ml + part * a.heads, a.part + part * a.heads * DP, lane);
      if (u >= end) break;
      w.next_pair(a);
      __syncwarp();
      heads.begin(a, w, extra, lane);
    }
  }
  if (!one) return;
  // one pair: the warps' outputs become the CTA's
  __syncthreads();
  const int nw = min(W, count);
  const long long part = (long long)blockIdx.x * W + pair0;
  for (int x = tid; x < a.heads * (DP / 4); x += W * 32) {
    const int g = x / (DP / 4), y = (x - g * (DP / 4)) * 4;
    float M = -INFINITY, L = 0.f;
    float2 v[W];
#pragma unroll
    for (int q = 0; q < W; ++q) {
      v[q] = q < nw ? ml[q * HM + g] : make_float2(-INFINITY, 0.f);
      M = fmaxf(M, v[q].x);
    }
    const float base = M == -INFINITY ? 0.f : M;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < W; ++q) {
      if (q >= nw) break;
      const float f = exp2_fast(v[q].x - base);
      const float4 z =
          *reinterpret_cast<const float4*>(smem + q * NST * R::STAGE + (g * DP + y) * 4);
      L = fmaf(v[q].y, f, L);
      o.x = fmaf(z.x, f, o.x);
      o.y = fmaf(z.y, f, o.y);
      o.z = fmaf(z.z, f, o.z);
      o.w = fmaf(z.w, f, o.w);
    }
    if (whole) {
      write_head<T>(a, b0, h0, g, y, o, final_ml(base, L).y);
      if (y == 0) write_lse(a, b0, h0, g, base, L);
    } else {
      *reinterpret_cast<float4*>(a.part + (part * a.heads + g) * DP + y) = o;
    }
    if (y == 0) {
      if constexpr (OWN)
        fin[g] = final_ml(base, L);
      else
        a.ml[part * a.heads + g] = make_float2(M, L);
    }
  }
  if (OWN && a.scores) {
    __syncthreads();
    add_scores(a, w, fin, tid, W * 32);
  }
}

// Maximum (0 where there is none) and sum over a pair's parts of query head g, a warp.
__device__ __forceinline__ float2 join_ml(const DecodeArgs& a, const Parts& p, int g, int lane) {
  float M = -INFINITY, L = 0.f;
  for (int x = lane; x < p.count; x += 32) {
    const float2 v = a.ml[p.place(x) * a.heads + g];
    const float mn = fmaxf(M, v.x), base = mn == -INFINITY ? 0.f : mn;
    L = L * exp2_fast(M - base) + v.y * exp2_fast(v.x - base);
    M = mn;
  }
  const float top = warp_max(M), base = top == -INFINITY ? 0.f : top;
  return make_float2(base, warp_sum(L * exp2_fast(M - base)));
}

// The parts of every query head joined, a warp each (the first blocks), and the scores,
// `blocks` CTAs a pair.
constexpr int JN_WARPS = 8, JN_THREADS = JN_WARPS * 32;
constexpr int JN_AHEAD = 8;  // places of a thread that are fetched before the sums are joined
template <typename T>
__global__ void __launch_bounds__(JN_THREADS) k_decode_join(DecodeArgs a, int W, int dp,
                                                            int out_blocks, int blocks) {
  __shared__ float2 fin[16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // Every CTA of k_decode was past its wait before this kernel could start: what ran before
  // k_decode is complete, and the lengths, which k_decode does not write, can be read (from
  // L2: kv_len) while it works.  Its parts, sums and logits are read after the wait.
  grid_dep_launch();
  const TurnRow row(a);
  Walk w;
  if ((int)blockIdx.x < out_blocks) {
    const int x = blockIdx.x * JN_WARPS + warp, pair = x / a.heads, g = x - pair * a.heads;
    if (pair >= a.c.B * a.c.Hkv) return;
    const int b = pair / a.c.Hkv;
    w.h = pair - b * a.c.Hkv;
    const int u = row.first(a, b, &w) + w.h * w.turns;
    const Parts p(row, W, u, w.turns, pair);
    grid_dep_wait();
    if (w.turns == 0) {  // it sees nothing
      for (int y = lane * 4; y < dp; y += 128)
        write_head<T>(a, b, w.h, g, y, make_float4(0.f, 0.f, 0.f, 0.f), 0.f);
      if (lane == 0) write_lse(a, b, w.h, g, 0.f, 0.f);
      return;
    }
    if (p.whole) return;
    for (int y = lane * 4; y < dp; y += 128) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float M = -INFINITY, L = 0.f;
      for (int q0 = 0; q0 < p.count; q0 += 8) {  // eight parts' loads in flight
        float4 z[8];
        float2 v[8];
        float top = M;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const long long at = p.place(min(q0 + q, p.count - 1)) * a.heads + g;
          z[q] = *reinterpret_cast<const float4*>(a.part + at * dp + y);
          v[q] = a.ml[at];
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (q0 + q >= p.count) v[q] = make_float2(-INFINITY, 0.f);
          top = fmaxf(top, v[q].x);
        }
        const float base = top == -INFINITY ? 0.f : top, old = exp2_fast(M - base);
        M = top;
        L *= old;
        o = make_float4(o.x * old, o.y * old, o.z * old, o.w * old);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float x = exp2_fast(v[q].x - base);
          L = fmaf(v[q].y, x, L);
          if (q0 + q >= p.count) continue;
          o.x = fmaf(z[q].x, x, o.x);
          o.y = fmaf(z[q].y, x, o.y);
          o.z = fmaf(z[q].z, x, o.z);
          o.w = fmaf(z[q].w, x, o.w);
        }
      }
      if (M == -INFINITY) M = 0.f;
      write_head<T>(a, b, w.h, g, y, o, final_ml(M, L).y);
      if (y == 0) write_lse(a, b, w.h, g, M, L);
    }
    return;
  }
  const int x = blockIdx.x - out_blocks, pair = x / blocks, b = pair / a.c.Hkv;
  w.h = pair - b * a.c.Hkv;
  const int u = row.first(a, b, &w) + w.h * w.turns;
  const int x0 = (x - pair * blocks) * JN_THREADS;
  const Parts p(row, W, u, w.turns, pair);
  grid_dep_wait();
  if (w.turns == 0) return;
  // this thread's logits and scores on their way while the sums are joined
#pragma unroll
  for (int i = 0; i < JN_AHEAD; ++i) {
    const int y = x0 + (int)threadIdx.x + i * blocks * JN_THREADS;
    if (y >= w.nv) break;
    fetch_l1(a.logits + ((long long)pair * a.places + y) * a.hs);
    fetch_l1(a.scores + (long long)pair * a.score_stride + w.seen.place(y));
  }
  for (int g = warp; g < a.heads; g += JN_WARPS) {
    const float2 v = join_ml(a, p, g, lane);
    if (lane == 0) fin[g] = final_ml(v.x, v.y);
  }
  __syncthreads();
  add_scores(a, w, fin, x0 + threadIdx.x, blocks * JN_THREADS);
}

// Query heads of a launch; key heads that have more take one launch after another.
int heads_per_launch(int dtype, int G) {
  return dtype == GMC_BF16 ? std::min(G, 16) : G > 4 ? std::min(G, 8) : G;
}
// Floats of a key's logits: whole 16-byte pieces, as many as rows hold them.
int logit_heads(int dtype, int G) {
  const int h = heads_per_launch(dtype, G);
  return h > 8 ? 16 : h > 4 ? 8 : h > 2 ? 4 : h;
}
int decode_dp(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

constexpr int D_WARPS = 8;  // of a CTA, at most; one CTA an SM

struct DecodeWs {
  size_t ml, part, logits, all;
};
DecodeWs decode_carve(const KV& c, int dtype, int H) {
  const int G = H / c.Hkv, heads = heads_per_launch(dtype, G);
  const size_t pairs = (size_t)c.B * c.Hkv, parts = pairs + (size_t)sm_count() * D_WARPS;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  DecodeWs w;
  w.ml = 0;
  w.part = up(parts * heads * 8);
  w.logits = w.part + up(parts * heads * decode_dp(c.d) * 4);
  w.all = w.logits + pairs * logit_heads(dtype, G) * 4 * (size_t)(ceil_div(c.cap, DT) * DT);
  return w;
}

template <class H, int DP, int W, int NST>
cudaError_t decode_launch(DecodeArgs a, cudaStream_t st, int* launches) {
  static_assert(W <= D_WARPS, "the workspace holds a part a warp");
  constexpr size_t smem = decode_smem<H, DP, W, NST>();
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  const int ctas = sm_count();
  const int pairs = a.c.B * a.c.Hkv;
  // A CTA a pair where that is a few turns a warp: no parts, no second launch.  32 sequences
  // of 512 keys and 4 key heads: 10.1 us, in stretches 11.3; with scores 12.6 and 14.7.  A
  // single sequence of 322 takes 9.0, in stretches 8.3, but its call 9.1 instead of 10.4:
  // the second launch is what the host takes time for; of 768 keys 14.0 and 8.3.
  const int most = ceil_div(a.c.cap, W * DT);
  const bool own = pairs <= ctas && most <= (2 * pairs >= ctas ? 6 : 3);
  a.warps = ctas * W;
  auto kernel = own ? k_decode<H, DP, W, NST, true> : k_decode<H, DP, W, NST, false>;
  cudaError_t e = set_smem_limit((const void*)kernel, smem);
  if (e != cudaSuccess) return e;
  if ((e = launch_k(kernel, dim3(own ? pairs : ctas), dim3(W * 32), smem, st, 1, a)) !=
      cudaSuccess)
    return e;
  ++*launches;
  if (own) return cudaSuccess;
  const int out_blocks = ceil_div(pairs * a.heads, JN_WARPS);
  int blocks = 0;  // of a pair's scores
  if (a.scores) {
    long long most = a.c.cap;
    if (a.window > 0) most = std::min(most, (long long)a.window + a.sinks);
    // two CTAs an SM, one place a thread at least (32 sequences of 2,085 keys: 41.0 us with
    // 256 places a CTA, 38.8 with 2,048; of 512 keys: 14.7 and 15.5)
    blocks = (int)std::min<long long>((most + JN_THREADS - 1) / JN_THREADS,
                                      std::max(1, 2 * ctas / pairs));
  }
  ++*launches;
  return launch_k(k_decode_join<typename H::T>, dim3(out_blocks + pairs * blocks),
                  dim3(JN_THREADS), 0, st, 1, a, W, DP, out_blocks, std::max(blocks, 1));
}
template <int DP, int W, int NST>
cudaError_t decode_f32(int heads, const DecodeArgs& a, cudaStream_t st, int* launches) {
  return heads == 1   ? decode_launch<HeadsF32<DP, 1>, DP, W, NST>(a, st, launches)
         : heads == 2 ? decode_launch<HeadsF32<DP, 2>, DP, W, NST>(a, st, launches)
         : heads <= 4 ? decode_launch<HeadsF32<DP, 4>, DP, W, NST>(a, st, launches)
                      : decode_launch<HeadsF32<DP, 8>, DP, W, NST>(a, st, launches);
}

}  // namespace

size_t decode_workspace(const KV& c, int dtype, int H) { return decode_carve(c, dtype, H).all; }

cudaError_t launch_decode(DecodeArgs a, int dtype, void* ws, cudaStream_t st, int* launches) {
  const int hm = heads_per_launch(dtype, a.G), dp = decode_dp(a.c.d);
  const DecodeWs w = decode_carve(a.c, dtype, a.H);
  a.ml = reinterpret_cast<float2*>((char*)ws + w.ml);
  a.part = reinterpret_cast<float*>((char*)ws + w.part);
  a.logits = reinterpret_cast<float*>((char*)ws + w.logits);
  a.hs = logit_heads(dtype, a.G);
  a.places = ceil_div(a.c.cap, DT) * DT;
  const long long esize = dtype == GMC_BF16 ? 2 : 4;
  const long long page16 = a.c.page_stride * esize / 16, head16 = a.c.head_stride * esize / 16,
                  slot16 = a.c.slot_stride * esize / 16;
  // pieces of 16 bytes from the pools' start: inside a page below 2^32 (gmc_decode checks
  // it), over the pool in all but the largest (page16 = 0: 64-bit offsets)
  a.head16 = (unsigned)head16;
  a.slot16 = (unsigned)slot16;
  a.page16 = page16 * (a.c.num_pages - 1) + head16 * (a.c.Hkv - 1) + slot16 * a.c.ps + 64 <=
                     0xffff0000LL
                 ? (unsigned)page16
                 : 0u;
  for (a.h0 = 0; a.h0 < a.G; a.h0 += hm) {
    a.heads = std::min(hm, a.G - a.h0);
    a.fresh = a.h0 == 0 && a.k_new != nullptr;
    if (a.h0 > 0) a.scores = a.scores ? a.out_scores : nullptr;  // on the launch before's
    cudaError_t e;
    if (dtype == GMC_BF16)
      e = dp == 64    ? decode_launch<HeadsBf16<64>, 64, 8, 4>(a, st, launches)
          : dp == 128 ? decode_launch<HeadsBf16<128>, 128, 8, 3>(a, st, launches)
                      : decode_launch<HeadsBf16<256>, 256, 4, 3>(a, st, launches);
    else
      e = dp == 64    ? decode_f32<64, 8, 3>(hm, a, st, launches)
          : dp == 128 ? decode_f32<128, 4, 3>(hm, a, st, launches)
                      : decode_f32<256, 2, 3>(hm, a, st, launches);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace gmc
