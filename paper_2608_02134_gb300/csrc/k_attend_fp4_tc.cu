// Causal attention of few new tokens a sequence over a cache held in 4 bits, on the tcgen05
// tensor cores (d of 64 and 128): one pass over the codes, which never become rows in memory.
//
// A CTA takes a tile of up to 128 rows, a row being one query head of one token (the G query
// heads of a key head and 128 / G consecutive tokens), and walks the seen keys 64 at a time.
// Four warps copy keys' codes, four values', seven turns ahead into rings of their own, multiply
// them with their scales and write them to shared memory as halves, which hold them exactly, the
// way the tensor cores read them.  One warp issues products; four warps turn the logits of even
// turns into weights, four those of odd ones, a row a thread, with an output and a maximum of
// their own in tensor memory and registers, so that neither waits for the other; the two outputs
// become one at the end.  The queries lie in tensor memory as halves,
// every row multiplied by a power of two that puts its largest value into [2^14, 2^15): what that
// makes too small for a half is 2^-39 of the largest.  Weights are rounded to half (2^-11, of
// small ones 2^-32 of the largest: FP4_UP), their sum is the unrounded ones'.  The base that they
// are taken against follows the running maximum only when that has grown by 2^8; then the output
// in tensor memory is rescaled.
//
// Measured: 16 tokens (28 query heads, 4 key heads of 128) on 8 x 16,004 keys 57 us, on one
// sequence of 16,004 20.  A turn takes 1,450 clocks, at half of the instructions that the SM could
// issue; the codes alone would allow 400.  Without converting and copying it would take 1,050.  On
// the way here, in us of the first: all eight weighing warps on one turn 67, taking turns 65; the
// loads of a turn's codes before its first store 64; rows in runs of a page 63; stores whose lanes
// need not swap halves 60; shared memory by 32-bit addresses 57.  Sixteen copying warps, in 72
// registers, 75 for 64; three or four turns of halves instead of two 60 and 65 for 57 and 63.
//
// Every tile of a sequence converts the same codes again, so this pays for few tiles: `direct` in
// k_attend_fp4.cu says where the rows are unpacked first instead.
//
// Keys that a row does not see get the weight 0.  Rows outside the seen ranges are not read; where
// a block read stands for NaN, the CTA computes its rows again one by one, each from the keys
// that it sees.
//
// Every wait is bounded (about two seconds); on timeout GMC_STATUS_TIMEOUT is set in
// the cache's status word, products in flight are drained and tensor memory is freed.
#include <algorithm>

#include "attend_tc.cuh"
#include "fp4.cuh"

namespace gmc {

namespace {
constexpr int QK = 64;       // keys of a turn
constexpr int Q_WEIGH = 8;   // warps that weigh
constexpr int Q_COPY = 8;    // warps that copy and convert
constexpr int Q_ISSUE = Q_WEIGH + Q_COPY;
constexpr int Q_THREADS = (Q_ISSUE + 1) * 32;
constexpr int Q_RING = 8;    // turns of a copying warp's ring
constexpr int Q_AHEAD = 2;   // turns of keys and values as halves
constexpr int Q_STAGE = 96;  // columns of a turn in tensor memory: 64 logits, 32 of weights

struct QCtl {
  uint64_t kfull[Q_AHEAD], kempty[Q_AHEAD], vfull[Q_AHEAD], vempty[Q_AHEAD];
  uint64_t qfull, sfull[2], pfull[2], ofull, drained;
  float top[2][TM], sum[2][TM];
  uint32_t tmem;
  volatile int abort;
  int strange;
};
constexpr int Q_ROWS = 2 * QK / Q_COPY;  // rows of a copying warp's turn: codes, then their scales
template <int DP> constexpr int Q_PART = Q_ROWS * (DP / 2 + DP / 16);
template <int DP> constexpr size_t q_smem() {
  // the output's rows pass through the keys' and values' place
  const size_t need =
      1024 + 2 * Q_AHEAD * (size_t)QK * DP * 2 + Q_COPY * Q_RING * Q_PART<DP> + sizeof(QCtl);
  // one CTA an SM: a second would wait for tensor memory
  return need > 120 * 1024 ? need : 120 * 1024;
}
// Shared memory by its own addresses: 32 bits, and no detour over generic ones.
template <int BYTES>
__device__ __forceinline__ void cp_async_to(uint32_t smem, const void* src, bool pred) {
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(src),
                 "r"(pred ? 16 : 0)
                 : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(smem), "l"(src), "n"(BYTES),
                 "r"(pred ? BYTES : 0)
                 : "memory");
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds1(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t at, const uint32_t* v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3])
               : "memory");
}
// Two floats as halves, the first one low.
__device__ __forceinline__ uint32_t halves(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
// 16 columns of 32 bits, without the wait.
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15])
      : "memory");
}
// The two warps of a lane quarter meet.
__device__ __forceinline__ void meet(int quarter) {
  asm volatile("bar.sync %0, 64;" ::"r"(quarter + 1) : "memory");
}

// One row from the keys j0 .. j1 - 1 that it sees, a warp a row: four channels a lane.
__device__ __noinline__ void row_alone4(const AttnArgs& a, int b, int h, long long row, int hq,
                                        int place, int j0, int j1, float* m_, float* l_,
                                        float o[4]) {
  const int lane = threadIdx.x & 31, x = lane * 4;
  float q[4] = {0.f, 0.f, 0.f, 0.f};
  if (x < a.c.d) {
    const __nv_bfloat16* p =
        reinterpret_cast<const __nv_bfloat16*>(a.q) + row * a.q_row + (long long)hq * a.q_head + x;
    for (int e = 0; e < 4; ++e) q[e] = to_f32(p[e]);
  }
  auto four = [&](const char* pool, long long part, int slot, float* f) {
    const uint32_t w = *reinterpret_cast<const uint16_t*>(pool + part +
                                                          (long long)slot * (a.c.d / 2) + x / 2);
    const uint32_t s2 = fp4_scale2((uint8_t)pool[part + fp4_scale_at(a.c, slot) + x / 16]);
    uint32_t r[4];
    fp4_halves(w, r);
    for (int e = 0; e < 2; ++e) {
      const uint32_t y = hmul2(r[e], s2);
      const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&y));
      f[2 * e] = z.x;
      f[2 * e + 1] = z.y;
    }
  };
  float m = *m_, l = *l_;
  for (int j = j0; j < j1; ++j) {
    if (!sees(place, j, a.window, a.sinks)) continue;
    const Slot at = kv_slot(a.c, b, j);
    const long long part = kv_row(a.c, h, Slot{at.page, 0});
    if (part < 0) continue;
    float s = 0.f, k[4], v[4] = {0.f, 0.f, 0.f, 0.f};
    if (x < a.c.d) {
      four(a.c.k, part, at.slot, k);
      four(a.c.v, part, at.slot, v);
      for (int e = 0; e < 4; ++e) s = fmaf(q[e], k[e], s);
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

template <int DP>
__global__ void __launch_bounds__(Q_THREADS, 1) k_attend_fp4(AttnArgs a, Div by_g, Div by_tokens,
                                                             Div by_ps) {
  constexpr int KT = QK * DP * 2, C = DP / 16, OC = DP / 2;
  // tensor memory: the queries, two turns of logits and weights, two outputs
  constexpr int STAGE = DP / 2, SUM = STAGE + 2 * Q_STAGE;
  static_assert(SUM + 2 * DP <= 512, "columns");
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  char* Ks = smem;  // [Q_AHEAD][DP / 64][64 rows][64]
  char* Vs = Ks + Q_AHEAD * KT;
  char* rings = Vs + Q_AHEAD * KT;  // [copying warp][Q_RING]
  QCtl* ctl = reinterpret_cast<QCtl*>(rings + Q_COPY * Q_RING * Q_PART<DP>);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    tc::mbar_init(&ctl->qfull, Q_WEIGH);
    tc::mbar_init(&ctl->ofull, 1);
    tc::mbar_init(&ctl->drained, 1);
    for (int x = 0; x < Q_AHEAD; ++x) {
      tc::mbar_init(&ctl->kfull[x], Q_COPY / 2);
      tc::mbar_init(&ctl->vfull[x], Q_COPY / 2);
      tc::mbar_init(&ctl->kempty[x], 1);
      tc::mbar_init(&ctl->vempty[x], 1);
    }
    for (int x = 0; x < 2; ++x) {
      tc::mbar_init(&ctl->sfull[x], 1);
      tc::mbar_init(&ctl->pfull[x], Q_WEIGH / 2);
    }
    ctl->abort = 0;
    ctl->strange = 0;
    tc::fence_mbar_init();
  }
  grid_dep_launch();
  grid_dep_wait();
  // key heads first: neighbouring CTAs are equally long, the longest ones start first
  const int h = blockIdx.x % a.c.Hkv, part = blockIdx.x / a.c.Hkv, split = part % a.splits;
  const int tpt = by_g.of(TM);  // tokens of a tile
  int b, tile, n;
  NewRows nr;
  if (!find_tile(a, part / a.splits, tpt, by_tokens, &b, &tile, &nr, &n)) return;
  const int t0 = (by_tokens.of(nr.T + tpt - 1) - 1 - tile) * tpt;
  const int nt = min(tpt, nr.T - t0);
  if (warp == Q_ISSUE) {
    tc::tmem_alloc(&ctl->tmem, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = ctl->tmem;
  const int i0 = n - nr.T + t0;  // place of the tile's first token
  const Seen seen = seen_keys(i0, i0 + nt - 1, a.window, a.sinks);
  const int na = ceil_div(seen.a, QK), all = na + ceil_div(seen.b1 - seen.b0, QK);
  const int per = ceil_div(all, a.splits), u0 = min(all, split * per);
  const int turns = min(all, u0 + per) - u0;
  auto key0 = [&](int x) { return u0 + x < na ? (u0 + x) * QK : seen.b0 + (u0 + x - na) * QK; };
  auto key1 = [&](int x) { return u0 + x < na ? seen.a : seen.b1; };

  if (turns > 0 && warp >= Q_WEIGH && warp < Q_ISSUE) {
    // ---- keys and values --------------------------------------------------------------
    // half of the warps the keys, half the values, Q_ROWS consecutive ones a warp: RW rows at a
    // time, a block of 16 channels a lane
    constexpr int W = Q_COPY / 2, RW = 32 / C, STEPS = QK / (W * RW);
    static_assert(STEPS * RW == Q_ROWS && Q_ROWS == 16, "a lane looks one row up, runs of 16");
    const int kv = (warp - Q_WEIGH) / W, w = warp - Q_WEIGH - kv * W;
    // eight lanes: two rows and four blocks, whose pieces lie in other banks
    const int c = C == 8 ? (lane & 3) | (lane >> 1 & 4) : lane & 3,
              rw = C == 8 ? (lane >> 2 & 1) | (lane >> 3 & 2) : lane >> 2;
    const char* pool = (kv ? a.c.v : a.c.k) + h * a.c.head_stride;
    const uint32_t tiles = tc::smem_u32(kv ? Vs : Ks);
    uint64_t *full = kv ? ctl->vfull : ctl->kfull, *empty = kv ? ctl->vempty : ctl->kempty;
    constexpr int CB = DP / 2, SB = DP / 16, P = CB / 16;  // bytes of a row, pieces of its codes
    const uint32_t ring = tc::smem_u32(rings + (warp - Q_WEIGH) * Q_RING * Q_PART<DP>);
    // a lane finds row `lane` of the warp's; where all 16 are seen and of one page, their first
    // one.  Its page is read a turn before it is needed, and looked at only then
    struct Place {
      int page, slot;
      bool run;
    };
    const bool runs = (a.c.ps & 15) == 0;  // 16 rows from a multiple of 16 on lie in one page
    auto look_up = [&](int x) {
      Place p = {0, -1, false};
      if (x >= turns) return p;
      int j = key0(x) + w * Q_ROWS;
      p.run = runs && (j & 15) == 0 && j + Q_ROWS <= key1(x);
      if (!p.run) j += lane;
      if (p.run || (lane < Q_ROWS && j < key1(x))) {
        const int y = by_ps.of(j);
        p.page = a.c.table[(long long)b * a.c.max_pages + y];
        p.slot = j - y * a.c.ps;
      }
      return p;
    };
    auto copy = [&](int x, const Place& p) {  // of rows that are not seen zeros
      if (x < turns) {
        const uint32_t to = ring + (x % Q_RING) * Q_PART<DP>;
        const bool there = p.slot >= 0 && (unsigned)p.page < (unsigned)a.c.num_pages;
        if (p.slot >= 0 && !there) set_status(a.c.status, CACHE_BAD);
        const char* part = pool + (there ? p.page * a.c.page_stride : 0);
        const long long codes = there ? (long long)p.slot * CB : 0,
                        scales = there ? fp4_scale_at(a.c, p.slot) : 0;
        if (p.run) {
#pragma unroll
          for (int y = 0; y < Q_ROWS * CB; y += 512)
            cp_async_to<16>(to + y + lane * 16, part + codes + (there ? y + lane * 16 : 0), there);
          if (lane < SB)
            cp_async_to<16>(to + Q_ROWS * CB + lane * 16, part + scales + (there ? lane * 16 : 0),
                       there);
        } else {
          const long long at = there ? part + codes - pool : -1;
#pragma unroll
          for (int r0 = 0; r0 < Q_ROWS; r0 += 32 / P) {
            const long long o = __shfl_sync(FULL, at, r0 + lane / P);
            cp_async_to<16>(to + r0 * CB + lane * 16, pool + (o >= 0 ? o + lane % P * 16 : 0),
                            o >= 0);
          }
          if (lane < Q_ROWS)
            cp_async_to<SB>(to + Q_ROWS * CB + lane * SB, part + scales, there);
        }
      }
      cp_async_commit();
    };
    {
      Place first[Q_RING - 1];
#pragma unroll
      for (int y = 0; y < Q_RING - 1; ++y) first[y] = look_up(y);
#pragma unroll
      for (int y = 0; y < Q_RING - 1; ++y) copy(y, first[y]);
    }
    // of the lane's block of its warp's first row
    const uint32_t place = (c >> 2) * QK * 128 + (w * Q_ROWS + rw) * 128 +
                           (((2 * (c & 3)) ^ (rw & 7)) * 16);
    uint32_t worst = 0;  // of the scales: from 0xf8 on not finite
    Place next = look_up(Q_RING - 1);
    for (int x = 0; x < turns; ++x) {
      const int stage = x % Q_AHEAD;
      if (x >= Q_AHEAD &&
          !__all_sync(FULL, wait_for(&empty[stage], (x / Q_AHEAD & 1) ^ 1, &ctl->abort)))
        break;
      cp_async_wait<Q_RING - 2>();
      __syncwarp();
      const uint32_t from = ring + (x % Q_RING) * Q_PART<DP> + rw * CB + c * 8,
                     from_z = ring + (x % Q_RING) * Q_PART<DP> + Q_ROWS * CB + rw * SB + c;
      // rows 4 further on: the other half of a swizzle's eight
      uint32_t dst[2];
      dst[0] = tiles + stage * KT + place;
      dst[1] = RW == 4 ? dst[0] ^ 64 : dst[0];
      uint2 code[STEPS];
      uint32_t scale[STEPS];
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        code[k] = lds8(from + k * RW * CB);
        scale[k] = lds1(from_z + k * RW * SB);
        worst = max(worst, scale[k]);
      }
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const uint32_t s2 = fp4_scale2(scale[k]);
        uint32_t v[8];
        fp4_halves(code[k].x, v);
        fp4_halves(code[k].y, v + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = hmul2(v[e], s2);
        const uint32_t row = dst[k & 1] + k * RW * 128;
        sts16(row, v);
        sts16(row ^ 16, v + 4);
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&full[stage]);
      copy(x + Q_RING - 1, next);  // into the place of turn x - 1
      next = look_up(x + Q_RING);
    }
    cp_async_wait<0>();
    if (worst >= 0xf8u) ctl->strange = 1;
  } else if (turns > 0 && warp == Q_ISSUE) {
    // ---- products -----------------------------------------------------------------------
    constexpr uint32_t BF16 = 1u << 7 | 1u << 10;  // the formats' bits: halves have none
    constexpr uint32_t sdesc = tc::idesc_bf16_f32(TM, QK) & ~BF16;
    constexpr uint32_t odesc = (tc::idesc_bf16_f32(TM, DP) & ~BF16) | (1u << 16);  // B is MN-major
    const uint32_t go = elect_one();
    const uint64_t kd = tc::desc_sw128_kmajor(Ks),
                   vd = desc_sw128_mnmajor(tc::smem_u32(Vs), QK * 128);
    auto ready = [&](uint64_t* bar, uint32_t parity) {
      const bool ok = wait_for(bar, parity, &ctl->abort);
      return __all_sync(FULL, ok) != 0;
    };
    auto logits = [&](int x) {
      const uint32_t d = tmem + STAGE + (x & 1) * Q_STAGE;
      const uint64_t kb = kd + x % Q_AHEAD * (KT / 16);
#pragma unroll
      for (int k = 0; k < DP / 16; ++k)
        mma_ts(go, d, tmem + k * 8, kb + ((k >> 2) * QK * 128 + (k & 3) * 32) / 16, sdesc, k > 0);
      commit(go, &ctl->sfull[x & 1]);
      commit(go, &ctl->kempty[x % Q_AHEAD]);
    };
    bool ok = ready(&ctl->qfull, 0);
    for (int x = 0; x < 2 && x < turns && ok; ++x) {
      ok = ready(&ctl->kfull[x], 0);
      tc::fence_after_sync();
      if (ok) logits(x);
    }
#pragma unroll 1
    for (int x = 0; x < turns && ok; ++x) {
      ok = ready(&ctl->pfull[x & 1], (x >> 1) & 1) &&
           ready(&ctl->vfull[x % Q_AHEAD], x / Q_AHEAD & 1);
      if (!ok) break;
      tc::fence_after_sync();
      const uint32_t p = tmem + STAGE + (x & 1) * Q_STAGE + 64, d = tmem + SUM + (x & 1) * DP;
      const uint64_t vb = vd + x % Q_AHEAD * (KT / 16);
#pragma unroll
      for (int k = 0; k < QK / 16; ++k)
        mma_ts(go, d, p + k * 8, vb + k * 2048 / 16, odesc, x > 1 || k > 0);
      commit(go, &ctl->vempty[x % Q_AHEAD]);
      if (x + 2 < turns) {  // into the place of logits that have become weights
        ok = ready(&ctl->kfull[(x + 2) % Q_AHEAD], (x + 2) / Q_AHEAD & 1);
        if (!ok) break;
        tc::fence_after_sync();
        logits(x + 2);
      } else if (x + 1 == turns) {
        commit(go, &ctl->ofull);
      }
    }
    if (!ok) {  // products in flight end before tensor memory is freed
      commit(go, &ctl->drained);
      const long long end = clock64() + T_WAIT;
      while (!tc::mbar_try_wait(&ctl->drained, 0) && clock64() < end) {
      }
    }
    __syncwarp();
  } else if (warp < Q_WEIGH) {
    // ---- weights ----------------------------------------------------------------------------
    const int half = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const int tok = by_g.of(r), g = r - tok * a.G;
    const bool valid = tok < nt;
    const int i = i0 + tok;
    const uint32_t lanes = tmem + ((uint32_t)quarter << 21);
    const int hq = h * a.G + g;
    const long long row = nr.off + t0 + tok;
    float factor = 1.f;
    if (turns > 0) {  // the queries: half a row a thread
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q) + row * a.q_row +
                               (long long)hq * a.q_head + half * OC;
      uint4 v[OC / 8];
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < OC / 8; ++c) {
        v[c] = make_uint4(0u, 0u, 0u, 0u);
        if (valid) v[c] = *reinterpret_cast<const uint4*>(q + c * 8);
        top = max(top, fp4_top(v[c]));
      }
      ctl->top[half][r] = __uint_as_float(top);
      meet(quarter);
      top = max(top, __float_as_uint(ctl->top[half ^ 1][r]));
      meet(quarter);  // both have read it
      const int e = (int)(top >> 7) - 127;
      const int k = top == 0 || top >= 0x7f80u ? 0 : min(14 - e, 126);
      const float up = __uint_as_float((uint32_t)(k + 127) << 23);
      factor = fmaxf(a.scale2 * __uint_as_float((uint32_t)(127 - k) << 23), 1e-37f);
#pragma unroll
      for (int c = 0; c < OC / 8; c += 4) {
        uint32_t p[16];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint32_t z[4] = {v[c + y].x, v[c + y].y, v[c + y].z, v[c + y].w};
#pragma unroll
          for (int f = 0; f < 4; ++f)
            p[4 * y + f] = halves(__uint_as_float(z[f] << 16) * up,
                                  __uint_as_float(z[f] & 0xffff0000u) * up);
        }
        tmem_st16_async(lanes + (half * OC + c * 8) / 2, p);
      }
      tmem_wait_st();
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&ctl->qfull);
    }
    float m = -INFINITY, l = 0.f;
    // a wait that runs out makes the next ones return at once; all threads stay in step
    for (int x = half; x < turns; x += 2) {  // the turns of this thread's warp, whole rows
      const uint32_t at = lanes + STAGE + half * Q_STAGE;
      const int j0 = key0(x), j1 = key1(x);
      wait_for(&ctl->sfull[half], (x >> 1) & 1, &ctl->abort);  // and products of turn x - 2
      __syncwarp();
      tc::fence_after_sync();
      // whether every row sees every key
      const bool whole = j0 + QK <= j1 && j0 + QK - 1 <= i0 &&
                         (a.window == 0 || i0 + nt - 1 - j0 < a.window || j0 + QK <= a.sinks);
      float s[32];
      auto load = [&](int z) {  // 32 logits, -inf where the row does not see the key
        tc::tmem_ld32(at + z * 32, s);
        if (!whole) {
          const int f = j0 + z * 32;                               // the first key
          const int hi = valid ? min(i + 1, j1) - f : 0;           // columns before hi,
          const int lo = a.window > 0 ? i - a.window + 1 - f : 0;  // from lo on
          const int sk = a.sinks - f;                              // or before sk
          const uint32_t in = below(hi) & (~below(lo) | below(sk));
#pragma unroll
          for (int y = 0; y < 32; ++y)
            if (!(in >> y & 1)) s[y] = -INFINITY;
        }
      };
      float top = -INFINITY;
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        load(z);
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int c = 4; c < 28; c += 8)
#pragma unroll
          for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], s[c + y], s[c + 4 + y]);
#pragma unroll
        for (int y = 0; y < 4; ++y) mx[y] = fmaxf(mx[y], s[28 + y]);
        top = max3(top, fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      }
      top = __fmul_ru(top, factor);
      const bool grew = top - m > FP4_ROOM;  // not of two infinities
      const float mn = grew ? fmaxf(top - FP4_UP, m) : m;
      const float f = m == -INFINITY || !grew ? 1.f : exp2_fast(m - mn);
      l *= f;
      m = mn;
      const float base = m == -INFINITY ? 0.f : m;
      const f32x2 scale = pair(factor, factor), off = pair(-base, -base);
      f32x2 sum[2] = {0ull, 0ull};
#pragma unroll
      for (int z = 1; z >= 0; --z) {
        if (z == 0) load(0);  // again: both halves do not fit the registers
        uint32_t p[16];
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          const float2 v = unpair(fma2(pair(s[2 * y], s[2 * y + 1]), scale, off));
          const float e0 = exp2_fast(v.x), e1 = exp2_fast(v.y);
          sum[y & 1] = add2(sum[y & 1], pair(e0, e1));
          p[y] = halves(e0, e1);
        }
        tmem_st16_async(at + 64 + z * 16, p);
      }
      const float2 both = unpair(add2(sum[0], sum[1]));
      l += both.x + both.y;
      if (x > 1 && __any_sync(FULL, f != 1.f)) {
#pragma unroll
        for (int c = 0; c < DP; c += 32) {
          float v[32];
          tc::tmem_ld32(lanes + SUM + half * DP + c, v);
#pragma unroll
          for (int y = 0; y < 32; ++y) v[y] *= f;
          tc::tmem_st32(lanes + SUM + half * DP + c, v);
        }
      }
      tmem_wait_st();
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&ctl->pfull[half]);
    }
    if (turns > 0) {
      wait_for(&ctl->ofull, 0, &ctl->abort);
      __syncwarp();
      tc::fence_after_sync();
    }
    // the two turns' sums become one
    ctl->top[half][r] = m;
    ctl->sum[half][r] = l;
    meet(quarter);
    const float m0 = ctl->top[0][r], m1 = ctl->top[1][r];
    m = fmaxf(m0, m1);
    const float base = m == -INFINITY ? 0.f : m;
    float f0 = exp2_fast(m0 - base), f1 = exp2_fast(m1 - base);
    l = ctl->sum[0][r] * f0 + ctl->sum[1][r] * f1;
    long long mine_at = -1;
    if (a.splits > 1) {
      const long long pr = part_row(a, split, b, t0 + tok) * a.H + hq;
      if (valid && half == 0) a.ml[pr] = make_float2(m, l);
      if (valid) mine_at = pr * a.c.d;
    } else {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      f0 *= inv;
      f1 *= inv;
      if (valid && half == 0 && a.lse)
        a.lse[row * a.H + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
      if (valid) mine_at = row * a.o_row + (long long)hq * a.o_head;
    }
    // 32 rows x OC columns a warp through the keys' and values' place, whole rows stored
    constexpr int PC = OC / 4, RPI = 32 / PC;
    char* st = Ks + warp * 32 * OC * 4;
#pragma unroll
    for (int c = 0; c < OC; c += 32) {
      float v[32];
#pragma unroll
      for (int y = 0; y < 32; ++y) v[y] = 0.f;
      if (turns > 0) {
        tc::tmem_ld32(lanes + SUM + half * OC + c, v);
#pragma unroll
        for (int y = 0; y < 32; ++y) v[y] *= f0;
      }
      if (turns > 1) {
        float w[32];
        tc::tmem_ld32(lanes + SUM + DP + half * OC + c, w);
#pragma unroll
        for (int y = 0; y < 32; ++y) v[y] = fmaf(w[y], f1, v[y]);
      }
#pragma unroll
      for (int y = 0; y < 32; y += 4)
        *reinterpret_cast<float4*>(st + lane * OC * 4 + ((((c + y) / 4) ^ (lane & 7)) * 16)) =
            make_float4(v[y], v[y + 1], v[y + 2], v[y + 3]);
    }
    __syncwarp();
    const int pc = lane % PC;
#pragma unroll 4
    for (int y0 = 0; y0 < 32; y0 += RPI) {
      const int y = y0 + lane / PC;
      const long long at = __shfl_sync(FULL, mine_at, y);
      if (at < 0) continue;
      const float4 v =
          *reinterpret_cast<const float4*>(st + y * OC * 4 + ((pc ^ (y & 7)) * 16));
      const long long to = at + half * OC + pc * 4;
      if (a.splits > 1)
        *reinterpret_cast<float4*>(a.part + to) = v;
      else
        *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + to) =
            make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == Q_ISSUE) tc::tmem_dealloc(tmem, 512);
  if (ctl->abort) {
    if (tid == 0) set_status(a.c.status, GMC_STATUS_TIMEOUT);
    return;
  }
  if (ctl->strange) {
    for (int rr = warp; rr < nt * a.G; rr += Q_THREADS / 32) {
      const int tk = rr / a.G, g = rr - tk * a.G, hq = h * a.G + g;
      const long long row = nr.off + t0 + tk;
      float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
      for (int x = 0; x < turns; ++x)
        row_alone4(a, b, h, row, hq, i0 + tk, key0(x), min(key1(x), key0(x) + QK), &m, &l, o);
      const int y = lane * 4;
      if (a.splits > 1) {
        const long long pr = part_row(a, split, b, t0 + tk) * a.H + hq;
        if (lane == 0) a.ml[pr] = make_float2(m, l);
        if (y < a.c.d)
          *reinterpret_cast<float4*>(a.part + pr * a.c.d + y) =
              make_float4(o[0], o[1], o[2], o[3]);
      } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (lane == 0 && a.lse)
          a.lse[row * a.H + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        if (y < a.c.d)
          *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + row * a.o_row +
                                    (long long)hq * a.o_head + y) =
              make_uint2(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv));
      }
    }
  }
}

// Tiles of one sequence and key head, all sequences: at most this many.
long long fp4_tiles(const KV& c, int G, long long rows, int T) {
  const int tokens = TM / G;
  return std::min((long long)c.B * ceil_div(T, tokens), rows / tokens + c.B);
}
}  // namespace

// Parts of the key axis where the tiles leave SMs idle: up to as many as fill them, two
// turns each at least.
int attend_direct_splits(const KV& c, int G, int T) {
  const long long rows = (long long)c.B * T, ctas = c.Hkv * fp4_tiles(c, G, rows, T);
  if (ctas > sm_count() / 2) return 1;
  return cheapest_parts(std::min<long long>({sm_count() / ctas, 32, c.cap / (2 * QK)}),
                        ceil_div(c.cap, QK), 0.76f, rows * G * c.Hkv * c.d);
}

cudaError_t launch_attend_direct(const AttnArgs& a, cudaStream_t st) {
  const long long grid = fp4_tiles(a.c, a.G, a.rows, a.T) * a.c.Hkv * a.splits;
  auto go = [&](auto kernel, size_t smem) {
    const cudaError_t e = set_smem_limit((const void*)kernel, smem);
    if (e != cudaSuccess) return e;
    return launch_k(kernel, dim3((unsigned)grid), dim3(Q_THREADS), smem, st, 1, a, make_div(a.G),
                    make_div(TM / a.G), make_div(a.c.ps));
  };
  return a.c.d == 64 ? go(k_attend_fp4<64>, q_smem<64>()) : go(k_attend_fp4<128>, q_smem<128>());
}

}  // namespace gmc
