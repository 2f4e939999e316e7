// Causal attention of new tokens over a paged key-value cache on the tcgen05 tensor
// cores: fp32 caches with d <= 128.
//
// The tensor cores multiply bf16.  A float cut into its upper 8 bits of mantissa, the next
// 8 and the last 8 is the sum of three bf16 exactly (cut, not rounded: no overflow, and the
// differences are exact), and of the nine products of two such sums the six down to
// 2^-16 of the largest are taken, the small ones first:
//     S = q0 k2 + q2 k0 + q1 k1 + q0 k1 + q1 k0 + q0 k0
// What is left out, q1 k2 + q2 k1 + q2 k2, is 2^-21 of |q| |k| at most (q1 reaches 2^-7 and
// q2 2^-15 of q's power of two) and 2^-24.6 on average, of the product's sign.  Products are
// exact and are added in fp32 in tensor memory over one turn of keys; across turns the output
// is added up in registers (the tensor cores' own adding cuts, and over thousands of keys that
// would show).
//
// A CTA takes a tile of up to 128 rows, a row being one query head of one token (the G
// query heads of a key head and 128 / G consecutive tokens), and walks the seen keys 64
// at a time.  Three warps load keys, three load values, cut them into bf16 and write them
// to shared memory the way the tensor cores read them; one issues products; eight turn
// logits into weights, cut them, write them to tensor memory, and add up the output: two
// threads a row, each with half of the turn's keys and half of the columns, which meet
// for the maximum.  The maximum that weights are taken against follows the running one
// only when it has grown by 2^8.
//
// The queries' parts lie in tensor memory, so a product reads 2 KB of shared memory for its
// keys alone, not 6 (which took the port's whole rate).
//
// Measured: 608 tokens of 32 heads 37 us, 1,000 tokens of 28 heads (4 key heads) 50 us,
// 144 TFLOP/s of fp32 products, where fp32 multiply-adds on the CUDA cores took 170 and
// 308 (their peak is 74 TFLOP/s).  Relative error (2-norm, against 64 bits) 5e-7, theirs
// was 9e-7; with the output added up in tensor memory over two turns 8e-7, over four
// 15e-7.  A turn takes 5,000 clocks; the tensor cores work for 3,100 of them, and the six
// warps that load and cut are its longest chain (some 800 instructions, half of them
// integer ones at half rate).
//
// Keys that a row does not see get the weight 0.  Slots outside the seen ranges are not
// read; where any key or value read is not finite, also one that every row sees (its parts
// would be NaN, and 0 x NaN would reach rows that do not see it), the CTA computes its rows
// again one by one, each from the keys that it sees.
//
// Every wait is bounded (about two seconds); on timeout GMC_STATUS_TIMEOUT is set in
// the cache's status word, products in flight are drained and tensor memory is freed.
#include <algorithm>

#include "attend_tc.cuh"

namespace gmc {

namespace {
constexpr int FK = 64;        // keys of a turn
constexpr int F_WEIGH = 8;    // warps that weigh and add up
constexpr int F_COPY = 6;     // warps that load and cut
constexpr int F_ISSUE = F_WEIGH + F_COPY;
constexpr int F_THREADS = (F_ISSUE + 1) * 32;
constexpr int F_STAGE = 96;   // columns of a turn in tensor memory: 64 logits, then 3 x 32 of weights

struct FCtl {
  uint64_t qfull, kfull[2], kempty[2], vfull[2], vempty[2], sfull[2], pfull[2], ofull, drained;
  float top[2][2][TM], sum[2][TM];
  uint32_t tmem;
  volatile int abort;
  int strange;
};

// One CTA an SM (a second one would wait for tensor memory).
template <int DP> constexpr size_t f_smem() {
  const size_t need = 1024 + 12 * (size_t)FK * DP * 2 + sizeof(FCtl);
  return need > 120 * 1024 ? need : 120 * 1024;
}

// The upper halves of two words, the first one's low.
__device__ __forceinline__ uint32_t uppers(float lo, float hi) {
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}
__device__ __forceinline__ float upper(float x) {
  return __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}
// Two floats as three pairs of bf16.
__device__ __forceinline__ void cut2(float x, float y, uint32_t* p0, uint32_t* p1, uint32_t* p2) {
  *p0 = uppers(x, y);
  const f32x2 minus = pair(-1.f, -1.f), one = fma2(pair(upper(x), upper(y)), minus, pair(x, y));
  const float2 v = unpair(one);
  *p1 = uppers(v.x, v.y);
  const float2 w = unpair(fma2(pair(upper(v.x), upper(v.y)), minus, one));
  *p2 = uppers(w.x, w.y);
}
// Eight floats into 16 bytes each of three tiles `step` bytes apart.
__device__ __forceinline__ void cut8(char* dst, int step, const float4& a, const float4& b) {
  uint4 w[3];
  cut2(a.x, a.y, &w[0].x, &w[1].x, &w[2].x);
  cut2(a.z, a.w, &w[0].y, &w[1].y, &w[2].y);
  cut2(b.x, b.y, &w[0].z, &w[1].z, &w[2].z);
  cut2(b.z, b.w, &w[0].w, &w[1].w, &w[2].w);
#pragma unroll
  for (int t = 0; t < 3; ++t) *reinterpret_cast<uint4*>(dst + t * step) = w[t];
}
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
// 8 columns of 32 bits, without the wait.
__device__ __forceinline__ void tmem_st8_async(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
// The two warps of a lane quarter meet.
__device__ __forceinline__ void meet(int quarter) {
  asm volatile("bar.sync %0, 64;" ::"r"(quarter + 1) : "memory");
}

template <int DP>
__global__ void __launch_bounds__(F_THREADS, 1) k_attend_f32(AttnArgs a, Div by_g, Div by_tokens) {
  constexpr int KT = FK * DP * 2, C = DP / 8;
  // tensor memory: the queries' three parts, two turns of logits and weights, one of output
  constexpr int QC = DP / 2, STAGE = 3 * QC, SUM = STAGE + 2 * F_STAGE;
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  char* Ks = smem;          // [2 turns][3][DP / 64][64 rows][64]
  char* Vs = Ks + 6 * KT;
  FCtl* ctl = reinterpret_cast<FCtl*>(Vs + 6 * KT);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    tc::mbar_init(&ctl->qfull, F_WEIGH);
    tc::mbar_init(&ctl->ofull, 1);
    tc::mbar_init(&ctl->drained, 1);
    for (int x = 0; x < 2; ++x) {
      tc::mbar_init(&ctl->kfull[x], F_COPY / 2);
      tc::mbar_init(&ctl->vfull[x], F_COPY / 2);
      tc::mbar_init(&ctl->kempty[x], 1);
      tc::mbar_init(&ctl->vempty[x], 1);
      tc::mbar_init(&ctl->sfull[x], 1);
      tc::mbar_init(&ctl->pfull[x], F_WEIGH);
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
  if (warp == F_ISSUE) {
    tc::tmem_alloc(&ctl->tmem, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = ctl->tmem;
  const int i0 = n - nr.T + t0;  // place of the tile's first token
  const Seen seen = seen_keys(i0, i0 + nt - 1, a.window, a.sinks);
  const int na = ceil_div(seen.a, FK), all = na + ceil_div(seen.b1 - seen.b0, FK);
  const int per = ceil_div(all, a.splits), u0 = min(all, split * per);
  const int turns = min(all, u0 + per) - u0;
  auto key0 = [&](int x) { return u0 + x < na ? (u0 + x) * FK : seen.b0 + (u0 + x - na) * FK; };
  auto key1 = [&](int x) { return u0 + x < na ? seen.a : seen.b1; };

  if (turns > 0 && warp >= F_WEIGH && warp < F_ISSUE) {
    // ---- keys and values --------------------------------------------------------------
    // three warps the keys, three the values: RW rows at a time, 8 columns a lane
    constexpr int W = F_COPY / 2, RW = 32 / C, STEPS = (FK + W * RW - 1) / (W * RW);
    const int kv = (warp - F_WEIGH) / W, w = warp - F_WEIGH - kv * W, c = lane % C, rw = lane / C;
    const char* pool = (kv ? a.c.v : a.c.k) + c * 32;
    char* tiles = kv ? Vs : Ks;
    uint64_t *full = kv ? ctl->vfull : ctl->kfull, *empty = kv ? ctl->vempty : ctl->kempty;
    const bool ok0 = c * 8 < a.c.d, ok1 = c * 8 + 4 < a.c.d;
    // the place of the warp's row (step, rw) = (lane / RW, lane % RW): its page is read a turn
    // before it is needed, and looked at only then
    struct Place {
      int page, slot;
    };
    auto look_up = [&](int x) {
      Place p = {0, -1};
      const int r = (lane / RW * W + w) * RW + lane % RW, j = key0(x) + r;
      if (lane < STEPS * RW && r < FK && x < turns && j < key1(x)) {
        const unsigned y = (unsigned)j / (unsigned)a.c.ps;
        p.page = a.c.table[(long long)b * a.c.max_pages + y];
        p.slot = j - (int)y * a.c.ps;
      }
      return p;
    };
    auto row_of = [&](const Place& p) {
      if (p.slot < 0) return -1LL;
      if ((unsigned)p.page >= (unsigned)a.c.num_pages) {
        set_status(a.c.status, CACHE_BAD);
        return -1LL;
      }
      return p.page * a.c.page_stride + h * a.c.head_stride + p.slot * a.c.slot_stride;
    };
    float4 v[STEPS][2];
    auto load = [&](long long rows) {
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const long long o = __shfl_sync(FULL, rows, k * RW + rw);
        v[k][0] = v[k][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (o >= 0) {
          const float4* src = reinterpret_cast<const float4*>(pool + o * 4);
          if (ok0) v[k][0] = src[0];
          if (ok1) v[k][1] = src[1];
        }
      }
    };
    f32x2 bad = 0ull;  // becomes NaN with a key or value that is not finite
    load(row_of(look_up(0)));
    Place next = look_up(1);
    for (int x = 0; x < turns; ++x) {
      if (x > 1 &&
          !__all_sync(FULL, wait_for(&empty[x & 1], ((x >> 1) & 1) ^ 1, &ctl->abort)))
        break;
      char* dst = tiles + (x & 1) * 3 * KT;
      const long long rows = row_of(next);
      next = look_up(x + 2);
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const int r = (k * W + w) * RW + rw;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          bad = fma2(pair(v[k][y].x, v[k][y].y), 0ull, bad);
          bad = fma2(pair(v[k][y].z, v[k][y].w), 0ull, bad);
        }
        if (k + 1 < STEPS || r < FK)
          cut8(dst + (c >> 3) * FK * 128 + r * 128 + (((c ^ r) & 7) * 16), KT, v[k][0], v[k][1]);
      }
      fence_async();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&full[x & 1]);
      load(rows);  // waited for at the next turn's stores
    }
    const float2 z = unpair(bad);
    if (!(z.x == 0.f && z.y == 0.f)) ctl->strange = 1;
  } else if (turns > 0 && warp == F_ISSUE) {
    // ---- products -----------------------------------------------------------------------
    constexpr uint32_t sdesc = tc::idesc_bf16_f32(TM, FK);
    constexpr uint32_t odesc = tc::idesc_bf16_f32(TM, DP) | (1u << 16);  // B is MN-major
    const uint32_t go = elect_one();
    const uint64_t kd = tc::desc_sw128_kmajor(Ks),
                   vd = desc_sw128_mnmajor(tc::smem_u32(Vs), FK * 128);
    auto ready = [&](uint64_t* bar, uint32_t parity) {
      const bool ok = wait_for(bar, parity, &ctl->abort);
      return __all_sync(FULL, ok) != 0;
    };
    // six products of parts, the smallest first
    auto logits = [&](int x) {
      const uint32_t d = tmem + STAGE + (x & 1) * F_STAGE;
      const uint64_t kb = kd + (x & 1) * (3 * KT / 16);
#pragma unroll
      for (int e = 0; e < 6; ++e) {
        constexpr int P[6] = {0, 2, 1, 0, 1, 0}, R[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          mma_ts(go, d, tmem + P[e] * QC + k * 8,
                 kb + (R[e] * KT + (k >> 2) * FK * 128 + (k & 3) * 32) / 16, sdesc, e > 0 || k > 0);
      }
      commit(go, &ctl->sfull[x & 1]);
      commit(go, &ctl->kempty[x & 1]);
    };
    bool ok = ready(&ctl->qfull, 0) && ready(&ctl->kfull[0], 0);
    tc::fence_after_sync();
    if (ok) logits(0);
#pragma unroll 1
    for (int x = 0; x < turns && ok; ++x) {
      if (x + 1 < turns) {
        ok = ready(&ctl->kfull[(x + 1) & 1], ((x + 1) >> 1) & 1);
        if (!ok) break;
        tc::fence_after_sync();
        logits(x + 1);
      }
      ok = ready(&ctl->pfull[x & 1], (x >> 1) & 1) && ready(&ctl->vfull[x & 1], (x >> 1) & 1);
      if (!ok) break;
      tc::fence_after_sync();
      const uint32_t p = tmem + STAGE + (x & 1) * F_STAGE, d = tmem + SUM;
      const uint64_t vb = vd + (x & 1) * (3 * KT / 16);
#pragma unroll
      for (int e = 0; e < 6; ++e) {
        constexpr int P[6] = {0, 2, 1, 0, 1, 0}, R[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
        for (int k = 0; k < FK / 16; ++k)
          mma_ts(go, d, p + P[e] * 32 + k * 8, vb + (R[e] * KT + k * 2048) / 16, odesc,
                 e > 0 || k > 0);
      }
      commit(go, &ctl->ofull);
      commit(go, &ctl->vempty[x & 1]);
    }
    if (!ok) {  // products in flight end before tensor memory is freed
      commit(go, &ctl->drained);
      const long long end = clock64() + T_WAIT;
      while (!tc::mbar_try_wait(&ctl->drained, 0) && clock64() < end) {
      }
    }
    __syncwarp();
  } else if (warp < F_WEIGH) {
    // ---- weights and output ---------------------------------------------------------------
    constexpr int OC = DP / 2;  // columns of a thread
    const int half = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const int tok = by_g.of(r), g = r - tok * a.G;
    const bool valid = tok < nt;
    const int i = i0 + tok;
    const uint32_t lanes = tmem + ((uint32_t)quarter << 21);
    const int hq = h * a.G + g;
    const long long row = nr.off + t0 + tok;
    if (turns > 0) {  // the queries: half a row a thread
      const float* q = reinterpret_cast<const float*>(a.q) + row * a.q_row +
                       (long long)hq * a.q_head + half * OC;
#pragma unroll
      for (int c = 0; c < OC; c += 16) {
        uint32_t p[3][8];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          if (valid && half * OC + c + 4 * y < a.c.d)
            v = *reinterpret_cast<const float4*>(q + c + 4 * y);
          cut2(v.x, v.y, &p[0][2 * y], &p[1][2 * y], &p[2][2 * y]);
          cut2(v.z, v.w, &p[0][2 * y + 1], &p[1][2 * y + 1], &p[2][2 * y + 1]);
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
          tmem_st8_async(lanes + e * QC + (half * OC + c) / 2, p[e]);
      }
      tmem_wait_st();
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&ctl->qfull);
    }
    float m = -INFINITY, l = 0.f;
    f32x2 o[OC / 2];
#pragma unroll
    for (int c = 0; c < OC / 2; ++c) o[c] = 0ull;
    // adds the products of turn x
    auto add_up = [&](int x) {
      wait_for(&ctl->ofull, x & 1, &ctl->abort);
      __syncwarp();
      tc::fence_after_sync();
#pragma unroll
      for (int c = 0; c < OC; c += 32) {
        float v[32];
        tc::tmem_ld32(lanes + SUM + half * OC + c, v);
#pragma unroll
        for (int y = 0; y < 16; ++y)
          o[c / 2 + y] = add2(o[c / 2 + y], pair(v[2 * y], v[2 * y + 1]));
      }
    };
    // a wait that runs out makes the next ones return at once; all threads stay in step
    for (int x = 0; x < turns; ++x) {
      const uint32_t at = lanes + STAGE + (x & 1) * F_STAGE;
      const int j0 = key0(x), j1 = key1(x);
      wait_for(&ctl->sfull[x & 1], (x >> 1) & 1, &ctl->abort);
      __syncwarp();
      tc::fence_after_sync();
      float s[32];
      tc::tmem_ld32(at + half * 32, s);
      // whether every row sees every key
      const bool whole = j0 + FK <= j1 && j0 + FK - 1 <= i0 &&
                         (a.window == 0 || i0 + nt - 1 - j0 < a.window || j0 + FK <= a.sinks);
      if (!whole) {
        const int f = j0 + half * 32;                            // this thread's first key
        const int hi = valid ? min(i + 1, j1) - f : 0;           // columns before hi,
        const int lo = a.window > 0 ? i - a.window + 1 - f : 0;  // from lo on
        const int sk = a.sinks - f;                              // or before sk
        const uint32_t in = below(hi) & (~below(lo) | below(sk));
#pragma unroll
        for (int y = 0; y < 32; ++y)
          if (!(in >> y & 1)) s[y] = -INFINITY;
      }
      float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int c = 4; c < 28; c += 8)
#pragma unroll
        for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], s[c + y], s[c + 4 + y]);
#pragma unroll
      for (int y = 0; y < 4; ++y) mx[y] = fmaxf(mx[y], s[28 + y]);
      float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale2;
      ctl->top[x & 1][half][r] = top;
      meet(quarter);  // both have read the logits, too
      top = fmaxf(top, ctl->top[x & 1][half ^ 1][r]);
      const bool grew = top > m + GROWN || (m == -INFINITY && top > m);
      const float mn = grew ? top : m;
      const float f = m == -INFINITY || !grew ? 1.f : exp2_fast(m - mn);
      l *= f;
      m = mn;
      const float base = m == -INFINITY ? 0.f : m;
      const f32x2 scale = pair(a.scale2, a.scale2), off = pair(-base, -base);
      f32x2 sum[2] = {0ull, 0ull};
#pragma unroll
      for (int c = 0; c < 16; c += 8) {
        uint32_t p[3][8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int z = 2 * (c + y);
          const float2 v = unpair(fma2(pair(s[z], s[z + 1]), scale, off));
          const float e0 = exp2_fast(v.x), e1 = exp2_fast(v.y);
          sum[y & 1] = add2(sum[y & 1], pair(e0, e1));
          cut2(e0, e1, &p[0][y], &p[1][y], &p[2][y]);
        }
#pragma unroll
        for (int e = 0; e < 3; ++e) tmem_st8_async(at + e * 32 + half * 16 + c, p[e]);
      }
      tmem_wait_st();
      const float2 both = unpair(add2(sum[0], sum[1]));
      l += both.x + both.y;
      if (x > 0) add_up(x - 1);  // its place is free for this turn's products after that
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&ctl->pfull[x & 1]);
      if (x > 0) {
        if (__any_sync(FULL, f != 1.f)) {
          const f32x2 ff = pair(f, f);
#pragma unroll
          for (int c = 0; c < OC / 2; ++c) o[c] = mul2(o[c], ff);
        }
      }
    }
    if (turns > 0) add_up(turns - 1);
    ctl->sum[half][r] = l;
    meet(quarter);
    l = ctl->sum[0][r] + ctl->sum[1][r];
    float* dst;
    long long mine_at = -1;
    float factor = 1.f;
    if (a.splits > 1) {
      const long long pr = part_row(a, split, b, t0 + tok) * a.H + hq;
      if (valid && half == 0) a.ml[pr] = make_float2(m, l);
      dst = a.part;
      if (valid) mine_at = pr * a.c.d;
    } else {
      factor = l == 0.f ? 0.f : 1.f / l;
      if (valid && half == 0 && a.lse)
        a.lse[row * a.H + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
      dst = reinterpret_cast<float*>(a.out);
      if (valid) mine_at = row * a.o_row + (long long)hq * a.o_head;
    }
    // 32 rows x OC columns a warp through the keys' place, whole rows stored
    constexpr int PC = OC / 4, RPI = 32 / PC;
    char* st = Ks + warp * 32 * OC * 4;
#pragma unroll
    for (int c = 0; c < PC; ++c) {
      const float2 lo = unpair(o[2 * c]), hi = unpair(o[2 * c + 1]);
      *reinterpret_cast<float4*>(st + lane * OC * 4 + ((c ^ (lane & 7)) * 16)) =
          make_float4(lo.x * factor, lo.y * factor, hi.x * factor, hi.y * factor);
    }
    __syncwarp();
    const int pc = lane % PC;
#pragma unroll 4
    for (int y0 = 0; y0 < 32; y0 += RPI) {
      const int y = y0 + lane / PC;
      const long long at = __shfl_sync(FULL, mine_at, y);
      if (at >= 0 && half * OC + pc * 4 < a.c.d)
        *reinterpret_cast<float4*>(dst + at + half * OC + pc * 4) =
            *reinterpret_cast<const float4*>(st + y * OC * 4 + ((pc ^ (y & 7)) * 16));
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == F_ISSUE) tc::tmem_dealloc(tmem, 512);
  if (ctl->abort) {
    if (tid == 0) set_status(a.c.status, GMC_STATUS_TIMEOUT);
    return;
  }
  if (ctl->strange) {
    for (int rr = warp; rr < nt * a.G; rr += F_THREADS / 32) {
      const int tk = rr / a.G, g = rr - tk * a.G, hq = h * a.G + g;
      const long long row = nr.off + t0 + tk;
      float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
      for (int x = 0; x < turns; ++x)
        row_alone<float>(a, b, h, row, hq, i0 + tk, key0(x), min(key1(x), key0(x) + FK), &m, &l,
                         o);
      const int y = lane * 4;
      float* dst;
      if (a.splits > 1) {
        const long long pr = part_row(a, split, b, t0 + tk) * a.H + hq;
        if (lane == 0) a.ml[pr] = make_float2(m, l);
        dst = a.part + pr * a.c.d;
      } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (lane == 0 && a.lse)
          a.lse[row * a.H + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        for (int e = 0; e < 4; ++e) o[e] *= inv;
        dst = reinterpret_cast<float*>(a.out) + row * a.o_row + (long long)hq * a.o_head;
      }
      if (y < a.c.d) *reinterpret_cast<float4*>(dst + y) = make_float4(o[0], o[1], o[2], o[3]);
    }
  }
}

// Tiles of one sequence and key head, all sequences: at most this many.
long long f32_tiles(const KV& c, int G, long long rows, int T) {
  const int tokens = TM / G;
  return std::min((long long)c.B * ceil_div(T, tokens), rows / tokens + c.B);
}
}  // namespace

bool attend_f32_takes(const KV& c, int dtype) { return dtype == GMC_F32 && c.d <= 128; }

// Parts of the key axis where the tiles leave SMs idle: up to as many as fill them, two
// turns each at least.
int attend_f32_splits(const KV& c, int G, int T) {
  const long long rows = (long long)c.B * T, ctas = c.Hkv * f32_tiles(c, G, rows, T);
  if (ctas > sm_count() / 2) return 1;
  return cheapest_parts(std::min<long long>({sm_count() / ctas, 32, c.cap / (2 * FK)}),
                        ceil_div(c.cap, FK), 2.4f, rows * G * c.Hkv * c.d);
}

cudaError_t launch_attend_f32(const AttnArgs& a, cudaStream_t st) {
  const long long grid = f32_tiles(a.c, a.G, a.rows, a.T) * a.c.Hkv * a.splits;
  auto go = [&](auto kernel, size_t smem) {
    const cudaError_t e = set_smem_limit((const void*)kernel, smem);
    if (e != cudaSuccess) return e;
    return launch_k(kernel, dim3((unsigned)grid), dim3(F_THREADS), smem, st, 1, a, make_div(a.G),
                    make_div(TM / a.G));
  };
  return a.c.d <= 64 ? go(k_attend_f32<64>, f_smem<64>()) : go(k_attend_f32<128>, f_smem<128>());
}

}  // namespace gmc
