// What the kernels of one new token's attention share (k_decode.cu, k_decode_fp4.cu): the
// row of turns and a warp's stretch of it, the kernel's outline over the query heads H of
// a warp, and the joining of parts and scores.
#pragma once

#include <algorithm>

#include "cache.cuh"

namespace gmc {

namespace {
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// ---- the row of turns ----------------------------------------------------------------
// The keys that the new token of a sequence of n tokens walks.  In turns of 32 (pages of 4
// bits) a turn starts at a multiple of 32 in the sequence, so that it can be copied whole:
// the sinks' and the window's first turns may hold keys that are not seen.
template <int DT> __device__ __forceinline__ Seen walked(const DecodeArgs& a, int n) {
  Seen s = seen_keys(n - 1, n - 1, a.window, a.sinks);
  if (DT == 32) {
    s.a = (s.a + 31) & ~31;
    s.b0 &= ~31;
    if (s.a >= s.b0) s.a = s.b0 = 0;
  }
  return s;
}

// A pair and a turn of it.
template <int DT> struct Walk {
  int b, h, t, turns, nv, n;
  Seen seen;
  int lo, hi;  // turns of 32: those from lo to hi - 1 hold cached keys of one range that are all
               // seen, key 32 t + off first
  int off;
  __device__ __forceinline__ void load(const DecodeArgs& a) { load(a, kv_len(a.c, b)); }
  __device__ __forceinline__ void load(const DecodeArgs& a, int tokens) {
    n = tokens;
    seen = walked<DT>(a, n);
    nv = seen.count();
    turns = ceil_div(nv, DT);
    if (DT == 32) {
      off = seen.b0 - seen.a;
      const int from = a.window > 0 ? max(n - a.window, 0) : 0;  // sinks' turns are not among them
      const int to = a.k_new ? n - 1 : n;
      lo = (max(from, seen.b0) - off + 31) >> 5;
      hi = (to - off) >> 5;
    }
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
template <int DT> struct TurnRow {
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
      mine += ceil_div(walked<DT>(a, n).count(), DT);
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
  __device__ __forceinline__ void find(const DecodeArgs& a, int at, Walk<DT>* w) const {
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
  // Turns of a CTA of W warps: of 4 bits, whose warps share them out, as many as the others'.
  __device__ __forceinline__ int of_cta(const DecodeArgs& a, int W) const {
    return DT == 32 ? max(ceil_div(all, a.warps / W), 1) : W * per;
  }
  // The first turn of sequence b, and its walk.
  __device__ __forceinline__ int first(const DecodeArgs& a, int b, Walk<DT>* w) const {
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
// Logits of a pair's turn, [key][heads of a launch].
template <int DT>
__device__ __forceinline__ float* logits_of(const DecodeArgs& a, const Walk<DT>& w) {
  return a.logits + (((long long)w.b * a.c.Hkv + w.h) * a.places + w.t * DT) * a.hs;
}
// ---- joining -------------------------------------------------------------------------------
// Whether a CTA, whose turns are lo .. hi - 1 of the row, joins its warps' parts and leaves one
// of a pair: where it has nothing else, and of 4 bits also where it has three pairs at most.
template <int DT>
__device__ __forceinline__ bool together(const DecodeArgs& a, const TurnRow<DT>& r, int lo,
                                         int hi) {
  Walk<DT> x, y;
  r.find(a, lo, &x);
  r.find(a, hi - 1, &y);
  return (y.b - x.b) * a.c.Hkv + y.h - x.h < (DT == 32 ? 3 : 1);
}

// The parts of a pair whose turns are u0 .. u0 + turns - 1 of the row: one of every CTA
// that joins its warps', one of every warp's run in the others.  Runs and pairs both only
// grow along the row, so the sum of their numbers numbers the parts' places.
struct Parts {
  int run0, n0, run1, mid, run2, count, W;
  long long pair;
  bool whole;  // one CTA had it all: its output is written
  template <int DT>
  __device__ __forceinline__ Parts(const DecodeArgs& a, const TurnRow<DT>& r, int W_, int u0,
                                   int turns, long long pair_) {
    W = W_;
    pair = pair_;
    const int cta = r.of_cta(a, W), u1 = u0 + turns;
    const int c0 = u0 / cta, c1 = (u1 - 1) / cta;
    if (turns == 0) {  // no part
      n0 = mid = count = 0;
      whole = false;
      return;
    }
    int n, first;
    auto of = [&](int c) {
      const int lo = c * cta, hi = r.all - lo < cta ? r.all : lo + cta;
      const bool one = DT == 32 ? together(a, r, lo, hi) : lo >= u0 && hi <= u1;
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
template <int DT>
__device__ __forceinline__ void add_scores(const DecodeArgs& a, const Walk<DT>& w, const float2* ml,
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
    // a turn of 32 may hold keys that are not seen: a NaN of the others' sum is not theirs
    const bool seen = DT != 32 || sees(w.n - 1, j, a.window, a.sinks);
    const float old = a.fresh && j == w.n - 1 ? 0.f : in[j];
    out[j] = seen ? old + s : old;
  }
  if (in != out)  // unseen keys keep what they had
    for (int j = w.seen.a + x0; j < w.seen.b0; j += step) out[j] = in[j];
}

// The turns of a CTA, and of a warp of its W: u, u + step, .. below end, the first one w.
template <int DT, int W> struct Stretch {
  int at, count, u, end, step;
  bool one, whole;  // all of the CTA's are of one pair; all the pair's
  bool few;         // of 4 bits: it joins its warps' parts (`together`)
  Walk<DT> w;
  // A whole pair, and no other.
  __device__ __forceinline__ void own(const DecodeArgs& a) {
    w.b = blockIdx.x / a.c.Hkv;
    w.h = blockIdx.x - w.b * a.c.Hkv;
    w.t = 0;
    w.load(a);
    at = 0;
    count = w.turns;
    one = whole = few = true;
  }
  // As many as every other CTA; false if there are none left.
  __device__ __forceinline__ bool share(const DecodeArgs& a, const TurnRow<DT>& turns) {
    const int cta = turns.of_cta(a, W);
    at = turns.all / cta < (int)blockIdx.x ? turns.all : (int)blockIdx.x * cta;
    count = min(cta, turns.all - at);
    if (count <= 0) return false;
    turns.find(a, at, &w);
    one = w.t + count <= w.turns;
    whole = one && count == w.turns;
    few = DT == 32 && together(a, turns, at, at + count);
    return true;
  }
  __device__ __forceinline__ void warp_of_one(int warp) {
    w.t += warp;
    u = at + warp;
    end = at + count;
    step = W;
  }
  // Of a CTA with a whole pair a warp's run of it.
  __device__ __forceinline__ void warp_of_own(int warp) {
    step = 1;
    u = warp * ceil_div(count, W);
    end = min(count, u + ceil_div(count, W));
    w.t = u;
  }
  __device__ __forceinline__ void warp_of_several(const DecodeArgs& a, const TurnRow<DT>& turns,
                                                  int warp) {
    u = at + warp * turns.per;
    end = min(at + count, u + turns.per);
    step = 1;
    if (u < end) turns.find(a, u, &w);
  }
};

// A pair without a seen key.
template <typename T, int DP>
__device__ __forceinline__ void write_nothing(const DecodeArgs& a, int b, int h) {
  for (int x = threadIdx.x; x < a.heads * (DP / 4); x += blockDim.x) {
    const int g = x / (DP / 4), y = (x - g * (DP / 4)) * 4;
    write_head<T>(a, b, h, g, y, make_float4(0.f, 0.f, 0.f, 0.f), 0.f);
    if (y == 0) write_lse(a, b, h, g, 0.f, 0.f);
  }
}

// The outputs of a CTA's first nw warps, all of one pair (b, h), become the CTA's: ml[warp][HM]
// maxima and sums, rows [HM][DP] at `rows`, `room` bytes a warp.  fin: of each head, where the pair
// is whole.
template <typename T, int HM, int DP, int W>
__device__ __forceinline__ void join_warps(const DecodeArgs& a, int b, int h, int nw, bool whole,
                                           const float2* ml, const char* rows, int room,
                                           float2* fin) {
  const long long part = (long long)blockIdx.x * W + b * a.c.Hkv + h;
  for (int x = threadIdx.x; x < a.heads * (DP / 4); x += W * 32) {
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
      const float4 z = *reinterpret_cast<const float4*>(rows + q * room + (g * DP + y) * 4);
      L = fmaf(v[q].y, f, L);
      o.x = fmaf(z.x, f, o.x);
      o.y = fmaf(z.y, f, o.y);
      o.z = fmaf(z.z, f, o.z);
      o.w = fmaf(z.w, f, o.w);
    }
    if (whole) {
      write_head<T>(a, b, h, g, y, o, final_ml(base, L).y);
      if (y == 0) write_lse(a, b, h, g, base, L);
    } else {
      *reinterpret_cast<float4*>(a.part + (part * a.heads + g) * DP + y) = o;
    }
    if (y == 0) {
      if (fin)
        fin[g] = final_ml(base, L);
      else
        a.ml[part * a.heads + g] = make_float2(M, L);
    }
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
constexpr int JN_AHEAD = 8;  // places of a thread that are fetched before the sums are joined
constexpr int JN_WARPS = 8, JN_THREADS = JN_WARPS * 32;
template <typename T, int DT>
__global__ void __launch_bounds__(JN_THREADS) k_decode_join(DecodeArgs a, int W, int dp,
                                                            int out_blocks, int blocks) {
  __shared__ float2 fin[16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // Every CTA of k_decode was past its wait before this kernel could start: what ran before
  // k_decode is complete, and the lengths, which k_decode does not write, can be read (from
  // L2: kv_len) while it works.  Its parts, sums and logits are read after the wait.
  grid_dep_launch();
  const TurnRow<DT> row(a);
  Walk<DT> w;
  if ((int)blockIdx.x < out_blocks) {
    const int x = blockIdx.x * JN_WARPS + warp, pair = x / a.heads, g = x - pair * a.heads;
    if (pair >= a.c.B * a.c.Hkv) return;
    const int b = pair / a.c.Hkv;
    w.h = pair - b * a.c.Hkv;
    const int u = row.first(a, b, &w) + w.h * w.turns;
    const Parts p(a, row, W, u, w.turns, pair);
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
  const Parts p(a, row, W, u, w.turns, pair);
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
inline int heads_per_launch(int dtype, int G, int d) {
  if (dtype == GMC_FP4) return std::min(G, d > 128 ? 8 : 16);
  return dtype == GMC_BF16 ? std::min(G, 16) : G > 4 ? std::min(G, 8) : G;
}
// Floats of a key's logits: whole 16-byte pieces, as many as rows hold them.
inline int logit_heads(int dtype, int G, int d) {
  const int h = heads_per_launch(dtype, G, d);
  return h > 8 ? 16 : h > 4 ? 8 : h > 2 ? 4 : h;
}
inline int decode_dp(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Warps of a CTA, at most (one CTA an SM), and keys of a turn.
inline int decode_warps(int dtype) { return dtype == GMC_FP4 ? 16 : 8; }
inline int decode_turn(int dtype) { return dtype == GMC_FP4 ? 32 : 16; }

struct DecodeWs {
  size_t ml, part, logits, all;
};
inline DecodeWs decode_carve(const KV& c, int dtype, int H) {
  const int G = H / c.Hkv, heads = heads_per_launch(dtype, G, c.d);
  const size_t pairs = (size_t)c.B * c.Hkv, parts = pairs + (size_t)sm_count() * decode_warps(dtype);
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  DecodeWs w;
  w.ml = 0;
  w.part = up(parts * heads * 8);
  w.logits = w.part + up(parts * heads * decode_dp(c.d) * 4);
  const int turn = decode_turn(dtype);
  w.all = w.logits + pairs * logit_heads(dtype, G, c.d) * 4 * (size_t)(ceil_div(c.cap, turn) * turn);
  return w;
}
// kernels: a CTA a pair, and equal stretches.
// Turns a warp of a CTA with a pair of its own has at most: where the pairs are half of the CTAs
// or more, and where they are fewer.
struct OwnTurns {
  int many, few;
};
template <typename T, int DT, int DP, int W>
cudaError_t decode_launch(DecodeArgs a, void (*own_kernel)(DecodeArgs), void (*kernel)(DecodeArgs),
                          OwnTurns most, size_t smem, cudaStream_t st, int* launches) {
  const int ctas = sm_count();
  const int pairs = a.c.B * a.c.Hkv;
  // A CTA a pair where that is a few turns a warp: no parts, no second launch.
  const int turns = ceil_div(a.c.cap, W * DT);
  const bool own = pairs <= ctas && turns <= (2 * pairs >= ctas ? most.many : most.few);
  a.warps = ctas * W;
  if (own) kernel = own_kernel;
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
  return launch_k(k_decode_join<T, DT>, dim3(out_blocks + pairs * blocks),
                  dim3(JN_THREADS), 0, st, 1, a, W, DP, out_blocks, std::max(blocks, 1));
}
}  // namespace
}  // namespace gmc
