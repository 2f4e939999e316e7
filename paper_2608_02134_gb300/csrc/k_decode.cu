// One new token's attention over a paged key-value cache: out = sum_j p_j v_j with
// p = softmax(scale q . k_j) over the seen keys, the new token's own key and value
// appended on the way, and optionally the weight that every key received added to
// its running score.
//
// Bound by memory: each key and value is read once for the G query heads that share
// it.  The seen keys of one (sequence, key head) are split over the CTAs of a
// cluster and over the warps of a CTA, 16 keys a turn; a warp copies its own keys
// and values ahead into its own ring in shared memory (cp.async, no barrier), keeps
// the running maxima and sums of its query heads and its part of the output in
// registers, and meets the other warps and CTAs only at the end.
#include <cooperative_groups.h>

#include <algorithm>

#include "cache.cuh"

namespace cg = cooperative_groups;

namespace gmc {

namespace {
constexpr int DT = 16;       // keys of a turn
constexpr int D_SMEM_LOGITS = 24 * 1024;  // logits kept in shared memory up to this many bytes

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

// One (sequence, key head, split) of a launch.
struct DecodeJob {
  int b, h, split, splits, n, v0, v1, heads;  // heads: query heads of this launch
  Seen seen;
  __device__ __forceinline__ void init(const DecodeArgs& a, int max_heads) {
    split = blockIdx.x;
    splits = gridDim.x;
    h = blockIdx.y;
    b = blockIdx.z;
    heads = min(max_heads, a.G - a.h0);
    n = kv_len(a.c, b);
    seen = seen_keys(n - 1, n - 1, a.window, a.sinks);
    const int nv = seen.count();
    v0 = min(nv, split * a.chunk);
    v1 = min(nv, v0 + a.chunk);
  }
};

// The appended row goes to its page (one CTA of the cluster, its last warp).
__device__ __forceinline__ void append_new(const DecodeArgs& a, const DecodeJob& J, int esize,
                                           int lane) {
  if (J.n < 1) return;
  const long long o = kv_row(a.c, J.b, J.h, J.n - 1);
  if (o < 0) return;
  const long long src = ((long long)J.b * a.c.Hkv + J.h) * a.c.d;
  for (int x = lane; x < a.c.d * esize / 16; x += 32) {
    *(int4*)(a.c.k + o * esize + x * 16) = *(const int4*)(a.k_new + src * esize + x * 16);
    *(int4*)(a.c.v + o * esize + x * 16) = *(const int4*)(a.v_new + src * esize + x * 16);
  }
}

// Lane's row pointer of turn t: lanes 0-15 the keys' rows, lanes 16-31 the values' of
// the same 16 places; nullptr past the end.
__device__ __forceinline__ const char* turn_row(const DecodeArgs& a, const DecodeJob& J, int t,
                                                int lane, int esize) {
  const int x = J.v0 + t * DT + (lane & 15);
  if (x >= J.v1) return nullptr;
  const int j = J.seen.place(x);
  if (a.k_new && j == J.n - 1)
    return (lane < 16 ? a.k_new : a.v_new) + ((long long)J.b * a.c.Hkv + J.h) * a.c.d * esize;
  const long long o = kv_row(a.c, J.b, J.h, j);
  return o < 0 ? nullptr : (lane < 16 ? a.c.k : a.c.v) + o * esize;
}

// Copies a turn's 16 keys and values into the stage (16-byte pieces of row r at
// piece ^ (r & 7), so that reads down a column of rows meet no bank twice); rows past
// the end and elements past d become zeros.
template <int ROWB>
__device__ __forceinline__ void turn_copy(const DecodeArgs& a, char* stage, const char* mine,
                                          int lane, int rowbytes) {
  constexpr int P = ROWB / 16;  // pieces of a row
  constexpr int RPI = P >= 32 ? 1 : 32 / P;
#pragma unroll
  for (int r0 = 0; r0 < 2 * DT; r0 += RPI) {
    const int r = r0 + (P >= 32 ? 0 : lane / P);
    const char* p = (const char*)__shfl_sync(FULL, (unsigned long long)mine, r);
#pragma unroll
    for (int p0 = 0; p0 < P; p0 += 32) {
      const int pc = P >= 32 ? p0 + lane : lane % P;
      const bool ok = p != nullptr && pc * 16 < rowbytes;
      cp_async16(stage + r * ROWB + ((pc ^ (r & 7)) * 16), ok ? p + pc * 16 : a.c.k, ok);
    }
  }
}

// What every warp leaves: maxima and sums of its query heads (powers of two), and
// the unnormalised output rows.
template <int DP, int W, int HM> struct Tail {
  float m[W][HM], l[W][HM];
  float cm[HM], cl[HM];  // of the CTA, for the cluster
  float fm[HM], fl[HM];  // of all keys
  float o[HM][DP];       // of the CTA
};

// Joins the warps, then the CTAs of the cluster, writes the output and the scores.
// wo: [W][HM][DP] the warps' output rows, in the ring.
template <int DP, int W, int HM, typename T>
__device__ __forceinline__ void decode_join(const DecodeArgs& a, const DecodeJob& J,
                                            Tail<DP, W, HM>* tl, const float* wo,
                                            const float* logits) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, nt = W * 32;
  __syncthreads();  // the warps' parts are written
  if (tid < HM) {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, tl->m[w][tid]);
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp2_fast(tl->m[w][tid] - base);
      L += tl->l[w][tid] * f;
      tl->m[w][tid] = f;
    }
    tl->cm[tid] = M;
    tl->cl[tid] = L;
  }
  __syncthreads();
  for (int x = tid; x < J.heads * DP; x += nt) {
    const int g = x / DP, y = x - g * DP;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) s += tl->m[w][g] * wo[(w * HM + g) * DP + y];
    tl->o[g][y] = s;
  }
  if (J.splits > 1)
    cluster.sync();
  else
    __syncthreads();
  if (tid < J.heads) {
    float M = -INFINITY, L = 0.f;
    for (int q = 0; q < J.splits; ++q)
      M = fmaxf(M, J.splits > 1 ? cluster.map_shared_rank(tl, q)->cm[tid] : tl->cm[tid]);
    const float base = M == -INFINITY ? 0.f : M;
    for (int q = 0; q < J.splits; ++q) {
      const Tail<DP, W, HM>* t = J.splits > 1 ? cluster.map_shared_rank(tl, q) : tl;
      L += t->cl[tid] * exp2_fast(t->cm[tid] - base);
    }
    tl->fm[tid] = base;
    tl->fl[tid] = L > 0.f || L != L ? 1.f / L : 0.f;
    if (a.lse && J.split == 0)
      a.lse[(long long)J.b * a.H + J.h * a.G + a.h0 + tid] =
          L == 0.f ? -INFINITY : (base + log2f(L)) * LN2;
  }
  __syncthreads();
  const int each = ceil_div(J.heads * a.c.d, J.splits);  // this CTA's elements of the output
  const int e1 = min(J.heads * a.c.d, (J.split + 1) * each);
  for (int e = J.split * each + tid; e < e1; e += nt) {
    const int g = e / a.c.d, y = e - g * a.c.d;
    float s = 0.f;
    for (int q = 0; q < J.splits; ++q) {
      const Tail<DP, W, HM>* t = J.splits > 1 ? cluster.map_shared_rank(tl, q) : tl;
      s += exp2_fast(t->cm[g] - tl->fm[g]) * t->o[g][y];
    }
    s *= tl->fl[g];
    const int hq = J.h * a.G + a.h0 + g;
    reinterpret_cast<T*>(a.out)[J.b * a.o_row + hq * a.o_head + y] = from_f32<T>(s);
  }
  if (J.splits > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  if (a.scores) {
    const long long row = ((long long)J.b * a.c.Hkv + J.h) * a.score_stride;
    const float* in = a.scores + row;
    float* out = a.out_scores + row;
    for (int x = J.v0 + tid; x < J.v1; x += nt) {
      float s = 0.f;
      for (int g = 0; g < J.heads; ++g)
        s += exp2_fast(logits[(long long)g * a.chunk + (x - J.v0)] - tl->fm[g]) * tl->fl[g];
      const int j = J.seen.place(x);
      out[j] = (a.fresh && j == J.n - 1 ? 0.f : in[j]) + s;
    }
    if (in != out) {  // unseen keys keep what they had
      const int u0 = J.seen.a, u1 = J.seen.b0;
      for (int x = u0 + J.split * nt + tid; x < u1; x += J.splits * nt) out[x] = in[x];
    }
  }
  if (J.splits > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------
// bf16: up to 16 query heads are the rows of mma m16n8k16 (fp32 accumulation); the
// keys' and values' fragments come from the ring by ldmatrix.  The products are far
// from the bound (48 instructions per 16 keys), so the rows that G leaves idle cost
// nothing that shows.
// ---------------------------------------------------------------------------
template <int DP, int W, int NST>
constexpr size_t decode_bf16_smem() {
  return (size_t)W * NST * 2 * DT * DP * 2 + sizeof(Tail<DP, W, 16>);
}

template <int DP, int W, int NST>
__global__ void __launch_bounds__(W * 32) k_decode_bf16(DecodeArgs a) {
  constexpr int HM = 16, ROWB = DP * 2, STAGE = 2 * DT * ROWB;
  static_assert(W * NST * STAGE >= W * HM * DP * 4, "the ring holds the warps' output rows");
  extern __shared__ __align__(128) char smem[];
  Tail<DP, W, HM>* tl = reinterpret_cast<Tail<DP, W, HM>*>(smem + W * NST * STAGE);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  char* ring = smem + warp * NST * STAGE;
  grid_dep_wait();
  DecodeJob J;
  J.init(a, HM);
  float* logits = nullptr;
  if (a.scores)
    logits = a.chunk_smem ? reinterpret_cast<float*>(tl + 1)
                          : a.logits + (((long long)J.b * a.c.Hkv + J.h) * J.splits + J.split) *
                                           HM * a.chunk;
  const int turns = ceil_div(J.v1 - J.v0, DT);
  const int rowbytes = a.c.d * 2;
  // turns warp, warp + W, ..: NST - 1 of them on their way before the first is used
#pragma unroll
  for (int p = 0; p < NST - 1; ++p) {
    const int t = warp + p * W;
    if (t < turns) turn_copy<ROWB>(a, ring + p * STAGE, turn_row(a, J, t, lane, 2), lane, rowbytes);
    cp_async_commit();
  }
  if (a.k_new && J.split == J.splits - 1 && warp == W - 1) append_new(a, J, 2, lane);
  // the query heads' fragments: rows lane/4 and lane/4 + 8
  uint32_t qf[DP / 16][4];
  {
    const int g0 = lane >> 2, c0 = (lane & 3) * 2;
    const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q) + J.b * a.q_row +
                             (long long)(J.h * a.G + a.h0) * a.q_head;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int g = g0 + (f & 1) * 8, col = ks * 16 + c0 + (f >> 1) * 8;
        qf[ks][f] = g < J.heads && col < a.c.d
                        ? *reinterpret_cast<const uint32_t*>(q + g * a.q_head + col)
                        : 0u;
      }
  }
  float o[DP / 8][4];
#pragma unroll
  for (int x = 0; x < DP / 8; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const char* next = nullptr;  // the row of the turn to be copied next, looked up a turn ahead
  if (warp + (NST - 1) * W < turns) next = turn_row(a, J, warp + (NST - 1) * W, lane, 2);

  int st = 0;
  for (int t = warp; t < turns; t += W) {
    cp_async_wait<NST - 2>();
    __syncwarp();
    {
      const int tn = t + (NST - 1) * W;
      int sn = st + NST - 1;
      if (sn >= NST) sn -= NST;
      if (tn < turns) turn_copy<ROWB>(a, ring + sn * STAGE, next, lane, rowbytes);
      cp_async_commit();
      if (tn + W < turns) next = turn_row(a, J, tn + W, lane, 2);
    }
    const uint32_t kb = (uint32_t)__cvta_generic_to_shared(ring + st * STAGE);
    const uint32_t vb = kb + DT * ROWB;
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    {
      const int r = ((lane >> 4) << 3) + (lane & 7);
      const uint32_t row = kb + r * ROWB;
      const int half = (lane >> 3) & 1;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) {
        uint32_t f[4];
        ldsm4(f, row + (((ks * 2 + half) ^ (r & 7)) * 16));
        mma16816(s[0], qf[ks], f[0], f[1]);
        mma16816(s[1], qf[ks], f[2], f[3]);
      }
    }
    // logits in powers of two; places past the end leave
    const int x0 = J.v0 + t * DT + (lane & 3) * 2;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const int x = x0 + nt * 8 + (f & 1);
        s[nt][f] = x < J.v1 ? s[nt][f] * a.scale2 : -INFINITY;
      }
    if (a.scores) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const int x = x0 + nt * 8 + (f & 1), g = (lane >> 2) + (f >> 1) * 8;
          if (x < J.v1 && g < J.heads) logits[(long long)g * a.chunk + (x - J.v0)] = s[nt][f];
        }
    }
    float mn[2], base[2];
    bool grew = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
      x = fmaxf(x, __shfl_xor_sync(FULL, x, 1));
      x = fmaxf(x, __shfl_xor_sync(FULL, x, 2));
      mn[r] = fmaxf(m[r], x);
      grew |= mn[r] > m[r];
      base[r] = mn[r] == -INFINITY ? 0.f : mn[r];
    }
    if (__any_sync(FULL, grew)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float f = exp2_fast(m[r] - base[r]);
        l[r] *= f;
#pragma unroll
        for (int x = 0; x < DP / 8; ++x) {
          o[x][2 * r] *= f;
          o[x][2 * r + 1] *= f;
        }
        m[r] = mn[r];
      }
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        s[nt][f] = exp2_fast(s[nt][f] - base[f >> 1]);
        l[f >> 1] += s[nt][f];
      }
    // the weights as two bf16 terms (relative error 2^-17), each multiplied with the
    // values: the second product hides behind the copies, and the output then carries its
    // own rounding only
    uint32_t pf[4], pl[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const float x = s[f >> 1][(f & 1) * 2], y = s[f >> 1][(f & 1) * 2 + 1];
      pf[f] = pack_bf16(x, y);
      pl[f] = pack_bf16(x - __uint_as_float(pf[f] << 16),
                        y - __uint_as_float(pf[f] & 0xffff0000u));
    }
    {
      const int r = (((lane >> 3) & 1) << 3) + (lane & 7);
      const uint32_t row = vb + r * ROWB;
      const int half = lane >> 4;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) {
        uint32_t f[4];
        ldsm4t(f, row + (((c * 2 + half) ^ (r & 7)) * 16));
        mma16816(o[2 * c], pf, f[0], f[1]);
        mma16816(o[2 * c + 1], pf, f[2], f[3]);
        mma16816(o[2 * c], pl, f[0], f[1]);
        mma16816(o[2 * c + 1], pl, f[2], f[3]);
      }
    }
    __syncwarp();  // every lane has read the stage
    if (++st == NST) st = 0;
  }
  cp_async_wait<0>();
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(FULL, l[r], 1);
    l[r] += __shfl_xor_sync(FULL, l[r], 2);
    if ((lane & 3) == 0) {
      tl->m[warp][(lane >> 2) + 8 * r] = m[r];
      tl->l[warp][(lane >> 2) + 8 * r] = l[r];
    }
  }
  __syncthreads();  // no warp reads the ring any more
  float* wo = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int g = (lane >> 2) + 8 * r;
    if (g < J.heads)
#pragma unroll
      for (int x = 0; x < DP / 8; ++x)
        *reinterpret_cast<float2*>(wo + (warp * HM + g) * DP + x * 8 + (lane & 3) * 2) =
            make_float2(o[x][2 * r], o[x][2 * r + 1]);
  }
  decode_join<DP, W, HM, __nv_bfloat16>(a, J, tl, wo, logits);
}

// ---------------------------------------------------------------------------
// fp32 on the CUDA cores, up to HM query heads a launch: a lane holds half a key's
// row for the products with q, and 4 columns of the output (or 2 x 4) for those with v.
// ---------------------------------------------------------------------------
template <int DP, int W, int NST, int HM>
constexpr size_t decode_f32_smem() {
  return (size_t)W * NST * 2 * DT * DP * 4 + HM * DP * 4 + W * DT * HM * 4 +
         sizeof(Tail<DP, W, HM>);
}

template <int DP, int W, int NST, int HM>
__global__ void __launch_bounds__(W * 32) k_decode_f32(DecodeArgs a) {
  constexpr int ROWB = DP * 4, STAGE = 2 * DT * ROWB, P = DP / 4;
  static_assert(W * NST * STAGE >= W * HM * DP * 4, "the ring holds the warps' output rows");
  extern __shared__ __align__(128) char smem[];
  float* qs = reinterpret_cast<float*>(smem + W * NST * STAGE);  // [HM][DP]
  float* ps = qs + HM * DP;                                      // [W][DT][HM]
  Tail<DP, W, HM>* tl = reinterpret_cast<Tail<DP, W, HM>*>(ps + W * DT * HM);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  char* ring = smem + warp * NST * STAGE;
  float* pw = ps + warp * DT * HM;
  grid_dep_wait();
  DecodeJob J;
  J.init(a, HM);
  float* logits = nullptr;
  if (a.scores)
    logits = a.chunk_smem ? reinterpret_cast<float*>(tl + 1)
                          : a.logits + (((long long)J.b * a.c.Hkv + J.h) * J.splits + J.split) *
                                           HM * a.chunk;
  const int turns = ceil_div(J.v1 - J.v0, DT);
  const int rowbytes = a.c.d * 4;
#pragma unroll
  for (int p = 0; p < NST - 1; ++p) {
    const int t = warp + p * W;
    if (t < turns) turn_copy<ROWB>(a, ring + p * STAGE, turn_row(a, J, t, lane, 4), lane, rowbytes);
    cp_async_commit();
  }
  if (a.k_new && J.split == J.splits - 1 && warp == W - 1) append_new(a, J, 4, lane);
  for (int x = threadIdx.x; x < HM * DP; x += W * 32) {
    const int g = x / DP, y = x - g * DP;
    qs[x] = g < J.heads && y < a.c.d
                ? reinterpret_cast<const float*>(a.q)[J.b * a.q_row +
                                                      (J.h * a.G + a.h0 + g) * a.q_head + y]
                : 0.f;
  }
  __syncthreads();
  constexpr int NC = P >= 32 ? P / 32 : 1;   // output pieces of a lane
  constexpr int KS = P >= 32 ? 1 : 32 / P;   // lanes that share a piece, alternate keys
  float o[HM][NC * 4];
  float m[HM], l[HM];
#pragma unroll
  for (int g = 0; g < HM; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int x = 0; x < NC * 4; ++x) o[g][x] = 0.f;
  }
  const char* next = nullptr;
  if (warp + (NST - 1) * W < turns) next = turn_row(a, J, warp + (NST - 1) * W, lane, 4);
  int st = 0;
  for (int t = warp; t < turns; t += W) {
    cp_async_wait<NST - 2>();
    __syncwarp();
    {
      const int tn = t + (NST - 1) * W;
      int sn = st + NST - 1;
      if (sn >= NST) sn -= NST;
      if (tn < turns) turn_copy<ROWB>(a, ring + sn * STAGE, next, lane, rowbytes);
      cp_async_commit();
      if (tn + W < turns) next = turn_row(a, J, tn + W, lane, 4);
    }
    const char* kb = ring + st * STAGE;
    const char* vb = kb + DT * ROWB;
    const int key = lane & 15, half = lane >> 4;
    float s[HM];
#pragma unroll
    for (int g = 0; g < HM; ++g) s[g] = 0.f;
#pragma unroll 4
    for (int c = 0; c < P / 2; ++c) {
      const int pc = half * (P / 2) + c;
      const float4 kv = *reinterpret_cast<const float4*>(kb + key * ROWB + ((pc ^ (key & 7)) * 16));
#pragma unroll
      for (int g = 0; g < HM; ++g) {
        const float4 qv = *reinterpret_cast<const float4*>(qs + g * DP + pc * 4);
        s[g] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, s[g]))));
      }
    }
    const int x = J.v0 + t * DT + key;
#pragma unroll
    for (int g = 0; g < HM; ++g) {
      s[g] += __shfl_xor_sync(FULL, s[g], 16);
      s[g] = x < J.v1 ? s[g] * a.scale2 : -INFINITY;
      if (a.scores && half == 0 && x < J.v1 && g < J.heads)
        logits[(long long)g * a.chunk + (x - J.v0)] = s[g];
      float mx = s[g];
#pragma unroll
      for (int w = 1; w < 16; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, w));
      const float mn = fmaxf(m[g], mx), base = mn == -INFINITY ? 0.f : mn;
      if (mn > m[g]) {  // the same in every lane
        const float f = exp2_fast(m[g] - base);
        l[g] *= f;
#pragma unroll
        for (int y = 0; y < NC * 4; ++y) o[g][y] *= f;
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
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int pc = piece + c * 32;
        const float4 vv = *reinterpret_cast<const float4*>(vb + k * ROWB + ((pc ^ (k & 7)) * 16));
#pragma unroll
        for (int g = 0; g < HM; ++g) {
          const float p = pw[k * HM + g];
          o[g][4 * c + 0] = fmaf(p, vv.x, o[g][4 * c + 0]);
          o[g][4 * c + 1] = fmaf(p, vv.y, o[g][4 * c + 1]);
          o[g][4 * c + 2] = fmaf(p, vv.z, o[g][4 * c + 2]);
          o[g][4 * c + 3] = fmaf(p, vv.w, o[g][4 * c + 3]);
        }
      }
    }
    __syncwarp();
    if (++st == NST) st = 0;
  }
  cp_async_wait<0>();
#pragma unroll
  for (int g = 0; g < HM; ++g) {
    const float L = warp_sum(l[g]);
    if (lane == 0) {
      tl->m[warp][g] = m[g];
      tl->l[warp][g] = L;
    }
    if (KS > 1) {
#pragma unroll
      for (int w = P; w < 32; w <<= 1)
#pragma unroll
        for (int y = 0; y < NC * 4; ++y) o[g][y] += __shfl_xor_sync(FULL, o[g][y], w);
    }
  }
  __syncthreads();
  float* wo = reinterpret_cast<float*>(smem);
  if (P >= 32 || lane < P) {
#pragma unroll
    for (int g = 0; g < HM; ++g)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        *reinterpret_cast<float4*>(wo + (warp * HM + g) * DP + (lane + c * 32) * 4) =
            make_float4(o[g][4 * c], o[g][4 * c + 1], o[g][4 * c + 2], o[g][4 * c + 3]);
  }
  decode_join<DP, W, HM, float>(a, J, tl, wo, logits);
}

constexpr int MAX_SPLITS = 16;

int heads_per_launch(int dtype, int G) { return dtype == GMC_BF16 ? 16 : G > 4 ? 8 : G > 2 ? 4 : G; }

// CTAs of a (sequence, key head): as many as fill the GPU twice, 64 seen keys each at
// least.  A power of two: clusters of other sizes leave more SMs of a group idle.
int decode_splits(const DecodeArgs& a) {
  long long most = a.c.cap;
  if (a.window > 0) most = std::min(most, (long long)a.window + a.sinks);
  int s = 1;
  while (s < MAX_SPLITS && (long long)a.c.B * a.c.Hkv * s < 2 * 152 && most > 64LL * s) s *= 2;
  return s;
}

template <typename K>
cudaError_t decode_launch(K kernel, size_t smem, size_t logits, int threads, int splits,
                          DecodeArgs a, cudaStream_t st) {
  a.chunk_smem = logits <= D_SMEM_LOGITS && smem + logits <= 227 * 1024;
  if (a.chunk_smem) smem += logits;
  cudaError_t e = set_smem_limit((const void*)kernel, smem);
  if (e != cudaSuccess) return e;
  if (splits > 8) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_k(kernel, dim3(splits, a.c.Hkv, a.c.B), dim3(threads), smem, st, splits, a);
}
}  // namespace

size_t decode_workspace(const KV& c, int dtype, int H) {
  // logits of the launches whose share does not fit shared memory
  const int hm = heads_per_launch(dtype, H / c.Hkv);
  return 256 + (size_t)c.B * c.Hkv * hm * 4 * ((size_t)c.cap + MAX_SPLITS * DT);
}

cudaError_t launch_decode(DecodeArgs a, int dtype, void* ws, cudaStream_t st, int* launches) {
  const int hm = heads_per_launch(dtype, a.G);
  const int splits = decode_splits(a);
  long long most = a.c.cap;
  if (a.window > 0) most = std::min(most, (long long)a.window + a.sinks);
  a.chunk = ceil_div(ceil_div((int)most, splits), DT) * DT;
  a.logits = reinterpret_cast<float*>(ws);
  const size_t lg = a.scores ? (size_t)a.chunk * hm * 4 : 0;
  const int dp = a.c.d <= 64 ? 64 : a.c.d <= 128 ? 128 : 256;
  for (a.h0 = 0; a.h0 < a.G; a.h0 += hm) {
    // key heads with more query heads than a launch takes: one launch after another,
    // each adding to the scores of the one before
    a.fresh = a.h0 == 0 && a.k_new != nullptr;
    if (a.h0 > 0) a.scores = a.scores ? a.out_scores : nullptr;
    cudaError_t e;
#define GMC_BF(DP, W, N) \
  decode_launch(k_decode_bf16<DP, W, N>, decode_bf16_smem<DP, W, N>(), lg, W * 32, splits, a, st)
#define GMC_F3(DP, W, N, HM)                                                                   \
  decode_launch(k_decode_f32<DP, W, N, HM>, decode_f32_smem<DP, W, N, HM>(), lg, W * 32,       \
                splits, a, st)
#define GMC_F3H(DP, W, N)                                                                      \
  (hm == 1 ? GMC_F3(DP, W, N, 1) : hm == 2 ? GMC_F3(DP, W, N, 2)                               \
   : hm == 4 ? GMC_F3(DP, W, N, 4) : GMC_F3(DP, W, N, 8))
    if (dtype == GMC_BF16)
      e = dp == 64 ? GMC_BF(64, 4, 4) : dp == 128 ? GMC_BF(128, 4, 3) : GMC_BF(256, 4, 2);
    else
      e = dp == 64 ? GMC_F3H(64, 4, 3) : dp == 128 ? GMC_F3H(128, 4, 3) : GMC_F3H(256, 2, 3);
#undef GMC_BF
#undef GMC_F3
#undef GMC_F3H
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

}  // namespace gmc
