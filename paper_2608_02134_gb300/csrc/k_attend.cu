// Causal attention of new tokens over a paged key-value cache on the CUDA cores: head
// sizes above 128, and bf16 caches whose pages are not a multiple of 8 slots.
//
// A CTA takes 64 rows, the query heads of one key head of some consecutive tokens (so
// each key is read once for all of them), and walks the seen keys 64 at a time with a
// running maximum and sum for every row.  A thread holds 8 (4 at d > 128) rows x 4 keys
// of the logits and 8 x 8 (4 x 16) of the output in registers; queries, keys, values and
// weights are fp32 in shared memory, read four at a time.  Two multiply-adds go into an
// instruction; two CTAs an SM (one at d > 128) wait for each other's loads.  The keys'
// copies run behind the products with the values and the values' behind the logits.
// Where the rows are too few to fill the GPU the keys are split over CTAs and a second
// kernel joins them.  1,000 tokens of 28 heads of 128 in bf16 (pages of 20 slots): 335 us,
// 21 TFLOP/s causal; of 16 heads of 256 in fp32: 344 us, 24.
#include <algorithm>

#include "cache.cuh"

namespace gmc {

namespace {
constexpr int AT_K = 64;
constexpr int AT_MAX_SPLITS = 32;

constexpr int AT_ROWS = 64;
template <int DP> constexpr int at_threads() { return DP > 128 ? 256 : 128; }
template <int DP> constexpr size_t at_smem() {
  return (size_t)AT_ROWS * DP * 4 + 2 * (size_t)AT_K * DP * 4 + AT_ROWS * AT_K * 4 +
         2 * AT_K * 8;
}

// o += weights x values of one tile; SKIP: zero weights are left out.
template <int RT, int NC, bool SKIP>
__device__ __forceinline__ void times_values(f32x2 (&o)[RT][NC * 2], const char* Pr,
                                             const char* Vs, int tx, int sw) {
#pragma unroll 1
  for (int k4 = 0; k4 < AT_K / 4; ++k4) {
    float4 pv[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
      pv[i] = *reinterpret_cast<const float4*>(Pr + i * AT_K * 4 + ((k4 ^ sw) * 16));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = k4 * 4 + e;
      ulonglong2 vv[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c)
        vv[c] = *reinterpret_cast<const ulonglong2*>(Vs + k * (NC * 256) +
                                                     (((tx + 16 * c) ^ (k & 7)) * 16));
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float p = e == 0 ? pv[i].x : e == 1 ? pv[i].y : e == 2 ? pv[i].z : pv[i].w;
        if (SKIP && p == 0.f) continue;
        const f32x2 pp = pair(p, p);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          o[i][2 * c] = fma2(pp, vv[c].x, o[i][2 * c]);
          o[i][2 * c + 1] = fma2(pp, vv[c].y, o[i][2 * c + 1]);
        }
      }
    }
  }
}

template <typename T, int DP>
__global__ void __launch_bounds__(at_threads<DP>(), DP > 128 ? 1 : 2) k_attend_simt(AttnArgs a, int gsub, int ntile) {
  constexpr int R = AT_ROWS, AT_THREADS = at_threads<DP>(), RT = R * 16 / AT_THREADS, P = DP / 4, NC = DP / 64, E = 16 / sizeof(T);
  extern __shared__ __align__(128) char smem[];
  char* Qs = smem;
  char* Ks = Qs + R * DP * 4;
  char* Vs = Ks + AT_K * DP * 4;
  char* Ps = Vs + AT_K * DP * 4;
  long long* offs = reinterpret_cast<long long*>(Ps + R * AT_K * 4);  // [2][AT_K]
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.z;
  const int ng = ceil_div(a.G, gsub);
  const int h = blockIdx.y / ng, hg = (blockIdx.y - h * ng) * gsub;
  const int split = blockIdx.x % a.splits;
  const int tpt = R / gsub;
  // the last tokens see the most keys: they go first
  const int t0 = (ntile - 1 - (int)blockIdx.x / a.splits) * tpt;
  const NewRows nr = new_rows(a.q_offsets, b, a.rows, a.T, a.c.status);
  const int nt = min(tpt, nr.T - t0);
  if (nt <= 0) return;
  const int n = kv_len(a.c, b);
  const int i0 = n - nr.T + t0;  // place of the first token of the tile
  const Seen seen = seen_keys(i0, i0 + nt - 1, a.window, a.sinks);
  const int na = ceil_div(seen.a, AT_K), nb = ceil_div(seen.b1 - seen.b0, AT_K);
  const int per = ceil_div(na + nb, a.splits);
  const int u0 = min(na + nb, split * per), u1 = min(na + nb, u0 + per);
  auto key0 = [&](int u) { return u < na ? u * AT_K : seen.b0 + (u - na) * AT_K; };
  auto key1 = [&](int u) { return u < na ? seen.a : seen.b1; };
  auto look_up = [&](int u) {
    if (tid < AT_K && u < u1) {
      const int j = key0(u) + tid;
      offs[(u & 1) * AT_K + tid] = j < key1(u) ? kv_row(a.c, b, h, j) : -1;
    }
  };
  // one tile's rows into shared memory as fp32, piece p of row r at p ^ (r & 7)
  auto copy_rows = [&](char* dst, const char* pool, int u) {
    for (int x = tid; x < AT_K * (DP / E); x += AT_THREADS) {
      const int r = x / (DP / E), p = x - r * (DP / E);
      const long long o = offs[(u & 1) * AT_K + r];
      const bool ok = o >= 0 && p * E < a.c.d;
      const char* src = ok ? pool + o * (long long)sizeof(T) + p * 16 : pool;
      if constexpr (sizeof(T) == 4) {
        cp_async16(dst + r * DP * 4 + ((p ^ (r & 7)) * 16), src, ok);
      } else {
        int4 raw = make_int4(0, 0, 0, 0);
        if (ok) raw = *reinterpret_cast<const int4*>(src);
        const __nv_bfloat162* e = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float2 lo = __bfloat1622float2(e[2 * q]), hi = __bfloat1622float2(e[2 * q + 1]);
          *reinterpret_cast<float4*>(dst + r * DP * 4 + (((2 * p + q) ^ (r & 7)) * 16)) =
              make_float4(lo.x, lo.y, hi.x, hi.y);
        }
      }
    }
    cp_async_commit();
  };
  look_up(u0);
  for (int x = tid; x < R * P; x += AT_THREADS) {
    const int r = x / P, p = x - r * P;
    const int t = r / gsub, g = hg + r - t * gsub;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t < nt && g < a.G && p * 4 < a.c.d) {
      const T* q = reinterpret_cast<const T*>(a.q) + (long long)(nr.off + t0 + t) * a.q_row +
                   (long long)(h * a.G + g) * a.q_head + p * 4;
      v = make_float4(to_f32(q[0]), to_f32(q[1]), to_f32(q[2]), to_f32(q[3]));
    }
    *reinterpret_cast<float4*>(Qs + r * DP * 4 + ((p ^ ((r / RT) & 7)) * 16)) = v;
  }
  __syncthreads();
  if (u0 < u1) copy_rows(Ks, a.c.k, u0);

  f32x2 o[RT][NC * 2];  // columns in pairs
  float m[RT], l[RT];
  int place[RT];  // of the row's token; below 0 also for rows that are none
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r = ty * RT + i, t = r / gsub;
    place[i] = t < nt ? i0 + t : -1;
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int y = 0; y < NC * 2; ++y) o[i][y] = 0ull;
  }
  const int sw = ty & 7;
  for (int u = u0; u < u1; ++u) {
    cp_async_wait<0>();
    look_up(u + 1);
    __syncthreads();  // the keys of u are there; the values of u - 1 are done with
    copy_rows(Vs, a.c.v, u);
    float s[RT][4];
    {
      f32x2 z[RT][4];  // sums over even and odd columns
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) z[i][c] = 0ull;
#pragma unroll 2
      for (int p = 0; p < P; ++p) {
        ulonglong2 kv[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int r = tx + 16 * c;
          kv[c] = *reinterpret_cast<const ulonglong2*>(Ks + r * DP * 4 + ((p ^ (r & 7)) * 16));
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const ulonglong2 qv =
              *reinterpret_cast<const ulonglong2*>(Qs + (ty * RT + i) * DP * 4 + ((p ^ sw) * 16));
#pragma unroll
          for (int c = 0; c < 4; ++c) z[i][c] = fma2(qv.y, kv[c].y, fma2(qv.x, kv[c].x, z[i][c]));
        }
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float2 v = unpair(z[i][c]);
          s[i][c] = v.x + v.y;
        }
    }
    const int j0 = key0(u), j1 = key1(u);
    // whether every row sees every key of the tile
    const bool whole = j0 + AT_K <= j1 && j0 + AT_K - 1 <= i0 &&
                       (a.window == 0 || i0 + nt - 1 - j0 < a.window || j0 + AT_K <= a.sinks);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = j0 + tx + 16 * c;
        const bool ok = whole || (j < j1 && sees(place[i], j, a.window, a.sinks));
        s[i][c] = ok ? s[i][c] * a.scale2 : -INFINITY;
        mx = fmaxf(mx, s[i][c]);
      }
#pragma unroll
      for (int w = 1; w < 16; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, w));
      const float mn = fmaxf(m[i], mx), base = mn == -INFINITY ? 0.f : mn;
      const float f = exp2_fast(m[i] - base);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float p = exp2_fast(s[i][c] - base);
        sum += p;
        const int k = tx + 16 * c;
        *reinterpret_cast<float*>(Ps + (ty * RT + i) * AT_K * 4 + (((k >> 2) ^ sw) * 16) +
                                  (k & 3) * 4) = p;
      }
      l[i] = l[i] * f + sum;
      if (f != 1.f) {
        const f32x2 ff = pair(f, f);
#pragma unroll
        for (int y = 0; y < NC * 2; ++y) o[i][y] = mul2(o[i][y], ff);
      }
    }
    __syncthreads();  // the keys of u are done with, the weights written
    if (u + 1 < u1) copy_rows(Ks, a.c.k, u + 1); else cp_async_commit();
    cp_async_wait<1>();
    __syncthreads();  // the values of u are there
    // a weight of zero does not meet a value that is not finite: a row that does not
    // see a key must not take a NaN from it
    bool strange = false;
    if (!whole) {
      for (int x = tid; x < AT_K * P; x += AT_THREADS) {
        const float4 v = reinterpret_cast<const float4*>(Vs)[x];
        strange |= !(fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY && fabsf(v.z) < INFINITY &&
                     fabsf(v.w) < INFINITY);
      }
      strange = __syncthreads_or(strange);
    }
    if (!strange)
      times_values<RT, NC, false>(o, Ps + ty * RT * AT_K * 4, Vs, tx, sw);
    else
      times_values<RT, NC, true>(o, Ps + ty * RT * AT_K * 4, Vs, tx, sw);
  }
  cp_async_wait<0>();
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    float L = l[i];
#pragma unroll
    for (int w = 1; w < 16; w <<= 1) L += __shfl_xor_sync(FULL, L, w);
    const int r = ty * RT + i, t = r / gsub, g = hg + r - t * gsub;
    if (t >= nt || g >= a.G) continue;
    const long long row = nr.off + t0 + t;
    const int hq = h * a.G + g;
    if (a.splits > 1) {
      const long long pr = part_row(a, split, b, t0 + t) * a.H + hq;
      if (tx == 0) a.ml[pr] = make_float2(m[i], L);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int x = (tx + 16 * c) * 4;
        const float2 lo = unpair(o[i][2 * c]), hi = unpair(o[i][2 * c + 1]);
        if (x < a.c.d)
          *reinterpret_cast<float4*>(a.part + pr * a.c.d + x) =
              make_float4(lo.x, lo.y, hi.x, hi.y);
      }
      continue;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (a.lse && tx == 0)
      a.lse[row * a.H + hq] = L == 0.f ? -INFINITY : (m[i] + log2f(L)) * LN2;
    T* out = reinterpret_cast<T*>(a.out) + row * a.o_row + hq * a.o_head;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int x = (tx + 16 * c) * 4;
      if (x >= a.c.d) continue;
      const float2 lo = unpair(o[i][2 * c]), hi = unpair(o[i][2 * c + 1]);
      out[x] = from_f32<T>(lo.x * inv);
      out[x + 1] = from_f32<T>(lo.y * inv);
      out[x + 2] = from_f32<T>(hi.x * inv);
      out[x + 3] = from_f32<T>(hi.y * inv);
    }
  }
}

// One warp a (new token, query head): out = sum_s w_s part_s / sum_s w_s l_s,
// w_s = 2^(m_s - max m).
template <typename T>
__global__ void __launch_bounds__(256) k_attend_join(AttnArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  const long long step = part_row(a, 1, 0, 0) * a.H;
  const long long x = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (x >= step) return;
  constexpr int U = 4;
  auto load = [&](int y0, int q0, float4* v) {  // of four parts
    const float* part = a.part + x * a.c.d + min(y0 + lane * 4, a.c.d - 4);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q0 + u < a.splits)
        v[u] = *reinterpret_cast<const float4*>(part + (q0 + u) * step * a.c.d);
  };
  float4 v[U];
  load(0, 0, v);  // on their way while the row and the weights are looked up
  // divisions of 32 bits where the numbers are: 57,344 rows of two parts 25.2 us, with 64 bits 26.4
  const bool small = step <= 0xffffffffLL;
  const long long token = small ? (unsigned)x / (unsigned)a.H : x / a.H;
  const int hq = (int)(x - token * a.H);
  const int b = (int)(small ? (unsigned)token / (unsigned)a.T : token / a.T);
  const int t = (int)(token - (long long)b * a.T);
  const NewRows nr = new_rows(a.q_offsets, b, a.rows, a.T, a.c.status);
  if (t >= nr.T) return;
  const long long row = nr.off + t;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < a.splits) ml = a.ml[lane * step + x];
  const float M = warp_max(ml.x), base = M == -INFINITY ? 0.f : M;
  const float w = exp2_fast(ml.x - base);
  const float L = warp_sum(ml.y * w);
  const float inv = L == 0.f ? 0.f : 1.f / L;
  if (a.lse && lane == 0)
    a.lse[row * a.H + hq] = L == 0.f ? -INFINITY : (base + log2f(L)) * LN2;
  T* out = reinterpret_cast<T*>(a.out) + row * a.o_row + hq * a.o_head;
  for (int y0 = 0; y0 < a.c.d; y0 += 128) {
    const int y = y0 + lane * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q0 = 0; q0 < a.splits; q0 += U) {
      if (y0 + q0 > 0) load(y0, q0, v);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int q = q0 + u;
        if (q >= a.splits) break;
        const float mq = __shfl_sync(FULL, ml.x, q), f = __shfl_sync(FULL, w, q);
        if (mq == -INFINITY) v[u] = make_float4(0.f, 0.f, 0.f, 0.f);  // no keys: wrote no row
        s.x += f * v[u].x;
        s.y += f * v[u].y;
        s.z += f * v[u].z;
        s.w += f * v[u].w;
      }
    }
    if (y < a.c.d) {  // rows and heads lie 16 bytes apart
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(out + y) =
            make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv);
      } else {
        const T z[4] = {from_f32<T>(s.x * inv), from_f32<T>(s.y * inv), from_f32<T>(s.z * inv),
                        from_f32<T>(s.w * inv)};
        uint2 both;
        memcpy(&both, z, 8);
        *reinterpret_cast<uint2*>(out + y) = both;
      }
    }
  }
}

// Parts of the key axis: where the rows' tiles leave SMs idle, as many as fill them,
// four turns of 64 keys each at least.
int simt_splits(const KV& c, int G, int T) {
  const int R = AT_ROWS, gsub = std::min(G, R);
  const long long ctas =
      (long long)c.B * c.Hkv * ceil_div(G, gsub) * ceil_div(T, std::max(1, R / gsub));
  const int fill = (c.d > 128 ? 1 : 2) * sm_count();
  if (ctas >= fill / 2) return 1;
  return (int)std::max<long long>(
      1, std::min<long long>({fill / ctas, AT_MAX_SPLITS, ceil_div(c.cap, 4 * AT_K)}));
}
int attend_splits(const KV& c, int dtype, int G, int T) {
  return attend_tc_takes(c, dtype, G) ? attend_tc_splits(c, G, T)
         : attend_f32_takes(c, dtype) ? attend_f32_splits(c, G, T)
                                      : simt_splits(c, G, T);
}
}  // namespace

size_t attend_workspace(const KV& c, int dtype, int H, int T, int splits) {
  const int G = H / c.Hkv;
  const int s = splits ? splits : attend_splits(c, dtype, G, T);
  if (s == 1) return 256;
  const size_t rows = (size_t)c.B * T * H * s;
  return 256 + ((rows * 8 + 255) & ~(size_t)255) + rows * c.d * 4;
}

cudaError_t launch_attend_join(const AttnArgs& a, int dtype, cudaStream_t st) {
  const unsigned grid = (unsigned)(((long long)a.c.B * a.T * a.H + 7) / 8);
  return dtype == GMC_BF16
             ? launch_k(k_attend_join<__nv_bfloat16>, dim3(grid), dim3(256), 0, st, 1, a)
             : launch_k(k_attend_join<float>, dim3(grid), dim3(256), 0, st, 1, a);
}

cudaError_t launch_attend(AttnArgs a, int dtype, void* ws, cudaStream_t st, int* launches,
                          int splits) {
  const int R = AT_ROWS, gsub = std::min(a.G, R), ng = ceil_div(a.G, gsub);
  const int ntile = ceil_div(a.T, R / gsub);
  a.splits = splits ? splits : attend_splits(a.c, dtype, a.G, a.T);
  if (a.splits > 1) {
    const size_t rows = (size_t)a.c.B * a.T * a.H * a.splits;
    a.ml = reinterpret_cast<float2*>(ws);
    a.part = reinterpret_cast<float*>((char*)ws + ((rows * 8 + 255) & ~(size_t)255));
  }
  const dim3 grid((unsigned)ntile * a.splits, a.c.Hkv * ng, a.c.B);
  cudaError_t e;
#define GMC_AT(T, DP)                                                                     \
  ((e = set_smem_limit((const void*)k_attend_simt<T, DP>, at_smem<DP>())) != cudaSuccess  \
       ? e                                                                                \
       : launch_k(k_attend_simt<T, DP>, grid, dim3(at_threads<DP>()), at_smem<DP>(), st, 1, a,  \
                  gsub, ntile))
  if (attend_tc_takes(a.c, dtype, a.G))
    e = launch_attend_tc(a, st);
  else if (attend_f32_takes(a.c, dtype))
    e = launch_attend_f32(a, st);
  else if (dtype == GMC_BF16)
    e = a.c.d <= 64 ? GMC_AT(__nv_bfloat16, 64)
                    : a.c.d <= 128 ? GMC_AT(__nv_bfloat16, 128) : GMC_AT(__nv_bfloat16, 256);
  else
    e = GMC_AT(float, 256);
#undef GMC_AT
  if (e != cudaSuccess) return e;
  ++*launches;
  if (a.splits > 1) {
    if ((e = launch_attend_join(a, dtype, st)) != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

}  // namespace gmc
