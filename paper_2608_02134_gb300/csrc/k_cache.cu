// The key-value cache's own kernels: new rows written to their pages, and the
// best-scored rows of a sequence moved to fresh pages.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "cache.cuh"

namespace gmc {

namespace {
constexpr int AP_THREADS = 256, AP_ROWS = 64;

// Rows t0 .. of one sequence's new keys and values.  Bound by memory: every byte is
// read once and written once, 16 bytes a lane, four keys' and four values' loads in
// flight; the rows' places in the pages are looked up once into shared memory.
// 8 x 16,004 rows of 4 heads of 128 in bf16: 81.4 us, 6.4 TB/s.
__global__ void __launch_bounds__(AP_THREADS)
    k_cache_append(KV c, const char* __restrict__ k_new, const char* __restrict__ v_new,
                   const int32_t* __restrict__ offsets, int rows, int T, int esize, int tile) {
  __shared__ long long at[AP_ROWS];
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.y, t0 = blockIdx.x * tile;
  // the length and the offsets on their way together
  const int len = __ldcg(c.lens + b);
  const NewRows nr = new_rows(offsets, b, rows, T, c.status);
  const int nt = min(tile, nr.T - t0);
  if (nt <= 0) return;
  const int first = kv_clamp(c, len) - nr.T + t0;
  if ((int)threadIdx.x < nt) {
    const int j = first + (int)threadIdx.x;
    if (j < 0) set_status(c.status, CACHE_BAD);
    at[threadIdx.x] = j < 0 ? -1 : kv_row(c, b, 0, j);
  }
  const int hc = c.d * esize / 16;  // 16-byte pieces of a head's row
  const int rc = hc * c.Hkv;
  const char *ks, *vs;
  if (v_new) {
    ks = k_new + (long long)(nr.off + t0) * rc * 16;
    vs = v_new + (long long)(nr.off + t0) * rc * 16;
  } else {
    ks = k_new + (2LL * nr.off + t0) * rc * 16;
    vs = k_new + (2LL * nr.off + nr.T + t0) * rc * 16;
  }
  const int total = nt * rc;
  constexpr int U = 4;
  bool looked = false;
  for (int x0 = threadIdx.x;; x0 += AP_THREADS * U) {
    int4 kv[U], vv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * AP_THREADS;
      if (x < total) {
        kv[u] = __ldcs((const int4*)ks + x);
        vv[u] = __ldcs((const int4*)vs + x);
      }
    }
    if (!looked) __syncthreads();  // the first rows load while their places are looked up
    looked = true;
    if (x0 >= total) break;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * AP_THREADS;
      if (x >= total) break;
      const int r = x / rc, y = x - r * rc, h = y / hc, z = y - h * hc;
      if (at[r] < 0) continue;
      const long long o = (at[r] + h * c.head_stride) * esize + z * 16;
      *(int4*)(c.k + o) = kv[u];
      *(int4*)(c.v + o) = vv[u];
    }
  }
}

// ---------------------------------------------------------------------------
// Eviction: S CTAs a (sequence, key head), each of which finds the same threshold from
// all of the pair's scores (they are a hundredth of the rows' bytes; finding it once and
// telling the others took a cluster's barriers, 17.4 us for 4 x 16,004 places where this
// took 14.9), and then writes and copies an equal part of the kept places.  12.4 us now,
// most of it the chain from the scores to the places; 32 sequences of up to 1,027 places,
// 385 kept, 13.7 us.
//
// The threshold, the keep-th largest of the scores' order-preserving 32-bit keys, is
// found in three passes of 11, 11 and 10 bits over a histogram in shared memory; keys
// equal to it are taken from the lowest place on.  A thread holds 2, 4, 8 or 16 consecutive
// keys in registers, through all passes where the sequence has no more than 16,384 places,
// so one scan over the threads' counts numbers the kept places.
// ---------------------------------------------------------------------------
constexpr int EV_THREADS = 1024, EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048, EV_COPIES = 4;  // copies by lane: fewer meet at one address
constexpr int EV_LIST = 8192;                 // kept places of a CTA held in shared memory

struct EvSmem {
  int hist[2][EV_BINS * EV_COPIES];  // one is cleared while the other counts
  int list[EV_LIST];
  long long src[EV_THREADS], dst[EV_THREADS];
  int wsum[2][EV_WARPS];
  uint32_t prefix;
  int need;
};

// Larger score, larger key; -0 equals 0, a NaN is as -infinity.
__device__ __forceinline__ uint32_t score_key(float s) {
  if (!(s == s)) return 0x007fffffu;  // -infinity's
  const uint32_t u = __float_as_uint(s + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// One more in a shared word, without a branch around it.
__device__ __forceinline__ void count_if(uint32_t addr, bool yes) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "@p red.shared.add.u32 [%0], 1;\n\t}" ::"r"(addr),
      "r"((uint32_t)yes)
      : "memory");
}

// Exclusive sums over the warp's lanes.
__device__ __forceinline__ int lanes_before(int v) {
  const int lane = threadIdx.x & 31;
  int sum = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(FULL, sum, o);
    if (lane >= o) sum += y;
  }
  return sum - v;
}

template <int E>
__global__ void __launch_bounds__(EV_THREADS, 1) k_evict(EvictArgs a, int esize, int vec) {
  extern __shared__ __align__(16) char ev_raw[];
  EvSmem* s = reinterpret_cast<EvSmem*>(ev_raw);
  const int r = blockIdx.x, S = gridDim.x, h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto clear = [&](int which) {
    for (int x = tid; x < EV_BINS * EV_COPIES / 4; x += EV_THREADS)
      reinterpret_cast<int4*>(s->hist[which])[x] = make_int4(0, 0, 0, 0);
  };
  clear(0);
  grid_dep_launch();
  grid_dep_wait();
  const long long pair = (long long)b * a.src.Hkv + h;
  const float* sc = a.scores + pair * a.score_stride;
  // this thread's places of a chunk: E from `at` on.  A row holds cap scores, so they are
  // on their way before the sequence's length is known
  constexpr int chunk = EV_THREADS * E;
  float v[E];
  uint32_t key[E];
  int at;
  auto fetch = [&](int c) {
    at = c * chunk + tid * E;
    if (E >= 4 && vec && at + E <= a.src.cap) {
#pragma unroll
      for (int x = 0; x < E; x += 4)
        *reinterpret_cast<float4*>(v + x) = *reinterpret_cast<const float4*>(sc + at + x);
    } else {
#pragma unroll
      for (int x = 0; x < E; ++x) v[x] = sc[min(at + x, a.src.cap - 1)];
    }
  };
  fetch(0);
  const int n = kv_len(a.src, b);
  const int k = min(a.keep, n), tail = n - a.recent;
  auto to_keys = [&]() {  // 0 is no key's value
    if (at >= a.sinks && at + E <= tail) {
#pragma unroll
      for (int x = 0; x < E; ++x) key[x] = score_key(v[x]);
    } else {
#pragma unroll
      for (int x = 0; x < E; ++x) {
        const int j = at + x;
        key[x] = j >= n ? 0u : j < a.sinks || j >= tail ? 0xffffffffu : score_key(v[x]);
      }
    }
  };
  int32_t* oi = a.out_idx + pair * a.keep;
  float* os = a.out_scores ? a.out_scores + pair * a.keep : nullptr;
  if (r == 0) {
    if (h == 0 && tid == 0) a.dst.lens[b] = k;
    for (int x = k + tid; x < a.keep; x += EV_THREADS) {
      oi[x] = -1;
      if (os) os[x] = 0.f;
    }
  }
  // this CTA's part of the kept places
  const int each = ceil_div(k, S), p0 = min(k, r * each), p1 = min(k, p0 + each);
  if (p0 >= p1) return;
  const int chunks = ceil_div(n, chunk);
  to_keys();
  uint32_t thr = 0;  // k == n: every key is larger
  int need = 0;      // keys equal to the threshold to take; all larger ones are
  if (k < n) {
    uint32_t prefix = 0;
    need = k;
    __syncthreads();
    auto pass = [&](auto number) {
      constexpr int p = decltype(number)::value, sh = p == 0 ? 21 : p == 1 ? 10 : 0,
                    bits = p == 2 ? 10 : 11;
      const uint32_t bins = (uint32_t)__cvta_generic_to_shared(s->hist[p & 1]) + (lane & 3) * 4;
      for (int c = 0; c < chunks; ++c) {
        if (chunks > 1) {
          fetch(c);
          to_keys();
        }
#pragma unroll
        for (int x = 0; x < E; ++x) {
          const uint32_t d = key[x] - prefix;
          count_if(bins + (d >> sh) * (EV_COPIES * 4),
                   p == 0 ? key[x] != 0 : d < 1u << (sh + bits));
        }
      }
      if (p < 2) clear((p + 1) & 1);
      __syncthreads();
      // bins from the largest on, two a thread: the one whose keys reach the need-th
      int c[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int4 v =
            reinterpret_cast<const int4*>(s->hist[p & 1])[EV_BINS - 1 - 2 * tid - y];
        c[y] = v.x + v.y + v.z + v.w;
      }
      const int here = __reduce_add_sync(FULL, c[0] + c[1]);
      if (lane == 0) s->wsum[0][warp] = here;
      __syncthreads();
      const int w = s->wsum[0][lane];  // EV_WARPS == 32 totals
      int before = __shfl_sync(FULL, lanes_before(w), warp);
      if (before < need && before + here >= need) {  // it is one of this warp's
        before += lanes_before(c[0] + c[1]);
        if (before < need && before + c[0] + c[1] >= need) {
          const int y = before + c[0] >= need ? 0 : 1;
          s->prefix = prefix | ((uint32_t)(EV_BINS - 1 - 2 * tid - y) << sh);
          s->need = need - before - (y ? c[0] : 0);
        }
      }
      __syncthreads();
      prefix = s->prefix;
      need = s->need;
    };
    pass(std::integral_constant<int, 0>());
    pass(std::integral_constant<int, 1>());
    pass(std::integral_constant<int, 2>());
    thr = prefix;
  }
  // the kept places in order: larger keys and equal ones before this thread's
  int g0 = 0, e0 = 0;
  for (int c = 0; c < chunks; ++c) {
    if (chunks > 1) {
      fetch(c);
      to_keys();
    }
    int gt = 0, eq = 0;
#pragma unroll
    for (int x = 0; x < E; ++x) {
      gt += key[x] > thr;
      eq += key[x] == thr;
    }
    if (thr == 0) eq = 0;
    const int both = (gt << 16) + eq;  // at most 16,384 each over the block
    const int here = __reduce_add_sync(FULL, both);
    int* ws = s->wsum[c & 1];
    if (lane == 0) ws[warp] = here;
    __syncthreads();
    const int w = ws[lane];
    const int before = __shfl_sync(FULL, lanes_before(w), warp) + lanes_before(both);
    const int total = __reduce_add_sync(FULL, w);
    int g = g0 + (before >> 16), e = e0 + (before & 0xffff);
    if (g + min(e, need) < p1 && g + gt + min(e + eq, need) > p0) {
      const unsigned held = min(p1 - p0, EV_LIST);
#pragma unroll
      for (int x = 0; x < E; ++x) {
        const bool isg = key[x] > thr, ise = key[x] == thr && thr != 0;
        const int slot = g + min(e, need) - p0;
        const bool take = isg || (ise && e < need);
        if (take && (unsigned)slot < held) s->list[slot] = at + x;
        if (p1 - p0 > EV_LIST && take && slot >= EV_LIST && slot < p1 - p0)
          oi[p0 + slot] = at + x;
        g += isg;
        e += ise;
      }
    }
    g0 += total >> 16;
    e0 += total & 0xffff;
  }
  __syncthreads();  // this CTA's places are written
  const int rc = a.src.d * esize / 16;
  for (int q0 = p0; q0 < p1; q0 += EV_THREADS) {
    const int nr = min(EV_THREADS, p1 - q0);
    if (tid < nr) {
      const int q = q0 + tid, j = q - p0 < EV_LIST ? s->list[q - p0] : oi[q];
      const Slot from = kv_slot(a.src, b, j), to = kv_slot(a.dst, b, q);  // together
      const float score = sc[j];
      const long long so = kv_row(a.src, h, from);
      const long long dto = kv_row(a.dst, h, to);
      oi[q] = j;
      if (os) os[q] = score;
      s->src[tid] = so < 0 || dto < 0 ? -1 : so * esize;
      s->dst[tid] = dto * esize;
    }
    __syncthreads();
    const int total = nr * rc;
    constexpr int U = 4;
    for (int x = tid; x < total; x += EV_THREADS * U) {
      int4 kv[U], vv[U];
      long long at[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int y = x + u * EV_THREADS;
        at[u] = -1;
        if (y < total) {
          const int row = y / rc, z = (y - row * rc) * 16;
          if (s->src[row] >= 0) {
            at[u] = s->dst[row] + z;
            kv[u] = *(const int4*)(a.src.k + s->src[row] + z);
            vv[u] = *(const int4*)(a.src.v + s->src[row] + z);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at[u] >= 0) {
          *(int4*)(a.dst.k + at[u]) = kv[u];
          *(int4*)(a.dst.v + at[u]) = vv[u];
        }
    }
    __syncthreads();
  }
}
}  // namespace

int sm_count() {
  static std::atomic<int> known[64];  // by device; a call asks several times
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) == cudaSuccess) {
    if (dev >= 0 && dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) {
      if (dev >= 0 && dev < 64) known[dev].store(sms, std::memory_order_relaxed);
      return sms;
    }
  }
  cudaGetLastError();
  return 152;
}

cudaError_t launch_cache_append(const KV& c, int dtype, const void* k_new, const void* v_new,
                                const int32_t* offsets, int rows, int T, cudaStream_t st) {
  const int esize = dtype == GMC_BF16 ? 2 : 4;
  int tile = AP_ROWS;  // rows of a block: fewer where the blocks would not fill the GPU twice
  const long long fill = 2LL * sm_count();
  while (tile > 4 && (long long)ceil_div(T, tile) * c.B < fill) tile /= 2;
  return launch_k(k_cache_append, dim3(ceil_div(T, tile), c.B), dim3(AP_THREADS), 0, st, 1, c,
                  (const char*)k_new, (const char*)v_new, offsets, rows, T, esize, tile);
}

cudaError_t launch_evict(const EvictArgs& a, int dtype, cudaStream_t st) {
  const int esize = dtype == GMC_BF16 ? 2 : 4;
  // CTAs of a pair: as many as fill the GPU, 32 kept rows each at least
  const long long pairs = (long long)a.src.B * a.src.Hkv;
  const int S = (int)std::max<long long>(
      1, std::min<long long>(sm_count() / pairs, ceil_div(a.keep, 32)));
  const int vec = (uintptr_t)a.scores % 16 == 0 && a.score_stride % 4 == 0;
  auto go = [&](auto kernel) {
    const cudaError_t e = set_smem_limit((const void*)kernel, sizeof(EvSmem));
    if (e != cudaSuccess) return e;
    return launch_k(kernel, dim3(S, a.src.Hkv, a.src.B), dim3(EV_THREADS), sizeof(EvSmem), st, 1,
                    a, esize, vec);
  };
  // keys of a thread: as few as hold the longest sequence
  const int each = ceil_div(a.src.cap, EV_THREADS);
  return each <= 2   ? go(k_evict<2>)
         : each <= 4 ? go(k_evict<4>)
         : each <= 8 ? go(k_evict<8>)
                     : go(k_evict<16>);
}

}  // namespace gmc
