// The key-value cache's own kernels: new rows written to their pages, and the
// best-scored rows of a sequence moved to fresh pages.
#include <cooperative_groups.h>

#include "cache.cuh"

namespace cg = cooperative_groups;

namespace gmc {

namespace {
constexpr int AP_THREADS = 256, AP_ROWS = 64;

// Rows t0 .. of one sequence's new keys and values.  Bound by memory: every byte is
// read once and written once, 16 bytes a lane, four keys' and four values' loads in
// flight; the rows' places in the pages are looked up once into shared memory.
__global__ void __launch_bounds__(AP_THREADS)
    k_cache_append(KV c, const char* __restrict__ k_new, const char* __restrict__ v_new,
                   const int32_t* __restrict__ offsets, int rows, int T, int esize, int tile) {
  __shared__ long long at[AP_ROWS];
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.y, t0 = blockIdx.x * tile;
  const NewRows nr = new_rows(offsets, b, rows, T, c.status);
  const int nt = min(tile, nr.T - t0);
  if (nt <= 0) return;
  const int first = kv_len(c, b) - nr.T + t0;
  if ((int)threadIdx.x < nt) {
    const int j = first + (int)threadIdx.x;
    if (j < 0) set_status(c.status, CACHE_BAD);
    at[threadIdx.x] = j < 0 ? -1 : kv_row(c, b, 0, j);
  }
  __syncthreads();
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
  for (int x0 = threadIdx.x; x0 < total; x0 += AP_THREADS * U) {
    int4 kv[U], vv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * AP_THREADS;
      if (x < total) {
        kv[u] = __ldcs((const int4*)ks + x);
        vv[u] = __ldcs((const int4*)vs + x);
      }
    }
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
// Eviction: one cluster per (sequence, key head), CTA r owning the r-th share of
// the sequence's places.  The keep-th largest score is found by a radix search
// over the scores' order-preserving 32-bit keys, eight bits a pass: every CTA
// counts its share, the counts meet through distributed shared memory.  Keys
// equal to the threshold are taken from the lowest place on.  Then each CTA
// writes its kept places in order and copies their rows.
// ---------------------------------------------------------------------------
constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_KEYS = 8192;  // keys of a share held in shared memory; the others are read again

struct EvSmem {
  int hist[2][256];
  int wgt[EV_WARPS], weq[EV_WARPS];
  int tot_gt, tot_eq;
  uint32_t prefix;
  int need;
  long long src[EV_THREADS], dst[EV_THREADS];
  uint32_t key[EV_KEYS];
};

// Larger score, larger key; -0 equals 0, a NaN is below every number's key.
__device__ __forceinline__ uint32_t score_key(float s) {
  if (!(s == s)) return 0x007fffffu;  // as -infinity
  const uint32_t u = __float_as_uint(s + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(EV_THREADS) k_evict(EvictArgs a, int esize) {
  extern __shared__ __align__(16) char ev_raw[];
  EvSmem* s = reinterpret_cast<EvSmem*>(ev_raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), r = (int)cluster.block_rank();
  const int h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dep_launch();
  grid_dep_wait();
  const int n = kv_len(a.src, b);
  const int k = min(a.keep, n);
  const long long pair = (long long)b * a.src.Hkv + h;
  const float* sc = a.scores + pair * a.score_stride;
  int32_t* oi = a.out_idx + pair * a.keep;
  float* os = a.out_scores ? a.out_scores + pair * a.keep : nullptr;
  if (r == 0) {
    if (h == 0 && tid == 0) a.dst.lens[b] = k;
    for (int x = k + tid; x < a.keep; x += EV_THREADS) {
      oi[x] = -1;
      if (os) os[x] = 0.f;
    }
  }
  // this CTA's places [j0, j0 + m), whole warps' worth each
  const int share = (ceil_div(n, C) + 31) & ~31;
  const int j0 = min(n, r * share), m = min(share, n - j0);
  const int tail = n - a.recent;
  auto fresh_key = [&](int x) -> uint32_t {
    const int j = j0 + x;
    return (j < a.sinks || j >= tail) ? 0xffffffffu : score_key(sc[j]);
  };
  auto key_at = [&](int x) -> uint32_t { return x < EV_KEYS ? s->key[x] : fresh_key(x); };
  for (int x = tid; x < min(m, EV_KEYS); x += EV_THREADS) s->key[x] = fresh_key(x);
  uint32_t thr = 0;
  int need = 0;       // keys equal to the threshold to take; all larger ones are
  if (k < n) {
    uint32_t prefix = 0;
    need = k;
    for (int p = 0; p < 4; ++p) {
      int* hist = s->hist[p & 1];
      for (int x = tid; x < 256; x += EV_THREADS) hist[x] = 0;
      __syncthreads();
      const int sh = 24 - 8 * p;
      for (int x0 = warp * 32; x0 < m; x0 += EV_THREADS) {
        const int x = x0 + lane;
        const uint32_t kx = x < m ? key_at(x) : 0;
        const bool in = x < m && (p == 0 || ((kx ^ prefix) >> (sh + 8)) == 0);
        const uint32_t d = in ? (kx >> sh) & 255u : 256u;
        const uint32_t same = __match_any_sync(FULL, d);
        if (in && lane == __ffs(same) - 1) atomicAdd(&hist[d], __popc(same));
      }
      cluster.sync();
      int cnt = 0;
      if (tid < 256)
        for (int q = 0; q < C; ++q) cnt += cluster.map_shared_rank(hist, q)[tid];
      // the digit whose keys reach the need-th from above
      int suf = cnt;  // counts of this digit and the larger ones of its warp
      if (tid < 256) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_down_sync(FULL, suf, o);
          if (lane + o < 32) suf += y;
        }
        if (lane == 0) s->wgt[warp] = suf;
      }
      __syncthreads();
      if (tid < 256) {
        for (int w = warp + 1; w < 8; ++w) suf += s->wgt[w];
        if (suf >= need && suf - cnt < need) {
          s->prefix = prefix | ((uint32_t)tid << sh);
          s->need = need - (suf - cnt);
        }
      }
      __syncthreads();
      prefix = s->prefix;
      need = s->need;
    }
    thr = prefix;
  }
  // what this CTA keeps: warp w counts the places of its own run of the share
  const int run = ceil_div(ceil_div(m, 32), EV_WARPS) * 32;
  const int x0 = min(m, warp * run), x1 = min(m, x0 + run);
  int gt = 0, eq = 0;
  for (int x = x0; x < x1; x += 32) {
    const uint32_t kx = x + lane < x1 ? key_at(x + lane) : 0;
    const bool in = x + lane < x1;
    gt += __popc(__ballot_sync(FULL, in && (k == n || kx > thr)));
    eq += __popc(__ballot_sync(FULL, in && k < n && kx == thr));
  }
  if (lane == 0) {
    s->wgt[warp] = gt;
    s->weq[warp] = eq;
  }
  __syncthreads();
  if (tid == 0) {
    int g = 0, e = 0;
    for (int w = 0; w < EV_WARPS; ++w) {
      g += s->wgt[w];
      e += s->weq[w];
    }
    s->tot_gt = g;
    s->tot_eq = e;
  }
  cluster.sync();
  int g0 = 0, e0 = 0;  // larger and equal keys before this CTA
  for (int q = 0; q < r; ++q) {
    g0 += *cluster.map_shared_rank(&s->tot_gt, q);
    e0 += *cluster.map_shared_rank(&s->tot_eq, q);
  }
  const int p0 = g0 + min(e0, need);
  const int p1 = g0 + s->tot_gt + min(e0 + s->tot_eq, need);
  // no CTA leaves while another may read its counts; the copies need no more of them
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  for (int w = 0; w < warp; ++w) {
    g0 += s->wgt[w];
    e0 += s->weq[w];
  }
  for (int x = x0; x < x1; x += 32) {
    const bool in = x + lane < x1;
    const uint32_t kx = in ? key_at(x + lane) : 0;
    const bool isg = in && (k == n || kx > thr), ise = in && k < n && kx == thr;
    const uint32_t mg = __ballot_sync(FULL, isg), me = __ballot_sync(FULL, ise);
    const uint32_t below = (1u << lane) - 1;
    const int e = e0 + __popc(me & below);
    if (isg || (ise && e < need)) {
      const int pos = g0 + __popc(mg & below) + min(e, need);
      oi[pos] = j0 + x + lane;
      if (os) os[pos] = sc[j0 + x + lane];
    }
    g0 += __popc(mg);
    e0 += __popc(me);
  }
  __syncthreads();  // this CTA's places are written
  const int rc = a.src.d * esize / 16;
  for (int q0 = p0; q0 < p1; q0 += EV_THREADS) {
    const int nr = min(EV_THREADS, p1 - q0);
    if (tid < nr) {
      const long long so = kv_row(a.src, b, h, oi[q0 + tid]);
      const long long dto = kv_row(a.dst, b, h, q0 + tid);
      s->src[tid] = so < 0 || dto < 0 ? -1 : so * esize;
      s->dst[tid] = dto * esize;
    }
    __syncthreads();
    const int total = nr * rc;
    constexpr int U = 4;
    for (int x = tid; x < total; x += EV_THREADS * U) {
      int4 kv[U], vv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int y = x + u * EV_THREADS;
        if (y < total) {
          const int row = y / rc, z = (y - row * rc) * 16;
          if (s->src[row] >= 0) {
            kv[u] = *(const int4*)(a.src.k + s->src[row] + z);
            vv[u] = *(const int4*)(a.src.v + s->src[row] + z);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int y = x + u * EV_THREADS;
        if (y < total) {
          const int row = y / rc, z = (y - row * rc) * 16;
          if (s->src[row] >= 0) {
            *(int4*)(a.dst.k + s->dst[row] + z) = kv[u];
            *(int4*)(a.dst.v + s->dst[row] + z) = vv[u];
          }
        }
      }
    }
    __syncthreads();
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
}  // namespace

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
    cudaGetLastError();
    return 152;
  }
  return sms;
}

cudaError_t launch_cache_append(const KV& c, int dtype, const void* k_new, const void* v_new,
                                const int32_t* offsets, int rows, int T, cudaStream_t st) {
  const int esize = dtype == GMC_BF16 ? 2 : 4;
  int tile = AP_ROWS;  // rows of a block: fewer where the blocks would not fill the GPU twice
  while (tile > 4 && (long long)ceil_div(T, tile) * c.B < 304) tile /= 2;
  return launch_k(k_cache_append, dim3(ceil_div(T, tile), c.B), dim3(AP_THREADS), 0, st, 1, c,
                  (const char*)k_new, (const char*)v_new, offsets, rows, T, esize, tile);
}

cudaError_t launch_evict(const EvictArgs& a, int dtype, cudaStream_t st) {
  const int esize = dtype == GMC_BF16 ? 2 : 4;
  // CTAs of a cluster: as many as fill the GPU, a few hundred places each at least
  int C = 1;
  while (C < 16 && (long long)a.src.B * a.src.Hkv * C < 152 && a.src.cap > 256 * C) C *= 2;
  cudaError_t e = set_smem_limit((const void*)k_evict, sizeof(EvSmem));
  if (e != cudaSuccess) return e;
  if (C > 8) {
    e = cudaFuncSetAttribute(k_evict, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_k(k_evict, dim3(C, a.src.Hkv, a.src.B), dim3(EV_THREADS), sizeof(EvSmem), st, C, a,
                  esize);
}

}  // namespace gmc
