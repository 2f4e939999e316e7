// New rows written to their pages with the position rotation applied on the way (and packed
// to 4 bits where the cache holds those), and rows read back out of their pages.
#include "cache.cuh"
#include "fp4.cuh"

namespace gmc {

namespace {
constexpr int RP_THREADS = 256, RP_ROWS = 64;
constexpr int RP_HEADS = 8;  // heads a thread turns by the same angles
constexpr int RP_AHEAD = 2;  // of them loaded at once
constexpr int RP_CTAS = 4, RP_CTAS4 = 3;  // an SM
constexpr int RP_BLOCKS = 2;  // blocks of 16 loaded at once
constexpr int RP_FILL = 4;   // blocks an SM, at least

__device__ __forceinline__ void to_floats(const uint4& v, float* x, float) {
  x[0] = __uint_as_float(v.x);
  x[1] = __uint_as_float(v.y);
  x[2] = __uint_as_float(v.z);
  x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void to_floats(const uint4& v, float* x, __nv_bfloat16) {
  unpack_bf16(v, x);
}
__device__ __forceinline__ uint4 from_floats(const float* x, float) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                    __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 from_floats(const float* x, __nv_bfloat16) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// a c - b s, rounded once: products and sum with their errors (Dekker's and Knuth's
// error-free forms).  What is packed to 4 bits is decided by which side of a border a value
// lies on, so it must not depend on how a sum was rounded on the way.
__device__ __forceinline__ float turned_exactly(float a, float c, float b, float s) {
  const float p = __fmul_rn(a, c), q = -__fmul_rn(b, s);
  const float ep = fmaf(a, c, -p), eq = fmaf(-b, s, -q);
  const float sum = __fadd_rn(p, q), z = __fsub_rn(sum, p);
  const float es = __fadd_rn(__fsub_rn(p, __fsub_rn(sum, z)), __fsub_rn(q, z));
  const float r = __fadd_rn(sum, __fadd_rn(es, __fadd_rn(ep, eq)));
  return isfinite(sum) ? r : sum;  // the errors of an infinity are NaN
}

// Two pairs turned, E of each, and rounded to bf16 as if exact: a[i] c - b[i] s and
// b[i] c + a[i] s in place.  A product, its error and a sum rounded once (Kahan) are off by less
// than two units; only where that reaches a border between two bf16 is the sum taken exactly.
template <int E, bool NEAR>
__device__ __forceinline__ void turn_to_bf16(float* z, const float* cs, const float* sn) {
  uint32_t near = 0xffffffffu;  // the smallest distance, in units, from 3 below such a border
  float w[2 * E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int i0 = NEAR ? 2 * i : i, i1 = NEAR ? 2 * i + 1 : i + E;
    const float a = z[i0], b = z[i1], p = __fmul_rn(b, sn[i]), q = __fmul_rn(a, sn[i]);
    w[i0] = __fadd_rn(fmaf(a, cs[i], -p), fmaf(-b, sn[i], p));
    w[i1] = __fadd_rn(fmaf(b, cs[i], q), fmaf(a, sn[i], -q));
    near = min(near, (__float_as_uint(w[i0]) & 0xffffu) - 0x7ffdu);
    near = min(near, (__float_as_uint(w[i1]) & 0xffffu) - 0x7ffdu);
  }
  if (near <= 6u) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int i0 = NEAR ? 2 * i : i, i1 = NEAR ? 2 * i + 1 : i + E;
      w[i0] = turned_exactly(z[i0], cs[i], z[i1], sn[i]);
      w[i1] = turned_exactly(z[i1], cs[i], -z[i0], sn[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 2 * E; ++i) z[i] = w[i];
}

// What a block knows of its rows.
struct RopeRows {
  long long at[RP_ROWS];  // of the row in the page of key head 0, -1: nowhere
  int slot[RP_ROWS];
  int pos[RP_ROWS][3];
};

// Rows t0 .. of one sequence.  Bound by memory: every byte of queries, keys and values is
// read once and written once, 16 bytes a load.  The rows' cosines and sines lie in shared
// memory; a thread takes 16 bytes of channels and the 16 bytes of their partners and turns up
// to `each` heads by the same angles.
template <typename T, bool FP4, bool NEAR, bool TURN>
__global__ void __launch_bounds__(RP_THREADS, !TURN ? 6 : FP4 ? RP_CTAS4 : RP_CTAS) k_append_rope(RopeArgs a, int tile) {
  constexpr int E = 16 / sizeof(T);  // elements of 16 bytes
  __shared__ RopeRows rr;
  extern __shared__ __align__(16) float turns[];  // [tile][rot]
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, b = blockIdx.y, t0 = blockIdx.x * tile;
  const int len = __ldcg(a.c.lens + b);
  const NewRows nr = new_rows(a.offsets, b, a.rows, a.T, a.c.status);
  const int nt = min(tile, nr.T - t0);
  if (nt <= 0) return;
  const int first = kv_clamp(a.c, len) - nr.T + t0;
  const int Hkv = a.c.Hkv, d = a.c.d;
  const T* q = reinterpret_cast<const T*>(a.q) + (long long)(nr.off + t0) * a.q_row;
  T* out = reinterpret_cast<T*>(a.out) + (long long)(nr.off + t0) * a.o_row;
  const T *ks, *vs;  // this block's first row
  if (a.v_new) {
    ks = reinterpret_cast<const T*>(a.k_new) + (long long)(nr.off + t0) * a.n_row;
    vs = reinterpret_cast<const T*>(a.v_new) + (long long)(nr.off + t0) * a.n_row;
  } else {
    ks = reinterpret_cast<const T*>(a.k_new) + (2LL * nr.off + t0) * a.n_row;
    vs = reinterpret_cast<const T*>(a.k_new) + (2LL * nr.off + nr.T + t0) * a.n_row;
  }
  // heads that turn: the queries', then the keys'; a thread's are h, h + groups, ..
  constexpr int U = RP_AHEAD;
  const int half = a.rot / 2, C = TURN ? half / E : 0;  // pieces of 2 E channels a head
  const int heads = TURN ? a.H + Hkv : 0;
  const int groups = min(heads, max(ceil_div(heads, RP_HEADS), RP_THREADS / max(nt * C, 1)));
  struct Task {
    int r, c, h;
  } at;
  uint4 v[U][2];
  auto begin = [&](int x) {
    const int y = x / C;
    at.c = x - y * C;
    at.r = y / groups;
    at.h = y - at.r * groups;
  };
  auto load = [&]() {
    const int lo = NEAR ? 2 * E * at.c : E * at.c, hi = NEAR ? lo + E : half + lo;
    const T* qr = q + (long long)at.r * a.q_row;
    const T* kr = ks + (long long)at.r * a.n_row;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = at.h + u * groups;
      if (h >= heads) break;
      const T* src = h < a.H ? qr + h * d : kr + (h - a.H) * d;
      v[u][0] = *reinterpret_cast<const uint4*>(src + lo);
      v[u][1] = *reinterpret_cast<const uint4*>(src + hi);
    }
  };
  int x = tid;
  const int tasks = nt * groups * C;
  if (TURN && x < tasks) {  // on their way while the rows' places and angles are looked up
    begin(x);
    load();
  }
  if (tid < nt) {
    const int j = first + tid;
    if (j < 0) set_status(a.c.status, CACHE_BAD);
    long long o = -1;
    int slot = 0;
    if (j >= 0) {
      const Slot s = kv_slot(a.c, b, j);
      slot = s.slot;
      o = kv_row(a.c, 0, FP4 ? Slot{s.page, 0} : s);
    }
    rr.at[tid] = o;
    rr.slot[tid] = slot;
  }
  if constexpr (TURN) {
    if (tid < nt * 3) {
      const int r = tid / 3, y = tid - r * 3, t = t0 + r;
      int p = first + r;
      if (a.pos)
        p = a.rows3 ? a.pos[3LL * nr.off + (long long)y * nr.T + t] : a.pos[(long long)nr.off + t];
      if (p < 0 || p >= a.max_pos) {
        set_status(a.c.status, CACHE_BAD);
        p = p < 0 ? 0 : a.max_pos - 1;
      }
      rr.pos[r][y] = p;
    }
    __syncthreads();
    const int quads = half / 4;  // of pairs
    auto sect = [&](int p) { return a.rows3 ? (p >= a.sect0) + (p >= a.sect1) : 0; };
    for (int y = tid; y < nt * quads; y += RP_THREADS) {
      const int r = y / quads, p = (y - r * quads) * 4;
      float* to = turns + r * a.rot + p;
      if (sect(p) == sect(p + 3)) {
        const float* f = a.table + (long long)rr.pos[r][sect(p)] * a.rot + p;
        *reinterpret_cast<float4*>(to) = __ldg(reinterpret_cast<const float4*>(f));
        *reinterpret_cast<float4*>(to + half) = __ldg(reinterpret_cast<const float4*>(f + half));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* f = a.table + (long long)rr.pos[r][sect(p + i)] * a.rot + p + i;
          to[i] = __ldg(f);
          to[half + i] = __ldg(f + half);
        }
      }
    }
  }
  __syncthreads();
  while (TURN && x < tasks) {
    const int r = at.r, lo = NEAR ? 2 * E * at.c : E * at.c, hi = NEAR ? lo + E : half + lo;
    float cs[E], sn[E];
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const float* f = turns + r * a.rot + E * at.c + i;
      *reinterpret_cast<float4*>(cs + i) = *reinterpret_cast<const float4*>(f);
      *reinterpret_cast<float4*>(sn + i) = *reinterpret_cast<const float4*>(f + half);
    }
    T* orow = out + (long long)r * a.o_row;
    while (true) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = at.h + u * groups;
        if (h >= heads) break;
        float z[2 * E];
        to_floats(v[u][0], z, T());
        to_floats(v[u][1], z + E, T());
        const bool key = h >= a.H;
        if (FP4 && key) {
          turn_to_bf16<E, NEAR>(z, cs, sn);
          const uint4 w0 = from_floats(z, T()), w1 = from_floats(z + E, T());
          // neighbours hold the two halves of the blocks (of pairs of neighbours one thread a
          // whole one): C is even, so both are here
          char* part = a.c.k + rr.at[r] + (h - a.H) * a.c.head_stride;
          char* codes = part + (long long)rr.slot[r] * (d / 2);
          char* scales = part + fp4_scale_at(a.c, rr.slot[r]);
          if constexpr (NEAR) {
            uint32_t s;
            const uint2 w = fp4_block(w0, w1, &s);
            if (rr.at[r] >= 0) {
              *reinterpret_cast<uint2*>(codes + lo / 2) = w;
              scales[lo / 16] = (char)s;
            }
          } else {
            // both blocks' largest magnitudes in one word
            const uint32_t mine = fp4_top(w0) | fp4_top(w1) << 16;
            const uint32_t top = max_u16x2(mine, __shfl_xor_sync(3u << (tid & 30), mine, 1));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const Fp4Scale f(i ? top >> 16 : top & 0xffffu);
              const uint32_t s = f.byte, w = f.codes(i ? w1 : w0);
              const int to = i ? hi : lo;
              if (rr.at[r] >= 0) {
                *reinterpret_cast<uint32_t*>(codes + to / 2) = w;
                if (!(tid & 1)) scales[to / 16] = (char)s;
              }
            }
          }
          continue;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
          float &p0 = z[NEAR ? 2 * i : i], &p1 = z[NEAR ? 2 * i + 1 : i + E];
          const float x0 = p0, x1 = p1;
          p0 = fmaf(x0, cs[i], -x1 * sn[i]);
          p1 = fmaf(x1, cs[i], x0 * sn[i]);
        }
        T* dst = orow + h * d;
        if (key) {
          if (rr.at[r] < 0) continue;
          dst = reinterpret_cast<T*>(a.c.k) + rr.at[r] + (h - a.H) * a.c.head_stride;
        }
        *reinterpret_cast<uint4*>(dst + lo) = from_floats(z, T());
        *reinterpret_cast<uint4*>(dst + hi) = from_floats(z + E, T());
      }
      if ((at.h += U * groups) >= heads) break;
      load();
    }
    if ((x += RP_THREADS) < tasks) {
      begin(x);
      load();
    }
  }
  // ---- channels that do not turn: the queries', keys' and all of the values' ----------------
  {
    const int rest = TURN ? (d - a.rot) / E : 0;
    const int still = (FP4 ? a.H : a.H + Hkv) * rest;
    const int per = still + (FP4 ? 0 : Hkv * (d / E));
    for (int x = tid; x < nt * per; x += RP_THREADS) {
      const int r = x / per;
      int y = x - r * per;
      const T* src;
      T* dst;
      if (y < still) {
        const int h = y / rest;
        y = a.rot + (y - h * rest) * E;
        if (h < a.H) {
          src = q + (long long)r * a.q_row + h * d + y;
          dst = out + (long long)r * a.o_row + h * d + y;
          if (src == dst) continue;
        } else {
          if (rr.at[r] < 0) continue;
          src = ks + (long long)r * a.n_row + (h - a.H) * d + y;
          dst = reinterpret_cast<T*>(a.c.k) + rr.at[r] + (h - a.H) * a.c.head_stride + y;
        }
      } else {
        if (rr.at[r] < 0) continue;
        y -= still;
        const int h = y / (d / E);
        y = (y - h * (d / E)) * E;
        src = vs + (long long)r * a.n_row + h * d + y;
        dst = reinterpret_cast<T*>(a.c.v) + rr.at[r] + h * a.c.head_stride + y;
      }
      *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    }
  }
  // ---- 4 bits: the values' blocks, and the keys' that do not turn ---------------------------
  if constexpr (FP4) {
    // a head's rows together: a warp's scales make whole sectors
    const int skip = TURN ? a.rot / 16 : 0, whole = d / 16, rest = whole - skip;
    const int still = Hkv * rest * nt, all = still + Hkv * whole * nt;
    constexpr int U = RP_BLOCKS;
    for (int x0 = tid; x0 < all; x0 += RP_THREADS * U) {
      uint4 v[U][2];
      char* part[U];
      int blk[U], slot[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int x = x0 + u * RP_THREADS;
        part[u] = nullptr;
        if (x >= all) continue;
        const bool key = x < still;
        if (!key) x -= still;
        const int n = key ? rest : whole, y = x / n, h = y / nt, r = y - h * nt;
        if (rr.at[r] < 0) continue;
        blk[u] = x - y * n + (key ? skip : 0);
        slot[u] = rr.slot[r];
        const uint4* src = reinterpret_cast<const uint4*>(
            (key ? ks : vs) + (long long)r * a.n_row + h * d + blk[u] * 16);
        v[u][0] = __ldcs(src);
        v[u][1] = __ldcs(src + 1);
        part[u] = (key ? a.c.k : a.c.v) + rr.at[r] + h * a.c.head_stride;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!part[u]) continue;
        uint32_t s;
        const uint2 w = fp4_block(v[u][0], v[u][1], &s);
        *reinterpret_cast<uint2*>(part[u] + (long long)slot[u] * (d / 2) + blk[u] * 8) = w;
        part[u][fp4_scale_at(a.c, slot[u]) + blk[u]] = (char)s;
      }
    }
  }
}

// The last rows of a sequence out of their pages, 16 bytes a lane.  Bound by memory.
__global__ void __launch_bounds__(RP_THREADS) k_cache_read(KV c, char* __restrict__ k_out,
                                                           char* __restrict__ v_out,
                                                           const int32_t* __restrict__ offsets,
                                                           int rows, int T, int esize, int tile) {
  __shared__ long long at[RP_ROWS];
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.y, t0 = blockIdx.x * tile;
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
  __syncthreads();
  const int hc = c.d * esize / 16, rc = hc * c.Hkv;
  const long long to = (long long)(nr.off + t0) * rc;
  constexpr int U = 4;
  for (int x0 = threadIdx.x; x0 < nt * rc; x0 += RP_THREADS * U) {
    uint4 w[U][2];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * RP_THREADS, r = x / rc;
      there[u] = x < nt * rc && at[r] >= 0;
      if (!there[u]) continue;
      const int y = x - r * rc, h = y / hc, z = y - h * hc;
      const long long o = (at[r] + h * c.head_stride) * esize + z * 16;
      w[u][0] = *reinterpret_cast<const uint4*>(c.k + o);
      w[u][1] = *reinterpret_cast<const uint4*>(c.v + o);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!there[u]) continue;
      const long long x = to + x0 + u * RP_THREADS;
      reinterpret_cast<uint4*>(k_out)[x] = w[u][0];
      reinterpret_cast<uint4*>(v_out)[x] = w[u][1];
    }
  }
}

// The same of 4 bits, unpacked: one key head, a block of 16 channels a lane, the loads of four
// before the first is stored.
template <int D>
__global__ void __launch_bounds__(RP_THREADS) k_cache_read4(KV c, char* __restrict__ k_out,
                                                            char* __restrict__ v_out,
                                                            const int32_t* __restrict__ offsets,
                                                            int rows, int T, int tile, int wide) {
  constexpr int HC = D / 16, U = 4;
  __shared__ long long at[RP_ROWS];
  __shared__ int slots[RP_ROWS];
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.z, h = blockIdx.y, t0 = blockIdx.x * tile;
  const int len = __ldcg(c.lens + b);
  const NewRows nr = new_rows(offsets, b, rows, T, c.status);
  const int nt = min(tile, nr.T - t0);
  if (nt <= 0) return;
  const int first = kv_clamp(c, len) - nr.T + t0;
  if ((int)threadIdx.x < nt) {
    const int j = first + (int)threadIdx.x;
    if (j < 0) set_status(c.status, CACHE_BAD);
    long long o = -1;
    int slot = 0;
    if (j >= 0) {
      const Slot s = kv_slot(c, b, j);
      slot = s.slot;
      o = kv_row(c, h, Slot{s.page, 0});
    }
    at[threadIdx.x] = o;
    slots[threadIdx.x] = slot;
  }
  __syncthreads();
  const long long to = ((long long)(nr.off + t0) * c.Hkv + h) * D, row = (long long)c.Hkv * D;
  const int items = 2 * nt * HC;
  for (int x0 = threadIdx.x; x0 < items; x0 += U * RP_THREADS) {
    uint2 w[U];
    uint32_t s[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * RP_THREADS, r = x / (2 * HC), v = x / HC & 1, z = x % HC;
      there[u] = x < items && at[r] >= 0;
      if (!there[u]) continue;
      const char* part = (v ? c.v : c.k) + at[r];
      w[u] = *reinterpret_cast<const uint2*>(part + (long long)slots[r] * (D / 2) + z * 8);
      s[u] = (uint8_t)part[fp4_scale_at(c, slots[r]) + z];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!there[u]) continue;
      const int x = x0 + u * RP_THREADS, r = x / (2 * HC), v = x / HC & 1, z = x % HC;
      const uint32_t s2 = fp4_scale2(s[u]);
      const uint4 lo = fp4_bf16(w[u].x, s2), hi = fp4_bf16(w[u].y, s2);
      char* p = (v ? v_out : k_out) + (to + r * row + z * 16) * 2;
      if (wide) {
        store32(p, lo, hi);
      } else {
        reinterpret_cast<uint4*>(p)[0] = lo;
        reinterpret_cast<uint4*>(p)[1] = hi;
      }
    }
  }
}

// Rows of a block: fewer where the blocks would not fill the GPU twice.
int rows_of_block(int T, int B) {
  int tile = RP_ROWS;
  const long long fill = (long long)RP_FILL * sm_count();
  while (tile > 1 && (long long)ceil_div(T, tile) * B < fill) tile /= 2;
  return tile;
}
}  // namespace

cudaError_t launch_append_rope(const RopeArgs& a, int dtype, cudaStream_t st) {
  const int tile = rows_of_block(a.T, a.c.B);
  auto go = [&](auto kernel) {
    const size_t smem = a.table ? (size_t)tile * a.rot * sizeof(float) : 0;
    const cudaError_t e = set_smem_limit((const void*)kernel, smem);
    if (e != cudaSuccess) return e;
    return launch_k(kernel, dim3(ceil_div(a.T, tile), a.c.B), dim3(RP_THREADS), smem, st, 1, a,
                    tile);
  };
  typedef __nv_bfloat16 bf16;
  if (!a.table) return go(k_append_rope<bf16, true, false, false>);  // packed alone
  if (dtype == GMC_FP4)
    return a.near ? go(k_append_rope<bf16, true, true, true>)
                  : go(k_append_rope<bf16, true, false, true>);
  if (dtype == GMC_BF16)
    return a.near ? go(k_append_rope<bf16, false, true, true>)
                  : go(k_append_rope<bf16, false, false, true>);
  return a.near ? go(k_append_rope<float, false, true, true>)
                : go(k_append_rope<float, false, false, true>);
}

cudaError_t launch_cache_read(const KV& c, int dtype, char* k_out, char* v_out,
                              const int32_t* offsets, int rows, int T, cudaStream_t st) {
  if (dtype == GMC_FP4) {
    const int tile = rows_of_block(T, c.B * c.Hkv);
    auto kernel = c.d == 64 ? k_cache_read4<64> : c.d == 128 ? k_cache_read4<128> : k_cache_read4<256>;
    return launch_k(kernel, dim3(ceil_div(T, tile), c.Hkv, c.B), dim3(RP_THREADS), 0, st, 1, c,
                    k_out, v_out, offsets, rows, T, tile,
                    (int)(((uintptr_t)k_out | (uintptr_t)v_out) % 32 == 0));
  }
  const int tile = rows_of_block(T, c.B);
  return launch_k(k_cache_read, dim3(ceil_div(T, tile), c.B), dim3(RP_THREADS), 0, st, 1, c, k_out,
                  v_out, offsets, rows, T, dtype == GMC_F32 ? 4 : 2, tile);
}

}  // namespace gmc
