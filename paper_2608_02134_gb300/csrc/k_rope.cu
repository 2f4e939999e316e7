// New rows written to their pages with the position rotation applied on the way (and packed
// to 4 bits where the cache holds those), and rows read back out of their pages.
#include "cache.cuh"
#include "fp4.cuh"

namespace gmc {

namespace {
constexpr int RP_THREADS = 256, RP_ROWS = 64;
constexpr int RP_HEADS = 8;  // heads a thread turns by the same angles

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

// What a block knows of its rows.
struct RopeRows {
  long long at[RP_ROWS];  // of the row in the page of key head 0, -1: nowhere
  int slot[RP_ROWS];
  int pos[RP_ROWS][3];
};

// cos and sin of E pairs from p0 on.
template <int E>
__device__ __forceinline__ void angles(const RopeArgs& a, const int* pos, int p0, float* cs,
                                       float* sn) {
  const int half = a.rot / 2;
#pragma unroll
  for (int i = 0; i < E; i += 4) {
    const int p = p0 + i;
    auto sect = [&](int x) { return a.rows3 ? (x >= a.sect0) + (x >= a.sect1) : 0; };
    if (sect(p) == sect(p + 3)) {
      const float* f = a.table + (long long)pos[sect(p)] * a.rot + p;
      const float4 c = __ldg(reinterpret_cast<const float4*>(f));
      const float4 s = __ldg(reinterpret_cast<const float4*>(f + half));
      cs[i] = c.x, cs[i + 1] = c.y, cs[i + 2] = c.z, cs[i + 3] = c.w;
      sn[i] = s.x, sn[i + 1] = s.y, sn[i + 2] = s.z, sn[i + 3] = s.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* f = a.table + (long long)pos[sect(p + j)] * a.rot + p + j;
        cs[i + j] = __ldg(f);
        sn[i + j] = __ldg(f + half);
      }
    }
  }
}

// Rows t0 .. of one sequence.  Bound by memory: every byte of queries, keys and values is
// read once and written once, 16 bytes a load.  A thread takes 16 bytes of channels and the
// 16 bytes of their partners, loads their angles once and turns up to 8 heads by them.
template <typename T, bool FP4, bool NEAR>
__global__ void __launch_bounds__(RP_THREADS) k_append_rope(RopeArgs a, int tile) {
  constexpr int E = 16 / sizeof(T);  // elements of 16 bytes
  __shared__ RopeRows rr;
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, b = blockIdx.y, t0 = blockIdx.x * tile;
  const int len = __ldcg(a.c.lens + b);
  const NewRows nr = new_rows(a.offsets, b, a.rows, a.T, a.c.status);
  const int nt = min(tile, nr.T - t0);
  if (nt <= 0) return;
  const int first = kv_clamp(a.c, len) - nr.T + t0;
  if (tid < nt) {
    const int j = first + tid;
    if (j < 0) set_status(a.c.status, CACHE_BAD);
    long long at = -1;
    int slot = 0;
    if (j >= 0) {
      const Slot s = kv_slot(a.c, b, j);
      slot = s.slot;
      at = kv_row(a.c, 0, FP4 ? Slot{s.page, 0} : s);
    }
    rr.at[tid] = at;
    rr.slot[tid] = slot;
  }
  if (a.table && tid < nt * 3) {
    const int r = tid / 3, x = tid - r * 3, t = t0 + r;
    int p = first + r;
    if (a.pos)
      p = a.rows3 ? a.pos[3LL * nr.off + (long long)x * nr.T + t] : a.pos[(long long)nr.off + t];
    if (p < 0 || p >= a.max_pos) {
      set_status(a.c.status, CACHE_BAD);
      p = p < 0 ? 0 : a.max_pos - 1;
    }
    rr.pos[r][x] = p;
  }
  __syncthreads();
  const int Hkv = a.c.Hkv, d = a.c.d;
  const T* q = reinterpret_cast<const T*>(a.q);
  T* out = reinterpret_cast<T*>(a.out);
  const T *ks, *vs;  // this block's first row
  if (a.v_new) {
    ks = reinterpret_cast<const T*>(a.k_new) + (long long)(nr.off + t0) * a.n_row;
    vs = reinterpret_cast<const T*>(a.v_new) + (long long)(nr.off + t0) * a.n_row;
  } else {
    ks = reinterpret_cast<const T*>(a.k_new) + (2LL * nr.off + t0) * a.n_row;
    vs = reinterpret_cast<const T*>(a.k_new) + (2LL * nr.off + nr.T + t0) * a.n_row;
  }
  // ---- heads that turn: the queries', then (but for 4 bits) the keys' ----------------------
  const int C = a.table ? a.rot / (2 * E) : 0;  // pieces of 2 E channels a head
  const int heads = FP4 ? a.H : a.H + Hkv, groups = ceil_div(heads, RP_HEADS);
  for (int x = tid; x < nt * groups * C; x += RP_THREADS) {
    const int y = x / C, c = x - y * C, r = y / groups, h0 = y - r * groups;
    float cs[E], sn[E];
    angles<E>(a, rr.pos[r], c * E, cs, sn);
    const int lo = NEAR ? 2 * E * c : E * c, hi = NEAR ? lo + E : a.rot / 2 + lo;
    const T* qr = q + (long long)(nr.off + t0 + r) * a.q_row;
    T* orow = out + (long long)(nr.off + t0 + r) * a.o_row;
    const T* kr = ks + (long long)r * a.n_row;
    T* kp = reinterpret_cast<T*>(a.c.k) + rr.at[r];
    constexpr int U = 4;
    for (int h1 = h0; h1 < heads; h1 += U * groups) {
      uint4 v[U][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h1 + u * groups;
        if (h >= heads) break;
        const T* src = h < a.H ? qr + h * d : kr + (h - a.H) * d;
        v[u][0] = *reinterpret_cast<const uint4*>(src + lo);
        v[u][1] = *reinterpret_cast<const uint4*>(src + hi);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h1 + u * groups;
        if (h >= heads) break;
        float p[2 * E], z[2 * E];
        to_floats(v[u][0], p, T());
        to_floats(v[u][1], p + E, T());
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const int i0 = NEAR ? 2 * i : i, i1 = NEAR ? 2 * i + 1 : i + E;
          z[i0] = fmaf(p[i0], cs[i], -p[i1] * sn[i]);
          z[i1] = fmaf(p[i1], cs[i], p[i0] * sn[i]);
        }
        T* dst = orow + h * d;
        if (!FP4 && h >= a.H) {
          if (rr.at[r] < 0) continue;
          dst = kp + (h - a.H) * a.c.head_stride;
        }
        *reinterpret_cast<uint4*>(dst + lo) = from_floats(z, T());
        *reinterpret_cast<uint4*>(dst + hi) = from_floats(z + E, T());
      }
    }
  }
  // ---- channels that do not turn: the queries', keys' and all of the values' ----------------
  {
    const int rest = C ? (d - a.rot) / E : d / E, skip = C ? a.rot : 0;
    const int still = heads * rest;
    const int per = still + (FP4 ? 0 : Hkv * (d / E));
    for (int x = tid; x < nt * per; x += RP_THREADS) {
      const int r = x / per;
      int y = x - r * per;
      const T* src;
      T* dst;
      if (y < still) {
        const int h = y / rest;
        y = skip + (y - h * rest) * E;
        if (h < a.H) {
          src = q + (long long)(nr.off + t0 + r) * a.q_row + h * d + y;
          dst = out + (long long)(nr.off + t0 + r) * a.o_row + h * d + y;
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
  // ---- 4 bits: keys' and values' blocks -----------------------------------------------------
  if constexpr (FP4) {
    auto put = [&](char* pool, int r, int h, int blk, const float* v) {
      char* part = pool + rr.at[r] + h * a.c.head_stride;
      uint32_t s;
      *reinterpret_cast<uint2*>(part + (long long)rr.slot[r] * (d / 2) + blk * 8) =
          fp4_block(v, &s);
      part[fp4_scale_at(a.c, rr.slot[r]) + blk] = (char)s;
    };
    auto get = [&](const T* row, int blk, float* v) {
      const uint4* src = reinterpret_cast<const uint4*>(row + blk * 16);
      const uint4 x = src[0], y = src[1];
      to_floats(x, v, T());
      to_floats(y, v + 8, T());
    };
    // two blocks of partners a thread
    const int pairs = a.table ? a.rot / 32 : 0;
    for (int x = tid; x < nt * Hkv * pairs; x += RP_THREADS) {
      const int y = x / pairs, c = x - y * pairs, r = y / Hkv, h = y - r * Hkv;
      if (rr.at[r] < 0) continue;
      const T* row = ks + (long long)r * a.n_row + h * d;
      const int lo = NEAR ? 2 * c : c, hi = NEAR ? lo + 1 : lo + a.rot / 32;
      float v[32], z[32], cs[16], sn[16];
      get(row, lo, v);
      get(row, hi, v + 16);
      angles<16>(a, rr.pos[r], c * 16, cs, sn);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int i0 = NEAR ? 2 * i : i, i1 = NEAR ? 2 * i + 1 : i + 16;
        z[i0] = __bfloat162float(
            __float2bfloat16_rn(turned_exactly(v[i0], cs[i], v[i1], sn[i])));
        z[i1] = __bfloat162float(
            __float2bfloat16_rn(turned_exactly(v[i1], cs[i], -v[i0], sn[i])));
      }
      put(a.c.k, r, h, lo, z);
      put(a.c.k, r, h, hi, z + 16);
    }
    const int whole = d / 16, still = whole - 2 * pairs, per = Hkv * (still + whole);
    for (int x = tid; x < nt * per; x += RP_THREADS) {
      const int r = x / per;
      int y = x - r * per;
      if (rr.at[r] < 0) continue;
      float v[16];
      if (y < Hkv * still) {
        const int h = y / still, blk = 2 * pairs + y - h * still;
        get(ks + (long long)r * a.n_row + h * d, blk, v);
        put(a.c.k, r, h, blk, v);
      } else {
        y -= Hkv * still;
        const int h = y / whole, blk = y - h * whole;
        get(vs + (long long)r * a.n_row + h * d, blk, v);
        put(a.c.v, r, h, blk, v);
      }
    }
  }
}

// The last rows of a sequence out of their pages, 16 bytes (of 4 bits a block of 16) a
// thread.  Bound by memory.
template <bool FP4>
__global__ void __launch_bounds__(RP_THREADS) k_cache_read(KV c, char* __restrict__ k_out,
                                                           char* __restrict__ v_out,
                                                           const int32_t* __restrict__ offsets,
                                                           int rows, int T, int esize, int tile) {
  __shared__ long long at[RP_ROWS];
  __shared__ int slots[RP_ROWS];
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
    long long o = -1;
    int slot = 0;
    if (j >= 0) {
      const Slot s = kv_slot(c, b, j);
      slot = s.slot;
      o = kv_row(c, 0, FP4 ? Slot{s.page, 0} : s);
    }
    at[threadIdx.x] = o;
    slots[threadIdx.x] = slot;
  }
  __syncthreads();
  const int hc = FP4 ? c.d / 16 : c.d * esize / 16, rc = hc * c.Hkv;
  const long long to = (long long)(nr.off + t0) * rc;
  constexpr int U = 4;
  for (int x0 = threadIdx.x; x0 < nt * rc; x0 += RP_THREADS * U) {
    uint4 w[U][2];
    uint32_t s[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * RP_THREADS;
      if (x >= nt * rc) break;
      const int r = x / rc, y = x - r * rc, h = y / hc, z = y - h * hc;
      if (at[r] < 0) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const char* pool = i ? c.v : c.k;
        if constexpr (FP4) {
          const char* part = pool + at[r] + h * c.head_stride;
          const uint2 v =
              *reinterpret_cast<const uint2*>(part + (long long)slots[r] * (c.d / 2) + z * 8);
          w[u][i] = make_uint4(v.x, v.y, 0u, 0u);
          s[u][i] = (uint8_t)part[fp4_scale_at(c, slots[r]) + z];
        } else {
          w[u][i] = *reinterpret_cast<const uint4*>(
              pool + (at[r] + h * c.head_stride) * esize + z * 16);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * RP_THREADS;
      if (x >= nt * rc) break;
      if (at[x / rc] < 0) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint4* dst = reinterpret_cast<uint4*>(i ? v_out : k_out);
        if constexpr (FP4) {
          const uint32_t s2 = fp4_scale2(s[u][i]);
          dst[(to + x) * 2] = fp4_bf16(w[u][i].x, s2);
          dst[(to + x) * 2 + 1] = fp4_bf16(w[u][i].y, s2);
        } else {
          dst[to + x] = w[u][i];
        }
      }
    }
  }
}

// Rows of a block: fewer where the blocks would not fill the GPU twice.
int rows_of_block(int T, int B) {
  int tile = RP_ROWS;
  const long long fill = 2LL * sm_count();
  while (tile > 1 && (long long)ceil_div(T, tile) * B < fill) tile /= 2;
  return tile;
}
}  // namespace

cudaError_t launch_append_rope(const RopeArgs& a, int dtype, cudaStream_t st) {
  const int tile = rows_of_block(a.T, a.c.B);
  auto go = [&](auto kernel) {
    return launch_k(kernel, dim3(ceil_div(a.T, tile), a.c.B), dim3(RP_THREADS), 0, st, 1, a, tile);
  };
  if (dtype == GMC_FP4)
    return a.near ? go(k_append_rope<__nv_bfloat16, true, true>)
                  : go(k_append_rope<__nv_bfloat16, true, false>);
  if (dtype == GMC_BF16)
    return a.near ? go(k_append_rope<__nv_bfloat16, false, true>)
                  : go(k_append_rope<__nv_bfloat16, false, false>);
  return a.near ? go(k_append_rope<float, false, true>) : go(k_append_rope<float, false, false>);
}

cudaError_t launch_cache_read(const KV& c, int dtype, char* k_out, char* v_out,
                              const int32_t* offsets, int rows, int T, cudaStream_t st) {
  const int esize = dtype == GMC_F32 ? 4 : 2, tile = rows_of_block(T, c.B);
  const dim3 grid(ceil_div(T, tile), c.B), block(RP_THREADS);
  return dtype == GMC_FP4
             ? launch_k(k_cache_read<true>, grid, block, 0, st, 1, c, k_out, v_out, offsets, rows,
                        T, esize, tile)
             : launch_k(k_cache_read<false>, grid, block, 0, st, 1, c, k_out, v_out, offsets, rows,
                        T, esize, tile);
}

}  // namespace gmc
