// Attention of new tokens over a cache held in 4 bits: the seen rows of every sequence are
// unpacked to bf16, which holds their values exactly, into pages of the workspace, and
// gmc_attend's kernels for bf16 run on these.
//
// The unpacking is bound by memory: 72 bytes a row of 128 channels read, 256 written.
#include <math.h>

#include <algorithm>

#include "cache.cuh"
#include "fp4.cuh"

namespace gmc {

namespace {
constexpr int UP_PAGE = 128;  // slots of a page of the workspace: whole turns of k_attend_tc
constexpr int UP_THREADS = 256, UP_ROWS = 32;

// UP_ROWS rows of one page and head; rows that no query sees become zeros, and pages without a
// seen row are left alone.  A lane takes a block of 16 channels, the loads of four blocks before
// the first is stored.
template <int D>
__global__ void __launch_bounds__(UP_THREADS) k_unpack(AttnArgs a, KV to) {
  constexpr int HC = D / 16, ITEMS = 2 * UP_ROWS * HC;  // keys' blocks, then the values'
  __shared__ long long at[UP_ROWS];
  __shared__ int slots[UP_ROWS];
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.z, h = blockIdx.y, j0 = blockIdx.x * UP_ROWS, page = j0 / UP_PAGE;
  const int n = kv_len(a.c, b);
  const NewRows nr = new_rows(a.q_offsets, b, a.rows, a.T, a.c.status);
  if (h == 0 && j0 % UP_PAGE == 0 && threadIdx.x == 0)
    const_cast<int32_t*>(to.table)[(long long)b * to.max_pages + page] = b * to.max_pages + page;
  if (nr.T == 0) return;
  const Seen seen = seen_keys(n - nr.T, n - 1, a.window, a.sinks);
  auto sees_any = [&](int lo, int hi) {  // of places lo .. hi - 1
    return lo < seen.a || (lo < seen.b1 && hi > seen.b0);
  };
  if (!sees_any(page * UP_PAGE, page * UP_PAGE + UP_PAGE)) return;
  if ((int)threadIdx.x < UP_ROWS) {
    const int j = j0 + (int)threadIdx.x;
    long long o = -1;
    int slot = 0;
    if (j < n && sees_any(j, j + 1)) {
      const Slot s = kv_slot(a.c, b, j);
      slot = s.slot;
      o = kv_row(a.c, h, Slot{s.page, 0});
    }
    at[threadIdx.x] = o;
    slots[threadIdx.x] = slot;
  }
  __syncthreads();
  const long long base = (long long)(b * to.max_pages + page) * to.page_stride +
                         h * to.head_stride + (long long)(j0 % UP_PAGE) * D;
  constexpr int U = ITEMS / UP_THREADS < 4 ? ITEMS / UP_THREADS : 4;
#pragma unroll
  for (int x0 = 0; x0 < ITEMS; x0 += U * UP_THREADS) {
    uint2 c[U];
    uint32_t s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * UP_THREADS + threadIdx.x, v = x / (UP_ROWS * HC),
                y = x % (UP_ROWS * HC), r = y / HC, z = y % HC;
      c[u] = make_uint2(0u, 0u);
      s[u] = 0;
      if (at[r] >= 0) {
        const char* part = (v ? a.c.v : a.c.k) + at[r];
        c[u] = *reinterpret_cast<const uint2*>(part + (long long)slots[r] * (D / 2) + z * 8);
        s[u] = (uint8_t)part[fp4_scale_at(a.c, slots[r]) + z];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + u * UP_THREADS + threadIdx.x, v = x / (UP_ROWS * HC),
                y = x % (UP_ROWS * HC);
      const uint32_t s2 = fp4_scale2(s[u]);
      store32((v ? to.v : to.k) + (base + y * 16) * 2, fp4_bf16(c[u].x, s2),
              fp4_bf16(c[u].y, s2));
    }
  }
}

// The cache as bf16, in the workspace from `at` on.
struct Unpacked {
  KV c;
  size_t table, pool, all;  // bytes of each part
};
Unpacked unpacked(const KV& c) {
  Unpacked u;
  u.c = c;
  u.c.ps = UP_PAGE;
  u.c.max_pages = ceil_div(c.cap, UP_PAGE);
  u.c.num_pages = c.B * u.c.max_pages;
  u.c.slot_stride = c.d;
  u.c.head_stride = (long long)UP_PAGE * c.d;
  u.c.page_stride = c.Hkv * u.c.head_stride;
  u.table = ((size_t)u.c.num_pages * 4 + 255) & ~(size_t)255;
  u.pool = (size_t)u.c.num_pages * u.c.page_stride * 2;
  u.all = u.table + 2 * u.pool;
  return u;
}
}  // namespace

namespace {
// Whether the attending kernel reads the codes itself (k_attend_fp4_tc.cu): where it takes less
// than unpacking and attending, in us by these two sums.  28 query and 4 key heads of 128, us so
// and so: 8 x 16,004 keys and 16 tokens (one tile) 57 and 114, 32 tokens 103 and 132, 48 (three
// tiles, a second wave) 189 and 149; 8 x 2,000 and 64 tokens 31 and 43, 96 tokens 59 and 44; one
// sequence of 16,004 and 64 tokens 33 and 40, 128 tokens 57 and 50; of 2,000 and 256 tokens (15
// tiles) 24 and 27; 32 x 500 and 18 tokens 14 and 23, 64 tokens 50 and 38.
bool direct(const KV& c, int G, int T) {
  if (c.d > 128) return false;
  const double sms = sm_count(), pairs = (double)c.B * c.Hkv, tiles = pairs * ceil_div(T, 128 / G);
  // a turn of 64 keys, and what a CTA has besides; joining as in cheapest_parts
  const int s = attend_direct_splits(c, G, T);
  double codes = ceil(tiles * s / sms) * (5.5 + 0.76 * ceil_div(ceil_div(c.cap, 64), s));
  if (s > 1) codes += 2.5 + 8. * s * c.B * T * G * c.Hkv * c.d / 5e6;
  // 2.56 bytes a value read and written, 2 read again, or a turn of 128 keys; joining
  const double values = pairs * c.cap * c.d * 2;
  double rows = 9 + values * 2.5625 / 6e6 +
                fmax(values * 2 / 6e6, tiles * ceil_div(c.cap, 128) / sms) +
                5 * ceil(tiles / (2 * sms));
  if (tiles < sms) rows += 5;
  return codes < rows;
}
// Parts of the key axis of the unpacked rows, whose attention need not add up as bf16's does: also
// where that fills a last wave (2,048 tokens on 16,004 keys: 392 us in one part, 364 in two).
int parts(const KV& c, int G, int T, long long most) {
  if (!attend_tc_takes(c, GMC_BF16, G) || attend_tc_splits(c, G, T) != 1) return 0;
  return attend_tc_wave_parts(c, G, T, most);
}
}  // namespace

size_t attend_fp4_workspace(const KV& c, int H, int T) {
  if (direct(c, H / c.Hkv, T)) {
    const int s = attend_direct_splits(c, H / c.Hkv, T);
    const size_t rows = (size_t)c.B * T * H * s;
    return s == 1 ? 256 : 256 + ((rows * 8 + 255) & ~(size_t)255) + rows * c.d * 4;
  }
  const Unpacked u = unpacked(c);
  return u.all + attend_workspace(u.c, GMC_BF16, H, T, parts(u.c, H / c.Hkv, T, c.cap));
}

cudaError_t launch_attend_fp4(AttnArgs a, void* ws, cudaStream_t st, int* launches) {
  if (direct(a.c, a.G, a.T)) {
    a.splits = attend_direct_splits(a.c, a.G, a.T);
    if (a.splits > 1) {
      const size_t rows = (size_t)a.c.B * a.T * a.H * a.splits;
      a.ml = reinterpret_cast<float2*>(ws);
      a.part = reinterpret_cast<float*>((char*)ws + ((rows * 8 + 255) & ~(size_t)255));
    }
    cudaError_t e = launch_attend_direct(a, st);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (a.splits > 1 && (e = launch_attend_join(a, GMC_BF16, st)) == cudaSuccess) ++*launches;
    return e;
  }
  Unpacked u = unpacked(a.c);
  u.c.table = reinterpret_cast<int32_t*>(ws);
  u.c.k = (char*)ws + u.table;
  u.c.v = u.c.k + u.pool;
  auto unpack = a.c.d == 64 ? k_unpack<64> : a.c.d == 128 ? k_unpack<128> : k_unpack<256>;
  const cudaError_t e =
      launch_k(unpack, dim3(u.c.max_pages * (UP_PAGE / UP_ROWS), a.c.Hkv, a.c.B),
               dim3(UP_THREADS), 0, st, 1, a, u.c);
  if (e != cudaSuccess) return e;
  ++*launches;
  a.c = u.c;
  int s = parts(a.c, a.G, a.T, a.c.cap);  // what the workspace has room for
  if (s > 1 && a.window > 0) {
    const long long most = (long long)a.window + a.sinks + 128;
    s = std::min(s, parts(a.c, a.G, a.T, std::min<long long>(a.c.cap, most)));
  }
  return launch_attend(a, GMC_BF16, (char*)ws + u.all, st, launches, s);
}

}  // namespace gmc
