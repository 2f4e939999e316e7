// Attention of new tokens over a cache held in 4 bits: the seen rows of every sequence are
// unpacked to bf16, which holds their values exactly, into pages of the workspace, and
// gmc_attend's kernels for bf16 run on these.
//
// The unpacking is bound by memory: 72 bytes a row of 128 channels read, 256 written.
#include <algorithm>

#include "cache.cuh"
#include "fp4.cuh"

namespace gmc {

namespace {
constexpr int UP_PAGE = 128;  // slots of a page of the workspace: whole turns of k_attend_tc
constexpr int UP_THREADS = 256, UP_ROWS = 32;

// UP_ROWS rows of one page; rows that no query sees become zeros, and pages without a seen
// row are left alone.
__global__ void __launch_bounds__(UP_THREADS) k_unpack(AttnArgs a, KV to) {
  __shared__ long long at[UP_ROWS];
  __shared__ int slots[UP_ROWS];
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.y, j0 = blockIdx.x * UP_ROWS, page = j0 / UP_PAGE;
  const int n = kv_len(a.c, b);
  const NewRows nr = new_rows(a.q_offsets, b, a.rows, a.T, a.c.status);
  if (j0 % UP_PAGE == 0 && threadIdx.x == 0)
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
      o = kv_row(a.c, 0, Slot{s.page, 0});
    }
    at[threadIdx.x] = o;
    slots[threadIdx.x] = slot;
  }
  __syncthreads();
  const int hc = a.c.d / 16, rc = UP_ROWS * hc;
  const long long base = (long long)(b * to.max_pages + page) * to.page_stride +
                         (long long)(j0 % UP_PAGE) * to.slot_stride;
  for (int x = threadIdx.x; x < rc * a.c.Hkv; x += UP_THREADS) {
    const int h = x / rc, y = x - h * rc, r = y / hc, z = y - r * hc;
    const long long dst = base + h * to.head_stride + r * to.slot_stride + z * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
      if (at[r] >= 0) {
        const char* part = (i ? a.c.v : a.c.k) + at[r] + h * a.c.head_stride;
        const uint2 v =
            *reinterpret_cast<const uint2*>(part + (long long)slots[r] * (a.c.d / 2) + z * 8);
        const uint32_t s2 = fp4_scale2((uint8_t)part[fp4_scale_at(a.c, slots[r]) + z]);
        lo = fp4_bf16(v.x, s2);
        hi = fp4_bf16(v.y, s2);
      }
      uint4* p = reinterpret_cast<uint4*>((i ? to.v : to.k) + dst * 2);
      p[0] = lo;
      p[1] = hi;
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

size_t attend_fp4_workspace(const KV& c, int H, int T) {
  const Unpacked u = unpacked(c);
  return u.all + attend_workspace(u.c, GMC_BF16, H, T);
}

cudaError_t launch_attend_fp4(AttnArgs a, void* ws, cudaStream_t st, int* launches) {
  Unpacked u = unpacked(a.c);
  u.c.table = reinterpret_cast<int32_t*>(ws);
  u.c.k = (char*)ws + u.table;
  u.c.v = u.c.k + u.pool;
  const cudaError_t e = launch_k(k_unpack, dim3(u.c.max_pages * (UP_PAGE / UP_ROWS), a.c.B),
                                 dim3(UP_THREADS), 0, st, 1, a, u.c);
  if (e != cudaSuccess) return e;
  ++*launches;
  a.c = u.c;
  return launch_attend(a, GMC_BF16, (char*)ws + u.all, st, launches);
}

}  // namespace gmc
