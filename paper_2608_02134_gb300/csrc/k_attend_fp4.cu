// Attention of new tokens over a cache held in 4 bits.  Few tokens, of 64 or 128 channels, go to
// the kernel that reads the codes (k_attend_fp4_tc.cu), of 256 token by token to gmc_decode's;
// else the seen rows of every sequence are unpacked to bf16, which holds their values exactly,
// into pages of the workspace, and gmc_attend's kernels for bf16 run on these.
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

// ---- d = 256: the new tokens one by one, as gmc_decode's sequences ---------------------------
// The tensor cores' kernels are built for up to 128 channels; decode's takes 256 and reads the
// codes, once for every token.  Token t of sequence b becomes sequence b T + t: its tokens are those up to its place, its pages
// are the same.  Of ragged calls the queries move there and the outputs back.
// Tokens of a launch: every warp of decode looks through their lengths (2,048 tokens on themselves
// 1,413 us in one launch, 589 in eight).
constexpr int AL_CHUNK = 256;
struct Alone {
  KV c;
  size_t lens, table, q, out, lse, all;  // bytes of each part, and of all with decode's own
};
Alone alone(const KV& c, int H, int T) {
  Alone x;
  x.c = c;
  x.c.B = c.B * T;
  x.c.max_pages = ceil_div(c.cap, c.ps);
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  const size_t n = x.c.B;
  x.lens = up(n * 4);
  x.table = up(n * x.c.max_pages * 4);
  x.q = x.out = n * H * c.d * 2;
  x.lse = up(n * H * 4);
  KV some = x.c;
  some.B = std::min(some.B, AL_CHUNK);
  x.all = x.lens + x.table + x.q + x.out + x.lse + decode_workspace(some, GMC_FP4, H, false);
  return x;
}
bool fits_alone(const KV& c, int T) {  // a table of 64 MB at most; turns are counted in 32 bits
  const long long n = (long long)c.B * T, some = std::min<long long>(n, AL_CHUNK);
  return c.d == 256 && n <= 16384 && n * ceil_div(c.cap, c.ps) <= (16 << 20) &&
         some * c.Hkv * (c.cap / 16 + 1) <= 0x40000000LL;
}
// Whether that takes less than unpacking and the CUDA cores, in us.  8 query and 2 key heads, us so
// and so: 3 tokens on 5 x 402 keys 12 and 92; 16 tokens on 16,004 49 and 187, on 8 x 16,004 277
// and 720; 700 tokens on themselves 155 and 222; 2,048 on 16,004 3,970 and 8,590; 64 on 32 x 500
// 450 and 339; 623 through a window of 329 141 and 125.
bool takes_alone(const KV& c, int G, int T, int window, int sinks) {
  if (!fits_alone(c, T)) return false;
  const double n = (double)c.B * T;
  const double seen = window > 0 ? fmin(c.cap, (double)window + sinks) : c.cap;
  const double turns = n * c.Hkv * ceil(seen / 32) * ceil_div(G, 8);
  return 45 * ceil(n / AL_CHUNK) + 0.0019 * turns < 90 + 36e-6 * n * G * c.Hkv * seen;
}

constexpr int AL_THREADS = 128;
__global__ void __launch_bounds__(AL_THREADS) k_alone(AttnArgs a, KV to, char* q) {
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.x / a.T, t = blockIdx.x - b * a.T, tid = threadIdx.x;
  const int n = kv_len(a.c, b);
  const NewRows nr = new_rows(a.q_offsets, b, a.rows, a.T, a.c.status);
  const int len = t < nr.T ? max(n - nr.T + t + 1, 0) : 0;
  if (tid == 0) to.lens[blockIdx.x] = len;
  const int32_t* from = a.c.table + (long long)b * a.c.max_pages;
  int32_t* pages = const_cast<int32_t*>(to.table) + (long long)blockIdx.x * to.max_pages;
  for (int x = tid; x < ceil_div(len, a.c.ps); x += AL_THREADS) pages[x] = from[x];
  if (!q || t >= nr.T) return;
  const char* row = a.q + (nr.off + t) * a.q_row * 2;
  const int each = a.c.d / 8;  // pieces of 16 bytes of a head
  for (int x = tid; x < a.H * each; x += AL_THREADS)
    reinterpret_cast<uint4*>(q)[(long long)blockIdx.x * a.H * each + x] =
        *reinterpret_cast<const uint4*>(row + (x / each * a.q_head + x % each * 8) * 2);
}
__global__ void __launch_bounds__(AL_THREADS) k_alone_back(AttnArgs a, const char* __restrict__ out,
                                                           const float* __restrict__ lse) {
  grid_dep_launch();
  grid_dep_wait();
  const int b = blockIdx.x / a.T, t = blockIdx.x - b * a.T, tid = threadIdx.x;
  const NewRows nr = new_rows(a.q_offsets, b, a.rows, a.T, a.c.status);
  if (t >= nr.T) return;
  char* row = a.out + (nr.off + t) * a.o_row * 2;
  const int each = a.c.d / 8;
  for (int x = tid; x < a.H * each; x += AL_THREADS)
    *reinterpret_cast<uint4*>(row + (x / each * a.o_head + x % each * 8) * 2) =
        reinterpret_cast<const uint4*>(out)[(long long)blockIdx.x * a.H * each + x];
  if (a.lse)
    for (int x = tid; x < a.H; x += AL_THREADS)
      a.lse[(long long)(nr.off + t) * a.H + x] = lse[(long long)blockIdx.x * a.H + x];
}

cudaError_t launch_alone(const AttnArgs& a, void* ws, cudaStream_t st, int* launches) {
  Alone x = alone(a.c, a.H, a.T);
  char* at = (char*)ws;
  auto next = [&](size_t bytes) {
    char* p = at;
    at += bytes;
    return p;
  };
  x.c.lens = reinterpret_cast<int32_t*>(next(x.lens));
  x.c.table = reinterpret_cast<int32_t*>(next(x.table));
  char *q = next(x.q), *out = next(x.out);
  float* lse = reinterpret_cast<float*>(next(x.lse));
  const bool moved = a.q_offsets != nullptr;
  cudaError_t e = launch_k(k_alone, dim3(x.c.B), dim3(AL_THREADS), 0, st, 1, a, x.c,
                           moved ? q : (char*)nullptr);
  if (e != cudaSuccess) return e;
  ++*launches;
  DecodeArgs d{};
  d.c = x.c;
  d.q = moved ? q : a.q;
  d.out = moved ? out : a.out;
  d.lse = moved ? lse : a.lse;
  d.q_row = moved ? (long long)a.H * a.c.d : a.q_row;
  d.q_head = moved ? a.c.d : a.q_head;
  d.o_row = moved ? (long long)a.H * a.c.d : a.o_row;
  d.o_head = moved ? a.c.d : a.o_head;
  d.H = a.H;
  d.G = a.G;
  d.window = a.window;
  d.sinks = a.sinks;
  d.scale2 = a.scale2;
  for (int n = x.c.B; n > 0; n -= AL_CHUNK) {
    d.c.B = std::min(n, AL_CHUNK);
    if ((e = launch_decode(d, GMC_FP4, at, st, launches)) != cudaSuccess) return e;
    d.c.lens += AL_CHUNK;
    d.c.table += (long long)AL_CHUNK * d.c.max_pages;
    d.q += AL_CHUNK * d.q_row * 2;
    d.out += AL_CHUNK * d.o_row * 2;
    if (d.lse) d.lse += (long long)AL_CHUNK * a.H;
  }
  if (!moved) return cudaSuccess;
  e = launch_k(k_alone_back, dim3(x.c.B), dim3(AL_THREADS), 0, st, 1, a, (const char*)out,
               (const float*)lse);
  if (e == cudaSuccess) ++*launches;
  return e;
}
}  // namespace

size_t attend_fp4_workspace(const KV& c, int H, int T) {
  if (direct(c, H / c.Hkv, T)) {
    const int s = attend_direct_splits(c, H / c.Hkv, T);
    const size_t rows = (size_t)c.B * T * H * s;
    return s == 1 ? 256 : 256 + ((rows * 8 + 255) & ~(size_t)255) + rows * c.d * 4;
  }
  const Unpacked u = unpacked(c);
  const size_t n = u.all + attend_workspace(u.c, GMC_BF16, H, T, parts(u.c, H / c.Hkv, T, c.cap));
  return fits_alone(c, T) ? std::max(n, alone(c, H, T).all) : n;  // a window may decide
}

cudaError_t launch_attend_fp4(AttnArgs a, void* ws, cudaStream_t st, int* launches) {
  if (takes_alone(a.c, a.G, a.T, a.window, a.sinks)) return launch_alone(a, ws, st, launches);
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
