// The paged key-value cache as the kernels see it, and which keys a query sees.
#pragma once

#include "common.cuh"
#include "kernels.cuh"

namespace gmc {

// Lets the next kernel on the stream be set up while this one runs (it waits in its
// own grid_dep_wait before it touches memory).
__device__ __forceinline__ void grid_dep_launch() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

constexpr uint32_t CACHE_BAD = GMC_STATUS_CACHE;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// gmc_kv_cache by value; cap = the longest a sequence may be.
struct KV {
  char *k, *v;
  const int32_t* table;
  int32_t* lens;
  uint32_t* status;
  long long page_stride, head_stride, slot_stride;  // elements
  int B, Hkv, d, ps, num_pages, max_pages, cap;
};

// Tokens of sequence b, clamped to what the cache can hold (read from L2, see
// k_decode_join).
__device__ __forceinline__ int kv_clamp(const KV& c, int n) {
  if (n < 0 || n > c.cap) {
    set_status(c.status, CACHE_BAD);
    return n < 0 ? 0 : c.cap;
  }
  return n;
}
__device__ __forceinline__ int kv_len(const KV& c, int b) {
  return kv_clamp(c, __ldcg(c.lens + b));
}

// Where token j lies: its page as the table has it, and the slot in it.
struct Slot {
  int page, slot;
};
__device__ __forceinline__ Slot kv_slot(const KV& c, int b, int j) {
  const unsigned p = (unsigned)j / (unsigned)c.ps;
  return {c.table[(long long)b * c.max_pages + p], (int)((unsigned)j - p * (unsigned)c.ps)};
}
// Element offset of that place's row of key head h (the same in both pools), or -1 where the
// table names a page outside the pool.
__device__ __forceinline__ long long kv_row(const KV& c, int h, const Slot& at) {
  const int page = at.page;
  if ((unsigned)page >= (unsigned)c.num_pages) {
    set_status(c.status, CACHE_BAD);
    return -1;
  }
  return page * c.page_stride + h * c.head_stride + at.slot * c.slot_stride;
}
__device__ __forceinline__ long long kv_row(const KV& c, int b, int h, int j) {
  return kv_row(c, h, kv_slot(c, b, j));
}

// New rows of a sequence: rows [off, off + T) of the packed input.
struct NewRows {
  int off, T;
};
__device__ __forceinline__ NewRows new_rows(int from, int to, int rows, int Tmax,
                                            uint32_t* status) {
  NewRows r;
  r.off = from;
  r.T = to - from;
  if (r.T < 0 || r.T > Tmax || r.off < 0 || (long long)r.off + r.T > rows) {
    set_status(status, CACHE_BAD);
    r.off = 0;
    r.T = 0;
  }
  return r;
}
__device__ __forceinline__ NewRows new_rows(const int32_t* offsets, int b, int rows, int Tmax,
                                            uint32_t* status) {
  if (!offsets) return {b * Tmax, Tmax};
  return new_rows(offsets[b], offsets[b + 1], rows, Tmax, status);
}

// The keys that the queries at places i0 .. i1 see between them: [0, a) and
// [b0, b1), a <= b0 (a = 0 without sinks before the window).
struct Seen {
  int a, b0, b1;
  __device__ __forceinline__ int count() const { return a + (b1 - b0); }
  __device__ __forceinline__ int place(int x) const { return x < a ? x : x - a + b0; }
};
__device__ __forceinline__ Seen seen_keys(int i0, int i1, int window, int sinks) {
  Seen s;
  s.b1 = i1 + 1 > 0 ? i1 + 1 : 0;
  s.b0 = window > 0 && i0 >= window ? i0 - window + 1 : 0;  // i0 may lie far below 0
  if (s.b0 > s.b1) s.b0 = s.b1;
  s.a = window > 0 && sinks < s.b0 ? sinks : s.b0;
  if (s.a == s.b0) {  // the sinks reach the window: one range
    s.a = 0;
    s.b0 = 0;
  }
  return s;
}
// 2^x (relative error 2^-22, ptx ex2.approx); 0 for x = -infinity.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 at a time.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float2 unpair(f32x2 v) {
  float2 d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(v));
  return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ bool sees(int i, int j, int window, int sinks) {
  return j <= i && (window == 0 || i - j < window || j < sinks);
}

struct AttnArgs {
  KV c;
  const char* q;
  char* out;
  float* lse;
  const int32_t* q_offsets;
  long long q_row, q_head, o_row, o_head;  // elements
  int H, G, window, sinks, rows, T;
  float scale2;  // scale * log2(e): softmax in powers of two
  // a key axis split over CTAs: partial sums [split][B][T][H][d], maxima and sums
  int splits;
  float* part;
  float2* ml;  // [split][B][T][H]
};
// Row of a split's part of new token t of sequence b.
__device__ __forceinline__ long long part_row(const AttnArgs& a, int split, int b, int t) {
  return ((long long)split * a.c.B + b) * a.T + t;
}

cudaError_t launch_cache_append(const KV&, int dtype, const void* k_new, const void* v_new,
                                const int32_t* offsets, int rows, int T, cudaStream_t);

size_t attend_workspace(const KV&, int dtype, int H, int T);
void* tensor_map_encoder();  // cuTensorMapEncodeTiled, or NULL
bool attend_tc_takes(const KV&, int dtype, int G);
int attend_tc_splits(const KV&, int G, int T);
cudaError_t launch_attend_tc(const AttnArgs&, cudaStream_t);
bool attend_f32_takes(const KV&, int dtype);
int attend_f32_splits(const KV&, int G, int T);
cudaError_t launch_attend_f32(const AttnArgs&, cudaStream_t);
cudaError_t launch_attend_join(const AttnArgs& a, int dtype, cudaStream_t);  // of part and ml
cudaError_t launch_attend(AttnArgs a, int dtype, void* ws, cudaStream_t, int* launches);

struct DecodeArgs {
  KV c;
  const char *q, *k_new, *v_new;
  char* out;
  float* lse;
  const float* scores;
  float* out_scores;
  long long score_stride;
  long long q_row, q_head, o_row, o_head;
  int H, G, window, sinks;
  float scale2;
  int h0, heads;      // query heads of a key head in this launch: from h0 on
  bool fresh;         // the appended key's score starts from 0
  // workspace, see k_decode.cu
  float2* ml;                  // [part][heads] maxima and sums
  float* part;                 // [part][heads][DP] outputs, unnormalised
  float* logits;               // [B][Hkv][places][hs]
  int places, hs;
  int warps;  // of the launch
  unsigned page16, head16, slot16;  // strides in pieces of 16 bytes
};
int sm_count();  // of the current device
size_t decode_workspace(const KV&, int dtype, int H);
cudaError_t launch_decode(DecodeArgs a, int dtype, void* ws, cudaStream_t, int* launches);

struct EvictArgs {
  KV src, dst;
  const float* scores;
  long long score_stride;
  int keep, sinks, recent;
  int32_t* out_idx;
  float* out_scores;
};
cudaError_t launch_evict(const EvictArgs&, int dtype, cudaStream_t);

}  // namespace gmc
