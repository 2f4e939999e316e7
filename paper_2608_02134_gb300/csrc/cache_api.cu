// C-ABI entry points of the key-value cache and its attention (declared and
// documented in include/gmc.h): argument checks, workspaces and launches.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "cache.cuh"
#include "fp4.cuh"

using namespace gmc;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

int cuda_rc(cudaError_t e) {
  if (e == cudaSuccess) return GMC_OK;
  cudaGetLastError();
  return GMC_ERR_CUDA;
}

constexpr int MAX_PLACES = 0x40000000;  // of a sequence, new ones too: tiles are counted in 32 bits

int esize_of(int dtype) { return dtype == GMC_FP4 ? 1 : dtype == GMC_BF16 ? 2 : 4; }  // in pages
int row_type(int dtype) { return dtype == GMC_FP4 ? GMC_BF16 : dtype; }  // of rows outside

// The cache's shape alone (what the workspace sizes need).
int check_shape(const gmc_kv_cache* c) {
  if (!c || c->B < 1 || c->Hkv < 1 || c->d < 1 || c->page_size < 1 || c->num_pages < 1 ||
      c->max_pages < 1 || c->max_len < 0)
    return GMC_ERR_ARG;
  if (c->dtype != GMC_F32 && c->dtype != GMC_BF16 && c->dtype != GMC_FP4) return GMC_ERR_ARG;
  // places are 32-bit; grids hold a sequence or a key head a block
  if ((long long)c->page_size * c->max_pages > MAX_PLACES || c->B > 65535 || c->Hkv > 65535)
    return GMC_ERR_UNSUPPORTED;
  if (c->max_len > c->page_size * c->max_pages) return GMC_ERR_ARG;
  // turns of 16 keys over all sequences and key heads are counted in 32 bits
  if ((long long)c->B * c->Hkv * (c->page_size * (long long)c->max_pages / 16 + 1) > 0x40000000LL)
    return GMC_ERR_UNSUPPORTED;
  if (c->dtype == GMC_FP4)
    return c->d == 64 || c->d == 128 || c->d == 256 ? GMC_OK : GMC_ERR_UNSUPPORTED;
  if (c->d > GMC_MAX_CACHE_D || c->d % (16 / esize_of(c->dtype)) != 0) return GMC_ERR_UNSUPPORTED;
  return GMC_OK;
}

bool stride_ok(int64_t s, int dtype) { return s >= 0 && s % (16 / esize_of(dtype)) == 0; }

int check_cache(const gmc_kv_cache* c) {
  const int rc = check_shape(c);
  if (rc != GMC_OK) return rc;
  if (!c->k || !c->v || !c->page_table || !c->lens) return GMC_ERR_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->page_table, 4) ||
      !aligned(c->lens, 4) || !aligned(c->status, 4))
    return GMC_ERR_ARG;
  if (!stride_ok(c->page_stride, c->dtype) || !stride_ok(c->head_stride, c->dtype) ||
      !stride_ok(c->slot_stride, c->dtype))
    return GMC_ERR_ARG;
  if (c->dtype == GMC_FP4) {  // slots lie as the format says, parts of pages apart
    const long long part = fp4_part(c->page_size, c->d);
    // n parts `inner` apart lie within `outer`
    auto within = [part](long long inner, int n, long long outer) {
      return outer >= part && (n == 1 || (inner >= part && inner <= (outer - part) / (n - 1)));
    };
    const long long head = c->Hkv > 1 ? c->head_stride : LLONG_MAX,
                    page = c->num_pages > 1 ? c->page_stride : LLONG_MAX;
    if (c->slot_stride != 0 ||
        !(within(head, c->Hkv, page) || within(page, c->num_pages, head)))
      return GMC_ERR_ARG;
  }
  return GMC_OK;
}

KV view(const gmc_kv_cache* c) {
  KV v;
  v.k = (char*)c->k;
  v.v = (char*)c->v;
  v.table = c->page_table;
  v.lens = c->lens;
  v.status = c->status;
  v.page_stride = c->page_stride;
  v.head_stride = c->head_stride;
  v.slot_stride = c->dtype == GMC_FP4 ? c->d / 2 : c->slot_stride;
  v.B = c->B;
  v.Hkv = c->Hkv;
  v.d = c->d;
  v.ps = c->page_size;
  v.num_pages = c->num_pages;
  v.max_pages = c->max_pages;
  v.cap = c->max_len > 0 ? c->max_len : c->page_size * c->max_pages;
  return v;
}

int check_heads(const gmc_kv_cache* c, int H) {
  if (H < 1 || H % c->Hkv != 0) return GMC_ERR_ARG;
  return H / c->Hkv > 128 ? GMC_ERR_UNSUPPORTED : GMC_OK;
}

int check_attn(const gmc_kv_cache* c, const gmc_attn* a) {
  if (!a || a->window < 0 || a->sinks < 0 || !(a->scale >= 0.f) || isinf(a->scale))
    return GMC_ERR_ARG;
  const int rc = check_heads(c, a->H);
  if (rc != GMC_OK) return rc;
  const int t = row_type(c->dtype);
  if (!stride_ok(a->q_row_stride, t) || !stride_ok(a->q_head_stride, t) ||
      !stride_ok(a->out_row_stride, t) || !stride_ok(a->out_head_stride, t))
    return GMC_ERR_ARG;
  return GMC_OK;
}

// rows rows of new tokens, T a sequence at most
int check_rows(const gmc_kv_cache* c, const int32_t* offsets, int rows, int T) {
  if (rows < 0 || T < 1 || !aligned(offsets, 4)) return GMC_ERR_ARG;
  if (T > MAX_PLACES) return GMC_ERR_UNSUPPORTED;
  if (!offsets && (long long)c->B * T != rows) return GMC_ERR_ARG;
  return GMC_OK;
}

// A window of all places is none; a smaller one can be taken from a place in 32 bits.
int window_of(const KV& c, const gmc_attn* at) { return at->window < c.cap ? at->window : 0; }

void heads_of(const gmc_kv_cache* c, const gmc_attn* at, long long* q_row, long long* q_head,
              long long* o_row, long long* o_head, float* scale2) {
  *q_row = at->q_row_stride ? at->q_row_stride : (long long)at->H * c->d;
  *q_head = at->q_head_stride ? at->q_head_stride : c->d;
  *o_row = at->out_row_stride ? at->out_row_stride : (long long)at->H * c->d;
  *o_head = at->out_head_stride ? at->out_head_stride : c->d;
  const double s = at->scale > 0.f ? (double)at->scale : 1.0 / sqrt((double)c->d);
  *scale2 = (float)(s * 1.4426950408889634074);
}

// One token a sequence over 4 bits goes the way of gmc_decode, which reads the codes themselves.
size_t attend_ws(const gmc_kv_cache* c, int H, int T) {
  if (c->dtype != GMC_FP4) return attend_workspace(view(c), c->dtype, H, T);
  const size_t n = attend_fp4_workspace(view(c), H, T);
  return T == 1 ? std::max(n, decode_workspace(view(c), c->dtype, H)) : n;
}
cudaError_t attend_one(const AttnArgs& a, void* ws, cudaStream_t st, int* launches) {
  DecodeArgs d{};
  d.c = a.c;
  d.q = a.q;
  d.out = a.out;
  d.lse = a.lse;
  d.q_row = a.q_row;
  d.q_head = a.q_head;
  d.o_row = a.o_row;
  d.o_head = a.o_head;
  d.H = a.H;
  d.G = a.G;
  d.window = a.window;
  d.sinks = a.sinks;
  d.scale2 = a.scale2;
  return launch_decode(d, GMC_FP4, ws, st, launches);
}

}  // namespace

extern "C" {

int gmc_cache_append(const gmc_kv_cache* cache, const void* k_new, const void* v_new,
                     const int32_t* offsets, int rows, int T, gmc_stream_t stream) {
  int rc = check_cache(cache);
  if (rc == GMC_OK) rc = check_rows(cache, offsets, rows, T);
  if (rc != GMC_OK || rows == 0) return rc;  // no rows: their pointers may be NULL
  if (!k_new || !aligned(k_new, 16) || !aligned(v_new, 16)) return GMC_ERR_ARG;
  rc = cuda_rc(launch_cache_append(view(cache), cache->dtype, k_new, v_new, offsets, rows, T,
                                   (cudaStream_t)stream));
  if (rc == GMC_OK) count_launches(1);
  return rc;
}

int gmc_cache_append_rope(const gmc_kv_cache* cache, const gmc_rope* rope,
                          const int32_t* positions, const void* k_new, const void* v_new,
                          const void* q, void* out, const int32_t* offsets, int rows, int T,
                          gmc_stream_t stream) {
  int rc = check_cache(cache);
  if (rc == GMC_OK) rc = check_rows(cache, offsets, rows, T);
  if (rc != GMC_OK) return rc;
  const int t = row_type(cache->dtype);
  const int d = cache->d, n = rope ? rope->rot / 2 : 0;
  if (!rope || !rope->table || !aligned(rope->table, 16) || rope->max_pos < 1 || rope->H < 0 ||
      rope->rot < 2 || rope->rot > d || (rope->interleaved != 0 && rope->interleaved != 1) ||
      !aligned(positions, 4) || !stride_ok(rope->q_row_stride, t) ||
      !stride_ok(rope->out_row_stride, t) || !stride_ok(rope->new_row_stride, t))
    return GMC_ERR_ARG;
  const int* sect = rope->sections;
  if (sect[0] < 0 || sect[1] < 0 || sect[2] < 0) return GMC_ERR_ARG;
  const long long pairs = (long long)sect[0] + sect[1] + sect[2];
  const bool rows3 = pairs != 0;
  if (rows3 && (pairs != n || !positions)) return GMC_ERR_ARG;
  if (rope->H > 0 && check_heads(cache, rope->H) != GMC_OK) return check_heads(cache, rope->H);
  // k_append_rope counts a row's channels, and the pieces of a block's 64 rows, in 32 bits
  if ((long long)rope->H * d > 1 << 26) return GMC_ERR_UNSUPPORTED;
  // pieces of 16 bytes hold whole pairs, of 4 bits whole blocks
  if (rope->rot % (cache->dtype == GMC_FP4 ? 32 : 16) != 0) return GMC_ERR_UNSUPPORTED;
  const int64_t dense = (int64_t)cache->Hkv * d, dense_q = (int64_t)rope->H * d;
  if ((rope->new_row_stride && (rope->new_row_stride < dense || (!v_new && rope->new_row_stride != dense))) ||
      (rope->q_row_stride && rope->q_row_stride < dense_q) ||
      (rope->out_row_stride && rope->out_row_stride < dense_q))
    return GMC_ERR_ARG;
  if (rows == 0) return GMC_OK;  // no rows: their pointers may be NULL
  if (!k_new || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q, 16) ||
      !aligned(out, 16) || (rope->H > 0) != (q != nullptr) || (rope->H > 0) != (out != nullptr))
    return GMC_ERR_ARG;
  RopeArgs a{};
  a.c = view(cache);
  a.table = rope->table;
  a.pos = positions;
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.q = (const char*)q;
  a.out = (char*)out;
  a.offsets = offsets;
  a.q_row = rope->q_row_stride ? rope->q_row_stride : dense_q;
  a.o_row = rope->out_row_stride ? rope->out_row_stride : dense_q;
  a.n_row = rope->new_row_stride ? rope->new_row_stride : dense;
  if (q == out && a.q_row != a.o_row) return GMC_ERR_ARG;
  a.max_pos = rope->max_pos;
  a.rot = rope->rot;
  a.near = rope->interleaved;
  a.rows3 = rows3;
  a.sect0 = sect[0];
  a.sect1 = sect[0] + sect[1];
  a.H = rope->H;
  a.rows = rows;
  a.T = T;
  rc = cuda_rc(launch_append_rope(a, cache->dtype, (cudaStream_t)stream));
  if (rc == GMC_OK) count_launches(1);
  return rc;
}

int gmc_cache_read(const gmc_kv_cache* cache, void* k_out, void* v_out, const int32_t* offsets,
                   int rows, int T, gmc_stream_t stream) {
  int rc = check_cache(cache);
  if (rc == GMC_OK) rc = check_rows(cache, offsets, rows, T);
  if (rc != GMC_OK || rows == 0) return rc;  // no rows: their pointers may be NULL
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return GMC_ERR_ARG;
  rc = cuda_rc(launch_cache_read(view(cache), cache->dtype, (char*)k_out, (char*)v_out, offsets,
                                 rows, T, (cudaStream_t)stream));
  if (rc == GMC_OK) count_launches(1);
  return rc;
}

size_t gmc_cache4_part_size(int page_size, int d) {
  if (page_size < 1 || page_size > MAX_PLACES || (d != 64 && d != 128 && d != 256)) return 0;
  return (size_t)((fp4_part(page_size, d) + 15) / 16 * 16);
}

size_t gmc_attend_workspace_size(const gmc_kv_cache* cache, int H, int T) {
  if (check_shape(cache) != GMC_OK || check_heads(cache, H) != GMC_OK || T < 1 ||
      T > MAX_PLACES)
    return 0;
  return attend_ws(cache, H, T);
}

int gmc_attend(const gmc_kv_cache* cache, const gmc_attn* attn, const void* q,
               const int32_t* q_offsets, int rows, int T, void* out, float* lse, void* workspace,
               size_t ws_bytes, gmc_stream_t stream) {
  int rc = check_cache(cache);
  if (rc == GMC_OK) rc = check_attn(cache, attn);
  if (rc == GMC_OK) rc = check_rows(cache, q_offsets, rows, T);
  if (rc != GMC_OK || rows == 0) return rc;  // no rows: their pointers may be NULL
  if (!q || !out || !workspace || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) ||
      !aligned(workspace, 256))
    return GMC_ERR_ARG;
  AttnArgs a{};
  a.c = view(cache);
  if (ws_bytes < attend_ws(cache, attn->H, T)) return GMC_ERR_WORKSPACE;
  a.q = (const char*)q;
  a.out = (char*)out;
  a.lse = lse;
  a.q_offsets = q_offsets;
  heads_of(cache, attn, &a.q_row, &a.q_head, &a.o_row, &a.o_head, &a.scale2);
  a.H = attn->H;
  a.G = attn->H / cache->Hkv;
  a.window = window_of(a.c, attn);
  a.sinks = attn->sinks;
  a.rows = rows;
  a.T = T;
  int launches = 0;
  rc = cuda_rc(cache->dtype == GMC_FP4 && T == 1 && !q_offsets
                   ? attend_one(a, workspace, (cudaStream_t)stream, &launches)
               : cache->dtype == GMC_FP4
                   ? launch_attend_fp4(a, workspace, (cudaStream_t)stream, &launches)
                   : launch_attend(a, cache->dtype, workspace, (cudaStream_t)stream, &launches));
  count_launches(launches);
  return rc;
}

size_t gmc_decode_workspace_size(const gmc_kv_cache* cache, int H) {
  if (check_shape(cache) != GMC_OK || check_heads(cache, H) != GMC_OK) return 0;
  return decode_workspace(view(cache), cache->dtype, H);
}

int gmc_decode(const gmc_kv_cache* cache, const gmc_attn* attn, const void* q, const void* k_new,
               const void* v_new, void* out, float* lse, const float* scores, float* out_scores,
               int64_t score_stride, void* workspace, size_t ws_bytes, gmc_stream_t stream) {
  int rc = check_cache(cache);
  if (rc == GMC_OK) rc = check_attn(cache, attn);
  if (rc != GMC_OK) return rc;
  if (!q || !out || !workspace || !k_new != !v_new || !scores != !out_scores) return GMC_ERR_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) ||
      !aligned(lse, 4) || !aligned(scores, 4) || !aligned(out_scores, 4) ||
      !aligned(workspace, 256))
    return GMC_ERR_ARG;
  DecodeArgs a{};
  a.c = view(cache);
  // offsets inside a page are kept as 32-bit numbers of 16 bytes
  const long long page = a.c.head_stride / 8 * (a.c.Hkv - 1) + a.c.slot_stride / 8 * (a.c.ps - 1);
  if (cache->dtype != GMC_FP4 && page * esize_of(cache->dtype) / 2 > 0xffff0000LL)
    return GMC_ERR_UNSUPPORTED;
  if (scores && score_stride < a.c.cap) return GMC_ERR_ARG;
  if (ws_bytes < decode_workspace(a.c, cache->dtype, attn->H)) return GMC_ERR_WORKSPACE;
  a.q = (const char*)q;
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.out = (char*)out;
  a.lse = lse;
  a.scores = scores;
  a.out_scores = out_scores;
  a.score_stride = score_stride;
  heads_of(cache, attn, &a.q_row, &a.q_head, &a.o_row, &a.o_head, &a.scale2);
  a.H = attn->H;
  a.G = attn->H / cache->Hkv;
  a.window = window_of(a.c, attn);
  a.sinks = attn->sinks;
  int launches = 0;
  rc = cuda_rc(launch_decode(a, cache->dtype, workspace, (cudaStream_t)stream, &launches));
  count_launches(launches);
  return rc;
}

size_t gmc_evict_workspace_size(const gmc_kv_cache* src, int keep) {
  if (check_shape(src) != GMC_OK || keep < 1) return 0;
  return 256;
}

int gmc_evict(const gmc_kv_cache* src, const gmc_kv_cache* dst, const float* scores,
              int64_t score_stride, int keep, int sinks, int recent, int32_t* out_idx,
              float* out_scores, void* workspace, size_t ws_bytes, gmc_stream_t stream) {
  int rc = check_cache(src);
  if (rc == GMC_OK) rc = check_cache(dst);
  if (rc != GMC_OK) return rc;
  if (src->B != dst->B || src->Hkv != dst->Hkv || src->d != dst->d || src->dtype != dst->dtype)
    return GMC_ERR_ARG;
  if (!scores || !out_idx || !workspace || !aligned(scores, 4) || !aligned(out_idx, 4) ||
      !aligned(out_scores, 4) || !aligned(workspace, 256))
    return GMC_ERR_ARG;
  EvictArgs a;
  a.src = view(src);
  a.dst = view(dst);
  if (keep < 1 || sinks < 0 || recent < 0 || (long long)sinks + recent > keep ||
      keep > a.dst.cap || score_stride < a.src.cap || src->lens == dst->lens)
    return GMC_ERR_ARG;
  if (ws_bytes < gmc_evict_workspace_size(src, keep)) return GMC_ERR_WORKSPACE;
  a.scores = scores;
  a.score_stride = score_stride;
  a.keep = keep;
  a.sinks = sinks;
  a.recent = recent;
  a.out_idx = out_idx;
  a.out_scores = out_scores;
  rc = cuda_rc(launch_evict(a, src->dtype, (cudaStream_t)stream));
  if (rc == GMC_OK) count_launches(1);
  return rc;
}

}  // extern "C"
