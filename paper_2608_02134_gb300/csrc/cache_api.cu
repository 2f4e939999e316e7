// C-ABI entry points of the key-value cache and its attention (declared and
// documented in include/gmc.h): argument checks, workspaces and launches.
#include <math.h>

#include "cache.cuh"

using namespace gmc;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

int cuda_rc(cudaError_t e) {
  if (e == cudaSuccess) return GMC_OK;
  cudaGetLastError();
  return GMC_ERR_CUDA;
}

constexpr int MAX_PLACES = 0x40000000;  // of a sequence, new ones too: tiles are counted in 32 bits

int esize_of(int dtype) { return dtype == GMC_BF16 ? 2 : 4; }

// The cache's shape alone (what the workspace sizes need).
int check_shape(const gmc_kv_cache* c) {
  if (!c || c->B < 1 || c->Hkv < 1 || c->d < 1 || c->page_size < 1 || c->num_pages < 1 ||
      c->max_pages < 1 || c->max_len < 0)
    return GMC_ERR_ARG;
  if (c->dtype != GMC_F32 && c->dtype != GMC_BF16) return GMC_ERR_ARG;
  // places are 32-bit; grids hold a sequence or a key head a block
  if ((long long)c->page_size * c->max_pages > MAX_PLACES || c->B > 65535 || c->Hkv > 65535)
    return GMC_ERR_UNSUPPORTED;
  if (c->max_len > c->page_size * c->max_pages) return GMC_ERR_ARG;
  // turns of 16 keys over all sequences and key heads are counted in 32 bits
  if ((long long)c->B * c->Hkv * (c->page_size * (long long)c->max_pages / 16 + 1) > 0x40000000LL)
    return GMC_ERR_UNSUPPORTED;
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
  v.slot_stride = c->slot_stride;
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
  if (!stride_ok(a->q_row_stride, c->dtype) || !stride_ok(a->q_head_stride, c->dtype) ||
      !stride_ok(a->out_row_stride, c->dtype) || !stride_ok(a->out_head_stride, c->dtype))
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

size_t gmc_attend_workspace_size(const gmc_kv_cache* cache, int H, int T) {
  if (check_shape(cache) != GMC_OK || check_heads(cache, H) != GMC_OK || T < 1 ||
      T > MAX_PLACES)
    return 0;
  return attend_workspace(view(cache), cache->dtype, H, T);
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
  if (ws_bytes < attend_workspace(a.c, cache->dtype, attn->H, T)) return GMC_ERR_WORKSPACE;
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
  rc = cuda_rc(launch_attend(a, cache->dtype, workspace, (cudaStream_t)stream, &launches));
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
  if (page * esize_of(cache->dtype) / 2 > 0xffff0000LL) return GMC_ERR_UNSUPPORTED;
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
