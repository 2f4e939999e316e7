// Causal attention of new tokens over a paged key-value cache on the tcgen05 tensor
// cores: bf16 caches with d <= 128.
//
// A CTA takes two tiles of up to 128 rows, a row being one query head of one token:
// the G query heads of a key head and 128 / G consecutive tokens make a tile, so each
// key and value is read once for all of them.  It walks the seen keys 128 at a time
// (whole pages where they are smaller).  One warp copies keys and values by TMA into a
// ring of five 128-row slots, one thread issues the products
//     S = Q K^T   (128 x 128, fp32 in tensor memory)
//     O += P V    (P bf16 in tensor memory over S's columns, V as the MN-major operand)
// and a warpgroup a tile turns S into P: a thread holds a row's 128 logits, so maxima
// and sums need no exchange.  The two tiles alternate: while one's logits become
// weights the tensor cores work for the other.  The maximum that weights are taken
// against follows the running one only when it has grown by 2^8 (weights up to 256
// lose nothing in bf16 or fp32), so the output in tensor memory is hardly ever
// rescaled, and a turn's weights need not wait for its maximum: they are taken against
// the one so far while it is looked for, and anew if it had grown (32 questions of 16 to
// 256 tokens on up to 513 keys: 52.1 -> 49.3 us, a question of 128 tokens on 16,004 keys:
// 41.8 -> 40.0).
//
// Weights are rounded to bf16 for their product with V (relative 2^-8, the same as the
// output's own rounding); sums, maxima and products are fp32.
//
// Rows of a tile that do not see a key give it the weight 0.  Slots past the sequence's
// end are zeroed in shared memory before the product reads them; where a tile of keys
// is seen by some rows only, its values are looked over, and if one is not finite
// (0 x NaN would reach rows that do not see it) the CTA computes its rows again one by
// one, each from the keys that it sees.
//
// Every wait is bounded (about two seconds); on timeout GMC_STATUS_TIMEOUT is set in
// the cache's status word, copies and products in flight are drained and tensor memory
// is freed.
#include <algorithm>

#include "attend_tc.cuh"

namespace gmc {

namespace {
// 128-row slots of the ring: what shared memory holds beside the queries, for one CTA of
// two tiles an SM or two CTAs of one.
template <int DP, int TILES> constexpr int t_slots() {
  return TILES == 2 ? (DP == 128 ? 5 : 8) : (DP == 128 ? 2 : 4);
}
template <int TILES> constexpr int t_threads() { return TILES * 128 + 64; }

struct TCtl {
  uint64_t full[8], empty[8], qfull, sfull[2], pfull[2][2], drained;
  uint32_t tmem;
  volatile int abort;
  int strange;
};

template <int DP, int TILES> constexpr size_t t_smem() {
  return 1024 + (size_t)(TILES + t_slots<DP, TILES>()) * TM * DP * 2 + sizeof(TCtl);
}

// Turns of keys: pages of up to 128 slots are taken as many as fit whole, larger ones
// in pieces of 128 (the last one short).
struct Turns {
  int ps, kt, ppt, tpp;
  Div by_ps, by_kt, by_tpp, by_g, by_tokens;
  __device__ __forceinline__ int of(int j) const {  // the turn that holds place j
    if (ps <= TM) return by_kt.of(j);
    const int p = by_ps.of(j);
    return p * tpp + (j - p * ps) / TM;
  }
  __device__ __forceinline__ int first(int u) const {
    if (ps <= TM) return u * kt;
    const int p = by_tpp.of(u);
    return p * ps + (u - p * tpp) * TM;
  }
  __device__ __forceinline__ int rows(int u) const {
    if (ps <= TM) return kt;
    return min(TM, ps - (u - by_tpp.of(u) * tpp) * TM);
  }
};
Turns make_turns(int ps, int G, int tiles) {
  Turns t;
  t.ps = ps;
  t.ppt = ps <= TM ? TM / ps : 1;
  t.kt = ps <= TM ? t.ppt * ps : TM;
  t.tpp = ceil_div(ps, TM);
  t.by_ps = make_div(ps);
  t.by_kt = make_div(t.kt);
  t.by_tpp = make_div(t.tpp);
  t.by_g = make_div(G);
  t.by_tokens = make_div(TM / G * tiles);
  return t;
}

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(tc::smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z,
                                            int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(tc::smem_u32(bar))
      : "memory");
}

// 128 consecutive fp32 columns of this warp's lanes (one row a thread), waited for.
__device__ __forceinline__ void tmem_ld128(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x128.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
      "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63, "
      "%64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, %76, %77, %78, %79, "
      "%80, %81, %82, %83, %84, %85, %86, %87, %88, %89, %90, %91, %92, %93, %94, %95, "
      "%96, %97, %98, %99, %100, %101, %102, %103, %104, %105, %106, %107, %108, %109, %110, %111, "
      "%112, %113, %114, %115, %116, %117, %118, %119, %120, %121, %122, %123, %124, %125, %126, %127}, [%128];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]),
        "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
        "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
        "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]),
        "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
        "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]),
        "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]),
        "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]),
        "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]),
        "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]), "=r"(r[64]),
        "=r"(r[65]), "=r"(r[66]), "=r"(r[67]), "=r"(r[68]), "=r"(r[69]),
        "=r"(r[70]), "=r"(r[71]), "=r"(r[72]), "=r"(r[73]), "=r"(r[74]),
        "=r"(r[75]), "=r"(r[76]), "=r"(r[77]), "=r"(r[78]), "=r"(r[79]),
        "=r"(r[80]), "=r"(r[81]), "=r"(r[82]), "=r"(r[83]), "=r"(r[84]),
        "=r"(r[85]), "=r"(r[86]), "=r"(r[87]), "=r"(r[88]), "=r"(r[89]),
        "=r"(r[90]), "=r"(r[91]), "=r"(r[92]), "=r"(r[93]), "=r"(r[94]),
        "=r"(r[95]), "=r"(r[96]), "=r"(r[97]), "=r"(r[98]), "=r"(r[99]),
        "=r"(r[100]), "=r"(r[101]), "=r"(r[102]), "=r"(r[103]), "=r"(r[104]),
        "=r"(r[105]), "=r"(r[106]), "=r"(r[107]), "=r"(r[108]), "=r"(r[109]),
        "=r"(r[110]), "=r"(r[111]), "=r"(r[112]), "=r"(r[113]), "=r"(r[114]),
        "=r"(r[115]), "=r"(r[116]), "=r"(r[117]), "=r"(r[118]), "=r"(r[119]),
        "=r"(r[120]), "=r"(r[121]), "=r"(r[122]), "=r"(r[123]), "=r"(r[124]),
        "=r"(r[125]), "=r"(r[126]), "=r"(r[127])
      : "r"(taddr)
      : "memory");
}
// The largest of a row's logits.
__device__ __forceinline__ float largest(const float (&s)[TM]) {
  float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
  for (int c = 4; c + 8 <= TM; c += 8)
#pragma unroll
    for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], s[c + y], s[c + 4 + y]);
#pragma unroll
  for (int y = 0; y < 4; ++y) mx[y] = fmaxf(mx[y], s[TM - 4 + y]);
  return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}

// The values of a turn that some rows of the CTA do not see, a row a thread of the first
// tile's warps: slots past the end become zeros, others are looked over for infinities
// and NaN.  false: the copy did not come.
template <int DP>
__device__ __forceinline__ bool look_over(TCtl* ctl, char* slot, int s, uint32_t parity, int r,
                                          bool there) {
  const int lane = threadIdx.x & 31;
  const bool ok = wait_for(&ctl->full[s], parity, &ctl->abort);
  if (!__all_sync(FULL, ok)) return false;
  char* row = slot + r * 128;
  if (there) {
    const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
    __nv_bfloat162 bad = zero;
#pragma unroll
    for (int c = 0; c < DP / 8; ++c) {
      const int4 w =
          *reinterpret_cast<const int4*>(row + (c >> 3) * TM * 128 + (((c ^ lane) & 7) * 16));
      const __nv_bfloat162* e = reinterpret_cast<const __nv_bfloat162*>(&w);
#pragma unroll
      for (int y = 0; y < 4; ++y) bad = __hfma2(e[y], zero, bad);
    }
    if (__hisnan(bad.x) || __hisnan(bad.y)) ctl->strange = 1;
  } else {
#pragma unroll
    for (int c = 0; c < DP / 8; ++c)
      *reinterpret_cast<int4*>(row + (c >> 3) * TM * 128 + (((c ^ lane) & 7) * 16)) =
          make_int4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  return true;
}

template <int DP, int TILES>
__global__ void __launch_bounds__(t_threads<TILES>(), 3 - TILES)
    k_attend_tc(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                const __grid_constant__ CUtensorMap vmap, AttnArgs a, Turns tn) {
  constexpr int NS = t_slots<DP, TILES>(), THREADS = t_threads<TILES>(), COPY = 4 * TILES,
                ISSUE = COPY + 1, SLOT = TM * DP * 2, HALF = TM * 128, NH = DP / 64;
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  char* Qs = smem;
  char* ring = Qs + TILES * SLOT;
  TCtl* ctl = reinterpret_cast<TCtl*>(ring + NS * SLOT);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (warp == COPY && lane == 0) {
    tc::prefetch_tmap(&qmap);
    tc::prefetch_tmap(&kmap);
    tc::prefetch_tmap(&vmap);
  }
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) {
      tc::mbar_init(&ctl->full[s], 1);
      tc::mbar_init(&ctl->empty[s], 1);
    }
    tc::mbar_init(&ctl->qfull, 1);
    tc::mbar_init(&ctl->drained, 1);
    for (int x = 0; x < TILES; ++x) {
      tc::mbar_init(&ctl->sfull[x], 1);
      tc::mbar_init(&ctl->pfull[x][0], 4);
      tc::mbar_init(&ctl->pfull[x][1], 4);
    }
    ctl->abort = 0;
    ctl->strange = 0;
    tc::fence_mbar_init();
  }
  grid_dep_launch();
  grid_dep_wait();
  const int h = blockIdx.y;
  int c = blockIdx.x, split = 0;
  if (a.splits > 1) {
    c = blockIdx.x / a.splits;
    split = blockIdx.x - c * a.splits;
  }
  const int tpt = tn.by_g.of(TM);  // tokens of a tile
  int b, tile, n;
  NewRows nr;
  if (!find_tile(a, c, tpt * TILES, tn.by_tokens, &b, &tile, &nr, &n)) return;
  // the last tokens see the most keys: they go first
  const int t0 = (tn.by_tokens.of(nr.T + tpt * TILES - 1) - 1 - tile) * tpt * TILES;
  const int nt = min(tpt * TILES, nr.T - t0);  // tokens of this CTA
  const int i0 = n - nr.T + t0;
  const int two = TILES == 2 && nt > tpt ? 2 : 1;
  int turns = 0, na = 0, ub0 = 0, x0 = 0;
  {
    const Seen seen = seen_keys(i0, i0 + nt - 1, a.window, a.sinks);
    if (seen.b1 > 0) {
      ub0 = tn.of(min(seen.b0, seen.b1 - 1));
      na = seen.a > 0 ? min(tn.of(seen.a - 1) + 1, ub0) : 0;
      const int all = na + tn.of(seen.b1 - 1) + 1 - ub0;
      const int per = a.splits > 1 ? ceil_div(all, a.splits) : all;
      x0 = min(all, split * per);
      turns = min(all, x0 + per) - x0;
    }
  }
  auto turn_at = [&](int x) { return x0 + x < na ? x0 + x : ub0 + x0 + x - na; };

  const int box = tn.ps <= TM ? tn.ps : TM;  // rows of a copy
  const int half = lane % NH, pg = lane / NH;
  // this lane's page of turn x; num_pages (past the pool, zeros) where there is none, or none
  // that a row of the CTA sees: such a page may have been given back, its entry be anything.
  // (The seen places are found here again: kept in registers from above, they cost the other
  // warps 0.7 % of a prompt's time.)
  auto look_up = [&](int x, int* slot) {
    *slot = 0;
    if (pg >= tn.ppt || x >= turns) return a.c.num_pages;
    const int u = turn_at(x), j = tn.first(u) + pg * tn.ps;
    const Seen seen = seen_keys(i0, i0 + nt - 1, a.window, a.sinks);
    if (j >= seen.b1 || (j >= seen.a && j + box <= seen.b0)) return a.c.num_pages;
    const int p = tn.by_ps.of(j);
    *slot = j - p * tn.ps;
    const int page = a.c.table[(long long)b * a.c.max_pages + p];
    if ((unsigned)page < (unsigned)a.c.num_pages) return page;
    set_status(a.c.status, CACHE_BAD);
    return a.c.num_pages;
  };
  int slot = 0, page = 0;
  if (warp == COPY) page = look_up(0, &slot);  // on its way while the CTA gets ready
  if (tn.kt < TM) {  // rows of a slot that no copy writes
    const int per = (TM - tn.kt) * 8;
    for (int x = tid; x < NS * NH * per; x += THREADS) {
      const int s = x / per, y = x - s * per;
      *reinterpret_cast<int4*>(ring + s * HALF + tn.kt * 128 + y * 16) = make_int4(0, 0, 0, 0);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == ISSUE) {
    tc::tmem_alloc(&ctl->tmem, 256 * TILES);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = ctl->tmem;
  int issued = 0;  // copies started (copying warp)
  if (turns > 0 && warp == COPY) {
    // ---- copies ---------------------------------------------------------------------
    if (lane == 0) {
      tc::mbar_arrive_expect_tx(&ctl->qfull, two * tpt * a.G * DP * 2);
      for (int t = 0; t < two; ++t)
        for (int c = 0; c < NH; ++c)
          tma_load_3d(Qs + t * SLOT + c * HALF, &qmap, c * 64, h * a.G, nr.off + t0 + t * tpt,
                      &ctl->qfull);
    }
    bool ok = true;
    for (int x = 0; x < turns && ok; ++x) {
      int nslot;
      const int npage = look_up(x + 1, &nslot);
      for (int kv = 0; kv < 2 && ok; ++kv) {
        const int s = issued % NS;
        ok = wait_for(&ctl->empty[s], ((uint32_t)(issued / NS) & 1u) ^ 1u, &ctl->abort);
        ok = __all_sync(FULL, ok);
        if (!ok) break;
        if (lane == 0) tc::mbar_arrive_expect_tx(&ctl->full[s], tn.ppt * box * DP * 2);
        __syncwarp();
        if (pg < tn.ppt)
          tma_load_4d(ring + s * SLOT + half * HALF + pg * tn.ps * 128, kv ? &vmap : &kmap,
                      half * 64, slot, h, page, &ctl->full[s]);
        ++issued;
      }
      page = npage;
      slot = nslot;
    }
  } else if (turns > 0 && warp == ISSUE) {
    // ---- products -------------------------------------------------------------------
    constexpr uint32_t sdesc = tc::idesc_bf16_f32(TM, TM);
    constexpr uint32_t odesc = tc::idesc_bf16_f32(TM, DP) | (1u << 16);  // B is MN-major
    const uint32_t go = elect_one();
    // advancing an address by x bytes adds x / 16 to its descriptor
    const uint64_t qd = tc::desc_sw128_kmajor(Qs), kd = tc::desc_sw128_kmajor(ring),
                   vd = desc_sw128_mnmajor(tc::smem_u32(ring), HALF);
    auto logits = [&](int t, int slot) {
      const uint64_t qa = qd + t * (SLOT / 16), kb = kd + slot * (SLOT / 16);
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        const int o = ((k >> 2) * HALF + (k & 3) * 32) / 16;
        mma_ss(go, tmem + t * TM, qa + o, kb + o, sdesc, k > 0);
      }
      commit(go, &ctl->sfull[t]);
    };
    auto ready = [&](uint64_t* bar, uint32_t parity) {
      const bool ok = wait_for(bar, parity, &ctl->abort);
      return __all_sync(FULL, ok) != 0;
    };
    bool ok = ready(&ctl->qfull, 0) && ready(&ctl->full[0], 0);
    tc::fence_after_sync();
    if (ok) {
      for (int t = 0; t < two; ++t) logits(t, 0);
      commit(go, &ctl->empty[0]);
    }
    int vs = 1, ks = 2 % NS;       // slots of this turn's values and the next one's keys
    uint32_t vp = 0, kp = 2 / NS;  // and their parities
#pragma unroll 1
    for (int x = 0; x < turns && ok; ++x) {
#pragma unroll 1
      for (int t = 0; t < two; ++t) {
        const uint64_t vb = vd + vs * (SLOT / 16);
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // 64 keys' weights at a time
          ok = ok && ready(&ctl->pfull[t][half], x & 1);
          if (half == 0 && t == 0) ok = ok && ready(&ctl->full[vs], vp);
          if (!ok) break;
          tc::fence_after_sync();
#pragma unroll
          for (int k = half * (TM / 32); k < (half + 1) * (TM / 32); ++k)
            mma_ts(go, tmem + TILES * TM + t * TM, tmem + t * TM + k * 8, vb + k * (2048 / 16), odesc,
                   x > 0 || k > 0);
        }
        if (!ok) break;
        if (t == two - 1) commit(go, &ctl->empty[vs]);
        if (x + 1 < turns) {
          if (t == 0) ok = ready(&ctl->full[ks], kp);
          if (!ok) break;
          tc::fence_after_sync();
          logits(t, ks);
          if (t == two - 1) commit(go, &ctl->empty[ks]);
        } else {
          commit(go, &ctl->sfull[t]);  // the output is complete
        }
      }
      vs += 2;
      if (vs >= NS) {
        vs -= NS;
        vp ^= 1;
      }
      ks += 2;
      if (ks >= NS) {
        ks -= NS;
        kp ^= 1;
      }
    }
    if (!ok) {  // products in flight end before tensor memory is freed
      commit(go, &ctl->drained);
      const long long end = clock64() + T_WAIT;
      while (!tc::mbar_try_wait(&ctl->drained, 0) && clock64() < end) {
      }
    }
    __syncwarp();
  } else if (warp < COPY) {
    // ---- weights --------------------------------------------------------------------
    const int t = warp >> 2, r = tid & (TM - 1);
    const int tok = tn.by_g.of(r), g = r - tok * a.G;
    const int mine = min(tpt, nt - t * tpt);  // tokens of this tile
    const bool valid = tok < mine;
    const int ti0 = i0 + t * tpt, i = ti0 + tok;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's lane quarter
    const uint32_t sa = tmem + lanes + t * TM, oa = tmem + lanes + TILES * TM + t * TM;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    if (mine > 0) {
      for (int x = 0; x < turns; ++x) {
        const int u = turn_at(x), j0 = tn.first(u), cnt = tn.rows(u);
        ok = wait_for(&ctl->sfull[t], x & 1, &ctl->abort);
        ok = __all_sync(FULL, ok);
        if (!ok) break;
        tc::fence_after_sync();
        const bool whole =
            cnt == TM && j0 + TM - 1 <= ti0 &&
            (a.window == 0 || ti0 + mine - 1 - j0 < a.window || j0 + TM <= a.sinks);
        const f32x2 scale = pair(a.scale2, a.scale2);
        float s[TM];
        f32x2 off, sum[2];
        uint32_t p[32];
        auto weigh = [&](int c) {  // 64 keys from c on
#pragma unroll
          for (int y = 0; y < 32; ++y) {
            const float2 v = unpair(fma2(pair(s[c + 2 * y], s[c + 2 * y + 1]), scale, off));
            const float e0 = exp2_fast(v.x), e1 = exp2_fast(v.y);
            sum[y & 1] = add2(sum[y & 1], pair(e0, e1));
            p[y] = pack2(e0, e1);
          }
        };
        auto hand_over = [&](int half) {
          tmem_st32_async(sa + half * 32, p);
          tmem_wait_st();
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&ctl->pfull[t][half]);
        };
        while (true) {
          tmem_ld128(sa, s);
          if (!whole) {
            const int hi = valid ? min(min(i + 1, n) - j0, cnt) : 0;  // columns before hi,
            const int lo = a.window > 0 ? i - a.window + 1 - j0 : 0;  // from lo on
            const int sk = a.sinks - j0;                              // or before sk
#pragma unroll
            for (int c = 0; c < TM; c += 32) {
              const uint32_t in = below(hi - c) & (~below(lo - c) | below(sk - c));
#pragma unroll
              for (int y = 0; y < 32; ++y)
                if (!(in >> y & 1)) s[c + y] = -INFINITY;
            }
          }
          if (x == 0) m = largest(s) * a.scale2;
          const float base = m == -INFINITY ? 0.f : m;
          off = pair(-base, -base);
          sum[0] = sum[1] = 0ull;
          // the first half's weights, against the maximum so far, beside this turn's maximum
          weigh(0);
          const float top = largest(s) * a.scale2;
          const bool grew = top > m + GROWN || (m == -INFINITY && top > m);
          if (!__any_sync(FULL, grew)) break;
          // hardly ever: the maximum follows, what there is is scaled, and the turn begins anew
          const float mn = grew ? top : m;
          const float f = m == -INFINITY || !grew ? 1.f : exp2_fast(m - mn);
          l *= f;
          m = mn;
          if (x > 0 && __any_sync(FULL, f != 1.f)) {
#pragma unroll
            for (int c = 0; c < DP; c += 32) {
              float o[32];
              tc::tmem_ld32(oa + c, o);
#pragma unroll
              for (int y = 0; y < 32; ++y) o[y] *= f;
              tmem_st32_async(oa + c, reinterpret_cast<const uint32_t*>(o));
            }
          }
        }
        // values of a turn that not every row of the CTA sees, before the first product
        if (t == 0 && !(cnt == TM && j0 + TM - 1 <= i0 &&
                        (a.window == 0 || i0 + nt - 1 - j0 < a.window || j0 + TM <= a.sinks))) {
          ok = look_over<DP>(ctl, ring + (2 * x + 1) % NS * SLOT, (2 * x + 1) % NS,
                             ((2 * x + 1) / NS) & 1, r, r < cnt && j0 + r < n);
          if (!ok) break;
        }
        hand_over(0);
        weigh(64);
        hand_over(1);
        const float2 both = unpair(add2(sum[0], sum[1]));
        l += both.x + both.y;
      }
      if (ok && turns > 0) {
        ok = wait_for(&ctl->sfull[t], turns & 1, &ctl->abort);
        ok = __all_sync(FULL, ok);
        tc::fence_after_sync();
      }
      const int hq = h * a.G + g;
      const long long row = nr.off + t0 + t * tpt + tok;
      if (a.splits > 1) {
        const long long pr = part_row(a, split, b, t0 + t * tpt + tok) * a.H + hq;
        if (valid) a.ml[pr] = ok ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
        if (ok && turns > 0)
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            float o[32];
            tc::tmem_ld32(oa + c, o);
            if (valid)
#pragma unroll
              for (int y = 0; y < 32; y += 4)
                if (c + y < a.c.d)
                  *reinterpret_cast<float4*>(a.part + pr * a.c.d + c + y) =
                      make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
          }
      } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (valid && a.lse)
          a.lse[row * a.H + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        const long long mine_at = valid ? row * a.o_row + (long long)hq * a.o_head : -1;
        // 32 rows a warp through its part of the queries' tile, whole rows stored
        char* st = Qs + t * SLOT + (warp & 3) * 32 * DP * 2;
        {
          float o[DP];
          if (ok && turns > 0) {
            if constexpr (DP == 128) {
              tmem_ld128(oa, o);
            } else {
              tc::tmem_ld32(oa, o);
              tc::tmem_ld32(oa + 32, o + 32);
            }
          } else {
#pragma unroll
            for (int y = 0; y < DP; ++y) o[y] = 0.f;
          }
#pragma unroll
          for (int y = 0; y < DP; y += 8) {
            const int pc = y / 8;
            *reinterpret_cast<int4*>(st + lane * DP * 2 + ((pc ^ (lane & 7)) * 16)) = make_int4(
                pack2(o[y] * inv, o[y + 1] * inv), pack2(o[y + 2] * inv, o[y + 3] * inv),
                pack2(o[y + 4] * inv, o[y + 5] * inv), pack2(o[y + 6] * inv, o[y + 7] * inv));
          }
        }
        __syncwarp();
        constexpr int PC = DP / 8, RPI = 32 / PC;
        const int pc = lane % PC;
#pragma unroll 8
        for (int y0 = 0; y0 < 32; y0 += RPI) {
          const int y = y0 + lane / PC;
          // the row's place in the output, from the thread that holds it
          const long long at = __shfl_sync(FULL, mine_at, y);
          if (at >= 0 && pc * 8 < a.c.d)
            *reinterpret_cast<int4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at + pc * 8) =
                *reinterpret_cast<const int4*>(st + y * DP * 2 + ((pc ^ (y & 7)) * 16));
        }
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == ISSUE) tc::tmem_dealloc(tmem, 256 * TILES);
  if (ctl->abort) {
    if (tid == 0) set_status(a.c.status, GMC_STATUS_TIMEOUT);
    if (warp == COPY && issued > 0) {  // copies in flight land before shared memory is given back
      const long long end = clock64() + T_WAIT;
      while (!tc::mbar_try_wait(&ctl->qfull, 0) && clock64() < end) {}
      for (int q = issued > NS ? issued - NS : 0; q < issued; ++q)
        while (!tc::mbar_try_wait(&ctl->full[q % NS], (q / NS) & 1) && clock64() < end) {}
    }
    return;
  }
  if (ctl->strange) {
    for (int rr = warp; rr < nt * a.G; rr += THREADS / 32) {
      const int tk = rr / a.G, g = rr - tk * a.G, hq = h * a.G + g;
      const long long row = nr.off + t0 + tk;
      float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
      for (int x = 0; x < turns; ++x) {
        const int u = turn_at(x), f = tn.first(u);
        row_alone<__nv_bfloat16>(a, b, h, row, hq, i0 + tk, f, min(n, f + tn.rows(u)), &m, &l, o);
      }
      const int y = lane * 4;
      if (a.splits > 1) {
        const long long pr = part_row(a, split, b, t0 + tk) * a.H + hq;
        if (lane == 0) a.ml[pr] = make_float2(m, l);
        if (y < a.c.d)
          *reinterpret_cast<float4*>(a.part + pr * a.c.d + y) = make_float4(o[0], o[1], o[2], o[3]);
      } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (lane == 0 && a.lse)
          a.lse[row * a.H + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        if (y < a.c.d)
          for (int e = 0; e < 4; ++e)
            reinterpret_cast<__nv_bfloat16*>(
                a.out)[row * a.o_row + (long long)hq * a.o_head + y + e] =
                __float2bfloat16_rn(o[e] * inv);
      }
    }
  }
}

// [dims] of bf16 elements, 128-byte swizzle, box of 64 elements.
cudaError_t make_map(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims,
                     const cuuint64_t* strides, const cuuint32_t* box) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                             const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  Encode fn = reinterpret_cast<Encode>(tensor_map_encoder());
  if (!fn) return cudaErrorNotSupported;
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  const CUresult r =
      fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box,
         ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// CTAs without a split: at most this many tiles of `tiles` x (128 / G) tokens.
long long tc_ctas(const KV& c, int G, long long rows, int T, int tiles) {
  const int tokens = TM / G * tiles;
  const long long each = (long long)c.B * ceil_div(T, tokens);
  return c.Hkv * std::min(each, rows / tokens + c.B);
}
// One tile a CTA and two CTAs an SM where the key axis is short and the CTAs are more than
// a wave: one's first copies and last stores (3 us each) hide behind the other's products
// (32 questions of 16 to 256 tokens on up to 513 keys: two tiles 52.8 us, one 49.2; 8 x
// 512 tokens on 2,048: 118 and 111); on longer axes two tiles share each key's copy
// (4,096 tokens: 110 and 119; 1,024 tokens, less than a wave: 20.5 and 21.3).
int tc_tiles(const AttnArgs& a) {
  long long most = a.c.cap;
  if (a.window > 0) most = std::min(most, (long long)a.window + a.sinks + a.T);
  return most <= 18 * TM && tc_ctas(a.c, a.G, a.rows, a.T, 2) > sm_count() ? 1 : 2;
}
}  // namespace

// Parts of the key axis where the tiles leave SMs idle: up to as many as fill them, two
// turns each at least.  2 x 256 tokens on 513 keys: 21.4 us in two parts, 13.6 in one; 20
// tokens on 700 keys: 13.5 in two, 15.1 in one.
int attend_tc_splits(const KV& c, int G, int T) {
  const long long rows = (long long)c.B * T, ctas = tc_ctas(c, G, rows, T, 1);
  const long long fill = 2LL * sm_count();
  if (ctas >= fill / 2) return 1;
  return cheapest_parts(std::min<long long>({fill / ctas, 32, c.cap / (2 * TM)}),
                        ceil_div(c.cap, TM), 1.6f, rows * G * c.Hkv * c.d);
}

bool attend_tc_takes(const KV& c, int dtype, int G) {
  // whole swizzle atoms of 8 slots a page; strides that a tensor map can hold
  auto fits = [](long long s, int n) { return n == 1 || (s > 0 && s * 2 < (1LL << 40)); };
  return dtype == GMC_BF16 && c.d <= 128 && G <= TM && c.ps % 8 == 0 &&
         fits(c.page_stride, c.num_pages) && fits(c.head_stride, c.Hkv) &&
         fits(c.slot_stride, c.ps);
}

namespace {
template <int DP, int TILES>
cudaError_t tc_launch(const AttnArgs& a, const CUtensorMap& qm, const CUtensorMap& km,
                      const CUtensorMap& vm, cudaStream_t st) {
  constexpr size_t smem = t_smem<DP, TILES>();
  const cudaError_t e = set_smem_limit((const void*)k_attend_tc<DP, TILES>, smem);
  if (e != cudaSuccess) return e;
  const long long tiles = tc_ctas(a.c, a.G, a.rows, a.T, TILES) / a.c.Hkv;
  return launch_k(k_attend_tc<DP, TILES>, dim3((unsigned)(tiles * a.splits), a.c.Hkv),
                  dim3(t_threads<TILES>()), smem, st, 1, qm, km, vm, a,
                  make_turns(a.c.ps, a.G, TILES));
}
}  // namespace

cudaError_t launch_attend_tc(const AttnArgs& a, cudaStream_t st) {
  const int tpt = TM / a.G;
  CUtensorMap qm, km, vm;
  auto stride = [&](long long s, int n) {
    return n == 1 ? (cuuint64_t)a.c.d * 2 : (cuuint64_t)s * 2;
  };
  cudaError_t e;
  {
    const cuuint64_t dims[3] = {(cuuint64_t)a.c.d, (cuuint64_t)a.H, (cuuint64_t)a.rows};
    const cuuint64_t strides[2] = {stride(a.q_head, a.H), stride(a.q_row, a.rows)};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.G, (cuuint32_t)tpt};
    if ((e = make_map(&qm, a.q, 3, dims, strides, box)) != cudaSuccess) return e;
  }
  {
    const cuuint64_t dims[4] = {(cuuint64_t)a.c.d, (cuuint64_t)a.c.ps, (cuuint64_t)a.c.Hkv,
                                (cuuint64_t)a.c.num_pages};
    const cuuint64_t strides[3] = {stride(a.c.slot_stride, a.c.ps),
                                   stride(a.c.head_stride, a.c.Hkv),
                                   stride(a.c.page_stride, a.c.num_pages)};
    const cuuint32_t box[4] = {64, (cuuint32_t)std::min(a.c.ps, TM), 1, 1};
    if ((e = make_map(&km, a.c.k, 4, dims, strides, box)) != cudaSuccess) return e;
    if ((e = make_map(&vm, a.c.v, 4, dims, strides, box)) != cudaSuccess) return e;
  }
  const bool one = a.splits > 1 || tc_tiles(a) == 1;
  if (a.c.d <= 64)
    return one ? tc_launch<64, 1>(a, qm, km, vm, st) : tc_launch<64, 2>(a, qm, km, vm, st);
  return one ? tc_launch<128, 1>(a, qm, km, vm, st) : tc_launch<128, 2>(a, qm, km, vm, st);
}

}  // namespace gmc
