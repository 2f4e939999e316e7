"""A compressed prompt goes on: cache, question, decoding, eviction.

One layer of a Qwen2.5-VL-shaped model after the boundary, with random states in place
of its weights (the calls are those of a real layer; only the projections are made up):

1. ``Compressor.run`` compresses B prompts of 36 x 36 visual tokens to K carriers each;
2. ``cache_append`` puts the compacted keys and values (``out_kv``) into a paged cache;
3. the tokens of a second question are appended and attend over the cache (``attend``);
4. tokens are decoded one after another (``decode``: appended, attended and every key's
   weight added to its running score);
5. whenever a sequence would outgrow its pages, ``evict`` keeps the rows that gathered the
   most attention, and decoding goes on from the smaller cache.

With ``--four-bits`` the cache holds 4 bits a value, and question and decoded tokens come as a
projection's output: queries and keys are turned by their (t, h, w) positions on the way
(``cache_append_rope``), then attended or decoded.

Run:  python examples/decode_after_compression.py [--four-bits]
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_02134_gb300 import gmc, workloads  # noqa: E402


def fresh_cache(B, Hkv, d, page, places, dtype, status):
    """An empty cache with room for `places` tokens a sequence."""
    per = -(-places // page)
    k = torch.zeros(B * per, Hkv, page, d, dtype=dtype, device="cuda")
    table = torch.randperm(B * per, device="cuda").to(torch.int32).reshape(B, per).contiguous()
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    return gmc.KVCache(k, torch.zeros_like(k), table, lens, status=status)


def fresh_cache4(B, Hkv, d, page, places, status):
    """The same with pages of 4 bits a value."""
    per = -(-places // page)
    k = torch.zeros(B * per, Hkv, gmc.cache4_part_size(page, d), dtype=torch.uint8, device="cuda")
    table = torch.randperm(B * per, device="cuda").to(torch.int32).reshape(B, per).contiguous()
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    return gmc.KVCache4(k, torch.zeros_like(k), table, lens, page, d, status=status)


def rotation(positions, d, base=1e6):
    """cos and sin of the pairs' angles at every position, from 64 bits; a quarter of the pairs
    turns by t, three eighths each by h and w."""
    n = d // 2
    rate = base ** (-torch.arange(n, dtype=torch.float64) / n)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * rate
    table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
    return gmc.Rope(table, sections=(n // 4, 3 * n // 8, 3 * n // 8))


def main(prompts=2, question=24, steps=60, places=384, keep=300, page=16, seed=0, verbose=True,
         four_bits=False):
    torch.manual_seed(seed)
    wl = workloads.make("qwen", B=prompts)
    arr = wl.abi_arrays()
    dev = {}
    for n, v in arr.items():
        if n != "text_offsets":
            t = torch.from_numpy(v)
            dev[n] = (t.view(torch.int16).view(torch.bfloat16) if v.dtype.name == "uint16"
                      else t).cuda()
    comp = gmc.Compressor(wl.B, wl.gh, wl.gw, wl.T_max, wl.H, wl.Hkv, wl.d, wl.D, wl.K,
                          gmc.GMC_BF16)
    out = comp.run(dev["hidden"], dev["keys"], dev["queries"], dev["pos_ids"], dev["vo_probe"])
    B, H, Hkv, d, rows = wl.B, wl.H, wl.Hkv, wl.d, out.K + wl.T_max

    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def fresh():
        if four_bits:
            return fresh_cache4(B, Hkv, d, page, places, status)
        return fresh_cache(B, Hkv, d, page, places, torch.bfloat16, status)

    cache = fresh()
    # the compressed prompt: every sequence's K carriers and its text
    cache.lens += rows
    gmc.cache_append(cache, out.kv, None, rows)

    def states(n, heads):
        return torch.randn(n, heads, d, device="cuda").to(torch.bfloat16)

    # a second question: appended, then attended over everything before it
    cache.lens += question
    answer = torch.empty(B * question, H, d, dtype=torch.bfloat16, device="cuda")
    if four_bits:
        # text positions go on behind the largest one of the prompt, (p, p, p) each
        last = out.pos.reshape(B, -1).amax(1)
        rope = rotation(int(last.max()) + 1 + question + steps, d)

        def positions(first, n):
            p = (last[:, None] + 1 + first + torch.arange(n, device="cuda")).to(torch.int32)
            return p[:, None].expand(B, 3, n).reshape(-1).contiguous()

        def turned(n, first):
            x = states(B * n, H + 2 * Hkv)  # a projection's output
            q = torch.empty(B * n, H, d, dtype=torch.bfloat16, device="cuda")
            gmc.cache_append_rope(cache, rope, x[:, H:H + Hkv], x[:, H + Hkv:], n,
                                  positions(first, n), x[:, :H], q)
            return q

        q = turned(question, 0)
    else:
        gmc.cache_append(cache, states(B * question, Hkv), states(B * question, Hkv), question)
        q = states(B * question, H)
    gmc.attend(cache, q, answer, question)

    # decoding; the scores start from the weights of the decoded tokens alone
    scores = torch.zeros(B, Hkv, places, device="cuda")
    token = torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda")
    workspace = gmc.alloc_workspace(gmc.decode_workspace_size(cache, H))
    length, evictions = rows + question, 0
    for step in range(steps):
        if length == places:
            kept = fresh()
            idx = torch.empty(B, Hkv, keep, dtype=torch.int32, device="cuda")
            best = torch.empty(B, Hkv, keep, device="cuda")
            gmc.evict(cache, kept, scores, keep, idx, best, sinks=4, recent=64)
            scores.zero_()
            scores[..., :keep] = best
            cache, length, evictions = kept, keep, evictions + 1
        cache.lens += 1
        length += 1
        if four_bits:
            gmc.decode(cache, turned(1, question + step), token, scores=scores, out_scores=scores,
                       workspace=workspace)
        else:
            gmc.decode(cache, states(B, H), token, k_new=states(B, Hkv), v_new=states(B, Hkv),
                       scores=scores, out_scores=scores, workspace=workspace)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and comp.status() == 0
    assert bool(torch.isfinite(answer.float()).all()) and bool(torch.isfinite(token.float()).all())
    if verbose:
        print(f"{B} prompts of {wl.N} visual tokens -> {out.K} carriers; {steps} tokens decoded, "
              f"{evictions} evictions, {length} tokens a sequence at the end")
    return {"length": length, "evictions": evictions, "scores": scores, "token": token}


if __name__ == "__main__":
    main(four_bits="--four-bits" in sys.argv[1:])
