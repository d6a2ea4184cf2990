"""From image tokens to the first generated tokens of one attention layer.

    python examples/kept_tokens_prefill.py [--images 4] [--keep 192] [--tokens 8]

Every image's 576 tokens are reduced to --keep (tr_reduce), projected
(tr_project) and enter one layer of a language model with the image's place
in the sequence as their first position axis and their rows and columns of the
24 x 24 grid as the other two: queries and keys are normed and rotated, keys
and values appended to a paged cache, and the prompt attends over it.  Then
each request generates --tokens tokens, one at a time, as a captured CUDA
graph whose lengths and positions advance on the device.  Random weights;
prints what each part took and checks the last step against a plain
computation.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_13500_gb300 as altr  # noqa: E402
import synth  # noqa: E402

HQ, HK, D, PAGE, GRID = 28, 4, 128, 16, 24


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--images", type=int, default=4)
    ap.add_argument("--keep", type=int, default=192)
    ap.add_argument("--tokens", type=int, default=8)
    a = ap.parse_args()
    dev, bf = torch.device("cuda", 0), torch.bfloat16
    torch.manual_seed(0)
    w = synth.make("llava576", seed=1, device=dev, batch=a.images, d=1024)
    width = HQ * D
    rnd = lambda *s: (torch.randn(*s, device=dev) / math.sqrt(s[-1])).to(bf)
    w_proj, w_qkv = rnd(width, 1024), rnd((HQ + 2 * HK) * D, width)
    q_weight, k_weight = torch.ones(D, device=dev), torch.ones(D, device=dev)
    rotary = altr.Rotary(D, dev, base=1e6, sections=(16, 24, 24))
    total = a.keep + a.tokens
    per = (total + PAGE - 1) // PAGE
    cache = altr.PagedCache.empty(a.images * per, HK, PAGE, D, device=dev)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    table = torch.randperm(a.images * per, device=dev).to(torch.int32).reshape(a.images, per)

    def layer(x, pos, lens, cu, max_new, max_len, out=None):
        """One attention layer's new rows x [T, width]; ends at the heads' output [T, HQ, D]."""
        rows = (x @ w_qkv.T).view(-1, HQ + 2 * HK, D)
        q = cache.append(rows[:, HQ:HQ + HK], rows[:, HQ + HK:], table, lens, cu, rotary=rotary, pos=pos,
                         k_weight=k_weight, q=rows[:, :HQ], q_weight=q_weight)
        return cache.attend(q, table, lens, cu, max_new=max_new, max_len=max_len, out=out), q

    def prefill():
        r = altr.reduce(w.x, w.x_pre, w.x_post, k=a.keep, seqlens=w.seqlens)
        z, err = altr.project(r.y, w_proj)
        # a kept token's axes: the image's start, its row and its column (the image starts at 0)
        pos = torch.stack([torch.zeros_like(r.idx), r.idx // GRID, r.idx % GRID]).to(torch.int32).contiguous()
        cu = i32([a.keep * b for b in range(a.images + 1)])
        return layer(z, pos, i32([a.keep] * a.images), cu, a.keep, a.keep)[0]

    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    prefill()
    begin.record()
    o = prefill()
    end.record()
    end.synchronize()
    print(f"{a.images} images of 576 tokens, {a.keep} kept: reduced, projected, appended and attended in "
          f"{begin.elapsed_time(end) * 1e3:.0f} us")

    # single tokens: the same step captured once, its lengths and positions advanced in place
    x = rnd(a.images, width)
    lens, pos = i32([a.keep] * a.images), torch.full((3, a.images), GRID - 1, dtype=torch.int32, device=dev)
    cu = i32(list(range(a.images + 1)))
    out = torch.empty(a.images, HQ, D, dtype=bf, device=dev)

    def step():
        lens.add_(1)
        pos.add_(1)
        return layer(x, pos, lens, cu, 1, total, out)

    step()  # outside the capture first: the kernels' shared-memory limit
    lens.sub_(1)
    pos.sub_(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, q = step()
    begin.record()
    for _ in range(a.tokens):
        graph.replay()
    end.record()
    end.synchronize()
    print(f"{a.tokens} generated tokens per image, one layer: {begin.elapsed_time(end) / a.tokens * 1e3:.1f} us a token")

    assert int(cache.error) == 0
    for b in range(a.images):
        k = cache.k[table[b].long()].transpose(1, 2).reshape(-1, HK, D)[:total].double()
        v = cache.v[table[b].long()].transpose(1, 2).reshape(-1, HK, D)[:total].double()
        for h in range(HQ):
            p = torch.softmax(k[:, h // (HQ // HK)] @ q[b, h].double() / math.sqrt(D), 0)
            ref = p @ v[:, h // (HQ // HK)]
            assert (out[b, h].double() - ref).abs().max() <= 2 ** -7 * (p @ v[:, h // (HQ // HK)].abs()).max() + 1e-6
    print("the last token's heads match a plain computation in 64 bits")


if __name__ == "__main__":
    main()
