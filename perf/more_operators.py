"""The paged cache held in 8 bits: appending keys and values (e4m3 codes, a
power-of-two scale for each 16 keys of a head), attention of new tokens over
it, and the block tables that both go by, kept on the GPU from what each
request brings and gives back.  Cases, inputs, plain forms and 64-bit values."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
DEV = "cuda"
EPS = 1e-6
BLOCK = 16              # keys that share a scale
LEAST, MOST = -117, 119  # exponents of a scale


# ------------------------------------------------------------------ cases
def _append(name, batch, new_lo, new_hi, past_lo, past_hi, hq, hk, d, page, axes, norm, dtype="bf16", layout="half"):
    return {"name": name, "op": "append", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo,
            "past_hi": past_hi, "hq": hq, "hk": hk, "d": d, "page": page, "axes": axes, "norm": norm, "dtype": dtype,
            "layout": layout}


def _attend(name, batch, new_lo, new_hi, past_lo, past_hi, hq, hk, d, page, dtype="bf16", causal=True, window=0,
            lse=False):
    return {"name": name, "op": "attend", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo,
            "past_hi": past_hi, "hq": hq, "hk": hk, "d": d, "page": page, "dtype": dtype, "causal": causal,
            "window": window, "lse": lse}


def _tables(name, batch, new_lo, new_hi, past_lo, past_hi, page, back):
    return {"name": name, "op": "tables", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo,
            "past_hi": past_hi, "page": page, "back": back}


def listed():
    return [
        # one generated token of 64 requests: its block of 16 keys is there already and may need a larger scale
        _append("append_tokens", 64, 1, 1, 256, 16384, 28, 4, 128, 16, 3, False),
        # the kept ninth of 32 dynamic-resolution images (256..16384 tokens) entering an empty cache, normed heads
        _append("append_prompts", 32, 29, 1820, 0, 0, 28, 4, 128, 64, 3, True),
        # odd chunks after odd pasts, half precision, 64-wide heads, neighbouring channels paired
        _append("append_chunks", 9, 61, 333, 7, 5001, 16, 16, 64, 32, 1, False, dtype="fp16", layout="pairs"),
        # one generated token after 576 visual and 35 text tokens, 32 heads: latency
        _attend("attend_token", 1, 1, 1, 610, 610, 32, 32, 128, 16),
        # one generated token of 64 requests with ragged histories: the codes once from memory
        _attend("attend_tokens", 64, 1, 1, 255, 16383, 28, 4, 128, 64),
        # a token and four drafts of 32 requests: 35 query rows on every key
        _attend("attend_drafts", 32, 5, 5, 1000, 12000, 28, 4, 128, 32),
        # a clip's 784 kept tokens as a chunk over what the cache holds already, half precision
        _attend("attend_clips", 4, 784, 784, 216, 5488, 28, 4, 128, 128, dtype="fp16"),
        # a 2048-token chunk of a long prompt
        _attend("attend_long", 1, 2048, 2048, 30720, 30720, 28, 4, 128, 64),
        # short ragged chunks over long histories, sliding window, 64-wide heads, statistics returned
        _attend("attend_window", 3, 17, 129, 9001, 30011, 16, 16, 64, 32, dtype="fp16", window=4096, lse=True),
        # one request's next token: latency
        _tables("tables_token", 1, 1, 1, 610, 610, 16, 0),
        # a token and up to four drafts of 256 requests, up to four of the last step's tokens refused
        _tables("tables_drafts", 256, 1, 5, 255, 16383, 16, 4),
        # chunks of 2000 prompts, what a step before them had reserved given back
        _tables("tables_prompts", 2000, 3, 131, 1, 2047, 64, 300),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["append", "attend", "attend", "tables"])
        hk = rng.choice([1, 2, 4, 8, 16, 32])
        hq = hk * rng.choice([g for g in (1, 2, 4, 5, 7, 8) if g * hk <= 40])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        page = rng.choice([16, 32, 64, 128])
        if op == "append":
            lo, past = _log(rng, 1, 1024), _log(rng, 1, 8192) - 1
            c = _append("", _log(rng, 1, 96), lo, lo * rng.choice([1, 2]), past, past * 2, hq, hk,
                        rng.choice([64, 80, 128]), page, rng.choice([1, 3]), rng.random() < 0.5, dtype,
                        rng.choice(["half", "pairs"]))
        elif op == "attend":
            lo, past = rng.choice([1, _log(rng, 1, 2048)]), _log(rng, 1, 20000) - 1
            c = _attend("", _log(rng, 1, 64), lo, lo * rng.choice([1, 1, 3]), past, past * rng.choice([1, 4]), hq, hk,
                        rng.choice([64, 96, 128]), page, dtype, rng.random() < 0.85,
                        rng.choice([0, 0, 0, _log(rng, 16, 8192)]), rng.random() < 0.3)
        else:
            lo, past = _log(rng, 1, 100), _log(rng, 1, 8192) - 1
            c = _tables("", _log(rng, 1, 3000), lo, lo * rng.choice([1, 3]), past, past * rng.choice([1, 2]), page,
                        rng.choice([0, _log(rng, 1, 500)]))
        del c["name"]
        if _cost(c) <= top and _room(c) <= 12e9:
            return c


def _sizes(case):
    """(new, past) tokens of each sequence: spread over the case's ranges, the same for every seed."""
    pairs = []
    for b in range(case["batch"]):
        u, v = (0.5 + 0.6180339887 * b) % 1.0, (0.25 + 0.7548776662 * b) % 1.0
        new = case["new_lo"] + round((case["new_hi"] - case["new_lo"]) * u)
        lo, hi = case["past_lo"] + 1, case["past_hi"] + 1
        pairs.append((new, round(lo * (hi / lo) ** v) - 1))
    return pairs


def _back(case):
    """Tokens that each sequence holds beyond its past before a pass."""
    return [(7 * b + 3) % (case["back"] + 1) for b in range(case["batch"])]


def _blocks(n, size):
    return (n + size - 1) // size


def _room(case):
    """Bytes of the plain form's padded scores (attend), of its rows in 64 bits (append), of its table."""
    pairs = _sizes(case)
    longest = max(n + p for n, p in pairs)
    if case["op"] == "tables":
        return 8.0 * case["batch"] * longest / case["page"]
    if case["op"] == "append":
        return 8.0 * sum(n + p for n, p in pairs) * (case["hq"] + 2 * case["hk"]) * case["d"]
    return 4.0 * case["batch"] * max(max(n for n, _ in pairs) * case["hq"], 2 * case["hk"] * case["d"]) * longest


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.8e12, w["flops"] / 1.9e15)


def work(case):
    pairs = _sizes(case)
    new = sum(n for n, _ in pairs)
    if case["op"] == "tables":
        # a length read and written, a count and a prefix; three numbers of each row; each page's id read and written
        page, moved = case["page"], 0
        for (n, p), back in zip(pairs, _back(case)):
            moved += _blocks(p + back, page) - _blocks(p, page) + _blocks(p + n, page) - _blocks(p, page)
        return {"bytes": 4 * (5 * case["batch"] + 3 * new + 2 * moved), "flops": 0}
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if case["op"] == "append":
        # rows in, queries and codes out; the first block of a sequence read and written again where it has older keys
        older = sum(p % BLOCK for _, p in pairs)
        scales = sum(_blocks(n + p, BLOCK) - p // BLOCK for n, p in pairs)
        return {"bytes": new * (4 * hq + 6 * hk) * d + 4 * older * hk * d + 2 * scales * hk + 4 * case["axes"] * new,
                "flops": new * (hq + hk) * (3 * d + (4 * d if case["norm"] else 0)) + 4 * new * hk * d}
    w = case["window"]
    seen = keys = 0
    for n, p in pairs:
        for i in range(n):
            last = p + i + 1 if case["causal"] else p + n
            first = max(0, p + i + 1 - w) if w else 0
            seen += last - first
        keys += p + n - (max(0, p + 1 - w) if w else 0)
    return {"bytes": 4 * new * hq * d + 2 * keys * hk * (d + 1.0 / BLOCK) + (4 * new * hq if case["lse"] else 0),
            "flops": 4 * d * hq * seen}


# ------------------------------------------------------------------ inputs
BASE = 1e6
MAX_POS = 1 << 16


def _axis_of(case):
    """The axis of each frequency: contiguous sections, the first axis taking what the others leave."""
    half, axes = case["d"] // 2, case["axes"]
    rest = half * 3 // 8 if axes == 3 else 0
    return [0] * (half - rest * (axes - 1)) + [a for a in range(1, axes) for _ in range(rest)]


def _positions(tokens, axes, g):
    """Kept tokens of frames of 14 x 14 patches: every first to fourth cell stays; one axis: text order."""
    offset = int(torch.randint(0, 30000, (1,), generator=g, device=DEV).item())
    if axes == 1:
        return (offset + torch.arange(tokens, device=DEV, dtype=torch.int32)).reshape(1, -1)
    cell = torch.cumsum(torch.randint(1, 5, (tokens,), generator=g, device=DEV), 0) % (196 * 2048)
    return (offset + torch.stack([cell // 196, (cell % 196) // 14, cell % 14])).to(torch.int32).contiguous()


def _randn(g, dtype, *shape, gain=1.0):
    return (gain * torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)).to(dtype)


def _held(g, pages, hk, page, d, gain):
    """A cache's codes and scales: normal values, their size another one in every block and head."""
    blocks = page // BLOCK
    x = torch.randn(pages, hk, blocks, BLOCK * d, generator=g, device=DEV)
    x.mul_(gain * torch.exp2(torch.randn(pages, hk, blocks, 1, generator=g, device=DEV)))
    part, power = torch.frexp(x.abs().amax(-1) / 448)
    power = power - (part == 0.5).int()
    codes = x.mul_(torch.exp2(-power.float())[..., None]).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return codes.reshape(pages, hk, page, d), (power + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _pages_of(lens, per, page, pages, g):
    """Every sequence's pages, drawn from all of them, and the pages left over."""
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    count = _blocks(torch.tensor(lens, device=DEV), page)
    here = torch.arange(per, device=DEV) < count[:, None]
    table = torch.full((len(lens), per), -1, dtype=torch.int32, device=DEV)
    used = int(count.sum())
    table[here] = order[:used]
    return table, order[used:]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    pairs, page = _sizes(case), case["page"]
    new, past = [n for n, _ in pairs], [p for _, p in pairs]
    lens = [n + p for n, p in pairs]
    if case["op"] == "tables":
        held = [p + b for p, b in zip(past, _back(case))]
        per = max(max(_blocks(n, page) for n in held), max(_blocks(n, page) for n in lens)) + 1
        pages = sum(max(_blocks(a, page), _blocks(b, page)) for a, b in zip(held, lens)) + 5
        table, left = _pages_of(held, per, page, pages, g)
        free = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
        free[:len(left)] = left
        s |= {"new": i32(new), "rows": sum(new), "keep": i32(past), "table": table, "lens": i32(held), "free": free,
              "count": i32([len(left)])}
        if own:
            import paper_2607_13500_gb300 as altr
            t = altr.PageTable(case["batch"], per, pages, page, DEV)
            t.table.copy_(table), t.lens.copy_(s["lens"]), t.free.copy_(free), t.free_count.copy_(s["count"])
            s["pages"] = t
        return s
    dt, hq, hk, d = DTYPES[case["dtype"]], case["hq"], case["hk"], case["d"]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    pages = sum(_blocks(n, page) for n in lens) + 3
    table, _ = _pages_of(lens, max(_blocks(n, page) for n in lens), page, pages, g)
    seq = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), torch.tensor(new, device=DEV))
    s |= {"table": table, "lens": i32(lens), "cu": i32(cu), "max_new": max(new), "max_len": max(lens), "seq": seq}
    s["k_codes"], s["k_scale"] = _held(g, pages, hk, page, d, 1.5)
    s["v_codes"], s["v_scale"] = _held(g, pages, hk, page, d, 1.0)
    tokens = cu[-1]
    if case["op"] == "attend":
        s["q"] = _randn(g, dt, tokens, hq, d, gain=1.5)
    else:
        # queries, keys and values as the one projection of a layer leaves them
        rows = _randn(g, dt, tokens, hq + 2 * hk, d)
        s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        s["q_weight"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV) if case["norm"] else None
        s["k_weight"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV) if case["norm"] else None
        s["pos"] = _positions(tokens, case["axes"], g)
        axis = _axis_of(case)
        s["axis"] = torch.tensor(axis, device=DEV)
        # the table of cosines and sines that a plain program keeps
        freq = BASE ** (-torch.arange(len(axis), dtype=torch.float64, device=DEV) / len(axis))
        angle = torch.arange(MAX_POS, dtype=torch.float64, device=DEV)[:, None] * freq
        s["cos"], s["sin"] = torch.cos(angle), torch.sin(angle)
    if own:
        import paper_2607_13500_gb300 as altr
        s["cache"] = altr.PagedCache8(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"])
        if case["op"] == "append":
            s["rotary"] = altr.Rotary(d, DEV, base=BASE, layout=case["layout"],
                                      sections=[axis.count(a) for a in range(case["axes"])])
    return s


# ------------------------------------------------------------------ the framework's calls
def _run_own(s):
    c = s["case"]
    if c["op"] == "tables":
        t = s["pages"]
        t.truncate(s["keep"])
        step = t.extend(s["new"], s["rows"])
        return {"table": t.table, "lens": t.lens, "free": t.free, "count": t.free_count, "cu_new": step.cu_new,
                "slots": step.slots, "pos": step.pos, "seq": step.seq}
    if c["op"] == "append":
        h = s["cache"]
        q = h.append(s["k"], s["v"], s["table"], s["lens"], s["cu"], rotary=s["rotary"], pos=s["pos"],
                     k_weight=s["k_weight"], q=s["q"], q_weight=s["q_weight"], eps=EPS)
        return {"q": q, "k": h.k, "v": h.v, "k_scale": h.k_scale, "v_scale": h.v_scale}
    o = s["cache"].attend(s["q"], s["table"], s["lens"], s["cu"], causal=c["causal"], window=c["window"],
                          max_new=s["max_new"], max_len=s["max_len"], return_lse=c["lse"])
    return {"o": o[0], "lse": o[1]} if c["lse"] else {"o": o}


# ------------------------------------------------------------------ plain forms
def _turn(x, cos, sin, layout):
    """Pairs of channels turned; x [T, H, d], cos [T, d/2]."""
    half = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    if layout == "half":
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _forward(x, weight, s):
    """Normed and rotated, in 64 bits: keys lie next to the borders between two codes."""
    y = x.double()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight
    place = s["pos"].long()[s["axis"]].T
    at = torch.arange(len(s["axis"]), device=DEV)
    return _turn(y, s["cos"][place, at], s["sin"][place, at], s["case"]["layout"])


def _exponents(scale):
    return scale.view(torch.uint8).int() - 127


def _code(x):
    """The nearest code of a 64-bit value: over 32 bits with the last one telling of what was cut off."""
    f = x.clamp(-448, 448).float()
    f = torch.where(f.double().abs() > x.abs(), torch.nextafter(f, torch.zeros_like(f)), f)
    odd = f.view(torch.int32) | ((f.double() != x) & (x.abs() < 448)).int()
    return odd.view(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)


def _put(codes, scale, rows, s):
    """New rows [T, hk, d] into their blocks; codes [pages, hk, page, d], scale [pages, hk, blocks], in place."""
    pages, hk, page, d = codes.shape
    blocks = page // BLOCK
    key = torch.arange(len(s["seq"]), device=DEV) - s["cu"][s["seq"] + 1] + s["lens"][s["seq"]]
    home, slot = s["table"][s["seq"], key // page].long(), key % page
    block = home * blocks + slot // BLOCK
    # what the new rows of every block need, and whether it has new rows or older keys
    most = torch.zeros(pages * blocks, hk, dtype=torch.float64, device=DEV)
    most.scatter_reduce_(0, block[:, None].expand(-1, hk), rows.abs().amax(-1), "amax")
    part, power = torch.frexp(most)
    need = torch.where(most > 0, power - 9 + (part > 0.875).int(), LEAST).clamp(LEAST, MOST)
    touched = torch.zeros(pages * blocks, 1, dtype=torch.bool, device=DEV)
    touched[block] = True
    first = s["lens"] - s["cu"].diff()  # a sequence's first new key
    older = first % BLOCK
    at = torch.where(older > 0, s["table"][torch.arange(len(first), device=DEV), first // page].long() * blocks
                     + first % page // BLOCK, pages * blocks)
    shared = torch.zeros(pages * blocks + 1, 1, dtype=torch.bool, device=DEV)
    shared[at] = True
    shared = shared[:-1]
    before = _exponents(scale).transpose(1, 2).reshape(pages * blocks, hk)
    after = torch.where(touched, torch.where(shared, torch.maximum(need, before), need), before)
    # older keys of those blocks move to the new scale
    raw = codes.view(torch.uint8).view(pages, hk, blocks, BLOCK, d)
    at = at.clamp(max=pages * blocks - 1)
    held = raw[at // blocks, :, at % blocks].view(torch.float8_e4m3fn).double()  # [batch, hk, BLOCK, d]
    moved = _code(held * torch.exp2((before - after)[at].double())[..., None, None])
    keep = torch.arange(BLOCK, device=DEV) < older[:, None]
    b, i = torch.where(keep)
    raw[at[b] // blocks, :, at[b] % blocks, i] = moved[b, :, i]
    codes.view(torch.uint8)[home, :, slot] = _code(rows * torch.exp2(-after[block].double())[..., None])
    scale.view(torch.uint8).copy_((after + 127).to(torch.uint8).view(pages, blocks, hk).transpose(1, 2))


def _run_append(s):
    q = _forward(s["q"], s["q_weight"], s).to(s["q"].dtype)
    _put(s["k_codes"], s["k_scale"], _forward(s["k"], s["k_weight"], s), s)
    _put(s["v_codes"], s["v_scale"], s["v"].double(), s)
    return {"q": q, "k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _values(codes, scale, table, n):
    """The first n keys of every sequence, [batch, hk, n, d] in 32 bits."""
    batch, hk, d = len(table), codes.shape[1], codes.shape[3]
    x = codes.view(torch.uint8)[table].view(torch.float8_e4m3fn).float()  # [batch, per, hk, page, d]
    x = x.unflatten(3, (-1, BLOCK)).mul_(torch.exp2(_exponents(scale)[table].float())[..., None, None])
    return x.flatten(3, 4).transpose(1, 2).reshape(batch, hk, -1, d)[:, :, :n]


def _run_attend(s):
    c, q, table = s["case"], s["q"], s["table"].long().clamp(min=0)
    batch, hk, d, group = c["batch"], c["hk"], c["d"], c["hq"] // c["hk"]
    top, n = s["max_new"], s["max_len"]
    # padded: sequence b's new token i in row i, its key j in column j
    row = torch.arange(len(s["seq"]), device=DEV) - s["cu"][s["seq"]]
    qs = torch.zeros(batch, top, c["hq"], d, device=DEV)
    qs[s["seq"], row] = q.float()
    qs = qs.reshape(batch, top, hk, group, d).permute(0, 2, 3, 1, 4).reshape(batch, hk, group * top, d)
    here = (s["lens"] - s["cu"].diff())[:, None] + torch.arange(top, device=DEV)  # [batch, top]
    j = torch.arange(n, device=DEV)
    seen = (j < s["lens"][:, None, None]).expand(batch, top, n)
    if c["causal"]:
        seen = seen & (j <= here[..., None])
    if c["window"]:
        seen = seen & (j > here[..., None] - c["window"])
    keys = _values(s["k_codes"], s["k_scale"], table, n)
    score = (qs @ keys.transpose(-1, -2)).mul_(1 / math.sqrt(d)).reshape(batch, hk, group, top, n)
    del keys
    score.masked_fill_(~seen[:, None, None], float("-inf"))
    most = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(most).exp_()
    total = p.sum(-1, keepdim=True)
    vals = _values(s["v_codes"], s["v_scale"], table, n)
    o = (p.reshape(batch, hk, group * top, n) @ vals).reshape(batch, hk, group, top, d) / total.clamp(min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(batch, top, c["hq"], d)[s["seq"], row].to(q.dtype)
    if not c["lse"]:
        return {"o": o}
    lse = (most + total.log())[..., 0].permute(0, 3, 1, 2).reshape(batch, top, c["hq"])[s["seq"], row]
    return {"o": o, "lse": lse}


def _run_tables(s):
    table, lens, free, count, page = s["table"], s["lens"], s["free"], s["count"], s["case"]["page"]
    pages, per = len(free), table.shape[1]
    j = torch.arange(per, device=DEV)
    spare = lambda at, ok: torch.where(ok, at, pages)  # (a place behind the last takes what is not meant)
    wide = torch.cat([free, free.new_zeros(1)])
    # back: the pages behind what is kept, in the table's order, the last of them deepest
    keep = torch.minimum(lens, s["keep"].clamp(min=0))
    gone = (j >= _blocks(keep, page)[:, None]) & (j < _blocks(lens, page)[:, None])
    nth = gone.flatten().cumsum(0) - 1
    back = nth[-1] + 1
    wide[spare(count + back - 1 - nth, gone.flatten())] = table.flatten()
    table.masked_fill_(gone, -1)
    have = count + back
    # on: every sequence's new pages, the topmost first
    grown = keep + s["new"]
    more = (j >= _blocks(keep, page)[:, None]) & (j < _blocks(grown, page)[:, None])
    nth = more.flatten().cumsum(0) - 1
    got = wide[spare(have - 1 - nth, more.flatten())].reshape(table.shape)
    table.copy_(torch.where(more, got, table))
    free.copy_(wide[:-1])
    count.copy_((have - nth[-1] - 1).int())
    lens.copy_(grown)
    cu = torch.cat([lens.new_zeros(1), s["new"].cumsum(0).int()])
    seq = torch.searchsorted(cu, torch.arange(s["rows"], device=DEV, dtype=torch.int32), right=True) - 1
    pos = keep[seq] + torch.arange(s["rows"], device=DEV) - cu[seq]
    slots = table[seq, pos // page] * page + pos % page
    return {"table": table, "lens": lens, "free": free, "count": count, "cu_new": cu, "slots": slots.int(),
            "pos": pos.int(), "seq": seq.int()}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _run_append, "attend": _run_attend, "tables": _run_tables}[state["case"]["op"]](state)


# ------------------------------------------------------------------ 64 bits
def _exact_forward(x, weight, case, pos):
    x, half = x.double(), case["d"] // 2
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    axis = torch.tensor(_axis_of(case), device=DEV)
    freq = torch.tensor([BASE ** (-i / half) for i in range(half)], dtype=torch.float64, device=DEV)
    theta = pos[axis].double().T * freq
    phase = torch.complex(torch.cos(theta), torch.sin(theta))[:, None]
    if case["layout"] == "half":
        z = torch.complex(x[..., :half], x[..., half:]) * phase
        return torch.cat([z.real, z.imag], -1)
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], half, 2).contiguous()) * phase
    return torch.view_as_real(z).flatten(-2)


def _e4m3(x):
    """The nearest value of sign, four bits of exponent and three of mantissa (ties to even), 448 at most."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_put(held, power, rows, table, past):
    """A sequence's new rows [n, hk, d], block by block; held and power (64-bit) are changed."""
    page = held.shape[2]
    n = len(rows)
    at = past
    while at < past + n:
        end = min(past + n, (at // BLOCK + 1) * BLOCK)
        home, slot, old = int(table[at // page]), at % page, at % BLOCK
        block = slot // BLOCK
        x = rows[at - past:end - past].transpose(0, 1)  # [hk, keys, d]
        top = x.abs().flatten(1).amax(-1)
        want = torch.ceil(torch.log2(top / 448))
        want = torch.where(top > 448 * torch.exp2(want), want + 1, want)
        want = torch.where(top <= 224 * torch.exp2(want), want - 1, want).clamp(LEAST, MOST)
        if old:
            want = torch.maximum(want, power[home, :, block])
            shift = torch.exp2(power[home, :, block] - want)
            sl = slice(slot - old, slot)
            held[home, :, sl] = _e4m3(held[home, :, sl] * shift[:, None, None])
        power[home, :, block] = want
        held[home, :, slot:slot + end - at] = _e4m3(x / torch.exp2(want)[:, None, None])
        at = end


def _exact_append(s):
    c = s["case"]
    k, v = s["k_codes"].double(), s["v_codes"].double()
    kp, vp = (torch.log2(s[x].double()).round() for x in ("k_scale", "v_scale"))
    rows = _exact_forward(s["k"], s["k_weight"], c, s["pos"])
    table, t = s["table"].cpu(), 0
    for b, (n, past) in enumerate(_sizes(c)):
        _exact_put(k, kp, rows[t:t + n], table[b], past)
        _exact_put(v, vp, s["v"][t:t + n].double(), table[b], past)
        t += n
    return {"q": _exact_forward(s["q"], s["q_weight"], c, s["pos"]), "k": k, "v": v, "k_scale": torch.exp2(kp),
            "v_scale": torch.exp2(vp)}


def _exact_attend(s):
    c = s["case"]
    d, group, page = c["d"], c["hq"] // c["hk"], c["page"]
    out, stat = [], []
    for b, (n, past) in enumerate(_sizes(c)):
        length = n + past
        home = s["table"][b, :_blocks(length, page)].long()
        first = int(s["cu"][b])
        j = torch.arange(length, device=DEV)
        i = past + torch.arange(n, device=DEV)[:, None]
        hidden = torch.zeros(n, length, dtype=torch.bool, device=DEV)
        if c["causal"]:
            hidden |= j > i
        if c["window"]:
            hidden |= j <= i - c["window"]
        heads, stats = [], []
        for h in range(c["hq"]):
            if h % group == 0:
                k, v = (s[x + "_codes"].view(torch.uint8)[home, h // group].view(torch.float8_e4m3fn).double().reshape(-1, BLOCK * d)
                        * s[x + "_scale"].view(torch.uint8)[home, h // group].view(torch.float8_e8m0fnu).double().reshape(-1, 1)
                        for x in "kv")
                k, v = k.reshape(-1, d)[:length], v.reshape(-1, d)[:length]
            x = (s["q"][first:first + n, h].double() @ k.T / math.sqrt(d)).masked_fill_(hidden, float("-inf"))
            z = torch.logsumexp(x, -1)
            heads.append(x.sub_(z[:, None]).exp_() @ v)
            stats.append(z)
        out.append(torch.stack(heads, 1))
        stat.append(torch.stack(stats, 1))
    return {"o": torch.cat(out), "lse": torch.cat(stat)} if c["lse"] else {"o": torch.cat(out)}


def exact(case, seed):
    if case["op"] == "tables":  # whole numbers
        return None
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)


if __name__ == "__main__":
    for n, c in enumerate(listed() + [draw(random.Random(i)) for i in range(8)]):
        w = work(c)
        print(f"{c.get('name', 'drawn %d' % n):20s} {w['bytes'] / 1e6:10.3f} MB {w['flops'] / 1e9:10.3f} GFLOP "
              f"{1e6 * _cost(c):8.1f} us  room {_room(c) / 1e9:.2f} GB")
