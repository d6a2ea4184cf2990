"""The operators that take kept visual tokens through an attention layer of
the language model: rotary positions with several axes (with the norm of each
head), appending keys and values to a paged cache, attention of new tokens
over that cache.  Cases, inputs, plain forms and 64-bit values."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
DEV = "cuda"
EPS = 1e-6


# ------------------------------------------------------------------ cases
def _rotary(name, direction, tokens, hq, hk, d, axes, norm, dtype="bf16", layout="half", rot=0):
    return {"name": name, "op": "rotary", "direction": direction, "tokens": tokens, "hq": hq, "hk": hk, "d": d,
            "rot": rot or d, "axes": axes, "norm": norm, "dtype": dtype, "layout": layout}


def _append(name, batch, new_lo, new_hi, past_lo, past_hi, hq, hk, d, page, axes, norm, dtype="bf16", layout="half"):
    return {"name": name, "op": "append", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo,
            "past_hi": past_hi, "hq": hq, "hk": hk, "d": d, "rot": d, "page": page, "axes": axes, "norm": norm,
            "dtype": dtype, "layout": layout}


def _attend(name, batch, new_lo, new_hi, past_lo, past_hi, hq, hk, d, page, dtype="bf16", causal=True, window=0,
            lse=False):
    return {"name": name, "op": "attend", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo,
            "past_hi": past_hi, "hq": hq, "hk": hk, "d": d, "page": page, "dtype": dtype, "causal": causal,
            "window": window, "lse": lse}


def listed():
    return [
        # one generated token of one request, 28 query and 4 key heads (D = 3584): latency
        _rotary("rotary_token", "forward", 1, 28, 4, 128, 3, False),
        # the kept tokens of a llava576 batch (64 images x 192, D = 4096), text-style positions
        _rotary("rotary_llava", "forward", 12288, 32, 32, 128, 1, False),
        # the kept tokens of a video6272 batch (8 clips x 784), three axes, normed heads
        _rotary("rotary_video", "forward", 6272, 28, 4, 128, 3, True),
        # the same tokens in training: gradients of queries, keys and both norm weights
        _rotary("rotary_video_back", "backward", 6272, 28, 4, 128, 3, True),
        # one generated token of 64 requests: queries and keys rotated, K and V appended
        _append("append_tokens", 64, 1, 1, 256, 16384, 28, 4, 128, 16, 3, False),
        # the kept ninth of 32 dynamic-resolution images (256..16384 tokens) entering an empty cache
        _append("append_prompts", 32, 29, 1820, 0, 0, 28, 4, 128, 64, 3, True),
        # one generated token after 576 visual and 35 text tokens, 32 heads: latency
        _attend("attend_token", 1, 1, 1, 610, 610, 32, 32, 128, 16),
        # one generated token of 64 requests with ragged histories: K and V once from memory
        _attend("attend_tokens", 64, 1, 1, 255, 16383, 28, 4, 128, 64),
        # prompts of 192 kept and 35 text tokens, empty cache
        _attend("attend_prompts", 16, 227, 227, 0, 0, 32, 32, 128, 16),
        # a clip's 784 kept tokens as a chunk over what the cache holds already, half precision
        _attend("attend_clips", 4, 784, 784, 216, 5488, 28, 4, 128, 128, dtype="fp16"),
        # a 2048-token chunk of a long prompt
        _attend("attend_long", 1, 2048, 2048, 30720, 30720, 28, 4, 128, 64),
        # short ragged chunks over long histories, sliding window, 64-wide heads, statistics returned
        _attend("attend_window", 3, 17, 129, 9001, 30011, 16, 16, 64, 32, dtype="fp16", window=4096, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["rotary", "append", "attend", "attend"])
        hk = rng.choice([1, 2, 4, 8, 16, 32])
        hq = hk * rng.choice([g for g in (1, 2, 4, 5, 7, 8) if g * hk <= 40])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        if op == "rotary":
            d = rng.choice([64, 80, 96, 128, 256])
            c = _rotary("", rng.choice(["forward", "backward"]), _log(rng, 1, 20000), hq, hk, d, rng.choice([1, 2, 3]),
                        rng.random() < 0.5, rng.choice([dtype, "fp32"]), rng.choice(["half", "pairs"]),
                        rng.choice([d, d, d // 2]))
        elif op == "append":
            lo, past = _log(rng, 1, 1024), _log(rng, 1, 8192) - 1
            c = _append("", _log(rng, 1, 96), lo, lo * rng.choice([1, 2]), past, past * 2, hq, hk,
                        rng.choice([64, 128]), rng.choice([16, 32, 64, 128]), rng.choice([1, 3]), rng.random() < 0.5,
                        dtype, rng.choice(["half", "pairs"]))
        else:
            lo, past = rng.choice([1, _log(rng, 1, 2048)]), _log(rng, 1, 20000) - 1
            c = _attend("", _log(rng, 1, 64), lo, lo * rng.choice([1, 1, 3]), past, past * rng.choice([1, 4]), hq, hk,
                        rng.choice([64, 128]), rng.choice([16, 32, 64, 128]), dtype, rng.random() < 0.85,
                        rng.choice([0, 0, 0, _log(rng, 16, 8192)]), rng.random() < 0.3)
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


def _room(case):
    """Bytes of the plain form's padded scores (attend) or of its rows in 32 bits."""
    if case["op"] == "rotary":
        return 4.0 * case["tokens"] * (case["hq"] + case["hk"]) * case["d"]
    pairs = _sizes(case)
    if case["op"] == "append":
        return 4.0 * sum(n + p for n, p in pairs) * (case["hq"] + 2 * case["hk"]) * case["d"]
    longest = max(n + p for n, p in pairs)
    return 4.0 * case["batch"] * max(max(n for n, _ in pairs) * case["hq"], 2 * case["hk"] * case["d"]) * longest


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.8e12, w["flops"] / 1.9e15)


def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if case["op"] == "rotary":
        rows = case["tokens"] * (hq + hk)
        passes = 2 if case["direction"] == "forward" or not case["norm"] else 3
        return {"bytes": passes * rows * d * es + 4 * case["axes"] * case["tokens"],
                "flops": rows * (3 * case["rot"] + (4 * passes * d if case["norm"] else 0))}
    pairs = _sizes(case)
    new = sum(n for n, _ in pairs)
    if case["op"] == "append":
        return {"bytes": 2 * new * (hq + 2 * hk) * d * es + 4 * case["axes"] * new,
                "flops": new * (hq + hk) * (3 * case["rot"] + (4 * d if case["norm"] else 0))}
    w = case["window"]
    seen = keys = 0
    for n, p in pairs:
        for i in range(n):
            last = p + i + 1 if case["causal"] else p + n
            first = max(0, p + i + 1 - w) if w else 0
            seen += last - first
        keys += p + n - (max(0, p + 1 - w) if w else 0)
    return {"bytes": 2 * new * hq * d * es + 2 * keys * hk * d * es + (4 * new * hq if case["lse"] else 0),
            "flops": 4 * d * hq * seen}


# ------------------------------------------------------------------ inputs
BASE = 1e6
MAX_POS = 1 << 16


def _axis_of(case):
    """The axis of each frequency: contiguous sections, the first axis taking what the others leave."""
    half, axes = case["rot"] // 2, case["axes"]
    rest = half * 3 // 8 if axes == 3 else half // 2 if axes == 2 else 0
    return [0] * (half - rest * (axes - 1)) + [a for a in range(1, axes) for _ in range(rest)]


def _positions(tokens, axes, g):
    """Kept tokens of frames of 14 x 14 patches: every first to fourth cell stays; one axis: text order."""
    offset = int(torch.randint(0, 30000, (1,), generator=g, device=DEV).item())
    if axes == 1:
        return (offset + torch.arange(tokens, device=DEV, dtype=torch.int32)).reshape(1, -1)
    cell = torch.cumsum(torch.randint(1, 5, (tokens,), generator=g, device=DEV), 0) % (196 * 2048)
    place = [cell // 196, (cell % 196) // 14, cell % 14]
    return (offset + torch.stack(place[:axes] if axes == 3 else place[1:])).to(torch.int32).contiguous()


def _randn(g, dtype, *shape, gain=1.0):
    return (gain * torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, hq, hk, d = DTYPES[case["dtype"]], case["hq"], case["hk"], case["d"]
    s = {"case": case}
    if case["op"] != "rotary":
        pairs = _sizes(case)
        new = [n for n, _ in pairs]
        lens = [n + p for n, p in pairs]
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        page = case["page"]
        per = max((n + page - 1) // page for n in lens)
        used = sum((n + page - 1) // page for n in lens)
        pages = used + 3
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((case["batch"], per), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(lens):
            k = (n + page - 1) // page
            table[b, :k] = order[at:at + k]
            at += k
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
        seq = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), torch.tensor(new, device=DEV))
        s |= {"table": table, "lens": i32(lens), "cu": i32(cu), "max_new": max(new), "max_len": max(lens), "seq": seq,
              "k_cache": _randn(g, dt, pages, hk, page, d, gain=1.5), "v_cache": _randn(g, dt, pages, hk, page, d)}
        tokens = cu[-1]
    else:
        tokens = case["tokens"]
    if case["op"] == "attend":
        s["q"] = _randn(g, dt, tokens, hq, d, gain=1.5)
    else:
        # queries, keys (and values) as the one projection of a layer leaves them
        heads = hq + hk if case["op"] == "rotary" else hq + 2 * hk
        rows = _randn(g, dt, tokens, heads, d)
        s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        if case["op"] == "rotary" and case["direction"] == "backward":
            grads = _randn(g, dt, tokens, heads, d)
            s["dq"], s["dk"] = grads[:, :hq], grads[:, hq:]
        s["q_weight"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV) if case["norm"] else None
        s["k_weight"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV) if case["norm"] else None
        s["pos"] = _positions(tokens, case["axes"], g)
        axis = _axis_of(case)
        s["axis"] = torch.tensor(axis, device=DEV)
        # the table of cosines and sines that a plain program keeps (angles in 64 bits)
        freq = BASE ** (-torch.arange(len(axis), dtype=torch.float64, device=DEV) / len(axis))
        angle = torch.arange(MAX_POS, dtype=torch.float64, device=DEV)[:, None] * freq
        s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    if own:
        import paper_2607_13500_gb300 as altr
        if case["op"] != "attend":
            s["rotary"] = altr.Rotary(d, DEV, base=BASE, rot_dim=case["rot"], layout=case["layout"],
                                      sections=[axis.count(a) for a in range(case["axes"])])
        if case["op"] != "rotary":
            s["cache"] = altr.PagedCache(s["k_cache"], s["v_cache"])
    return s


# ------------------------------------------------------------------ the framework's calls
def _run_own(s):
    c = s["case"]
    if c["op"] == "rotary" and c["direction"] == "forward":
        q, k = s["rotary"].apply(s["q"], s["k"], s["pos"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
        return {"q": q, "k": k}
    if c["op"] == "rotary":
        g = s["rotary"].backward(s["dq"], s["dk"], s["pos"], q=s["q"] if c["norm"] else None,
                                 k=s["k"] if c["norm"] else None, q_weight=s["q_weight"], k_weight=s["k_weight"],
                                 eps=EPS)
        out = {"dq": g.q, "dk": g.k}
        return out | {"dq_weight": g.q_weight, "dk_weight": g.k_weight} if c["norm"] else out
    if c["op"] == "append":
        q = s["cache"].append(s["k"], s["v"], s["table"], s["lens"], s["cu"], rotary=s["rotary"], pos=s["pos"],
                              k_weight=s["k_weight"], q=s["q"], q_weight=s["q_weight"], eps=EPS)
        return {"q": q, "k_cache": s["cache"].k, "v_cache": s["cache"].v}
    o = s["cache"].attend(s["q"], s["table"], s["lens"], s["cu"], causal=c["causal"], window=c["window"],
                          max_new=s["max_new"], max_len=s["max_len"], return_lse=c["lse"])
    return {"o": o[0], "lse": o[1]} if c["lse"] else {"o": o}


# ------------------------------------------------------------------ plain forms
def _turn(x, cos, sin, layout):
    """Pairs of the first 2 * cos.shape[-1] channels turned, the others kept; x [T, H, d], cos [T, R/2]."""
    half = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    if layout == "half":
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _angles(s):
    place = s["pos"].long()[s["axis"]].T
    at = torch.arange(len(s["axis"]), device=DEV)
    return s["cos"][place, at], s["sin"][place, at]


def _forward(x, weight, s):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight
    return _turn(y, *_angles(s), s["case"]["layout"]).to(x.dtype)


def _backward(dy, x, weight, s):
    cos, sin = _angles(s)
    g = _turn(dy.float(), cos, -sin, s["case"]["layout"])
    if weight is None:
        return g.to(dy.dtype), None
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    wg = weight * g
    dx = r * wg - x * (r * r * r) * (x * wg).mean(-1, keepdim=True)
    return dx.to(dy.dtype), (g * x * r).sum((0, 1))


def _run_append(s):
    page = s["k_cache"].shape[2]
    at = torch.arange(len(s["seq"]), device=DEV) - s["cu"][s["seq"] + 1] + s["lens"][s["seq"]]
    home, slot = s["table"][s["seq"], at // page].long(), at % page
    s["k_cache"][home, :, slot] = _forward(s["k"], s["k_weight"], s)
    s["v_cache"][home, :, slot] = s["v"]
    return {"q": _forward(s["q"], s["q_weight"], s), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _run_attend(s):
    c, q, table = s["case"], s["q"], s["table"].long().clamp(min=0)
    batch, hk, d, group = c["batch"], c["hk"], c["d"], c["hq"] // c["hk"]
    top, n = s["max_new"], s["max_len"]
    # padded: sequence b's new token i in row i, its key j in column j
    row = torch.arange(len(s["seq"]), device=DEV) - s["cu"][s["seq"]]
    qs = torch.zeros(batch, top, c["hq"], d, device=DEV)
    qs[s["seq"], row] = q.float()
    qs = qs.reshape(batch, top, hk, group, d).permute(0, 2, 3, 1, 4).reshape(batch, hk, group * top, d)
    keys = s["k_cache"][table].transpose(1, 2).reshape(batch, hk, -1, d)[:, :, :n].float()
    vals = s["v_cache"][table].transpose(1, 2).reshape(batch, hk, -1, d)[:, :, :n].float()
    here = (s["lens"] - s["cu"].diff())[:, None] + torch.arange(top, device=DEV)  # [batch, top]
    j = torch.arange(n, device=DEV)
    seen = (j < s["lens"][:, None, None]).expand(batch, top, n)
    if c["causal"]:
        seen = seen & (j <= here[..., None])
    if c["window"]:
        seen = seen & (j > here[..., None] - c["window"])
    score = (qs @ keys.transpose(-1, -2)).mul_(1 / math.sqrt(d)).reshape(batch, hk, group, top, n)
    score.masked_fill_(~seen[:, None, None], float("-inf"))
    most = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(most).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(batch, hk, group * top, n) @ vals).reshape(batch, hk, group, top, d) / total.clamp(min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(batch, top, c["hq"], d)[s["seq"], row].to(q.dtype)
    if not c["lse"]:
        return {"o": o}
    lse = (most + total.log())[..., 0].permute(0, 3, 1, 2).reshape(batch, top, c["hq"])[s["seq"], row]
    return {"o": o, "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "append":
        return _run_append(state)
    if c["op"] == "attend":
        return _run_attend(state)
    if c["direction"] == "forward":
        return {"q": _forward(state["q"], state["q_weight"], state), "k": _forward(state["k"], state["k_weight"], state)}
    dq, dqw = _backward(state["dq"], state["q"], state["q_weight"], state)
    dk, dkw = _backward(state["dk"], state["k"], state["k_weight"], state)
    return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw} if c["norm"] else {"dq": dq, "dk": dk}


# ------------------------------------------------------------------ 64 bits
def _phase(case, pos):
    """exp(i theta) of each token and pair, complex128."""
    axis = torch.tensor(_axis_of(case), device=DEV)
    half = len(axis)
    freq = torch.tensor([BASE ** (-i / half) for i in range(half)], dtype=torch.float64, device=DEV)
    theta = pos[axis].double().T * freq
    return torch.complex(torch.cos(theta), torch.sin(theta))[:, None]


def _as_pairs(x, case):
    r = case["rot"]
    if case["layout"] == "half":
        return torch.complex(x[..., :r // 2], x[..., r // 2:r])
    return torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous())


def _of_pairs(z, x, case):
    r = case["rot"]
    out = x.clone()
    if case["layout"] == "half":
        out[..., :r // 2], out[..., r // 2:r] = z.real, z.imag
    else:
        out[..., 0:r:2], out[..., 1:r:2] = z.real, z.imag
    return out


def _exact_forward(x, weight, phase, case):
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    return _of_pairs(_as_pairs(x, case) * phase, x, case)


def _exact_backward(dy, x, weight, phase, case):
    dy = dy.double()
    g = _of_pairs(_as_pairs(dy, case) * phase.conj(), dy, case)
    if weight is None:
        return g, None
    # y = u w with u = x / sqrt(mean x^2 + eps): du = g w, dx = (du - u mean(u du)) / sqrt(...)
    x = x.double()
    rms = torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
    u = x / rms
    du = g * weight.double()
    return (du - u * (u * du).sum(-1, keepdim=True) / x.shape[-1]) / rms, (g * u).sum((0, 1))


def _exact_attend(s):
    c = s["case"]
    d, group, page = c["d"], c["hq"] // c["hk"], c["page"]
    out, stat = [], []
    for b, (n, past) in enumerate(_sizes(c)):
        length = n + past
        home = s["table"][b, :(length + page - 1) // page].long()
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
            k = s["k_cache"][home, h // group].reshape(-1, d)[:length].double()
            v = s["v_cache"][home, h // group].reshape(-1, d)[:length].double()
            x = (s["q"][first:first + n, h].double() @ k.T / math.sqrt(d)).masked_fill_(hidden, float("-inf"))
            z = torch.logsumexp(x, -1)
            heads.append(x.sub_(z[:, None]).exp_() @ v)
            stats.append(z)
        out.append(torch.stack(heads, 1))
        stat.append(torch.stack(stats, 1))
    return {"o": torch.cat(out), "lse": torch.cat(stat)} if c["lse"] else {"o": torch.cat(out)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    phase = _phase(case, s["pos"])
    if case["op"] == "append":
        k, v = s["k_cache"].double(), s["v_cache"].double()
        rows, page, t = _exact_forward(s["k"], s["k_weight"], phase, case), case["page"], 0
        for b, (n, past) in enumerate(_sizes(case)):
            at = past + torch.arange(n, device=DEV)
            home = s["table"][b].long()[at // page]
            k[home, :, at % page], v[home, :, at % page] = rows[t:t + n], s["v"][t:t + n].double()
            t += n
        return {"q": _exact_forward(s["q"], s["q_weight"], phase, case), "k_cache": k, "v_cache": v}
    if case["direction"] == "forward":
        return {"q": _exact_forward(s["q"], s["q_weight"], phase, case),
                "k": _exact_forward(s["k"], s["k_weight"], phase, case)}
    dq, dqw = _exact_backward(s["dq"], s["q"], s["q_weight"], phase, case)
    dk, dkw = _exact_backward(s["dk"], s["k"], s["k_weight"], phase, case)
    return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw} if case["norm"] else {"dq": dq, "dk": dk}


if __name__ == "__main__":
    for n, c in enumerate(listed() + [draw(random.Random(i)) for i in range(8)]):
        w = work(c)
        print(f"{c.get('name', 'drawn %d' % n):20s} {w['bytes'] / 1e6:10.3f} MB {w['flops'] / 1e9:10.3f} GFLOP "
              f"{1e6 * _cost(c):8.1f} us  room {_room(c) / 1e9:.2f} GB")
