"""The operators between the linears of a decoder that serves several requests at once, as cases that
can be measured: the norm with the residual's addition (and its gradient), the writer of a paged cache,
the attention that reads it, and the adapters of many requests beside a shared 4-bit linear.

`run` computes each in its plain form, from elementary torch operations in 32 bits, or, where `own` is
true, by the library's entry points.  `exact` is the same from the definitions in 64 bits.

Sizes are those of the Llama-2-7B backbone (hidden size 4096, 32 heads of 128, the four linears of a
layer) and generic ones around them: grouped heads, heads of 64, other widths, ragged lengths.
"""
from __future__ import annotations

import math
import random

import torch

own = False

LAYER = "12288x4096+4096x4096+22016x4096+4096x11008"
EPS = 1e-5
THETA = 10000.0
MOST_SCORES = 0.8e9        # values of a padded score matrix: the plain form holds three of them
MOST_KEYS = 2.1e9          # bytes of a cache of 16 bits that is attended to
MOST_KEPT = 3.9e8          # ... that is written to
MOST_NEW = 8000
MOST_NORM = 4096 * 4096
MOST_MACS = 1024 * 202_375_168


def listed():
    def norm(name, rows, width, **more):
        return dict(name=name, kind="norm", rows=rows, width=width, **{**dict(residual=True, eight=False), **more})

    def cached(name, kind, requests, new, longest, past, **more):
        return dict(name=name, kind=kind, requests=requests, new=new, longest=longest, past=past, mix=7,
                    **{**dict(heads=32, kv_heads=32, dim=128, page=64, eight=False), **more})

    return [
        # a decode step of a few requests: the norm before a 4-bit linear, with the residual's addition.  The smallest call
        norm("norm_decode", 7, 4096),
        # a prompt, normalised straight to the 8-bit activations of an 8-bit linear
        norm("norm_prompt_8bit", 2048, 4096, eight=True),
        # training: the gradient of a short batch, an odd number of rows, and of a long one
        dict(name="norm_gradient", kind="gradient", rows=289, width=4096, residual=True),
        dict(name="norm_gradient_long", kind="gradient", rows=4096, width=4096, residual=True),
        # a decode step of 16 requests: rotated queries, keys and values into the cache
        cached("append_decode", "append", 16, 1, 1500, True),
        # packed prompts of different lengths into a cache of 8 bits
        cached("append_prompts_8bit", "append", 5, 1600, 1600, False, eight=True),
        # the action tokens of one robot: about 290 tokens of prompt, one new token
        cached("attend_one", "attend", 1, 1, 295, True, page=16),
        # a decode step of many requests with long histories, grouped heads and a cache of 8 bits
        cached("attend_many_8bit", "attend", 64, 1, 8000, True, kv_heads=8, eight=True),
        # new tokens of some requests behind long histories, grouped heads
        cached("attend_chunks", "attend", 3, 384, 13000, True, kv_heads=8),
        # whole prompts of different lengths, packed
        cached("attend_prompts", "attend", 4, 2500, 2500, False),
        # a decode step of a layer for 16 requests that each have an adapter of their own
        dict(name="adapters_decode", kind="adapters", rows=16, requests=16, adapters=16, rank=32, linears=LAYER, group=128, mix=7),
        # packed prompts, each with its adapter, one without
        dict(name="adapters_prompts", kind="adapters", rows=1000, requests=5, adapters=8, rank=32, linears=LAYER, group=128, mix=7),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_norm(rng, kind):
    width = rng.choice((1024, 2048, 4096, 5120, 8192, 16384, 8 * (2 * _log(rng, 8, 1023) + 1), 8 * (2 * _log(rng, 8, 1023) + 1)))
    case = dict(kind=kind, rows=_log(rng, 1, max(1, min(16384, MOST_NORM // width))), width=width, residual=rng.random() < 0.7)
    return dict(case, eight=rng.random() < 0.5) if kind == "norm" else case


def _draw_cached(rng, kind):
    shape = rng.choice(("decode", "decode", "chunk", "prompt"))
    kv_heads = rng.choice((1, 2, 4, 8, 8, 32))
    group = 1 if kv_heads == 32 else rng.choice((1, 2, 4, 4, 8))
    dim = rng.choice((64, 128, 128))
    heads = kv_heads * group
    while True:
        if shape == "decode":
            requests, new, longest = _log(rng, 1, 128), 1, _log(rng, 16, 16000)
        elif shape == "chunk":
            requests, new = _log(rng, 1, 8), _log(rng, 2, 600)
            longest = new + _log(rng, 16, 12000)
        else:
            requests, new = _log(rng, 1, 8), _log(rng, 16, 2600)
            longest = new
        if requests * heads * new * longest <= MOST_SCORES and requests * longest * kv_heads * dim * 4 <= (MOST_KEYS if kind == "attend" else MOST_KEPT) and \
                (kind == "attend" or requests * new <= MOST_NEW):
            break
    return dict(kind=kind, requests=requests, new=new, longest=longest, past=shape != "prompt", mix=rng.randint(1, 10 ** 6), heads=heads,
                kv_heads=kv_heads, dim=dim, page=rng.choice((16, 32, 64, 64, 128, 256)), eight=rng.random() < 0.4)


def _draw_adapters(rng):
    h = 256 * rng.choice((5, 6, 7, 8, 9, 10, 11, 14, 16, 18))
    f = 256 * int(round(2.6875 * h / 256))
    linears = rng.choice(("%dx%d" % (h, h), "%dx%d+%dx%d+%dx%d+%dx%d" % (3 * h, h, h, h, 2 * f, h, h, f), "%dx%d" % (2 * _log(rng, 250, 6000) + 1, h)))
    macs = sum(n * k for n, k in _shapes(linears))
    rows = max(1, min(_log(rng, 1, 1024), MOST_MACS // macs))
    return dict(kind="adapters", rows=rows, requests=min(rows, _log(rng, 1, 64)), adapters=_log(rng, 1, 48), rank=rng.choice((8, 16, 16, 24, 32, 32, 64)),
                linears=linears, group=128, mix=rng.randint(1, 10 ** 6))


def draw(rng):
    kind = rng.choice(("norm", "gradient", "append", "attend", "attend", "adapters"))
    if kind in ("norm", "gradient"):
        return _draw_norm(rng, kind)
    return _draw_adapters(rng) if kind == "adapters" else _draw_cached(rng, kind)


# ------------------------------------------------------------------------------------- inputs --

def _rng(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1009 * int(seed) + stream)


def _normal(shape, seed, stream, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=_rng(seed, stream), device="cuda") * std).to(dtype)


def _hidden(rows, width, seed, stream):
    """Hidden states: a few columns are ten times as large."""
    t = torch.randn((rows, width), generator=_rng(seed, stream), device="cuda")
    t[:, torch.randperm(width, generator=_rng(seed, stream + 1), device="cuda")[: math.ceil(0.005 * width)]] *= 10
    return t.to(torch.bfloat16)


def _shapes(linears):
    return [tuple(int(v) for v in s.split("x")) for s in linears.split("+")]


def _lengths(case):
    """(new tokens, length with them) of each request: the first has the most of both."""
    rng = random.Random(case["mix"])
    new = [case["new"]] + [rng.randint(max(1, case["new"] // 8), case["new"]) for _ in range(case["requests"] - 1)]
    if not case["past"]:
        return new, list(new)
    before = case["longest"] - case["new"]
    return new, [n + (rng.randint(before // 16, before) if i else before) for i, n in enumerate(new)]


def _pages(case):
    return [-(-n // case["page"]) for n in _lengths(case)[1]]


def _spread(case):
    """The adapter of each row: requests of consecutive rows, from two requests on the last one without an adapter."""
    rng = random.Random(case["mix"])
    cuts = sorted(rng.sample(range(1, case["rows"]), case["requests"] - 1)) if case["requests"] < case["rows"] else list(range(1, case["rows"]))
    which = list(range(case["adapters"]))
    rng.shuffle(which)
    of = [which[i % len(which)] for i in range(case["requests"])]
    if case["requests"] > 1 and case["requests"] < case["rows"]:
        of[-1] = -1
    rows, at = [], 0
    for a, end in zip(of, cuts + [case["rows"]]):
        rows += [a] * (end - at)
        at = end
    return rows


def _prepare_norm(case, seed):
    rows, width = case["rows"], case["width"]
    st = dict(x=_hidden(rows, width, seed, 1), weight=(1 + _normal((width,), seed, 3, 0.2, torch.float32)).to(torch.bfloat16),
              residual=_hidden(rows, width, seed, 4) if case["residual"] else None)
    if case["kind"] == "gradient":
        st.update(dy=_normal((rows, width), seed, 6), dres=_normal((rows, width), seed, 7) if case["residual"] else None)
        st["dy"] += 0.2 * st["x"] * st["weight"].sign()     # gradients pull towards what the layer said: the weight's is no sum of noise alone
    return st


def _prepare_cached(case, seed):
    new, total = _lengths(case)
    pages = _pages(case)
    heads, kv_heads, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    T, R, used = sum(new), case["requests"], sum(pages)
    pool = used + 3
    order = torch.randperm(pool, generator=_rng(seed, 1), device="cuda")[:used].to(torch.int32)
    filled = torch.arange(max(pages), device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    table = torch.full((R, max(pages)), -1, dtype=torch.int32, device="cuda")
    table[filled] = order
    shape = (pool, kv_heads, page, dim)
    if case["eight"]:
        k, v = (torch.randint(-127, 128, shape, generator=_rng(seed, s), device="cuda", dtype=torch.int8) for s in (2, 3))
        scales = tuple(0.02 + 0.01 * torch.rand(shape[:3], generator=_rng(seed, s), device="cuda") for s in (4, 5))
    else:
        k, v = _normal(shape, seed, 2), _normal(shape, seed, 3)
        scales = (None, None)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    qkv = _normal((T, (heads + 2 * kv_heads) * dim), seed, 6)   # what the fused linear of a layer writes
    at = torch.arange(max(total), device="cuda", dtype=torch.float64)[:, None]
    angle = at * THETA ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) * 2 / dim)
    return dict(k=k, v=v, k_scale=scales[0], v_scale=scales[1], table=table, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                total=torch.tensor(total, dtype=torch.int32, device="cuda"), qkv=qkv, cos=angle.cos().float(), sin=angle.sin().float(),
                tokens=T, scale=1 / math.sqrt(dim))


def _prepare_adapters(case, seed):
    rows, n, r = case["rows"], case["adapters"], case["rank"]
    items = []
    for i, (N, K) in enumerate(_shapes(case["linears"])):
        G = K // case["group"]
        words = lambda shape, s: torch.randint(-2 ** 31, 2 ** 31 - 1, shape, generator=_rng(seed, s), device="cuda", dtype=torch.int64).to(torch.int32)  # noqa: E731
        items.append(dict(N=N, K=K, qweight=words((N, K // 8), 10 * i), zeros=words((N, -(-G // 8)), 10 * i + 1),
                          scales=(0.002 + 0.002 * torch.rand((N, G), generator=_rng(seed, 10 * i + 2), device="cuda")).half(),
                          x=_hidden(rows, K, seed, 10 * i + 3), A=_normal((n, r, K), seed, 10 * i + 5, 0.02), B=_normal((n, N, r), seed, 10 * i + 6, 0.05),
                          scaling=0.5 + 1.5 * torch.rand((n,), generator=_rng(seed, 10 * i + 7), device="cuda")))
    return dict(items=items, row_adapter=torch.tensor(_spread(case), dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    make = {"norm": _prepare_norm, "gradient": _prepare_norm, "append": _prepare_cached, "attend": _prepare_cached, "adapters": _prepare_adapters}
    return dict(make[case["kind"]](case, seed), case=case)


# -------------------------------------------------------------------------------- plain forms --

def _plain_norm(st):
    h = st["x"].float()
    if st["residual"] is not None:
        h = h + st["residual"].float()
    r = (h.square().mean(1, keepdim=True) + EPS).rsqrt()
    out = {"h": h.to(torch.bfloat16)} if st["residual"] is not None else {}
    if not st["case"]["eight"]:
        return dict(out, y=(h * r * st["weight"].float()).to(torch.bfloat16))
    # codes of h * weight: the row's factor r is in the scale alone, so no rounding of r decides a code
    u = h * st["weight"].float()
    most = u.abs().amax(1, keepdim=True)
    step = torch.where(most > 0, most / torch.full_like(most, 127.0), torch.ones_like(most))
    code = (u / step).round().clamp(-127, 127)
    scale = step * r
    return dict(out, y=code * scale, scale=scale.reshape(-1))


def _plain_gradient(st):
    h, w, dy = st["x"].float(), st["weight"].float(), st["dy"].float()
    r = (h.square().mean(1, keepdim=True) + EPS).rsqrt()
    n = h * r
    g = dy * w
    dx = r * (g - n * (g * n).mean(1, keepdim=True))
    if st["dres"] is not None:
        dx = dx + st["dres"].float()
    return dict(dx=dx.to(torch.bfloat16), dweight=(dy * n).sum(0))


def _token_places(st):
    """Of each new token: its request and its position in it."""
    starts = st["starts"].long()
    t = torch.arange(st["tokens"], device="cuda")
    r = torch.searchsorted(starts, t, right=True) - 1
    return r, t - starts[r + 1] + st["total"].long()[r]


def _split(st):
    """q [tokens, heads, dim], k and v [tokens, kv_heads, dim]: views of what the fused linear wrote."""
    c, T = st["case"], st["tokens"]
    a, b = c["heads"] * c["dim"], c["kv_heads"] * c["dim"]
    q, k, v = st["qkv"].split((a, b, b), dim=1)
    return q.view(T, c["heads"], c["dim"]), k.view(T, c["kv_heads"], c["dim"]), v.view(T, c["kv_heads"], c["dim"])


def _rotated(t, cos, sin):
    half = t.shape[-1] // 2
    a, b = t[..., :half], t[..., half:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _cached_values(st):
    """The cache as the values it stands for."""
    if st["case"]["eight"]:
        return dict(k=torch.mul(st["k"], st["k_scale"][..., None]), v=torch.mul(st["v"], st["v_scale"][..., None]))
    return dict(k=st["k"], v=st["v"])


def _plain_append(st):
    c = st["case"]
    r, at = _token_places(st)
    q, k, v = (t.float() for t in _split(st))
    cos, sin = st["cos"][at][:, None], st["sin"][at][:, None]
    k = _rotated(k, cos, sin)
    page, slot = st["table"].long()[r, at // c["page"]], at % c["page"]
    for into, scales, t in ((st["k"], st["k_scale"], k), (st["v"], st["v_scale"], v)):
        if c["eight"]:
            most = t.abs().amax(-1)
            step = torch.where(most > 0, most / torch.full_like(most, 127.0), torch.ones_like(most))
            into[page, :, slot] = (t / step[..., None]).round().clamp(-127, 127).to(torch.int8)
            scales[page, :, slot] = step
        else:
            into[page, :, slot] = t.to(torch.bfloat16)
    return dict(q=_rotated(q, cos, sin).to(torch.bfloat16), **_cached_values(st))


def _plain_attend(st):
    c = st["case"]
    R, H, D, group = c["requests"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    r, at = _token_places(st)
    i = torch.arange(st["tokens"], device="cuda") - st["starts"].long()[r]
    q = torch.zeros((R, c["new"], H, group, D), device="cuda")
    q[r, i] = _split(st)[0].float().view(-1, H, group, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(R * H, c["new"] * group, D)
    held = torch.arange(st["table"].shape[1] * c["page"], device="cuda")[None] < st["total"][:, None]
    pages = st["table"].long().clamp(min=0)

    def gathered(t, scales):   # [R * H, keys, D]
        t = t[pages].float()
        if scales is not None:
            t = t * scales[pages][..., None]
        t = t.permute(0, 2, 1, 3, 4).reshape(R, H, -1, D)
        return torch.where(held[:, None, :, None], t, 0.0).reshape(R * H, -1, D)

    s = torch.bmm(q, gathered(st["k"], st["k_scale"]).transpose(1, 2)).mul_(st["scale"]).view(R, H, c["new"], group, -1)
    key = torch.arange(s.shape[-1], device="cuda")
    new = st["starts"].long().diff()
    last = (st["total"].long() - new)[:, None] + torch.arange(c["new"], device="cuda")
    s.masked_fill_(~(key <= last[..., None])[:, None, :, None], -math.inf)
    most = s.amax(-1, keepdim=True)
    s = s.sub_(torch.where(most > -math.inf, most, 0.0)).exp_()
    s = s.div_(s.sum(-1, keepdim=True))
    o = torch.bmm(s.view(R * H, c["new"] * group, -1), gathered(st["v"], st["v_scale"]))
    return o.view(R, H, c["new"], group, D).permute(0, 2, 1, 3, 4)[r, i].reshape(st["tokens"], c["heads"], D).to(torch.bfloat16)


def _nibbles(words, count):
    shift = torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)
    return ((words[..., None] >> shift) & 15).flatten(1)[:, :count].float()


def _plain_adapters(st):
    rows = st["row_adapter"].long()
    group = st["case"]["group"]

    def one(e):
        q, z, s = _nibbles(e["qweight"], e["K"]), _nibbles(e["zeros"], e["K"] // group), e["scales"].float()
        w = ((q.view(e["N"], -1, group) - z[..., None]) * s[..., None]).view(e["N"], e["K"])
        x, (n, r, _) = e["x"].float(), e["A"].shape
        mine = (rows[:, None] == torch.arange(n, device="cuda")).float() * e["scaling"]
        down = (x @ e["A"].float().view(n * r, -1).t()).view(-1, n, r) * mine[..., None]
        up = e["B"].float().permute(0, 2, 1).reshape(n * r, -1)
        return (x @ w.t() + down.view(-1, n * r) @ up).to(torch.bfloat16)

    return [one(e) for e in st["items"]]


# -------------------------------------------------------------------------- the library's calls --

def _own_norm(st):
    from paper_2412_01034_amd import binding as B
    if "out" not in st:
        new = lambda dtype: torch.empty_like(st["x"], dtype=dtype)  # noqa: E731
        st["out"] = {"h": new(torch.bfloat16)} if st["residual"] is not None else {}
        if st["case"]["eight"]:
            st["codes"] = new(torch.int8)
            st["out"]["scale"] = torch.empty(st["x"].shape[0], device="cuda")
        else:
            st["out"]["y"] = new(torch.bfloat16)
    out = st["out"]
    B.qail_rmsnorm(st["x"], st["weight"], EPS, residual=st["residual"], residual_out=out.get("h"), y=out.get("y"), y_s8=st.get("codes"),
                   y_scale=out.get("scale"))
    return dict(out, y=torch.mul(st["codes"], out["scale"][:, None])) if st["case"]["eight"] else out


def _own_gradient(st):
    from paper_2412_01034_amd import binding as B
    if "out" not in st:
        rows, width = st["x"].shape
        st["out"] = dict(dx=torch.empty_like(st["x"]), dweight=torch.empty(width, device="cuda"))
        st["workspace"] = torch.empty(B.qail_rmsnorm_backward_workspace(rows, width), dtype=torch.uint8, device="cuda")
    B.qail_rmsnorm_backward(st["x"], st["weight"], EPS, st["dy"], st["out"]["dx"], st["out"]["dweight"], st["workspace"], dres=st["dres"])
    return st["out"]


def _handles(B, st):
    new, total = _lengths(st["case"])
    st["cache"] = B.make_kv_cache(st["k"], st["v"], st["k_scale"], st["v_scale"])
    st["requests"] = B.make_requests(st["table"], st["starts"], st["total"], tokens=st["tokens"], max_new=max(new), max_len=max(total))
    st["q"], st["new_k"], st["new_v"] = _split(st)
    st["out"] = torch.empty((st["tokens"], st["case"]["heads"], st["case"]["dim"]), dtype=torch.bfloat16, device="cuda")


def _own_append(st):
    from paper_2412_01034_amd import binding as B
    if "cache" not in st:
        _handles(B, st)
    B.qail_kv_append(st["cache"], st["requests"], st["new_k"], st["new_v"], q=st["q"], q_out=st["out"], cos=st["cos"], sin=st["sin"])
    return dict(q=st["out"], **_cached_values(st))


def _own_attend(st):
    from paper_2412_01034_amd import binding as B
    if "cache" not in st:
        _handles(B, st)
        n = B.qail_paged_attention_workspace(st["cache"], st["requests"], st["case"]["heads"])
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    B.qail_paged_attention(st["cache"], st["requests"], st["q"], st["out"], st["scale"], st["workspace"])
    return st["out"]


def _own_adapters(st):
    from paper_2412_01034_amd import binding as B
    rows, count = st["case"]["rows"], len(st["items"])
    if "handle" not in st:
        st["y"] = [torch.empty((rows, e["N"]), dtype=torch.bfloat16, device="cuda") for e in st["items"]]
        st["handle"] = B.make_w4a16_items([dict(e, y=y, group_size=st["case"]["group"]) for e, y in zip(st["items"], st["y"])], rows)
        st["adapters"] = B.make_adapters(st["items"])
        n = B.qail_w4a16_adapters_workspace(st["handle"], st["adapters"], count, rows)
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    B.qail_w4a16_linear_adapters_batch(st["handle"], st["adapters"], st["row_adapter"], count, rows, st["workspace"])
    return st["y"]


def run(st):
    plain = {"norm": _plain_norm, "gradient": _plain_gradient, "append": _plain_append, "attend": _plain_attend, "adapters": _plain_adapters}
    mine = {"norm": _own_norm, "gradient": _own_gradient, "append": _own_append, "attend": _own_attend, "adapters": _own_adapters}
    return (mine if own else plain)[st["case"]["kind"]](st)


# --------------------------------------------------------------------------------------- work --

def work(case):
    kind = case["kind"]
    if kind in ("norm", "gradient"):
        n = case["rows"] * case["width"]
        if kind == "gradient":
            return dict(bytes=n * (8 if case["residual"] else 6) + 6 * case["width"], flops=12 * n)
        out = (1 if case["eight"] else 2) + (4 if case["residual"] else 0)
        return dict(bytes=n * (2 + out) + 2 * case["width"] + (4 * case["rows"] if case["eight"] else 0), flops=6 * n)
    if kind == "adapters":
        rows, r, n = case["rows"], case["rank"], len({a for a in _spread(case) if a >= 0})
        byte = flops = 0
        for N, K in _shapes(case["linears"]):
            G = K // case["group"]
            byte += N * K // 2 + N * G * 2 + N * -(-G // 8) * 4 + 2 * rows * (K + N) + 2 * n * r * (K + N)
            flops += 2 * rows * (N * K + r * (N + K))
        return dict(bytes=byte, flops=flops)
    new, total = _lengths(case)
    D, H, heads = case["dim"], case["kv_heads"], case["heads"]
    row = H * (D + 4 if case["eight"] else 2 * D)    # a token's keys, or values
    T = sum(new)
    if kind == "append":
        angles = len(set().union(*(range(t - n, t) for n, t in zip(new, total)))) * D * 4
        return dict(bytes=T * (2 * (heads + 2 * H) * D + 2 * heads * D + 2 * row) + angles, flops=6 * T * (heads + H) * D)
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(new, total))
    return dict(bytes=4 * T * heads * D + sum(total) * 2 * row, flops=4 * pairs * heads * D)


# -------------------------------------------------------------------------------------- exact --

def _exact_norm(st):
    h = st["x"].double() + (st["residual"].double() if st["residual"] is not None else 0)
    if st["case"]["eight"]:
        # the codes are those of 32-bit arithmetic (one rounding a line), everything else is not
        f = h.float()
        u = f * st["weight"].float()
        step = u.abs().max(1).values
        step = torch.where(step > 0, (step.double() / 127).float(), 1.0)
        code = torch.round((u.double() / step.double()[:, None]).float()).clamp(-127, 127)
        scale = step.double() / torch.sqrt(torch.mean(h * h, 1) + EPS)
        out = dict(y=code.double() * scale[:, None], scale=scale)
    else:
        out = dict(y=h / torch.sqrt(torch.mean(h * h, 1) + EPS)[:, None] * st["weight"].double())
    return dict(out, h=h) if st["residual"] is not None else out


def _exact_gradient(st):
    h, w, dy = (st[k].double() for k in ("x", "weight", "dy"))
    rms = torch.sqrt(torch.mean(h * h, 1, keepdim=True) + EPS)
    dx = dy * w / rms - h * torch.sum(dy * w * h, 1, keepdim=True) / (h.shape[1] * rms ** 3)
    return dict(dx=dx + st["dres"].double() if st["dres"] is not None else dx, dweight=torch.sum(dy * h / rms, 0))


def _exact_append(st):
    c = st["case"]
    new, total = _lengths(c)
    D, H, heads = c["dim"], c["kv_heads"], c["heads"]
    x = st["qkv"].view(-1, heads + 2 * H, D)
    table, cos, sin = st["table"].cpu(), st["cos"].double(), st["sin"].double()
    out = {n: st[n].double() * (st[n + "_scale"].double()[..., None] if c["eight"] else 1) for n in ("k", "v")}
    q, t = torch.empty((len(x), heads, D), dtype=torch.float64, device="cuda"), 0
    for r, (n, length) in enumerate(zip(new, total)):
        at = torch.arange(length - n, length, device="cuda")
        a, b = x[t:t + n, :heads + H].double().chunk(2, -1)
        cs, sn = cos[at][:, None], sin[at][:, None]
        turned = torch.cat((a * cs - b * sn, b * cs + a * sn), -1)
        q[t:t + n] = turned[:, :heads]
        where = table[r].cuda().long()[at // c["page"]], at % c["page"]
        keys, values = turned[:, heads:], x[t:t + n, heads + H:].double()
        if c["eight"]:    # codes of 32-bit arithmetic, each operation rounded once
            a, b, cs, sn = a[:, heads:].float(), b[:, heads:].float(), cs.float(), sn.float()
            keys = torch.cat(((a * cs).sub(b * sn), (b * cs).add(a * sn)), -1).double()
        for name, rows in (("k", keys), ("v", values)):
            if c["eight"]:
                step = rows.abs().max(-1).values
                step = torch.where(step > 0, (step / 127).float().double(), 1.0)
                rows = torch.round((rows / step[..., None]).float()).double() * step[..., None]
            out[name][where[0], :, where[1]] = rows
        t += n
    return dict(out, q=q)


def _exact_attend(st):
    c = st["case"]
    new, total = _lengths(c)
    D, H, heads = c["dim"], c["kv_heads"], c["heads"]
    x = st["qkv"].view(-1, heads + 2 * H, D)
    table = st["table"].cpu()
    out, t = torch.empty((st["tokens"], heads, D), dtype=torch.float64, device="cuda"), 0
    for r, (n, length) in enumerate(zip(new, total)):
        held = table[r][:-(-length // c["page"])].cuda().long()
        future = torch.arange(length, device="cuda")[None, :] > torch.arange(length - n, length, device="cuda")[:, None]
        for h in range(H):
            kv = []
            for name in ("k", "v"):
                rows = st[name][held, h].double()
                if c["eight"]:
                    rows = rows * st[name + "_scale"][held, h].double()[..., None]
                kv.append(rows.reshape(-1, D)[:length])
            for g in range(h * (heads // H), (h + 1) * (heads // H)):
                s = (x[t:t + n, g].double() @ kv[0].t()) / math.sqrt(D)
                s[future] = -math.inf
                out[t:t + n, g] = torch.softmax(s, 1) @ kv[1]
        t += n
    return out


def _exact_adapters(st):
    group, rows = st["case"]["group"], st["row_adapter"].long()
    out = []
    for e in st["items"]:
        codes = torch.stack([(e["qweight"] >> (4 * j)) & 15 for j in range(8)], -1).reshape(e["N"], e["K"] // group, group).double()
        zeros = torch.stack([(e["zeros"] >> (4 * j)) & 15 for j in range(8)], -1).reshape(e["N"], -1)[:, :e["K"] // group].double()
        x = e["x"].double()
        y = x @ ((codes - zeros[..., None]) * e["scales"].double()[..., None]).reshape(e["N"], -1).t()
        for a in sorted(set(rows.tolist()) - {-1}):
            at = rows == a
            y[at] += e["scaling"][a].double() * (x[at] @ e["A"][a].double().t()) @ e["B"][a].double().t()
        out.append(y)
    return out


def exact(case, seed):
    if case["kind"] == "attend" and work(case)["flops"] > 2e12:
        return None
    st = prepare(case, seed)
    how = {"norm": _exact_norm, "gradient": _exact_gradient, "append": _exact_append, "attend": _exact_attend, "adapters": _exact_adapters}
    return how[case["kind"]](st)
