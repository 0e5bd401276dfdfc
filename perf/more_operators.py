"""What stands between the products of a decoder layer, as cases that can be
timed and checked.

Four kinds, all through the public binding (paper_2410_14740_amd.attention and
paper_2410_14740_amd.norms):

  norm    the residual stream takes a block's output, normed before if the layer
          norms after its blocks, times a gate and a scale, and is normed for the
          next block
  rotate  queries and keys turned by their positions, which may have several
          axes (time, height, width)
  append  keys turned by their positions on the way into the 8-bit cache, with
          their values, and the queries beside them. Prompts are read back as
          well: what codes and scales stand for is their outcome
  chunk   a chunk of new tokens attends over the cache: over what it holds, its
          last tokens the chunk's own ("held"), or over what it holds and then
          the chunk's keys and values, which are not in it yet ("new")

The cache holds blocks of `block` tokens of one kv head as signed bytes with one
fp32 scale per block (s = amax / 127, q = clamp(rne(x / s))), for keys and values
apart; the tokens of a sequence's last block stay in their 16-bit type too and
are attended from there until the block is full. Head counts and widths are those
of the 7B, 13B and 70B configurations (d_model 4096, 5120, 8192 at 128 per head;
the 70B one with eight kv heads) and of the tiny one (d_model 1024, as 16 heads
of 64).

With `own` False the operators are computed by elementary torch operations in
32 bits (angles in 64); with `own` True by the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HEADS = {"tiny": (16, 16, 64), "7b": (32, 32, 128), "13b": (40, 40, 128), "70b": (64, 8, 128)}
NORM_MOST = 10692 * 8192            # elements of the largest norm
ROTATE_MOST = 16385 * 72 * 128      # elements of the largest rotation
APPEND_MOST = 40000 * 8 * 128       # elements of the largest append's keys
CHUNK_MOST = 64 * 128 * (2048 * 32048 + 700 * 17085)  # heads x width x pairs of the largest chunk
CACHE_MOST = 8 * 128 * 270000       # heads x width x tokens of the largest cache


def _norm(name, rows, d, x, y, norm="rms", post=False, gate="none", weight="f16", scale=1.0, pad=0):
    return {"name": name, "kind": "norm", "rows": rows, "d": d, "x": x, "y": y, "norm": norm, "post": post,
            "gate": gate, "weight": weight, "scale": scale, "pad": pad}


def _heads(name, kind, model, dtype, **more):
    hq, hk, d = HEADS[model]
    return {"name": name, "kind": kind, "hq": hq, "hk": hk, "d": d, "dtype": dtype, **more}


def _turn(axes="64", rot=128, interleaved=False, base=10000.0):
    return {"axes": axes, "rot": rot, "interleaved": interleaved, "base": base}


def listed():
    return [
        # one token of a small model between attention and FFN: launch and latency
        _norm("norm-tiny-token", 1, 1024, "f32", "f16"),
        # a chunk of ragged prompts at 13B, mean and variance, blocks scaled down by depth
        _norm("norm-13b-chunk", 889, 5120, "f16", "f16", norm="layer", scale=0.22),
        # long documents at 70B, normed after the block as well and gated per channel
        _norm("norm-70b-long", 10692, 8192, "f32", "bf16", post=True, gate="channel", weight="f32"),
        # a batch of ragged 7B prompts, rows of one fused projection
        _heads("rotate-7b-packed", "rotate", "7b", "f16", lens="1,7,64,129,515,1000,2380", **_turn()),
        # text around images at 70B: positions of time, height and width
        _heads("rotate-70b-image", "rotate", "70b", "bf16", lens="16385", **_turn("16,24,24", base=1e6)),
        # one token of a small model's sequence: latency
        _heads("append-tiny-token", "append", "tiny", "f16", lens="100", block=64, token=True, **_turn("32", 64)),
        # a batch of eight at 7B, a token each
        _heads("append-7b-b8", "append", "7b", "f16", lens="191,350,511,640,1100,1535,1999,2047", block=64,
               token=True, **_turn()),
        # long 70B prompts into the cache, half of each head turned
        _heads("append-70b-long", "append", "70b", "bf16", lens="24000,8191,4001,3808", block=64, token=False,
               **_turn("32", 64, base=5e5)),
        # a small model's second turn: few tokens on a short cache
        _heads("chunk-tiny", "chunk", "tiny", "f16", lens="100", q_lens="33", block=64, how="new"),
        # chunked prefill at 13B
        _heads("chunk-13b", "chunk", "13b", "bf16", lens="3500,1511,2323", q_lens="512,300,77", block=64, how="new"),
        # long documents at 70B, a large chunk on what is there
        _heads("chunk-70b-long", "chunk", "70b", "bf16", lens="30000,16385", q_lens="2048,700", block=64, how="new"),
        # drafted tokens checked at 70B: five rows on each of sixteen long sequences, appended before
        _heads("chunk-70b-drafts", "chunk", "70b", "f16", lens=",".join(str(700 + 1913 * i + 11 * i * i) for i in range(16)),
               q_lens=",".join(["5"] * 16), block=64, how="held"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def text(v):
        return ",".join(str(x) for x in v)

    kind = rng.choice(["norm", "norm", "rotate", "append", "append", "chunk", "chunk", "chunk"])
    if kind == "norm":
        d = rng.choice([log_int(64, 16384), 8 * log_int(8, 2048), 1024, 4096, 5120, 8192])
        rows = log_int(1, max(1, min(16000, int(0.9 * NORM_MOST) // d)))
        y = rng.choice(["f16", "bf16"])
        return {"kind": kind, "rows": rows, "d": d, "x": rng.choice(["f32", y]), "y": y,
                "norm": rng.choice(["rms", "layer"]), "post": rng.random() < 0.5,
                "gate": rng.choice(["none", "channel", "row"]) if rows * d < 0.6 * NORM_MOST else "none",
                "weight": rng.choice(["f32", y]), "scale": rng.choice([1.0, 0.22, 1.41]), "pad": rng.choice([0, 0, 8, 72])}
    hk = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    hq = hk * rng.choice([g for g in (1, 2, 3, 4, 5, 8, 16) if hk * g <= 64])
    d = rng.choice([64, 128, 128])
    c = {"kind": kind, "hq": hq, "hk": hk, "d": d, "dtype": rng.choice(["f16", "bf16"])}
    n = log_int(1, 24)
    if kind != "chunk":
        rot = rng.choice([d, d, d // 2])
        half = rot // 2
        a = rng.randint(1, half - 2)
        b = rng.randint(1, half - a - 1)
        c |= _turn(rng.choice([str(half), str(half), f"{a},{half - a}", f"{a},{b},{half - a - b}"]), rot,
                   rng.random() < 0.4, rng.choice([1e4, 5e5, 1e6]))
    if kind == "rotate":
        lens = [log_int(1, 16000) for _ in range(n)]
        while (hq + hk) * d * sum(lens) > 0.9 * ROTATE_MOST:
            lens = [max(1, x // 2) for x in lens]
        return {**c, "lens": text(lens)}
    block = rng.choice([32, 64, 64, 128])
    if kind == "append":
        token = rng.random() < 0.5
        lens = [log_int(1, 24000) for _ in range(n)]
        while (hk * sum(lens) * d > 0.9 * CACHE_MOST if token else max(hk, hq / 8) * d * sum(lens) > 0.9 * APPEND_MOST):
            lens = [max(1, x // 2) for x in lens]
        return {**c, "lens": text(lens), "block": block, "token": token}
    lens = [log_int(1, 60000 if n == 1 else 20000) for _ in range(n)]
    q = [log_int(1, rng.choice([8, 600, 2500])) for _ in range(n)]
    how = rng.choice(["new", "new", "held"])
    if rng.random() < 0.3:
        lens[rng.randrange(n)] = 0  # a sequence that begins with this chunk
    while hq * d * sum(a * (a + b) for a, b in zip(q, lens)) > 0.4 * CHUNK_MOST:
        q = [max(1, a // 2) for a in q]
        if max(q) == 1:
            lens = [b // 2 for b in lens]
    while hk * d * n * max(lens) > 0.9 * CACHE_MOST:
        lens = [b // 2 for b in lens]
    if how == "held":  # the chunk's own tokens among the held ones (but for a row or two that see nothing)
        lens = [max(b, a - rng.randint(0, 2), 1) for a, b in zip(q, lens)]
    return {**c, "lens": text(lens), "q_lens": text(q), "block": block, "how": how}


# ---------------------------------------------------------------------------
# inputs, from the seed alone

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + what)
    return g


def _normal(seed, what, shape, dtype, sigma=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=_gen(seed, what))


def _ints(text):
    return [int(x) for x in text.split(",")]


def _starts(lens):
    return torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device="cuda")


def _freq(c):
    """Radians per position of each pair, fp32: what a user's program holds."""
    half = c["rot"] // 2
    return torch.tensor([c["base"] ** (-i / half) for i in range(half)], dtype=torch.float32, device="cuda")


def _positions(c, seed):
    """[axes][tokens]: a document of text (all axes alike) around pictures of 32 rows."""
    axes = _ints(c["axes"])
    parts = []
    for n in _ints(c["lens"]):
        t = torch.arange(n, dtype=torch.int32)
        rows = [t]
        if len(axes) > 1:
            picture = (t // 1024) % 2 == 1
            h, w = (t % 1024) // 32, t % 32
            start = t // 1024 * 1024
            rows = [torch.where(picture, start, t), torch.where(picture, start + h, t), torch.where(picture, start + w, t)]
        parts.append(torch.stack(rows[:len(axes)]))
    return torch.cat(parts, 1).to(dtype=torch.int32, device="cuda")


def _cache_tensors(c, seed, more):
    """A cache with random codes in pages that lie in no order, `lens` tokens in
    each sequence and room for `more`."""
    lens = _ints(c["lens"])
    n, H, D, B = len(lens), c["hk"], c["d"], c["block"]
    mb = -(-(max(lens) + more) // B)
    P, dt = n * H * mb, DTYPES[c["dtype"]]
    t = {"table": torch.randperm(P, generator=_gen(seed, 1), device="cuda").int().view(n, H, mb),
         "len": torch.tensor(lens, dtype=torch.int32, device="cuda"), "weight": torch.zeros((n, H, mb), device="cuda")}
    for i, name in enumerate(("k", "v")):
        g = _gen(seed, 8 + i)
        codes = t[name + "_codes"] = torch.empty((P, B, D), dtype=torch.int8, device="cuda")
        step = max(1, (1 << 27) // (B * D))
        for p in range(0, P, step):
            m = min(step, P - p)
            codes[p:p + m] = torch.randn((m, B, D), generator=g, device="cuda").mul_(36).round_().clamp_(-127, 127)
        t[name + "_scale"] = torch.empty(P, device="cuda").uniform_(0.02, 0.04, generator=g)
        t["tail_" + name] = torch.empty((n, H, B, D), dtype=dt, device="cuda").normal_(generator=g)
    return t


def prepare(case, seed):
    c = case
    s = {"case": c}
    if c["kind"] == "norm":
        r, d, pad = c["rows"], c["d"], c["pad"]
        x, y = (_normal(seed, i, (r, d + pad), DTYPES[c[n]], 2.0 - i)[:, :d] for i, n in enumerate(("x", "y")))
        x[:, ::61] *= 12.0  # the wide channels of a residual stream
        s |= {"x": x, "y": y}
        w = DTYPES[c["weight"]]
        for i, name in enumerate(("weight", "bias", "post_weight", "post_bias")):
            used = ("bias" not in name or c["norm"] == "layer") and ("post" not in name or c["post"])
            s[name] = (_normal(seed, 2 + i, (d,), w, 0.2) + (0 if "bias" in name else 1)) if used else None
        shape = {"none": None, "channel": (d,), "row": (r, d)}[c["gate"]]
        s["gate"] = _normal(seed, 6, shape, w, 0.5) if shape else None
        return s
    hq, hk, d, dt = c["hq"], c["hk"], c["d"], DTYPES[c["dtype"]]
    lens = _ints(c["lens"])
    n = len(lens)
    if c["kind"] == "chunk":
        ql = _ints(c["q_lens"])
        s["cache"] = _cache_tensors(c, seed, 1)
        x = _normal(seed, 2, (sum(ql), hq + 2 * hk, d), dt)  # rows of one fused projection
        x[:, :hq] *= 1.5
        s |= {"q": x[:, :hq], "k": x[:, hq:hq + hk], "v": x[:, hq + hk:], "lens": lens, "q_lens": ql, "cu": _starts(ql)}
    else:
        token = c["kind"] == "append" and c["token"]
        rows = n if token else sum(lens)
        x = _normal(seed, 2, (rows, hq + 2 * hk, d), dt)
        x[:, :, ::29] *= 3.0  # a few wide channels
        s |= {"q": x[:, :hq], "k": x[:, hq:hq + hk], "v": x[:, hq + hk:], "freq": _freq(c)}
        at = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["positions"] = at.expand(len(_ints(c["axes"])), n).contiguous() if token else _positions(c, seed)
        if c["kind"] == "append":
            s["cache"] = _cache_tensors(c, seed, 1)
            s |= {"cu": _starts([1] * n if token else lens), "pos": at if token else torch.zeros_like(at), "total": rows}
    if own:
        from paper_2410_14740_amd import attention
        if "cache" in s:
            t = s["cache"]
            s["own"] = attention.KVCache(n, hk, d, t["table"].shape[2], block_tokens=c["block"], dtype=dt, tensors=t)
        if "freq" in s:
            s["rotary"] = attention.Rotary(s["freq"], sections=_ints(c["axes"]), interleaved=c["interleaved"])
    return s


# ---------------------------------------------------------------------------
# one pass

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["kind"]](state)


def _own_norm(s):
    from paper_2410_14740_amd import norms
    c = s["case"]
    x, out = norms.residual_norm(s["x"], s["y"], weight=s["weight"], bias=s["bias"], post=c["post"],
                                 post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"],
                                 scale=c["scale"], kind=c["norm"], eps=1e-5)
    return {"x": x, "out": out}


def _own_rotate(s):
    q, k = s["rotary"].rotate(s["q"], s["positions"], k=s["k"])
    return {"q": q, "k": k}


def _own_append(s):
    c, t = s["own"], s["cache"]
    if s["case"]["token"]:
        q, _ = c.append_rotated(s["rotary"], s["k"], s["v"], s["positions"], q=s["q"], pos=s["pos"])
        return {"q": q, "len": t["len"], "tail_k": t["tail_k"], "tail_v": t["tail_v"]}
    q, _ = c.append_rotated(s["rotary"], s["k"], s["v"], s["positions"], q=s["q"], cu=s["cu"], pos=s["pos"])
    k, v = c.read(s["cu"], s["total"])
    return {"q": q, "k": k, "v": v, "len": t["len"]}


def _own_chunk(s):
    c, new = s["case"], s["case"]["how"] == "new"
    out, lse = s["own"].attend_chunk(s["q"], s["cu"], s["k"] if new else None, s["v"] if new else None,
                                     max_q=max(s["q_lens"]), max_len=max(s["lens"]), return_lse=True)
    return {"out": out, "lse": lse}


_run_own = {"norm": _own_norm, "rotate": _own_rotate, "append": _own_append, "chunk": _own_chunk}


def _plain_normed(x, kind, weight, bias):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5)
    x = x if weight is None else x * weight.float()
    return x if bias is None else x + bias.float()


def _plain_norm(s):
    c = s["case"]
    t = s["y"].float()
    if c["post"]:
        t = _plain_normed(t, c["norm"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        t = t * s["gate"].float()
    x = s["x"].float() + c["scale"] * t
    out = _plain_normed(x, c["norm"], s["weight"], s["bias"])
    return {"x": x.to(s["x"].dtype), "out": out.to(s["y"].dtype)}


def _plain_turn(x, s):
    c = s["case"]
    axes, rot = _ints(c["axes"]), c["rot"]
    axis = torch.repeat_interleave(torch.arange(len(axes), device="cuda"), torch.tensor(axes, device="cuda"))
    angle = s["positions"].double()[axis].t() * s["freq"].double()  # [tokens][pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float()
    lo, hi = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = lo * cos - hi * sin, hi * cos + lo * sin
    turned = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _plain_rotate(s):
    return {"q": _plain_turn(s["q"], s), "k": _plain_turn(s["k"], s)}


def _quantized(x):
    """Codes and scales of fp32 blocks [..., block, d]."""
    scale = x.abs().amax((-1, -2)) / 127.0
    div = torch.where(scale > 0, scale, torch.ones_like(scale))[..., None, None]
    return (x / div).round_().clamp_(-127, 127), scale


def _plain_append(s):
    c, t = s["case"], s["cache"]
    n, H, mb = t["table"].shape
    B, D = c["block"], c["d"]
    q, k = _plain_turn(s["q"], s), _plain_turn(s["k"], s)
    table, rows = t["table"].long(), torch.arange(n, device="cuda")
    if c["token"]:
        pos = s["pos"].long()
        blk, off = pos // B, pos % B
        page, done = table[rows, :, blk], (off == B - 1)[:, None]
        for name, x in (("k", k), ("v", s["v"])):
            t["tail_" + name][rows, :, off] = x
            codes, scale = _quantized(t["tail_" + name].float())
            t[name + "_codes"][page] = torch.where(done[..., None, None], codes.char(), t[name + "_codes"][page])
            t[name + "_scale"][page] = torch.where(done, scale, t[name + "_scale"][page])
        t["len"].copy_(pos + 1)
        return {"q": q, "len": t["len"], "tail_k": t["tail_k"], "tail_v": t["tail_v"]}
    cu = s["cu"].long()
    lens = cu[1:] - cu[:-1]
    row = cu[:-1, None] + torch.arange(mb * B, device="cuda")
    full = (torch.arange(mb, device="cuda") < (lens // B)[:, None])[:, None, :, None, None]
    last = (lens - 1).clamp(min=0)
    tail = (last // B)[:, None, None, None, None].expand(n, H, 1, B, D)
    at = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(cu[1:], at, right=True)
    at = at - cu[seq]
    in_tail = (torch.arange(B, device="cuda") <= (last % B)[:, None])[:, None, :, None]
    result = {"q": q}
    for name, x in (("k", k), ("v", s["v"])):
        y = x[row.clamp(max=s["total"] - 1)].float().view(n, mb, B, H, D).permute(0, 3, 1, 2, 4)
        codes, scale = _quantized(y)
        rest = y.gather(2, tail).squeeze(2)
        t[name + "_codes"][table] = torch.where(full, codes.char(), t[name + "_codes"][table])
        t[name + "_scale"][table] = torch.where(full[..., 0, 0], scale, t[name + "_scale"][table])
        t["tail_" + name].copy_(torch.where(in_tail, rest.to(x.dtype), t["tail_" + name]))
        held = torch.where(full, codes * scale[..., None, None], y).permute(0, 2, 3, 1, 4).reshape(n, mb * B, H, D)
        result[name] = held[seq, at].to(x.dtype)
    t["len"].copy_(lens)
    t["weight"].zero_()
    return {**result, "len": t["len"]}


def _plain_chunk(s):
    c, t = s["case"], s["cache"]
    hq, hk, d, B = c["hq"], c["hk"], c["d"], c["block"]
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    a = 0
    for b, (n, ql) in enumerate(zip(s["lens"], s["q_lens"])):  # the scores of all sequences at once would not fit
        page = t["table"][b, :, :n // B].long()
        held = []
        for name in ("k", "v"):
            x = t[name + "_codes"][page].float() * t[name + "_scale"][page][..., None, None]
            x = torch.cat((x.view(hk, -1, d), t["tail_" + name][b, :, :n % B].float()), 1)
            held.append(torch.cat((x, s[name][a:a + ql].float().transpose(0, 1)), 1) if c["how"] == "new" else x)
        k, v = held
        kl = k.shape[1]
        q = s["q"][a:a + ql].float().mul_(d ** -0.5).transpose(0, 1).reshape(hk, -1, d)
        x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(hk, hq // hk, ql, kl)
        i = torch.arange(ql, device="cuda")[:, None] + (kl - ql)
        x.masked_fill_(torch.arange(kl, device="cuda")[None, :] > i, -math.inf)
        m = x.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        x = x.sub_(m).exp_()
        total = x.sum(-1, keepdim=True)
        o = torch.bmm(x.view(hk, -1, kl), v.contiguous()).view(hk, hq // hk, ql, d)
        out[a:a + ql] = (o / torch.where(total > 0, total, torch.ones_like(total))).view(hq, ql, d).transpose(0, 1)
        lse[a:a + ql] = (m + total.log()).view(hq, ql).t()
        a += ql
    return {"out": out, "lse": lse}


_run_plain = {"norm": _plain_norm, "rotate": _plain_rotate, "append": _plain_append, "chunk": _plain_chunk}


# ---------------------------------------------------------------------------
# what a pass cannot do without

def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    c = case
    if c["kind"] == "norm":
        n, w = c["rows"] * c["d"], _size(c["weight"])
        vectors = (1 + c["post"]) * (2 if c["norm"] == "layer" else 1) + (c["gate"] == "channel")
        byte = n * (2 * _size(c["x"]) + 2 * _size(c["y"]) + (w if c["gate"] == "row" else 0)) + vectors * c["d"] * w
        return {"bytes": byte, "flops": n * (6 + 4 * c["post"] + (c["gate"] != "none"))}
    hq, hk, d = c["hq"], c["hk"], c["d"]
    lens = _ints(c["lens"])
    if c["kind"] == "rotate":
        T = sum(lens)
        return {"bytes": T * ((hq + hk) * d * 4 + 4 * len(_ints(c["axes"]))), "flops": T * (hq + hk) * 3 * c["rot"]}
    B, row = c["block"], 2 * hk * d  # keys and values of one token
    if c["kind"] == "append" and c["token"]:
        n, done = len(lens), sum((x + 1) % B == 0 for x in lens)  # tokens, and blocks that they fill
        return {"bytes": n * (hq * d * 4 + 4 * row + 16) + done * (B * row * 3 + 8 * hk),
                "flops": n * (hq + hk) * 3 * c["rot"] + done * 2 * B * row}
    if c["kind"] == "append":  # 16-bit rows read, pages written and read, rows written
        T, full, left = sum(lens), sum(x // B for x in lens), sum(x % B for x in lens)
        return {"bytes": T * (hq * d * 4 + 4 * row) + full * 2 * (B * row + 8 * hk) + left * 4 * row,
                "flops": T * ((hq + hk) * 3 * c["rot"] + 4 * row)}
    ql, new = _ints(c["q_lens"]), c["how"] == "new"
    pairs = 0
    for n, m in zip(lens, ql):
        off = n if new else n - m
        pairs += m * off + m * (m + 1) // 2 if off >= 0 else n * (n + 1) // 2
    full, left = sum(x // B for x in lens), sum(x % B for x in lens) + (sum(ql) if new else 0)
    return {"bytes": full * (B * row + 12 * hk) + left * 2 * row + sum(ql) * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    return {"norm": _exact_norm, "rotate": _exact_rotate, "append": _exact_append,
            "chunk": _exact_chunk}[case["kind"]](prepare(case, seed))


def _exact_norm(s):
    c = s["case"]

    def normed(x, weight, bias):
        mean = x.mean(1) if c["norm"] == "layer" else torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
        rms = ((x - mean[:, None]).square().mean(1) + 1e-5).sqrt()
        z = (x - mean[:, None]) / rms[:, None]
        return z * (1.0 if weight is None else weight.double()) + (0.0 if bias is None else bias.double())

    t = s["y"].double()
    t = normed(t, s["post_weight"], s["post_bias"]) if c["post"] else t
    x = s["x"].double() + c["scale"] * t * (1.0 if s["gate"] is None else s["gate"].double())
    return {"x": x, "out": normed(x, s["weight"], s["bias"])}


def _exact_turn(x, s):
    """A pair is a complex number, turned by e^(i position freq)."""
    c = s["case"]
    half = c["rot"] // 2
    first = np.cumsum([0, *_ints(c["axes"])])
    turn = torch.empty((x.shape[0], half), dtype=torch.complex128, device="cuda")
    for a in range(len(first) - 1):
        part = slice(int(first[a]), int(first[a + 1]))
        angle = torch.outer(s["positions"][a].double(), s["freq"][part].double())
        turn[:, part] = torch.polar(torch.ones_like(angle), angle)
    y = x.double().clone()
    even, odd = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["interleaved"] else (slice(0, half), slice(half, c["rot"]))
    z = torch.complex(y[:, :, even].contiguous(), y[:, :, odd].contiguous()) * turn[:, None]
    y[:, :, even], y[:, :, odd] = z.real, z.imag
    return y


def _exact_rotate(s):
    return {"q": _exact_turn(s["q"], s), "k": _exact_turn(s["k"], s)}


def _block64(x):
    """What a full block [..., block, d] reads back as: the scale and the quotient are fp32 by definition."""
    x = x.double()
    scale = (x.abs().flatten(-2).max(-1).values / 127.0).float().double()[..., None, None]
    codes = torch.round((x / scale.clamp(min=1e-300)).float().double()).clamp(-127, 127)
    return codes * scale


def _exact_append(s):
    c, t, B = s["case"], s["cache"], s["case"]["block"]
    k = _exact_turn(s["k"], s)
    result = {"q": _exact_turn(s["q"], s), "len": None}
    lens = _ints(c["lens"])
    if c["token"]:
        result |= {"tail_k": t["tail_k"].double(), "tail_v": t["tail_v"].double()}
        for b, n in enumerate(lens):
            result["tail_k"][b, :, n % B], result["tail_v"][b, :, n % B] = k[b], s["v"][b].double()
        return result
    # codes are of the keys as their 16-bit type holds them
    for name, out, x in (("k", k, k.to(s["k"].dtype)), ("v", s["v"].double(), s["v"])):
        a = 0
        for n in lens:
            full = n // B * B
            y = x[a:a + full].reshape(-1, B, c["hk"], c["d"]).transpose(1, 2)
            out[a:a + full] = _block64(y).transpose(1, 2).reshape(full, c["hk"], c["d"])
            a += n
        result[name] = out
    return result


def _exact_chunk(s):
    c, t = s["case"], s["cache"]
    B, G = c["block"], c["hq"] // c["hk"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    ends = np.cumsum(s["q_lens"])
    for b, (n, m) in enumerate(zip(s["lens"], s["q_lens"])):
        rows = slice(int(ends[b]) - m, int(ends[b]))
        for h in range(c["hk"]):
            page = t["table"][b, h, :n // B].long()
            kv = []
            for name in ("k", "v"):
                parts = [(t[name + "_codes"][page].double() * t[name + "_scale"][page].double()[:, None, None]).reshape(-1, c["d"]),
                         t["tail_" + name][b, h, :n % B].double()]
                kv.append(torch.cat(parts + ([s[name][rows, h].double()] if c["how"] == "new" else [])))
            k, v = kv
            seen = (k.shape[0] - m + 1 + torch.arange(m, device="cuda")).clamp(min=0)
            for g in range(h * G, (h + 1) * G):
                x = s["q"][rows, g].double() @ k.t() / math.sqrt(c["d"])
                x[torch.arange(k.shape[0], device="cuda")[None, :] >= seen[:, None]] = -math.inf
                e = torch.logsumexp(x, 1)
                out[rows, g] = torch.exp(x - torch.where(e.isinf(), torch.zeros_like(e), e)[:, None]) @ v
                lse[rows, g] = e
    return {"out": out, "lse": lse}
