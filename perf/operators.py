"""The attention half of a decoder layer next to the sparse FFN, as cases that
can be timed and checked.

Four kinds, all through the public binding (paper_2410_14740_amd.attention):

  prompt  attention over whole prompts: packed sequences of different lengths,
          grouped heads, causal (bottom-right aligned where keys are more or
          fewer than queries) or not
  store   a prompt's keys and values into the 8-bit cache (append), and read
          back as 16-bit rows, as the next chunk of a chunked prompt needs them
  decode  one token per sequence: its key and value appended, then its query
          attended over the cache, with the weight of every block of tokens
          added up where an eviction policy wants it
  evict   the blocks of lowest accumulated weight leave every sequence and
          head that holds more than its budget (the last block always stays)

The cache holds blocks of `block` tokens of one kv head as signed bytes with
one fp32 scale per block (s = amax / 127, q = clamp(rne(x / s))), for keys and
values apart; the tokens of a sequence's last block also stay in their 16-bit
type, and are attended from there until the block is full. Head counts and widths are those of the 7B, 13B and 70B configurations
(d_model 4096, 5120, 8192 at 128 per head; the 70B one with eight kv heads) and
of the tiny one (d_model 1024, as 16 heads of 64).

With `own` False the operators are computed by elementary torch operations in
32 bits; with `own` True by the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
HEADS = {"tiny": (16, 16, 64), "7b": (32, 32, 128), "13b": (40, 40, 128), "70b": (64, 8, 128)}
PROMPT_MOST = 64 * 128 * (8192 * 8192 + 2500 * 2500)  # heads x width x pairs of the largest prompt case
CACHE_MOST = 32 * 8 * 128 * 9000                      # sequences x heads x width x tokens of the largest cache


def _prompt(name, model, dtype, q_lens, k_lens="", causal=True):
    hq, hk, d = HEADS[model]
    return {"name": name, "kind": "prompt", "hq": hq, "hk": hk, "d": d, "dtype": dtype,
            "q_lens": q_lens, "k_lens": k_lens or q_lens, "causal": causal}


def _cache(name, kind, model, dtype, lens, block=64, **more):
    hq, hk, d = HEADS[model]
    return {"name": name, "kind": kind, "hq": hq, "hk": hk, "d": d, "dtype": dtype, "lens": lens,
            "block": block, **more}


def listed():
    return [
        # the first prompt of a small model: launch and one tile's latency
        _prompt("prompt-tiny", "tiny", "f16", "33"),
        # a served batch of ragged prompts, from one token to a long one, at 7B
        _prompt("prompt-7b-packed", "7b", "f16", "1,7,64,129,515,1000,2380"),
        # chunked prefill at 13B: chunks of new tokens against the keys so far
        _prompt("prompt-13b-chunk", "13b", "bf16", "512,300,77", "3584,1811,2400"),
        # long documents at 70B (eight query heads to a kv head)
        _prompt("prompt-70b-long", "70b", "bf16", "8192,2500"),
        # ragged 7B prompts into the cache and back
        _cache("store-7b", "store", "7b", "f16", "1,64,700,1023,2048"),
        # the same for long 70B prompts
        _cache("store-70b-long", "store", "70b", "bf16", "32768,16385,8191,4000"),
        # one token of a small model's single sequence: latency
        _cache("decode-tiny", "decode", "tiny", "f16", "100", track=False),
        # a batch of eight at 7B, as the batched FFN workload decodes
        _cache("decode-7b-b8", "decode", "7b", "f16", "191,350,511,640,1100,1535,1999,2047", track=False),
        # thirty-two ragged sequences at 70B whose blocks are weighed for eviction
        _cache("decode-70b-b32", "decode", "70b", "bf16", ",".join(
            str(500 + 517 * i + 7 * i * i) for i in range(32)), track=True),
        # one very long sequence: the length itself has to be split
        _cache("decode-70b-1x131k", "decode", "70b", "f16", "131071", track=False),
        # steady state of a budget: every sequence one block over it
        _cache("evict-7b", "evict", "7b", "f16", ",".join(str(33 * 64 + 5 * i) for i in range(8)),
               keep=32, first=1, recent=4),
        # long 70B prompts cut to a fifth
        _cache("evict-70b-long", "evict", "70b", "bf16", ",".join(
            str(131072 - 3001 * i) for i in range(32)), keep=400, first=2, recent=32),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def text(v):
        return ",".join(str(x) for x in v)

    kind = rng.choice(["prompt", "prompt", "store", "decode", "decode", "evict"])
    hk = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    hq = hk * rng.choice([g for g in (1, 2, 3, 4, 5, 8, 16) if hk * g <= 64])
    d = rng.choice([64, 128, 128])
    c = {"kind": kind, "hq": hq, "hk": hk, "d": d, "dtype": rng.choice(["f16", "bf16"])}
    n = log_int(1, 32 if kind != "prompt" else 12)
    if kind == "prompt":
        q = [log_int(1, 6000) for _ in range(n)]
        k = list(q)
        how = rng.random()
        if how < 0.3:
            k = [x + log_int(1, 4000) for x in q]
        elif how < 0.4:
            k = [rng.randint(0, 2 * x) for x in q]
            k[0] += 1
        while hq * d * sum(a * max(a, b) for a, b in zip(q, k)) > 0.5 * PROMPT_MOST:
            q, k = [max(1, x // 2) for x in q], [x // 2 for x in k]
        k[0] = max(1, k[0])
        return {**c, "q_lens": text(q), "k_lens": text(k), "causal": rng.random() < 0.8}
    block = rng.choice([32, 64, 64, 128])
    if kind == "evict":
        lens = [log_int(block, 2000 * block) for _ in range(n)]
        keep = log_int(4, max(5, max(lens) // block))
        first = rng.randint(0, keep // 4)
        return {**c, "lens": text(lens), "block": block, "keep": keep, "first": first,
                "recent": rng.randint(0, keep // 2)}
    lens = [log_int(1, 100000 if n == 1 else 16000) for _ in range(n)]
    while hk * d * n * max(lens) > 0.8 * CACHE_MOST:
        lens = [max(1, x // 2) for x in lens]
    c = {**c, "lens": text(lens), "block": block}
    return c if kind == "store" else {**c, "track": rng.random() < 0.5}


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


def _blocks_max(c):
    most = max(_ints(c["lens"]))
    return -(-(most + 1) // c["block"])


def _cache_tensors(c, seed, pages=True):
    """An empty cache whose pages lie in no order."""
    n, H, D, B, mb = len(_ints(c["lens"])), c["hk"], c["d"], c["block"], _blocks_max(c)
    P = n * H * mb
    dt = DTYPES[c["dtype"]]
    at = P if pages else 1  # an eviction moves entries of the table, not pages
    return {
        "k_codes": torch.zeros((at, B, D), dtype=torch.int8, device="cuda"),
        "v_codes": torch.zeros((at, B, D), dtype=torch.int8, device="cuda"),
        "k_scale": torch.zeros(at, device="cuda"), "v_scale": torch.zeros(at, device="cuda"),
        "tail_k": torch.zeros((n, H, B, D), dtype=dt, device="cuda"),
        "tail_v": torch.zeros((n, H, B, D), dtype=dt, device="cuda"),
        "table": torch.randperm(P, generator=_gen(seed, 1), device="cuda").int().view(n, H, mb),
        "len": torch.zeros(n, dtype=torch.int32, device="cuda"),
        "weight": torch.zeros((n, H, mb), device="cuda"),
    }


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    hq, hk, d = c["hq"], c["hk"], c["d"]
    s = {"case": c}
    if c["kind"] == "prompt":
        ql, kl = _ints(c["q_lens"]), _ints(c["k_lens"])
        if ql == kl:  # rows of one fused projection
            x = _normal(seed, 0, (sum(ql), hq + 2 * hk, d), dt)
            x[:, :hq] *= 1.5
            s |= {"q": x[:, :hq], "k": x[:, hq:hq + hk], "v": x[:, hq + hk:]}
        else:
            x = _normal(seed, 0, (sum(kl), 2 * hk, d), dt)
            s |= {"q": _normal(seed, 2, (sum(ql), hq, d), dt, 1.5), "k": x[:, :hk], "v": x[:, hk:]}
        s |= {"q_lens": ql, "k_lens": kl, "cu_q": _starts(ql), "cu_k": _starts(kl)}
        return s
    lens = _ints(c["lens"])
    n, B = len(lens), c["block"]
    t = _cache_tensors(c, seed, pages=c["kind"] != "evict")
    s["cache"] = t
    if c["kind"] == "store":
        x = _normal(seed, 2, (sum(lens), 2 * hk, d), dt)
        x[:, :, ::29] *= 4.0  # a few wide channels
        s |= {"k": x[:, :hk], "v": x[:, hk:], "cu": _starts(lens), "total": sum(lens),
              "pos": torch.zeros(n, dtype=torch.int32, device="cuda")}
    elif c["kind"] == "decode":
        for i, name in enumerate(("k", "v")):
            codes = t[name + "_codes"]
            step = max(1, (1 << 27) // (B * d))
            g = _gen(seed, 8 + i)
            for p in range(0, codes.shape[0], step):
                m = min(step, codes.shape[0] - p)
                codes[p:p + m] = torch.randn((m, B, d), generator=g, device="cuda").mul_(36).round_().clamp_(-127, 127)
            t[name + "_scale"].uniform_(0.02, 0.04, generator=g)
            t["tail_" + name].normal_(generator=g)
        t["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        held = (torch.arange(t["weight"].shape[2], device="cuda") * B)[None, :] < t["len"][:, None]
        t["weight"].uniform_(0.0, 4.0, generator=_gen(seed, 3)).mul_(held[:, None])
        x = _normal(seed, 2, (n, hq + 2 * hk, d), dt)
        x[:, :hq] *= 1.5
        s |= {"q": x[:, :hq], "k": x[:, hq:hq + hk], "v": x[:, hq + hk:], "pos": t["len"].clone(),
              "max_len": max(lens) + 1}
    else:
        t["len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        held = (torch.arange(t["weight"].shape[2], device="cuda") * B)[None, :] < t["len"][:, None]
        w = torch.randn(t["weight"].shape, generator=_gen(seed, 3), device="cuda").mul_(1.5).exp_()
        t["weight"] = w.bfloat16().float().mul_(held[:, None])  # with equal ones among them
        s["out"] = {k: torch.empty_like(t[k]) for k in ("table", "weight", "len")}
    if own:
        from paper_2410_14740_amd import attention
        s["own"] = attention.KVCache(n, hk, d, t["table"].shape[2], block_tokens=B, dtype=dt, tensors=t)
    return s


# ---------------------------------------------------------------------------
# one pass

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["kind"]](state)


def _own_prompt(s):
    from paper_2410_14740_amd import attention
    out, lse = attention.prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"],
                                          max_q=max(s["q_lens"]), causal=s["case"]["causal"], return_lse=True)
    return {"out": out, "lse": lse}


def _own_store(s):
    c = s["own"]
    c.append(s["k"], s["v"], cu=s["cu"], pos=s["pos"])
    k, v = c.read(s["cu"], s["total"])
    return {"k": k, "v": v, "len": c.len}


def _own_decode(s):
    c = s["own"]
    c.append(s["k"], s["v"], pos=s["pos"])
    out, lse = c.attend(s["q"], max_len=s["max_len"], track=s["case"]["track"], return_lse=True)
    return _decoded(out, lse, s)


def _decoded(out, lse, s):
    t = s["cache"]
    r = {"out": out, "lse": lse, "len": t["len"], "tail_k": t["tail_k"], "tail_v": t["tail_v"]}
    return {**r, "weight": t["weight"]} if s["case"]["track"] else r


def _own_evict(s):
    c = s["case"]
    s["own"].evict(c["keep"], c["first"], c["recent"], out=s["out"])
    return s["out"]


_run_own = {"prompt": _own_prompt, "store": _own_store, "decode": _own_decode, "evict": _own_evict}


def _softmax_rows(x):
    """(exp(x - max), its row sums, ln sum exp) along the last axis; a row of -inf alone gives zeros and -inf."""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    return x, total, (m + total.log()).squeeze(-1)


def _plain_prompt(s):
    c = s["case"]
    hq, hk, d = c["hq"], c["hk"], c["d"]
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    q0 = k0 = 0
    for ql, kl in zip(s["q_lens"], s["k_lens"]):  # the scores of all sequences at once would not fit
        q = s["q"][q0:q0 + ql].float().mul_(d ** -0.5).transpose(0, 1).reshape(hk, -1, d)
        if kl == 0:
            out[q0:q0 + ql], lse[q0:q0 + ql] = 0, -math.inf
            q0 += ql
            continue
        k = s["k"][k0:k0 + kl].float().permute(1, 2, 0).contiguous()
        v = s["v"][k0:k0 + kl].float().transpose(0, 1).contiguous()
        x = torch.bmm(q, k).view(hk, hq // hk, ql, kl)
        if c["causal"]:
            i = torch.arange(ql, device="cuda")[:, None] + (kl - ql)
            x.masked_fill_(torch.arange(kl, device="cuda")[None, :] > i, -math.inf)
        p, total, e = _softmax_rows(x)
        o = torch.bmm(p.view(hk, -1, kl), v).view(hq, ql, d)
        total = total.view(hq, ql, 1)
        out[q0:q0 + ql] = (o / torch.where(total > 0, total, torch.ones_like(total))).transpose(0, 1)
        lse[q0:q0 + ql] = e.view(hq, ql).t()
        q0, k0 = q0 + ql, k0 + kl
    return {"out": out, "lse": lse}


def _quantized(x):
    """Codes and scales of fp32 blocks [..., block, d]."""
    scale = x.abs().amax((-1, -2)) / 127.0
    div = torch.where(scale > 0, scale, torch.ones_like(scale))[..., None, None]
    return (x / div).round_().clamp_(-127, 127), scale


def _plain_store(s):
    c, t = s["case"], s["cache"]
    n, H, mb = t["table"].shape
    B, D = c["block"], c["d"]
    cu = s["cu"].long()
    lens = cu[1:] - cu[:-1]
    row = cu[:-1, None] + torch.arange(mb * B, device="cuda")
    full = (torch.arange(mb, device="cuda") < (lens // B)[:, None])[:, None, :, None, None]
    table = t["table"].long()
    last = (lens - 1).clamp(min=0)
    tail = (last // B)[:, None, None, None, None].expand(n, H, 1, B, D)
    at = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(cu[1:], at, right=True)
    at = at - cu[seq]
    in_tail = (torch.arange(B, device="cuda") <= (last % B)[:, None])[:, None, :, None]
    result = {}
    for name in ("k", "v"):
        x = s[name][row.clamp(max=s["total"] - 1)].float().view(n, mb, B, H, D).permute(0, 3, 1, 2, 4)
        codes, scale = _quantized(x)
        rest = x.gather(2, tail).squeeze(2)
        t[name + "_codes"][table] = torch.where(full, codes.char(), t[name + "_codes"][table])
        t[name + "_scale"][table] = torch.where(full[..., 0, 0], scale, t[name + "_scale"][table])
        t["tail_" + name].copy_(torch.where(in_tail, rest.to(t["tail_" + name].dtype), t["tail_" + name]))
        dense = torch.where(full, codes * scale[..., None, None], x).permute(0, 2, 3, 1, 4).reshape(n, mb * B, H, D)
        result[name] = dense[seq, at].to(s[name].dtype)
    t["len"].copy_(s["pos"] + lens)
    t["weight"].zero_()
    return {**result, "len": t["len"]}


def _plain_decode(s):
    c, t = s["case"], s["cache"]
    n, H, mb = t["table"].shape
    B, D, G = c["block"], c["d"], c["hq"] // c["hk"]
    pos = s["pos"].long()
    blk, off = pos // B, pos % B
    table, rows = t["table"].long(), torch.arange(n, device="cuda")
    done = (off == B - 1)[:, None]
    page = table[rows, :, blk]
    for name in ("k", "v"):
        t["tail_" + name][rows, :, off] = s[name]
        codes, scale = _quantized(t["tail_" + name].float())
        t[name + "_codes"][page] = torch.where(done[..., None, None], codes.char(), t[name + "_codes"][page])
        t[name + "_scale"][page] = torch.where(done, scale, t[name + "_scale"][page])
    t["len"].copy_(pos + 1)
    t["weight"][rows, :, blk] *= (off != 0)[:, None]  # a block that this token opens has no weight yet
    used = -(-s["max_len"] // B)
    nb, left = t["len"].long() // B, t["len"].long() % B
    idx = torch.arange(used, device="cuda")
    is_open = (idx == nb[:, None])[:, None, :, None, None]

    def dense(name):
        x = t[name + "_codes"][table[:, :, :used]].float().mul_(t[name + "_scale"][table[:, :, :used]][..., None, None])
        return torch.where(is_open, t["tail_" + name].float()[:, :, None], x).view(n * H, used * B, D)

    at = torch.arange(used * B, device="cuda")
    hide = at[None, :] >= (nb * B + left)[:, None]
    q = s["q"].float().mul_(D ** -0.5).view(n * H, G, D)
    x = torch.bmm(q, dense("k").transpose(1, 2).contiguous()).view(n, H, G, used * B)
    x.masked_fill_(hide[:, None, None, :], -math.inf)
    p, total, lse = _softmax_rows(x)
    p.div_(total)
    v = dense("v").masked_fill_(hide[:, None, :, None].expand(n, H, used * B, 1).reshape(n * H, used * B, 1), 0)
    out = torch.bmm(p.view(n * H, G, -1), v).view(n, c["hq"], D).to(s["q"].dtype)
    if c["track"]:
        t["weight"][:, :, :used] += p.view(n, H, G, used, B).sum((2, 4))
    return _decoded(out, lse.view(n, c["hq"]), s)


def _plain_evict(s):
    c, t = s["case"], s["cache"]
    n, H, mb = t["table"].shape
    nb = ((t["len"].long() - 1).clamp(min=0) // c["block"])[:, None, None]  # the last block stays
    i = torch.arange(mb, device="cuda").view(1, 1, mb)
    u = t["weight"].view(torch.int32).long()
    key = torch.where(u < 0, -1 - u - (1 << 31), u)  # the order of the bit patterns
    key = torch.where((i < c["first"]) | (i >= nb - c["recent"]), torch.full_like(key, 1 << 40), key)
    key = torch.where(i >= nb, torch.full_like(key, -(1 << 40)), key)
    order = torch.sort(key, dim=2, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, i.expand(n, H, mb))
    keep = torch.minimum(nb, torch.full_like(nb, c["keep"]))
    gone = (i < nb) & (rank >= keep)
    group = torch.where(gone, 2, torch.where(i < nb, 0, 1))  # kept, last and unused, evicted
    new = torch.sort(group, dim=2, stable=True).indices
    return {"table": t["table"].gather(2, new), "weight": t["weight"].masked_fill(gone, 0).gather(2, new),
            "len": t["len"] - ((nb - keep).view(n) * c["block"]).int()}


_run_plain = {"prompt": _plain_prompt, "store": _plain_store, "decode": _plain_decode, "evict": _plain_evict}


# ---------------------------------------------------------------------------
# what a pass cannot do without

def _pairs(ql, kl, causal):
    """(query, key) pairs that a bottom-right aligned causal mask leaves."""
    if not causal:
        return ql * kl
    return sum(max(0, kl - ql + i + 1) for i in range(ql)) if kl < ql else ql * (kl - ql) + ql * (ql + 1) // 2


def work(case):
    c = case
    hq, hk, d = c["hq"], c["hk"], c["d"]
    if c["kind"] == "prompt":
        ql, kl = _ints(c["q_lens"]), _ints(c["k_lens"])
        pairs = sum(_pairs(a, b, c["causal"]) for a, b in zip(ql, kl))
        return {"bytes": sum(ql) * hq * (4 * d + 4) + sum(kl) * hk * 4 * d, "flops": 4 * d * hq * pairs}
    lens = _ints(c["lens"])
    n, B = len(lens), c["block"]
    rows = 2 * hk * d  # keys and values of one token
    if c["kind"] == "store":  # 16-bit rows read, pages written and read, rows written
        full = sum(x // B for x in lens)
        left = sum(x % B for x in lens)
        return {"bytes": sum(lens) * 4 * rows + full * 2 * (B * rows + 8 * hk) + left * 4 * rows,
                "flops": 4 * sum(lens) * rows}
    if c["kind"] == "decode":
        full, left = sum((x + 1) // B for x in lens), sum((x + 1) % B for x in lens)
        byte = full * (B * rows + 12 * hk) + left * 2 * rows + n * 4 * rows + n * hq * (4 * d + 4)
        return {"bytes": byte + (8 * hk * sum(-(-(x + 1) // B) for x in lens) if c["track"] else 0),
                "flops": 4 * d * hq * (sum(lens) + n)}
    return {"bytes": n * hk * _blocks_max(c) * 16 + 8 * n, "flops": n * hk * _blocks_max(c)}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    return {"prompt": _exact_prompt, "store": _exact_store, "decode": _exact_decode,
            "evict": _exact_evict}[case["kind"]](prepare(case, seed))


def _attention64(q, k, v, seen):
    """One head in 64 bits: q [m][d], k and v [l][d]; row i sees the first seen[i] keys."""
    x = q.double() @ k.double().t() * (1.0 / math.sqrt(q.shape[1]))
    x[torch.arange(k.shape[0], device="cuda")[None, :] >= seen[:, None]] = -math.inf
    lse = torch.logsumexp(x, 1)
    w = torch.exp(x - torch.where(lse.isinf(), torch.zeros_like(lse), lse)[:, None])
    return w @ v.double(), lse, w


def _exact_prompt(s):
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    cq, ck = np.cumsum([0, *s["q_lens"]]), np.cumsum([0, *s["k_lens"]])
    for b, (ql, kl) in enumerate(zip(s["q_lens"], s["k_lens"])):
        if kl == 0:
            continue
        seen = torch.full((ql,), kl, device="cuda")
        if c["causal"]:
            seen = (kl - ql + 1 + torch.arange(ql, device="cuda")).clamp(min=0)
        for h in range(c["hq"]):
            g = h // (c["hq"] // c["hk"])
            o, e, _ = _attention64(s["q"][cq[b]:cq[b + 1], h], s["k"][ck[b]:ck[b + 1], g],
                                   s["v"][ck[b]:ck[b + 1], g], seen)
            out[cq[b]:cq[b + 1], h], lse[cq[b]:cq[b + 1], h] = o, e
    return {"out": out, "lse": lse}


def _block64(x):
    """What a full block [..., block, d] reads back as: the scale and the quotient are fp32 by definition."""
    x = x.double()
    scale = (x.abs().flatten(-2).max(-1).values / 127.0).float().double()[..., None, None]
    codes = torch.round((x / scale.clamp(min=1e-300)).float().double()).clamp(-127, 127)
    return codes * scale


def _exact_store(s):
    c, B = s["case"], s["case"]["block"]
    lens = _ints(c["lens"])
    result = {"len": None}
    for name in ("k", "v"):
        out = s[name].double()
        a = 0
        for n in lens:
            full = n // B * B
            x = s[name][a:a + full].reshape(-1, B, c["hk"], c["d"]).transpose(1, 2)
            out[a:a + full] = _block64(x).transpose(1, 2).reshape(full, c["hk"], c["d"])
            a += n
        result[name] = out
    return result


def _exact_decode(s):
    c, t = s["case"], s["cache"]
    B, G = c["block"], c["hq"] // c["hk"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    weight = t["weight"].double()
    for b, n in enumerate(_ints(c["lens"])):
        blocks, rest = n // B, n % B
        for h in range(c["hk"]):
            page = t["table"][b, h, :blocks].long()
            kv = []
            for name in ("k", "v"):
                old = t[name + "_codes"][page].double() * t[name + "_scale"][page].double()[:, None, None]
                last = torch.cat([t["tail_" + name][b, h, :rest], s[name][b, h][None]]).double()
                last = _block64(last) if rest == B - 1 else last
                kv.append(torch.cat([old.reshape(-1, c["d"]), last]))
            o, e, w = _attention64(s["q"][b, h * G:(h + 1) * G], kv[0], kv[1],
                                   torch.full((G,), n + 1, device="cuda"))
            out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = o, e
            by = torch.nn.functional.pad(w.sum(0), (0, -(n + 1) % B)).view(-1, B).sum(1)
            weight[b, h, :by.numel()] += by
    r = {"out": out, "lse": lse, "len": None, "tail_k": None, "tail_v": None}
    return {**r, "weight": weight} if c["track"] else r


def _exact_evict(s):
    c, t = s["case"], s["cache"]
    w = t["weight"].cpu().numpy()
    got = np.zeros(w.shape, np.float64)
    for b, n in enumerate(_ints(c["lens"])):
        nb = (n - 1) // c["block"]
        for h in range(c["hk"]):
            row = w[b, h]
            kept = np.arange(nb)
            if nb > c["keep"]:
                middle = np.arange(c["first"], nb - c["recent"])
                best = middle[np.lexsort((middle, -row[middle]))][:c["keep"] - c["first"] - c["recent"]]
                kept = np.concatenate([kept[:c["first"]], np.sort(best), kept[nb - c["recent"]:]])
            got[b, h, :kept.size] = row[kept]
            got[b, h, kept.size:kept.size + row.size - nb] = row[nb:]
    return {"table": None, "weight": torch.from_numpy(got), "len": None}
