"""Edges of the attention calls. The bounds are those of test_gpu_attention.py."""
import math

import numpy as np
import pytest
import torch

from helpers import say
from paper_2410_14740_amd import m2c
from paper_2410_14740_amd.attention import KVCache, prompt_attention
from test_gpu_attention import BF16, F16, SPLITS, check_attend, check_prompt, rand, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [192, 200])
@pytest.mark.parametrize("qs,ks,scale", [(1e-34, 1e34, 0.2), (1e-36, 1e36, 0.2), (1e-38, 2e37, 1.0)])
def test_attend_tiny_queries(qs, ks, scale, n):
    """bf16 queries down to the type's subnormal numbers, and keys that give
    them scores of some units."""
    say(f"attend tiny queries {qs} {n}")
    c = KVCache(1, 2, 64, 4, dtype=BF16)
    c.append(rand((n, 2, 64), BF16, 301, ks), rand((n, 2, 64), BF16, 302), cu=starts([n]))
    q = rand((1, 6, 64), BF16, 303, qs)
    out, lse = c.attend(q, scale=scale, return_lse=True)
    check_attend(c, q, out, lse, [0], scale=scale)


def item_before_the_first(cu, per, more, total):
    """Some work item of packed sequences falls before the first item of the
    sequence that a count of the starts at or before it names."""
    first = [c // per + b * more for b, c in enumerate(cu[:-1])]
    for x in range(total // per + (len(cu) - 1) * more):
        b = sum(f <= x for f in first) - 1
        if b >= 0 and x < first[b] and cu[b + 1] > cu[b]:
            return True
    return False


BACKWARDS = [[0, 1000, 1100, 10, 20], [5, 1000, 1064, 0, 300, 20], [64, 900, 1000, 3, 1100, 2]]


@pytest.mark.parametrize("cu", BACKWARDS)
def test_starts_that_do_not_ascend_stay_in_range(cu):
    """They are the caller's mistake: the call says so, and touches no other
    sequence's page, tail, weight or length and no row outside its arrays."""
    say(f"starts that do not ascend {cu}")
    H, d, B, T, n = 2, 64, 64, 1100, len(cu) - 1
    assert item_before_the_first(cu, B, 2, T) and item_before_the_first(cu, B, 1, T)
    starts_ = torch.tensor(cu, dtype=torch.int32, device="cuda")
    seqs = torch.tensor([1, 3, 5, 7, 9][:n], dtype=torch.int32, device="cuda")
    others = [0, 2, 4, 6, 8, 10] + [9] * (n < 5)
    c = KVCache(11, H, d, 20, block_tokens=B)
    c.append(rand((11 * 70, H, d), F16, 310), rand((11 * 70, H, d), F16, 311), cu=starts([70] * 11))
    c.check()
    c.weight.fill_(3.0)
    pages = c.table[others].long()

    def held():
        rows = {"table": c.table, **{name: getattr(c, name)[others] for name in ("len", "weight", "tail_k", "tail_v")},
                **{name: getattr(c, name)[pages] for name in ("k_codes", "v_codes", "k_scale", "v_scale")}}
        return {name: t.contiguous().view(torch.uint8).clone() for name, t in rows.items()}  # unused places hold anything

    def same():
        now = held()
        return all(torch.equal(now[name], before[name]) for name in now)

    before = held()
    room = rand((T + 400, H, d), F16, 312)
    c.append(room[200:200 + T], room[200:200 + T], cu=starts_, seqs=seqs)
    with pytest.raises(m2c.M2CError) as e:
        c.check()
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and "ascend" in str(e.value)
    assert same()
    k, v = (torch.full((T + 4000, H, d), 9.0, dtype=F16, device="cuda") for _ in range(2))
    c.read(starts_, seqs=seqs, k=k[2000:2000 + T], v=v[2000:2000 + T])
    with pytest.raises(m2c.M2CError) as e:
        c.check()
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and "ascend" in str(e.value)
    for t in (k, v):
        assert bool((t[:2000] == 9).all()) and bool((t[2000 + T:] == 9).all())
    assert same()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("many", [False, True])
def test_prompt_starts_that_do_not_ascend_stay_in_range(many, causal):
    say(f"prompt starts that do not ascend {many} {causal}")
    hq, d, T = 2, 64, 3000
    cu = [0, 2000, 2500, 10, 20] if not many else [0, 2000, 2500, 10, 20] + [20 + 7 * i for i in range(80)]
    assert item_before_the_first([2 * c for c in cu], 128, 1, 2 * T)
    room = torch.full((T + 8000, hq, d), 9.0, dtype=F16, device="cuda")
    x = torch.zeros((T + 8000, hq, d), dtype=F16, device="cuda")
    q = x[4000:4000 + T]
    starts_ = torch.tensor(cu, dtype=torch.int32, device="cuda")
    for cu_k in (starts_, torch.zeros_like(starts_)):
        prompt_attention(q, q[:, :1], q[:, :1], starts_, cu_k, causal=causal, out=room[4000:4000 + T])
        torch.cuda.synchronize()
        assert bool((room[:4000] == 9).all()) and bool((room[4000 + T:] == 9).all())


@pytest.mark.parametrize("n,hq,hk,d,dt,longest,hints", [
    (70, 16, 8, 64, F16, 9000, (9000, 0)),      # chunks of 16 units
    (66, 8, 8, 128, BF16, 30000, (30000,)),     # larger ones
    (65, 40, 2, 64, BF16, 20000, (20000, 700)),  # two tiles of heads, a hint far too short
    (66, 128, 128, 64, F16, 16500, (16500,)),   # whole rows of more units than a wave's lanes hold at once
])
def test_attend_more_sequences_than_lanes(n, hq, hk, d, dt, longest, hints):
    say(f"attend {n} sequences {hq}/{hk}x{d} {dt} up to {longest}")
    lens = [(53 * i) % 200 if i % 5 else i % 3 for i in range(n)]
    lens[n // 2], lens[n - 2] = longest, longest // 3
    if hk == 128:
        lens = [min(x, 70) for x in lens]
        lens[n // 2] = longest
    c = KVCache(n, hk, d, longest // 64 + 2, dtype=dt, n_pages=sum(x // 64 for x in lens) * hk + 1)
    pages = torch.randperm(c.k_codes.shape[0], generator=torch.Generator().manual_seed(320)).int().cuda()
    c.table.fill_(-1)
    at = 0
    for b, x in enumerate(lens):
        c.table[b, :, :x // 64] = pages[at:at + x // 64 * hk].view(hk, x // 64)
        at += x // 64 * hk
    c.append(rand((sum(lens), hk, d), dt, 321), rand((sum(lens), hk, d), dt, 322), cu=starts(lens))
    q = rand((n, hq, d), dt, 323, 1.5)
    some = sorted({0, 1, 5, n // 2, n // 2 + 1, n - 2, n - 1})
    for hint in hints:
        for track in (False, True):
            before = c.weight.clone()
            out, lse = c.attend(q, max_len=hint, track=track, return_lse=True)
            c.check()
            check_attend(c, q[some], out[some], lse[some], some, before=before if track else None)
            assert track or torch.equal(c.weight, before)
            assert bool((out[[i for i, x in enumerate(lens) if x == 0]] == 0).all())


def call_desc(q, k, v, out, causal):
    d = m2c.AttnDesc(m2c.DTYPE_BF16 if q.dtype == BF16 else m2c.DTYPE_FP16, q.shape[1], k.shape[1], q.shape[2], causal, 0,
                     0.0, 0)
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        setattr(d, name + "_stride", t.stride()[:2])
    return d


@pytest.mark.parametrize("hq,hk,d,dt,ql,kl,causal", SPLITS)
def test_rows_of_few_queries_are_cut(hq, hk, d, dt, ql, kl, causal):
    """The plan on the device cuts some row of each of these calls: the first
    word of the workspace says so."""
    say(f"prompt is cut {hq}/{hk}x{d} {dt} {ql} {kl}")
    q, k, v = rand((sum(ql), hq, d), dt, 330, 1.5), rand((sum(kl), hk, d), dt, 331), rand((sum(kl), hk, d), dt, 332)
    out, cu, ck = torch.empty_like(q), starts(ql), starts(kl)
    desc = call_desc(q, k, v, out, causal)
    room = torch.zeros(m2c.m2c_prompt_attention_workspace(desc, cu, ck, len(ql), sum(ql), sum(kl)), dtype=torch.uint8,
                       device="cuda")
    desc.workspace, desc.workspace_bytes = room.data_ptr(), room.numel()
    m2c.m2c_prompt_attention(desc, q, k, v, cu, ck, len(ql), sum(ql), sum(kl), out)
    assert int(room[:4].view(torch.int32)) != 0
    check_prompt(q, k, v, ql, kl, causal, out, None)


@pytest.mark.parametrize("layout", ["fused", "head_major", "padded", "shared_row"])
@pytest.mark.parametrize("dt,d", [(F16, 128), (BF16, 64)])
def test_prompt_cut_strides(layout, dt, d):
    """Rows cut along their keys: a part's start, the join's and whole rows'
    writes with strides of their own."""
    hq, hk, ql, kl = 4, 2, [33, 3, 140], [3000, 1500, 900]
    tq, tk = sum(ql), sum(kl)
    say(f"prompt cut strides {layout} {dt}")
    if layout == "fused":
        x = rand((tk, 2 * hk + 1, d), dt, 340)
        k, v = x[:, :hk], x[:, hk:2 * hk]
        q = rand((tq, hq + 2 * hk, d), dt, 341)[:, :hq]
        out = torch.zeros((tq, hq + 3, d), dtype=dt, device="cuda")[:, 1:1 + hq]
    elif layout == "head_major":
        q, k, v = (rand((h, n, d), dt, 342 + i).transpose(0, 1) for i, (h, n) in enumerate(((hq, tq), (hk, tk), (hk, tk))))
        out = torch.zeros((hq, tq, d), dtype=dt, device="cuda").transpose(0, 1)
    elif layout == "padded":
        q, k, v = (rand((n, h, d + 24), dt, 345 + i)[:, :, 8:8 + d] for i, (h, n) in enumerate(((hq, tq), (hk, tk), (hk, tk))))
        out = torch.zeros((tq, hq, d + 8), dtype=dt, device="cuda")[:, :, :d]
    else:
        q = rand((tq, hq, d), dt, 348)
        k, v = (rand((tk, 1, d), dt, 349 + i).expand(tk, hk, d) for i in range(2))
        out = torch.zeros((tq, hq, d), dtype=dt, device="cuda")
    whole = out._base if out._base is not None else out
    got, lse = prompt_attention(q, k, v, starts(ql), starts(kl), out=out, return_lse=True)
    assert got is out
    check_prompt(q, k, v, ql, kl, True, out, lse)
    beside = torch.ones_like(whole, dtype=torch.bool)
    beside.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool((whole[beside] == 0).all())
    # a key in the last part that no row but the last ones of its sequence sees
    k2, v2 = k.clone(), v.clone()
    k2[kl[0] - 9], v2[kl[0] - 9] = math.nan, math.inf
    prompt_attention(q, k2, v2, starts(ql), starts(kl), out=out)
    blind = ql[0] - 9
    check_prompt(q[:blind], k[:kl[0] - 9], v[:kl[0] - 9], [blind], [kl[0] - 9], True, out[:blind], None)
    assert not torch.isfinite(out[blind:ql[0]].float()).any()
    check_prompt(q[ql[0]:], k[kl[0]:], v[kl[0]:], ql[1:], kl[1:], True, out[ql[0]:], None)


def test_prompt_cut_extreme_scores():
    say("prompt cut extreme scores")
    d, ql, kl = 64, [40], [4000]
    for dt in (F16, BF16):
        q, k, v = rand((40, 2, d), dt, 351, 30.0), rand((4000, 2, d), dt, 352, 30.0), rand((4000, 2, d), dt, 353)
        for scale in (None, 0.7, 1e-6):
            out, lse = prompt_attention(q, k, v, starts(ql), starts(kl), scale=scale, return_lse=True)
            check_prompt(q, k, v, ql, kl, True, out, lse, scale=scale)


@pytest.mark.parametrize("dt,d", [(F16, 128), (BF16, 64)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_prompt_values_that_are_seen_enter_every_row(dt, d, what):
    """A value that is not finite reaches all rows and heads that see its key."""
    say(f"prompt seen {what} {dt}")
    q, k, v = rand((200, 4, d), dt, 360), rand((200, 2, d), dt, 361), rand((200, 2, d), dt, 362)
    v[157] = what
    for causal in (True, False):
        out = prompt_attention(q, k, v, starts([200]), causal=causal)
        sees = 157 if causal else 0
        assert not torch.isfinite(out[sees:].float()).any()
        assert bool(torch.isfinite(out[:sees].float()).all())


def test_codes_of_subnormal_blocks():
    """Blocks whose largest magnitude is a subnormal number of their type; bf16's
    then have subnormal scales, of 516 of the smallest fp32 number or more, and
    the largest quotient is up to 127 (1 + 2^-10), which rounds to 127 still."""
    say("codes of subnormal blocks")
    B, D = 32, 64
    for dt, bits in ((F16, 10), (BF16, 7)):
        n = 1 << bits
        tops = torch.arange(1, n, dtype=torch.int32) if dt == BF16 else torch.arange(1, n, 5, dtype=torch.int32)
        mags = torch.arange(B * D, dtype=torch.int32)[None] % (tops[:, None] + 1)  # 0 .. the largest, again and again
        mags[:, 0] = tops
        mags[:, 1::2] |= 0x8000
        x = mags.to(torch.int16).view(dt).view(-1, 1, D)
        T = x.shape[0]
        c = KVCache(1, 1, D, T // B, block_tokens=B, dtype=dt)
        c.append(x.cuda(), x.cuda(), cu=starts([T]))
        c.check()
        f = x.float().view(-1, B * D).numpy()
        s = np.abs(f).max(1, keepdims=True) / np.float32(127)
        q = f / s
        assert np.abs(q).max() < 127.5
        for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)):
            assert np.array_equal(scale.cpu().numpy(), s[:, 0])
            assert np.array_equal(codes.view(-1, B * D).cpu().numpy(), np.rint(q).astype(np.int8))
        k, _ = c.read(starts([T]), T)
        want = torch.from_numpy(np.rint(q).astype(np.float32) * s).to(dt).view(-1, 1, D)
        assert torch.equal(k.cpu().view(torch.int16) & 0x7fff, want.view(torch.int16) & 0x7fff)
