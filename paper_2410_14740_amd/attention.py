"""Attention of a decoder layer next to the sparse FFN, on torch tensors.

`prompt_attention` attends over whole packed prompts; `KVCache` holds keys and
values in 8 bits, block by block (`append`, `read`), attends single tokens over
them (`attend`) and drops the blocks of least accumulated weight (`evict`). The
work is done by libm2c.so (include/m2c.h has the definitions); this module
checks tensors and passes addresses.

Every call only enqueues on `stream` (default: torch's current stream) and
returns. Tensors of a call must stay alive, and not be written elsewhere, until
its work is done; for outputs that a call allocates torch's allocator sees to
that on the stream of the call.
"""
from __future__ import annotations

import torch

from . import m2c

_DTYPES = {torch.float16: m2c.DTYPE_FP16, torch.bfloat16: m2c.DTYPE_BF16}
_I64x2 = m2c._I64x2
_check = m2c._check
# the address of a device's current stream without building a Stream object,
# which takes as long as a launch
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _raw(stream, device):
    if stream is None:
        return _current(device.index)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _alloc(stream, device, *wanted):
    """Tensors (shape, dtype) that torch's allocator keeps for `stream`."""
    if stream is None:
        return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in wanted]
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in wanted]


def _like(q, stream):
    """An output like q, contiguous (the usual case by the shorter call)."""
    if stream is None and q.is_contiguous():
        return torch.empty_like(q)
    return _alloc(stream, q.device, (q.shape, q.dtype))[0]


def _address(t):
    return None if t is None else t.data_ptr()


def _bad(msg):
    raise m2c.M2CError(m2c.M2C_ERR_INVALID_ARG, msg)


def _rows(name, t, dtype, device, heads, dim):
    """Strides (tokens, heads) of rows [tokens][heads][dim]."""
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        _bad(f"{name}: shape {tuple(shape)}, need [tokens, {heads}, {dim}]")
    if t.dtype != dtype or t.device != device:
        _bad(f"{name}: {t.dtype} on {t.device}, need {dtype} on {device}")
    a, b, c = t.stride()
    if c != 1:
        _bad(f"{name}: the elements of a head must be contiguous")
    return _I64x2(a if shape[0] > 1 else dim, b if heads > 1 else 0)  # a single row's stride is free


def _ints(name, t, n, device):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != n or t.device != device or \
            not t.is_contiguous():
        _bad(f"{name}: need a contiguous int32 tensor of {n} on {device}")
    return t


_prompt_need = {}  # workspace bytes by call shape


def prompt_attention(q, k, v, cu_q, cu_k=None, max_q=0, causal=True, scale=None, out=None,
                     return_lse=False, stream=None):
    """Attention of packed prompts.

    q [total_q, n_heads, head_dim]; k, v [total_k, n_kv_heads, head_dim], fp16 or
    bf16, any token and head strides that are multiples of 8 elements (rows of
    a fused projection, for example). cu_q, cu_k: int32 [sequences + 1] row
    starts (cu_k None: the same). causal: query i of lq sees keys 0 .. lk - lq
    + i of its sequence. max_q: longest query sequence if known (a hint
    for whether rows are split along their keys).
    scale: of q.k, None or 0 for 1 / sqrt(head_dim).
    Returns out like q (contiguous unless given), or (out, lse) with lse fp32
    [total_q, n_heads] = ln sum exp(scale q.k)."""
    if q.dim() != 3 or k.dim() != 3 or q.dtype not in _DTYPES or not q.is_cuda:
        _bad("q, k, v: need fp16 or bf16 GPU tensors [tokens, heads, head_dim]")
    dev, (tq, hq, d), hk = q.device, q.shape, k.shape[1]
    if v.shape != k.shape:
        _bad(f"v: shape {tuple(v.shape)}, k has {tuple(k.shape)}")
    n = cu_q.shape[0] - 1 if cu_q.dim() == 1 else 0
    if n < 1:
        _bad("cu_q: need the row starts of at least one sequence and the end")
    _ints("cu_q", cu_q, n + 1, dev)
    cu_k = cu_q if cu_k is None else _ints("cu_k", cu_k, n + 1, dev)
    dt, tk = q.dtype, k.shape[0]
    if out is None:
        out, out_strides = _like(q, stream), _I64x2(hq * d, d)
    elif out.shape != q.shape:
        _bad(f"out: shape {tuple(out.shape)}, need {tuple(q.shape)}")
    else:
        out_strides = _rows("out", out, dt, dev, hq, d)
    lse = _alloc(stream, dev, ((tq, hq), torch.float32))[0] if return_lse else None
    desc = m2c.AttnDesc(_DTYPES[dt], hq, hk, d, 1 if causal else 0, dev.index,
                        0.0 if scale is None else scale, max_q, _rows("q", q, dt, dev, hq, d),
                        _rows("k", k, dt, dev, hk, d), _rows("v", v, dt, dev, hk, d),
                        out_strides)
    starts, key_starts = cu_q.data_ptr(), cu_k.data_ptr()
    key = (n, tq, tk, max_q, hq, hk, d, starts == key_starts)
    need = _prompt_need.get(key)
    if need is None:
        if len(_prompt_need) >= 4096:
            _prompt_need.clear()
        need = _prompt_need[key] = m2c.m2c_prompt_attention_workspace(desc, cu_q, cu_k, n, tq, tk)
    if need:
        work, = _alloc(stream, dev, ((need,), torch.uint8))
        desc.workspace, desc.workspace_bytes = work.data_ptr(), need
    _check(m2c.load().m2c_prompt_attention(
        desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), starts, key_starts, n, tq, tk, out.data_ptr(),
        _address(lse), _raw(stream, dev)))
    return (out, lse) if return_lse else out


class Rotary:
    """How positions turn the pairs of a head's first 2 len(freq) elements.

    freq: fp32 GPU tensor [pairs], a multiple of 8, radians per position of each
    pair. sections: pairs of each axis of a position, in order (default: one axis).
    interleaved: pair i is elements 2i and 2i + 1, not i and i + pairs. scale:
    a factor of the turned elements."""

    def __init__(self, freq, sections=None, interleaved=False, scale=1.0):
        if freq.dim() != 1 or freq.dtype != torch.float32 or not freq.is_cuda or not freq.is_contiguous():
            _bad("freq: need a contiguous fp32 GPU tensor [pairs]")
        pairs = freq.shape[0]
        sections = [pairs] if sections is None else list(sections)
        if pairs % 8 or not 8 <= pairs <= 64:
            _bad(f"freq: {pairs} pairs, need a multiple of 8, 8 to 64")
        if not 1 <= len(sections) <= 4 or min(sections) < 0 or sum(sections) != pairs:
            _bad(f"sections {sections}: need 1 to 4 counts of pairs, {pairs} in all")
        if not 0.0 < abs(scale) <= 1e30:
            _bad(f"scale {scale}: need a finite number other than 0")
        self.freq, self.axes = freq, len(sections)
        self.desc = m2c.RotaryDesc(2 * pairs, 1 if interleaved else 0, len(sections),
                                   (m2c.ctypes.c_int32 * 4)(*sections), scale, freq.data_ptr())

    def _positions(self, positions, rows, device):
        """Address and axis stride of checked positions."""
        want = (rows,) if self.axes == 1 and positions.dim() == 1 else (self.axes, rows)
        if positions.shape != want or positions.dtype != torch.int32 or positions.device != device or \
                self.freq.device != device or (rows > 1 and positions.stride(-1) != 1):
            _bad(f"positions: {positions.dtype} {tuple(positions.shape)} on {positions.device}, need int32 "
                 f"{want} on {device}, as freq is, the coordinates of an axis contiguous")
        return positions.data_ptr(), (positions.stride(0) if self.axes > 1 else rows)

    def rotate(self, q, positions, k=None, q_out=None, k_out=None, stream=None):
        """q [tokens, n_heads, head_dim], and k [tokens, n_kv_heads, head_dim] if
        given, turned by positions (int32 [axes, tokens], or [tokens] for one axis).
        q_out, k_out: what gets them (may be q and k; allocated if not given).
        Returns q_out, or (q_out, k_out) where k is given."""
        if q.dim() != 3 or q.dtype not in _DTYPES or not q.is_cuda:
            _bad("q: need an fp16 or bf16 GPU tensor [tokens, heads, head_dim]")
        dev, (n, hq, d) = q.device, q.shape
        at, step = self._positions(positions, n, dev)
        q_out, qs, qos = _turned("q", q, q_out, n, hq, d, q.dtype, dev, stream)
        hk, ks, kos = 0, _NONE, _NONE
        if k is not None:
            hk = k.shape[1] if k.dim() == 3 else 0
            k_out, ks, kos = _turned("k", k, k_out, n, hk, d, q.dtype, dev, stream)
        elif k_out is not None:
            _bad("k_out: there is no k")
        _check(m2c.load().m2c_rotate(self.desc, _DTYPES[q.dtype], d, dev.index, n, at, step, hq, q.data_ptr(), qs,
                                     q_out.data_ptr(), qos, hk, _address(k), ks, _address(k_out), kos,
                                     _raw(stream, dev)))
        return q_out if k is None else (q_out, k_out)


_NONE = _I64x2(0, 0)


def _turned(name, t, out, tokens, heads, dim, dtype, device, stream):
    """Where rows go, and the strides of both."""
    strides = _rows(name, t, dtype, device, heads, dim)
    if t.shape[0] != tokens:
        _bad(f"{name}: {t.shape[0]} tokens, need {tokens}")
    if out is None:
        return _like(t, stream), strides, _I64x2(heads * dim, dim)
    if out.shape != t.shape:
        _bad(f"{name}_out: shape {tuple(out.shape)}, need {tuple(t.shape)}")
    return out, strides, _rows(name + "_out", out, dtype, device, heads, dim)


class KVCache:
    """Keys and values of `n_seqs` sequences in 8 bits, one fp32 scale per
    block of `block_tokens` tokens of a key/value head.

    Owns (or takes over, with `tensors` naming all but the last two) the arrays
    of m2c_kv_cache as attributes of the same names: k_codes, v_codes, k_scale,
    v_scale, tail_k, tail_v, table, len, weight, arrive, status. `n_pages`
    defaults to one page for every table entry, and `table` to those in order;
    with fewer pages it is -1 and the caller sets entries before blocks fill."""

    def __init__(self, n_seqs, n_kv_heads, head_dim, max_blocks, block_tokens=64,
                 dtype=torch.float16, n_pages=None, device=None, tensors=None):
        if dtype not in _DTYPES:
            _bad(f"dtype {dtype}: need torch.float16 or torch.bfloat16")
        if tensors is not None:
            codes = tensors.get("k_codes")
            if codes is None or not codes.is_cuda or codes.dim() != 3:
                _bad("tensors: need GPU tensors, k_codes [pages, block_tokens, head_dim] among them")
            dev, n_pages = codes.device, codes.shape[0]
        else:
            dev = torch.device("cuda", torch.cuda.current_device()) if device is None \
                else torch.device(device)
            if dev.type != "cuda":
                _bad(f"device {dev}: need a GPU")
            if dev.index is None:
                dev = torch.device("cuda", torch.cuda.current_device())
        entries = n_seqs * n_kv_heads * max_blocks
        n_pages = entries if n_pages is None else n_pages
        page, tail = (n_pages, block_tokens, head_dim), (n_seqs, n_kv_heads, block_tokens, head_dim)
        entry = (n_seqs, n_kv_heads, max_blocks)
        want = {"k_codes": (page, torch.int8), "v_codes": (page, torch.int8),
                "k_scale": ((n_pages,), torch.float32), "v_scale": ((n_pages,), torch.float32),
                "tail_k": (tail, dtype), "tail_v": (tail, dtype), "table": (entry, torch.int32),
                "len": ((n_seqs,), torch.int32), "weight": (entry, torch.float32),
                "arrive": ((n_seqs,), torch.int32), "status": ((1,), torch.int32)}
        for name, (shape, dt) in want.items():
            t = tensors.get(name) if tensors is not None else None
            if t is None and (tensors is None or name in ("arrive", "status")):
                make = torch.empty if name in ("k_codes", "v_codes", "tail_k", "tail_v") else torch.zeros
                t = make(shape, dtype=dt, device=dev)
                if name == "table":
                    t = torch.arange(entries, dtype=torch.int32, device=dev).view(shape) if n_pages >= entries \
                        else t.fill_(-1)
            if t is None or tuple(t.shape) != shape or t.dtype != dt or t.device != dev or \
                    not t.is_contiguous():
                _bad(f"{name}: need a contiguous {dt} tensor {shape} on {dev}")
            setattr(self, name, t)
        self._lib, self._need = m2c.load(), {}  # _need: workspace bytes by call shape
        self.device, self.dtype = dev, dtype
        self.n_seqs, self.n_kv_heads, self.head_dim = n_seqs, n_kv_heads, head_dim
        self.max_blocks, self.block_tokens = max_blocks, block_tokens
        self.desc = m2c.KvCacheDesc(_DTYPES[dtype], n_seqs, n_kv_heads, head_dim, block_tokens,
                                    max_blocks, dev.index, 0, n_pages,
                                    *(getattr(self, n).data_ptr() for n in want))

    def _n(self, seqs, n):
        """Rows of a call, and its checked sequence list."""
        if seqs is None:
            return n, None
        return seqs.shape[0], _ints("seqs", seqs, n, self.device)

    def reset(self, seqs=None, stream=None):
        """Forget the tokens of the listed sequences (default: all)."""
        n = self.n_seqs if seqs is None else seqs.shape[0]
        n, seqs = self._n(seqs, n)
        _check(self._lib.m2c_kv_reset(self.desc, _address(seqs), n, _raw(stream, self.device)))

    def append(self, k, v, cu=None, seqs=None, pos=None, stream=None):
        """Append rows of k and v [tokens, n_kv_heads, head_dim]: rows cu[b] ..
        cu[b + 1] - 1 to sequence seqs[b] (default: b), or with cu None one row
        each. pos: int32 places of the first new tokens (default: the ends)."""
        n = k.shape[0] if cu is None else cu.shape[0] - 1
        n, seqs = self._n(seqs, n)
        _ints("cu", cu, n + 1, self.device)
        _ints("pos", pos, n, self.device)
        ks = _rows("k", k, self.dtype, self.device, self.n_kv_heads, self.head_dim)
        vs = _rows("v", v, self.dtype, self.device, self.n_kv_heads, self.head_dim)
        if v.shape[0] != k.shape[0]:
            _bad(f"v: {v.shape[0]} tokens, k has {k.shape[0]}")
        _check(self._lib.m2c_kv_append(self.desc, _address(seqs), n, _address(cu), k.shape[0],
                                       _address(pos), k.data_ptr(), v.data_ptr(), ks, vs,
                                       _raw(stream, self.device)))

    def append_rotated(self, rotary, k, v, positions, q=None, cu=None, seqs=None, pos=None, q_out=None, k_out=None,
                       stream=None):
        """`append` of keys that `rotary` turns by `positions` (as in Rotary.rotate;
        pos is the place in the cache) on the way, and of the queries q [tokens,
        n_heads, head_dim] of the same tokens beside them. q_out: what gets the
        queries (may be q; allocated if not given). k_out: rows that get the turned
        keys as well (not k), True to allocate them. Returns (q_out, k_out), None for
        what there is not."""
        n = k.shape[0] if cu is None else cu.shape[0] - 1
        n, seqs = self._n(seqs, n)
        dev, hk, d = self.device, self.n_kv_heads, self.head_dim
        _ints("cu", cu, n + 1, dev)
        _ints("pos", pos, n, dev)
        ks = _rows("k", k, self.dtype, dev, hk, d)
        vs = _rows("v", v, self.dtype, dev, hk, d)
        rows = k.shape[0]
        if v.shape[0] != rows:
            _bad(f"v: {v.shape[0]} tokens, k has {rows}")
        at, step = rotary._positions(positions, rows, dev)
        hq, qs, qos, kos = 0, _NONE, _NONE, _NONE
        if q is not None:
            hq = q.shape[1] if q.dim() == 3 else 0
            q_out, qs, qos = _turned("q", q, q_out, rows, hq, d, self.dtype, dev, stream)
        elif q_out is not None:
            _bad("q_out: there is no q")
        if k_out is not None:
            k_out, _, kos = _turned("k", k, None if k_out is True else k_out, rows, hk, d, self.dtype, dev, stream)
        _check(self._lib.m2c_kv_append_rotated(
            self.desc, rotary.desc, _address(seqs), n, _address(cu), rows, _address(pos), at, step, k.data_ptr(),
            v.data_ptr(), ks, vs, _address(k_out), kos, hq, _address(q), qs, _address(q_out), qos,
            _raw(stream, dev)))
        return q_out, k_out

    def read(self, cu, total=None, seqs=None, k=None, v=None, stream=None):
        """Tokens 0, 1, .. of sequence seqs[b] into rows cu[b] .. cu[b + 1] - 1
        of k and v (allocated with `total` rows if not given; rows past a
        sequence's length are not written). Returns (k, v)."""
        n, seqs = self._n(seqs, cu.shape[0] - 1)
        _ints("cu", cu, n + 1, self.device)
        if (k is None) != (v is None) or (k is None) == (total is None):
            _bad("read: give k and v, or total")
        if k is None:
            rows = ((total, self.n_kv_heads, self.head_dim), self.dtype)
            k, v = _alloc(stream, self.device, rows, rows)
        ks = _rows("k", k, self.dtype, self.device, self.n_kv_heads, self.head_dim)
        vs = _rows("v", v, self.dtype, self.device, self.n_kv_heads, self.head_dim)
        if v.shape[0] != k.shape[0]:
            _bad(f"v: {v.shape[0]} rows, k has {k.shape[0]}")
        _check(self._lib.m2c_kv_read(self.desc, _address(seqs), n, cu.data_ptr(), k.shape[0],
                                     k.data_ptr(), v.data_ptr(), ks, vs, _raw(stream, self.device)))
        return k, v

    def attend(self, q, seqs=None, max_len=0, scale=None, track=False, out=None, return_lse=False,
               stream=None):
        """Attention of one token per sequence, q [n, n_heads, head_dim], over
        all that sequence seqs[b] (default: b) holds. max_len: the longest of
        them if known. scale: as in prompt_attention. track: add the blocks' attention weights to `weight`.
        Returns out like q, or (out, lse) with lse fp32 [n, n_heads]."""
        if q.dim() != 3:
            _bad("q: need [n, n_heads, head_dim]")
        hq = q.shape[1]
        n, seqs = self._n(seqs, q.shape[0])
        qs = _rows("q", q, self.dtype, self.device, hq, self.head_dim)
        track = 1 if track else 0
        key = (n, hq, track, max_len)
        need = self._need.get(key)
        if need is None:
            if len(self._need) >= 4096:
                self._need.clear()
            need = self._need[key] = m2c.m2c_kv_attend_workspace(self.desc, *key)
        if out is None:
            out, os = _like(q, stream), _I64x2(hq * self.head_dim, self.head_dim)
        elif out.shape != q.shape:
            _bad(f"out: shape {tuple(out.shape)}, need {tuple(q.shape)}")
        else:
            os = _rows("out", out, self.dtype, self.device, hq, self.head_dim)
        lse = _alloc(stream, self.device, ((n, hq), torch.float32))[0] if return_lse else None
        work = _alloc(stream, self.device, ((need,), torch.uint8))[0] if need else None
        _check(self._lib.m2c_kv_attend(self.desc, _address(seqs), n, hq, 0.0 if scale is None else scale,
                                       q.data_ptr(), qs, out.data_ptr(), os, _address(lse), track,
                                       max_len, _address(work), need, _raw(stream, self.device)))
        return (out, lse) if return_lse else out

    def attend_chunk(self, q, cu, k=None, v=None, seqs=None, max_q=0, max_len=0, scale=None, out=None,
                     return_lse=False, stream=None):
        """Attention of chunks of tokens: rows cu[b] .. cu[b + 1] - 1 of q [tokens,
        n_heads, head_dim] are sequence seqs[b]'s (default: b). Its keys are what the
        cache holds of it and then the same rows of k and v [tokens, n_kv_heads,
        head_dim], the chunk's own, which are appended afterwards; without them the
        cache holds the chunk already. Of nk keys in all, query i of lq sees keys 0
        .. nk - lq + i. max_q, max_len: longest chunk, and most tokens of a sequence
        in the cache, if known. scale: as in prompt_attention.
        Returns out like q, or (out, lse) with lse fp32 [tokens, n_heads]."""
        if q.dim() != 3 or cu.dim() != 1:
            _bad("q: need [tokens, n_heads, head_dim]; cu: row starts and the end")
        total, hq, dev = q.shape[0], q.shape[1], self.device
        n, seqs = self._n(seqs, cu.shape[0] - 1)
        _ints("cu", cu, n + 1, dev)
        qs = _rows("q", q, self.dtype, dev, hq, self.head_dim)
        if (k is None) != (v is None):
            _bad("attend_chunk: give k and v, or neither")
        ks = vs = _NONE
        if k is not None:
            ks = _rows("k", k, self.dtype, dev, self.n_kv_heads, self.head_dim)
            vs = _rows("v", v, self.dtype, dev, self.n_kv_heads, self.head_dim)
            if k.shape[0] != total or v.shape[0] != total:
                _bad(f"k, v: {k.shape[0]} and {v.shape[0]} tokens, q has {total}")
        key = (n, total, hq, max_q, max_len)
        need = self._need.get(key)
        if need is None:
            if len(self._need) >= 4096:
                self._need.clear()
            need = self._need[key] = m2c.m2c_kv_attend_chunk_workspace(self.desc, *key)
        if out is None:
            out, os = _like(q, stream), _I64x2(hq * self.head_dim, self.head_dim)
        elif out.shape != q.shape:
            _bad(f"out: shape {tuple(out.shape)}, need {tuple(q.shape)}")
        else:
            os = _rows("out", out, self.dtype, dev, hq, self.head_dim)
        lse = _alloc(stream, dev, ((total, hq), torch.float32))[0] if return_lse else None
        work = _alloc(stream, dev, ((need,), torch.uint8))[0] if need else None
        _check(self._lib.m2c_kv_attend_chunk(
            self.desc, _address(seqs), n, cu.data_ptr(), total, hq, 0.0 if scale is None else scale, q.data_ptr(), qs,
            _address(k), ks, _address(v), vs, out.data_ptr(), os, _address(lse), max_q, max_len, _address(work), need,
            _raw(stream, dev)))
        return (out, lse) if return_lse else out

    def evict(self, keep, first=0, recent=0, seqs=None, out=None, stream=None):
        """Keep `keep` blocks before the last one of every listed sequence and
        head: the first `first`, the last `recent`, else the heaviest. out: a
        dict of tensors "table", "weight", "len" that get the rows instead of
        the cache's own."""
        n, seqs = self._n(seqs, self.n_seqs if seqs is None else seqs.shape[0])
        for name, v in (("keep", keep), ("first", first), ("recent", recent)):
            if not 0 <= v < 1 << 31:  # a larger one would be cut to 32 bits on the way
                _bad(f"{name} {v}: need [0, 2^31 - 1]")
        to = (None, None, None)
        if out is not None:
            to = (out["table"], out["weight"], out["len"])
            for name, t, own in zip(("table", "weight", "len"), to, (self.table, self.weight, self.len)):
                if t.shape != own.shape or t.dtype != own.dtype or t.device != own.device or \
                        not t.is_contiguous():
                    _bad(f"out[{name!r}]: need a tensor like the cache's")
        _check(self._lib.m2c_kv_evict(self.desc, _address(seqs), n, keep, first, recent,
                                      *map(_address, to), _raw(stream, self.device)))

    def check(self, stream=None):
        """Wait for `stream`; raise what the calls so far found on the device
        (a sequence or page out of range, row starts that do not ascend, a full
        sequence, a bad place)."""
        _check(self._lib.m2c_kv_status(self.desc, _raw(stream, self.device)))
