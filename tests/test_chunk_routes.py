"""Which way a decoder layer attends a later chunk (no GPU is touched)."""
from types import SimpleNamespace

import pytest

from paper_2410_14740_amd import decoder


@pytest.mark.parametrize("lens,before,heads,back", [
    ([2048, 700], [30000, 16385], (64, 8, 128), True), ([4096], [4000], (64, 8, 128), True), ([1024], [60000], (32, 8, 64), True),
    ([2048], [4000], (64, 8, 128), False), ([512, 300, 77], [3500, 1511, 2323], (40, 40, 128), False),
    ([4096], [16000], (40, 40, 128), False), ([512], [60000], (32, 8, 64), False), ([5] * 16, [30000] * 16, (64, 8, 128), False),
    ([0, 0], [7, 0], (16, 4, 64), False),
])
def test_by_the_work(lens, before, heads, back):
    assert decoder.reads_back(lens, before, *heads) is back


@pytest.mark.parametrize("budget,back", [(0, True), (4, False)])
def test_a_layer_with_a_budget_attends_codes(budget, back, monkeypatch):
    """Its cache may hold fewer tokens than the rows before the chunk were."""
    layer = object.__new__(decoder.DecoderLayer)
    layer.budget, layer.n_heads, layer.n_kv_heads, layer.dim = budget, 64, 8, 128
    calls = []

    class Stop(Exception):
        pass

    def read(*a):
        calls.append("read")
        raise Stop

    monkeypatch.setattr(decoder, "_starts", lambda lens: None)
    layer.cache = SimpleNamespace(read=read, attend_chunk=lambda *a, **k: calls.append("chunk"))
    try:
        layer.attend(None, None, None, None, [2048], [60000])
    except Stop:
        pass
    assert calls == ["read" if back else "chunk"]
