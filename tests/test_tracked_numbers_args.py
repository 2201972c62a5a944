"""Numbers beyond 32 bits in the Python calls around an evicting cache (no GPU)."""
import types

import pytest

import paper_2502_08910_amd as ih
from paper_2502_08910_amd import binding


def stand_ins(heads=2):
    """What the calls look at before their numbers go to the library, which is not reached."""
    import torch
    device = torch.device("cpu")
    track = types.SimpleNamespace(check=lambda *a: None, ref=lambda: None, before=lambda *a: None)
    return types.SimpleNamespace(B=4, tokens=64, Hkv=heads, device=device, ref=lambda: None), track, torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("numbers", [dict(keep=2 ** 32 + 16), dict(n_sink=2 ** 32), dict(n_recent=2 ** 32 + 4), dict(n_recent=-2 ** 32), dict(n_sink=2 ** 31)])
def test_evict(monkeypatch, numbers):
    """They are refused; their lower 32 bits were taken for them."""
    gone_on = []
    monkeypatch.setattr(binding, "_enqueue", lambda device, fn, *args: gone_on.append(args))
    store, track, lens = stand_ins()
    want = dict(keep=16, n_sink=0, n_recent=0)
    want.update(numbers)
    import torch
    with pytest.raises(ih.IhipError, match="2\\^31"):
        ih.kv_evict(store, track, lens, 64, new_lens=lens, ws=lens, kept=torch.zeros(4 * 2 * min(want["keep"], 16), dtype=torch.int32), **want)
    assert not gone_on


def test_window_and_max_q(monkeypatch):
    """Bounds that are loose are bounds; what is negative stays it, and is refused by the library."""
    import torch
    got = []
    monkeypatch.setattr(binding, "_enqueue", lambda device, fn, *args: got.append((args[7], args[0]._obj.max_q)))
    monkeypatch.setattr(binding, "_packed_tensor", lambda *a: None)
    _, track, cu = stand_ins()
    q, lse = torch.zeros((5, 2, 128), dtype=torch.bfloat16), torch.zeros((5, 2))
    most = 2 ** 31 - 1
    for window, max_q, want in ((-2 ** 32 + 5, 5, (-1, 5)), (0, 0, (0, 0)), (5, 2 ** 32 + 1, (5, most)), (2 ** 40, -2 ** 32 + 7, (most, -1)), (None, most, (most, most))):
        ih.prompt_key_weights(q, q, cu, max_q, lse, track, window=window, ws=cu)
        assert got.pop() == want
