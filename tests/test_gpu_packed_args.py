"""kv_append and prompt_attn refuse, before anything is launched, a packed tensor that is narrower than the others (one at a time), and
leave all tensors as they were."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ihip():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_08910_amd as pkg
    pkg.lib()
    return pkg


def tensors(narrow, **heads):
    return {n: torch.ones((6, h, 64 if n == narrow else 128), dtype=torch.bfloat16, device="cuda") for n, h in heads.items()}


def refused(ihip, call, t, narrow):
    if narrow is None:
        return call()
    with pytest.raises(ihip.IhipError):
        call()
    torch.cuda.synchronize()
    assert all(bool((x == 1).all()) for x in t.values())


@pytest.mark.parametrize("narrow", [None, "q", "k", "v", "out"])
def test_prompt_attn(ihip, narrow):
    t = tensors(narrow, q=4, k=2, v=2, out=4)
    cu = torch.tensor([0, 6], dtype=torch.int32).cuda()
    refused(ihip, lambda: ihip.prompt_attn(t["q"], t["k"], t["v"], cu, 6, out=t["out"]), t, narrow)


@pytest.mark.parametrize("narrow", [None, "q", "k", "v", "q_out", "k_out"])
def test_kv_append(ihip, narrow):
    t = tensors(narrow, q=4, k=2, v=2, q_out=4, k_out=2)
    cache = [torch.ones((1, 2, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cu, lens = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([0, 6], [6]))
    store = ihip.KVStore.bf16(*cache)
    refused(ihip, lambda: ihip.kv_append(store, t["k"], t["v"], cu, lens, 8, q=t["q"], q_out=t["q_out"], k_out=t["k_out"]), t, narrow)
    assert all(bool((x == 1).all()) for x in cache)
