"""Tensors of another GPU than the current one, or of two: refused before anything is launched.  (Played: there is one GPU here.)"""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def calls(ev):
    """Every call of the decode operators, as (name, function of the cache)."""
    import torch
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    t, at, off = i32([[0, 1]]), i32([0]), i32([0, 3])
    z, u = torch.zeros(2, 10, device="cuda"), torch.zeros(2, device="cuda")
    return [("write", lambda c: ev.kv_write(c, k, k, t, at, off, 3)), ("read", lambda c: ev.kv_read(c, t, at, off, 3, 3)),
            ("attention", lambda c: ev.kv_attention(k, c, t, i32([3]), off, 3)), ("sample", lambda c: ev.sample(z, u))]


def test_another_current_gpu(ev, monkeypatch):
    from paper_2605_27390_amd import decode
    c = ev.KVCache(2, 32, 2, 64)
    c.data.zero_()
    c.scales.fill_(1.0)
    todo = calls(ev)
    for _, call in todo:
        call(c)
    here = decode._get_device()
    monkeypatch.setattr(decode, "_get_device", lambda: here + 1)
    for name, call in todo:
        with pytest.raises(ValueError, match="GPU"):
            call(c)


def test_a_cache_on_another_gpu(ev):
    c = ev.KVCache(2, 32, 2, 64)
    c._device += 1
    for name, call in calls(ev)[:3]:
        with pytest.raises(ValueError, match="GPU"):
            call(c)
