"""The distillation loss on the retained support and its gradient, against the definition in 64 bits."""
import numpy as np
import pytest

import adapt_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    return t.to("cuda", dtype or t.dtype)


def problem(E, K, d, V, seed=0, size=1.0):
    rng = np.random.default_rng(seed)
    h, W = ref.bf16(rng.normal(size=(E, d))), ref.bf16(rng.normal(size=(V, d)) * size / np.sqrt(d))
    support = rng.integers(0, V, size=(E, K)).astype(np.int32)
    target = np.float32(rng.normal(size=(E, K)) * 2).astype(np.float64)
    weight = np.float32(rng.random(E)).astype(np.float64)
    return h, W, support, target, weight


def call(ev, h, W, support, target, weight, T=1.0, dtype=None, **kw):
    import torch
    dtype = dtype or torch.bfloat16
    return ev.kd_loss(dev(h, torch.bfloat16), dev(W, torch.bfloat16), dev(support), dev(target, torch.float32),
                      None if weight is None else dev(weight, torch.float32), T=T, dtype=dtype, **kw)


def check(got, h, W, support, target, weight, T, half):
    loss, lb, dh, db, draft, zb = ref.kd_loss(h, W, support, target, weight, T, half)
    for name, g, want, bound in zip(("loss", "dh", "draft"), got, (loss, dh, draft), (lb, db, zb)):
        g = g.double().cpu().numpy()
        assert np.array_equal(np.isnan(g), np.isnan(want)), name
        far = np.nan_to_num(np.abs(g - want) - bound)
        assert not (far > 0).any(), (name, float(far.max()), np.argwhere(far > 0)[:3])


@pytest.mark.parametrize("E,K,d,V,T", [(1, 1, 8, 3, 1.0), (1, 256, 4096, 700, 1.0), (3, 256, 512, 999, 2.0), (7, 37, 520, 200, 0.5),
                                       (600, 9, 64, 100, 1.0), (2, 1024, 2056, 3000, 1.3), (40, 256, 1000, 1000, 1.0), (5, 100, 4104, 300, 1.0),
                                       (2, 65, 8200, 300, 1.0), (3, 20, 16384, 128, 1.0), (513, 33, 136, 77, 4.0), (1, 7, 1032, 50, 1.0)])
@pytest.mark.parametrize("fp32", [False, True])
def test_against_the_definition(ev, E, K, d, V, T, fp32):
    import torch
    p = problem(E, K, d, V, seed=E + K + d, size=3.0)
    got = call(ev, *p, T=T, dtype=torch.float32 if fp32 else torch.bfloat16)
    check(got, *p, T, ref.U if fp32 else ref.BF16)
    again = call(ev, *p, T=T, dtype=torch.float32 if fp32 else torch.bfloat16)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("E,K", [(4, 40), (600, 24)])
def test_entries_that_are_not_in_the_support(ev, E, K):
    import torch
    h, W, support, target, weight = problem(E, K, 200, 90, seed=3)
    support[0] = -1                                                   # an event without any
    support[1, 1:] = -1                                               # of one token: p = q = 1
    support[2, ::3], support[2, 1::3] = 90, 2 ** 31 - 1               # ids past the vocabulary
    support[3, K - 5:] = -2 ** 31
    target[0, :], target[3, K - 5:] = np.nan, np.nan                  # (as kl_gate leaves them)
    for w in (weight, None):
        got = call(ev, h, W, support, target, w, dtype=torch.float32)
        check(got, h, W, support, target, w, 1.0, ref.U)
        assert got[0][0] == 0 and not got[1][0].any() and got[2][0].isnan().all()
        assert abs(float(got[0][1])) == 0


def test_targets_that_are_not_numbers(ev):
    """-inf is a probability of zero; nothing but -inf gives no loss; NaN and +inf give NaN, to their event alone."""
    import torch
    for E in (8, 600):
        h, W, support, target, weight = problem(E, 40, 128, 70, seed=4)
        target[0, ::2] = -np.inf
        target[1] = -np.inf
        target[2, 7], target[3, 8] = np.nan, np.inf
        got = call(ev, h, W, support, target, weight, dtype=torch.float32)
        rest = np.array([i for i in range(E) if i not in (2, 3)])
        check([t[dev(rest)] for t in got], h[rest], W, support[rest], target[rest], weight[rest], 1.0, ref.U)
        assert got[0][1] == 0 and not got[1][1].any()
        assert got[0][2:4].isnan().all() and got[1][2:4].isnan().all() and got[2][2:4].isfinite().all()


def test_rows_that_are_not_numbers(ev):
    """A NaN in a row of W_lm or in h makes its own events NaN."""
    import torch
    for E in (6, 600):
        h, W, support, target, weight = problem(E, 40, 128, 70, seed=5)
        support[support == 11] = 12
        support[1, 3] = 11
        W[11, 9] = np.nan
        h[2, 100] = np.inf
        got = call(ev, h, W, support, target, weight, dtype=torch.float32)
        rest = np.array([i for i in range(E) if i not in (1, 2)])
        W[11, 9] = 0
        check([t[dev(rest)] for t in got], h[rest], W, support[rest], target[rest], weight[rest], 1.0, ref.U)
        assert got[0][1].isnan() and got[1][1].isnan().all() and got[2][1].isnan().sum() == 1
        assert got[0][2].isnan() and got[1][2].isnan().all()


def test_far_logits(ev):
    """Logits of hundreds: the running maximum moves, shares underflow, and a small temperature makes it worse."""
    import torch
    h, W, support, target, weight = problem(5, 256, 64, 300, seed=6, size=40.0)
    target *= 50
    for T in (1.0, 0.25, 16.0):
        check(call(ev, h, W, support, target, weight, T=T, dtype=torch.float32), h, W, support, target, weight, T, ref.U)


def test_a_draft_that_equals_the_target(ev):
    """Near the minimum the loss is a small difference of large terms: still to the bound of the logits' errors, which vanishes with q - p."""
    import torch
    h, W, support, _, weight = problem(30, 256, 256, 400, seed=7, size=3.0)
    z = np.take_along_axis(h @ W.T, support.astype(np.int64), 1)
    target = np.float32(z + np.random.default_rng(8).normal(size=z.shape) * 1e-3).astype(np.float64)
    check(call(ev, h, W, support, target, weight, dtype=torch.float32), h, W, support, target, weight, 1.0, ref.U)


def test_behind_the_gate(ev):
    """Support, target logits and draft logits are kl_gate's; loss without weight is its divergence."""
    import torch
    rng = np.random.default_rng(9)
    E, V, d, K = 12, 5000, 512, 256
    h, W = dev(ref.bf16(rng.normal(size=(E, d))), torch.bfloat16), dev(ref.bf16(rng.normal(size=(V, d)) * 0.1), torch.bfloat16)
    z = dev(np.float32(rng.normal(size=(E, V)) * 3))
    z[3, 100:] = float("nan")                                        # fewer numbers than K
    support, zt, zq, kl = ev.kl_gate(z, h, W, K=K, T=1.5)
    loss, dh, draft = ev.kd_loss(h, W, support, zt, T=1.5)
    mine = support >= 0
    assert not mine[3].all() and torch.equal(draft.isnan(), ~mine)
    assert float((draft - zq)[mine].abs().max()) <= 1e-4             # (two orders of 512 products of about 0.1)
    good = torch.arange(E, device="cuda") != 3
    assert float(((loss - 1.5 ** 2 * kl) / loss)[good].abs().max()) < 1e-4


def test_refusals(ev):
    import torch
    h, W, support, target, weight = problem(4, 20, 64, 50)
    ok = dict(h=dev(h, torch.bfloat16), W_lm=dev(W, torch.bfloat16), support=dev(support), target=dev(target, torch.float32))
    for bad in (dict(h=ok["h"].float()), dict(W_lm=ok["W_lm"].float()), dict(support=ok["support"].long()), dict(target=ok["target"].double()),
                dict(dtype=torch.float16)):
        with pytest.raises(TypeError):
            ev.kd_loss(**{**ok, **bad})
    for bad in (dict(h=ok["h"][:3]), dict(W_lm=ok["W_lm"][:, :56].contiguous()), dict(target=ok["target"][:, :19].contiguous()),
                dict(weight=torch.ones(3, device="cuda")), dict(out_dh=torch.empty(4, 56, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            ev.kd_loss(**{**ok, **bad})
    for bad in (dict(T=0.0), dict(T=float("nan")), dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ev.EvospecError):
            ev.kd_loss(**{**ok, **bad})
    none = ev.kd_loss(ok["h"][:0], ok["W_lm"], ok["support"][:0], ok["target"][:0])
    assert [tuple(t.shape) for t in none] == [(0,), (0, 64), (0, 20)]


def test_outputs_that_are_inputs(ev):
    import torch
    h, W, support, target, weight = problem(4, 20, 64, 50)
    ok = dict(h=dev(h, torch.bfloat16), W_lm=dev(W, torch.bfloat16), support=dev(support), target=dev(target, torch.float32))
    for bad in (dict(out_draft=ok["target"]), dict(out_draft=ok["support"].view(torch.float32)), dict(out_dh=ok["h"]), dict(out_dh=ok["W_lm"][46:])):
        with pytest.raises(ValueError, match="overlaps"):
            ev.kd_loss(**{**ok, **bad})


@pytest.mark.parametrize("E", [3, 520])
def test_streams_and_graphs(ev, E):
    import torch
    h, W, support, target, weight = problem(E, 48, 264, 90, seed=11)
    th, tW, ts, tt, tw = dev(h, torch.bfloat16), dev(W, torch.bfloat16), dev(support), dev(target, torch.float32), dev(weight, torch.float32)
    want = ev.kd_loss(th, tW, ts, tt, weight=tw)
    ws = torch.empty(ev.kd_loss_workspace_bytes(E, 48, 264) + 16, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()

    def one():
        return ev.kd_loss(th, tW, ts, tt, weight=tw, out_loss=outs[0], out_dh=outs[1], out_draft=outs[2], workspace=ws)
    with torch.cuda.stream(s):
        one()
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            one()
    for k in range(4):
        th.copy_(dev(ref.bf16(h * (k + 1)), torch.bfloat16))
        ts.copy_(dev(np.roll(support, k, 1)))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ev.kd_loss(th, tW, ts, tt, weight=tw))), k


def test_another_gpu_than_the_current_one(ev, monkeypatch):
    """Played: there is one GPU here."""
    import torch
    from paper_2605_27390_amd import decode
    h, W, support, target, _ = problem(2, 5, 64, 20)
    here = decode._get_device()
    monkeypatch.setattr(decode, "_get_device", lambda: here + 1)
    with pytest.raises(ValueError, match="GPU"):
        call(ev, h, W, support, target, None)
