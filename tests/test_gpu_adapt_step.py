"""The updates of examples/adapt_step.py: what its calls give on each other's results, and the adapters' gradients against the formula and against
differences of the loss."""
import importlib.util
import os

import numpy as np
import pytest

import adapt_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("adapt_step", os.path.join(ROOT, "examples", "adapt_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def host(t):
    return t.double().cpu().numpy()


def updates_of(example, n, **kw):
    """The first n updates: the adapters and moments before, what the update saw, and the loop after it."""
    loop = example.Loop(**kw)
    while n:
        a, b = host(loop.a), host(loop.b)
        masters = host(loop.opt.master)
        kl, seen = loop.step()
        assert kl.isfinite().all()
        if seen is not None:
            n -= 1
            yield loop, a, b, masters, seen


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_updates(example, state):
    for loop, a, b, masters, s in updates_of(example, 3, state=state, seed=2):
        x, W, W_lm = host(s["x"]), host(loop.W), host(loop.W_lm)
        off, adapter, scale = s["row_off"].tolist(), s["adapter"].tolist(), host(loop.bank.scale)
        # forward: the shared projection is torch's, in bf16
        y = host(s["x"] @ loop.W.t())
        want, bound, h, hb = ref.lora_forward(x, a, b, scale, off, adapter, y)
        assert (np.abs(host(s["hidden"]) - want) <= bound).all() and (np.abs(host(s["h"]) - h) <= hb).all()
        # loss and gradient at the hidden states that came out
        got = ref.kd_loss(host(s["hidden"]), W_lm, s["support"].cpu().numpy(), host(s["target"]), host(s["weight"]), loop.T, ref.BF16)
        for name, w, wb in (("loss", got[0], got[1]), ("dh", got[2], got[3]), ("draft", got[4], got[5])):
            assert (np.abs(host(s[name]) - w) <= wb).all(), name
        # the adapters' gradients from that gradient
        da, dab, db, dbb, _, _ = ref.lora_backward(x, host(s["dh"]), a, b, scale, off, adapter, None)
        assert (np.abs(host(loop.grads[0]) - da) <= dab).all() and (np.abs(host(loop.grads[1]) - db) <= dbb).all()
        # and the adapters are their masters, rounded
        for t, at in zip((loop.a, loop.b), loop.opt.offsets):
            assert (loop.opt.master[at:at + t.numel()].to(t.dtype) == t.reshape(-1)).all()
        assert not np.array_equal(host(loop.opt.master), masters)


def test_gradients_against_differences(example):
    """The loss of the whole way, in 64 bits, as A and B are changed: its slope is what comes out of the calls, to the roundings on the
    way (hidden states and their gradient to bf16: 2^-8 of each, through at most d products)."""
    loop, a, b, _, s = list(updates_of(example, 2, seed=5))[-1]
    x, W, W_lm = host(s["x"]), host(loop.W), host(loop.W_lm)
    off, adapter, scale = s["row_off"].tolist(), s["adapter"].tolist(), host(loop.bank.scale)
    support, target, weight = s["support"].cpu().numpy(), host(s["target"]), host(s["weight"])

    def loss(a, b):
        hidden = ref.lora_forward(x, a, b, scale, off, adapter, x @ W.T)[0]
        return ref.kd_loss(hidden, W_lm, support, target, weight, loop.T, 0.0)[0].sum()

    rng = np.random.default_rng(0)
    got = [host(g) for g in loop.grads]
    for which in (0, 1):
        for _ in range(6):
            way = rng.normal(size=got[which].shape)
            way /= np.linalg.norm(way)
            step = 1e-4
            up, down = [a, b], [a, b]
            up[which], down[which] = up[which] + step * way, down[which] - step * way
            slope = (loss(*up) - loss(*down)) / (2 * step)
            # a gradient that is off by 2^-6 of its length in any direction (four roundings of 2^-8)
            assert abs(slope - np.sum(got[which] * way)) <= 2.0 ** -6 * np.linalg.norm(got[which])


def test_command_line(example, capsys, monkeypatch):
    for state in ("fp32", "8bit"):
        monkeypatch.setattr("sys.argv", ["adapt_step.py", "--steps", "6", "--state", state])
        example.main()
        assert "update 1" in capsys.readouterr().out
