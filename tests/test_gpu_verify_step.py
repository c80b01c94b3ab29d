"""The decode loop of examples/verify_step.py: what its calls give on each other's results, step after step."""
import importlib.util
import os

import numpy as np
import pytest

import decode_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("verify_step", os.path.join(ROOT, "examples", "verify_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def host_cache(c):
    h = ref.Cache(c.pages, c.page, c.heads, c.dim, c.kind)
    h.data = c.data.cpu().numpy().reshape(h.data.shape)
    h.scales = c.scales.cpu().numpy().reshape(h.scales.shape)
    return h


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_steps(example, kind):
    loop = example.Loop(S=3, kind=kind, seed=1)
    for i in range(6):
        before = list(loop.lens)
        last = list(loop.last)
        r = loop.step(temperature=0.0 if i % 2 else 0.7)
        # attention: the cache after the step differs from the one it saw where accepted nodes were moved, so compare on the
        # root, which sees the older tokens and itself
        h = host_cache(loop.cache)
        table = loop.table.cpu().numpy()
        q = r["q"].double().cpu().numpy()
        for s in range(loop.S):
            root = r["row_off"][s]
            out, lse, weight, _ = ref.attention(h, q[root:root + 1], table[s:s + 1], [before[s] + 1], [0, 1], loop.group, None,
                                                loop.dim ** -0.5)
            got = r["out"][root].double().cpu().numpy()
            # the root's block may have been scaled up by tree nodes in between: one more rounding of the codes
            step = 2.0 ** -4 if kind == "e4m3" else 1 / 127
            v_max = np.abs(h.values(table[s:s + 1], 0, before[s] + 1)[1]).max()
            assert np.abs(got - out[0]).max() <= 2.0 ** -7 * np.abs(out).max() + 2 * step * v_max
            assert last[s] == loop.tokens[s][-len(r["grown"][s]) - 1]
        z = r["logits"].double().cpu().numpy()
        if i % 2:
            drawn = r["drawn"].cpu().numpy()
            assert (z[np.arange(len(z)), drawn] == z.max(1)).all() and (r["logprob"].cpu().numpy() == 0).all()
        assert all(1 <= len(g) <= example.DEPTH + 1 for g in r["grown"])
        assert loop.lens == [a + len(g) for a, g in zip(before, r["grown"])]
        # the cache holds the accepted tokens' keys: those of the tokens themselves, to the codes' rounding
        for s in range(loop.S):
            _, _, k, v = loop.project(loop.tokens[s][:loop.lens[s]])
            hk, hv, there = h.values(table[s:s + 1], 0, loop.lens[s])
            assert there.all()
            for got, want in ((hk, k), (hv, v)):
                want = want.double().cpu().numpy()
                top = np.abs(want).max()
                # a code's half step, of the value or of the block's scale, twice where the block was rescaled
                assert np.abs(got - want).max() <= 2 * (2.0 ** -4 if kind == "e4m3" else 1 / 127) * 2 * top


def test_command_line(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["verify_step.py", "--steps", "2"])
    example.main()
    assert "step 1" in capsys.readouterr().out


def test_a_full_cache(example, capsys, monkeypatch):
    """The last tree that fits is taken, the next one is refused, and the command ends in front of it."""
    loop = example.Loop(S=2, capacity=64, seed=3)
    nodes = 1 + example.WIDTH * example.DEPTH
    while max(loop.lens) + nodes <= 64:
        before = list(loop.lens)
        loop.step()
        assert all(a < b for a, b in zip(before, loop.lens))
    before, tokens = list(loop.lens), [list(t) for t in loop.tokens]
    with pytest.raises(ValueError, match="do not fit"):
        loop.step()
    assert loop.lens == before and loop.tokens == tokens
    whole = example.Loop
    monkeypatch.setattr(example, "Loop", lambda: whole(S=2, capacity=64, seed=3))
    monkeypatch.setattr("sys.argv", ["verify_step.py", "--steps", "100"])
    example.main()
    assert "no room" in capsys.readouterr().out


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_every_call_of_a_step(example, kind, monkeypatch):
    """What each call finds and leaves, against the definition: writes value by value, attention of every node of every tree within its bounds, and
    tokens equal."""
    import attention_bounds as bounds
    ev, seen = example.ev, []
    write, attend, sample = ev.kv_write, ev.kv_attention, ev.sample

    def checked_write(c, k, v, table, starts, row_off, max_rows):
        h = host_cache(c)
        h.data, h.scales = h.data.copy(), h.scales.copy()
        write(c, k, v, table, starts, row_off, max_rows)
        h.write(k.float().cpu().numpy(), v.float().cpu().numpy(), table.cpu().numpy(), starts.tolist(), row_off.tolist())
        after = host_cache(c)
        assert (after.scales == h.scales).all()
        rows = np.diff(row_off.tolist())
        for s, (a, n) in enumerate(zip(starts.tolist(), rows)):  # (what lies behind the last token is nobody's)
            for got, want in zip(after.values(table.cpu().numpy(), s, a + n), h.values(table.cpu().numpy(), s, a + n)):
                assert (got == want).all()
        seen.append("write")

    def checked_attention(q, c, table, lens, row_off, max_rows, tree=None):
        out, lse = attend(q, c, table, lens, row_off, max_rows, tree=tree)
        want = bounds.attention(host_cache(c), q.double().cpu().numpy(), table.cpu().numpy(), lens.tolist(), row_off.tolist(),
                                q.shape[1] // c.heads, "bf16", tree.tolist())
        assert bounds.differs(out.double().cpu().numpy(), lse.double().cpu().numpy(), want) is None
        seen.append("attention")
        return out, lse

    def checked_sample(logits, u, **kw):
        got, lp = sample(logits, u, **kw)
        host = {k: x.cpu().numpy() for k, x in kw.items()}
        want, want_lp, margin = ref.sample(logits.double().cpu().numpy(), u.cpu().numpy(), **host)
        sure = margin > logits.shape[1] * 2.0 ** -43 + 2.0 ** -38
        assert sure.any() and np.array_equal(got.cpu().numpy()[sure], want[sure])
        seen.append("sample")
        return got, lp

    loop = example.Loop(S=2, kind=kind, seed=5, V=4096, active=1024)
    loop.cache.data.zero_()
    loop.cache.scales.fill_(1.0)
    for name, f in (("kv_write", checked_write), ("kv_attention", checked_attention), ("sample", checked_sample)):
        monkeypatch.setattr(ev, name, f)
    for _ in range(4):
        loop.step()
    assert seen == ["write", "attention", "sample", "write"] * 4
