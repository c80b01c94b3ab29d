"""AdamW over many tensors, with moments in 32 and in 8 bits, against the definition in 64 bits."""
import numpy as np
import pytest

import adapt_reference as ref

pytestmark = pytest.mark.gpu
BLOCK = 256


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def types():
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def host(t):
    return t.double().cpu().numpy().reshape(-1)


class Problem:
    def __init__(self, ev, sizes, ptype, gtype, state, master, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        P, G = types()[ptype], types()[gtype]
        self.sizes, self.ptype, self.state = sizes, ptype, state
        dev = lambda x, t: torch.from_numpy(np.asarray(x)).to("cuda", t)   # noqa: E731
        self.params = [dev(rng.normal(size=n) * 0.1, P) for n in sizes]
        self.grads = [dev(rng.normal(size=n) * 10.0 ** rng.uniform(-4, -1, size=n), G) for n in sizes]
        self.opt = ev.AdamW(self.params, self.grads, state=state, master=master)
        self.total = self.opt.blocks * BLOCK
        self.at = self.opt.offsets
        assert self.at == list(np.cumsum([0] + [-(-n // BLOCK) * BLOCK for n in sizes[:-1]]))

    def moments(self):
        o = self.opt
        if self.state == "fp32":
            return host(o.m), host(o.v)
        s = host(o.scales).reshape(-1, 2).repeat(BLOCK, 0)
        return ref.m_values(o.m.cpu().numpy()) * s[:, 0], ref.v_values(o.v.cpu().numpy()) * s[:, 1]

    def flat(self, tensors):
        out = np.zeros(self.total)
        for a, t in zip(self.at, tensors):
            out[a:a + t.numel()] = host(t)
        return out

    def check_step(self, ev, lr, t, seed=0, grad_scale=1.0, call=None, **kw):
        """One step from the state as it is, against the definition."""
        import torch
        o = self.opt
        opts = dict(betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
        opts.update(kw)
        p0 = host(o.master) if o.master is not None else self.flat(self.params)
        m0, v0 = self.moments()
        p, pb, m, mb, v, vb = ref.adamw(p0, self.flat(self.grads), m0, v0, lr, t, grad_scale=grad_scale, **opts)
        if call is None:
            gs = None if grad_scale == 1.0 else torch.tensor([grad_scale], device="cuda")
            ev.adamw_step(o, lr, t, seed=seed, grad_scale=gs, **opts)
        else:
            call()
        half = ref.HALF[self.ptype]
        mine = np.zeros(self.total, bool)
        for a, n in zip(self.at, self.sizes):
            mine[a:a + n] = True
        got = self.flat(self.params)
        if o.master is not None:
            gm = host(o.master)
            assert (np.abs(gm - p)[mine] <= pb[mine]).all()
            want = np.concatenate([host(o.master[a:a + n].to(types()[self.ptype])) for a, n in zip(self.at, self.sizes)])
            assert np.array_equal(got[mine], want)
        else:
            tiny = 2.0 ** -25 if self.ptype == "fp16" else 0.0       # (fp16 below its normal numbers)
            far = np.abs(got - p) - (pb + half * (np.abs(p) + pb) + tiny)
            assert not (far[mine] > 0).any(), float(far[mine].max())
        if self.state == "fp32":
            gm, gv = self.moments()
            assert (np.abs(gm - m) <= mb)[mine].all() and (np.abs(gv - v) <= vb)[mine].all()
        else:
            self.check_codes(m, mb, v, vb, seed, t)
        assert not self.moments()[0][~mine].any() and not self.moments()[1][~mine].any()

    def check_codes(self, m, mb, v, vb, seed, t):
        o = self.opt
        scales = host(o.scales).reshape(-1, 2)
        r = ref.random_bits(np.arange(self.total), seed, t)
        for codes, x, b, col, bias, largest, bits in ((o.m, m, mb, 0, 7, 448.0, r & 0xffff), (o.v, v, vb, 1, 15, 61440.0, r >> 16)):
            c = codes.cpu().numpy().astype(np.int64)
            top = np.abs(x).reshape(-1, BLOCK)
            low, high = (top - b.reshape(-1, BLOCK)).max(1), (top + b.reshape(-1, BLOCK)).max(1)
            for k in range(len(scales)):
                s = scales[k, col]
                assert ref.scale_for(max(low[k], 0.0), largest) <= s <= ref.scale_for(high[k], largest), (k, s)
            s = scales[:, col].repeat(BLOCK)
            if bias == 7:
                # (what the sign of a moment next to zero is does not matter)
                sure = np.abs(x) > b
                assert ((c >= 128) == (x < 0))[sure].all()
                c = c & 127
            # the moment's error, and a rounding where the smallest normal number is added to tiny ones
            err = b / s + ref.U * 2.0 ** (2 - bias)
            lo, hi = ref.grid(np.maximum(np.abs(x) / s - err, 0.0), bits, bias, largest), ref.grid(np.abs(x) / s + err, bits, bias, largest)
            if bias == 15:
                lo, hi = np.where(x > b, np.maximum(lo, 1), lo), np.where(x > 0, np.maximum(hi, 1), hi)
            assert ((c >= lo) & (c <= hi)).all(), np.argwhere((c < lo) | (c > hi))[:4]
            # (and nearly all of them are a single code)
            assert np.mean(lo == hi) > 0.99 or len(c) < 1000


SIZES = [[1], [3, 256, 255, 257, 5], [1000, 1, 2, 3, 4, 5, 6, 7, 8, 0, 100000], [517] * 130, [70000]]


@pytest.mark.parametrize("sizes", range(len(SIZES)))
@pytest.mark.parametrize("ptype,gtype,master", [("bf16", "bf16", False), ("bf16", "bf16", True), ("bf16", "fp32", True), ("bf16", "fp32", False),
                                                ("fp16", "fp16", False), ("fp16", "fp32", True), ("fp16", "fp16", True), ("fp32", "fp32", False)])
@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_steps(ev, sizes, ptype, gtype, master, state):
    p = Problem(ev, SIZES[sizes], ptype, gtype, state, master, seed=sizes)
    p.check_step(ev, 1e-2, 1, seed=5)
    p.check_step(ev, 1e-3, 2, seed=5, grad_scale=0.37)
    p.check_step(ev, 1e-3, 1000, seed=2 ** 32 - 1, betas=(0.0, 0.9), eps=1e-5, weight_decay=0.0)
    p.check_step(ev, 0.0, 12345678, seed=9, betas=(0.95, 0.9999))


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_moments_to_the_bit(ev, state):
    """Those of the formulas computed one operation after the other in fp32, and their codes, step after step."""
    p = Problem(ev, [70000, 300, 256, 1], "bf16", "bf16", state, False, seed=90)
    b1, b2, g = 0.9, 0.98, p.flat(p.grads).astype(np.float32)
    f = np.float32
    for t in (1, 2, 3):
        m, v = (x.astype(np.float32) for x in p.moments())
        m, v = f(b1) * m + f(1 - b1) * g, f(b2) * v + f(1 - b2) * (g * g)
        ev.adamw_step(p.opt, 1e-3, t, betas=(b1, b2), seed=77)
        if state == "fp32":
            gm, gv = p.moments()
            assert np.array_equal(gm, m) and np.array_equal(gv, v)
            continue
        s = host(p.opt.scales).reshape(-1, 2)
        r = ref.random_bits(np.arange(p.total), 77, t)
        for codes, x, col, bias, largest, bits in ((p.opt.m, m, 0, 7, 448.0, r & 0xffff), (p.opt.v, v, 1, 15, 61440.0, r >> 16)):
            assert [ref.scale_for(float(top), largest) for top in np.abs(x).reshape(-1, BLOCK).max(1)] == list(s[:, col])
            y, least = np.abs(x) / s[:, col].repeat(BLOCK).astype(np.float32), f(2.0 ** (1 - bias))
            y = np.where(y < least, (y + least).astype(np.float64) - least, y)
            want = ref.grid(y, bits, bias, largest)
            want = np.where(x > 0, np.maximum(want, 1), want) if bias == 15 else want + np.where(np.signbit(x), 128, 0)
            assert np.array_equal(codes.cpu().numpy(), want)


def test_gradients_of_zero_and_far_apart(ev):
    """A block of zeros; magnitudes from 1e-18 to 1e6 within one: those that do not fit a block's codes become the smallest, not zero, for v."""
    for state in ("fp32", "8bit"):
        p = Problem(ev, [256, 256, 300], "fp32", "fp32", state, False, seed=3)
        p.grads[0].zero_()
        import torch
        p.grads[1].copy_(10.0 ** torch.linspace(-18, 6, 256, device="cuda"))
        p.check_step(ev, 1e-3, 1)
        p.check_step(ev, 1e-3, 2)
        if state == "8bit":
            assert not p.opt.m[:256].any() and not p.opt.v[:256].any() and (p.opt.v[256:512] >= 1).all()


def test_what_is_not_finite(ev):
    """NaN and infinity stay with their element; an infinite scale changes nothing."""
    import torch
    for state in ("fp32", "8bit"):
        p = Problem(ev, [600, 40], "bf16", "bf16", state, True, seed=4)
        before = [t.clone() for t in (*p.params, p.opt.master, p.opt.m, p.opt.v)]
        for x in (float("inf"), float("nan"), -float("inf")):
            ev.adamw_step(p.opt, 1e-2, 1, grad_scale=torch.tensor([x], device="cuda"))
            assert all(torch.equal(a, b) for a, b in zip(before, (*p.params, p.opt.master, p.opt.m, p.opt.v)))
        q = Problem(ev, [600, 40], "bf16", "bf16", state, True, seed=4)
        q.grads[0][5], q.grads[0][300], q.grads[1][39] = float("nan"), float("inf"), -float("inf")
        for t in (1, 2):
            ev.adamw_step(p.opt, 1e-2, t)
            ev.adamw_step(q.opt, 1e-2, t)
        bad = np.zeros(p.total, bool)
        bad[[5, 300, q.at[1] + 39]] = True
        assert np.isnan(q.flat(q.params)[bad]).all() and np.array_equal(p.flat(p.params)[~bad], q.flat(q.params)[~bad])
        (m, v), (m2, v2) = p.moments(), q.moments()
        assert np.array_equal(m[~bad], m2[~bad]) and np.array_equal(v[~bad], v2[~bad])
        if state == "8bit":
            assert (q.opt.m.cpu().numpy()[bad] == 0x7f).all() and (q.opt.v.cpu().numpy()[bad] == 0xf7).all()


def test_moments_move_on_average(ev):
    """v under a constant gradient: 0.1 % a step, far below half a step of its codes, and still it arrives, on average over elements."""
    import torch
    n = 1 << 16
    p, g = [torch.zeros(n, device="cuda")], [torch.full((n,), 2.0, device="cuda")]
    opt = ev.AdamW(p, g, state="8bit")
    steps = 200
    for t in range(1, steps + 1):
        ev.adamw_step(opt, 0.0, t, seed=11)
    m, v = ev.adamw_moments(opt, dtype=torch.float32)
    want_m, want_v = 2.0 * (1 - 0.9 ** steps), 4.0 * (1 - 0.999 ** steps)
    # an element is off by a random walk with steps of at most 1/8 of it; the mean of 65,536 by 1/256 of that
    assert abs(float(m.mean()) / want_m - 1) < 0.01 and abs(float(v.mean()) / want_v - 1) < 0.01
    # (m ends at 2, a code whose next value 0.9 2 + 0.1 2 is itself, where nothing is left to round)
    assert float(v.std()) > 0


def test_moments_as_values(ev):
    import torch
    p = Problem(ev, [1000, 77], "bf16", "bf16", "8bit", False, seed=6)
    ev.adamw_step(p.opt, 1e-3, 1, seed=3)
    want = p.moments()
    for dtype in (torch.bfloat16, torch.float32):
        for got, w in zip(ev.adamw_moments(p.opt, dtype=dtype), want):
            assert got.dtype is dtype and np.array_equal(host(got), w)   # (both types have all values of a code exactly)
    q = Problem(ev, [1000], "bf16", "bf16", "fp32", False)
    assert ev.adamw_moments(q.opt)[0] is q.opt.m
    # every code
    p.opt.m[:256] = torch.arange(256, device="cuda").to(torch.uint8)
    p.opt.v[:256] = torch.arange(256, device="cuda").clamp(max=247).to(torch.uint8)
    m, v = ev.adamw_moments(p.opt, dtype=torch.float32)
    want = p.moments()
    assert np.array_equal(host(m), want[0], equal_nan=True) and np.array_equal(host(v), want[1])


def test_schedule_and_graph(ev):
    """lr and t from the GPU, in a captured step that is replayed: the same as eager steps to what their functions differ."""
    import torch
    for state in ("fp32", "8bit"):
        p = Problem(ev, [3000, 41], "bf16", "fp32", state, True, seed=7)
        schedule, scale = torch.tensor([1e-2, 1.0], device="cuda"), torch.ones(1, device="cuda")
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                ev.adamw_step(p.opt, 99.0, 77, seed=5, schedule=schedule, grad_scale=scale)
        torch.cuda.synchronize()
        for t in (1, 2, 3, 500):
            schedule.copy_(torch.tensor([1e-2 / t, float(t)]))
            scale.fill_(1.0 / t)
            for g in p.grads:
                g.mul_(-1.1)

            def replay():
                graph.replay()
                torch.cuda.synchronize()
            lr, gs = float(schedule[0]), float(scale[0])
            p.check_step(ev, lr, t, seed=5, grad_scale=gs, call=replay)


def test_two_handles_on_two_streams(ev):
    import torch
    a = [Problem(ev, [50000, 3], "bf16", "bf16", "8bit", False, seed=8) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for t in (1, 2, 3):
        for p, s in zip(a, streams):
            with torch.cuda.stream(s):
                ev.adamw_step(p.opt, 1e-3, t, seed=1)
    torch.cuda.synchronize()
    for x, y in zip((*a[0].params, a[0].opt.m, a[0].opt.v, a[0].opt.scales), (*a[1].params, a[1].opt.m, a[1].opt.v, a[1].opt.scales)):
        assert torch.equal(x, y)


def test_refusals(ev):
    import torch
    w = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")      # noqa: E731
    with pytest.raises(ValueError):
        ev.AdamW([w(4)], [])
    with pytest.raises(TypeError):
        ev.AdamW([w(4), w(4, t=torch.float32)], [w(4), w(4)])
    with pytest.raises(TypeError):
        ev.AdamW([w(4, t=torch.float32)], [w(4)])
    with pytest.raises(TypeError):
        ev.AdamW([w(4, t=torch.float64)], [w(4, t=torch.float64)])
    with pytest.raises(ValueError):
        ev.AdamW([w(4, 2)], [w(2, 4)])
    with pytest.raises(ValueError):
        ev.AdamW([w(4, 2).t()], [w(4, 2).t()])
    with pytest.raises(ValueError):
        ev.AdamW([w(4)], [w(4)], scales=torch.ones(1, 2, device="cuda"))
    with pytest.raises(ValueError):
        ev.AdamW([w(4)], [w(4)], m=torch.zeros(4, device="cuda"))
    with pytest.raises(TypeError):
        ev.AdamW([w(4)], [w(4)], state="8bit", m=torch.zeros(256, device="cuda"))
    both = w(512)
    for pair in ([both, both], [both[:300], both[256:]]):
        with pytest.raises(ValueError, match="same memory"):
            ev.AdamW(pair, [torch.zeros_like(p) for p in pair])
    ev.AdamW([both[:256], both[256:]], [w(256), w(256)])
    opt = ev.AdamW([w(4)], [w(4)])
    for bad in (dict(t=0), dict(eps=0.0), dict(betas=(1.0, 0.9)), dict(lr=float("nan"))):
        with pytest.raises(ev.EvospecError):
            ev.adamw_step(opt, **{**dict(lr=1e-3, t=1), **bad})
    with pytest.raises(TypeError):
        ev.adamw_step(opt, 1e-3, 1, grad_scale=torch.ones(1, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        ev.adamw_step(opt, 1e-3, 1, schedule=torch.ones(3, device="cuda"))
    odd = w(20)[1:]
    with pytest.raises(ev.EvospecError):                             # not on 16 bytes
        ev.adamw_step(ev.AdamW([odd], [w(19)]), 1e-3, 1)


def test_tensors_of_a_handle_stay(ev):
    """Their addresses went to the library: another tensor in their place would not be seen."""
    import torch
    p = Problem(ev, [300, 5], "bf16", "bf16", "8bit", True)
    for name in ("params", "grads", "m", "v", "scales", "master"):
        with pytest.raises(AttributeError):
            setattr(p.opt, name, getattr(p.opt, name))
    with pytest.raises(TypeError):
        p.opt.grads[0] = torch.zeros_like(p.grads[0])
    bank = ev.LoraBank(torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 32, 8, dtype=torch.bfloat16, device="cuda"))
    for name in ("a", "b", "scale"):
        with pytest.raises(AttributeError):
            setattr(bank, name, getattr(bank, name))


def test_another_gpu_than_the_current_one(ev, monkeypatch):
    """Played: there is one GPU here."""
    from paper_2605_27390_amd import decode
    p = Problem(ev, [100], "bf16", "bf16", "8bit", False)
    here = decode._get_device()
    monkeypatch.setattr(decode, "_get_device", lambda: here + 1)
    with pytest.raises(ValueError, match="GPU"):
        ev.adamw_step(p.opt, 1e-3, 1)
    with pytest.raises(ValueError, match="GPU"):
        ev.adamw_moments(p.opt)
