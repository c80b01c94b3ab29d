"""Low-rank adapters against the definition in 64 bits: forward, backward, masks that leave requests empty, strides, streams, graphs."""
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


class Problem:
    def __init__(self, ev, rows, adapter, n, r, d_in, d_out, seed=0, lead=0, tail=0, scale=True, wide=0):
        import torch
        rng = np.random.default_rng(seed)
        off = np.concatenate([[0], np.cumsum(rows)]) + lead
        self.T = int(off[-1]) + tail
        self.off, self.adapter = off.astype(np.int32), np.asarray(adapter, np.int32)
        normal = lambda *s: ref.bf16(rng.normal(size=s))             # noqa: E731
        self.x, self.y, self.dy, self.dx = normal(self.T, d_in), normal(self.T, d_out), normal(self.T, d_out), normal(self.T, d_in)
        self.A, self.B = normal(n, r, d_in) * 2.0 ** -4, normal(n, d_out, r) * 2.0 ** -2
        self.scale = np.float32(rng.normal(size=n)).astype(np.float64) if scale else None

        def rows_of(x):
            t = torch.full((x.shape[0], x.shape[1] + wide), 7.0, dtype=torch.bfloat16, device="cuda")[:, wide // 2:wide // 2 + x.shape[1]]
            t.copy_(dev(x, torch.bfloat16))
            return t
        self.rows_of = rows_of
        self.tx, self.ty, self.tdy, self.tdx = rows_of(self.x), rows_of(self.y), rows_of(self.dy), rows_of(self.dx)
        self.toff, self.tad = dev(self.off), dev(self.adapter)
        self.bank = ev.LoraBank(dev(self.A, torch.bfloat16), dev(self.B, torch.bfloat16), None if self.scale is None else dev(self.scale, torch.float32))

    def check_forward(self, y, h=None):
        want, bound, wh, hb = ref.lora_forward(self.x, self.A, self.B, self.scale, self.off, self.adapter, self.y)
        got = y.double().cpu().numpy()
        untouched = np.isnan(wh[0])
        assert np.array_equal(got[untouched], self.y[untouched])
        far = np.abs(got - want) - bound
        assert not (far > 0).any(), (float(far.max()), np.argwhere(far > 0)[:4])
        if h is not None:
            got = h.double().cpu().numpy()[:, ~untouched]
            assert (np.abs(got - wh[:, ~untouched]) <= hb[:, ~untouched]).all()

    def check_backward(self, da, db, dx=None):
        a, ab, b, bb, x, xb = ref.lora_backward(self.x, self.dy, self.A, self.B, self.scale, self.off, self.adapter, self.dx if dx is not None else None)
        for name, got, want, bound in (("da", da, a, ab), ("db", db, b, bb), ("dx", dx, x, xb)):
            if got is not None:
                far = np.abs(got.double().cpu().numpy() - want) - bound
                assert not (far > 0).any(), (name, float(far.max()), np.argwhere(far > 0)[:4])


CASES = [
    # rows, adapters, n, r, d_in, d_out
    ([1], [0], 1, 8, 8, 8),
    ([1], [0], 1, 32, 4096, 4096),
    ([1] * 16, [i % 5 for i in range(16)], 5, 16, 520, 264),
    ([1] * 70, [(i * 3) % 7 - 1 for i in range(70)], 6, 32, 256, 128),
    ([3, 0, 5, 1, 0], [1, 0, -1, 2, 1], 3, 24, 72, 200),
    ([16, 17, 15, 32, 33, 31], [0, 1, 0, 2, 9, 1], 3, 40, 1000, 136),
    ([64], [0], 2, 64, 512, 1032),
    ([100, 129, 1], [1, 0, 1], 2, 48, 264, 2056),
    ([700], [0], 1, 8, 136, 64),
    ([300, 301], [3, 3], 4, 56, 2048, 8),
    ([0, 0], [0, 1], 2, 16, 64, 64),
    ([5, 6], [-1, 7], 2, 16, 64, 64),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("wide", [0, 48])
def test_forward(ev, case, wide):
    rows, adapter, n, r, d_in, d_out = CASES[case]
    p = Problem(ev, rows, adapter, n, r, d_in, d_out, seed=case, lead=case % 3, tail=case % 4, scale=case % 2 == 0, wide=wide)
    import torch
    h = torch.full((r, p.T), 9.0, dtype=torch.float32, device="cuda")
    assert ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, out_h=h) is h
    p.check_forward(p.ty, h)
    none = np.isnan(ref.lora_forward(p.x, p.A, p.B, p.scale, p.off, p.adapter, p.y)[2][0])
    assert not h.cpu().numpy()[:, none].any()
    again = p.rows_of(p.y)
    assert ev.lora_forward(p.tx, p.bank, p.toff, p.tad, again) is again
    assert torch.equal(again, p.ty)                                  # the same bits, whether h is kept or not


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("kept", [True, False])
def test_backward(ev, case, kept):
    import torch
    rows, adapter, n, r, d_in, d_out = CASES[case]
    p = Problem(ev, rows, adapter, n, r, d_in, d_out, seed=50 + case, lead=case % 2, tail=case % 3, scale=case % 2 == 1, wide=(case % 2) * 16)
    h = None
    if kept:
        h = torch.full((r, p.T), float("nan"), device="cuda")        # (columns of rows without an adapter are not read)
        ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, out_h=h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)
    outs = [torch.full_like(t, float("nan")) for t in (da, db)]
    da2, db2 = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, out_da=outs[0], out_db=outs[1])
    assert da2 is outs[0] and torch.equal(da, da2) and torch.equal(db, db2)


def test_many_requests_and_rows(ev):
    """More than 64 requests, some empty, with rows of several tiles each; and a large number of rows of one adapter."""
    rng = np.random.default_rng(3)
    rows = [int(v) for v in rng.integers(0, 90, size=150)]
    p = Problem(ev, rows, [int(v) for v in rng.integers(-1, 9, size=150)], 9, 16, 128, 192, seed=4)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    p.check_forward(p.ty, h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)
    p = Problem(ev, [9000], [0], 1, 32, 64, 72, seed=5)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    p.check_forward(p.ty, h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)


@pytest.mark.parametrize("seed", range(6))
def test_requests_that_follow_one_another(ev, seed):
    """Runs of requests with one adapter, that begin and end at and between multiples of 16 and 32 rows, with empty ones among them."""
    rng = np.random.default_rng(seed)
    S = [40, 64, 65, 130, 200, 500][seed]
    rows = rng.choice([0, 1, 1, 2, 3, 5, 15, 16, 17, 32, 48], size=S) if seed % 2 else rng.choice([0, 1, 1, 1, 2, 16, 32], size=S)
    adapter = np.repeat(rng.integers(-1, 3, size=S), rng.integers(1, 20, size=S))[:S]
    p = Problem(ev, [int(v) for v in rows], [int(v) for v in adapter], 3, [16, 40][seed // 3], 64, 72, seed=20 + seed, lead=int(rng.integers(0, 40)),
                tail=seed)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    p.check_forward(p.ty, h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)


@pytest.mark.parametrize("seed", range(3))
def test_requests_that_follow_one_another_at_rank_64(ev, seed):
    """The same in tiles of 32 rows."""
    rng = np.random.default_rng(40 + seed)
    S = [30, 64, 90][seed]
    rows = rng.choice([0, 1, 16, 31, 32, 33, 64, 70], size=S)
    adapter = np.repeat(rng.integers(-1, 3, size=S), rng.integers(1, 20, size=S))[:S]
    p = Problem(ev, [int(v) for v in rows], [int(v) for v in adapter], 3, 64, 72, 136, seed=43 + seed, lead=int(rng.integers(0, 40)), tail=seed)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    p.check_forward(p.ty, h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)


@pytest.mark.parametrize("r,d", [(8, 4096), (32, 4096), (64, 4096), (16, 64), (40, 72), (64, 64)])
def test_more_tiles_than_units(ev, r, d):
    """Rows so many that a compute unit has several tiles, and (4,096) so large that they do not fit the caches."""
    p = Problem(ev, [4000, 5001, 17], [1, 0, 1], 2, r, d, d, seed=80 + r, lead=3)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    p.check_forward(p.ty, h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)


@pytest.mark.parametrize("S", [0, 1, 9, 64, 70, 300, 5000])
@pytest.mark.parametrize("r", [8, 64])
def test_kept_columns_of_rows_without_an_adapter(ev, S, r):
    """h is written whole: zeros for requests without an adapter, and before, between and behind the requests' rows."""
    import torch
    rng = np.random.default_rng(S)
    adapter = [-1 if s % 9 == 8 or s % 64 == 63 else s // 3 % 2 for s in range(S)]
    for rows in ([int(v) for v in rng.integers(0, 40 if S < 1000 else 3, size=S)], [1] * S):
        p = Problem(ev, rows, adapter, 2, r, 64, 72, seed=70 + S, lead=37, tail=50)
        h = torch.full((r, p.T), float("nan"), device="cuda")
        ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, out_h=h)
        p.check_forward(p.ty, h)
        none = np.isnan(ref.lora_forward(p.x, p.A, p.B, p.scale, p.off, p.adapter, p.y)[2][0])
        assert not h.cpu().numpy()[:, none].any()


@pytest.mark.parametrize("r", [8, 24, 64])
@pytest.mark.parametrize("adapter", [[1] * 6, [1, 1, 1, 1, 4, 0], [0, 1, 2, 3, 4, -1], [-1] * 6, [2, 9, -1, -1, 2, 9]])
def test_shares_of_adapters(ev, adapter, r):
    """Rows enough for an adapter's to be split, by its share of them: all of them, most, alike, none; twice the same."""
    import torch
    p = Problem(ev, [600, 500, 601, 433, 37, 700], adapter, 5, r, 136, 200, seed=60, lead=2, tail=1)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h)
    p.check_backward(da, db)
    outs = [torch.full_like(t, float("nan")) for t in (da, db)]
    need = ev.lora_backward_workspace_bytes(p.bank, 6, p.T)
    ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, out_da=outs[0], out_db=outs[1],
                     workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(da, outs[0]) and torch.equal(db, outs[1])


def test_thousands_of_requests(ev):
    rng = np.random.default_rng(30)
    for S, adapters in ((5000, rng.integers(-1, 5, size=5000)), (4200, np.where(np.arange(4200) % 700 == 699, 1, -1)), (4097, np.zeros(4097, int))):
        p = Problem(ev, [int(v) for v in rng.integers(0, 4, size=S)], [int(v) for v in adapters], 5, 8, 16, 24, seed=31, lead=3)
        h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
        p.check_forward(p.ty, h)
        da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
        p.check_backward(da, db, p.tdx)


def test_rows_far_into_memory(ev):
    """Rows whose place passes 2^31 elements and 2^32 bytes: only the last ones belong to a request."""
    import torch
    T, stride = 70000, 32768
    p = Problem(ev, [5, 3], [1, 0], 2, 16, 64, 64, seed=6)
    buf = torch.empty((T, stride), dtype=torch.bfloat16, device="cuda")
    view = lambda at: buf[:, at:at + 64]                             # noqa: E731
    x, y, dy, dx = view(0), view(64), view(128), view(192)
    for t, src in ((x, p.tx), (y, p.ty), (dy, p.tdy), (dx, p.tdx)):
        t[-8:] = src
    off = p.toff + (T - 8)
    h = ev.lora_forward(x, p.bank, off, p.tad, y, keep=True)
    p.check_forward(y[-8:], h[:, -8:])
    da, db = ev.lora_backward(x, dy, p.bank, off, p.tad, h=h, dx=dx)
    p.check_backward(da, db, dx[-8:])


def test_offsets_that_pass_the_rows(ev):
    """Values of row_off are clamped to the rows there are, and a request that ends before it begins has none."""
    import torch
    p = Problem(ev, [4, 5, 6], [0, 1, 0], 2, 16, 64, 72, seed=7)
    p.off = np.array([-3, 4, 9, 1 << 30], np.int32)
    p.toff = dev(p.off)
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    p.check_forward(p.ty, h)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    p.check_backward(da, db, p.tdx)
    p = Problem(ev, [4, 5, 6], [0, 1, 0], 2, 16, 64, 72, seed=7)
    p.off = np.array([15, 7, 7, 7], np.int32)
    p.toff = dev(p.off)
    ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty)
    assert torch.equal(p.ty, dev(p.y, torch.bfloat16))
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad)
    assert not da.any() and not db.any()


def test_no_rows(ev):
    import torch
    bank = ev.LoraBank(torch.ones(2, 8, 16, dtype=torch.bfloat16, device="cuda"), torch.ones(2, 24, 8, dtype=torch.bfloat16, device="cuda"))
    none = lambda d: torch.empty(0, d, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")        # noqa: E731
    for off, ad in ((i32([0, 0]), i32([1])), (i32([0]), i32([]))):
        ev.lora_forward(none(16), bank, off, ad, none(24))
        da, db = ev.lora_backward(none(16), none(24), bank, off, ad, dx=none(16), out_da=torch.full((2, 8, 16), 3.0, device="cuda"),
                                  out_db=torch.full((2, 24, 8), 3.0, device="cuda"))
        assert not da.any() and not db.any()
    x, y = torch.ones(5, 16, dtype=torch.bfloat16, device="cuda"), torch.ones(5, 24, dtype=torch.bfloat16, device="cuda")
    ev.lora_forward(x, bank, i32([0]), i32([]), y)
    assert (y == 1).all()


def test_what_is_not_finite_stays_where_it_is(ev):
    """A row with NaN or infinity changes its own row of y and dx, and the gradients of its own adapter; rows without an adapter nothing."""
    import torch
    rows, adapter = [20, 7, 40], [0, -1, 1]
    p = Problem(ev, rows, adapter, 3, 16, 128, 96, seed=8)
    bad_x, bad_dy = p.tx.clone(), p.tdy.clone()
    bad_x[3, 5], bad_x[4, 6], bad_dy[10, 7] = float("nan"), float("inf"), float("-inf")
    bad_x[22], bad_dy[23] = float("nan"), float("nan")
    y, dx = p.ty.clone(), p.tdx.clone()
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    hb = ev.lora_forward(bad_x, p.bank, p.toff, p.tad, y, keep=True)
    good = torch.ones(p.T, dtype=torch.bool, device="cuda")
    good[[3, 4]] = False
    assert torch.equal(y[good], p.ty[good]) and y[3].isnan().all() and not y[4].isfinite().any()
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    da2, db2 = ev.lora_backward(bad_x, bad_dy, p.bank, p.toff, p.tad, h=hb, dx=dx)
    good[[3, 4]], good[10] = True, False
    assert torch.equal(dx[good], p.tdx[good]) and not dx[10].isfinite().any()
    assert torch.equal(da[1:], da2[1:]) and torch.equal(db[1:], db2[1:])
    assert da2[0, :, 5].isnan().all() and not da2[0].isfinite().all(0)[5] and not db2[0].isfinite().any()
    # an infinite input whose weight is not zero: infinite, not NaN
    one = torch.zeros(1, 16, dtype=torch.bfloat16, device="cuda")
    one[0, 2] = float("inf")
    bank = ev.LoraBank(torch.ones(1, 8, 16, dtype=torch.bfloat16, device="cuda").abs(), torch.ones(1, 8, 8, dtype=torch.bfloat16, device="cuda"))
    out = torch.zeros(1, 8, dtype=torch.bfloat16, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")        # noqa: E731
    ev.lora_forward(one, bank, i32([0, 1]), i32([0]), out)
    assert (out == float("inf")).all()


def test_large_and_small_magnitudes(ev):
    """h and g have fp32's range on their way."""
    for up in (2.0 ** 60, 2.0 ** -60):
        p = Problem(ev, [40, 9], [0, 1], 2, 16, 64, 64, seed=9, scale=False)
        import torch
        p.x, p.dy, p.A, p.B = p.x * up, p.dy * up, p.A * up ** 0.5, p.B / up ** 1.5
        p.tx, p.tdy = dev(p.x, torch.bfloat16), dev(p.dy, torch.bfloat16)
        p.bank = ev.LoraBank(dev(p.A, torch.bfloat16), dev(p.B, torch.bfloat16))
        h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
        p.check_forward(p.ty, h)


def test_refusals(ev):
    import torch
    p = Problem(ev, [5, 6], [0, 1], 2, 16, 64, 72, seed=10)
    f32 = torch.zeros(11, 64, device="cuda")
    with pytest.raises(TypeError):
        ev.lora_forward(f32, p.bank, p.toff, p.tad, p.ty)
    with pytest.raises(TypeError):
        ev.lora_forward(p.tx, p.bank, p.toff.long(), p.tad, p.ty)
    with pytest.raises(ValueError):
        ev.lora_forward(p.tx, p.bank, p.toff[:2], p.tad, p.ty)
    with pytest.raises(ValueError):
        ev.lora_forward(p.tx[:5], p.bank, p.toff, p.tad, p.ty)
    with pytest.raises(ValueError):
        ev.lora_forward(p.tx.t().contiguous().t(), p.bank, p.toff, p.tad, p.ty)
    with pytest.raises(ValueError):
        ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty[:1].expand(11, 72))
    with pytest.raises(ValueError):
        ev.lora_forward(p.tx[:1].expand(11, 64), p.bank, p.toff, p.tad, p.ty)
    with pytest.raises(ValueError):
        ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, out_h=torch.zeros(11, 16, device="cuda"))
    with pytest.raises(ev.EvospecError):                             # rows that do not begin on 16 bytes
        ev.lora_forward(torch.zeros(11, 68, dtype=torch.bfloat16, device="cuda")[:, 4:], p.bank, p.toff, p.tad, p.ty)
    with pytest.raises(ev.EvospecError):
        ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ev.EvospecError):
        ev.LoraBank(torch.zeros(1, 12, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 64, 12, dtype=torch.bfloat16, device="cuda"))
    square = Problem(ev, [4], [0], 1, 8, 64, 64)
    with pytest.raises(ValueError, match="overlaps"):
        ev.lora_forward(square.tx, square.bank, square.toff, square.tad, square.tx)
    with pytest.raises(ValueError, match="overlaps"):
        ev.lora_backward(square.tx, square.tdy, square.bank, square.toff, square.tad, dx=square.tdy)
    assert torch.equal(p.ty, dev(p.y, torch.bfloat16))


def test_streams_and_graphs(ev):
    """On a stream of its own; and captured, with the caller's buffers, replayed between eager calls."""
    import torch
    p = Problem(ev, [33, 1, 64, 5], [1, 0, -1, 1], 2, 32, 512, 256, seed=11)
    y0, dx0 = p.ty.clone(), p.tdx.clone()
    h = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty, keep=True)
    da, db = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=h, dx=p.tdx)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y, dx = y0.clone(), dx0.clone()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hs = ev.lora_forward(p.tx, p.bank, p.toff, p.tad, y, keep=True)
        das, dbs = ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad, h=hs, dx=dx)
    s.synchronize()
    mine = ~torch.isnan(torch.from_numpy(ref.lora_forward(p.x, p.A, p.B, p.scale, p.off, p.adapter, p.y)[2][0])).cuda()
    assert torch.equal(hs[:, mine], h[:, mine])
    for a, b in ((y, p.ty), (dx, p.tdx), (das, da), (dbs, db)):
        assert torch.equal(a, b)
    S, T = p.tad.numel(), p.T
    ws = torch.empty(ev.lora_backward_workspace_bytes(p.bank, S, T), dtype=torch.uint8, device="cuda")
    x, dy, h2, da2, db2 = p.tx.clone(), p.tdy.clone(), torch.zeros_like(h), torch.empty_like(da), torch.empty_like(db)

    def both():
        y.copy_(y0)
        dx.copy_(dx0)
        ev.lora_forward(x, p.bank, p.toff, p.tad, y, out_h=h2)
        ev.lora_backward(x, dy, p.bank, p.toff, p.tad, h=h2, dx=dx, out_da=da2, out_db=db2, workspace=ws)
    with torch.cuda.stream(s):
        both()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            both()
    for k in range(4):
        x.copy_(p.tx * (k + 1))
        dy.copy_(p.tdy * (2 - k))
        graph.replay()
        torch.cuda.synchronize()
        ye, dxe = y0.clone(), dx0.clone()
        he = ev.lora_forward(x, p.bank, p.toff, p.tad, ye, keep=True)
        dae, dbe = ev.lora_backward(x, dy, p.bank, p.toff, p.tad, h=he, dx=dxe)
        for a, b in ((y, ye), (dx, dxe), (da2, dae), (db2, dbe)):
            assert torch.equal(a, b), k


def test_another_gpu_than_the_current_one(ev, monkeypatch):
    """Played: there is one GPU here."""
    from paper_2605_27390_amd import decode
    p = Problem(ev, [3], [0], 1, 8, 64, 64)
    here = decode._get_device()
    monkeypatch.setattr(decode, "_get_device", lambda: here + 1)
    with pytest.raises(ValueError, match="GPU"):
        ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty)
    with pytest.raises(ValueError, match="GPU"):
        ev.lora_backward(p.tx, p.tdy, p.bank, p.toff, p.tad)
    monkeypatch.undo()
    p.bank._device += 1
    with pytest.raises(ValueError, match="GPU"):
        ev.lora_forward(p.tx, p.bank, p.toff, p.tad, p.ty)
