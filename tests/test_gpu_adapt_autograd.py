"""What the calls change in place is seen by autograd: a graph that saved the old values says so, and what requires a gradient is refused while
gradients are recorded."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def problem(ev):
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)        # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")                        # noqa: E731
    return normal, ev.LoraBank(normal(1, 8, 64), normal(1, 32, 8)), i32([0, 5]), i32([0])


def graph_on(t):
    """A loss whose gradient needs t as it is now."""
    import torch
    w = torch.ones_like(t, requires_grad=True)
    return (w * t).sum()


def test_a_graph_that_saved_what_changes(ev):
    import torch
    normal, bank, off, ad = problem(ev)
    x, dy, support = normal(5, 64), normal(5, 32), torch.arange(8, dtype=torch.int32, device="cuda").expand(5, 8).contiguous()
    f32 = lambda *s: torch.zeros(s, device="cuda")                   # noqa: E731
    params, grads = [normal(300), normal(7)], [normal(300), normal(7)]
    opt = ev.AdamW(params, grads, master=True)
    small = ev.AdamW([normal(300)], [normal(300)], state="8bit")
    y, h, dx, da, db = normal(5, 32), f32(8, 5), normal(5, 64), f32(1, 8, 64), f32(1, 32, 8)
    loss, dh, draft, out = f32(5), normal(5, 64), f32(5, 8), normal(512)
    forward = lambda **kw: ev.lora_forward(x, bank, off, ad, y, **kw)                                        # noqa: E731
    backward = lambda **kw: ev.lora_backward(x, dy, bank, off, ad, **kw)                                     # noqa: E731
    distil = lambda **kw: ev.kd_loss(x, bank.a[0], support, f32(5, 8), **kw)                                 # noqa: E731
    step = lambda: ev.adamw_step(opt, 1e-3, 1)                       # noqa: E731
    calls = [(y, forward), (h, lambda: forward(out_h=h)), (dx, lambda: backward(dx=dx)), (da, lambda: backward(out_da=da)),
             (db, lambda: backward(out_db=db)), (loss, lambda: distil(out_loss=loss)), (dh, lambda: distil(out_dh=dh)),
             (draft, lambda: distil(out_draft=draft)), (out, lambda: ev.adamw_moments(small, out_m=out)), (out, lambda: ev.adamw_moments(small, out_v=out)),
             *((t, step) for t in (*params, opt.m, opt.v, opt.master))]
    for t, call in calls:
        graph_on(t).backward()                                       # (unchanged: fine)
        saved = graph_on(t)
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            saved.backward()
    kept = graph_on(x)                                               # what is read only
    forward(), backward(dx=dx), distil(), step()
    kept.backward()


def test_what_requires_a_gradient(ev):
    import torch
    normal, bank, off, ad = problem(ev)
    x, y, dy, dx = normal(5, 64), normal(5, 32).requires_grad_(), normal(5, 32), normal(5, 64).requires_grad_()
    was = y.detach().clone(), dx.detach().clone()
    with pytest.raises(ValueError, match="requires a gradient"):
        ev.lora_forward(x, bank, off, ad, y)
    with pytest.raises(ValueError, match="requires a gradient"):     # (part of a graph)
        ev.lora_forward(x, bank, off, ad, y * 2)
    with pytest.raises(ValueError, match="requires a gradient"):
        ev.lora_backward(x, dy, bank, off, ad, dx=dx)
    with pytest.raises(ValueError, match="requires a gradient"):
        ev.lora_forward(x, bank, off, ad, y.detach(), out_h=torch.zeros(8, 5, device="cuda", requires_grad=True))
    with pytest.raises(ValueError, match="requires a gradient"):
        ev.lora_backward(x, dy, bank, off, ad, out_da=torch.zeros(1, 8, 64, device="cuda", requires_grad=True))
    support = torch.arange(8, dtype=torch.int32, device="cuda").expand(5, 8).contiguous()
    with pytest.raises(ValueError, match="requires a gradient"):
        ev.kd_loss(x, bank.a[0], support, torch.zeros(5, 8, device="cuda"), out_dh=normal(5, 64).requires_grad_())
    assert torch.equal(y, was[0]) and torch.equal(dx, was[1])
    with torch.no_grad():
        ev.lora_forward(x, bank, off, ad, y)
        ev.lora_backward(x, dy, bank, off, ad, dx=dx)
    assert not torch.equal(y, was[0]) and not torch.equal(dx, was[1])
    # adapters that are leaves with a gradient, the parameters of an optimiser: read as they are, and stepped
    a, b = bank.a.clone().requires_grad_(), bank.b.clone().requires_grad_()
    again = ev.LoraBank(a, b)
    da, db = ev.lora_backward(x, dy, again, off, ad)
    opt = ev.AdamW([a, b], [da, db])
    ev.adamw_step(opt, 1e-3, 1)
    assert not torch.equal(a, bank.a) and a.requires_grad
    ev.kd_loss(x.clone().requires_grad_(), bank.a[0], support, torch.zeros(5, 8, device="cuda"))


def test_inference_tensors(ev):
    import torch
    normal, bank, off, ad = problem(ev)
    with torch.inference_mode():
        x, y = normal(5, 64), normal(5, 32)
        was = y.clone()
        ev.lora_forward(x, bank, off, ad, y)
    ev.lora_forward(x, bank, off, ad, y)                             # (and outside)
    assert not torch.equal(y, was)
