"""Outputs, updated tensors and workspaces that share memory with an input or one another are refused before anything runs."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def arena(n=1 << 16):
    """Zeros, and views of them: of a type and shape, from a byte on."""
    import torch
    buf = torch.zeros(n, dtype=torch.uint8, device="cuda")

    def view(at, dtype, *shape):
        size = torch.empty(0, dtype=dtype).element_size()
        for s in shape:
            size *= s
        return buf[at:at + size].view(dtype).view(shape)
    return buf, view


def test_adapters(ev):
    import torch
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    buf, view = arena()
    T, r, d = 6, 8, 16
    # x and y, and dy and dx, in the same rows
    rows, grads = view(0, bf16, T, 2 * d), view(1024, bf16, T, 2 * d)
    x, y, dy, dx = rows[:, :d], rows[:, d:], grads[:, :d], grads[:, d:]
    a, b, scale = view(4096, bf16, 1, r, d), view(6144, bf16, 1, d, r), view(8192, f32, 1)
    off, ad = view(9216, i32, 2), view(10240, i32, 1)
    off[1] = T
    h, da, db = view(12288, f32, r, T), view(16384, f32, 1, r, d), view(20480, f32, 1, d, r)
    bank = ev.LoraBank(a, b, scale)
    ws = view(24576, torch.uint8, ev.lora_backward_workspace_bytes(bank, 1, T))
    ev.lora_forward(x, bank, off, ad, y, out_h=h)
    ok = dict(x=x, dy=dy, bank=bank, row_off=off, adapter=ad, h=h, dx=dx, out_da=da, out_db=db, workspace=ws)
    ev.lora_backward(**ok)
    was = buf.clone()
    for bad in (4096, 4096 + 32 * (r - 1), 6144, 8192 - 64, 9216 - 32, 10240, 0):
        with pytest.raises(ValueError, match="overlaps"):
            ev.lora_forward(x, bank, off, ad, view(bad, bf16, T, d))
    for bad in (0, 32 * T, 4096 + 64, 6144, 8192 - 32, 9216, 10240 - 4):
        with pytest.raises(ValueError, match="overlaps"):
            ev.lora_forward(x, bank, off, ad, y, out_h=view(bad, f32, r, T))
    for bad in (0, 1024, 4096, 6144, 8192, 9216, 10240, 12288):
        for name, shape, dtype in (("dx", (T, d), bf16), ("out_da", (1, r, d), f32), ("out_db", (1, d, r), f32), ("workspace", tuple(ws.shape), torch.uint8)):
            with pytest.raises(ValueError, match="overlaps"):
                ev.lora_backward(**{**ok, name: view(bad, dtype, *shape)})
    for bad in (dict(out_db=view(16384, f32, 1, d, r)), dict(out_da=view(20480 + 256, f32, 1, r, d)),
                dict(workspace=view(16384 + 16, torch.uint8, ws.numel())), dict(workspace=view(20480, torch.uint8, ws.numel())),
                dict(dx=view(16384, bf16, T, d)), dict(h=grads.view(f32).view(-1)[:r * T].view(r, T))):
        with pytest.raises(ValueError, match="overlaps"):
            ev.lora_backward(**{**ok, **bad})
    assert torch.equal(buf, was)


def test_distillation(ev):
    import torch
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    buf, view = arena(1 << 17)
    E, K, d, V = 3, 16, 64, 20
    h, W, support, target, weight = view(0, bf16, E, d), view(1024, bf16, V, d), view(8192, i32, E, K), view(12288, f32, E, K), view(16384, f32, E)
    loss, dh, draft = view(20480, f32, E), view(24576, bf16, E, d), view(28672, f32, E, K)
    n = ev.kd_loss_workspace_bytes(E, K, d)
    assert n > 0
    ok = dict(h=h, W_lm=W, support=support, target=target, weight=weight, out_loss=loss, out_dh=dh, out_draft=draft, workspace=view(32768, torch.uint8, n))
    ev.kd_loss(**ok)
    was = buf.clone()
    for at in (0, 1024, 8192, 12288, 16384):
        for name, shape, dtype in (("out_loss", (E,), f32), ("out_dh", (E, d), bf16), ("out_draft", (E, K), f32), ("workspace", (n,), torch.uint8)):
            with pytest.raises(ValueError, match="overlaps"):
                ev.kd_loss(**{**ok, name: view(at, dtype, *shape)})
    for bad in (dict(out_dh=view(20480, bf16, E, d)), dict(out_draft=view(24576, f32, E, K)), dict(workspace=view(28672, torch.uint8, n)),
                dict(workspace=view(20480, torch.uint8, n)), dict(out_loss=view(28672 + 4, f32, E))):
        with pytest.raises(ValueError, match="overlaps"):
            ev.kd_loss(**{**ok, **bad})
    assert torch.equal(buf, was)


@pytest.mark.parametrize("state", ["fp32", "8bit"])
def test_adamw(ev, state):
    import torch
    bf16, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    buf, view = arena()
    sizes, kind = (256, 300), f32 if state == "fp32" else u8
    flat = 256 + 512
    params, grads = [view(0, bf16, 256), view(512, bf16, 300)], [view(2048, bf16, 256), view(2560, bf16, 300)]
    ok = dict(m=view(4096, kind, flat), v=view(8192, kind, flat), master=view(16384, f32, flat))
    if state == "8bit":
        ok["scales"] = view(12288, f32, 3, 2)
    opt = ev.AdamW(params, grads, state=state, **ok)
    ev.adamw_step(opt, 1e-3, 1)
    was = buf.clone()
    for name, shape, dtype in (("m", (flat,), kind), ("v", (flat,), kind), ("master", (flat,), f32), ("scales", (3, 2), f32)):
        if name not in ok:
            continue
        for at in {0, 512, 2048, 2560, 4096, 8192, 16384} - {dict(m=4096, v=8192, master=16384).get(name)}:
            with pytest.raises(ValueError, match="overlaps"):
                ev.AdamW(params, grads, state=state, **{**ok, name: view(at, dtype, *shape)})
    with pytest.raises(ValueError, match="overlaps"):
        ev.AdamW(params, [view(0, bf16, 256), grads[1]], state=state, **ok)
    ev.AdamW(params, [grads[0], view(2048, bf16, 300)], state=state, **ok)           # (gradients are only read)
    if state == "8bit":
        for bad in (dict(out_m=view(4096, bf16, flat)), dict(out_v=view(8192, bf16, flat)), dict(out_m=view(12288, bf16, flat)),
                    dict(out_m=view(24576, bf16, flat), out_v=view(24576 + 1024, bf16, flat))):
            with pytest.raises(ValueError, match="overlaps"):
                ev.adamw_moments(opt, **bad)
        ev.adamw_moments(opt, out_m=view(24576, bf16, flat), out_v=view(28672, bf16, flat))
        buf[24576:32768], was[24576:32768] = 0, 0
    assert torch.equal(buf, was)
