"""AdamW with the least eps: what never had a gradient stays as it is; and moments of more elements than one launch takes."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state", ["fp32", "8bit"])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30])
def test_elements_without_gradients(state, eps):
    import torch
    import paper_2605_27390_amd as ev
    for n in (1, 700):
        p = torch.randn(n, device="cuda").to(torch.bfloat16)
        g = torch.zeros_like(p)
        was = p.clone()
        opt = ev.AdamW([p], [g], state=state, master=True)
        for t in (1, 2):
            ev.adamw_step(opt, 1e-3, t, eps=eps, weight_decay=0.0, seed=3)
        assert torch.equal(p, was) and torch.equal(opt.master[:n], was.float()) and not opt.master[n:].any()
        assert not any(t.any() for t in ev.adamw_moments(opt))
        g[-1] = 1.0                                                  # (and one that has one moves by the rate, whatever eps)
        ev.adamw_step(opt, 1e-3, 3, eps=eps, weight_decay=0.0, seed=3)
        assert torch.equal(p[:-1], was[:-1]) and opt.master.isfinite().all() and float((opt.master[n - 1] - was[-1].float()).abs()) > 0


def test_moments_of_more_than_one_launch():
    """2^33 elements and three blocks, the codes of the last five blocks and of the first one not zero."""
    import torch
    import paper_2605_27390_amd as ev
    from paper_2605_27390_amd.adapt import lib
    blocks = 2 ** 25 + 3
    m, v = (torch.zeros(blocks * 256, dtype=torch.uint8, device="cuda") for _ in range(2))
    scales = torch.ones(blocks, 2, device="cuda")
    some = [0, *range(2 ** 25 - 2, 2 ** 25 + 3)]
    for b in some:
        m[256 * b:256 * b + 256] = 0x38                              # 1
        v[256 * b:256 * b + 256] = 0x78                              # 1
        scales[b, 0], scales[b, 1] = 2.0 ** (b % 8), 2.0 ** (b % 5)
    out = [torch.full((blocks * 256,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ev.adapt._check(lib.evospec_adamw_moments(m.data_ptr(), v.data_ptr(), scales.data_ptr(), blocks, 0, out[0].data_ptr(), out[1].data_ptr(),
                                              torch.cuda.current_stream().cuda_stream), "evospec_adamw_moments")
    for b in some:
        assert (out[0][256 * b:256 * b + 256] == 2.0 ** (b % 8)).all() and (out[1][256 * b:256 * b + 256] == 2.0 ** (b % 5)).all()
    assert not out[0][256:256 * (2 ** 25 - 2)].view(torch.int64).any() and not out[1][256:256 * (2 ** 25 - 2)].view(torch.int64).any()
    del m, v, out
    torch.cuda.empty_cache()
