"""The operators that learn from what the KL gate admits, as cases that can be measured: low-rank adapters of many requests beside
a shared projection, the distillation loss on the retained support with its gradient, and an AdamW step over many tensors.

Where `own` is false, `run` computes them in plain torch operations; where it is true, by the package's calls.
Inputs are the same for both.

Kinds:
  lora       y[t] += s (x[t] A^T) B^T with the adapter (A, B, s) of the request that row t belongs to; h = x A^T is kept for training
  lora_grad  its backward pass: dx += s (dy B) A, and the gradients of every adapter's A and B
  kd         per event: w T^2 KL(softmax(target / T) || softmax(draft / T)) on K tokens, draft = h . W[id], and its gradient to h
  adamw      one step over tensors of different sizes; moments in 32 bits, or in 8 bits and read back

Moments in 8 bits: 256 elements of a tensor share a scale for m and one for v, powers of two (the least that takes the block's largest
magnitude).  m is e4m3 (sign, 4 exponent bits, bias 7, 3 mantissa bits, largest 448); v, which has no sign, has 5 exponent bits (bias 15)
and 3 mantissa bits, largest 61,440; a v above zero is at least its smallest code.  Both are rounded at random: 16 bits for each out of a
counter's hash decide whether the magnitude goes up.  Tensors follow one another in flat buffers, each from a multiple of 256 on.
"""
import math

import torch

own = False

DEV = "cuda"
FLOATS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GROUP = 256
HYPER = {"lr": 1e-3, "betas": (0.9, 0.999), "eps": 1e-8, "weight_decay": 0.01, "t": 20, "seed": 1234}


def listed():
    return [
        # the next token of one request: a call is launches and latency
        {"name": "adapter, 1 token", "kind": "lora", "S": 1, "rows": 1, "n": 1, "r": 32, "d_in": 4096, "d_out": 4096, "keep": False},
        # a decode step of 64 requests over 16 adapters, the value projection
        {"name": "adapters, 64 tokens", "kind": "lora", "S": 64, "rows": 1, "n": 16, "r": 32, "d_in": 4096, "d_out": 1024, "keep": False},
        # the prompts of four requests, kept for training on them
        {"name": "adapters, 4 x 2,500", "kind": "lora", "S": 4, "rows": 2500, "n": 3, "r": 16, "d_in": 4096, "d_out": 4096, "keep": True},
        # a full replay buffer: 32 events of up to 6 draft steps, one adapter
        {"name": "gradients, 32 x 6", "kind": "lora_grad", "S": 32, "rows": 6, "n": 1, "r": 32, "d_in": 4096, "d_out": 4096, "kept": True,
         "dx": True},
        # a small model's, whose forward pass kept nothing
        {"name": "gradients, 5 x 333, odd", "kind": "lora_grad", "S": 5, "rows": 333, "n": 4, "r": 24, "d_in": 1000, "d_out": 520,
         "kept": False, "dx": True},
        # eight long sequences of two requests' adapters
        {"name": "gradients, 8 x 1,500", "kind": "lora_grad", "S": 8, "rows": 1500, "n": 2, "r": 32, "d_in": 4096, "d_out": 4096,
         "kept": True, "dx": True},
        # one admitted event
        {"name": "distil 1 event", "kind": "kd", "E": 1, "K": 256, "d": 4096, "V": 151936, "type": "bf16"},
        # a full replay buffer: 32 events of 6 draft steps
        {"name": "distil 192 steps", "kind": "kd", "E": 192, "K": 256, "d": 4096, "V": 151936, "type": "bf16"},
        # the adapters of two projections, with 32-bit masters
        {"name": "step, 4 tensors", "kind": "adamw", "tensors": 4, "size": 131072, "type": "bf16", "state": "fp32", "master": True},
        # those of many layers
        {"name": "step, 48 tensors, 8 bits", "kind": "adamw", "tensors": 48, "size": 262147, "type": "bf16", "state": "8bit",
         "master": False},
        # a whole draft layer
        {"name": "step, 8 x 16.8M", "kind": "adamw", "tensors": 8, "size": 16777216, "type": "bf16", "state": "fp32", "master": False},
        {"name": "step, 8 x 16.8M, 8 bits", "kind": "adamw", "tensors": 8, "size": 16777216, "type": "bf16", "state": "8bit",
         "master": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lora", "lora", "lora_grad", "lora_grad", "kd", "kd", "adamw", "adamw"])
    if kind in ("lora", "lora_grad"):
        d_in, d_out = 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 1024)
        S = _log(rng, 1, 64)
        most = 12000 * 4096 // max(4096, (d_in + d_out) // 2)
        c = {"kind": kind, "S": S, "rows": _log(rng, 1, max(1, most // S)), "n": _log(rng, 1, 16),
             "r": rng.choice([8, 16, 16, 24, 32, 32, 40, 64]), "d_in": d_in, "d_out": d_out}
        if kind == "lora":
            c["keep"] = rng.random() < 0.4
        else:
            c.update(kept=rng.random() < 0.6, dx=rng.random() < 0.8)
        return c
    if kind == "kd":
        d = 8 * _log(rng, 8, 1024)
        K = rng.choice([256, 256, _log(rng, 1, 256), _log(rng, 1, 1024)])
        V = _log(rng, 2000, min(151936, 151936 * 4096 // d))
        return {"kind": kind, "E": _log(rng, 1, max(1, min(1000, 192 * 256 * 4096 // (K * d)))), "K": K, "d": d, "V": V,
                "type": rng.choice(["bf16", "bf16", "fp32"])}
    tensors = _log(rng, 1, 48)
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    return {"kind": kind, "tensors": tensors, "size": _log(rng, 1, 16000000 // tensors), "type": dtype,
            "state": rng.choice(["fp32", "8bit"]), "master": dtype != "fp32" and rng.random() < 0.5}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _spread(most, S):
    """S whole numbers up to `most`: the largest first, the others anywhere in the upper half.  The case's own, whatever the seed."""
    low = (most + 1) // 2
    return [most] + [low + int((i * 0.6180339887) % 1.0 * (most - low + 1)) for i in range(1, S)]


def _requests(case):
    """How many rows each request has, and whose adapter: every ninth has none."""
    rows = _spread(case["rows"], case["S"])
    return rows, [-1 if s % 9 == 8 else (5 * s + 1) % case["n"] for s in range(case["S"])]


def _sizes(case):
    """Elements of every tensor, and where they start in the flat buffers."""
    sizes = _spread(case["size"], case["tensors"])
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // GROUP) * GROUP)
    return sizes, at


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = _gen(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV)      # noqa: E731
    s = {"case": case}
    if case["kind"] == "kd":
        E, K, d, V = case["E"], case["K"], case["d"], case["V"]
        s["W"] = torch.empty((V, d), dtype=torch.bfloat16, device=DEV).normal_(0, 0.02 * math.sqrt(4096 / d), generator=g)
        s["h"] = normal(E, d).to(torch.bfloat16)
        s["support"] = torch.rand((E, V), generator=g, device=DEV).topk(K, dim=1).indices.to(torch.int32)
        # the target's largest logits, by size: a few stand out
        z = torch.rand((E, K), generator=g, device=DEV).pow_(3).mul_(9).add_(2)
        s["target"] = z.sort(dim=1, descending=True).values
        # now and then an event has fewer tokens
        short = torch.arange(E, device=DEV) % 16 == 7
        s["support"][short, K - K // 10:] = -1
        s["target"][short, K - K // 10:] = math.nan
        # a step's weight falls with its depth, more where the loss is large
        s["weight"] = torch.exp(-0.3 * (0.5 + torch.rand(E, generator=g, device=DEV)) * (torch.arange(E, device=DEV) % 6))
        return s
    if case["kind"] == "adamw":
        sizes, at = _sizes(case)
        total, dtype = at[-1], FLOATS[case["type"]]
        w, grad = normal(total).mul_(0.02), torch.exp2(normal(total)).mul_(1e-3) * normal(total)
        m, v = normal(total).mul_(3e-4), (torch.exp2(normal(total)) * 1e-3).square_()
        own_part = torch.zeros(total, dtype=torch.bool, device=DEV)
        for a, n in zip(at, sizes):
            own_part[a:a + n] = True
        m, v, w = m * own_part, v * own_part, w * own_part
        s["params"] = [w[a:a + n].to(dtype) for a, n in zip(at, sizes)]
        s["grads"] = [grad[a:a + n].to(dtype) for a, n in zip(at, sizes)]
        if dtype is torch.float32:
            s["params"] = [p.clone() for p in s["params"]]
            s["grads"] = [p.clone() for p in s["grads"]]
        s["master"] = w if case["master"] else None
        if case["state"] == "8bit":
            r = torch.randint(0, 1 << 32, (total,), generator=g, device=DEV)
            s["m"], s["v"], s["scales"] = _plain_codes(m, v, r)
        else:
            s["m"], s["v"], s["scales"] = m, v, None
        if own:
            import paper_2605_27390_amd as ev
            s["opt"] = ev.AdamW(s["params"], s["grads"], state=case["state"], m=s["m"], v=s["v"], scales=s["scales"], master=s["master"])
        return s
    n, r, d_in, d_out = case["n"], case["r"], case["d_in"], case["d_out"]
    rows, adapter = _requests(case)
    T = sum(rows)
    s["row_off"] = _i32([0] + torch.tensor(rows).cumsum(0).tolist())
    s["adapter"] = _i32(adapter)
    s["A"] = (normal(n, r, d_in) / math.sqrt(d_in)).to(torch.bfloat16)
    s["B"] = (normal(n, d_out, r) * 0.03).to(torch.bfloat16)
    s["scale"] = 0.5 + torch.rand(n, generator=g, device=DEV)
    s["x"] = normal(T, d_in).to(torch.bfloat16)
    if case["kind"] == "lora":
        # what the shared projection left, as a part of a fused one's rows
        s["y"] = normal(T, d_out + 64).to(torch.bfloat16)[:, :d_out]
    else:
        s["dy"] = (normal(T, d_out) * 1e-3).to(torch.bfloat16)
        s["dx"] = (normal(T, d_in) * 1e-3).to(torch.bfloat16) if case["dx"] else None
        s["h"] = None
        if case["kept"]:
            s["h"] = _plain_down(s["x"], s["A"], _which(s), n).t().contiguous()
    if own:
        import paper_2605_27390_amd as ev
        s["bank"] = ev.LoraBank(s["A"], s["B"], s["scale"])
    return s


# ---------------------------------------------------------------- the plain forms

def _which(s):
    """Every row's adapter, -1 for none."""
    off = s["row_off"].long()
    return torch.repeat_interleave(s["adapter"].long(), off[1:] - off[:-1], output_size=s["x"].shape[0])


def _plain_down(x, w, which, n):
    """[T, r]: x times the transposed [r, d] of each row's adapter; zero for rows without one."""
    T, r = x.shape[0], w.shape[1]
    every = (x.float() @ w.reshape(n * r, -1).float().t()).view(T, n, r)
    return every.gather(1, which.clamp(min=0)[:, None, None].expand(T, 1, r))[:, 0] * (which >= 0)[:, None]


def _plain_placed(h, which, n):
    """[T, n r]: each row's h at its adapter's place."""
    T, r = h.shape
    every = torch.zeros((T, n, r), dtype=h.dtype, device=DEV)
    every.scatter_(1, which.clamp(min=0)[:, None, None].expand(T, 1, r), (h * (which >= 0)[:, None])[:, None])
    return every.view(T, n * r)


def _plain_lora(s):
    A, B, which, n = s["A"], s["B"], _which(s), s["case"]["n"]
    h = _plain_down(s["x"], A, which, n)
    up = _plain_placed(h * s["scale"][which.clamp(min=0)][:, None], which, n) @ B.transpose(1, 2).reshape(-1, B.shape[1]).float()
    s["y"].copy_(torch.where((which >= 0)[:, None], s["y"].float() + up, s["y"].float()))
    return {"y": s["y"], "h": h.t()} if s["case"]["keep"] else {"y": s["y"]}


def _plain_lora_grad(s):
    A, B, which, n = s["A"], s["B"], _which(s), s["case"]["n"]
    r, d_in = A.shape[1:]
    factor = s["scale"][which.clamp(min=0)][:, None]
    h = s["h"].t() if s["h"] is not None else _plain_down(s["x"], A, which, n)
    x, dy = s["x"].float(), s["dy"].float()
    g = _plain_placed(_plain_down(dy, B.transpose(1, 2), which, n) * factor, which, n)
    dA = (g.t() @ x).view(n, r, d_in)
    dB = (dy.t() @ _plain_placed(h * factor, which, n)).view(-1, n, r).transpose(0, 1)
    out = {"dA": dA, "dB": dB.contiguous()}
    if s["dx"] is not None:
        s["dx"].copy_(s["dx"].float() + g @ A.reshape(n * r, d_in).float())
        out["dx"] = s["dx"]
    return out


def _plain_kd(s):
    ids, w = s["support"].long(), s["weight"]
    mine = ids >= 0
    W = s["W"][ids.clamp(min=0)].float()                                                      # [E, K, d]
    z = torch.bmm(W, s["h"].float()[:, :, None])[:, :, 0]
    la = torch.log_softmax(torch.where(mine, s["target"], -math.inf).double(), 1)             # (temperature 1)
    lq = torch.log_softmax(torch.where(mine, z, -math.inf).double(), 1)
    a, q = la.exp(), lq.exp()
    loss = w.double() * torch.where(mine & (a > 0), a * (la - lq), 0.0).sum(1)
    c = torch.where(mine, w.double()[:, None] * (q - a), 0.0).float()
    dh = torch.bmm(c[:, None, :], W)[:, 0]
    return {"loss": loss.float(), "dh": dh.to(FLOATS[s["case"]["type"]]), "draft": torch.where(mine, z, math.nan)}


def _plain_hash(total, seed, t):
    """32 random bits for each element of the flat buffers, from its place, the seed and the step."""
    M = 0xffffffff
    x = torch.arange(total, device=DEV)
    x = x * 0x9e3779b1 + ((seed * 0x85ebca6b + t * 0xc2b2ae35) & M) & M
    x = (x ^ (x >> 16)) * 0x21f0aaad & M
    x = (x ^ (x >> 15)) * 0x735a2d97 & M
    return x ^ (x >> 15)


def _plain_power(x, most, least_exponent):
    """The least power of two, from 2^-100 to 2^100, with x <= most * power; most = 1.75 or 1.875 times 2^least_exponent."""
    f, e = torch.frexp(x)                                                                     # x = f 2^e, f in [1/2, 1)
    top = most / 2.0 ** (least_exponent + 1)
    return torch.ldexp(torch.ones_like(x), torch.where(x > 0, e - 1 - least_exponent + (f > top), -100).clamp(-100, 100))


def _plain_round(y, bits, bias):
    """Codes of magnitudes y with 3 mantissa bits: the low 20 of fp32's 23 are dropped, after 16 random ones are added at their
    top; below the smallest normal number with its exponent."""
    tiny = y < 2.0 ** (1 - bias)
    b = torch.where(tiny, y + 2.0 ** (1 - bias), y).view(torch.int32).long() + (bits << 4)
    return (b >> 20) - torch.where(tiny, (128 - bias) * 8, (127 - bias) * 8)


def _plain_codes(m, v, r):
    """m and v [blocks * 256] to codes (uint8) and scales [blocks, 2]."""
    mb, vb = m.view(-1, GROUP), v.view(-1, GROUP)
    sm, sv = _plain_power(mb.abs().amax(1), 448.0, 8), _plain_power(vb.amax(1), 61440.0, 15)
    cm = _plain_round((mb.abs() / sm[:, None]).view(-1), r & 0xffff, 7) + torch.where(m < 0, 128, 0)
    cv = _plain_round((vb / sv[:, None]).view(-1), r >> 16, 15)
    cv = torch.where((v > 0) & (cv == 0), 1, cv)
    return cm.to(torch.uint8), cv.to(torch.uint8), torch.stack([sm, sv], 1)


def _plain_values(m, v, scales):
    per = scales.repeat_interleave(GROUP, 0)
    e, f = (v >> 3).int(), (v & 7).float()
    return (m.view(torch.float8_e4m3fn).float() * per[:, 0],
            torch.where(e == 0, f * 2.0 ** -17, torch.ldexp(8 + f, e - 18)) * per[:, 1])


def _plain_flat(tensors, sizes, at):
    out = torch.zeros(at[-1], dtype=torch.float32, device=DEV)
    torch._foreach_copy_([out[a:a + n] for a, n in zip(at, sizes)], tensors)
    return out


def _plain_adamw(s):
    sizes, at = _sizes(s["case"])
    (b1, b2), t, lr = HYPER["betas"], HYPER["t"], HYPER["lr"]
    grad = _plain_flat(s["grads"], sizes, at)
    p = s["master"] if s["master"] is not None else _plain_flat(s["params"], sizes, at)
    small = s["case"]["state"] == "8bit"
    m, v = _plain_values(s["m"], s["v"], s["scales"]) if small else (s["m"], s["v"])
    m = m * b1 + grad * (1 - b1)
    v = v * b2 + grad * grad * (1 - b2)
    p = p * (1 - lr * HYPER["weight_decay"])
    p = p - lr / (1 - b1 ** t) * m / (torch.sqrt(v) / math.sqrt(1 - b2 ** t) + HYPER["eps"])
    torch._foreach_copy_(s["params"], [p[a:a + n] for a, n in zip(at, sizes)])
    if s["master"] is not None:
        s["master"].copy_(p)
    if small:
        for name, x in zip(("m", "v", "scales"), _plain_codes(m, v, _plain_hash(at[-1], HYPER["seed"], t))):
            s[name].copy_(x)
        m, v = (x.to(torch.bfloat16) for x in _plain_values(s["m"], s["v"], s["scales"]))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adamw_out(s, m, v)


def _adamw_out(s, m, v):
    out = {"params": s["params"], "m": m, "v": v}
    if s["master"] is not None:
        out["master"] = s["master"]
    return out


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2605_27390_amd as ev
        if kind == "lora":
            h = ev.lora_forward(s["x"], s["bank"], s["row_off"], s["adapter"], s["y"], keep=case["keep"])
            return {"y": s["y"], "h": h} if case["keep"] else {"y": s["y"]}
        if kind == "lora_grad":
            dA, dB = ev.lora_backward(s["x"], s["dy"], s["bank"], s["row_off"], s["adapter"], h=s["h"], dx=s["dx"])
            return {"dA": dA, "dB": dB} if s["dx"] is None else {"dA": dA, "dB": dB, "dx": s["dx"]}
        if kind == "kd":
            loss, dh, z = ev.kd_loss(s["h"], s["W"], s["support"], s["target"], weight=s["weight"], T=1.0, dtype=FLOATS[case["type"]])
            return {"loss": loss, "dh": dh, "draft": z}
        ev.adamw_step(s["opt"], HYPER["lr"], HYPER["t"], betas=HYPER["betas"], eps=HYPER["eps"], weight_decay=HYPER["weight_decay"],
                      seed=HYPER["seed"])
        m, v = ev.adamw_moments(s["opt"]) if case["state"] == "8bit" else (s["m"], s["v"])
        return _adamw_out(s, m, v)
    return {"lora": _plain_lora, "lora_grad": _plain_lora_grad, "kd": _plain_kd, "adamw": _plain_adamw}[kind](s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "kd":
        E, K, d = case["E"], case["K"], case["d"]
        return {"bytes": E * (K * (2 * d + 12) + d * (2 + (2 if case["type"] == "bf16" else 4)) + 8), "flops": 4 * E * K * d}
    if case["kind"] == "adamw":
        sizes, _ = _sizes(case)
        N = sum(sizes)
        size = 4 if case["type"] == "fp32" else 2
        a = 2 * size + (8 + size if case["master"] else size)                                 # gradient; parameter and master, in and out
        # (moments of 8 bits are read back as 16)
        b = 16 if case["state"] == "fp32" else 4 + 2 + 4
        return {"bytes": N * (a - size + b) if case["master"] else N * (a + b), "flops": 0}
    n, r, d_in, d_out = case["n"], case["r"], case["d_in"], case["d_out"]
    rows, adapter = _requests(case)
    T = sum(c for c, a in zip(rows, adapter) if a >= 0)
    used = len({a for a in adapter if a >= 0})
    weights = used * r * (d_in + d_out) * 2
    if case["kind"] == "lora":
        return {"bytes": weights + T * (2 * d_in + 4 * d_out) + (4 * r * T if case["keep"] else 0), "flops": 2 * T * r * (d_in + d_out)}
    inputs = T * 2 * (d_in + d_out) + (4 * r * T if case["kept"] else 0) + (4 * T * d_in if case["dx"] else 0)
    products = 2 * T * r * (d_in + 2 * d_out + (d_in if case["dx"] else 0) + (0 if case["kept"] else d_in))
    return {"bytes": weights + inputs + n * r * (d_in + d_out) * 4, "flops": products}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_kd(s):
    loss, dh, draft = [], [], []
    for e in range(s["h"].shape[0]):
        ids = s["support"][e].long()
        at = torch.nonzero(ids >= 0)[:, 0]
        W = s["W"][ids[at]].double()
        z = W @ s["h"][e].double()
        t = s["target"][e, at].double()
        a, q = torch.softmax(t, 0), torch.softmax(z, 0)
        w = float(s["weight"][e].double())
        loss.append(w * float((a * (t - torch.logsumexp(t, 0) - z + torch.logsumexp(z, 0))).sum()))
        dh.append(w * ((q - a) @ W))
        draft.append(torch.full(ids.shape, math.nan, dtype=torch.float64, device=DEV).index_copy_(0, at, z))
    return {"loss": torch.tensor(loss, dtype=torch.float64), "dh": torch.stack(dh), "draft": torch.stack(draft)}


def _exact_lora(s):
    case = s["case"]
    off, adapter = s["row_off"].tolist(), s["adapter"].tolist()
    forward = case["kind"] == "lora"
    n, r, d_in, d_out = case["n"], case["r"], case["d_in"], case["d_out"]
    T = off[-1]
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)                  # noqa: E731
    y = s["y"].double() if forward else None
    dx = s["dx"].double() if not forward and s["dx"] is not None else None
    h_all, dA, dB = new(r, T), new(n, r, d_in), new(n, d_out, r)
    for i, a in enumerate(adapter):
        if a < 0:
            continue
        rows = slice(off[i], off[i + 1])
        A, B, c = s["A"][a].double(), s["B"][a].double(), float(s["scale"][a].double())
        x = s["x"][rows].double()
        h = x @ A.t()
        if forward:
            h_all[:, rows] = h.t()
            y[rows] += c * (h @ B.t())
            continue
        dy = s["dy"][rows].double()
        g = c * (dy @ B)
        dA[a] += g.t() @ x
        dB[a] += c * (dy.t() @ h)
        if dx is not None:
            dx[rows] += g @ A
    if forward:
        return {"y": y, "h": h_all} if case["keep"] else {"y": y}
    return {"dA": dA, "dB": dB} if dx is None else {"dA": dA, "dB": dB, "dx": dx}


def _exact_rounded(x, scale, r, least, steps):
    """Magnitudes x of a block's scale on the grid of 3 mantissa bits, normal from 2^least on: up where 16 random bits say so."""
    y = x / scale
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** least))).clamp(min=least) - 3)
    whole = torch.floor(y / step + r.double() / 65536)
    return whole * step * scale, steps * scale


def _exact_adamw(s):
    case = s["case"]
    sizes, at = _sizes(case)
    (b1, b2), t, lr = HYPER["betas"], HYPER["t"], HYPER["lr"]
    small = case["state"] == "8bit"
    params, ms, vs = [], torch.zeros(at[-1], dtype=torch.float64, device=DEV), torch.zeros(at[-1], dtype=torch.float64, device=DEV)
    master = torch.zeros(at[-1], dtype=torch.float64, device=DEV)
    for a, n, p, g in zip(at, sizes, s["params"], s["grads"]):
        whole = -(-n // GROUP) * GROUP
        g = g.double()
        p = s["master"][a:a + n].double() if s["master"] is not None else p.double()
        if small:
            c = s["m"][a:a + n].long()
            low, e = c & 7, (c >> 3) & 15
            m = torch.where(e == 0, low * 2.0 ** -9, (8 + low) * torch.exp2(e.double() - 10)) * torch.where(c > 127, -1.0, 1.0)
            c = s["v"][a:a + n].long()
            low, e = c & 7, c >> 3
            v = torch.where(e == 0, low * 2.0 ** -17, (8 + low) * torch.exp2(e.double() - 18))
            block = (torch.arange(n, device=DEV) + a) // GROUP
            m, v = m * s["scales"][block, 0].double(), v * s["scales"][block, 1].double()
        else:
            m, v = s["m"][a:a + n].double(), s["v"][a:a + n].double()
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        p = p - lr * HYPER["weight_decay"] * p - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + HYPER["eps"])
        params.append(p)
        master[a:a + n] = p
        if small:
            x = (torch.arange(n, device=DEV) + a) * 0x9e3779b1 + HYPER["seed"] * 0x85ebca6b + t * 0xc2b2ae35
            for shift, factor in ((16, 0x21f0aaad), (15, 0x735a2d97)):
                x = x % (1 << 32)
                x = (x ^ (x >> shift)) * factor
            x = x % (1 << 32)
            x = x ^ (x >> 15)
            for value, bits, dst, least, largest in ((m, x & 0xffff, ms, -6, 448.0), (v, x >> 16, vs, -14, 61440.0)):
                pad = torch.zeros(whole, dtype=torch.float64, device=DEV)
                pad[:n] = value.abs()
                amax = pad.view(-1, GROUP).amax(1)
                scale = torch.exp2(torch.ceil(torch.log2((amax / largest).clamp(min=2.0 ** -100)))).repeat_interleave(GROUP)[:n]
                out, one = _exact_rounded(value.abs(), scale, bits, least, 2.0 ** (least - 3))
                if least == -14:
                    out = torch.where((value > 0) & (out == 0), one, out)
                dst[a:a + n] = torch.where(value < 0, -out, out)
        else:
            ms[a:a + n], vs[a:a + n] = m, v
    out = {"params": params, "m": ms, "v": vs}
    if s["master"] is not None:
        out["master"] = master
    return out


def exact(case, seed):
    global own
    s, mine = None, own
    own = False                                                                               # (no handle is needed)
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    return {"lora": _exact_lora, "lora_grad": _exact_lora, "kd": _exact_kd, "adamw": _exact_adamw}[case["kind"]](s)
