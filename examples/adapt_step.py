"""Adapters that learn while they serve: requests decode with an adapter each, the KL gate admits the events where the draft is far from the target,
and a full buffer of them gives the adapters one step.

    python examples/adapt_step.py [--steps 12] [--state 8bit]

The draft's body is one projection with random weights, the target another one near it; they stand for the places at which a
program has these calls, not for language models.  Every decode step, for all requests:

  1. the shared projection, and beside it each request's adapter (lora_forward), give the draft's hidden states;
  2. the gate compares them with the target's logits (kl_gate) and admits what diverges;
  3. admitted events go to the buffer: input, support, target logits, adapter, depth.

Once the buffer is full, its events are put in order by adapter, and
  4. the forward pass runs again on them, with the adapters as they are now (lora_forward, which keeps h for the way back);
  5. the loss on the retained support gives its gradient to the hidden states (kd_loss), deeper steps count less;
  6. lora_backward gives the adapters' gradients, adamw_step their next values, and the buffer is empty again.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_27390_amd as ev  # noqa: E402

EPS_ALIGN = 0.1                                               # divergence from which an event is admitted
BUFFER = 32                                                   # events of an update
SUPPORT = 64                                                  # target logits that are kept of an event
DEPTH = 6                                                     # draft steps of a round
BETA = 0.3                                                    # how fast their weights fall


class Loop:
    def __init__(self, requests=9, adapters=4, V=4096, d=256, r=16, state="fp32", T=1.0, lr=2e-3, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weights(*shape, size=1.0):
            return torch.randn(shape, generator=g, device="cuda").mul_(size / math.sqrt(shape[-1])).to(torch.bfloat16)

        self.g, self.T, self.lr, self.d, self.r = g, T, lr, d, r
        self.W, self.W_lm = weights(d, d), weights(V, d, size=3.0)
        self.W_target = (self.W.float() + weights(d, d, size=0.5).float()).to(torch.bfloat16)
        # A from random numbers, B from zero: an adapter begins as none
        self.a, self.b = weights(adapters, r, d), torch.zeros(adapters, d, r, dtype=torch.bfloat16, device="cuda")
        self.bank = ev.LoraBank(self.a, self.b, torch.full((adapters,), 2.0, device="cuda"))
        self.grads = [torch.zeros(self.a.shape, device="cuda"), torch.zeros(self.b.shape, device="cuda")]
        self.opt = ev.AdamW([self.a, self.b], self.grads, state=state, master=True)
        # the last request has no adapter; row_off and adapter do not change as long as the requests do not
        self.adapter = [s % adapters for s in range(requests - 1)] + [-1]
        self.row_off = self._i32(range(requests + 1))
        self.of_request = self._i32(self.adapter)
        self.buffer, self.depth, self.updates = [], 0, 0

    def _i32(self, x):
        return torch.tensor(list(x), dtype=torch.int32, device="cuda")

    def forward(self, x, row_off, adapter, keep=False):
        """Hidden states of the draft: the shared projection and the adapters beside it; with keep also what the way back needs."""
        y = x @ self.W.t()
        h = ev.lora_forward(x, self.bank, row_off, adapter, y, keep=keep)
        return (y, h) if keep else y

    def step(self):
        """One decode step of all requests: (divergences, whether there was an update, which then returns what it saw)."""
        S = len(self.adapter)
        x = torch.randn((S, self.d), generator=self.g, device="cuda").to(torch.bfloat16)
        hidden = self.forward(x, self.row_off, self.of_request)
        z = (x @ self.W_target.t()).float() @ self.W_lm.float().t()
        support, target, _, kl = ev.kl_gate(z, hidden, self.W_lm, K=SUPPORT, T=self.T)
        self.depth = self.depth % DEPTH + 1
        for s, far in enumerate(kl.tolist()):
            if far > EPS_ALIGN and self.adapter[s] >= 0 and len(self.buffer) < BUFFER:
                self.buffer.append((self.adapter[s], x[s], support[s], target[s], self.depth, far))
        return kl, self.update() if len(self.buffer) == BUFFER else None

    def update(self):
        """One step of the adapters on the events of the buffer."""
        events = sorted(self.buffer, key=lambda e: e[0])
        self.buffer = []
        x, support, target = (torch.stack([e[i] for e in events]) for i in (1, 2, 3))
        base = sum(e[5] for e in events) / len(events)
        weight = torch.tensor([math.exp(-BETA * base * (e[4] - 1)) / len(events) for e in events], device="cuda")
        row_off, adapter = self._i32(range(len(events) + 1)), self._i32(e[0] for e in events)
        hidden, h = self.forward(x, row_off, adapter, keep=True)
        loss, dh, draft = ev.kd_loss(hidden, self.W_lm, support, target, weight=weight, T=self.T)
        ev.lora_backward(x, dh, self.bank, row_off, adapter, h=h, out_da=self.grads[0], out_db=self.grads[1])
        self.updates += 1
        ev.adamw_step(self.opt, self.lr, self.updates, weight_decay=0.0, seed=1)
        return {"x": x, "support": support, "target": target, "weight": weight, "row_off": row_off, "adapter": adapter, "hidden": hidden, "h": h,
                "loss": loss, "dh": dh, "draft": draft}


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=12)
    p.add_argument("--state", choices=("fp32", "8bit"), default="fp32")
    a = p.parse_args()
    loop = Loop(state=a.state)
    for i in range(a.steps):
        kl, update = loop.step()
        line = f"step {i}: mean divergence {float(kl.mean()):.3f}, {len(loop.buffer)} events wait"
        print(line if update is None else line + f"; update {loop.updates}: loss {float(update['loss'].sum()):.4f}")


if __name__ == "__main__":
    main()
