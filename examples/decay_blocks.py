"""Residual blocks of decayed attention over a long sequence, trained under a
checkpointing schedule of this package, and generating token by token.

A block is h += dropout(Wo attention(Wqkv norm(h))).  The sequence is cut into n
segments; what a segment passes to the next is the blocks' attention states, and
that is what the schedule's slots hold.  The reverse sweep evaluates a segment
again from the state in a slot: the norms and the attention give the same bits,
and dropout finds the same masks from its counters, so the gradients are those
of a sweep that stores every state, bit for bit.

    python examples/decay_blocks.py            # a few training steps, then tokens

The products with the weights are torch's.
"""
from __future__ import annotations

import dataclasses
import os
import sys

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1806_01117_amd as amb


@dataclasses.dataclass
class Config:
    width: int = 512
    heads: int = 8         # query heads
    kv_heads: int = 4      # key/value heads, each with a state
    depth: int = 2         # blocks
    batch: int = 4
    segments: int = 12     # n of the schedule
    steps: int = 96        # tokens per segment
    slots: int = 3         # segments' states held at a time
    p: float = 0.1         # dropout
    dtype: torch.dtype = torch.bfloat16

    @property
    def size(self) -> int:
        return self.width // self.heads


class Blocks:
    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg, self.seed = cfg, seed
        gen = torch.Generator().manual_seed(seed)
        c, kv = cfg, cfg.kv_heads * cfg.size
        make = lambda *shape: (torch.randn(*shape, generator=gen) / shape[-1] ** 0.5).to(device, c.dtype)  # noqa: E731
        self.params = {}
        for i in range(c.depth):
            self.params[f"norm{i}"] = torch.ones(c.width, device=device)
            self.params[f"qkv{i}"] = make(c.width + 2 * kv, c.width)
            self.params[f"out{i}"] = make(c.width, c.width)
        self.params["norm_last"] = torch.ones(c.width, device=device)
        # memories from 8 tokens to 1024
        far = torch.linspace(10.0, 3.0, c.kv_heads)
        self.log_decay = torch.log1p(-torch.exp2(-far)).to(device)

    def first_state(self, batch=None):
        c = self.cfg
        return [torch.zeros(batch or c.batch, c.kv_heads, c.size, c.size, device=self.log_decay.device) for _ in range(c.depth)]

    def _drop(self, t, i, h):
        """Dropout behind block i in segment t: a counter range of its own."""
        return dict(p=self.cfg.p, seed=self.seed, offset=(t * self.cfg.depth + i) * amb.dropout_counters(h))

    def _split(self, qkv):
        """q, k and v as they lie in one projection's output."""
        c = self.cfg
        kv = c.kv_heads * c.size
        q, k, v = qkv.split([c.width, kv, kv], dim=-1)
        head = lambda x: x.unflatten(-1, (-1, c.size))  # noqa: E731
        return head(q), head(k), head(v)

    def forward(self, t, x, state):
        """Segment t's inputs x [B, steps, width] and the blocks' states: its
        outputs, the states after it, and what the segment's gradients need."""
        c, kept, after, drop, residual = self.cfg, [], [], {}, None
        for i in range(c.depth):
            n = amb.add_norm(x, self.params[f"norm{i}"], residual=residual, **drop)
            qkv = n["y"] @ self.params[f"qkv{i}"].t()
            a = amb.decay_attention(*self._split(qkv), self.log_decay, s0=state[i])
            x = a["o"].flatten(2) @ self.params[f"out{i}"].t()
            kept.append((n["h"], n["y"], qkv, a["o"]))
            after.append(a["sn"])
            residual, drop = n["h"], self._drop(t, i, n["h"])
        n = amb.add_norm(x, self.params["norm_last"], residual=residual, **drop)
        return n["y"], after, (kept, n["h"])

    def backward(self, t, dy, state, dstate, kept, grads):
        """Gradients of segment t from those of its outputs and of the states
        after it; adds the parameters' to grads, returns the states' before it."""
        c, before = self.cfg, [None] * self.cfg.depth
        layers, h = kept
        rows = lambda z: z.reshape(-1, z.shape[-1])  # noqa: E731

        def add(name, g):
            grads[name] = g if name not in grads else grads[name] + g

        g = amb.add_norm_backward(dy, h, self.params["norm_last"], **self._drop(t, c.depth - 1, h))
        add("norm_last", g["dw"])
        for i in reversed(range(c.depth)):
            h, y, qkv, o = layers[i]
            dx, dh = g.get("dx", g["dresidual"]), g["dresidual"]
            add(f"out{i}", (rows(dx).t() @ rows(o.flatten(2))).float())
            do = (dx @ self.params[f"out{i}"]).unflatten(-1, (c.heads, c.size))
            dqkv = torch.empty_like(qkv)
            dq, dk, dv = self._split(dqkv)
            a = amb.decay_attention_backward(*self._split(qkv), self.log_decay, do, s0=state[i], dsn=dstate[i],
                                             out={"dq": dq, "dk": dk, "dv": dv})
            before[i] = a["ds0"]
            add(f"qkv{i}", (rows(dqkv).t() @ rows(y)).float())
            drop = self._drop(t, i - 1, h) if i else {}
            g = amb.add_norm_backward(dqkv @ self.params[f"qkv{i}"], h, self.params[f"norm{i}"], dh=dh, **drop)
            add(f"norm{i}", g["dw"])
        return before


def gradients(blocks: Blocks, xs, targets, slots=None):
    """Loss (half the mean square of the outputs' distance from the targets) and
    gradients over all segments, under the schedule for `slots` (None: the
    configuration's) slots; also how many segments were evaluated."""
    n = len(xs)
    scale = 1.0 / targets[0].numel() / n
    live, dstate, kept, grads, held = (0, blocks.first_state()), None, None, {}, {}
    loss, evaluated = torch.zeros((), device=targets[0].device), 0
    for line in amb.schedule_text(n, slots or blocks.cfg.slots).splitlines()[1:]:
        op, *num = line.split()
        num = [int(v) for v in num]
        if op == "A":  # advance the live state
            for t in range(*num):
                live = (t + 1, blocks.forward(t, xs[t], live[1])[1])
                evaluated += 1
        elif op == "S":
            held[num[0]] = live
        elif op == "R":
            live = held[num[0]]
        else:  # "F" or "Y": the last segment whose gradients are still wanted
            t, state = num[0], live[1]
            assert live[0] == t
            y, after, kept = blocks.forward(t, xs[t], state)
            evaluated += 1
            d = y.float() - targets[t].float()
            loss = loss + 0.5 * scale * d.square().sum()
            if dstate is None:
                dstate = [torch.zeros_like(s) for s in after]
            dstate = blocks.backward(t, (d * scale).to(y.dtype), state, dstate, kept, grads)
    return loss, grads, evaluated


@torch.no_grad()
def generate(blocks: Blocks, prompt, tokens: int):
    """Feeds the outputs back as inputs, token by token, after a prompt
    [B, T, width]; without dropout.  The last norm's outputs are in 8 bits."""
    c = blocks.cfg
    state, out = blocks.first_state(prompt.shape[0]), []
    x = prompt
    for _ in range(tokens):
        residual = None
        for i in range(c.depth):
            n = amb.add_norm(x, blocks.params[f"norm{i}"], residual=residual)
            q, k, v = blocks._split(n["y"] @ blocks.params[f"qkv{i}"].t())
            if x.shape[1] == 1:
                o = amb.decay_attention_step(q, k, v, blocks.log_decay, state[i])
            else:
                o = amb.decay_attention(q, k, v, blocks.log_decay, s0=state[i], out={"sn": state[i]})["o"]
            x, residual = o.flatten(2) @ blocks.params[f"out{i}"].t(), n["h"]
        last = amb.add_norm(x[:, -1:], blocks.params["norm_last"], residual=residual[:, -1:], out_dtype="f8")
        x = (last["y"].float() * last["scale"]).to(c.dtype)
        out.append(x)
    return torch.cat(out, 1)


def main():
    cfg = Config()
    gen = torch.Generator(device="cuda").manual_seed(1)
    # a slow wave in noise: the target is the wave
    t = torch.arange(cfg.segments * cfg.steps + 1, device="cuda") / 40.0
    phase = 6.28 * torch.rand(cfg.batch, 1, cfg.width, generator=gen, device="cuda")
    wave = torch.sin(t[None, :, None] + phase)
    noisy = (wave + 0.5 * torch.randn(wave.shape, generator=gen, device="cuda")).to(cfg.dtype)
    xs = [s.contiguous() for s in noisy[:, :-1].split(cfg.steps, 1)]
    targets = [s.contiguous().to(cfg.dtype) for s in wave[:, 1:].split(cfg.steps, 1)]
    blocks = Blocks(cfg)
    for step in range(8):
        loss, grads, evaluated = gradients(blocks, xs, targets)
        print(f"step {step}: loss {float(loss):.4f}, {evaluated} evaluations of {cfg.segments} segments with {cfg.slots} slots")
        for name, p in blocks.params.items():
            p -= (20.0 * grads[name]).to(p.dtype)
    made = generate(blocks, xs[0], 40)
    print("generated", tuple(made.shape), "mean square", float(made.float().square().mean()))


if __name__ == "__main__":
    main()
