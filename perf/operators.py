"""The operators of a residual block over a long sequence: what is timed and checked.

Three operators belong to such a block: attention whose state decays (a
recurrence over the sequence, whose state is what a checkpoint holds), dropout
whose mask is generated again wherever a step is evaluated again, and the
root-mean-square norm behind the residual's addition.  A case is one call (or
a forward call and its backward call) on inputs that already lie in HBM.

``own`` false: plain torch operations in 32 bits.  ``own`` true: the calls of
this package.

Definitions (lambda = exp(log_decay[head]), one state per key/value head):

* attention: S_i = lambda S_{i-1} + k_i v_i^T, o_i = scale S_i^T q_i for the
  first ``lengths[b]`` tokens of row b; further outputs and gradients are zero.
* dropout: row r, column c takes half (c % 2) of word ((c % 8) / 2) of
  Philox-4x32-10 (Salmon, Moraes, Dror and Shaw 2011) at the 64-bit counter
  offset + r ceil(cols / 8) + c / 8 under the 64-bit key `seed`; the element is
  kept where these 16 bits are >= t = round(65536 p), and then scaled by
  65536 / (65536 - t).
* norm: h = residual + dropout(x), y = w h / sqrt(mean(h^2) + eps); in 8 bits
  y = scale * e4m3 with scale = max|y| / 448 of a row or of 128 columns.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = "f32", "bf16"
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
SIZE = {F32: 4, BF16: 2}
EPS = 1e-6


def _attn(name, do, dtype, batch, steps, heads, group, dk, dv, layout="bthd", ragged=False, state=True):
    """`heads` key/value heads with `group` query heads each; do: "step", "fwd", "bwd" or "train" (both)."""
    return {"name": name, "op": "attn", "do": do, "dtype": dtype, "batch": batch, "steps": steps, "heads": heads,
            "group": group, "dk": dk, "dv": dv, "layout": layout, "ragged": ragged, "state": state}


def _norm(name, do, dtype, rows, cols, p, out="same", block=0):
    """do: "fwd" or "train"; out: "same" (the dtype) or "f8" with one scale per `block` columns (0: per row)."""
    return {"name": name, "op": "norm", "do": do, "dtype": dtype, "rows": rows, "cols": cols, "p": p, "out": out,
            "block": block}


def _drop(name, dtype, rows, cols, p, residual):
    return {"name": name, "op": "drop", "do": "train", "dtype": dtype, "rows": rows, "cols": cols, "p": p,
            "residual": residual}


def listed():
    return [
        # one token of a small generator, batch 4 and width 256 (as 4 heads of
        # 64): nothing but latency
        _attn("step_b4", "step", F32, 4, 1, 4, 1, 64, 64),
        # one token for each of 128 sequences at width 2048 (16 query heads
        # that share 8 states): reads and writes every state once
        _attn("step_b128", "step", BF16, 128, 1, 8, 2, 128, 128),
        # a prompt of 20000 tokens at width 4096, one sequence: the state is
        # carried over a long sequence by few heads; q, k, v as they lie in
        # one projection's output
        _attn("prompt_t20000", "fwd", BF16, 1, 20000, 8, 4, 128, 128, layout="packed", state=False),
        # prompts of different lengths in one batch, one of them empty; head
        # sizes that fill no tile, heads shared by three
        _attn("prompt_ragged", "fwd", BF16, 6, 1999, 5, 3, 80, 112, ragged=True),
        # training at the sizes of the 512-wide LSTM over 1000 steps (batch 64),
        # steps first in memory as that LSTM's inputs are
        _attn("train_h512_t1000", "train", F32, 64, 1000, 8, 1, 64, 64, layout="tbhd"),
        # the backward call at the sizes of the 2048-wide bf16 LSTM over 10000 steps
        _attn("backward_h2048_t10000", "bwd", BF16, 16, 10000, 16, 1, 128, 128),
        # a batch of single tokens on its way into an 8-bit product
        _norm("norm_f8_b128", "fwd", BF16, 128, 2048, 0.0, out="f8"),
        # a prompt of 20000 tokens on its way into an 8-bit product
        _norm("norm_f8_t20000", "fwd", BF16, 20000, 4096, 0.0, out="f8", block=128),
        # training, width 4096: the residual's addition with dropout, the norm,
        # and the gradients of both
        _norm("norm_train_w4096", "train", BF16, 65536, 4096, 0.1),
        # training in 32 bits, a width that no vector divides
        _norm("norm_train_odd", "train", F32, 1999, 1001, 0.25),
        # dropout of one step's output (batch 64, width 512)
        _drop("drop_b64", F32, 64, 512, 0.5, False),
        # dropout of a whole sequence's outputs into the residual, and its gradient
        _drop("drop_t10000", BF16, 160000, 2048, 0.1, True),
    ]


def _between(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm."""
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    most = {op: max(work(c)["bytes"] for c in listed() if c["op"] == op) for op in ("attn", "norm", "drop")}
    while True:
        op = rng.choice(["attn", "attn", "norm", "drop"])
        dtype = rng.choice([F32, BF16])
        if op == "attn":
            do = rng.choice(["step", "fwd", "bwd", "train"])
            c = _attn("", do, dtype, _between(rng, 1, 128), 1 if do == "step" else _between(rng, 1, 20000),
                      _between(rng, 1, 16), rng.randint(1, 4), 16 * rng.randint(1, 8), 16 * rng.randint(1, 8),
                      rng.choice(["bthd", "tbhd", "packed"]), rng.random() < 0.4, rng.random() < 0.7)
        elif op == "norm":
            out = rng.choice(["same", "f8"])
            c = _norm("", "fwd" if out == "f8" else "train", dtype, _between(rng, 1, 65536), _between(rng, 16, 8192),
                      rng.choice([0.0, rng.uniform(0.02, 0.6)]), out, rng.choice([0, 128]) if out == "f8" else 0)
        else:
            c = _drop("", dtype, _between(rng, 1, 160000), _between(rng, 16, 8192), rng.uniform(0.02, 0.9),
                      rng.random() < 0.5)
        if work(c)["bytes"] <= most[op]:
            del c["name"]
            return c


def work(case):
    c, size = case, SIZE[case["dtype"]]
    if c["op"] == "attn":
        B, T, H, G, dk, dv = (c[k] for k in ("batch", "steps", "heads", "group", "dk", "dv"))
        q, k, v, o = B * T * H * G * dk, B * T * H * dk, B * T * H * dv, B * T * H * G * dv
        S = B * H * dk * dv * 4
        n = 0 if not c["state"] else 1
        if c["do"] == "step":
            return {"bytes": (q + k + v + o) * size + 2 * S, "flops": B * H * dk * dv * (3 + 2 * G)}
        # the recurrence itself: the state's update and its product with each
        # query, and for the gradients the same for dS and its three products
        fwd = {"bytes": (q + k + v + o) * size + (1 + n) * S, "flops": B * T * H * dk * dv * 2 * (1 + G)}
        bwd = {"bytes": (2 * (q + k + v) + o) * size + 3 * n * S, "flops": B * T * H * dk * dv * 2 * (4 + 2 * G)}
        if c["do"] == "train":  # q, k, v are read by both calls
            return {"bytes": fwd["bytes"] + bwd["bytes"], "flops": fwd["flops"] + bwd["flops"]}
        return fwd if c["do"] == "fwd" else bwd
    n, rows, cols = c["rows"] * c["cols"], c["rows"], c["cols"]
    if c["op"] == "norm":
        if c["do"] == "fwd":
            scales = rows * (-(-cols // c["block"]) if c["block"] else 1) * 4 if c["out"] == "f8" else 0
            # x, residual, w in; h, y and scales out
            return {"bytes": 3 * n * size + n * (1 if c["out"] == "f8" else size) + cols * 4 + scales, "flops": 8 * n}
        # forward: x, residual, w in, h, y out; backward: dy, dh, h, w in,
        # dresidual, dx and dw out
        return {"bytes": (4 + 4 + (1 if c["p"] else 0)) * n * size + 3 * cols * 4, "flops": 20 * n}
    # x (and residual) in, y out; dy in, dx out
    return {"bytes": (4 + (1 if c["residual"] else 0)) * n * size, "flops": 6 * n}


# ---- inputs -----------------------------------------------------------------


def _qkv(c, gen, heads_of):
    """Tensors [B, T, heads, size] for (heads, size) of heads_of, laid out as the case says."""
    B, T, dt = c["batch"], c["steps"], DTYPE[c["dtype"]]
    if c["layout"] == "packed":
        flat = torch.randn(B, T, sum(h * d for h, d in heads_of), generator=gen, device="cuda").to(dt)
        return [x.view(B, T, h, d) for x, (h, d) in zip(flat.split([h * d for h, d in heads_of], dim=2), heads_of)]
    if c["layout"] == "tbhd":
        return [torch.randn(T, B, h, d, generator=gen, device="cuda").to(dt).transpose(0, 1) for h, d in heads_of]
    return [torch.randn(B, T, h, d, generator=gen, device="cuda").to(dt) for h, d in heads_of]


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "attn":
        B, T, H, G, dk, dv = (c[k] for k in ("batch", "steps", "heads", "group", "dk", "dv"))
        s["q"], s["k"], s["v"] = _qkv(c, gen, [(H * G, dk), (H, dk), (H, dv)])
        # memories from 8 tokens to 4096 and, for the first head of several, without end
        far = torch.linspace(12.0, 3.0, H, device="cuda")
        s["log_decay"] = torch.log1p(-torch.exp2(-far))
        if H > 1:
            s["log_decay"][0] = 0.0
        s["s0"] = torch.randn(B, H, dk, dv, generator=gen, device="cuda") if c["state"] or c["do"] == "step" else None
        s["lengths"] = None
        if c["ragged"]:
            n = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            n[0] = T
            if B > 1:
                n[1] = 0
            if B > 2:
                n[2] = 1
            s["lengths"] = n
        if c["do"] in ("bwd", "train"):
            s["do"] = _qkv(dict(c, layout="bthd" if c["layout"] == "packed" else c["layout"]), gen, [(H * G, dv)])[0]
            s["dsn"] = torch.randn(B, H, dk, dv, generator=gen, device="cuda") if c["state"] else None
        s["scale"] = dk ** -0.5
        return s
    rows, cols, dt = c["rows"], c["cols"], DTYPE[c["dtype"]]
    make = lambda: torch.randn(rows, cols, generator=gen, device="cuda").to(dt)  # noqa: E731
    # a key and a counter as a training program has them: the counter has
    # passed 32 bits
    s["seed"], s["offset"] = 0x1806_0111_7000_0000 + seed, (1 << 33) + 977 * seed
    s["x"] = make()
    if c["op"] == "norm":
        s["residual"] = make()
        s["w"] = 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")
        if c["do"] == "train":
            s["dy"], s["dh"] = make(), make()
    else:
        s["residual"] = make() if c["residual"] else None
        s["dy"] = make()
    return s


# ---- the plain forms --------------------------------------------------------

CHUNK = 256


def _decayed(q, k, v, g):
    """o_i = sum over j <= i of lambda^(i-j) (q_i . k_j) v_j, over whole chunks at once.

    q [B, H, G, T, a], k [B, H, 1, T, a], v [B, H, 1, T, e], all fp32; or k and v
    with G heads and q with one, whose results the caller adds up.
    """
    B, H, T = q.shape[0], q.shape[1], q.shape[3]
    n = -(-T // CHUNK)
    C = min(CHUNK, T)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0, 0, n * C - T)).reshape(*x.shape[:3], n, C, x.shape[4])  # noqa: E731
    q, k, v = cut(q), cut(k), cut(v)
    g = g.view(1, H, 1, 1, 1, 1)
    i = torch.arange(C, device=q.device, dtype=torch.float32)
    gap = i[:, None] - i[None, :]
    inside = torch.where(gap >= 0, torch.exp(g * gap.clamp(min=0)), 0.0)
    o = torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * inside, v)
    if n > 1:
        # each chunk's contribution to the state at its end, and the states at
        # the chunks' starts as sums of those before
        local = torch.matmul((k * torch.exp(g * (C - 1 - i).view(C, 1))).transpose(-1, -2), v)
        c = torch.arange(n, device=q.device, dtype=torch.float32)
        steps = c[:, None] - 1 - c[None, :]
        across = torch.where(steps >= 0, torch.exp(g[..., 0] * C * steps.clamp(min=0)), 0.0)
        start = torch.matmul(across, local.flatten(-2)).view(local.shape)
        o = o + torch.matmul(q * torch.exp(g * (i + 1).view(C, 1)), start)
    return o.flatten(3, 4)[:, :, :, :T]


def _heads(x, H, alive):
    """[B, T, H G, d] to fp32 [B, H, G, T, d], with zeros past each row's length."""
    B, T, HG, d = x.shape
    x = x.float().view(B, T, H, HG // H, d).permute(0, 2, 3, 1, 4)
    return x if alive is None else torch.where(alive, x, 0.0)


def _tokens(x, dtype):
    """fp32 [B, H, G, T, d] to [B, T, H G, d]."""
    B, H, G, T, d = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(B, T, H * G, d).to(dtype)


def _plain_attn(s):
    c, g, scale = s["case"], s["log_decay"], s["scale"]
    B, T, H, G, dk, dv = (c[k] for k in ("batch", "steps", "heads", "group", "dk", "dv"))
    dt = DTYPE[c["dtype"]]
    if c["do"] == "step":
        live = 1.0 if s["lengths"] is None else (s["lengths"] > 0).view(B, 1, 1, 1)
        q, k, v = (s[n].float().view(B, H, -1, d) for n, d in (("q", dk), ("k", dk), ("v", dv)))
        S = torch.exp(g).view(1, H, 1, 1) * s["s0"] + k.transpose(-1, -2) * v
        o = scale * torch.matmul(q, S)
        if s["lengths"] is not None:
            S, o = torch.where(live, S, s["s0"]), torch.where(live, o, 0.0)
        s["s0"].copy_(S)
        return {"o": o.reshape(B, 1, H * G, dv).to(dt), "sn": s["s0"]}
    n = torch.full((B,), T, device=g.device, dtype=torch.int32) if s["lengths"] is None else s["lengths"]
    t = torch.arange(T, device=g.device, dtype=torch.float32).view(1, 1, 1, T, 1)
    n = n.float().view(B, 1, 1, 1, 1)
    alive = None if s["lengths"] is None else t < n
    q, k, v = (_heads(s[x], H, alive) for x in ("q", "k", "v"))
    g5 = g.view(1, H, 1, 1, 1)
    fore = torch.exp(g5 * (t + 1))  # lambda^(i+1): from the initial state to token i
    back = torch.exp(g5 * (n - 1 - t).clamp(min=0))  # lambda^(n-1-j): from token j to the last state
    s0, out = s["s0"], {}
    whole = torch.exp(g5 * n)[..., 0, :, :]
    if c["do"] in ("fwd", "train"):
        o = _decayed(q, k, v, g)
        sn = torch.matmul((k * back).transpose(-1, -2), v)[:, :, 0]
        if s0 is not None:
            o = o + torch.matmul(q, s0[:, :, None]) * fore
            sn = sn + whole * s0
        out["o"], out["sn"] = _tokens(o * scale, dt), sn
    if c["do"] in ("bwd", "train"):
        do = _heads(s["do"], H, alive) * scale
        dq = _decayed(do, v, k, g)
        flip = lambda x: x.flip(3)  # noqa: E731
        shape = lambda x: x.expand(B, H, G, T, x.shape[-1])  # noqa: E731
        dv = flip(_decayed(flip(shape(k)), flip(q), flip(do), g)).sum(2, keepdim=True)
        dk = flip(_decayed(flip(shape(v)), flip(do), flip(q), g)).sum(2, keepdim=True)
        if s0 is not None:
            dq = dq + torch.matmul(do, s0[:, :, None].transpose(-1, -2)) * fore
            dsn = s["dsn"][:, :, None]
            dv = dv + torch.matmul(k, dsn) * back
            dk = dk + torch.matmul(v, dsn.transpose(-1, -2)) * back
            ds0 = torch.matmul((q * fore).transpose(-1, -2), do).sum(2) + whole * s["dsn"]
            out["ds0"] = ds0
        if alive is not None:
            dq, dk, dv = (torch.where(alive, x, 0.0) for x in (dq, dk, dv))
            out.update({} if "o" not in out else {"o": torch.where(alive[:, 0, 0].view(B, T, 1, 1), out["o"], 0.0)})
        out["dq"], out["dk"], out["dv"] = _tokens(dq, dt), _tokens(dk, dt), _tokens(dv, dt)
    elif alive is not None:
        out["o"] = torch.where(alive[:, 0, 0].view(B, T, 1, 1), out["o"], 0.0)
    return out


def _product(a, b):
    """High and low 32 bits of a b, a an int64 tensor of 32-bit values, b a 32-bit constant."""
    low, high = (a & 0xFFFF) * b, (a >> 16) * b
    whole = high + (low >> 16)
    return whole >> 16, ((whole & 0xFFFF) << 16) | (low & 0xFFFF)


def _round(x, key):
    """One round of Philox-4x32 on four tensors of 32-bit words."""
    h0, l0 = _product(x[0], 0xD2511F53)
    h1, l1 = _product(x[2], 0xCD9E8D57)
    return h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0


def _keep(s, rows, cols):
    """The factors of dropout, fp32 [rows, cols], or 1.0."""
    at = round(65536 * s["case"]["p"])
    if at == 0:
        return 1.0
    wide = -(-cols // 8)
    n = s["offset"] + torch.arange(rows * wide, device="cuda", dtype=torch.int64)
    x = n & 0xFFFFFFFF, n >> 32, torch.zeros_like(n), torch.zeros_like(n)
    key = s["seed"] & 0xFFFFFFFF, s["seed"] >> 32
    for r in range(10):
        x = _round(x, ((key[0] + r * 0x9E3779B9) & 0xFFFFFFFF, (key[1] + r * 0xBB67AE85) & 0xFFFFFFFF))
    words = torch.stack(x, dim=1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=2).view(rows, wide * 8)[:, :cols]
    return torch.where(halves >= at, 65536.0 / (65536 - at) if at < 65536 else 0.0, 0.0)


def _times(x, keep):
    """x where it is kept, scaled; zero, whatever x is, where it is not."""
    return x if isinstance(keep, float) else torch.where(keep > 0, x * keep, 0.0)


def _plain_norm(s):
    c, dt = s["case"], DTYPE[s["case"]["dtype"]]
    keep = _keep(s, c["rows"], c["cols"])
    h = s["residual"].float() + _times(s["x"].float(), keep)
    y = s["w"] * (h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS))
    out = {"h": h.to(dt)}
    if c["out"] == "f8":
        wide = c["block"] or c["cols"]
        pad = torch.nn.functional.pad(y, (0, -c["cols"] % wide)).view(c["rows"], -1, wide)
        scale = pad.abs().amax(2) / 448.0
        scale = torch.where(scale > 0, scale, 1.0)
        y = (pad / scale[:, :, None]).view(c["rows"], -1)[:, : c["cols"]]
        out["y"], out["scale"] = y.to(torch.float8_e4m3fn), scale
        return out
    out["y"] = y.to(dt)
    if c["do"] == "train":
        h = out["h"].float()
        r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        dy = s["dy"].float()
        a = dy * s["w"]
        dr = s["dh"].float() + r * (a - h * (r * r * (a * h).mean(1, keepdim=True)))
        out["dresidual"], out["dw"] = dr.to(dt), (dy * (h * r)).sum(0)
        if round(65536 * c["p"]):
            out["dx"] = _times(dr, keep).to(dt)
    return out


def _plain_drop(s):
    c, dt = s["case"], DTYPE[s["case"]["dtype"]]
    keep = _keep(s, c["rows"], c["cols"])
    y = _times(s["x"].float(), keep)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dt), "dx": _times(s["dy"].float(), keep).to(dt)}


# ---- this package's calls -----------------------------------------------------


def _own_attn(s):
    import paper_1806_01117_amd as amb
    c, out = s["case"], {}
    args = s["q"], s["k"], s["v"], s["log_decay"]
    if c["do"] == "step":
        return {"o": amb.decay_attention_step(*args, s["s0"], lengths=s["lengths"], scale=s["scale"]), "sn": s["s0"]}
    if c["do"] in ("fwd", "train"):
        out.update(amb.decay_attention(*args, s0=s["s0"], lengths=s["lengths"], scale=s["scale"]))
    if c["do"] in ("bwd", "train"):
        out.update(amb.decay_attention_backward(*args, s["do"], s0=s["s0"], dsn=s["dsn"], lengths=s["lengths"],
                                                scale=s["scale"]))
    return out


def _own_norm(s):
    import paper_1806_01117_amd as amb
    c = s["case"]
    drop = dict(p=c["p"], seed=s["seed"], offset=s["offset"])
    out = amb.add_norm(s["x"], s["w"], residual=s["residual"], eps=EPS, out_dtype="f8" if c["out"] == "f8" else None,
                       scale_block=c["block"], **drop)
    if c["do"] == "train":
        out.update(amb.add_norm_backward(s["dy"], out["h"], s["w"], dh=s["dh"], eps=EPS, **drop))
    return out


def _own_drop(s):
    import paper_1806_01117_amd as amb
    drop = dict(p=s["case"]["p"], seed=s["seed"], offset=s["offset"])
    return {"y": amb.dropout(s["x"], residual=s["residual"], **drop), "dx": amb.dropout(s["dy"], **drop)}


def run(state):
    forms = (_own_attn, _own_norm, _own_drop) if own else (_plain_attn, _plain_norm, _plain_drop)
    return forms[("attn", "norm", "drop").index(state["case"]["op"])](state)


# ---- the definitions in 64 bits ------------------------------------------------


def _exact_attn(s):
    """Token by token."""
    c = s["case"]
    B, T, H, G, dk, dv = (c[k] for k in ("batch", "steps", "heads", "group", "dk", "dv"))
    lam = torch.exp(s["log_decay"].double()).view(1, H, 1, 1)
    row = lambda x, t, d: x[:, t].double().view(B, H, -1, d)  # noqa: E731
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(T, device="cuda")[:, None] < s["lengths"]).view(T, B, 1, 1, 1)
    pick = lambda t, a, b: a if live is None else torch.where(live[t], a, b)  # noqa: E731
    zero = torch.zeros(B, H, dk, dv, device="cuda", dtype=torch.float64)
    nothing = torch.zeros((), device="cuda", dtype=torch.float64)
    out = {}
    S = zero if s["s0"] is None else s["s0"].double()
    if c["do"] != "bwd":
        o = torch.empty(B, T, H * G, dv, device="cuda", dtype=torch.float64)
    if c["do"] in ("bwd", "train"):
        dq = torch.empty(B, T, H * G, dk, device="cuda", dtype=torch.float64)
        dk_ = torch.empty(B, T, H, dk, device="cuda", dtype=torch.float64)
        dv_ = torch.empty(B, T, H, dv, device="cuda", dtype=torch.float64)
    for t in range(T):
        S = pick(t, lam * S + row(s["k"], t, dk).transpose(-1, -2) * row(s["v"], t, dv), S)
        if c["do"] != "bwd":
            o[:, t] = pick(t, s["scale"] * torch.matmul(row(s["q"], t, dk), S), nothing).reshape(B, H * G, dv)
        if c["do"] in ("bwd", "train"):
            dq[:, t] = pick(t, s["scale"] * torch.matmul(row(s["do"], t, dv), S.transpose(-1, -2)), nothing).reshape(B, H * G, dk)
    if c["do"] != "bwd":
        out["o"], out["sn"] = o, S
    if c["do"] in ("bwd", "train"):
        D = zero if s["dsn"] is None else s["dsn"].double()
        for t in reversed(range(T)):
            add = s["scale"] * torch.matmul(row(s["q"], t, dk).transpose(-1, -2), row(s["do"], t, dv))
            A = D + add  # the gradient of S_t
            dk_[:, t] = pick(t, torch.matmul(row(s["v"], t, dv), A.transpose(-1, -2)), nothing)[:, :, 0]
            dv_[:, t] = pick(t, torch.matmul(row(s["k"], t, dk), A), nothing)[:, :, 0]
            D = pick(t, lam * A, D)
        out["dq"], out["dk"], out["dv"] = dq, dk_, dv_
        if s["s0"] is not None:
            out["ds0"] = D
    return out


def _exact_keep(s, rows, cols):
    """Philox by 64-bit products that wrap, and which elements it keeps."""
    t = round(65536 * s["case"]["p"])
    wide, m32 = (cols + 7) // 8, 0xFFFFFFFF
    c = torch.arange(rows, device="cuda")[:, None] * wide + torch.arange(wide, device="cuda") + s["offset"]
    w = [c & m32, (c >> 32) & m32, c * 0, c * 0]
    k0, k1 = s["seed"] & m32, (s["seed"] >> 32) & m32
    for _ in range(10):
        lo = [w[0] * 0xD2511F53, w[2] * 0xCD9E8D57]
        # the products wrap modulo 2^64, which changes none of their 64 bits
        hi = [(x >> 32) & m32 for x in lo]
        w = [hi[1] ^ w[1] ^ k0, lo[1] & m32, hi[0] ^ w[3] ^ k1, lo[0] & m32]
        k0, k1 = (k0 + 0x9E3779B9) & m32, (k1 + 0xBB67AE85) & m32
    bits = torch.stack([w[j // 2] >> 16 * (j % 2) & 0xFFFF for j in range(8)], dim=2)
    kept = bits.reshape(rows, wide * 8)[:, :cols] >= t
    return kept, 65536.0 / (65536 - t) if t < 65536 else 0.0


def _exact_norm(s):
    c = s["case"]
    kept, up = _exact_keep(s, c["rows"], c["cols"])
    x, w = s["x"].double(), s["w"].double()
    h = s["residual"].double() + torch.where(kept, x * up, x * 0)
    y = w * h / torch.sqrt((h * h).sum(1, keepdim=True) / c["cols"] + EPS)
    out = {"h": h, "y": y}
    if c["out"] == "f8":
        wide = c["block"] or c["cols"]
        scale = torch.stack([a.abs().amax(1) for a in y.split(wide, dim=1)], dim=1) / 448
        out["scale"] = scale
        out["y"] = y / scale.repeat_interleave(wide, dim=1)[:, : c["cols"]]  # before its rounding to 8 bits
        return out
    if c["do"] == "train":
        h = h.to(DTYPE[c["dtype"]]).double()  # the backward call's input is the stored h
        r = 1 / torch.sqrt((h * h).sum(1, keepdim=True) / c["cols"] + EPS)
        a = s["dy"].double() * w
        dr = s["dh"].double() + r * a - h * r ** 3 * (a * h).sum(1, keepdim=True) / c["cols"]
        out["dresidual"], out["dw"] = dr, (s["dy"].double() * h * r).sum(0)
        if round(65536 * c["p"]):
            out["dx"] = torch.where(kept, dr * up, dr * 0)
    return out


def _exact_drop(s):
    kept, up = _exact_keep(s, s["case"]["rows"], s["case"]["cols"])
    x, dy = s["x"].double(), s["dy"].double()
    y = torch.where(kept, x * up, x * 0)
    return {"y": y if s["residual"] is None else y + s["residual"].double(), "dx": torch.where(kept, dy * up, dy * 0)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "norm": _exact_norm, "drop": _exact_drop}[case["op"]](s)
