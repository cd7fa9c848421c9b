"""The operators of a residual block against their float64 definitions.

Bars, from what is rounded where (u = 2^-24 for fp32, 2^-9 for bf16, both the
largest relative error of one rounding):

* fp32 results: sums of a few hundred products and decays lambda^n taken with a
  relative error of |n log lambda| u; 100 u = 6e-6 of a tensor's 2-norm, and of
  its rms (or the entry itself, if that is larger) five standard deviations
  for an entry: 3e-5.
* bf16 results: the result's own rounding and, in attention, those of the
  weighted products and of the states on their way into the matrix cores, each
  at most u and u / sqrt(3) rms: 2 u = 4e-3 of the 2-norm, 10 u = 2e-2 for an
  entry.
* 8 bits: half a unit of e4m3's three-bit mantissa is 2^-4 of the value, half
  its smallest step 2^-10 of the scale.
"""
import numpy as np
import pytest

from oracle import ops as O

pytestmark = pytest.mark.gpu

BARS = {"f32": (6e-6, 3e-5), "bf16": (4e-3, 2e-2)}


@pytest.fixture(scope="module")
def amb():
    import torch  # noqa: F401  (its HIP runtime is the one that the library then shares)

    import paper_1806_01117_amd as amb
    amb.load()
    return amb


def _torch():
    import torch
    return torch


def _dt(dtype):
    torch = _torch()
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _np(t):
    return t.detach().cpu().double().numpy()


def _near(got, want, dtype, what):
    got = _np(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    if not want.size:
        return
    rms = np.sqrt((want * want).mean())
    if rms == 0.0:
        assert (got == 0.0).all(), what
        return
    d = np.abs(got - want)
    norm, entry = BARS[dtype]
    assert np.sqrt((d * d).mean()) <= norm * rms, (what, np.sqrt((d * d).mean()) / rms)
    worst = (d / np.maximum(np.abs(want), rms)).max()
    assert worst <= entry, (what, worst)


DECAYS = [-0.02, 0.0, -0.0005, -1.5, -0.1, -0.007]


class Attn:
    """Seeded inputs of one attention problem, laid out as asked."""

    def __init__(self, dtype, B, T, H, G, dk, dv, layout="bthd", lengths=None, state=True, poison=True, seed=0,
                 decays=None):
        torch = _torch()
        print("[case]", dtype, B, T, H, G, dk, dv, layout, lengths, flush=True)
        self.dtype, self.shape, self.lengths = dtype, (B, T, H, G, dk, dv), lengths
        gen = torch.Generator().manual_seed(seed)
        self.scale = dk ** -0.5
        dt = _dt(dtype)
        dims = dict(q=(H * G, dk), k=(H, dk), v=(H, dv), do=(H * G, dv))
        dense = {n: torch.randn(B, T, h, d, generator=gen).to(dt) for n, (h, d) in dims.items()}
        if layout == "broadcast":  # one row's k and v for the whole batch
            for n in "kv":
                dense[n] = dense[n][:1].expand(B, T, *dims[n])
        self.g = (DECAYS if decays is None else decays)[:H]
        self.g = (self.g * H)[:H]
        self.np = {n: t.double().numpy() for n, t in dense.items()}
        if lengths is not None and poison:  # nothing past a row's length is used
            for n, t in dense.items():
                for b in range(B):
                    t[b, max(0, lengths[b]):] = float("nan")
        self.dev = {n: self._lay(t, layout, n) for n, t in dense.items()}
        f32 = dict(dtype=torch.float32)
        self.s0 = torch.randn(B, H, dk, dv, generator=gen, **f32) if state else None
        self.dsn = torch.randn(B, H, dk, dv, generator=gen, **f32) if state else None
        cu = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.args = [self.dev[n] for n in "qkv"] + [torch.tensor(self.g, **f32).cuda()]
        self.more = dict(scale=self.scale, lengths=None if lengths is None else
                         torch.tensor(lengths, dtype=torch.int32).cuda())
        self.s0d, self.dsnd = cu(self.s0), cu(self.dsn)

    def _lay(self, t, layout, n):
        torch = _torch()
        B, T, h, d = t.shape
        if layout == "tbhd":
            return t.transpose(0, 1).contiguous().cuda().transpose(0, 1)
        if layout == "bhtd":
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        if layout == "odd":  # rows that no vector is aligned to
            buf = torch.zeros(B * T * h * (d + 3) + 1, dtype=t.dtype, device="cuda")
            v = buf[1:].view(B, T, h, d + 3)[..., :d]
            v.copy_(t)
            return v
        if layout == "broadcast" and n in "kv":
            return t[:1].cuda().expand(B, T, h, d)
        return t.contiguous().cuda()

    def forward(self):
        i = self.np
        return O.attention(i["q"], i["k"], i["v"], self.g, None if self.s0 is None else self.s0.double().numpy(),
                           self.lengths, self.scale)

    def backward(self):
        i = self.np
        f = lambda t: None if t is None else t.double().numpy()  # noqa: E731
        return O.attention_backward(i["q"], i["k"], i["v"], self.g, i["do"], f(self.s0), f(self.dsn), self.lengths,
                                    self.scale)


LENGTHS = [0, 1, 2, 15, 17, 63, 64, 65, 127, 129, 300]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", LENGTHS)
def test_attention_lengths(amb, dtype, T):
    c = Attn(dtype, 2, T, 2, 2, 64, 64)
    r = amb.decay_attention(*c.args, s0=c.s0d, **c.more)
    o, sn = c.forward()
    _near(r["o"], o, dtype, "o")
    _near(r["sn"], sn, "f32", "sn")
    g = amb.decay_attention_backward(*c.args, c.dev["do"], s0=c.s0d, dsn=c.dsnd, **c.more)
    for name, want in zip(("dq", "dk", "dv", "ds0"), c.backward()):
        _near(g[name], want, "f32" if name == "ds0" else dtype, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,G,dk,dv", [(1, 1, 16, 16), (3, 1, 16, 128), (2, 3, 128, 16), (5, 2, 80, 112), (1, 4, 48, 64),
                                       (2, 1, 128, 128), (6, 1, 32, 96)])
def test_attention_heads(amb, dtype, H, G, dk, dv):
    c = Attn(dtype, 2, 150, H, G, dk, dv, lengths=[150, 77])
    r = amb.decay_attention(*c.args, s0=c.s0d, **c.more)
    o, sn = c.forward()
    _near(r["o"], o, dtype, "o")
    _near(r["sn"], sn, "f32", "sn")
    g = amb.decay_attention_backward(*c.args, c.dev["do"], s0=c.s0d, dsn=c.dsnd, **c.more)
    for name, want in zip(("dq", "dk", "dv", "ds0"), c.backward()):
        _near(g[name], want, "f32" if name == "ds0" else dtype, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["tbhd", "bhtd", "odd", "broadcast"])
def test_attention_layouts(amb, dtype, layout):
    c = Attn(dtype, 3, 100, 2, 2, 48, 64, layout=layout)
    r = amb.decay_attention(*c.args, s0=c.s0d, **c.more)
    o, sn = c.forward()
    _near(r["o"], o, dtype, "o")
    _near(r["sn"], sn, "f32", "sn")
    g = amb.decay_attention_backward(*c.args, c.dev["do"], s0=c.s0d, dsn=c.dsnd, **c.more)
    for name, want in zip(("dq", "dk", "dv", "ds0"), c.backward()):
        _near(g[name], want, "f32" if name == "ds0" else dtype, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_ragged_rows(amb, dtype):
    # rows of every kind in one batch; NaNs lie past each row's length, and
    # lengths outside the range count as its ends
    T = 200
    c = Attn(dtype, 8, T, 2, 2, 64, 32, lengths=[T, 0, 1, 64, 65, 199, -7, T + 9])
    r = amb.decay_attention(*c.args, s0=c.s0d, **c.more)
    o, sn = c.forward()
    _near(r["o"], o, dtype, "o")
    _near(r["sn"], sn, "f32", "sn")
    assert _torch().equal(r["sn"][1].cpu(), c.s0[1]) and not r["o"][1].any()  # an empty row
    g = amb.decay_attention_backward(*c.args, c.dev["do"], s0=c.s0d, dsn=c.dsnd, **c.more)
    for name, want in zip(("dq", "dk", "dv", "ds0"), c.backward()):
        _near(g[name], want, "f32" if name == "ds0" else dtype, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H", [(1, 1000, 1), (1, 2300, 3), (40, 70, 2)])
def test_attention_few_and_many_rows(amb, dtype, B, T, H):
    # few rows over a long sequence, and many over a short one; no states given
    c = Attn(dtype, B, T, H, 1, 32, 48, state=False)
    r = amb.decay_attention(*c.args, **c.more)
    o, sn = c.forward()
    _near(r["o"], o, dtype, "o")
    _near(r["sn"], sn, "f32", "sn")
    g = amb.decay_attention_backward(*c.args, c.dev["do"], **c.more)
    assert g["ds0"] is None
    for name, want in zip(("dq", "dk", "dv"), c.backward()):
        _near(g[name], want, dtype, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,G,dk,dv", [(2, 150, 2, 2, 64, 64), (1, 1000, 1, 1, 128, 128), (1, 90, 3, 1, 32, 112)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_attention_keeps_infinities_to_their_side(amb, dtype, B, T, H, G, dk, dv, value):
    """A value at token j is in the results that depend on it, and in no others: those keep every bit."""
    torch = _torch()
    j = 69
    clean = Attn(dtype, B, T, H, G, dk, dv)
    want = dict(amb.decay_attention(*clean.args, s0=clean.s0d, **clean.more))
    want.update(amb.decay_attention_backward(*clean.args, clean.dev["do"], s0=clean.s0d, dsn=clean.dsnd, **clean.more))
    # by operand: the results' tokens that see it, of o, dq, dk and dv
    before, own, after, none = slice(0, j + 1), slice(j, j + 1), slice(j, T), slice(0, 0)
    seen = dict(q=dict(o=own, dq=none, dk=before, dv=before), k=dict(o=after, dq=after, dk=none, dv=own),
                v=dict(o=after, dq=after, dk=own, dv=none), do=dict(o=none, dq=own, dk=before, dv=before))
    for name, sides in seen.items():
        c = Attn(dtype, B, T, H, G, dk, dv)
        c.dev[name][-1, j, 0, 5] = value
        got = dict(amb.decay_attention(*c.args, s0=c.s0d, **c.more))
        got.update(amb.decay_attention_backward(*c.args, c.dev["do"], s0=c.s0d, dsn=c.dsnd, **c.more))
        for r, side in sides.items():
            free = torch.ones(got[r].shape[1], dtype=torch.bool)
            free[side] = False
            heads = range(G) if r in ("o", "dq") and name in "kv" else [0]
            for h in range(got[r].shape[2]):
                if h not in heads:
                    assert torch.equal(got[r][-1, :, h], want[r][-1, :, h]), (name, r, h)
                    continue
                assert torch.equal(got[r][-1, free, h], want[r][-1, free, h]), (name, r, h)
                hit = ~torch.isfinite(got[r][-1, ~free, h])
                assert hit.any(-1).all(), (name, r, h)
            assert torch.equal(got[r][:-1], want[r][:-1]), (name, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_decays_at_their_ends(amb, dtype):
    # no memory at all (lambda = 0), next to none, and without end
    c = Attn(dtype, 1, 140, 4, 1, 32, 32, decays=[-float("inf"), -80.0, 0.0, -1e-6])
    r = amb.decay_attention(*c.args, s0=c.s0d, **c.more)
    o, sn = c.forward()
    for h in range(4):
        _near(r["o"][:, :, h], o[:, :, h], dtype, ("o", h))
        _near(r["sn"][:, h], sn[:, h], "f32", ("sn", h))
    g = amb.decay_attention_backward(*c.args, c.dev["do"], s0=c.s0d, dsn=c.dsnd, **c.more)
    for name, want in zip(("dq", "dk", "dv"), c.backward()):
        for h in range(4):
            _near(g[name][:, :, h], want[:, :, h], dtype, (name, h))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,G,dk,dv", [(1, 1, 1, 16, 16), (5, 3, 2, 64, 64), (3, 2, 4, 128, 112), (70, 4, 1, 48, 128)])
def test_attention_step_is_the_sequence(amb, dtype, B, H, G, dk, dv):
    # token by token in place: the outputs and the state of the whole sequence
    torch = _torch()
    T, lengths = 4, [0 if b % 5 == 3 else 4 for b in range(B)]
    c = Attn(dtype, B, T, H, G, dk, dv, lengths=lengths)
    s = c.s0d.clone()
    q, k, v, g = c.args
    live = c.more["lengths"].clamp(max=1)
    o = [amb.decay_attention_step(q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1], g, s, lengths=live, scale=c.scale)
         for t in range(T)]
    want, sn = c.forward()
    _near(torch.cat(o, 1), want, dtype, "o")
    _near(s, sn, "f32", "s")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_step_leaves_a_finished_row(amb, dtype):
    # a row without a token keeps its state, whatever it holds, in place and in another buffer
    torch = _torch()
    c = Attn(dtype, 2, 1, 3, 2, 32, 48, lengths=[0, 1])
    s = c.s0d.clone()
    s[0, 1, 4, 5], s[0, 2, 7, 1], s[0, 0, 0, 0] = float("inf"), float("nan"), -0.0
    keep = s[0].clone()
    r = amb.decay_attention(*c.args, s0=s, **c.more)
    o = amb.decay_attention_step(*c.args, s, lengths=c.more["lengths"], scale=c.scale)
    for t in (r["sn"][0], s[0]):
        assert torch.equal(t.view(torch.int32), keep.view(torch.int32))
    assert not o[0].any() and not r["o"][0].any() and torch.equal(s[1], r["sn"][1])


def test_attention_offsets_past_32_bits(amb):
    # tokens 2^26 elements apart: the offsets pass 2^32
    torch = _torch()
    T, H, d = 70, 1, 32
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    c = Attn("bf16", 1, T, H, 1, d, d)
    far = torch.empty(T, 1 << 26, dtype=torch.bfloat16, device="cuda")
    at = {}
    for i, n in enumerate(("q", "k", "v", "do")):
        at[n] = far.as_strided((1, T, 1, d), (T << 26, 1 << 26, d, 1), 64 * i)
        at[n].copy_(c.dev[n])
    out = {n: far.as_strided((1, T, 1, d), (T << 26, 1 << 26, d, 1), 64 * (i + 4))
           for i, n in enumerate(("o", "dq", "dk", "dv"))}
    r = amb.decay_attention(at["q"], at["k"], at["v"], c.args[3], s0=c.s0d, out={"o": out["o"]}, **c.more)
    o, sn = c.forward()
    _near(r["o"], o, "bf16", "o")
    _near(r["sn"], sn, "f32", "sn")
    g = amb.decay_attention_backward(at["q"], at["k"], at["v"], c.args[3], at["do"], s0=c.s0d, dsn=c.dsnd,
                                     out={n: out[n] for n in ("dq", "dk", "dv")}, **c.more)
    for name, want in zip(("dq", "dk", "dv", "ds0"), c.backward()):
        _near(g[name], want, "f32" if name == "ds0" else "bf16", name)
    del far, at, out, r, g
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_in_two_parts_and_on_another_stream(amb, dtype):
    # a sequence in two calls carries its state and its gradient; on a stream
    # of its own; the same inputs give the same bits
    torch = _torch()
    c = Attn(dtype, 2, 181, 2, 2, 64, 80)
    q, k, v, g = c.args
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cut = 83
        a = amb.decay_attention(q[:, :cut], k[:, :cut], v[:, :cut], g, s0=c.s0d, **c.more)
        b = amb.decay_attention(q[:, cut:], k[:, cut:], v[:, cut:], g, s0=a["sn"], **c.more)
        do = c.dev["do"]
        gb = amb.decay_attention_backward(q[:, cut:], k[:, cut:], v[:, cut:], g, do[:, cut:], s0=a["sn"], dsn=c.dsnd, **c.more)
        ga = amb.decay_attention_backward(q[:, :cut], k[:, :cut], v[:, :cut], g, do[:, :cut], s0=c.s0d, dsn=gb["ds0"], **c.more)
        again = amb.decay_attention_backward(q[:, :cut], k[:, :cut], v[:, :cut], g, do[:, :cut], s0=c.s0d, dsn=gb["ds0"], **c.more)
    side.synchronize()
    o, sn = c.forward()
    _near(torch.cat([a["o"], b["o"]], 1), o, dtype, "o")
    _near(b["sn"], sn, "f32", "sn")
    for name, want in zip(("dq", "dk", "dv"), c.backward()):
        _near(torch.cat([ga[name], gb[name]], 1), want, dtype, name)
    _near(ga["ds0"], c.backward()[3], "f32", "ds0")
    assert all(torch.equal(ga[n], again[n]) for n in ga)


def test_attention_in_a_graph(amb):
    # captured and replayed on new values, with eager work between the replays
    torch = _torch()
    c, d = (Attn("bf16", 2, 333, 2, 2, 64, 64, seed=s) for s in (0, 1))
    ins = [t.clone() for t in c.args[:3]] + [c.dev["do"].clone()]
    f = lambda: (amb.decay_attention(*ins[:3], c.args[3], s0=c.s0d, **c.more),  # noqa: E731
                 amb.decay_attention_backward(*ins[:3], c.args[3], ins[3], s0=c.s0d, dsn=c.dsnd, **c.more))
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = f()
    for x in (c, d, c):
        for t, n in zip(ins, ("q", "k", "v", "do")):
            t.copy_(x.dev[n])
        graph.replay()
        torch.cuda.synchronize()
        want = f()
        for a, b in zip(got, want):
            for n in a:
                assert torch.equal(a[n], b[n]), n


def test_attention_refusals(amb):
    torch = _torch()
    c = Attn("bf16", 2, 8, 2, 2, 32, 32)
    q, k, v, g = c.args
    for bad in ([q[0], k, v, g], [q, k[:, :4], v, g], [q, k.float(), v, g], [q[:, :, :3], k, v, g], [q, k, v, g.double()],
                [q, k, v, g[:1]], [q.half(), k.half(), v.half(), g], [q.transpose(2, 3), k, v, g], [q.cpu(), k.cpu(), v.cpu(), g.cpu()]):
        with pytest.raises(ValueError):
            amb.decay_attention(*bad)
    with pytest.raises(ValueError):
        amb.decay_attention(*c.args, lengths=torch.tensor([1, 2], device="cuda"))  # int64
    with pytest.raises(ValueError):
        amb.decay_attention(*c.args, s0=c.s0d.transpose(2, 3))
    with pytest.raises(ValueError):
        amb.decay_attention_step(q[:, :1], k[:, :1], v[:, :1], g, None)
    with pytest.raises(amb.AmbpttError) as e:
        amb.decay_attention(q[..., :24], k[..., :24], v, g)
    assert e.value.status == -4
    with pytest.raises(amb.AmbpttError) as e:  # an output whose rows lie on one another
        amb.decay_attention(*c.args, out={"o": torch.empty(1, 8, 4, 32, dtype=torch.bfloat16, device="cuda").expand(2, 8, 4, 32)})
    assert e.value.status == -1


# ---- dropout --------------------------------------------------------------------


def _rows_of(dtype, rows, cols, lay, seed):
    torch = _torch()
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)).to(_dt(dtype))
    if lay == "wide":  # rows apart from each other, and off every vector's alignment
        buf = torch.zeros(rows * (cols + 5) + 3, dtype=x.dtype, device="cuda")
        v = buf[3:].view(rows, cols + 5)[:, :cols]
        v.copy_(x)
        return x.double().numpy(), v
    return x.double().numpy(), x.cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,lay", [(1, 1, "dense"), (3, 7, "dense"), (5, 8, "dense"), (9, 64, "dense"), (4, 129, "dense"),
                                           (33, 40, "wide"), (2, 2100, "dense"), (300, 16, "dense")])
def test_dropout(amb, dtype, rows, cols, lay):
    torch = _torch()
    print("[case]", dtype, rows, cols, lay, flush=True)
    seed, offset, p = 0xFEDCBA9876543210, (1 << 32) - 2, 0.3  # the counter passes 32 bits within the call
    x, xd = _rows_of(dtype, rows, cols, lay, 1)
    r, rd = _rows_of(dtype, rows, cols, lay, 2)
    f = O.dropout_factors(rows, cols, p, seed, offset)
    y = amb.dropout(xd, p, seed, offset)
    assert ((_np(y) != 0) == ((f > 0) & (x != 0))).all()  # the mask is the definition's, bit for bit
    _near(y, O.dropped(x, f), dtype, "y")
    _near(amb.dropout(xd, p, seed, offset, residual=rd), r + O.dropped(x, f), dtype, "y + r")
    z = xd.clone()
    assert amb.dropout(z, p, seed, offset, out=z) is z and torch.equal(z, y)
    assert amb.dropout_counters(xd) == rows * -(-cols // 8)


def test_dropout_of_parts_is_dropout_of_the_whole(amb):
    torch = _torch()
    x = torch.randn(40, 24, device="cuda")
    whole = amb.dropout(x, 0.5, 7, 100)
    first = amb.dropout(x[:15], 0.5, 7, 100)
    second = amb.dropout(x[15:], 0.5, 7, 100 + amb.dropout_counters(x[:15]))
    assert torch.equal(torch.cat([first, second]), whole)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_ends_and_infinities(amb, dtype):
    torch = _torch()
    x = torch.full((4, 40), float("inf"), dtype=_dt(dtype), device="cuda")
    x[1] = float("nan")
    f = O.dropout_factors(4, 40, 0.5, 3, 4)
    y = _np(amb.dropout(x, 0.5, 3, 4))
    assert (y[f == 0] == 0).all() and (y[(0, 2, 3), :][f[(0, 2, 3), :] > 0] == np.inf).all() and np.isnan(y[1][f[1] > 0]).all()
    assert not amb.dropout(x, 1.0, 3, 4).any()
    assert torch.equal(amb.dropout(x[2:], 0.0, 3, 4), x[2:])
    r = torch.ones(4, 40, dtype=_dt(dtype), device="cuda")
    assert torch.equal(amb.dropout(x, 1.0, 3, 4, residual=r), r)
    assert amb.dropout(x[:0], 0.5, 3, 4).shape == (0, 40)


def test_dropout_refusals(amb):
    torch = _torch()
    x = torch.randn(4, 6, 8, device="cuda")
    for bad in (lambda: amb.dropout(x.half(), 0.5, 1), lambda: amb.dropout(x.cpu(), 0.5, 1), lambda: amb.dropout(x.transpose(1, 2), 0.5, 1),
                lambda: amb.dropout(x, 0.5, 1, residual=x[0]), lambda: amb.dropout(x[:, :4], 0.5, 1, residual=x[:, :4].bfloat16())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):  # rows without a common stride
        amb.dropout(x[:, :4], 0.5, 1)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(amb.AmbpttError):
            amb.dropout(x, p, 1)


# ---- norm -------------------------------------------------------------------------


SIZES = [(1, 1), (3, 7), (5, 8), (4, 127), (7, 128), (2, 129), (130, 64), (3, 1001), (9, 2048), (2, 4096), (3, 5000), (2, 8192),
         (1, 16384), (2, 20001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_norm(amb, dtype, rows, cols, p):
    torch = _torch()
    print("[case]", dtype, rows, cols, p, flush=True)
    eps, seed, offset = 1e-5, 11, 1 << 35
    x, xd = _rows_of(dtype, rows, cols, "dense", 1)
    r, rd = _rows_of(dtype, rows, cols, "dense", 2)
    dy, dyd = _rows_of(dtype, rows, cols, "dense", 3)
    dh, dhd = _rows_of(dtype, rows, cols, "dense", 4)
    w = 1 + 0.3 * np.random.default_rng(5).normal(size=cols)
    wd = torch.tensor(w, dtype=torch.float32).cuda()
    w = _np(wd)
    f = O.dropout_factors(rows, cols, p, seed, offset) if p else np.ones((rows, cols))
    drop = dict(p=p, seed=seed, offset=offset)
    h = r + O.dropped(x, f)
    got = amb.add_norm(xd, wd, residual=rd, eps=eps, **drop)
    _near(got["h"], h, dtype, "h")
    _near(got["y"], O.norm(h, w, eps), dtype, "y")
    hs = _np(got["h"])
    dr, dw = O.norm_backward(dy, hs, w, dh, eps)
    g = amb.add_norm_backward(dyd, got["h"], wd, dh=dhd, eps=eps, **drop)
    if cols > 1:  # with one column the norm's gradient is a difference of equals
        _near(g["dresidual"], dr, dtype, "dr")
        _near(g["dw"], dw, "f32", "dw")
        if p:
            _near(g["dx"], O.dropped(dr, f), dtype, "dx")
    assert ("dx" in g) == (p > 0)
    g = amb.add_norm_backward(dyd, got["h"], wd, eps=eps)
    if cols > 1:
        _near(g["dresidual"], O.norm_backward(dy, hs, w, 0 * dh, eps)[0], dtype, "dr without dh")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 100), (2, 128), (5, 300), (4, 1024), (3, 2048), (2, 4100), (2, 9000)])
@pytest.mark.parametrize("block", [0, 128])
def test_norm_in_8_bits(amb, dtype, rows, cols, block):
    torch = _torch()
    print("[case]", dtype, rows, cols, block, flush=True)
    x, xd = _rows_of(dtype, rows, cols, "dense", 1)
    w = 1 + 0.3 * np.random.default_rng(5).normal(size=cols)
    wd = torch.tensor(w, dtype=torch.float32).cuda()
    got = amb.add_norm(xd, wd, eps=1e-5, out_dtype="f8", scale_block=block)
    assert torch.equal(got["h"], xd)
    y = O.norm(x, _np(wd), 1e-5)
    wide = block or cols
    want = np.stack([np.abs(y[:, i:i + wide]).max(1) for i in range(0, cols, wide)], 1) / 448
    scale = _np(got["scale"])
    assert np.allclose(scale, want, rtol=1e-5)
    s = np.repeat(scale, wide, 1)[:, :cols]
    d = np.abs(_np(got["y"].float()) * s - y)
    assert (d <= 1.001 * np.abs(y) * 2.0 ** -4 + s * 2.0 ** -10).all() and np.abs(_np(got["y"].float())).max() <= 448


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(2, 16), (100, 20), (37, 33), (2000, 61), (70, 65), (41, 128), (33, 200), (40000, 24), (19, 256),
                                       (9, 257), (1500, 512)])
def test_norm_of_narrow_rows(amb, dtype, rows, cols):
    # a part of a wave to a row: full and partial waves and workgroups, with and without 8 bits
    test_norm(amb, dtype, rows, cols, 0.25)
    for block in (0, 128):
        test_norm_in_8_bits(amb, dtype, rows, cols, block)


@pytest.mark.parametrize("block", [0, 128])
def test_norm_in_8_bits_below_the_normal_numbers(amb, block):
    # a scale that lost its bits would take the stored values past 448: it is 2^-126 at least
    torch = _torch()
    x = torch.randn(3, 200, device="cuda")
    for size in (1e-36, 1e-38, 1e-40, 2e-44):
        w = torch.full((200,), size, device="cuda")
        got = amb.add_norm(x, w, out_dtype="f8", scale_block=block)
        y = O.norm(_np(x), _np(w), 1e-6)
        scale = _np(got["scale"])
        assert (scale >= 2.0 ** -126).all()
        s = np.repeat(scale, block or 200, 1)[:, :200]
        d = np.abs(_np(got["y"].float()) * s - y)
        assert (d <= 1.001 * np.abs(y) * 2.0 ** -4 + s * 2.0 ** -10 + 2.0 ** -147).all()


def test_norm_rows_and_views(amb):
    torch = _torch()
    # rows apart from each other and off every alignment; h in place of the
    # residual; a row of zeros, one that holds an infinity, one a NaN
    rows, cols = 6, 300
    for dtype in ("f32", "bf16"):
        x, xd = _rows_of(dtype, rows, cols, "wide", 1)
        r, rd = _rows_of(dtype, rows, cols, "wide", 2)
        w = torch.ones(cols, device="cuda")
        out = {"h": rd}
        want = r + x
        got = amb.add_norm(xd, w, residual=rd, out=out)
        assert got["h"] is rd
        _near(rd, want, dtype, "h")
        _near(got["y"], O.norm(want, 1.0, 1e-6), dtype, "y")
        z = torch.randn(4, cols, device="cuda").to(_dt(dtype))
        z[0] = 0.0
        z[1, 3], z[2, 5] = float("inf"), float("nan")
        for block in (0, 128):
            q = amb.add_norm(z, w, out_dtype="f8", scale_block=block)
            assert not q["y"][0].float().any() and (q["scale"][0] == 1).all()
            assert torch.isfinite(q["y"][3].float()).all()
        y = amb.add_norm(z, w)["y"]
        assert not y[0].any() and not torch.isfinite(y[1]).all() and torch.isnan(y[2]).all() and torch.isfinite(y[3]).all()
        assert amb.add_norm(z[:0], w)["y"].shape == (0, cols)
        g = amb.add_norm_backward(z[:0], z[:0], w)
        assert not g["dw"].any()
        a = torch.randn(2, 3, cols, device="cuda").to(_dt(dtype))
        assert torch.equal(amb.add_norm(a, w)["y"].view(6, cols), amb.add_norm(a.view(6, cols), w)["y"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_weight_gradient_over_many_rows(amb, dtype):
    torch = _torch()
    for rows, cols in ((5000, 72), (1300, 520), (700, 2056)):
        h, hd = _rows_of(dtype, rows, cols, "dense", 1)
        dy, dyd = _rows_of(dtype, rows, cols, "dense", 2)
        w = torch.ones(cols, device="cuda")
        g = amb.add_norm_backward(dyd, hd, w)
        dr, dw = O.norm_backward(dy, h, 1.0, 0.0, 1e-6)
        _near(g["dw"], dw, "f32", "dw")
        _near(g["dresidual"], dr, dtype, "dr")
        again = amb.add_norm_backward(dyd, hd, w)
        assert all(torch.equal(g[n], again[n]) for n in g)


def test_norm_in_a_graph(amb):
    torch = _torch()
    x = torch.randn(50, 640, device="cuda", dtype=torch.bfloat16)
    r, dy, w = torch.randn_like(x), torch.randn_like(x), torch.rand(640, device="cuda")
    drop = dict(p=0.2, seed=5, offset=6)

    def f():
        a = amb.add_norm(x, w, residual=r, **drop)
        return {**a, **amb.add_norm_backward(dy, a["h"], w, **drop), "f8": amb.add_norm(x, w, out_dtype="f8")["y"],
                "d": amb.dropout(x, **drop)}

    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = f()
    for seed in (1, 2, 3):
        torch.manual_seed(seed)
        for t in (x, r, dy):
            t.copy_(torch.randn_like(t))
        graph.replay()
        torch.cuda.synchronize()
        want = f()
        for n in got:
            assert torch.equal(got[n].view(torch.uint8), want[n].view(torch.uint8)), n


def test_norm_refusals(amb):
    torch = _torch()
    x, w = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for bad in (lambda: amb.add_norm(x, w[:32]), lambda: amb.add_norm(x, w.bfloat16()), lambda: amb.add_norm(x, w, residual=x[:2]),
                lambda: amb.add_norm(x.double(), w), lambda: amb.add_norm(x, w, out_dtype="f16"),
                lambda: amb.add_norm(x.t(), w[:4]), lambda: amb.add_norm_backward(x[:2], x, w),
                lambda: amb.add_norm(x, w, out={"h": x.bfloat16()})):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(scale_block=128), dict(out_dtype="f8", scale_block=64), dict(p=2.0), dict(eps=-1.0)):
        with pytest.raises(amb.AmbpttError):
            amb.add_norm(x, w, **bad)
