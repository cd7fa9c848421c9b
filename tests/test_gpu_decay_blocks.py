"""The example of residual blocks over a long sequence: its gradients do not
depend on the schedule, agree with differences, and training uses them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decay_blocks", os.path.join(ROOT, "examples", "decay_blocks.py"))
    m = importlib.util.module_from_spec(spec)
    import sys
    sys.modules["decay_blocks"] = m
    spec.loader.exec_module(m)
    return m


def _data(ex, cfg, seed=1):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda: [torch.randn(cfg.batch, cfg.steps, cfg.width, generator=gen, device="cuda").to(cfg.dtype)  # noqa: E731
                    for _ in range(cfg.segments)]
    return make(), make()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_gradients_do_not_depend_on_the_schedule(ex, dtype):
    import torch
    cfg = ex.Config(width=128, heads=4, kv_heads=2, batch=2, segments=7, steps=70, p=0.2, dtype=getattr(torch, dtype))
    blocks, (xs, ts) = ex.Blocks(cfg), _data(ex, cfg)
    want_loss, want, once = ex.gradients(blocks, xs, ts, slots=cfg.segments)
    for slots in (1, 2, 3):
        loss, grads, evaluated = ex.gradients(blocks, xs, ts, slots=slots)
        assert evaluated > once  # segments were evaluated again
        assert torch.equal(loss, want_loss)
        for name in want:
            assert torch.equal(grads[name], want[name]), (slots, name)


def test_gradients_against_differences(ex):
    # the loss along a direction of each parameter in fp32: the difference's own
    # rounding is some 2^-24 of the loss over the step 2e-2, and its curvature
    # stays below the bar's 2 % of the slope
    import torch
    torch.manual_seed(0)
    cfg = ex.Config(width=64, heads=2, kv_heads=1, batch=2, segments=3, steps=40, p=0.2, dtype=torch.float32)
    blocks, (xs, ts) = ex.Blocks(cfg), _data(ex, cfg)
    _, grads, _ = ex.gradients(blocks, xs, ts)
    for name, p in blocks.params.items():
        u = grads[name] / grads[name].norm()
        old, e = p.clone(), 2e-2
        p.copy_(old + e * u)
        up = ex.gradients(blocks, xs, ts)[0].double()
        p.copy_(old - e * u)
        down = ex.gradients(blocks, xs, ts)[0].double()
        p.copy_(old)
        slope, want = float((up - down) / (2 * e)), float(grads[name].double().norm())
        assert abs(slope - want) <= 0.02 * want + 2e-5, (name, slope, want)


def test_tokens_one_by_one_are_the_sequence(ex):
    # generation's steps against one call over the same inputs, without dropout;
    # bf16 activations through two blocks
    import torch
    cfg = ex.Config(width=128, heads=4, kv_heads=2, batch=3, segments=1, steps=9, p=0.0)
    blocks, (xs, _) = ex.Blocks(cfg), _data(ex, cfg)
    made = ex.generate(blocks, xs[0], 5)
    whole = torch.cat([xs[0], made[:, :-1]], 1)
    y, _, _ = blocks.forward(0, whole, blocks.first_state())
    want, got = y[:, -5:].float(), made.float()
    # e4m3 rounds to 2^-4 of a value, bf16 products and states to some 2^-8
    assert ((got - want).norm() / want.norm()) <= 0.05
