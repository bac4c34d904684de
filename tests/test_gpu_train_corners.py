"""Ends of the ranges of the training step's calls on an MI355X."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

gift = pytest.importorskip("paper_2607_07494_amd.gift")
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gift.Context()
    yield c
    torch.cuda.synchronize()
    c.close()


def test_norm_past_float32(ctx):
    """Finite gradients whose norm is past float32's range: out[0] rounds to infinity, out[1] clips (it is below
    float32's normal range, where neighbours are 2^-149 apart)."""
    x = torch.full((2,), 3e38, device=DEV)
    out = torch.empty(2, device=DEV)
    gift.grad_norm(ctx, [x], out, max_norm=1.0)
    torch.cuda.synchronize()
    norm = float(x[0].double()) * math.sqrt(2)
    got = out.double().cpu().tolist()
    assert math.isinf(got[0]) and abs(got[1] - 1 / norm) <= 2.0 ** -150 + 1e-15 / norm


def test_only_empty_tensors(ctx):
    out = torch.full((2,), 5.0, device=DEV)
    empty = [torch.zeros(0, device=DEV), torch.zeros((3, 0), device=DEV)]
    gift.grad_norm(ctx, empty, out, max_norm=1.0)
    torch.cuda.synchronize()
    assert out.tolist() == [0.0, 1.0]
    for moments in ("f32", "e4m3"):
        opt = gift.AdamW(ctx, [torch.zeros(0, device=DEV), torch.zeros((3, 0), device=DEV)], moments=moments)
        opt.step([g.clone() for g in empty], lr=1.0)
        assert opt.steps == 1
        opt.close()


def test_steps_after_set_stream(ctx):
    """A context moved to another stream between two steps: the second runs after the first."""
    s = torch.cuda.Stream()
    p, g = torch.ones(5000, device=DEV), torch.ones(5000, device=DEV)
    a = torch.randn(4096, 4096, device=DEV)
    c = gift.Context()
    opt = gift.AdamW(c, [p])
    torch.cuda.synchronize()
    for _ in range(10):
        a @ a
    opt.step([g], lr=0.25)
    c.set_stream(s.cuda_stream)
    opt.step([g], lr=0.25)           # equal gradients: m / sqrt(v) is 1 after the corrections, twice
    opt.close()
    assert float((p - 0.5).abs().max()) <= 1e-5
    c.close()
