"""AdamW on an MI355X where its tensors' memory changes between steps.

The float32 step equals the oracle bit for bit, so it also tells which memory
a step read and wrote.
"""

import numpy as np
import pytest
import torch

from oracle import train

pytestmark = pytest.mark.gpu

gift = pytest.importorskip("paper_2607_07494_amd.gift")
DEV = "cuda"
F = np.float32
LR, B1, B2, EPS = 3e-3, 0.9, 0.95, 1e-8


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gift.Context()
    yield c
    torch.cuda.synchronize()
    c.close()


def test_parameters_copies_and_moments_moved_between_steps(ctx):
    n = 3000
    rng = np.random.default_rng(1)
    p = rng.standard_normal(n).astype(F)
    m, v = np.zeros(n, F), np.zeros(n, F)
    param, copy = torch.from_numpy(p).to(DEV), torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    opt = gift.AdamW(ctx, [param], betas=(B1, B2), eps=EPS, copies=[copy])
    left = []                      # memory that was given up, and what it held

    def step(number):
        nonlocal p, m, v
        g = rng.standard_normal(n).astype(F)
        opt.step([torch.from_numpy(g).to(DEV)], lr=LR)
        torch.cuda.synchronize()
        m, v = train.adamw_moments(m, v, g, B1, B2)
        p = train.adamw_param(p, m, v, LR, B1, B2, EPS, 0.0, number)
        np.testing.assert_array_equal(param.cpu().numpy(), p)
        np.testing.assert_array_equal(copy.cpu().view(torch.int16).numpy().view(np.uint16), train.to_bf16(p))
        np.testing.assert_array_equal(opt.state["m"][:n].cpu().numpy(), m)
        np.testing.assert_array_equal(opt.state["v"][:n].cpu().numpy(), v)
        for t, held in left:
            assert torch.equal(t.view(torch.uint8), held)

    def leave(t):
        old = t.detach()
        left.append((old, old.clone().view(torch.uint8)))

    step(1)
    leave(param)
    param.data = param.detach().clone()
    step(2)
    leave(copy)
    copy.data = torch.zeros(n + 5, dtype=torch.bfloat16, device=DEV)[5:]     # (off the 16-byte grid)
    step(3)
    leave(opt.state["m"])
    opt.state["m"] = opt.state["m"].clone()
    step(4)
    p = rng.standard_normal(n).astype(F)
    leave(param)
    param.data = torch.from_numpy(p).to(DEV)
    step(5)
    param.data = param.data.to(torch.bfloat16)
    with pytest.raises(TypeError, match="float32"):
        opt.step([torch.zeros(n, device=DEV)], lr=LR)


def test_moments_made_by_the_object_are_kept_until_their_step_is_done(ctx):
    """state["m"] replaced while the step that uses the old one waits behind other work on another stream: the memory
    is not handed out again before that step has run."""
    n = 1 << 20
    s = torch.cuda.Stream()
    p, g = torch.ones(n, device=DEV), torch.ones(n, device=DEV)
    a = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    other = gift.Context(stream=s.cuda_stream)
    opt = gift.AdamW(other, [p])
    fresh = torch.zeros_like(opt.state["m"])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            a @ a
    opt.step([g], lr=0.5)
    opt.state["m"] = fresh
    opt.step([g], lr=0.0)            # binds the new one and lets go of the old one
    taken = [torch.full((n,), 7.0, device=DEV) for _ in range(4)]     # on the current stream, which waits for nothing
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in taken)
    np.testing.assert_allclose(p.cpu().numpy(), 0.5, rtol=1e-6)       # the first step moves by lr
    opt.close()
    other.close()


@pytest.mark.parametrize("null", [True, False])
def test_close_waits_for_the_step(null):
    """Also where the context works on the null stream, behind work that takes some milliseconds."""
    s = torch.cuda.default_stream() if null else torch.cuda.Stream()
    p, g = torch.ones(300, device=DEV), torch.ones(300, device=DEV)
    a = torch.randn(8192, 8192, device=DEV)
    done = torch.cuda.Event()
    torch.cuda.synchronize()
    c = gift.Context(stream=s.cuda_stream)
    assert (c._stream == 0) == null
    opt = gift.AdamW(c, [p])
    with torch.cuda.stream(s):
        a @ a                        # (the library's first product loads its code)
        s.synchronize()
        for _ in range(20):
            a @ a
        opt.step([g], lr=0.5)
        done.record(s)
    opt.close()
    assert done.query()
    torch.cuda.synchronize()
    np.testing.assert_allclose(p.cpu().numpy(), 0.5, rtol=1e-6)
    c.close()
