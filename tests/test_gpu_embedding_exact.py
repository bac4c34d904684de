"""Embedding gradient of frequent ids on an MI355X, bit for bit.

The output gradients are whole numbers of -3 .. 3 (exact in bfloat16), the scale
is a power of two, and what is added to are whole numbers: with L terms in a row
every partial sum is a whole number of at most 3 L < 2^24, so float32 additions
are exact in any order and a part that is lost, doubled or added to another
row shows, however long the row is.
"""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

gift = pytest.importorskip("paper_2607_07494_amd.gift")
DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gift.Context()
    yield c
    torch.cuda.synchronize()
    c.close()


def ids(pattern, N, T, V, gen):
    if pattern == "one":
        return torch.full((N, T), V - 1)
    if pattern == "few":
        return torch.randint(0, min(3, V), (N, T), generator=gen)
    if pattern == "half":         # every other position holds one id, between two others of many
        tok = torch.randint(0, V, (N, T), generator=gen)
        tok[:, ::2] = V // 2
        return tok
    if pattern == "padded":       # an id for padding inside the table, behind it
        tok = torch.randint(1, V, (N, T), generator=gen)
        tok[:, T // 5:] = 0
        return tok
    # lengths of 1, 2, 4, ... positions, then what is left
    return (torch.arange(T) + 1).log2().floor().long().clamp(max=V - 1).expand(N, T)[:, torch.randperm(T, generator=gen)]


CASES = [
    # N, T, V, d, dout, pattern: rows of 2 to 4096 runs
    (1, 63, 2, 1, "f32", "one"),
    (1, 257, 3, 5, "bf16", "one"),
    (1, 288, 5, 64, "bf16", "one"),           # at 8 entries a run: 36 runs
    (1, 520, 5, 130, "f32", "one"),           # 65
    (2, 2048, 40, 260, "bf16", "half"),
    (1, 2049, 7, 300, "f32", "one"),
    (3, 8192, 9, 70, "bf16", "few"),
    (1, 8193, 300, 33, "f32", "padded"),
    (2, 20000, 500, 257, "bf16", "lengths"),
    (1, 40000, 9, 12, "f32", "one"),
    (1, 65536, 32000, 128, "bf16", "half"),
    (1, 65536, 2000, 515, "bf16", "padded"),
    (1, 65537, 30, 260, "f32", "lengths"),
    (1, 131072, 700, 8, "bf16", "few"),
    (1, 131071, 4, 3, "f32", "one"),
    (5, 30011, 64, 16, "bf16", "lengths"),
]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,T,V,d,dtype,pattern", CASES)
def test_whole_numbers(ctx, N, T, V, d, dtype, pattern, accumulate):
    print("exact", N, T, V, d, dtype, pattern, accumulate, flush=True)
    gen = torch.Generator().manual_seed(T + V + d)
    tok = ids(pattern, N, T, V, gen)
    dout = torch.randint(-3, 4, (N, T, d), generator=gen).float()
    old = torch.randint(-1000, 1001, (N, V, d), generator=gen).float()
    scale = 0.25
    want = (old if accumulate else torch.zeros_like(old)).double()
    for j in range(N):
        want[j].index_add_(0, tok[j], dout[j].double() * scale)
    grads = old.to(DEV) if accumulate else torch.full((N, V, d), float("nan"), device=DEV)
    gift.embedding_grad(ctx, tok.to(DEV), dout.to(DT[dtype]).to(DEV), grads, scale=scale, accumulate=accumulate)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(grads.cpu().double().numpy(), want.numpy())


def test_random_values_within_the_chain_of_additions(ctx):
    """A row of L terms: at most 32 additions in a run; its runs' sums, at most L / 8 + 2, in four shares of one quarter
    each, then the shares: (32 + (L / 8 + 2) / 4 + 4 + 2) 2^-24 of the terms' magnitudes with scale and rounding."""
    gen = torch.Generator().manual_seed(4)
    for T, V, d in ((40000, 9, 12), (131072, 3, 8)):
        print("chain", T, V, d, flush=True)
        tok, dout = torch.full((1, T), V - 1), torch.randn((1, T, d), generator=gen)
        grads = torch.empty((1, V, d), device=DEV)
        gift.embedding_grad(ctx, tok.to(DEV), dout.to(DEV), grads, scale=0.7)
        torch.cuda.synchronize()
        scale = float(np.float32(0.7))
        want, size = scale * dout[0].double().sum(0), scale * dout[0].double().abs().sum(0)
        bound = (32 + (T / 8 + 2) / 4 + 6) * 2.0 ** -24 * size
        assert bool(((grads[0, V - 1].cpu().double() - want).abs() <= bound).all())
        assert not bool(grads[0, :V - 1].any())
