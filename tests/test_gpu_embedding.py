"""Embedding lookup and gradient on an MI355X.

The lookup multiplies once in float32 and rounds once to its output type: equal
to the oracle bit for bit.  The gradient of a row with L terms is a sum of
float32 additions: every term passes through the additions of its run (8 to 32
entries, at most RUN = 64), those of the row's at most L / 8 + 2 run sums, one
multiplication by the scale and, with accumulate, one addition; each rounding
is off by at most 2^-24 of a partial sum, and no partial sum exceeds the sum S
of the terms' magnitudes:

    |error| <= (RUN + L / 8 + 4) 2^-24 (scale S + |old|)
"""

import numpy as np
import pytest
import torch

from oracle import train

pytestmark = pytest.mark.gpu

gift = pytest.importorskip("paper_2607_07494_amd.gift")
DEV = "cuda"
RUN = 64
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print(*a, flush=True)


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = gift.Context()
    yield c
    torch.cuda.synchronize()
    c.close()


def values(gen, shape, dtype):
    return torch.randn(shape, generator=gen, dtype=torch.float32).to(DT[dtype])


def guarded(shape, dtype, offset, fill):
    """A tensor inside a larger one, `offset` elements from its start, and the whole."""
    n = int(np.prod(shape))
    whole = torch.full((n + offset + 64,), fill, dtype=dtype, device=DEV)
    return whole[offset:offset + n].view(shape), whole


def untouched(whole, n, offset, fill):
    return bool((whole[:offset] == fill).all()) and bool((whole[offset + n:] == fill).all())


# ---------------------------------------------------------------------------
# Lookup
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("T,V,d,table,out,ids,offset", [
    (1, 1, 1, "f32", "f32", 64, 0),
    (1, 7, 64, "bf16", "bf16", 32, 0),
    (5, 9, 63, "f32", "bf16", 64, 1),
    (7, 33, 65, "bf16", "f32", 32, 0),
    (9, 50, 127, "bf16", "bf16", 64, 3),
    (9, 50, 129, "f32", "f32", 32, 2),
    (33, 100, 257, "bf16", "bf16", 64, 1),
    (257, 1000, 771, "bf16", "f32", 64, 0),
    (300, 1000, 1024, "f32", "bf16", 32, 0),
    (64, 500, 1536, "f32", "f32", 64, 5),
])
def test_lookup(ctx, T, V, d, table, out, ids, offset):
    say("lookup", T, V, d, table, out, ids, offset)
    gen = torch.Generator().manual_seed(T + d)
    E = values(gen, (V, d), table)
    tok = torch.randint(0, V, (T,), generator=gen)
    if T > 4:
        tok[1], tok[2], tok[3] = -1, V, V - 1
        if ids == 64:
            tok[4] = 2 ** 40      # an id whose low half would lie inside the table
    want = train.lookup(E.float().numpy(), tok.numpy(), 1.7)
    tok_g = tok.to(torch.int64 if ids == 64 else torch.int32).to(DEV)
    E_g, _ = guarded((V, d), DT[table], offset, 0)
    E_g.copy_(E)
    got, whole = guarded((T, d), DT[out], offset, 5.0)
    gift.embedding(ctx, E_g, tok_g, got, scale=1.7)
    torch.cuda.synchronize()
    assert untouched(whole, T * d, offset, 5.0)
    if out == "f32":
        np.testing.assert_array_equal(got.cpu().numpy(), want)
    else:
        np.testing.assert_array_equal(got.cpu().view(torch.int16).numpy().view(np.uint16), train.to_bf16(want))


def test_lookup_keeps_special_values_and_the_shape_of_the_ids(ctx):
    E = torch.tensor([[float("nan"), float("inf"), -0.0, 1e-40]], device=DEV)
    tok = torch.zeros((2, 3), dtype=torch.int32, device=DEV)
    out = torch.empty((2, 3, 4), device=DEV)
    gift.embedding(ctx, E, tok, out)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int32), E.view(torch.int32).expand(2, 3, 4))
    half = torch.empty((2, 3, 4), dtype=torch.bfloat16, device=DEV)
    gift.embedding(ctx, E, tok, half)
    gift.embedding(ctx, E, tok[:0, 0], half[:0, 0])
    torch.cuda.synchronize()
    assert bool(torch.isnan(half[..., 0]).all()) and bool(torch.isinf(half[..., 1]).all())


# ---------------------------------------------------------------------------
# Gradient
# ---------------------------------------------------------------------------
def tokens_of(pattern, N, T, V, gen):
    if pattern == "zipf":
        tok = (torch.exp(torch.rand((N, T), generator=gen, dtype=torch.float64) * np.log(V + 1.0)) - 1).long().clamp(0, V - 1)
    elif pattern == "one":
        tok = torch.full((N, T), V // 2)
    elif pattern == "distinct":
        tok = torch.stack([torch.randperm(V, generator=gen)[:T] for _ in range(N)])
    elif pattern == "few":
        tok = torch.randint(0, min(3, V), (N, T), generator=gen)
    elif pattern == "none":
        tok = torch.full((N, T), -1)
    else:
        tok = torch.randint(-V // 2 - 1, V + V // 2 + 1, (N, T), generator=gen)      # a third and more outside
    return tok


CASES = [
    # N, T, V, d, dout, ids, pattern
    (1, 1, 1, 1, "f32", 64, "one"),
    (1, 1, 300, 65, "bf16", 32, "distinct"),
    (1, 31, 40, 64, "f32", 64, "few"),
    (1, 32, 40, 128, "bf16", 64, "one"),
    (1, 33, 40, 129, "bf16", 32, "one"),
    (2, 64, 70, 257, "bf16", 64, "few"),
    (3, 65, 255, 256, "f32", 32, "zipf"),
    (2, 100, 256, 63, "bf16", 64, "outside"),
    (2, 500, 257, 130, "f32", 64, "outside"),
    (1, 200, 1000, 100, "f32", 64, "none"),
    (1, 1000, 65536, 72, "bf16", 64, "distinct"),
    (2, 2047, 5000, 96, "bf16", 32, "zipf"),
    (2, 2048, 65535, 40, "f32", 64, "zipf"),
    (2, 2049, 300, 260, "bf16", 64, "zipf"),
    (1, 4097, 70000, 200, "f32", 32, "zipf"),
    (1, 6000, 17, 515, "bf16", 64, "zipf"),
    (1, 20000, 32000, 64, "bf16", 64, "zipf"),
    (1, 9000, 11, 33, "f32", 64, "one"),
    (17, 130, 90, 48, "bf16", 32, "outside"),
    # the borders of the sort's forms: 2048 and 8192 positions in a workgroup, 64 tiles of 2048, more
    (2, 8192, 300, 20, "f32", 64, "zipf"),
    (2, 8193, 3000, 24, "bf16", 32, "outside"),
    (1, 65536, 2000, 16, "bf16", 64, "zipf"),
    (1, 40000, 9, 12, "f32", 64, "one"),
    (1, 30000, 255, 12, "f32", 64, "zipf"),
    (1, 30000, 256, 12, "f32", 32, "few"),
    (1, 131072, 700, 8, "bf16", 64, "few"),
    (2, 131073, 65536, 4, "f32", 64, "outside"),
    (1, 600_000, 70000, 2, "f32", 32, "zipf"),
    (1, 300, 1_048_577, 3, "f32", 64, "zipf"),
    (1, 300, 1_048_576, 3, "f32", 64, "outside"),
    (2, 5000, 140_000, 9, "bf16", 64, "outside"),
    (1, 9000, 3, 1030, "bf16", 64, "one"),
    (2, 40, 30, 5000, "bf16", 64, "few"),
    (300, 5, 7, 3, "f32", 32, "outside"),
]


def run_grad(ctx, tok, dout, V, scale, accumulate, old, offset=0, **kw):
    N, T, d = dout.shape
    grads, whole = guarded((N, V, d), torch.float32, offset, 7.0)
    grads.copy_(old) if accumulate else grads.fill_(float("nan"))
    x, _ = guarded(dout.shape, dout.dtype, offset, 0)
    x.copy_(dout)
    gift.embedding_grad(ctx, tok, x, grads, scale=scale, accumulate=accumulate, **kw)
    torch.cuda.synchronize()
    assert untouched(whole, N * V * d, offset, 7.0)
    return grads.cpu()


def check_grad(got, tok, dout, V, scale, old):
    N, T, d = dout.shape
    want = train.lookup_grad(tok.numpy(), dout.float().numpy(), V, scale)
    size = train.lookup_grad(tok.numpy(), dout.float().abs().numpy(), V, abs(scale))
    terms = np.zeros((N, V, 1))
    for j in range(N):
        t = tok[j][(tok[j] >= 0) & (tok[j] < V)].numpy()
        np.add.at(terms[j, :, 0], t, 1)
    before = old.double().numpy() if old is not None else np.zeros_like(want)
    err = np.abs(got.double().numpy() - (want + before))
    bound = (RUN + terms / 8 + 4) * 2.0 ** -24 * (size + np.abs(before))
    assert np.all(err <= bound), float((err - bound).max())
    empty = np.broadcast_to(terms == 0, want.shape)
    np.testing.assert_array_equal(got.numpy()[empty], before[empty])     # zeros, or what was there


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,T,V,d,dtype,ids,pattern", CASES)
def test_grad(ctx, N, T, V, d, dtype, ids, pattern, accumulate):
    say("grad", N, T, V, d, dtype, ids, pattern, accumulate)
    gen = torch.Generator().manual_seed(T + d)
    tok, dout = tokens_of(pattern, N, T, V, gen), values(gen, (N, T, d), dtype)
    old = torch.randn((N, V, d), generator=gen) if accumulate else None
    tok_g = tok.to(torch.int64 if ids == 64 else torch.int32).to(DEV)
    offset = d % 4
    got = run_grad(ctx, tok_g, dout, V, -1.3, accumulate, old, offset)
    check_grad(got, tok, dout, V, -1.3, old)
    again = run_grad(ctx, tok_g, dout, V, -1.3, accumulate, old, offset)
    assert torch.equal(got, again)


def test_grad_of_no_positions(ctx):
    tok, dout = torch.zeros((2, 0), dtype=torch.int64, device=DEV), torch.zeros((2, 0, 5), device=DEV)
    grads = torch.full((2, 100, 5), 3.0, device=DEV)
    gift.embedding_grad(ctx, tok, dout, grads, accumulate=True)
    torch.cuda.synchronize()
    assert bool((grads == 3).all())
    gift.embedding_grad(ctx, tok, dout, grads)
    torch.cuda.synchronize()
    assert bool((grads == 0).all())


def test_padding_rows_are_not_read(ctx):
    """NaN in the gradients of padded positions reaches nothing."""
    tok = torch.tensor([[4, -1, 4, 99, 0, 2 ** 40]], device=DEV)
    dout = torch.ones((1, 6, 70), device=DEV)
    dout[0, [1, 3, 5]] = float("nan")
    grads = torch.empty((1, 6, 70), device=DEV)
    gift.embedding_grad(ctx, tok, dout, grads)
    torch.cuda.synchronize()
    assert grads[0, :, 0].tolist() == [1.0, 0.0, 0.0, 0.0, 2.0, 0.0] and not bool(torch.isnan(grads).any())


def test_infinities_and_nans_stay_in_their_row(ctx):
    tok = torch.tensor([[3, 1, 3, 2]], device=DEV)
    dout = torch.ones((1, 4, 9), device=DEV)
    dout[0, 0, 0], dout[0, 2, 0], dout[0, 1, 1] = float("inf"), float("-inf"), float("inf")
    grads = torch.empty((1, 5, 9), device=DEV)
    gift.embedding_grad(ctx, tok, dout, grads)
    torch.cuda.synchronize()
    g = grads[0].cpu()
    assert torch.isnan(g[3, 0]) and torch.isinf(g[1, 1])
    assert torch.isnan(g).sum() == 1 and torch.isinf(g).sum() == 1


def test_gradient_is_the_lookups_difference_quotient(ctx):
    """The lookup is linear, so (f(E + D) - f(E - D)) / 2 = <grad, D> for f(E) = <dout, lookup(E)>; each of the two
    lookups is off by 2^-24 of its values (and of E +- D's), f in float64."""
    gen = torch.Generator().manual_seed(3)
    T, V, d, s = 200, 60, 130, 2.5
    tok = tokens_of("outside", 1, T, V, gen).to(DEV)
    E, D = (torch.randn((V, d), generator=gen).to(DEV) for _ in range(2))
    dout = torch.randn((1, T, d), generator=gen).to(DEV)
    grads, out = torch.empty((1, V, d), device=DEV), torch.empty((1, T, d), device=DEV)
    gift.embedding_grad(ctx, tok, dout, grads, scale=s)
    f, size = [], 0.0
    for table in (E + D, E - D):
        gift.embedding(ctx, table, tok, out, scale=s)
        torch.cuda.synchronize()
        f.append(float((out.double() * dout.double()).sum()))
        size += float((out.double() * dout.double()).abs().sum())
    terms = torch.bincount(tok[0][(tok[0] >= 0) & (tok[0] < V)], minlength=V).max()
    slack = 2.0 ** -24 * size + (RUN + float(terms) / 8 + 4) * 2.0 ** -24 * s * float(
        (dout[0].double().abs()[(tok[0] >= 0) & (tok[0] < V)] * D.double().abs()[tok[0][(tok[0] >= 0) & (tok[0] < V)]]).sum())
    assert abs((f[0] - f[1]) / 2 - float((grads[0].double() * D.double()).sum())) <= slack


def test_offsets_past_32_bits(ctx):
    """A gradient and a table of more than 2^31 elements and 2^33 bytes."""
    V, d = 2_200_000, 1000
    tok = torch.tensor([[V - 1, 0, V - 2, V - 1]], device=DEV)
    dout = torch.arange(4 * d, device=DEV).float().view(1, 4, d) % 251
    grads = torch.empty((1, V, d), device=DEV).fill_(float("nan"))
    gift.embedding_grad(ctx, tok, dout, grads)
    out = torch.empty((1, 4, d), device=DEV)
    gift.embedding(ctx, grads[0], tok, out)
    torch.cuda.synchronize()
    assert torch.equal(grads[0, V - 1], dout[0, 0] + dout[0, 3]) and torch.equal(grads[0, V - 2], dout[0, 2])
    assert torch.equal(grads[0, 0], dout[0, 1])
    assert torch.equal(out[0], torch.stack([dout[0, 0] + dout[0, 3], dout[0, 1], dout[0, 2], dout[0, 0] + dout[0, 3]]))
    grads[0, [V - 1, V - 2, 0]] = 0
    assert not bool(grads.any())      # (a NaN is true)


# ---------------------------------------------------------------------------
# Streams, scratch, capture
# ---------------------------------------------------------------------------
def test_other_stream_and_own_scratch(ctx):
    gen = torch.Generator().manual_seed(9)
    N, T, V, d = 2, 700, 400, 200
    tok, dout = tokens_of("zipf", N, T, V, gen).to(DEV), values(gen, (N, T, d), "bf16").to(DEV)
    want = run_grad(ctx, tok, dout, V, 1.0, False, None)
    need = gift.embedding_grad_scratch(N, T, V, d)
    scratch = torch.empty(need + 512, dtype=torch.uint8, device=DEV).fill_(255)
    start = -scratch.data_ptr() % 256
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = gift.Context(stream=s.cuda_stream)
    got = run_grad(other, tok, dout, V, 1.0, False, None, scratch=scratch[start:start + need])
    assert torch.equal(got, want) and bool((scratch[start + need:] == 255).all())
    with pytest.raises(gift.GiftError, match="too small"):
        run_grad(other, tok, dout, V, 1.0, False, None, scratch=scratch[start:start + need - 1])
    with pytest.raises(gift.GiftError, match="misaligned"):
        run_grad(other, tok, dout, V, 1.0, False, None, scratch=scratch[start + 1:])
    other.close()


def test_captured_calls(ctx):
    """Two graphs of one context with scratch of their own, replayed between eager calls on new inputs."""
    gen = torch.Generator().manual_seed(11)
    N, T, V, d = 2, 3000, 500, 96
    tok, dout = torch.zeros((N, T), dtype=torch.int64, device=DEV), torch.zeros((N, T, d), device=DEV)
    s = torch.cuda.Stream()
    c = gift.Context(stream=s.cuda_stream)
    need = gift.embedding_grad_scratch(N, T, V, d)
    outs, graphs = [], []
    keep = []
    for _ in range(2):
        grads, rows = torch.empty((N, V, d), device=DEV), torch.empty((N, T, d), device=DEV)
        scratch = torch.empty(need, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            with pytest.raises(gift.GiftError, match="scratch"):
                gift.embedding_grad(c, tok, dout, grads)
            gift.embedding_grad(c, tok, dout, grads, scratch=scratch)
            gift.embedding(c, grads[0], tok, rows)
        outs.append((grads, rows))
        graphs.append(graph)
        keep.append(scratch)
    for k in range(4):
        tok.copy_(tokens_of("zipf" if k % 2 else "outside", N, T, V, gen))
        dout.copy_(torch.randn(dout.shape, generator=gen))
        torch.cuda.synchronize()
        for graph, (grads, rows) in zip(graphs, outs):
            grads.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            eager, eager_rows = torch.empty_like(grads), torch.empty_like(rows)
            gift.embedding_grad(ctx, tok, dout, eager)
            gift.embedding(ctx, eager[0], tok, eager_rows)
            torch.cuda.synchronize()
            assert torch.equal(grads, eager) and torch.equal(rows, eager_rows), k
    c.close()
