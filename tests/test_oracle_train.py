"""Pins of the training-step oracle (CPU)."""

import numpy as np

from oracle import e4m3, train

F = np.float32


def test_lookup_grad_is_the_one_hot_product_and_the_difference_quotient():
    rng = np.random.default_rng(0)
    N, T, V, d, s = 2, 9, 5, 3, 1.5
    tokens = rng.integers(-1, V + 1, (N, T))
    dout = rng.standard_normal((N, T, d))
    got = train.lookup_grad(tokens, dout, V, s)
    hot = (tokens[..., None] == np.arange(V)).astype(float)
    np.testing.assert_allclose(got, s * np.einsum("ntv,ntd->nvd", hot, dout), atol=1e-14)
    table, move = rng.standard_normal((V, d)), rng.standard_normal((V, d))
    for j in range(N):
        f = lambda E: (dout[j] * s * np.where(((tokens[j] >= 0) & (tokens[j] < V))[:, None],
                                              E[np.clip(tokens[j], 0, V - 1)], 0)).sum()
        np.testing.assert_allclose((f(table + move) - f(table - move)) / 2, (got[j] * move).sum(), atol=1e-12)


def test_first_adamw_step_is_the_sign_step():
    """From zero moments m / (1 - b1) = g and v / (1 - b2) = g^2: p moves by lr g / (|g| + eps)."""
    g = np.array([3.0, -2e-4, 0.0, 1e-9])
    p, m, v = train.adamw_formula(np.ones(4), np.zeros(4), np.zeros(4), g, 0.1, 0.9, 0.95, 1e-8, 0.5, 1)
    np.testing.assert_allclose(p, 0.95 - 0.1 * g / (np.abs(g) + 1e-8), rtol=1e-13)
    m32, v32 = train.adamw_moments(np.zeros(4, F), np.zeros(4, F), g.astype(F), 0.9, 0.95)
    np.testing.assert_allclose(m32, m, rtol=2e-7)
    np.testing.assert_allclose(v32, v, rtol=3e-7)
    np.testing.assert_allclose(train.adamw_param(np.ones(4, F), m32, v32, 0.1, 0.9, 0.95, 1e-8, 0.5, 1), p, rtol=3e-7)


def test_block_rounding_takes_a_neighbour_and_is_right_in_the_mean():
    """Every value goes to one of its two neighbours on E4M3's grid, over all 2^16 numbers in the proportion that
    makes the mean right: the share of the upper one is the fraction to 2^-16 (and
    below 2^-6 to the 2^-21 of a step that y + 2^-6 is rounded to)."""
    grid = np.sort(np.unique(np.abs(e4m3.decode_table()[:127])))
    rng = np.random.default_rng(1)
    values = np.concatenate([rng.uniform(0, 448, 20), 2.0 ** rng.uniform(-9.5, 8.8, 60), grid[1:20]]).astype(F)
    r = np.arange(65536)
    for y in values:
        x = np.full(65536, y)
        x[::256] = 448            # the block's maximum: multiplier 448 fl(1 / 448)
        codes, scales = train.stochastic_codes(x, r, False)
        np.testing.assert_array_equal(scales, F(448) * (F(1) / F(448)))
        q = e4m3.dequantize(codes).astype(np.float64)
        keep = np.arange(65536) % 256 != 0
        y = F(y) * (F(448) * (F(1) / F(448)))
        lo = grid[np.searchsorted(grid, y, "right") - 1]
        hi = grid[min(np.searchsorted(grid, y, "right"), len(grid) - 1)]
        assert np.all((q[keep] == lo) | (q[keep] == hi)), y
        if hi > lo:
            # 256 of the 65536 numbers are left out, one of every 256 neighbours
            share = (q[keep] == hi).mean()
            assert abs(share - (float(y) - lo) / (hi - lo)) <= 2 ** -16 + 2 ** -21 + 1 / 256, y


def test_block_rounding_corners():
    x = np.zeros(512, F)
    x[:256] = 1e-6
    x[0] = 448
    x[1], x[2] = -1e-6, 0
    codes, scales = train.stochastic_codes(x, np.zeros(512, np.int64), True)
    assert scales[0] == F(448) * (F(1) / F(448)) and scales[1] == 0 and np.all(codes[256:] == 0)
    assert codes[3] == 1 and codes[2] == 0 and codes[1] == 0x81      # positive never 0; the sign is kept
    x[5] = np.nan
    codes, scales = train.stochastic_codes(x, np.zeros(512, np.int64), True)
    assert np.isnan(scales[0]) and np.all(codes[:256] & 0x7F == 0x7F) and scales[1] == 0


def test_random_numbers_take_the_words_in_order():
    from oracle.subspace import philox4x32_10
    r = train.random_numbers(1100, 3, 7, (5 << 32) | 9)
    w = [int(np.asarray(a).ravel()[0]) for a in philox4x32_10(np.array([2]), np.array([0]), np.array([3]), np.array([7]), 9, 5)]
    # call 2: elements 8..11 (words 0, 1) and 264..267 (words 2, 3)
    want = [h for x in w for h in (x & 0xFFFF, x >> 16)]
    assert [int(x) for x in r[8:12]] + [int(x) for x in r[264:268]] == want
    assert abs(r.mean() / 65535 - 0.5) < 0.05


def test_bf16_rounding():
    x = np.array([1.0, 1.00390625, 1.01171875, -3.4e38, np.inf, np.nan, 1e-45], F)
    got = train.to_bf16(x)
    assert list(got[:3]) == [0x3F80, 0x3F80, 0x3F82] and got[4] == 0x7F80 and (got[5] & 0x7FFF) > 0x7F80 and got[6] == 0


def test_norm():
    assert train.grad_norm([np.array([3.0]), np.array([[4.0]])], 1.0) == (5.0, 1.0 / (5.0 + 1e-6))
    assert np.isnan(train.grad_norm([np.array([np.inf])], 1.0)[1])
