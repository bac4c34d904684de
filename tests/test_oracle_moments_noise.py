"""How far 8-bit moments move the AdamW step (oracle, CPU).

Gradients are normal noise of constant variance, beta1 is 0.9; both moments are
stored as codes after every step and compared with the exact moving averages,
over the elements, after several time constants 1 / (1 - beta2).

Tolerances: n elements give a standard deviation, or a root of a mean square,
to a standard error of sqrt((k - 1) / (4 n)) of itself for a kurtosis k; with
k = 20 that is 3.5 % at n = 4096 and 6.9 % at 1024: 15 and 28 % are four of
them.  A mean of n elements is known to sd / sqrt(n), and four of those are asked.
"""

import numpy as np
import pytest

from oracle import train

F = np.float32


def noise(beta2, n, steps, beta1=0.9):
    """Standard deviation and mean of the stored v over the exact one, and the root mean square of the update's
    difference, relative to the update's: with both moments stored, and with v alone."""
    rng = np.random.default_rng(int(beta2 * 1000))
    zero = np.zeros(n, np.uint8), np.zeros(n // 256, F)
    m_codes, v_codes = zero, zero
    m_exact = v_exact = np.zeros(n)
    for _ in range(steps):
        g = (rng.standard_normal(n) * 1e-3).astype(F)
        m_exact = beta1 * m_exact + (1 - beta1) * g.astype(float)
        v_exact = beta2 * v_exact + (1 - beta2) * g.astype(float) ** 2
        m, v = train.adamw_moments(train.decode_moment(*m_codes), train.decode_moment(*v_codes), g, beta1, beta2)
        r = rng.integers(0, 65536, n)
        m_codes, v_codes = train.stochastic_codes(m, r, False), train.stochastic_codes(v, r, True)
    ratio = train.decode_moment(*v_codes) / v_exact
    exact, root = m_exact / np.sqrt(v_exact), np.sqrt(v.astype(float))

    def rms(x):
        return np.sqrt(np.mean(x * x))

    return ratio.std(), ratio.mean() - 1, rms(m / root - exact) / rms(exact), rms(m_exact / root - exact) / rms(exact)


@pytest.mark.parametrize("beta2,n,steps,v_noise,both,v_alone", [
    (0.95, 4096, 120, 0.12, 0.082, 0.055),
    (0.99, 4096, 600, 0.20, 0.115, 0.094),
    (0.999, 1024, 3000, 0.23, 0.135, 0.111),
])
def test_noise_of_8_bit_moments(beta2, n, steps, v_noise, both, v_alone):
    got = noise(beta2, n, steps)
    tol = 4 * np.sqrt(19 / (4 * n))
    assert abs(got[0] / v_noise - 1) <= tol
    assert abs(got[1]) <= 4 * v_noise / np.sqrt(n)
    assert abs(got[2] / both - 1) <= tol
    assert abs(got[3] / v_alone - 1) <= tol
