"""Pins of the training oracle: its gradients against differences, its moments' codes by what they promise."""

import numpy as np
import pytest

import oracle.training as ot


def inputs(seed, r, k, s):
    g = np.random.default_rng([230611268, 40, seed])
    x = g.standard_normal((r, k)).astype(np.float32)
    a = g.integers(0, k, (s, r)).astype(np.int32)
    lp = ot.policy_logp(x, a)
    old = (lp + 0.2 * g.standard_normal((s, r))).astype(np.float32)
    ref = (lp + 0.4 * g.standard_normal((s, r))).astype(np.float32)
    return g, x, a, old, ref


@pytest.mark.parametrize("reference,entropy,per_choice", [(False, 0.0, False), (True, 0.0, True), (True, 0.3, False)])
def test_policy_gradient_against_differences(reference, entropy, per_choice):
    r, k, s = 3, 5, 6
    g, x, a, old, ref = inputs(1, r, k, s)
    a[2, 1] = -1
    adv = g.standard_normal((s, r) if per_choice else s).astype(np.float32)
    kw = dict(ref_logp=ref if reference else None, clip_low=0.15, clip_high=0.25, kl_coef=0.4, entropy_coef=entropy,
              scale=0.125)
    grad = ot.policy_loss(x, a, old, adv, **kw)[2]
    h = 1e-6
    for row in range(r):
        for col in range(k):
            up, down = x.astype(np.float64), x.astype(np.float64)
            up[row, col] += h
            down[row, col] -= h
            diff = (ot.policy_loss(up, a, old, adv, **kw)[0] - ot.policy_loss(down, a, old, adv, **kw)[0]) / (2 * h)
            # (central differences: h^2 of third derivatives, and 2^-53 / h of the loss)
            assert abs(diff - grad[row, col]) < 1e-8


def test_a_rollout_at_the_old_policy_has_the_plain_policy_gradient():
    r, k, s = 4, 6, 3
    g, x, a, old, _ = inputs(2, r, k, s)
    adv = g.standard_normal(s).astype(np.float32)
    lp = ot.log_softmax(x)
    loss, terms, grad, *_ = ot.policy_loss(x, a, ot.policy_logp(x, a), adv, scale=1.0)
    want = np.zeros((r, k))
    for i in range(s):
        for row in range(r):
            want[row] += adv[i] * np.exp(lp[row])
            want[row, a[i, row]] -= adv[i]
    assert np.allclose(grad, want, atol=1e-12) and terms[3] == 0
    assert abs(loss + adv.astype(np.float64).sum() * r) < 1e-12


def test_codes_are_ordered_and_cover_what_they_promise():
    m, v = ot.code_values(-14, 128), ot.code_values(-30, 256)
    for values, least in ((m, -14), (v, -30)):
        assert values[0] == 0 and np.all(np.diff(values) > 0)
        assert values[8] == 2.0 ** least and values[1] == 2.0 ** (least - 3)
        assert values[120 if least == -14 else 248] == 1.0
        # (neighbours are at most an eighth apart from the smallest normal value on)
        assert np.all(np.diff(values[8:]) <= values[8:-1] / 8)


def test_stored_moments_are_right_in_the_mean():
    """Rounding at random: a value's mean over many seeds is the value."""
    n, seeds = 512, 4000
    g = np.random.default_rng(5)
    m = (g.standard_normal(n) * 10.0 ** g.uniform(-4, 0, n)).astype(np.float32)
    v = (g.standard_normal(n) ** 2 * 10.0 ** g.uniform(-7, 0, n)).astype(np.float32)
    sums = np.zeros((2, n))
    for seed in range(seeds):
        cm, cv, sc = ot.encode(m, v, ot.random_bits(seed, 3, np.arange(n)))
        for i, d in enumerate(ot.decode(cm, cv, sc)):
            sums[i] += d
    for i, (x, least) in enumerate(((np.abs(m), -14), (v, -30))):
        u = 2 * np.repeat(sc[:, i].astype(np.float64), ot.BLOCK)
        values = ot.code_values(least, 257)
        low = np.searchsorted(values, x / u, side="right") - 1
        # A value at the part q of the distance D between two codes is stored as the upper one with probability q:
        # the mean of n draws is off by D sqrt(q (1 - q) / n) <= D / (2 sqrt n) in the mean square, and by five
        # times that in one of 10^6 cases (1024 values are looked at).
        bound = 5 * (values[low + 1] - values[low]) * u / (2 * np.sqrt(seeds))
        off = np.abs(sums[i] / seeds - (m if i == 0 else x))
        held = (low == 0) & (x > 0) & (i == 1)  # a v above zero takes the first code at least
        assert np.all(off[~held] <= bound[~held])
        assert np.allclose(sums[i][held] / seeds, (values[1] * u)[held], rtol=1e-12)


def test_random_bits_differ_between_tensors_seeds_and_halves():
    i = np.arange(1 << 16)
    base = ot.random_bits(7, 0, i)
    for other in (ot.random_bits(8, 0, i), ot.random_bits(7, 1, i), ot.random_bits(7, 0, i + (1 << 32))):
        # (two unrelated 32-bit numbers agree once in 2^32)
        assert np.count_nonzero(other == base) <= 2
    u = base / 2.0 ** 32
    # mean of n uniform numbers: 1/2 +- 5 / sqrt(12 n); correlation of neighbours: 0 +- 5 / sqrt(n)
    assert abs(u.mean() - 0.5) < 5 / np.sqrt(12 * u.size)
    assert abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 5 / np.sqrt(u.size)


def test_adamw_is_adam_without_decay_and_clipping():
    import oracle.donn as od
    g = np.random.default_rng(9)
    p, gr, m = (g.standard_normal(100).astype(np.float32) for _ in range(3))
    v = (g.standard_normal(100) ** 2).astype(np.float32)
    q, m1, v1 = ot.adamw(p, gr, m, v, 3, 0.5)
    f = lambda t: float(np.float32(t))  # noqa: E731
    ref = od.adam_update(p.astype(np.float64), gr.astype(np.float64), m.astype(np.float64), v.astype(np.float64), 3,
                         0.5, f(0.9), f(0.999), f(1e-8))
    # float32 moments: 2^-24 of each product and sum
    assert np.allclose(q, ref[0], rtol=0, atol=3e-6) and np.allclose(m1, ref[1], atol=4e-7)
    assert np.allclose(v1, ref[2], rtol=1e-6)
