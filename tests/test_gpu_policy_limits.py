"""The policy calls at the limits of their arguments, against 64 bits.

Tolerances.  u = 2^-24 is half a step of float32.  A row's sum of exponentials is off, relative to itself, by

  the additions one after another: one fewer than a lane has values, 6 steps over the lanes of a wave, one fewer than
    there are waves;
  3 u for every round that a workgroup's thread takes of a row, whose running sum is brought to a new maximum;
  the exponentials, 2 u each and (rounded difference, rounded product, the constant in it) 2.22 u for every unit of the
    distance from the maximum, whose mean under the row's probabilities is at most log(levels):

sum_bound below, in u: 38 at 1024 levels, 56 at 2048, 74 at 8192, 191 at 65536.  A log-probability d - log(sum) adds the rounding of
d, of the logarithm (2 u of it) and of the difference: (2 |d| + 3 |log sum| + sum_bound) u.

A gradient's value is made of products (slope of a choice) x (probability).  A slope holds exponentials of a
log-probability minus another number z: that log-probability's error, 3.22 u |z| of the difference, the product and the
constant, and 6 u of the exponential and the products; z reaches 8 upwards, and below zero e^z loses what |z| gains
against the 1 beside it.  A probability: 2.22 u |d| + (sum_bound + 5) u.  The sum over S slopes S u, what remains 8 u.
All of it relative to the parts' sizes as the oracle adds them up.
"""

import numpy as np
import pytest

import oracle.training as ot
from test_gpu_policy import U, dev, host, loss_inputs, rng

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lrb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2306_11268_amd import binding
    binding.load()
    return binding


def sum_bound(k):
    values, waves, rounds = (16, 1, 0) if k <= 1024 else (32, 1, 0) if k <= 2048 else (32, 4, 4) if k <= 8192 else (128, 8, 8)
    return values - 1 + 6 + waves - 1 + 3 * rounds + 2 + 2.22 * np.log(k)


def distances(x):
    x = x.astype(np.float64)
    d = x - x.max(-1, keepdims=True)
    return d, np.log(np.exp(d).sum(-1))


def check_logp(x, a, got):
    d, lz = distances(x)
    want = ot.policy_logp(x, a)
    da = np.take_along_axis(d, a.T, axis=1).T
    tol = (2 * np.abs(da) + 3 * np.abs(lz) + sum_bound(x.shape[1])) * U
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


def parts_bound(x, s):
    d, lz = distances(x)
    far = np.abs(d[np.isfinite(d)]).max()
    b = sum_bound(x.shape[1])
    return (2 * far + 3 * lz.max() + b + 3.22 * 8 + 6 + 2.22 * far + b + 5 + s + 8) * U


@pytest.mark.parametrize("k", (3, 16, 40, 100, 256, 1500, 3000, 6000, 40007))
@pytest.mark.parametrize("far", (-np.inf, -1e30, -1e8, -1000.0, -100.0))
def test_references_far_below_the_policy(lrb, k, far):
    """d = ref_logp - logp from far below zero to 8: dl/dlogp has kl_coef (1 - e^d), which is kl_coef where the reference
    bars the level, however large e^d - d - 1 is there."""
    g = rng(20, k)
    r, s = 9, 5
    x, a, old, adv, _ = loss_inputs(g, r, k, s, True, True)
    ref = (ot.policy_logp(x, a) + g.uniform(-30.0, 8.0, a.shape)).astype(np.float32)
    hit = g.uniform(size=a.shape) < 0.4
    hit[0, 0] = True
    ref[hit] = far
    a[2, 5] = a[0, 3] = -1
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.1, entropy_coef=0.05, scale=1.0 / a.size)
    with np.errstate(invalid="ignore"):
        want, terms, grad, size, sizes = ot.policy_loss(x, a, old, adv, ref_logp=ref, **kw)
    parts = parts_bound(x, s)
    t_tol = parts * sizes + U * np.abs(terms)
    for dt, half in ((torch.float32, U), (torch.bfloat16, 2.0 ** -8)):
        loss, got_terms, got = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), ref_logp=dev(ref), grad_dtype=dt, **kw)
        got, got_terms = host(got), host(got_terms)
        assert np.isfinite(got).all()
        off, tol = np.abs(got - grad), parts * size + half * np.abs(grad) + 1e-40
        assert np.all(off <= tol), (off / tol).max()
        fine = [0, 2, 3] if np.isinf(far) else [0, 1, 2, 3]
        assert np.all(np.abs(got_terms[fine] - terms[fine]) <= t_tol[fine] + 1e-40), (got_terms, terms)
        if np.isinf(far):
            assert got_terms[1] == np.inf and float(loss) == np.inf
        else:
            assert abs(float(loss) - want) <= t_tol[0] + 0.1 * t_tol[1] + 0.05 * t_tol[2] + U * abs(want)
    # no KL term in the loss: the reference is only reported
    loss, got_terms, got = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), ref_logp=dev(ref), **dict(kw, kl_coef=0.0))
    assert np.isfinite(float(loss)) and np.isfinite(host(got)).all()


def test_a_step_with_a_reference_that_bars_drawn_levels(lrb):
    """The reference policy's own log-probabilities, -inf where it bars a level: the step is taken."""
    g = rng(21)
    x = dev(g.standard_normal((50, 12)).astype(np.float32))
    before = x.clone()
    ref_scores = x.clone()
    ref_scores[:, 4] = -np.inf
    t = lrb.TrainTensors([x], [torch.zeros_like(x)])
    a, lp, _ = lrb.lr_policy_draw(x, dev(g.gumbel(size=(8, 50, 12)).astype(np.float32)))
    ref = lrb.lr_policy_logp(ref_scores, a)
    assert bool(torch.isinf(ref).any())
    _, _, norm = lrb.policy_train_step(t, a, lp, dev(g.standard_normal(8).astype(np.float32)), 1, lr=0.1, ref_logp=ref,
                                       kl_coef=0.1)
    assert np.isfinite(float(norm)) and not torch.equal(x, before)
    assert bool(torch.isfinite(x).all())


@pytest.mark.parametrize("k", (2, 16, 60, 300, 2000, 5000, 40007))
@pytest.mark.parametrize("reference", (False, True))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_an_action_out_of_range_shows_in_every_term(lrb, k, reference, dtype):
    x, a, old, adv, ref = loss_inputs(rng(22, k), 9, k, 3, False, reference)
    a[1, 4] = k
    for kl in (0.0, 0.1):
        loss, terms, grad = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), kl_coef=kl, entropy_coef=0.1,
                                               ref_logp=dev(ref) if reference else None, grad_dtype=dtype)
        assert np.isnan(float(loss)) and np.all(np.isnan(host(terms)))
        bad = np.isnan(host(grad))
        assert bad[4].all() and not np.delete(bad, 4, axis=0).any()


@pytest.mark.parametrize("rollouts,pixels", [(0, 5), (3, 0), (3, 5)])
def test_a_refused_loss_leaves_its_outputs(lrb, rollouts, pixels):
    x = torch.ones((pixels, 16), device="cuda")
    a = torch.zeros((rollouts, pixels), dtype=torch.int32, device="cuda")
    old, adv = torch.zeros((rollouts, pixels), device="cuda"), torch.ones(rollouts, device="cuda")
    out = torch.full((7, 16), 3.0, device="cuda")
    fit = out[:pixels]
    for args, kw in (((x, a, old.double(), adv), dict(out_grad=fit)), ((x, a.long(), old, adv), dict(out_grad=fit)),
                     ((x, a, old, adv[:0] if rollouts else torch.ones(2, device="cuda")), dict(out_grad=fit)),
                     ((x, a, old, adv), dict(out_grad=fit, ref_logp=old.half())),
                     ((x, a, old, adv), dict(out_grad=out)),
                     ((x, a, old, adv), dict(out_grad=fit, grad_dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            lrb.lr_policy_loss(*args, **kw)
    with pytest.raises(lrb.LrError):
        lrb.lr_policy_loss(x, a, old, adv, out_grad=fit, clip_low=2.0)
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("rollouts,pixels", [(0, 5), (3, 0), (0, 0)])
def test_a_gradient_of_no_choices_alone(lrb, rollouts, pixels):
    x = torch.ones((pixels, 16), device="cuda")
    a = torch.zeros((rollouts, pixels), dtype=torch.int32, device="cuda")
    old, adv = torch.zeros((rollouts, pixels), device="cuda"), torch.ones(rollouts, device="cuda")
    loss, terms, grad = lrb.lr_policy_loss(x, a, old, adv, want_loss=False)
    assert loss is None and terms is None and grad.shape == x.shape and not bool(grad.any())
    loss, terms, grad = lrb.lr_policy_loss(x, a, old, adv, want_grad=False)
    assert float(loss) == 0 and not bool(terms.any()) and grad is None


@pytest.mark.parametrize("k,rows", [(2051, 9), (5000, 6), (8192, 5), (10007, 4), (40007, 3)])
@pytest.mark.parametrize("s", (4, 5, 7, 8, 9, 13))
def test_draws_of_many_rollouts_from_long_rows(lrb, k, rows, s):
    """More rollouts than one pass over the scores takes, and groups of them that are not full."""
    g = rng(23, k, s)
    x = (2 * g.standard_normal((rows, k))).astype(np.float32)
    noise = g.gumbel(size=(s, rows, k)).astype(np.float32)
    noise[-1, 0, k - 1] = 100.0  # the last level, of the last rollout
    noise[s // 2, 1] = -np.inf   # (every score equal: the first)
    levels = g.uniform(0, 6, k).astype(np.float32)
    a, lp, phi = lrb.lr_policy_draw(dev(x), dev(noise), dev(levels))
    want = ot.policy_draw(x, noise)
    assert want[-1, 0] == k - 1 and want[s // 2, 1] == 0
    assert np.array_equal(host(a), want) and np.array_equal(host(phi), levels[want])
    check_logp(x, want, host(lp))
    # each rollout drawn alone gives the same
    for i in range(s):
        one = lrb.lr_policy_draw(dev(x), dev(noise[i:i + 1]))
        assert torch.equal(one[0][0], a[i]) and torch.equal(one[1][0], lp[i])


def test_draws_of_more_long_rows_than_workgroups(lrb):
    k, rows, s, n = 2051, 65536 + 97, 5, 61
    g = rng(24)
    x = dev((2 * g.standard_normal((n, k))).astype(np.float32))
    noise = dev(g.gumbel(size=(s, n, k)).astype(np.float32))
    small = lrb.lr_policy_draw(x, noise)
    assert np.array_equal(host(small[0]), ot.policy_draw(host(x), host(noise)))
    first = torch.arange(rows, device="cuda") % n
    big = lrb.lr_policy_draw(x[first], noise[:, first])
    assert torch.equal(big[0], small[0][:, first]) and torch.equal(big[1], small[1][:, first])


@pytest.mark.parametrize("k", (100, 2000, 3000, 10007))
@pytest.mark.parametrize("s", (257, 513, 1024))
def test_log_probabilities_of_more_rollouts_than_threads(lrb, k, s):
    g = rng(25, k, s)
    x = (2 * g.standard_normal((3, k))).astype(np.float32)
    a = g.integers(0, k, (s, 3)).astype(np.int32)
    a[0], a[-1] = 0, k - 1
    check_logp(x, a, host(lrb.lr_policy_logp(dev(x), dev(a))))


@pytest.mark.parametrize("k", (8192, 10007, 40007, 65536))
@pytest.mark.parametrize("spread", (0.1, 2.0, 6.0))
def test_clip_borders_of_long_rows(lrb, k, spread):
    """Ratios within float32's error of a border, where a row's sum is longest: the side is the one that 64 bits say."""
    g = rng(26, k)
    r, s = 12, 24
    low, high = 1.0 - float(np.float32(0.2)), 1.0 + float(np.float32(0.28))
    x = (spread * g.standard_normal((r, k))).astype(np.float32)
    a = g.integers(0, k, (s, r)).astype(np.int32)
    lp = ot.policy_logp(x, a)
    adv = np.where(g.uniform(size=(s, r)) < 0.5, 1.0, -1.0).astype(np.float32)
    border = np.where(adv > 0, np.log(high), np.log(low))
    away = g.uniform(-300 * U, 300 * U, (s, r))
    old = (lp - border + away).astype(np.float32)
    off = lp - old.astype(np.float64) - border
    a[np.abs(off) < 1e-9] = -1
    over = (a >= 0) & np.where(adv > 0, off > 0, off < 0)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.0, entropy_coef=0.0, scale=1.0)
    _, terms, grad, size, _ = ot.policy_loss(x, a, old, adv, **kw)
    assert terms[3] == over.sum() and 0.3 < over.mean() < 0.7
    _, got_terms, got = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), **kw)
    assert float(got_terms[3]) == over.sum()
    assert np.all(np.abs(host(got) - grad) <= parts_bound(x, s) * size + U * np.abs(grad) + 1e-40)
