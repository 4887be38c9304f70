"""Levels drawn for rollouts and the clipped policy loss on the GPU, against 64 bits.

Tolerances.  u = 2^-24 is half a step of float32.  The sum of a row's
exponentials adds at most 64 values a lane and 10 levels of lanes, each
exponential within 4 u and 2 u for every unit of its argument, whose share falls
with e^-|argument| (less than 2 u altogether): 80 u of the sum, and as much of
its logarithm.  A log-probability d - log(sum), d = logit - maximum, is then
within (2 |d| + |log sum| + 84) u.  A gradient's parts are products of a ratio
exp(logp - old) and a probability: off by both arguments' errors, for logits
within 20 of the maximum 2 (40 + 12 + 84) u < 300 u = 1.8e-5 of the parts'
sum, and by half a step of the type it is kept in.
"""

import numpy as np
import pytest

import oracle.training as ot

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
PARTS = 300 * U


@pytest.fixture(scope="module")
def lrb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2306_11268_amd import binding
    binding.load()
    return binding


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def host(t):
    return t.detach().float().cpu().numpy() if t.dtype == torch.bfloat16 else t.detach().cpu().numpy()


def rng(*seed):
    return np.random.default_rng([230611268, 41, *seed])


def unaligned(x):
    """The same values on the GPU, four bytes behind a 16-byte border."""
    flat = torch.empty(x.size + 1, dtype=torch.from_numpy(x).dtype, device="cuda")
    flat[1:] = dev(x).reshape(-1)
    return flat[1:].view(x.shape)


def check_logp(x, a, got):
    lp = ot.policy_logp(x, a)
    x = x.astype(np.float64)
    with np.errstate(invalid="ignore"):
        d = x - x.max(-1, keepdims=True)
        lz = np.log(np.exp(d).sum(-1))
    da = np.take_along_axis(d, np.clip(a, 0, x.shape[1] - 1).T, axis=1).T
    made = (a >= 0) & (a < x.shape[1]) & np.isfinite(lp)
    tol = np.where(made, (2 * np.abs(np.where(made, da, 0)) + np.abs(np.where(made, lz, 0)) + 84) * U, 0)
    assert np.all(np.abs(got - lp)[made] <= tol[made]), np.max((np.abs(got - lp) / (tol + 1e-30))[made])
    assert np.array_equal(got[~made], lp[~made].astype(np.float32), equal_nan=True)


LEVELS = (1, 2, 3, 4, 5, 8, 15, 16, 17, 32, 33, 60, 64, 65, 100, 128, 129, 255, 256, 257, 260, 500, 512, 513, 1000, 1023,
          1024, 1025, 1100, 2048, 2051, 4096, 4100, 5000, 8192, 10007, 16384, 16388, 20000, 32768, 32772, 40007, 65535, 65536)


@pytest.mark.parametrize("k", LEVELS)
def test_draw_and_logp(lrb, k):
    g = rng(0, k)
    for rows, s in ((1, 1), (13, 3), (70 if k < 5000 else 5, 2)):
        x = (2 * g.standard_normal((rows, k))).astype(np.float32)
        noise = g.gumbel(size=(s, rows, k)).astype(np.float32)
        levels = g.uniform(0, 6, k).astype(np.float32)
        a, lp, phi = lrb.lr_policy_draw(dev(x), dev(noise), dev(levels))
        want = ot.policy_draw(x, noise)
        assert np.array_equal(host(a), want)
        assert np.array_equal(host(phi), levels[want])
        check_logp(x, want, host(lp))
        assert torch.equal(lrb.lr_policy_logp(dev(x), a), lp)
        # another alignment, another order of the sums: the same levels
        a2, lp2, none = lrb.lr_policy_draw(unaligned(x), unaligned(noise), None)
        assert none is None and torch.equal(a2, a)
        check_logp(x, want, host(lp2))


@pytest.mark.parametrize("k", (4, 16, 30, 256, 1000, 3000, 40000))
def test_draw_ties_nan_and_barred_levels(lrb, k):
    g = rng(1, k)
    x = np.zeros((6, k), np.float32)
    noise = np.round(g.uniform(0, 3, (2, 6, k))).astype(np.float32)  # many ties
    x[1] = -np.inf
    x[1, k - 1] = 1.0  # one level left
    x[2] = np.nan      # none: level 0
    x[3, : k // 2] = np.nan
    x[4] = -np.inf     # all barred: all equal, the first
    x[5] = np.finfo(np.float32).min
    noise[0, 0] = -np.inf
    a, lp, _ = lrb.lr_policy_draw(dev(x), dev(noise))
    assert np.array_equal(host(a), ot.policy_draw(x, noise))
    assert host(a)[0, 1] == k - 1 and host(lp)[0, 1] == 0.0
    assert np.all(host(a)[:, 2] == 0) and np.all(host(a)[:, 4] == 0)


def test_logp_without_choice_and_out_of_range(lrb):
    x = rng(2).standard_normal((9, 37)).astype(np.float32)
    a = rng(3).integers(0, 37, (5, 9)).astype(np.int32)
    a[1, 2], a[4, 8], a[0, 0], a[3, 3] = -1, -2147483648, 37, 2147483647
    got = host(lrb.lr_policy_logp(dev(x), dev(a)))
    assert got[1, 2] == 0 and got[4, 8] == 0 and np.isnan(got[0, 0]) and np.isnan(got[3, 3])
    check_logp(x, a, got)


def loss_inputs(g, r, k, s, per_choice, reference, spread=1.5):
    x = (spread * g.standard_normal((r, k))).astype(np.float32)
    p = np.exp(ot.log_softmax(x))
    cdf = np.cumsum(p, -1)
    a = np.stack([np.minimum((cdf < g.uniform(0, 1, (r, 1))).sum(-1), k - 1) for _ in range(s)]).astype(np.int32)
    lp = ot.policy_logp(x, a)
    old = (lp + 0.2 * g.standard_normal((s, r))).astype(np.float32)
    ref = (lp + 0.4 * g.standard_normal((s, r))).astype(np.float32) if reference else None
    adv = g.standard_normal((s, r) if per_choice else s).astype(np.float32)
    return x, a, old, adv, ref


KW = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.1, entropy_coef=0.05)


def check_loss(lrb, x, a, old, adv, ref, grad_dtype=torch.float32, put=dev, **kw):
    kw = {**KW, **kw}
    scale = kw.setdefault("scale", 1.0 / a.size)
    want, terms, grad, size, sizes = ot.policy_loss(x, a, old, adv, ref_logp=ref, **kw)
    loss, got_terms, got = lrb.lr_policy_loss(put(x), put(a), put(old), put(adv),
                                              ref_logp=None if ref is None else put(ref), grad_dtype=grad_dtype, **kw)
    assert got.dtype == grad_dtype
    half = U if grad_dtype == torch.float32 else 2.0 ** -8
    off = np.abs(host(got) - grad)
    tol = PARTS * size + half * np.abs(grad) + 1e-40
    assert np.all(off <= tol), (off / tol).max()
    # the loss's terms: each choice's as exactly as its gradient, the entropy as a sum of p log p
    t_tol = PARTS * sizes + U * np.abs(terms)
    assert np.all(np.abs(host(got_terms) - terms) <= t_tol + 1e-40), (host(got_terms), terms, t_tol)
    l_tol = t_tol[0] + kw["kl_coef"] * t_tol[1] + kw["entropy_coef"] * t_tol[2] + U * abs(want)
    assert abs(float(loss) - want) <= l_tol + 1e-40
    return loss, got_terms, got


@pytest.mark.parametrize("k", LEVELS)
def test_loss_and_gradient(lrb, k):
    g = rng(4, k)
    for i, (r, s) in enumerate(((1, 1), (19, 3), (67 if k < 2000 else 3, 6))):
        per, reference = bool((i + k) % 2), bool(i)
        x, a, old, adv, ref = loss_inputs(g, r, k, s, per, reference)
        check_loss(lrb, x, a, old, adv, ref)
        check_loss(lrb, x, a, old, adv, ref, put=unaligned)
        check_loss(lrb, x, a, old, adv, ref, grad_dtype=torch.bfloat16)


@pytest.mark.parametrize("s", (1, 2, 7, 16, 63, 64, 65, 100, 257, 1024))
@pytest.mark.parametrize("k", (3, 40, 256, 1001, 3000))
def test_many_rollouts_that_choose_the_same_levels(lrb, s, k):
    g = rng(5, s, k)
    r = 5 if s * k < 300000 else 2
    x, a, old, adv, ref = loss_inputs(g, r, k, s, True, True, spread=3.0)
    a[:, 0] = k - 1  # the same level every time
    old[:, 0] = ot.policy_logp(x, a)[:, 0] + 0.1
    ref[:, 0] = ot.policy_logp(x, a)[:, 0] - 0.1
    check_loss(lrb, x, a, old, adv, ref)


@pytest.mark.parametrize("k", (2, 16, 100, 256, 1024, 5000, 40007))
def test_missing_choices_barred_levels_and_empty_rows(lrb, k):
    g = rng(6, k)
    r, s = (41, 5) if k < 3000 else (6, 5)
    x, a, old, adv, ref = loss_inputs(g, r, k, s, True, True)
    barred = g.uniform(size=x.shape) < 0.3
    barred[np.arange(r)[None, :], a] = False  # (levels that were drawn stay open)
    x[barred] = -np.inf
    lp = ot.policy_logp(x, a)
    old, ref = (lp + 0.1).astype(np.float32), (lp - 0.2).astype(np.float32)
    gone = g.uniform(size=a.shape) < 0.3
    gone[:, 0] = gone[:, r - 1] = True  # rows without any choice
    gone[:, 1] = False
    a[gone] = -1 - g.integers(0, 5, int(gone.sum()))
    x[0], x[r - 1] = -np.inf, np.nan
    for t in (old, ref, adv):
        t[gone] = np.where(g.uniform(size=int(gone.sum())) < 0.5, np.nan, np.inf)
    # (the oracle leaves such places out; its softmax of rows 0 and r - 1 is not used)
    ox = x.copy()
    ox[0] = ox[r - 1] = 0
    kw = dict(KW, scale=1.0 / (~gone).sum())
    want, terms, grad, size, sizes = ot.policy_loss(ox, a, old, np.nan_to_num(adv), ref_logp=ref, **kw)
    for dt, half in ((torch.float32, U), (torch.bfloat16, 2.0 ** -8)):
        loss, got_terms, got = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), ref_logp=dev(ref), grad_dtype=dt,
                                                  **kw)
        got = host(got)
        assert np.all(got[0] == 0) and np.all(got[r - 1] == 0)
        assert np.all(np.abs(got - grad) <= PARTS * size + half * np.abs(grad) + 1e-40)
        assert np.all(np.abs(host(got_terms) - terms) <= PARTS * sizes + U * np.abs(terms))
    # nothing chosen anywhere
    loss, got_terms, got = lrb.lr_policy_loss(dev(x), dev(np.full_like(a, -1)), dev(old), dev(adv), ref_logp=dev(ref))
    assert float(loss) == 0 and not got_terms.any() and not got.any()


@pytest.mark.parametrize("k", (16, 300, 5000))
def test_an_action_out_of_range_shows(lrb, k):
    x, a, old, adv, ref = loss_inputs(rng(7, k), 9, k, 3, False, True)
    a[1, 4] = k
    loss, terms, grad = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), ref_logp=dev(ref), **KW)
    assert np.isnan(float(loss)) and np.all(np.isnan(host(terms)))
    bad = np.isnan(host(grad))
    assert bad[4].all() and not np.delete(bad, 4, axis=0).any()


@pytest.mark.parametrize("k", (2, 16, 256, 1024, 3000))
def test_ratios_next_to_the_clip_borders(lrb, k):
    """Choices a few 1e-8 on either side of a border: the gradient is there on one side and not on the other."""
    g = rng(8, k)
    r, s = (200, 16) if k < 3000 else (30, 16)
    x = (2 * g.standard_normal((r, k))).astype(np.float32)
    a = g.integers(0, k, (s, r)).astype(np.int32)
    lp = ot.policy_logp(x, a)
    adv = np.where(g.uniform(size=(s, r)) < 0.5, 1.0, -1.0).astype(np.float32)
    border = np.where(adv > 0, np.log(1.0 + float(np.float32(0.28))), np.log(1.0 - float(np.float32(0.2))))
    old = (lp - border).astype(np.float32)  # (rounding puts it a little to this side or that)
    ratio = np.exp(lp - old.astype(np.float64))
    over = np.where(adv > 0, ratio > 1.0 + float(np.float32(0.28)), ratio < 1.0 - float(np.float32(0.2)))
    clear = np.abs(lp - old.astype(np.float64) - border) > 1e-9
    assert 0.3 < over.mean() < 0.7 and clear.mean() > 0.9
    a[~clear] = -1
    _, terms, _ = check_loss(lrb, x, a, old, adv, None, scale=1.0)
    assert int(round(float(terms[3]))) == int((over & clear).sum())


@pytest.mark.parametrize("k", (3, 16, 40, 256, 3000))
@pytest.mark.parametrize("low,high", [(1.0, 1e6), (1.0, 0.0), (0.0, 0.0), (0.0, 3e38)])
def test_clips_at_their_limits_and_far_references(lrb, k, low, high):
    """Ratios of e^-3 to e^3, none within e^0.05 of one; references e^-4 to e^4 away, where e^d - d - 1 is formed as it
    stands (off by at most 1.7 times the error of d, which is below 150 u)."""
    g = rng(15, k)
    x, a, _, adv, _ = loss_inputs(g, 33, k, 5, True, True)
    lp = ot.policy_logp(x, a)
    away = g.uniform(0.05, 3.0, a.shape) * np.where(g.uniform(size=a.shape) < 0.5, 1, -1)
    old = (lp - away).astype(np.float32)
    ref = (lp + g.uniform(-4.0, 4.0, a.shape)).astype(np.float32)
    a[2, 5] = a[0, 0] = -1
    check_loss(lrb, x, a, old, adv, ref, clip_low=low, clip_high=high, kl_coef=0.03)
    check_loss(lrb, x, a, old, adv, None, clip_low=low, clip_high=high, entropy_coef=0.0)


def test_outputs_on_their_own_and_together_are_the_same(lrb):
    x, a, old, adv, ref = (dev(t) for t in loss_inputs(rng(9), 300, 64, 4, False, True))
    loss, terms, grad = lrb.lr_policy_loss(x, a, old, adv, ref_logp=ref, **KW)
    l2, t2, none = lrb.lr_policy_loss(x, a, old, adv, ref_logp=ref, want_grad=False, **KW)
    n1, n2, g2 = lrb.lr_policy_loss(x, a, old, adv, ref_logp=ref, want_loss=False, **KW)
    assert none is None and n1 is None and n2 is None
    assert torch.equal(loss, l2) and torch.equal(terms, t2) and torch.equal(grad, g2)
    again = lrb.lr_policy_loss(x, a, old, adv, ref_logp=ref, **KW)
    assert torch.equal(again[0], loss) and torch.equal(again[2], grad)


def test_gradient_against_differences_of_the_loss(lrb):
    """Central differences of the GPU's own loss along random directions."""
    g = rng(10)
    x, a, old, adv, ref = loss_inputs(g, 40, 24, 5, True, True)
    # (no ratio within 2e-2 of a border, so that none crosses one)
    ratio = np.exp(ot.policy_logp(x, a) - old)
    near = (np.abs(ratio - 1.28) < 3e-2) | (np.abs(ratio - 0.8) < 3e-2)
    a[near] = -1
    scale = 1.0
    args = (dev(a), dev(old), dev(adv))
    _, _, grad = lrb.lr_policy_loss(dev(x), *args, ref_logp=dev(ref), scale=scale, **KW)
    size = ot.policy_loss(x, a, old, adv, ref_logp=ref, scale=scale, **KW)[3].sum()
    h = 4e-3
    for i in range(5):
        d = g.choice((-1.0, 1.0), x.shape).astype(np.float32)
        d *= np.float32(h)
        up, down = x + d, x - d
        f = [float(lrb.lr_policy_loss(dev(t), *args, ref_logp=dev(ref), scale=scale, want_grad=False, **KW)[0])
             for t in (up, down)]
        moved = ((up - down).astype(np.float64) * host(grad)).sum()
        # h^3 / 3 of third derivatives (each at most 8 times a gradient's parts) and float32 losses and logits
        assert abs((f[0] - f[1]) - moved) <= 8 * h ** 3 * size + 4 * U * (abs(f[0]) + abs(f[1])) + 8 * PARTS * h * size


def test_empty_calls_do_nothing(lrb):
    x = torch.zeros((0, 16), device="cuda")
    a, lp, phi = lrb.lr_policy_draw(x, torch.zeros((3, 0, 16), device="cuda"))
    assert a.shape == (3, 0)
    x = torch.zeros((5, 16), device="cuda")
    a, lp, _ = lrb.lr_policy_draw(x, torch.zeros((0, 5, 16), device="cuda"))
    assert a.shape == (0, 5) and lrb.lr_policy_logp(x, a).shape == (0, 5)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("rollouts,pixels", [(0, 5), (3, 0), (0, 0)])
def test_a_loss_of_no_choices_is_zero(lrb, dtype, rollouts, pixels):
    """Also where the outputs' memory held something else: the step that follows takes them as they are."""
    x = torch.ones((pixels, 16), device="cuda")
    a = torch.zeros((rollouts, pixels), dtype=torch.int32, device="cuda")
    old, adv = torch.zeros((rollouts, pixels), device="cuda"), torch.ones(rollouts, device="cuda")
    out = torch.full((pixels, 16), 3.0, dtype=dtype, device="cuda")
    loss, terms, grad = lrb.lr_policy_loss(x, a, old, adv, grad_dtype=dtype, out_grad=out)
    assert float(loss) == 0 and not bool(terms.any()) and grad is out and not bool(grad.any())
    assert not bool(lrb.lr_policy_loss(x, a, old, adv, grad_dtype=dtype)[2].any())


def test_too_many_levels_or_rollouts_are_refused(lrb):
    x = torch.zeros((1, 65537), device="cuda")
    a = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        lrb.lr_policy_draw(x, x[None])
    with pytest.raises(ValueError):
        lrb.lr_policy_logp(x, a)
    with pytest.raises(ValueError):
        lrb.lr_policy_loss(x, a, a.float(), torch.ones(1, device="cuda"))
    with pytest.raises(ValueError):
        lrb.lr_policy_logp(x[:, :16].contiguous(), a.expand(1025, 1).contiguous())


def test_shapes_of_masks_pass_through(lrb):
    g = rng(11)
    x = g.standard_normal((2, 5, 7, 12)).astype(np.float32)
    noise = g.gumbel(size=(3, 2, 5, 7, 12)).astype(np.float32)
    a, lp, phi = lrb.lr_policy_draw(dev(x), dev(noise), dev(np.arange(12, dtype=np.float32)))
    assert a.shape == lp.shape == phi.shape == (3, 2, 5, 7)
    adv = g.standard_normal(3).astype(np.float32)
    loss, terms, grad = lrb.lr_policy_loss(dev(x), a, lp, dev(adv))
    assert grad.shape == x.shape
    want = ot.policy_loss(x.reshape(70, 12), host(a).reshape(3, 70), host(lp).reshape(3, 70), adv, scale=1 / 210)
    assert np.all(np.abs(host(grad).reshape(70, 12) - want[2]) <= PARTS * want[3] + 1e-40)


def test_rows_behind_2_31_values(lrb):
    """Offsets beyond 32 bits: the last rows of 2^31 and more logits, and nothing behind them."""
    k, r, s = 256, (1 << 23) + 5, 2
    x = torch.zeros((r, k), device="cuda")
    g = rng(12)
    tail = g.standard_normal((3, k)).astype(np.float32)
    x[-3:] = dev(tail)
    a = torch.full((s, r), -1, dtype=torch.int32, device="cuda")
    ta = g.integers(0, k, (s, 3)).astype(np.int32)
    a[:, -3:] = dev(ta)
    lp = lrb.lr_policy_logp(x, a)
    check_logp(tail, ta, host(lp[:, -3:]))
    old = lp - 0.1
    adv = np.array([1.0, -0.5], np.float32)
    _, _, grad = lrb.lr_policy_loss(x, a, old, dev(adv), scale=1.0)
    want = ot.policy_loss(tail, ta, host(old[:, -3:]), adv, scale=1.0)
    assert np.all(np.abs(host(grad[-3:]) - want[2]) <= PARTS * want[3] + 1e-40)
    assert not bool(grad[:-3].any())


@pytest.mark.parametrize("k,rows", [(2, 700001), (4, 660001), (7, 400003), (16, 330001), (31, 170003), (64, 90001),
                                    (128, 70001), (255, 36001), (512, 19001), (1000, 9001), (2048, 6301), (3001, 3301),
                                    (6000, 3101), (12000, 2203)])
def test_more_tiles_than_workgroups(lrb, k, rows):
    """Workgroups that take several tiles each: rows that repeat give what the first of them give, bit for bit."""
    g = rng(13, k)
    n, s = 97, 3
    x, a, old, adv, ref = loss_inputs(g, n, k, s, False, True)
    adv = np.array([0.7, -1.1, 0.4], np.float32)
    a[1, ::7] = -1
    noise = g.gumbel(size=(s, n, k)).astype(np.float32)
    kw = dict(KW, scale=0.5)
    one = lrb.lr_policy_loss(dev(x), dev(a), dev(old), dev(adv), ref_logp=dev(ref), **kw)
    first = torch.arange(rows, device="cuda") % n
    big = [dev(x)[first]] + [dev(t)[:, first].contiguous() for t in (a, old, ref)]
    loss, terms, grad = lrb.lr_policy_loss(big[0], big[1], big[2], dev(adv), ref_logp=big[3], **kw)
    assert torch.equal(grad, one[2][first])
    lp = lrb.lr_policy_logp(big[0], big[1])
    assert torch.equal(lp, lrb.lr_policy_logp(dev(x), dev(a))[:, first])
    # the loss's terms: those of the rows that repeat, and of the few behind the last whole round
    whole, rest = divmod(rows, n)
    part = lrb.lr_policy_loss(dev(x[:rest]), dev(a[:, :rest]), dev(old[:, :rest]), dev(adv), ref_logp=dev(ref[:, :rest]),
                              **kw)
    want = host(one[1]).astype(np.float64) * whole + (host(part[1]) if rest else 0)
    sizes = ot.policy_loss(x, a, old, adv, ref_logp=ref, **kw)[4] * (whole + 1)
    assert np.all(np.abs(host(terms) - want) <= PARTS * sizes)
    if rows * k * s < 3e8:
        big_noise = dev(noise)[:, first].contiguous()
        got = lrb.lr_policy_draw(big[0], big_noise)
        small = lrb.lr_policy_draw(dev(x), dev(noise))
        assert torch.equal(got[0], small[0][:, first]) and torch.equal(got[1], small[1][:, first])


@pytest.mark.parametrize("k", (2, 16, 100, 256, 1024, 2000, 3000, 5000, 12000, 40007))
@pytest.mark.parametrize("low", (-np.inf, float(np.finfo(np.float32).min), -1e30, -200.0))
def test_levels_barred_by_very_low_scores(lrb, k, low):
    """Most levels far below the others, in runs as long as a thread's share of a row: nothing of them is left."""
    g = rng(14, k)
    r, s = 5, 4
    x, a, old, adv, ref = loss_inputs(g, r, k, s, True, True)
    keep = np.zeros((r, k), bool)
    keep[np.arange(r)[None, :], a] = True
    keep[:, -1] = True
    x = np.where(keep, x, np.float32(low))
    x[3] = np.where(keep[3], x[3] + np.float32(50), x[3])
    lp = ot.policy_logp(x, a)
    old, ref = (lp + 0.1).astype(np.float32), (lp - 0.2).astype(np.float32)
    _, terms, grad = check_loss(lrb, x, a, old, adv, ref)
    assert np.isfinite(host(grad)).all() and np.isfinite(host(terms)).all()
    check_logp(x, a, host(lrb.lr_policy_logp(dev(x), dev(a))))
    noise = g.gumbel(size=(2, r, k)).astype(np.float32)
    got, glp, _ = lrb.lr_policy_draw(dev(x), dev(noise))
    assert np.array_equal(host(got), ot.policy_draw(x, noise))
    check_logp(x, host(got), host(glp))


@pytest.mark.parametrize("k,rows", [(12, 330001), (20, 200003), (24, 220001), (25, 190001), (40, 130001), (47, 90001),
                                    (48, 110001), (49, 90001), (63, 90001)])
def test_level_counts_between_the_powers_of_two(lrb, k, rows):
    test_loss_and_gradient(lrb, k)
    test_missing_choices_barred_levels_and_empty_rows(lrb, k)
    test_more_tiles_than_workgroups(lrb, k, rows)
