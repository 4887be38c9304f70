"""Refusals of the calls that train device levels by reward: on the host, before anything is launched."""

import ctypes
import os

import pytest

from paper_2306_11268_amd import binding as lb

pytestmark = pytest.mark.skipif(not os.path.exists(lb.LIB_PATH), reason="liblr.so not built")

P = ctypes.c_void_p
A = [P(0x100000000 * (i + 1)) for i in range(12)]  # far from each other
SIZE, ARG, NULL, WORK, ALIAS = 2, 3, 1, 6, 7


def draw(logits=A[0], noise=A[1], levels=A[2], s=4, n=100, k=16, actions=A[3], logp=A[4], phi=A[5]):
    return lb.load().lr_policy_draw(logits, noise, levels, s, n, k, actions, logp, phi, None)


def test_draw():
    for k in (0, -1, 65537):
        assert draw(k=k) == SIZE
    assert draw(s=-1) == SIZE and draw(s=1025) == SIZE and draw(n=-1) == SIZE
    assert draw(n=1 << 60) == SIZE and draw(n=1 << 45, k=65536) == SIZE  # bytes beyond 2^63
    assert draw(logits=None) == NULL and draw(noise=None) == NULL and draw(actions=None) == NULL
    assert draw(levels=None) == NULL  # phases need the levels
    assert draw(actions=A[1]) == ALIAS and draw(logp=A[3]) == ALIAS and draw(phi=A[0]) == ALIAS
    assert draw(logp=P(A[0].value + 100 * 16 * 4 - 4)) == ALIAS
    assert draw(phi=P(A[1].value + 4 * 100 * 16 * 4 - 4)) == ALIAS  # inside the last rollout's noise
    assert draw(s=0, logits=None) == 0 and draw(n=0, logits=None) == 0


def test_logp():
    f = lambda logits=A[0], actions=A[1], s=4, n=100, k=16, logp=A[2]: lb.load().lr_policy_logp(  # noqa: E731
        logits, actions, s, n, k, logp, None)
    assert f(k=0) == SIZE and f(s=-1) == SIZE and f(n=-5) == SIZE
    assert f(logits=None) == NULL and f(actions=None) == NULL and f(logp=None) == NULL
    assert f(logp=A[1]) == ALIAS and f(logp=P(A[0].value + 8)) == ALIAS
    assert f(n=0, logp=None) == 0


def loss(policy=(0.2, 0.2, 0.1, 0.1, 1.0), logits=A[0], actions=A[1], old=A[2], ref=A[3], adv=A[4], per=0, s=4, n=100,
         k=16, out=A[5], terms=A[6], gt=0, grad=A[7], work=A[8], size=None):
    lib = lb.load()
    size = lib.lr_policy_workspace_size() if size is None else size
    p = None if policy is None else ctypes.byref(lb.LrPolicy(*policy))
    return lib.lr_policy_loss(p, logits, actions, old, ref, adv, per, s, n, k, out, terms, gt, grad, work, size, None)


def test_loss():
    nan, inf = float("nan"), float("inf")
    assert loss(policy=None) == NULL
    for bad in ((-0.1, 0.2, 0, 0, 1), (1.5, 0.2, 0, 0, 1), (nan, 0.2, 0, 0, 1), (0.2, -0.1, 0, 0, 1), (0.2, inf, 0, 0, 1),
                (0.2, nan, 0, 0, 1), (0.2, 0.2, inf, 0, 1), (0.2, 0.2, 0, nan, 1), (0.2, 0.2, 0, 0, nan),
                (0.2, 0.2, 0, 0, inf)):
        assert loss(policy=bad) == ARG, bad
    assert loss(gt=2) == ARG and loss(gt=-1) == ARG
    assert loss(k=0) == SIZE and loss(k=65537) == SIZE and loss(s=-1) == SIZE and loss(s=1025) == SIZE
    assert loss(n=-1) == SIZE
    assert loss(out=None, terms=None, grad=None) == NULL
    for name in ("logits", "actions", "old", "adv", "work"):
        assert loss(**{name: None}) == NULL, name
    assert loss(size=lb.load().lr_policy_workspace_size() - 1) == WORK
    assert loss(work=P(A[8].value + 4)) == WORK  # not aligned
    # every output over every input, and over each other
    for o in ("out", "terms", "grad", "work"):
        for at in (A[0], A[1], A[2], A[3], A[4]):
            assert loss(**{o: at}) == ALIAS, (o, at)
    assert loss(out=A[6]) == ALIAS and loss(grad=A[8]) == ALIAS and loss(terms=P(A[7].value + 96)) == ALIAS
    # the advantages of every choice are longer than those of the rollouts
    assert loss(out=P(A[4].value + 16), per=1) == ALIAS
    assert loss(n=0, logits=None) == 0 and loss(s=0, logits=None) == 0


def param(i=0, n=1000, **kw):
    base = 0x10000000000 * (i + 1)
    at = dict(d_param=base, d_grad=base + 0x100000000, d_m=base + 0x200000000, d_v=base + 0x300000000,
              d_scales=base + 0x400000000, count=n)
    at.update(kw)
    return lb.LrParam(**at)


def table(*params):
    return (lb.LrParam * len(params))(*params)


def test_grad_norm():
    lib = lb.load()
    w = lib.lr_grad_norm_workspace_size(2)
    assert w > 0 and lib.lr_grad_norm_workspace_size(0) == w
    # one set of partial sums for each launch, of a few dozen tensors
    sizes = [lib.lr_grad_norm_workspace_size(n) for n in range(1, 500)]
    assert all(b >= a and b % w == 0 for a, b in zip(sizes, sizes[1:])) and sizes[-1] <= 16 * w
    assert lib.lr_grad_norm_workspace_size(-1) == -SIZE and lib.lr_grad_norm_workspace_size(65537) == -SIZE
    f = lambda t, num, gt=0, norm=A[0], work=A[1], size=w: lib.lr_grad_norm(t, num, gt, norm, work, size, None)  # noqa: E731
    t = table(param(0), param(1))
    assert f(t, 2, gt=2) == ARG
    assert f(t, -1) == SIZE and f(t, 65537) == SIZE and f(table(param(n=-1)), 1) == SIZE
    assert f(table(param(n=1 << 56), param(1, n=1)), 2) == SIZE  # counts that do not add up
    assert f(None, 1) == NULL and f(t, 2, norm=None) == NULL and f(t, 2, work=None) == NULL
    assert f(table(param(d_grad=None)), 1) == NULL
    assert f(t, 2, size=w - 1) == WORK and f(t, 2, work=P(A[1].value + 4)) == WORK
    assert f(t, 2, norm=P(A[1].value + 64)) == ALIAS
    assert f(table(param(d_grad=A[0].value - 8)), 1) == ALIAS
    assert f(table(param(d_grad=A[1].value + w - 4)), 1) == ALIAS


def adamw(t, num, gt=0, st=0, step=1, lr=0.1, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, norm=None, top=1.0, seed=0):
    return lb.load().lr_adamw_update(t, num, gt, st, step, lr, b1, b2, eps, wd, norm, top, seed, None)


def test_adamw():
    nan, inf = float("nan"), float("inf")
    t = table(param(0), param(1))
    assert adamw(t, 2, step=0) == SIZE and adamw(t, -1) == SIZE and adamw(t, 65537) == SIZE
    assert adamw(table(param(n=-1)), 1) == SIZE
    for bad in (dict(gt=2), dict(st=2), dict(st=-1), dict(lr=nan), dict(lr=inf), dict(b1=1.0), dict(b1=-0.1),
                dict(b1=nan), dict(b2=1.0), dict(b2=nan), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(wd=-0.1),
                dict(wd=nan), dict(wd=inf), dict(top=0.0), dict(top=-1.0), dict(top=nan)):
        assert adamw(t, 2, **bad) == ARG, bad
    assert adamw(None, 1) == NULL
    for name in ("d_param", "d_grad", "d_m", "d_v"):
        assert adamw(table(param(0), param(1, **{name: None})), 2) == NULL, name
    assert adamw(table(param(d_scales=None)), 1, st=1) == NULL
    # nothing to do: no tensors, or empty ones whose pointers are not looked at
    assert adamw(None, 0) == 0
    assert adamw(table(lb.LrParam(None, None, None, None, None, 0)), 1) == 0


def test_adamw_refuses_overlapping_buffers():
    a, b = param(0), param(1)
    assert adamw(table(a, a), 2) == ALIAS  # the same tensor twice
    for name in ("d_param", "d_m", "d_v"):
        for other in ("d_param", "d_grad", "d_m", "d_v"):
            # the last value of one inside the first of another tensor's
            at = getattr(a, other) + 4 * 999
            assert adamw(table(a, param(1, **{name: at})), 2) == ALIAS, (name, other)
            if name != other:
                assert adamw(table(param(0, **{name: getattr(a, other)})), 1) == ALIAS, (name, other)
    # 8-bit moments: 1000 bytes, scales of four blocks
    assert adamw(table(a, param(1, d_m=a.d_m + 999)), 2, st=1) == ALIAS
    assert adamw(table(a, param(1, d_v=a.d_scales + 4 * 8 - 1)), 2, st=1) == ALIAS
    # the norm is read while the parameters are written
    assert adamw(table(a, b), 2, norm=P(b.d_param + 3996)) == ALIAS
    assert adamw(table(a, b), 2, norm=P(b.d_v)) == ALIAS
    # a bf16 gradient ends after 2000 bytes, a float32 one does not
    assert adamw(table(param(0, d_param=a.d_grad + 2000)), 1, gt=0) == ALIAS


def test_moments():
    lib = lb.load()
    arr = lambda *p: (P * len(p))(*p)  # noqa: E731
    t = table(param())
    assert lib.lr_adamw_moments(t, -1, None, None, None) == SIZE
    assert lib.lr_adamw_moments(None, 1, arr(A[0]), arr(A[1]), None) == NULL
    assert lib.lr_adamw_moments(t, 1, None, arr(A[1]), None) == NULL
    assert lib.lr_adamw_moments(t, 1, arr(A[0]), arr(None), None) == NULL
    assert lib.lr_adamw_moments(table(param(d_scales=None)), 1, arr(A[0]), arr(A[1]), None) == NULL
    assert lib.lr_adamw_moments(t, 1, arr(A[0]), arr(A[0]), None) == ALIAS
    assert lib.lr_adamw_moments(t, 1, arr(t[0].d_m), arr(A[1]), None) == ALIAS
    assert lib.lr_adamw_moments(t, 1, arr(A[0]), arr(t[0].d_scales), None) == ALIAS
    assert lib.lr_adamw_moments(None, 0, None, None, None) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        lb.lr_policy_draw(x, torch.zeros(2, 4, 8))
    with pytest.raises(ValueError):
        lb.lr_policy_logp(x, torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        lb.lr_policy_loss(x, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 4), torch.zeros(2))
    with pytest.raises(ValueError):
        lb.TrainTensors([x], [x])
    with pytest.raises(ValueError):
        lb.TrainTensors([x], [x], bits=16)
