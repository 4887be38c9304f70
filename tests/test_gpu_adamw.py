"""The optimiser step over many tensors on the GPU: gradient norm, AdamW with moments of 32 and of 8 bits.

Moments are compared bit for bit: they are float32 products and sums in a stated
order, and their codes a function of them and of the random bits.  A parameter
p k - rate m / (sqrt(v) root + eps) is rounded in keep, rate, root (half a step
each), the product, the root (one step), the sum, the quotient (1.5 steps), the
last product and the difference: within 10 u of the change and 2 u of the value,
u = 2^-24.
"""

import numpy as np
import pytest

import oracle.training as ot

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


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
    return t.detach().cpu().numpy()


def rng(*seed):
    return np.random.default_rng([230611268, 42, *seed])


def bf16(x):
    """float32 values that bfloat16 holds."""
    return torch.from_numpy(x).to(torch.bfloat16).float().numpy()


COUNTS = (
    [1], [7, 255, 256, 257, 0, 1, 1000], [2048, 2049, 4096 * 3 + 5], [100003], list(range(1, 130)),
    [50000 - 37 * i for i in range(60)],
)


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_grad_norm(lrb, counts, dtype):
    grads = [bf16(rng(0, n, i).standard_normal(n).astype(np.float32)) for i, n in enumerate(counts)]
    want = ot.grad_norm(grads)
    got = lrb.lr_grad_norm([dev(g).to(dtype) for g in grads])
    # (summed in float64, rounded once)
    assert abs(float(got) - want) <= 2 * U * want
    # at any alignment: one buffer without gaps
    flat = torch.cat([torch.zeros(1, device="cuda")] + [dev(g) for g in grads]).to(dtype)
    at, cut = 1, []
    for n in counts:
        cut.append(flat[at:at + n])
        at += n
    assert torch.equal(lrb.lr_grad_norm(cut), lrb.lr_grad_norm(cut))
    assert abs(float(lrb.lr_grad_norm(cut)) - want) <= 2 * U * want


def test_grad_norm_of_nothing_of_large_and_of_broken_values(lrb):
    assert float(lrb.lr_grad_norm([])) == 0
    assert float(lrb.lr_grad_norm([torch.zeros(0, device="cuda"), torch.zeros(5, device="cuda")])) == 0
    big = torch.full((300,), 1e30, device="cuda")  # squares beyond float32
    assert abs(float(lrb.lr_grad_norm([big])) - 1e30 * 300 ** 0.5) <= 1e30 * 300 ** 0.5 * 4 * U
    small = torch.full((300,), 1e-30, device="cuda")
    assert abs(float(lrb.lr_grad_norm([small])) - 1e-30 * 300 ** 0.5) <= 1e-30 * 300 ** 0.5 * 4 * U
    for bad in (float("nan"), float("inf"), -float("inf")):
        t = torch.ones(5000, device="cuda")
        t[4321] = bad
        got = float(lrb.lr_grad_norm([torch.ones(7, device="cuda"), t]))
        assert np.isnan(got) if np.isnan(bad) else got == float("inf")


def moments32(g, n):
    return (g.standard_normal(n) * 1e-3).astype(np.float32), (g.standard_normal(n) ** 2 * 1e-6).astype(np.float32)


def check_params(p0, want, got):
    change = np.abs(want - p0)
    # (the change is a difference of the decay and the update: each at most as large as |p| or the update)
    assert np.all(np.abs(got - want) <= 12 * U * (change + np.abs(p0)) + 1e-38), np.max(np.abs(got - want))


OPT = dict(lr=0.05, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("packed", (False, True))
def test_adamw_32(lrb, counts, dtype, packed):
    g = rng(1, sum(counts))
    data = []
    for n in counts:
        m, v = moments32(g, n)
        data.append((g.standard_normal(n).astype(np.float32), bf16((g.standard_normal(n) * 1e-2).astype(np.float32)), m, v))
    kinds = [[dev(d[i]) for d in data] for i in range(4)]
    kinds[1] = [t.to(dtype) for t in kinds[1]]
    guard = None
    if packed:
        # one buffer for each kind, its tensors without gaps between two guards
        flat = [torch.cat([torch.full((1,), 7.0, device="cuda", dtype=k[0].dtype)] + k
                          + [torch.full((3,), 7.0, device="cuda", dtype=k[0].dtype)]) for k in kinds]
        starts = 1 + np.concatenate([[0], np.cumsum(counts)])
        kinds = [[f[a:a + n] for a, n in zip(starts, counts)] for f in flat]
        guard = flat
    norm = torch.tensor(2.0, device="cuda")
    t = lrb.TrainTensors(kinds[0], kinds[1], m=kinds[2], v=kinds[3])
    lrb.lr_adamw_update(t, 4, norm=norm, max_norm=0.7, **OPT)
    for (p, gr, m, v), tp, tm, tv in zip(data, kinds[0], kinds[2], kinds[3]):
        wp, wm, wv = ot.adamw(p, gr, m, v, 4, norm=2.0, max_norm=0.7, **OPT)
        assert np.array_equal(host(tm), wm) and np.array_equal(host(tv), wv)
        check_params(p, wp, host(tp))
    if guard:
        for f in guard:
            assert float(f[0]) == 7.0 and bool((f[-3:] == 7.0).all())


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("packed", (False, True))
def test_adamw_8_over_several_steps(lrb, counts, dtype, packed):
    g = rng(2, sum(counts))
    ps = [g.standard_normal(n).astype(np.float32) for n in counts]
    size = [10.0 ** g.uniform(-4, 1, n) for n in counts]
    if packed:
        cut = lambda dt, per=1: [b[3 if per == 1 else 0:][sum(-(-c // per) if per > 1 else c for c in counts[:i]):][:-(-n // per)]  # noqa: E731
                                 for b in [torch.zeros(sum(counts) + 2048, dtype=dt, device="cuda")]
                                 for i, n in enumerate(counts)]
        dp, dg, m, v = cut(torch.float32), cut(dtype), cut(torch.uint8), cut(torch.uint8)
        for a, b in zip(dp, ps):
            a.copy_(dev(b))
        t = lrb.TrainTensors(dp, dg, bits=8, m=m, v=v)
    else:
        dp, dg = [dev(p) for p in ps], [torch.zeros(n, device="cuda", dtype=dtype) for n in counts]
        t = lrb.TrainTensors(dp, dg, bits=8)
    state = [(np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros((-(-n // 256), 2), np.float32)) for n in counts]
    for step in range(1, 5):
        grads = [bf16((s * g.standard_normal(n) * (g.uniform(size=n) < 0.9)).astype(np.float32))
                 for s, n in zip(size, counts)]
        for a, b in zip(dg, grads):
            a.copy_(dev(b))
        lrb.lr_adamw_update(t, step, seed=1000 + step, **OPT)
        for i, n in enumerate(counts):
            p0 = ps[i]
            m, v = (x.astype(np.float32) for x in ot.decode(*state[i]))
            wp, wm, wv = ot.adamw(p0, grads[i], m, v, step, **OPT)
            cm, cv, sc = ot.encode(wm, wv, ot.random_bits(1000 + step, i, np.arange(n)))
            assert np.array_equal(host(t.m[i]), cm), (step, i)
            assert np.array_equal(host(t.v[i]), cv), (step, i)
            assert np.array_equal(host(t.scales[i]), sc), (step, i)
            check_params(p0, wp, host(dp[i]))
            ps[i], state[i] = host(dp[i]).copy(), (cm, cv, sc)
    m, v = lrb.lr_adamw_moments(t)
    for i in range(len(counts)):
        wm, wv = ot.decode(*state[i])
        assert np.array_equal(host(m[i]), wm.astype(np.float32)) and np.array_equal(host(v[i]), wv.astype(np.float32))


def test_adamw_8_extreme_moments(lrb):
    """Blocks of zeros, of the smallest and of the largest values, one value far above the rest, and broken ones."""
    n = 256 * 8 + 9
    g = rng(3)
    gr = np.zeros(n, np.float32)
    gr[256:512] = 1e-30 * g.standard_normal(256)       # squares below float32's smallest
    gr[512:768] = 1e15 * g.standard_normal(256)
    gr[768:1024] = g.standard_normal(256) * 1e-5
    gr[800] = 100.0
    gr[1100] = np.inf                                   # block 4
    gr[1300] = np.nan                                   # block 5
    gr[1600] = 3e19                                     # its square is beyond 2^126: block 6's v
    gr[256 * 8:] = g.standard_normal(9)
    p = g.standard_normal(n).astype(np.float32)
    dp = dev(p)
    t = lrb.TrainTensors([dp], [dev(gr)], bits=8)
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        lrb.lr_adamw_update(t, 1, seed=5, **OPT)
        wp, wm, wv = ot.adamw(p, gr, np.zeros(n, np.float32), np.zeros(n, np.float32), 1, **OPT)
    sc = host(t.scales[0])
    for block, (bad_m, bad_v) in enumerate([(0, 0)] * 4 + [(1, 1), (1, 1), (0, 1), (0, 0), (0, 0)]):
        assert np.isnan(sc[block, 0]) == bool(bad_m) and np.isnan(sc[block, 1]) == bool(bad_v), block
    good = np.repeat(~np.isnan(sc).any(1), 256)[:n]
    with np.errstate(invalid="ignore"):
        cm, cv, want = ot.encode(wm, wv, ot.random_bits(5, 0, np.arange(n)))
    assert np.array_equal(sc, want, equal_nan=True)
    assert np.array_equal(host(t.m[0])[good], cm[good]) and np.array_equal(host(t.v[0])[good], cv[good])
    fine = np.isfinite(wp)
    assert np.array_equal(np.isfinite(host(dp)), fine)
    check_params(p[fine], wp[fine], host(dp)[fine])
    m, v = lrb.lr_adamw_moments(t)
    assert np.all(np.isnan(host(m[0])[256 * 4:256 * 6])) and np.all(np.isnan(host(v[0])[256 * 4:256 * 7]))
    # a second moment above zero is not stored as zero
    assert np.all(host(t.v[0])[good][wv[good] > 0] > 0)


@pytest.mark.parametrize("bits", (8, 32))
def test_a_norm_that_is_not_finite_leaves_everything(lrb, bits):
    g = rng(4)
    p, gr = dev(g.standard_normal(3000).astype(np.float32)), dev(g.standard_normal(3000).astype(np.float32))
    t = lrb.TrainTensors([p], [gr], bits=bits)
    lrb.lr_adamw_update(t, 1, **OPT)
    held = [x.clone() for x in (p, t.m[0], t.v[0])]
    for bad in (float("nan"), float("inf"), -float("inf")):
        lrb.lr_adamw_update(t, 2, norm=torch.tensor(bad, device="cuda"), **OPT)
        assert all(torch.equal(a, b) for a, b in zip(held, (p, t.m[0], t.v[0])))
    lrb.lr_adamw_update(t, 2, norm=torch.tensor(1.0, device="cuda"), **OPT)
    assert not torch.equal(held[0], p)


@pytest.mark.parametrize("norm,max_norm", [(0.5, 1.0), (1.0, 1.0), (3.0, 1.0), (1e30, 1e-3), (2.0, float("inf")), (0.0, 1.0)])
def test_clipping(lrb, norm, max_norm):
    g = rng(5)
    p, gr = g.standard_normal(777).astype(np.float32), g.standard_normal(777).astype(np.float32)
    m, v = moments32(g, 777)
    dp, dm, dv = dev(p), dev(m), dev(v)
    t = lrb.TrainTensors([dp], [dev(gr)], m=[dm], v=[dv])
    lrb.lr_adamw_update(t, 7, norm=torch.tensor(norm, device="cuda"), max_norm=max_norm, **OPT)
    wp, wm, wv = ot.adamw(p, gr, m, v, 7, norm=norm, max_norm=max_norm, **OPT)
    assert np.array_equal(host(dm), wm) and np.array_equal(host(dv), wv)
    check_params(p, wp, host(dp))


def test_same_step_as_lr_adam_update(lrb):
    """Without decay and clipping it is the Adam step of the phase masks."""
    g = rng(6)
    phi, gr = g.uniform(0, 6, 40000).astype(np.float32), g.standard_normal(40000).astype(np.float32)
    a, m, v = dev(phi), torch.zeros(40000, device="cuda"), torch.zeros(40000, device="cuda")
    b = dev(phi)
    t = lrb.TrainTensors([b], [dev(gr)])
    for step in (1, 2, 3):
        lrb.lr_adam_update(a, dev(gr), m, v, step, lr=0.5)
        lrb.lr_adamw_update(t, step, lr=0.5)
    # three steps of at most 0.5 each way, 12 u of change and value in both
    assert float((a - b).abs().max()) <= 2 * 3 * 12 * U * (0.6 + 8)


def test_tensors_behind_2_32_values(lrb):
    """One tensor of more than 2^32 values, 8-bit moments: its last block, and the random bits' upper half."""
    n = (1 << 32) + 300
    p = torch.zeros(n, device="cuda")
    gr = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = rng(7)
    tail = bf16(g.standard_normal(300).astype(np.float32))
    gr[-300:] = dev(tail).to(torch.bfloat16)
    t = lrb.TrainTensors([p], [gr], bits=8)
    assert abs(float(lrb.lr_grad_norm(t)) - ot.grad_norm([tail])) <= 2 * U * ot.grad_norm([tail])
    lrb.lr_adamw_update(t, 1, seed=77, **OPT)
    z = np.zeros(300, np.float32)
    wp, wm, wv = ot.adamw(z, tail, z, z, 1, **OPT)
    cm, cv, sc = ot.encode(wm, wv, ot.random_bits(77, 0, np.arange(n - 300, n)))
    assert np.array_equal(host(t.m[0][-300:]), cm) and np.array_equal(host(t.v[0][-300:]), cv)
    assert np.array_equal(host(t.scales[0][-2:]), sc)
    check_params(z, wp, host(p[-300:]))
    assert not bool(p[:-300].any())


def test_the_object_keeps_the_memory_it_was_given(lrb):
    p, gr = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    t = lrb.TrainTensors([p], [gr])
    p.data = torch.zeros(1000, device="cuda")  # the caller's tensor goes elsewhere
    held = t._held["d_param"][0]
    lrb.lr_adamw_update(t, 1, lr=0.1)
    keep = torch.empty(0, device="cuda").set_(held)
    assert float(p.abs().max()) == 0 and keep.numel() == 1000 and float(keep.max()) < 1
    with pytest.raises(ValueError):
        lrb.policy_train_step(t, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), gr, gr, 1, lr=0.1)
    with pytest.raises(ValueError):
        t.set_grads([torch.ones(999, device="cuda")])
    with pytest.raises(ValueError):
        t.set_grads([torch.ones(2000, device="cuda")[::2]])
    with pytest.raises(ValueError):
        lrb.TrainTensors([p], [gr, gr])
    with pytest.raises(ValueError):
        lrb.TrainTensors([p.half()], [gr])
    t.set_grads([torch.zeros(1000, dtype=torch.bfloat16, device="cuda")])
    lrb.lr_adamw_update(t, 2, lr=0.1)
    same = torch.ones(1000, device="cuda")
    with pytest.raises(lrb.LrError):
        lrb.lr_adamw_update(lrb.TrainTensors([same, same], [gr, gr]), 1, lr=0.1)


def test_a_step_beyond_32_bits_is_refused(lrb):
    p = torch.ones(8, device="cuda")
    t = lrb.TrainTensors([p], [torch.ones(8, device="cuda")])
    with pytest.raises(ValueError):
        lrb.lr_adamw_update(t, 2 ** 32 + 1, lr=0.1)
    with pytest.raises(lrb.LrError):
        lrb.lr_adamw_update(t, 0, lr=0.1)
    assert bool((p == 1).all())
    lrb.lr_adamw_update(t, 2 ** 31 - 1, lr=0.5)
    # m = 1 - beta1, v = 1 - beta2, uncorrected, with the call's float32 betas (1 - float32(0.999) is 1.3e-5 below 0.001,
    # the step 1.58 times half of that: 1.0e-5)
    b1, b2 = float(np.float32(0.9)), float(np.float32(0.999))
    assert abs(float(p[0]) - (1 - 0.5 * (1 - b1) / ((1 - b2) ** 0.5 + 1e-8))) < 16 * 2 ** -24
