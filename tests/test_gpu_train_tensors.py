"""What an optimiser step's tensors may go through between steps, on the GPU."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lrb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2306_11268_amd import binding
    binding.load()
    return binding


def scores_and_bias():
    x, bias = torch.zeros((6, 8), device="cuda"), torch.zeros(9, device="cuda")
    return [x, bias], [torch.zeros_like(x), torch.ones_like(bias)]


def rollouts(lrb, x, s=3):
    g = np.random.default_rng([230611268, 45])
    noise = torch.from_numpy(g.gumbel(size=(s, *x.shape)).astype(np.float32)).cuda()
    a, lp, _ = lrb.lr_policy_draw(x, noise)
    return a, lp, torch.ones(s, device="cuda")


@pytest.mark.parametrize("which", ("params", "grads"))
@pytest.mark.parametrize("i", (0, 1))
def test_a_policy_step_refuses_any_tensor_that_moved(lrb, which, i):
    params, grads = scores_and_bias()
    t = lrb.TrainTensors(params, grads)
    a, lp, adv = rollouts(lrb, params[0])
    moved = (params, grads)[which == "grads"][i]
    moved.data = moved.clone()
    with pytest.raises(ValueError):
        lrb.policy_train_step(t, a, lp, adv, 1, lr=0.1)
    assert not any(bool(z.any()) for z in (*params, grads[0], *t.m, *t.v))
    # put in place by the calls that are there for it
    t = lrb.TrainTensors(params, [g.clone() for g in grads])
    t.set_grads(grads)
    lrb.policy_train_step(t, a, lp, adv, 1, lr=0.1)
    assert bool(params[1].any())


def calls(lrb, t, field):
    """The calls that use a field."""
    yield lambda: lrb.lr_adamw_update(t, 1, lr=0.1)
    if field == "grads":
        yield lambda: lrb.lr_grad_norm(t)
    if field in ("m", "v", "scales") and t.bits == 8:
        yield lambda: lrb.lr_adamw_moments(t)


@pytest.mark.parametrize("bits,field", [(bits, f) for bits in (32, 8) for f in ("params", "grads", "m", "v", "scales")
                                        if bits == 8 or f != "scales"])
@pytest.mark.parametrize("size", (0, 16, 1 << 16))
def test_a_resized_storage_is_refused(lrb, bits, field, size):
    """Its memory has gone back to the allocator: the addresses that the object holds are no longer its own."""
    ones = lambda: [torch.ones(700, device="cuda") for _ in range(3)]  # noqa: E731
    p, g = ones(), ones()
    t = lrb.TrainTensors(p, g, bits=bits)
    for call in calls(lrb, t, field):
        call()
    tensors = getattr(t, field)
    others = [z for z in (*p, *g, *t.m, *t.v) if z is not tensors[1]]
    before = [z.clone() for z in others]
    tensors[1].untyped_storage().resize_(size)
    for call in calls(lrb, t, field):
        with pytest.raises(ValueError):
            call()
    assert all(torch.equal(a, b) for a, b in zip(others, before))


def test_gradients_put_in_place_of_resized_ones(lrb):
    g = [torch.ones(700, device="cuda") for _ in range(3)]
    t = lrb.TrainTensors(None, g)
    g[2].untyped_storage().resize_(0)
    with pytest.raises(ValueError):
        lrb.lr_grad_norm(t)
    t.set_grads([torch.ones(700, device="cuda") for _ in range(3)])
    assert abs(float(lrb.lr_grad_norm(t)) - 2100 ** 0.5) < 1e-5


def test_tensors_that_share_a_storage_or_have_no_values(lrb):
    flat = torch.ones(1000, device="cuda")
    p = [flat[:300], torch.zeros(0, device="cuda"), flat[300:]]
    g = [torch.ones(300, device="cuda"), torch.zeros(0, device="cuda"), torch.ones(700, device="cuda")]
    t = lrb.TrainTensors(p, g)
    lrb.lr_adamw_update(t, 1, lr=0.1)
    p[1].untyped_storage().resize_(64)  # (an empty tensor has nothing to lose)
    lrb.lr_adamw_update(t, 2, lr=0.1)
    assert bool((flat < 1).all())
    flat.untyped_storage().resize_(0)
    with pytest.raises(ValueError):
        lrb.lr_adamw_update(t, 3, lr=0.1)


def test_steps_beyond_32_bits_either_way_are_refused(lrb):
    p = torch.ones(8, device="cuda")
    t = lrb.TrainTensors([p], [torch.ones(8, device="cuda")])
    for step in (-(1 << 32) + 5, -(1 << 31) - 1, 1 << 31, (1 << 32) + 5):
        with pytest.raises(ValueError):
            lrb.lr_adamw_update(t, step, lr=0.1)
    for step in (0, -1, -(1 << 31)):
        with pytest.raises(lrb.LrError):
            lrb.lr_adamw_update(t, step, lr=0.1)
    assert bool((p == 1).all())


@pytest.mark.parametrize("bits", (32, 8))
@pytest.mark.parametrize("eps", (1e-45, 1e-40, 2.0 ** -127, 2.0 ** -126))
def test_a_subnormal_eps_does_not_move_values_without_gradient(lrb, bits, eps):
    """0 / (0 + eps) is 0; beside a second moment above zero (its root is past 1e-23) such an eps is nothing."""
    g = torch.linspace(-1, 1, 601, device="cuda")
    g[::3] = 0
    p, q = torch.ones(601, device="cuda"), torch.ones(601, device="cuda")
    lrb.lr_adamw_update(lrb.TrainTensors([p], [g], bits=bits), 1, lr=0.1, eps=eps, weight_decay=0.5)
    lrb.lr_adamw_update(lrb.TrainTensors([q], [g], bits=bits), 1, lr=0.1, eps=0.0, weight_decay=0.5)
    still = g == 0
    assert bool((p[still] == np.float32(1 - float(np.float32(0.1)) * 0.5)).all())
    assert torch.equal(p[~still], q[~still])
