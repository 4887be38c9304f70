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
