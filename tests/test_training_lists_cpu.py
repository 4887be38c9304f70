"""Lists of an optimiser step that do not fit each other: refused before anything is looked up on a device."""

import pytest

from paper_2306_11268_amd import binding as lb

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("params,grads", [(0, 1), (1, 0), (2, 1), (1, 2)])
def test_parameters_and_gradients_of_different_number(params, grads):
    with pytest.raises(ValueError, match=f"{params} parameters for {grads} gradients"):
        lb.TrainTensors([torch.zeros(4)] * params, [torch.zeros(4)] * grads)
