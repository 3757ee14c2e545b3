"""Dual tensors of forward mode are refused by every operator: what they would return has no tangent."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2202_05008_b200 import EvoError, build as B, operators


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build_library()


X, PLACE, W = torch.zeros(4, 3), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
OFF, WEIGHT, ROW = torch.tensor([0, 2, 4]), torch.zeros(2, 3, 3), torch.zeros(4)
CALLS = {
    "orthogonalize": lambda g: operators.orthogonalize(g(X)),
    "muon_step": lambda g: operators.muon_step(ROW, ROW, ROW, g(ROW), [], 1, lr=0.1),
    "grouped_linear": lambda g: operators.grouped_linear(X, g(WEIGHT), OFF),
    "grouped_linear of a bias": lambda g: operators.grouped_linear(X, WEIGHT, OFF, g(torch.zeros(2, 3))),
    "mlp_actions": lambda g: operators.mlp_actions(g(torch.zeros(2, 12)), (3, 3), X, OFF),
    "take_rows": lambda g: operators.take_rows(g(X), PLACE),
    "take_rows with weights": lambda g: operators.take_rows(X, PLACE, g(W)),
    "combine_rows": lambda g: operators.combine_rows(g(X), PLACE, W),
    "combine_rows_backward": lambda g: operators.combine_rows_backward(X, X, PLACE, g(W)),
    "grouped_linear_backward": lambda g: operators.grouped_linear_backward(g(X), X, WEIGHT, OFF),
    "grouped_linear_backward of y": lambda g: operators.grouped_linear_backward(X, X, WEIGHT, OFF, g(X), activation="tanh"),
    "policy_loss": lambda g: operators.policy_loss(g(X), PLACE[:, 0], ROW, ROW),
    "policy_loss of weights": lambda g: operators.policy_loss(X, PLACE[:, 0], ROW, ROW, weights=g(ROW)),
}


@pytest.mark.parametrize("call", CALLS, ids=lambda name: name.replace(" ", "-"))
def test_a_dual_tensor_is_refused(call):
    with forward_ad.dual_level():
        for mode in (torch.enable_grad, torch.no_grad):
            with mode(), pytest.raises(EvoError) as e:
                CALLS[call](lambda t: forward_ad.make_dual(t.clone(), torch.ones_like(t)))
            assert e.value.code == 1 and "tangent" in str(e.value)
        with pytest.raises(EvoError) as e:                   # (not on a GPU, which is the next thing that is looked at)
            CALLS[call](lambda t: t)
        assert "tangent" not in str(e.value)


def test_a_derivative_by_forward_mode_is_refused():
    with pytest.raises(EvoError) as e:
        torch.func.jvp(lambda x: operators.take_rows(x, PLACE), (X,), (X,))
    assert "tangent" in str(e.value)
