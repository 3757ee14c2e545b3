"""What the Python calls of the matrix operators refuse before they touch a GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2202_05008_b200 import EvoError, build as B, operators


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build_library()


def test_a_stream_of_another_device_is_refused():
    for index in (0, 1):
        stream = SimpleNamespace(device=torch.device("cuda", 1 - index))
        with pytest.raises(EvoError) as e:
            operators._On(torch.device("cuda", index), stream, "orthogonalize").__enter__()
        assert e.value.code == 1 and "stream" in str(e.value)


@pytest.mark.parametrize("coefficients,eps", [((1e-50, 0.0, 0.0), 1e-7), ((0.0, -1e-46, 0.0), 1e-7), (operators.COEFFICIENTS, 1e-50), (operators.COEFFICIENTS, 1e-46),
                                              (operators.COEFFICIENTS, float("nan")), ((0.0, 0.0, 0.0), 1e-7)])
def test_numbers_that_are_zero_in_fp32_do_not_select_the_defaults(coefficients, eps):
    with pytest.raises(EvoError):
        operators._newton_schulz(5, coefficients, eps, "orthogonalize")
    assert operators._newton_schulz(5, (1e-30, 0.0, 0.0), 1e-30, "orthogonalize").steps == 5


def test_arguments_whose_gradient_would_be_lost_are_refused():
    x, m, theta = torch.zeros(4, 4), torch.zeros(16), torch.zeros(2, 24)
    off = torch.tensor([0, 2, 4])
    calls = [lambda g: operators.orthogonalize(g(x)), lambda g: operators.orthogonalize(x, out=g(x)),
             lambda g: operators.muon_step(m, m, m, g(m), [], 1, lr=0.1), lambda g: operators.muon_step(m, m, m, m, [], 1, lr=0.1, out=(g(m), m, m)),
             lambda g: operators.grouped_linear(g(x), torch.zeros(2, 4, 4), off), lambda g: operators.grouped_linear(x, g(torch.zeros(2, 4, 4)), off),
             lambda g: operators.grouped_linear(x, torch.zeros(2, 4, 4), off, g(torch.zeros(2, 4))),
             lambda g: operators.mlp_actions(g(theta), (4, 4), x, off), lambda g: operators.mlp_actions(theta, (4, 4), g(x), off)]

    def wanting(t):
        return t.clone().requires_grad_()
    for call in calls:
        with pytest.raises(EvoError) as e:
            call(wanting)
        assert e.value.code == 1 and "backward" in str(e.value)
        with torch.no_grad(), pytest.raises(EvoError) as e:         # (these are not on a GPU, which is the next thing that is looked at)
            call(wanting)
        assert "backward" not in str(e.value)
