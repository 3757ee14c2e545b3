"""What the Python calls of the matrix operators refuse before they touch a GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2202_05008_b200 import EvoError, operators


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
