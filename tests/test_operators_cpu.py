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
