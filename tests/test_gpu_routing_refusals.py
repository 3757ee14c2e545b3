"""Tensors of another number of dimensions are refused like any others that do not match."""
import pytest
import torch

from paper_2202_05008_b200 import EvoError, combine_rows, combine_rows_backward, grouped_linear_backward, policy_loss, route_rows, take_rows

pytestmark = pytest.mark.gpu


def test_tensors_without_rows_are_refused():
    x, place, w = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    one, row, off, weight = torch.zeros((), device="cuda"), torch.zeros(4, device="cuda"), torch.tensor([0, 4], device="cuda"), torch.zeros(1, 8, 8, device="cuda")
    for call in (lambda: take_rows(one, place), lambda: take_rows(row, place), lambda: take_rows(x, place[0, 0]), lambda: take_rows(x, place, one), lambda: take_rows(x, place, out=one),
                 lambda: take_rows(x, place, out=row), lambda: take_rows(x, place, out=x[None]), lambda: combine_rows(one, place), lambda: combine_rows(x, place[0, 0]),
                 lambda: combine_rows(x, place, out=one), lambda: combine_rows_backward(one, x, place, w), lambda: combine_rows_backward(x, one, place, w),
                 lambda: combine_rows_backward(x, x, place, one), lambda: combine_rows_backward(x, x, place, w, out=one), lambda: route_rows(place[0, 0], 3),
                 lambda: grouped_linear_backward(one, x, weight, off), lambda: grouped_linear_backward(x, one, weight, off), lambda: grouped_linear_backward(x, x, one, off),
                 lambda: grouped_linear_backward(x, x, weight, one), lambda: grouped_linear_backward(x, x, weight, off, one), lambda: grouped_linear_backward(x, x, weight, off, out=(one, None, None)),
                 lambda: grouped_linear_backward(x, x, weight, off, out=(None, one, None)), lambda: grouped_linear_backward(x, x, weight, off, out=(None, None, one)),
                 lambda: policy_loss(one, place[:, 0], row, row), lambda: policy_loss(x, place[0, 0], row, row), lambda: policy_loss(x, place[:, 0].contiguous(), one, row),
                 lambda: policy_loss(x, place[:, 0].contiguous(), row, row, weights=one), lambda: policy_loss(x, place[:, 0].contiguous(), row, row, out=one)):
        with pytest.raises(EvoError) as e:
            call()
        assert e.value.code == 1
