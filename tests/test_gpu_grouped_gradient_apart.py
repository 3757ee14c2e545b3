"""The gradients of products one by one, and for offsets that are none: against the formulas in 64 bits, bit for bit where the same kernel runs, and with every output
inside a wider room."""
import pytest
import torch

from paper_2202_05008_b200 import grouped_linear_backward
from test_gpu_grouped_gradient import close, exact, make

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("act", ["none", "tanh", "relu"])
@pytest.mark.parametrize("lengths,n_in,n_out", [([3, 9, 0], 200, 136), ([150, 260, 90], 200, 136), ([400], 130, 70), ([2] * 30, 300, 7), ([64] * 20, 131, 264)])
def test_each_gradient_by_itself(dtype, act, lengths, n_in, n_out):
    dy, x, w, off, y = make(len(lengths), lengths, n_in, n_out, dtype, act, 1.5)
    together = grouped_linear_backward(dy, x, w, off, y, activation=act, scale=1.5)
    want = exact(dy, x, w, off, y, act, 1.5)
    for i in range(3):
        wanted = tuple(k == i for k in range(3))
        alone = grouped_linear_backward(dy, x if i == 1 else None, w, off, y, activation=act, scale=1.5, wanted=wanted)
        assert [a is not None for a in alone] == list(wanted)
        for got in (alone[i], together[i]):
            close(got, *want[i], n_out if i == 0 else max(lengths))
        if i < 2:                                            # (db alone is another kernel's, with other splits)
            assert torch.equal(alone[i], together[i])


# few rows; both on the tensor cores, as they lie and laid out; rows split; a policy's action layer
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("act", ["none", "tanh"])
@pytest.mark.parametrize("rows,groups,n_in,n_out", [(100, 4, 72, 40), (1200, 4, 136, 264), (1200, 4, 131, 101), (3000, 2, 40, 24), (200, 4, 300, 7), (40, 4, 300, 1031)])
def test_offsets_that_fall_or_leave_the_rows_touch_nothing_outside_of_any_output(dtype, act, rows, groups, n_in, n_out):
    dy, x, w, _, y = make(groups, [rows // groups] * groups, n_in, n_out, dtype, act)
    pitch = n_out * n_in + n_out + 24
    for wide, edges in ((False, [-5, rows // 2, 30, 2 * rows, 100]), (False, [rows, 0, rows // 2, 10, rows]), (False, [2 ** 31 - 1] * 5), (False, [-2 ** 31] * 5), (True, [2 ** 62, -2 ** 62, 5, rows, 3]),
                        (True, [0, rows, 0, rows, 0])):
        off = torch.tensor(edges[:groups + 1], dtype=torch.int64 if wide else torch.int32, device="cuda")
        rooms = [torch.full((rows + 20, n_in + 16), 5.0, dtype=dtype, device="cuda"), torch.full((groups + 2, pitch), 5.0, dtype=dtype, device="cuda")]
        dx, inner = rooms[0][10:-10, 8:-8], rooms[1][1:-1]
        dw, db = inner[:, 8:8 + n_out * n_in].unflatten(1, (n_out, n_in)), inner[:, 16 + n_out * n_in:16 + n_out * n_in + n_out]
        grouped_linear_backward(dy, x, w, off, y, activation=act, out=(dx, dw, db))
        torch.cuda.synchronize()
        outside = [torch.ones_like(room, dtype=torch.bool) for room in rooms]
        outside[0][10:-10, 8:-8] = False
        outside[1][1:-1, 8:8 + n_out * n_in] = False
        outside[1][1:-1, 16 + n_out * n_in:16 + n_out * n_in + n_out] = False
        assert all((room[m] == 5).all() for room, m in zip(rooms, outside))
        assert x.isfinite().all() and dy.isfinite().all() and w.isfinite().all()
