"""Sizes whose products leave 64 bits are refused, and ranges that only touch are not overlaps (no GPU needed: the checks come before the
first CUDA call, and the pointers are never used)."""
import ctypes as C

import pytest

from test_matrix_ops import FAR, INVALID, OK, UNSUPPORTED, WORKSPACE, _actions, _grouped, _ns, _x, lib  # noqa: F401

MOST = 1 << 40
# weights, biases and rows far behind y, below which nothing of the small case lies
LOW = dict(d_x=FAR * 2, d_weight=FAR * 3, d_bias=FAR * 4, d_offsets=FAR * 5, d_y=FAR)


@pytest.mark.parametrize("kw", [dict(rows=MOST, ld_x=MOST, ld_y=20), dict(rows=MOST, ld_y=MOST), dict(rows=1 << 25, ld_x=MOST - 1, ld_y=MOST - 1),
                                dict(groups=(1 << 31) - 1, weight_stride=MOST), dict(groups=1 << 30, bias_stride=MOST), dict(n_out=1 << 20, ld_weight=MOST, ld_y=1 << 20),
                                dict(groups=1 << 24, weight_stride=MOST, d_y=FAR + (1 << 62)), dict(groups=1 << 22, weight_stride=MOST - 1),
                                dict(type=1, rows=MOST, ld_x=1 << 23, ld_y=1 << 23)])
def test_grouped_sizes_beyond_64_bits(lib, kw):                       # noqa: F811
    p = _grouped(**dict(LOW, **kw))
    assert lib.evo_grouped_linear(C.byref(p), FAR * 64, 1 << 62, None) == INVALID


@pytest.mark.parametrize("kw", [dict(rows=MOST, ld_observations=MOST, ld_actions=1), dict(rows=MOST, ld_actions=MOST), dict(members=(1 << 31) - 1, ld_theta=MOST),
                                dict(members=1 << 24, ld_theta=MOST), dict(rows=1 << 24, ld_observations=MOST)])
def test_policy_sizes_beyond_64_bits(lib, kw):                        # noqa: F811
    p = _actions(**dict(dict(d_theta=FAR * 2, d_observations=FAR * 3, d_offsets=FAR * 5, d_actions=FAR), **kw))
    assert lib.evo_mlp_actions(C.byref(p), FAR * 64, 1 << 62, None) == INVALID


@pytest.mark.parametrize("kw", [dict(batch=(1 << 32) - 1, batch_stride=MOST), dict(batch=1 << 24, batch_stride=MOST)])
def test_batches_beyond_64_bits(lib, kw):                             # noqa: F811
    for x, out in ((_x(FAR * 2, rows=4, cols=4, **kw), _x(FAR, rows=4, cols=4, **kw)), (_x(FAR, rows=4, cols=4, **kw), _x(FAR * 2, rows=4, cols=4, **kw))):
        assert lib.evo_orthogonalize(C.byref(_ns()), C.byref(x), C.byref(out), FAR * 64, 1 << 62, None) == INVALID


def test_actions_behind_the_last_members_parameters_do_not_overlap(lib):   # noqa: F811
    """Parameter rows need no padding behind the last one: what begins there is another array.  (Wide layers: the workspace is asked for last.)"""
    sizes = (40, 700, 700, 3)
    dim = 40 * 700 + 700 + 700 * 700 + 700 + 3 * 700 + 3
    ld = (dim + 31) // 32 * 32
    end = FAR + 4 * (3 * ld + dim)
    for at, code in ((end, WORKSPACE), (end - 4, INVALID), (FAR - 4 * 300, WORKSPACE), (FAR - 4 * 299, INVALID)):
        p = _actions(sizes, ld_theta=ld, d_theta=FAR, d_observations=2 * FAR, d_offsets=3 * FAR, d_actions=at, rows=100, ld_actions=3)
        assert lib.evo_mlp_actions(C.byref(p), FAR * 64, 256, None) == code, (at, code)



def test_more_small_matrices_than_blocks_of_a_launch(lib):             # noqa: F811
    n = C.c_size_t()
    for batch, rows, cols in ((1 << 31, 1, 1), (1 << 28, 4, 8000), (1 << 29, 40, 300), ((1 << 32) - 1, 3, 2)):
        assert lib.evo_orthogonalize_bytes(batch, rows, cols, C.byref(n)) == UNSUPPORTED, (batch, rows, cols)
        x, out = _x(FAR, type_=1, batch=batch, rows=rows, cols=cols), _x(1 << 55, type_=1, batch=batch, rows=rows, cols=cols)
        assert lib.evo_orthogonalize(C.byref(_ns()), C.byref(x), C.byref(out), None, 0, None) == UNSUPPORTED
    assert lib.evo_orthogonalize_bytes((1 << 31) - 1, 1, 1, C.byref(n)) == OK and n.value == 0
