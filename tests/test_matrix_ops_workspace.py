"""Sizes of workspaces asked for before the buffers exist (no GPU needed)."""
import ctypes as C

import pytest

from test_matrix_ops import FAR, INVALID, OK, WORKSPACE, _grouped, lib  # noqa: F401


@pytest.mark.parametrize("type_,rows,pitch", [(1, 4000, 48), (2, 4000, 48), (1, 4000, 49), (0, 4000, 48), (1, 12, 48), (0, 12, 48)])
def test_without_addresses_the_size_is_enough_for_any(lib, type_, rows, pitch):       # noqa: F811
    kw = dict(type=type_, rows=rows, n_in=48, ld_x=pitch, ld_weight=48, weight_stride=960, n_out=20, d_y=FAR * 16)
    n = C.c_size_t()

    def need(**more):
        assert lib.evo_grouped_linear_bytes(C.byref(_grouped(**dict(kw, **more))), C.byref(n)) == OK
        return n.value
    size = 4 if type_ == 0 else 2
    most = max(need(d_x=FAR + a, d_weight=2 * FAR + b) for a in (0, size, 8) for b in (0, size))
    for missing in (dict(d_x=None), dict(d_weight=None), dict(d_x=None, d_weight=None), dict(d_x=None, d_weight=None, d_y=None, d_bias=None, d_offsets=None)):
        assert need(**missing) >= most, missing
    # a call whose rows lie at an odd address takes what the size without addresses said, and no less than its own
    if most:
        without = need(d_x=None, d_weight=None)
        p = _grouped(**dict(kw, d_x=FAR + size, d_offsets=FAR * 8 + 4))
        assert lib.evo_grouped_linear(C.byref(p), FAR * 32, most - 1, None) == WORKSPACE and without >= most
    assert lib.evo_grouped_linear(C.byref(_grouped(**dict(kw, d_x=None))), FAR * 32, 1 << 40, None) == INVALID


def test_rows_a_group_from_which_operands_are_laid_out(lib):          # noqa: F811
    n = C.c_size_t()

    def need(type_, rows, n_in, groups=10):
        p = _grouped(type=type_, rows=rows, groups=groups, n_in=n_in, ld_x=n_in, ld_weight=n_in, n_out=20, weight_stride=20 * n_in + 1)
        assert lib.evo_grouped_linear_bytes(C.byref(p), C.byref(n)) == OK
        return n.value
    for type_, n_in, least in ((0, 1000, 332), (0, 100, 467), (0, 10, 1817), (1, 1000, 95), (2, 1000, 95), (1, 100, 230), (1, 10, 1580)):
        assert need(type_, least - 1, n_in) == 0 and need(type_, least, n_in) > 0, (type_, n_in)
