"""Refusals of the matrix operators' C entry points, and the numbers their launches are planned with (no GPU needed: every check
comes before the first CUDA call, and the pointers are never used)."""
import ctypes as C

import pytest

from paper_2202_05008_b200 import build as B
from paper_2202_05008_b200.binding import Actions, Grouped, Matrices, Matrix, Muon, NewtonSchulz, load_library

OK, INVALID, WORKSPACE, UNSUPPORTED = 0, 1, 3, 7
FAR = 1 << 40          # addresses far apart: 1 FAR, 2 FAR, ...


@pytest.fixture(scope="module")
def lib():
    B.build_library()
    return load_library()


def _ns(steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7):
    return NewtonSchulz(C.sizeof(NewtonSchulz), steps, a, b, c, eps)


def _x(data=FAR, type_=0, batch=2, rows=300, cols=200, batch_stride=None, row_stride=None):
    row_stride = cols if row_stride is None else row_stride
    return Matrices(data, type_, batch, rows, cols, rows * row_stride if batch_stride is None else batch_stride, row_stride)


def test_workspace_of_small_matrices_is_nothing_and_grows_with_large_ones(lib):
    n = C.c_size_t(7)
    for rows, cols in ((1, 1), (128, 128), (64, 64), (256, 128), (12, 512), (8, 25)):
        assert lib.evo_orthogonalize_bytes(5, rows, cols, C.byref(n)) == OK and n.value == 0, (rows, cols)
    sizes = []
    for batch, rows, cols in ((1, 129, 129), (1, 300, 200), (1, 200, 300), (2, 300, 200)):
        assert lib.evo_orthogonalize_bytes(batch, rows, cols, C.byref(n)) == OK
        sizes.append(n.value)
        m, k = min(rows, cols), max(rows, cols)
        assert n.value >= batch * (2 * 4 * m * k + 2 * 4 * m * m)
    assert sizes[1] == sizes[2] and sizes[3] > sizes[2]
    for args in ((0, 4, 4), (1, 0, 4), (1, 4, 0), (1, (1 << 20) + 1, 4)):
        assert lib.evo_orthogonalize_bytes(*args, C.byref(n)) == INVALID
    assert lib.evo_orthogonalize_bytes(1, 4, 4, None) == INVALID
    # more tiles than 32 bits number
    assert lib.evo_orthogonalize_bytes(1 << 16, 1 << 20, 1 << 20, C.byref(n)) == UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=FAR + 2), dict(type_=3), dict(batch=0), dict(rows=0), dict(cols=0),
                                 dict(row_stride=199), dict(batch_stride=300 * 200 - 1), dict(rows=(1 << 20) + 1),
                                 dict(row_stride=1 << 33, batch_stride=1 << 42)])
def test_matrices_that_are_refused(lib, bad):
    good = _x(2 * FAR)
    assert lib.evo_orthogonalize(C.byref(_ns()), C.byref(_x(**bad)), C.byref(good), FAR * 8, 1 << 40, None) == INVALID
    assert lib.evo_orthogonalize(C.byref(_ns()), C.byref(good), C.byref(_x(**bad)), FAR * 8, 1 << 40, None) == INVALID


def test_orthogonalize_refuses_what_does_not_match_or_overlaps(lib):
    x, ws = _x(), FAR * 8

    def call(out, ns=None, work=ws, size=1 << 40):
        return lib.evo_orthogonalize(C.byref(ns if ns is not None else _ns()), C.byref(x), C.byref(out), work, size, None)
    for other in (dict(type_=1), dict(batch=1), dict(rows=299), dict(cols=199)):
        assert call(_x(2 * FAR, **other)) == INVALID, other
    assert call(_x(FAR + 4)) == INVALID                                     # overlaps, but is not x itself
    assert call(_x(FAR, row_stride=208)) == INVALID                         # x's memory, other strides
    assert call(_x(FAR + 4 * (2 * 300 * 200 - 1))) == INVALID               # the last element
    assert call(_x(2 * FAR), work=ws + 128) == INVALID and call(_x(2 * FAR), work=None) == INVALID
    assert call(_x(2 * FAR), size=4096) == WORKSPACE
    for ns in (_ns(steps=65), _ns(eps=-1.0), _ns(eps=float("nan")), _ns(eps=1e-38), _ns(eps=float("inf"))):
        assert call(_x(2 * FAR), ns=ns) == INVALID
    wrong = _ns()
    wrong.struct_size = 4
    assert call(_x(2 * FAR), ns=wrong) == INVALID
    # coefficients that do not keep [0, 1] small, or are no numbers
    for abc in ((3.4445, 4.7750, 2.0315), (70.0, 0.0, 0.0), (float("nan"), 0.0, 0.0), (2.0, float("inf"), 0.0), (1.9, 0.0, 0.0)):
        assert call(_x(2 * FAR), ns=_ns(10, *abc)) == UNSUPPORTED, abc
    assert lib.evo_orthogonalize(None, None, C.byref(x), ws, 1 << 40, None) == INVALID
    assert lib.evo_orthogonalize(None, C.byref(x), None, ws, 1 << 40, None) == INVALID


def _muon(**kw):
    m = Muon(C.sizeof(Muon), 0, 0.01, 0.95, 0.0, 0.9, 0.999, 1e-8, _ns())
    for k, v in kw.items():
        setattr(m, k, v)
    return m


def _list(*items):
    return (Matrix * max(1, len(items)))(*(Matrix(*x) for x in items)), len(items)


def test_muon_lists(lib):
    n = C.c_size_t()
    ok, k = _list((0, 28, 128), (3712, 128, 128), (20224, 8, 128))
    assert lib.evo_muon_bytes(ok, k, 21256, C.byref(n)) == OK and n.value == 0
    assert lib.evo_muon_bytes(None, 0, 10, C.byref(n)) == OK and n.value == 0
    large, k = _list((4, 300, 300))
    assert lib.evo_muon_bytes(large, k, 4 + 90000, C.byref(n)) == OK and n.value > 0
    many, k = _list(*((i * 90000, 300, 300) for i in range(70)))               # more than a launch lists
    assert lib.evo_muon_bytes(many, k, 70 * 90000, C.byref(n)) == OK
    for items, dim in ((((0, 4, 4), (15, 4, 4)), 100), (((20, 4, 4), (0, 4, 4)), 100), (((90, 4, 4),), 100), (((0, 0, 4),), 100),
                       (((0, 4, 0),), 100), (((101, 1, 1),), 100), (((0, 1 << 20, 1 << 20),), 100), ((((1 << 64) - 1, 2, 2),), 100)):
        bad, k = _list(*items)
        assert lib.evo_muon_bytes(bad, k, dim, C.byref(n)) == INVALID, items
    assert lib.evo_muon_bytes(None, 1, 100, C.byref(n)) == INVALID
    assert lib.evo_muon_bytes(ok, 1, 21256, None) == INVALID


def test_muon_step_refusals(lib):
    items, n = _list((0, 300, 300))
    apart = [FAR * i for i in range(1, 8)]

    def call(cfg=None, ptrs=apart, step=1, dim=90010, work=FAR * 9, size=1 << 40):
        return lib.evo_muon_step(C.byref(cfg if cfg is not None else _muon()), items, n, dim, step, *ptrs, work, size, None)
    for kw in (dict(lr=float("inf")), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-1.0), dict(beta1=1.0), dict(beta2=1.0),
               dict(adam_eps=-1.0), dict(adam_eps=float("nan")), dict(struct_size=8), dict(newton_schulz=_ns(steps=100))):
        assert call(_muon(**kw)) == INVALID, kw
    assert call(_muon(newton_schulz=_ns(8, 9.0, 9.0, 9.0))) == UNSUPPORTED
    assert call(step=0) == INVALID and call(dim=0) == INVALID and call(dim=89999) == INVALID
    for i in range(7):
        assert call(ptrs=[None if j == i else p for j, p in enumerate(apart)]) == INVALID
        assert call(ptrs=[p + 2 if j == i else p for j, p in enumerate(apart)]) == INVALID
    # an output over another vector, or beside its own input
    for out, where in ((4, 1), (4, 3), (5, 0), (6, 4), (5, 3)):
        assert call(ptrs=[apart[where] if j == out else p for j, p in enumerate(apart)]) == INVALID, (out, where)
    assert call(ptrs=apart[:4] + [apart[0] + 4] + apart[5:]) == INVALID
    assert call(work=None) == INVALID and call(work=FAR * 9 + 8) == INVALID and call(size=1024) == WORKSPACE
    assert lib.evo_muon_step(None, items, n, 90010, 1, *apart, FAR * 9, 1 << 40, None) == INVALID


def _grouped(**kw):
    p = Grouped(C.sizeof(Grouped), 0, 4, 10, 20, 1, 1.0, 0, 100, FAR, 10, 2 * FAR, 10, 200, 3 * FAR, 20, 4 * FAR, 5 * FAR, 20)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad", [dict(struct_size=8), dict(type=3), dict(groups=0), dict(n_in=0), dict(n_out=0), dict(n_in=(1 << 20) + 1), dict(activation=3),
                                 dict(scale=float("inf")), dict(offsets_64=2), dict(rows=1 << 41), dict(d_x=None), dict(d_weight=None), dict(d_y=None),
                                 dict(d_offsets=None), dict(d_x=FAR + 2), dict(d_bias=3 * FAR + 1), dict(d_offsets=4 * FAR + 2),
                                 dict(offsets_64=1, d_offsets=4 * FAR + 4), dict(ld_x=9), dict(ld_y=19), dict(ld_weight=9), dict(weight_stride=1 << 41),
                                 dict(d_y=FAR + 4), dict(d_y=2 * FAR - 4), dict(d_y=3 * FAR), dict(d_y=4 * FAR), dict(groups=1 << 31)])
def test_grouped_refusals(lib, bad):
    assert lib.evo_grouped_linear(C.byref(_grouped(**bad)), FAR * 32, 1 << 40, None) == INVALID


def test_grouped_without_rows_is_nothing_to_do(lib):
    assert lib.evo_grouped_linear(C.byref(_grouped(rows=0, d_x=None, d_y=None)), None, 0, None) == OK
    assert lib.evo_grouped_linear(None, None, 0, None) == INVALID
    assert lib.evo_grouped_linear(C.byref(_grouped(groups=(1 << 31) - 1, n_out=1 << 20, ld_weight=12, weight_stride=0, ld_y=1 << 20, d_y=FAR * 64)), None, 0, None) in (INVALID, UNSUPPORTED)


def test_grouped_workspace(lib):
    n = C.c_size_t()

    def need(**kw):
        assert lib.evo_grouped_linear_bytes(C.byref(_grouped(**kw)), C.byref(n)) == OK, kw
        return n.value
    assert need() == 0 and need(rows=0) == 0                                    # few rows a group
    many = dict(rows=4000, n_in=48, ld_x=48, ld_weight=48, weight_stride=960, n_out=20)
    assert need(type=1, **many) == 0                                            # aligned 16-bit rows are taken as they lie
    assert need(type=1, **dict(many, ld_x=49)) >= 2 * 48 * (4 * 20 + 4000)
    assert need(type=0, **many) >= 3 * 2 * 48 * (4 * 20 + 4000)
    p = _grouped(**many)
    assert lib.evo_grouped_linear(C.byref(p), FAR * 32, n.value - 1, None) == WORKSPACE
    assert lib.evo_grouped_linear(C.byref(p), FAR * 32 + 16, 1 << 40, None) == INVALID
    assert lib.evo_grouped_linear(C.byref(p), None, 1 << 40, None) == INVALID
    assert lib.evo_grouped_linear_bytes(C.byref(p), None) == INVALID


def _actions(sizes=(5, 16, 16, 1), **kw):
    p = Actions(C.sizeof(Actions), 4, len(sizes) - 1, (C.c_uint32 * 9)(*sizes), 1.0, 0, 100, FAR, 416, 2 * FAR, sizes[0], 3 * FAR, 4 * FAR, sizes[-1])
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_actions_refusals(lib):
    n = C.c_size_t(9)
    assert lib.evo_mlp_actions_bytes(C.byref(_actions()), C.byref(n)) == OK and n.value == 0
    wide = _actions((40, 700, 700, 3), ld_theta=700 * 41 + 700 * 701 + 3 * 701 + 1)
    wide.ld_theta = (wide.ld_theta + 3) // 4 * 4
    assert lib.evo_mlp_actions_bytes(C.byref(wide), C.byref(n)) == OK and n.value == 2 * 100 * 700 * 4
    assert lib.evo_mlp_actions(C.byref(wide), FAR * 8, n.value - 1, None) == WORKSPACE
    assert lib.evo_mlp_actions(C.byref(wide), None, n.value, None) == INVALID
    for bad in (dict(struct_size=4), dict(members=0), dict(n_layers=0), dict(n_layers=9), dict(ld_theta=384), dict(ld_theta=387),
                dict(action_scale=float("nan")), dict(offsets_64=7), dict(rows=1 << 41)):
        assert lib.evo_mlp_actions_bytes(C.byref(_actions(**bad)), C.byref(n)) == INVALID, bad
    for bad in (dict(d_theta=None), dict(d_theta=FAR + 8), dict(d_observations=None), dict(d_observations=2 * FAR + 2), dict(d_offsets=None),
                dict(d_actions=None), dict(ld_observations=4), dict(d_actions=FAR), dict(d_actions=2 * FAR + 4), dict(d_actions=3 * FAR)):
        assert lib.evo_mlp_actions(C.byref(_actions(**bad)), None, 0, None) == INVALID, bad
    assert lib.evo_mlp_actions(C.byref(_actions(rows=0, d_actions=None)), None, 0, None) == OK
    assert lib.evo_mlp_actions_bytes(C.byref(_actions((5, 0, 1))), C.byref(n)) == INVALID


def test_a_configuration_without_the_fields_of_muon_is_still_taken(lib):
    from paper_2202_05008_b200 import workloads as W
    from paper_2202_05008_b200.binding import EvoConfig, make_config
    first = EvoConfig.muon_momentum.offset
    a, b = C.c_size_t(), C.c_size_t()
    cfg = make_config(W.CFG4)
    assert cfg.struct_size == C.sizeof(EvoConfig) and lib.evo_workspace_bytes(C.byref(cfg), C.byref(a)) == OK
    cfg.struct_size, cfg.muon_momentum, cfg.muon_steps = first, 7.0, 1000        # what lies behind it is not read
    assert lib.evo_workspace_bytes(C.byref(cfg), C.byref(b)) == OK and a.value == b.value
    cfg.struct_size = first + 4
    assert lib.evo_workspace_bytes(C.byref(cfg), C.byref(b)) == INVALID


def test_muon_solvers_have_their_workspace(lib):
    from paper_2202_05008_b200 import workloads as W
    from paper_2202_05008_b200.binding import make_config
    n, m = C.c_size_t(), C.c_size_t()
    for w, large in ((W.CFG4, False), (W.CFG3, False), (W.SEQ2SEQ, False),
                     (W.Workload("x", 4, 300 * 201 + 201 * 5, 1, policy_kind=W.POLICY_MLP, layer_sizes=(200, 300, 3)), True)):
        w = w.with_(param_dim=W.mlp_param_count(w.layer_sizes)) if w.name == "x" else w
        assert lib.evo_workspace_bytes(C.byref(make_config(w)), C.byref(n)) == OK
        assert lib.evo_workspace_bytes(C.byref(make_config(w.with_(optimizer=W.OPT_MUON))), C.byref(m)) == OK
        assert (m.value > n.value) == large, w.name
    assert lib.evo_workspace_bytes(C.byref(make_config(W.CFG5.with_(optimizer=W.OPT_MUON))), C.byref(m)) == UNSUPPORTED


def test_policies_that_go_layer_by_layer_need_room_for_hidden_rows(lib):
    n = C.c_size_t()
    sizes, ld = (28, 128, 128, 8), 21280
    for members, rows, layers in ((4096, 16384, True), (100, 400, False), (4096, 40000, False)):
        p = _actions(sizes, members=members, rows=rows, ld_theta=ld)
        assert lib.evo_mlp_actions_bytes(C.byref(p), C.byref(n)) == OK
        assert n.value == (2 * rows * 128 * 4 if layers else 0), (members, rows)
