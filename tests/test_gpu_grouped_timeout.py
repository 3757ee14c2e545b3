"""A wait inside the tensor-core kernels of the grouped products and their gradients that runs out: the block that gave up leaves NaN in what it still had to write, everything else has the bits it
always has, and the call and those after it return.  In the checked build the first block of a launch can be told to leave out the first stage's completion, and waits to give up after 2^20
clocks, half a millisecond."""
import pytest
import torch

from paper_2202_05008_b200 import binding, build as B, grouped_linear, grouped_linear_backward, operators

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture()
def checked(monkeypatch):
    B.build_library(debug=True)
    lib = binding.load_library(debug=True)
    monkeypatch.setattr(operators, "load_library", lambda: lib)
    yield lib
    assert lib.evo_debug_grouped_waits(31, 0) == 0


def make(groups, rows_each, n_in, n_out, dtype, act):
    gen = torch.Generator(device="cuda").manual_seed(groups)
    rows = groups * rows_each
    x, dy = torch.randn(rows, n_in, generator=gen, device="cuda").to(dtype), torch.randn(rows, n_out, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(groups, n_out, n_in, generator=gen, device="cuda") / n_in ** 0.5).to(dtype)
    y = torch.tanh(torch.randn(rows, n_out, generator=gen, device="cuda")).to(dtype) if act == "tanh" else None
    return dy, x, w, torch.arange(groups + 1, device="cuda", dtype=torch.int32) * rows_each, y


def run_out(lib, call, may, must):
    """The call as ever, with the completion left out, and as ever again; `may` and `must`: what the first block may leave NaN in (of the result), and what it has to."""
    plain = call()
    assert plain.isfinite().all()
    assert lib.evo_debug_grouped_waits(20, 1) == 0
    got = call()
    torch.cuda.synchronize()
    assert lib.evo_debug_grouped_waits(31, 0) == 0
    again = call()
    assert torch.equal(again, plain)
    bad = got.isnan()
    assert bad[must].all() and not bad[~may].any() and torch.equal(got[~bad], plain[~bad])


def mask(t, *boxes):
    m = torch.zeros_like(t, dtype=torch.bool)
    for box in boxes:
        m[box] = True
    return m


# Blocks take tiles in order: the first has the first and, with 160 of them on 148 SMs, the 149th.  With more stages' worth of steps in the first tile than there are stages the wait runs out in it; a
# later one (450 rows are eight steps, of as many stages) in the 149th.
@pytest.mark.parametrize("dtype,act", [(BF16, "none"), (F16, "tanh"), (F32, "none")])
@pytest.mark.parametrize("groups,rows,n_in,n_out", [(160, 1600, 64, 64), (160, 450, 64, 64), (2, 24000, 256, 256)])
def test_gradients_of_weights(checked, dtype, act, groups, rows, n_in, n_out):
    dy, x, w, off, y = make(groups, rows, n_in, n_out, dtype, act)
    call = lambda: grouped_linear_backward(dy, x, w, off, y, activation=act, wanted=(False, True, False))[1]
    dw = call()
    if groups == 2:                                          # (two halves of the outputs by 74 splits by two sets: tiles 0 and 148 are the first half of each set's first split)
        may = mask(dw, (slice(None), slice(0, 128)))
        must = may
    else:
        may = mask(dw, 0, 148)
        must = mask(dw, 148) if rows < 512 and dtype == BF16 else may
    run_out(checked, call, may, must)


@pytest.mark.parametrize("dtype,act", [(BF16, "none"), (F16, "tanh"), (F32, "none")])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("groups,rows,n_in,n_out", [(160, 128, 2048, 64), (3, 256, 1600, 300)])
def test_products_and_gradients_of_rows(checked, dtype, act, back, groups, rows, n_in, n_out):
    # (the contracted index is the long one: of the gradient that of the outputs)
    dy, x, w, off, y = make(groups, rows, *((n_out, n_in) if back else (n_in, n_out)), dtype, act)
    call = (lambda: grouped_linear_backward(dy, x, w, off, y, activation=act, wanted=(True, False, False))[0]) if back else (lambda: grouped_linear(x, w, off, activation=act))
    out = call()
    if groups == 160:
        may = mask(out, slice(0, rows), slice(148 * rows, 149 * rows))
        must = may
    else:                                                    # (a tile is 128 outputs of up to 256 rows; which rows go together is the launch's)
        may = mask(out, (slice(0, rows), slice(0, 128)))
        must = mask(out, (slice(0, 16), slice(0, 128)))
    run_out(checked, call, may, must)
