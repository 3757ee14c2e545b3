"""Products grouped by member and the MLP policy's actions for ragged rows, against the same formulas in 64 bits.

Tolerances, relative to S = sum of |x_k w_k| (+ |b|): fp32 operands are two tf32 numbers each, off by 2^-21 at worst (two operands), the product
of the low parts (2^-22) is left out, the tensor core cuts each of the 8 sums of a chunk of 64 (2^-23 each), and chunks are added
in fp32 (2^-24 each).  Products of 16-bit numbers are exact and the tensor core cuts a sum every 8 or 16 of the contracted index.  The
result is rounded to its type; tanh adds two units of fp32 and never makes an error larger."""
import ctypes as C
import math

import pytest
import torch

from paper_2202_05008_b200 import EvoError, Solver, grouped_linear, mlp_actions, workloads as W

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def slack(dtype, k):
    return 2.25 * 2.0 ** -20 + k / 64 * 2.0 ** -24 if dtype == F32 else (k / 8 + 2) * 2.0 ** -23


def exact(x, weight, offsets, bias, act="none", scale=1.0):
    """(result, S); rows outside all groups are NaN."""
    y = torch.full((x.shape[0], weight.shape[1]), float("nan"), dtype=torch.float64, device=x.device)
    s = torch.zeros_like(y)
    edges = offsets.tolist()
    for g, (p, q) in enumerate(zip(edges[:-1], edges[1:])):
        if q > p:
            w, b = weight[g].double(), 0.0 if bias is None else bias[g].double()
            y[p:q] = x[p:q].double() @ w.t() + b
            s[p:q] = x[p:q].double().abs() @ w.abs().t() + (0.0 if bias is None else b.abs())
    y = torch.tanh(y) if act == "tanh" else y.relu() if act == "relu" else y
    return scale * y, abs(scale) * s


def check(got, x, weight, offsets, bias=None, act="none", scale=1.0):
    want, s = exact(x, weight, offsets, bias, act, scale)
    inside = ~want.isnan()
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    bound = slack(x.dtype, x.shape[1]) * s + (half + 2.0 ** -22) * (want.abs() + slack(x.dtype, x.shape[1]) * s) + tiny
    err = (got.double() - want).abs()
    assert (err[inside] <= bound[inside]).all(), float((err / bound)[inside].max())


def make(groups, lengths, n_in, n_out, dtype, seed=0, lead=0, tail=0, wide=False):
    gen = torch.Generator(device="cuda").manual_seed(seed + n_in * 31 + n_out)
    rows = lead + sum(lengths) + tail
    x = torch.randn(rows, n_in, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(groups, n_out, n_in, generator=gen, device="cuda") / math.sqrt(n_in)).to(dtype)
    b = torch.randn(groups, n_out, generator=gen, device="cuda").to(dtype)
    edges = [lead]
    for n in lengths:
        edges.append(edges[-1] + n)
    return x, w, b, torch.tensor(edges, dtype=torch.int64 if wide else torch.int32, device="cuda")


SHAPES = [
    (1, [1], 1, 1), (3, [1, 0, 2], 5, 3), (4, [0, 0, 0, 7], 16, 16), (2, [8, 9], 17, 33), (5, [3, 40, 0, 1, 33], 28, 128),
    (3, [31, 32, 65], 64, 64), (2, [100, 1], 130, 70), (2, [5, 300], 1000, 90), (1, [17], 2048, 40), (6, [1] * 6, 512, 260),
    (70, [i % 5 for i in range(70)], 24, 40), (3, [129, 257, 40], 264, 264), (2, [513, 16], 72, 512),
]


@pytest.mark.parametrize("groups,lengths,n_in,n_out", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sizes_and_types(groups, lengths, n_in, n_out, dtype):
    x, w, b, off = make(groups, lengths, n_in, n_out, dtype, wide=n_in % 2 == 0)
    check(grouped_linear(x, w, off), x, w, off)
    check(grouped_linear(x, w, off, b, activation="tanh", scale=2.5), x, w, off, b, "tanh", 2.5)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n_in,n_out", [(72, 130), (648, 500), (264, 1200), (1032, 1500)])      # tiles of up to 64, 128, 192 and 256 rows
def test_groups_of_every_part_of_a_tile(n_in, n_out, dtype):
    x, w, b, off = make(18, [1, 31, 33, 0, 63, 65, 97, 129, 161, 191, 193, 225, 255, 257, 300, 511, 513, 7], n_in, n_out, dtype, tail=3)
    y = torch.full((x.shape[0], n_out), 7.0, dtype=dtype, device="cuda")
    check(grouped_linear(x, w, off, b, activation="relu", scale=0.5, out=y), x, w, off, b, "relu", 0.5)
    assert (y[-3:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_in,n_out,shift", [(64, 48, 0), (64, 48, 1), (61, 48, 0), (256, 136, 3), (256, 136, 8)])
def test_strides_alignment_and_rows_outside_of_the_groups(dtype, n_in, n_out, shift):
    lengths = [3, 0, 20, 90, 1]
    x, w, b, off = make(5, lengths, n_in, n_out, dtype, lead=2, tail=4)
    # a layer of a wider parameter row, observations and results inside wider rows
    theta = torch.full((5, shift + n_out * n_in + n_out + 24), float("nan"), dtype=dtype, device="cuda")
    theta[:, shift:shift + n_out * n_in] = w.flatten(1)
    theta[:, shift + n_out * n_in:shift + n_out * n_in + n_out] = b
    wv = theta[:, shift:shift + n_out * n_in].unflatten(1, (n_out, n_in))
    bv = theta[:, shift + n_out * n_in:shift + n_out * n_in + n_out]
    xs = torch.full((x.shape[0], n_in + 13), float("nan"), dtype=dtype, device="cuda")
    xs[:, 8:8 + n_in] = x
    ys = torch.full((x.shape[0], n_out + 9), 7.0, dtype=dtype, device="cuda")
    xv, yv = xs[:, 8:8 + n_in], ys[:, 5:5 + n_out]
    xs[:2] = float("nan")                                       # rows that no group has
    assert grouped_linear(xv, wv, off, bv, activation="relu", out=yv) is yv
    check(yv, x, w, off, b, "relu")
    assert (ys[:, :5] == 7).all() and (ys[:, 5 + n_out:] == 7).all() and (ys[:2] == 7).all() and (ys[-4:] == 7).all()
    # weights shared by all groups, and a pitch between weight rows
    shared = w[:1].expand(5, n_out, n_in)
    check(grouped_linear(x, shared, off, b), x, shared, off, b)
    pitch = torch.full((5, n_out, n_in + 8), float("nan"), dtype=dtype, device="cuda")
    pitch[:, :, :n_in] = w
    check(grouped_linear(x, pitch[:, :, :n_in], off), x, w, off)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_infinities_and_nan_stay_with_their_rows_and_groups(dtype):
    x, w, b, off = make(4, [5, 6, 40, 3], 64, 80, dtype)
    clean = grouped_linear(x, w, off, b)
    x2, w2 = x.clone(), w.clone()
    x2[2, 7] = float("nan")
    x2[20, 63] = float("inf")
    w2[3, 11, 5] = float("-inf")
    got = grouped_linear(x2, w2, off, b)
    want = exact(x2, w2, off, b)[0]
    bad = ~want.isfinite()
    assert torch.equal(got.isnan()[bad], want.isnan()[bad]) and torch.equal(got[bad & want.isinf()].double(), want[bad & want.isinf()])
    assert torch.equal(got[~bad], clean[~bad]) and int(bad.sum()) == 80 + 80 + 3


def test_offsets_beyond_the_rows_touch_nothing_else():
    x, w, b, _ = make(3, [4, 4, 4], 16, 16, F32)
    ys = torch.full((14, 16), 3.0, device="cuda")
    for edges in ([-5, 4, 100, 1 << 30], [0, 12, 4, 12], [9, 2, 2, 2]):
        grouped_linear(x, w, torch.tensor(edges, dtype=torch.int32, device="cuda"), b, out=ys[1:13])
        assert (ys[0] == 3).all() and (ys[13] == 3).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_streams_graphs_and_repetition(dtype):
    x, w, b, off = make(6, [10, 0, 33, 128, 1, 64], 128, 192, dtype)
    first = grouped_linear(x, w, off, b)
    for _ in range(3):
        assert torch.equal(grouped_linear(x, w, off, b), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = grouped_linear(x, w, off, b, stream=side)
    again = grouped_linear(x, w, off, b)
    side.synchronize()
    assert torch.equal(other, first) and torch.equal(again, first)
    off2 = torch.tensor([0, 50, 50, 60, 100, 230, 236], dtype=torch.int32, device="cuda")
    live, graph = off.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = grouped_linear(x, w, live, b)
    for o in (off2, off):                                       # the sizes of the groups are read when the graph runs
        live.copy_(o)
        graph.replay()
        check(y, x, w, o, b)


def test_refusals():
    x, w, b, off = make(2, [3, 4], 8, 8, F32)
    y = torch.empty(7, 8, device="cuda")
    bad = [dict(x=x.cpu()), dict(x=x.double()), dict(x=x.t()), dict(weight=w[0]), dict(weight=w.bfloat16()), dict(weight=w[:, :, :7]),
           dict(offsets=off[:-1]), dict(offsets=off.float()), dict(offsets=off.cpu()), dict(bias=b[:1]), dict(bias=b.half()),
           dict(out=y[:6]), dict(out=y.half()), dict(out=x), dict(weight=w.transpose(1, 2)), dict(activation="gelu"), dict(scale=float("nan"))]
    for kw in bad:
        args = dict(x=x, weight=w, offsets=off, bias=b, out=y)
        args.update(kw)
        with pytest.raises((EvoError, KeyError)):
            grouped_linear(args.pop("x"), args.pop("weight"), args.pop("offsets"), args.pop("bias"), **args)
    assert grouped_linear(x[:0], w, torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 8)


def theta_for(members, sizes, seed=0):
    dim = W.mlp_param_count(sizes)
    gen = torch.Generator(device="cuda").manual_seed(seed + dim)
    return torch.randn(members, (dim + 31) // 32 * 32, generator=gen, device="cuda") * 0.3


def actions_exact(theta, sizes, obs, offsets, scale):
    """(actions, bound): errors of a layer are at most the sum of |w| times those of the one before, and tanh makes none larger."""
    y = torch.full((obs.shape[0], sizes[-1]), float("nan"), dtype=torch.float64, device=obs.device)
    bound = torch.zeros_like(y)
    edges = offsets.tolist()
    for m, (p, q) in enumerate(zip(edges[:-1], edges[1:])):
        if q <= p:
            continue
        h, e, at = obs[p:q].double(), torch.zeros(q - p, sizes[0], dtype=torch.float64, device=obs.device), 0
        for n_in, n_out in zip(sizes[:-1], sizes[1:]):
            w = theta[m, at:at + n_out * n_in].view(n_out, n_in).double()
            b = theta[m, at + n_out * n_in:at + n_out * n_in + n_out].double()
            at += n_out * n_in + n_out
            e = e @ w.abs().t() + slack(F32, n_in) * (h.abs() @ w.abs().t() + b.abs())
            h = torch.tanh(h @ w.t() + b)
            e = e + 2.0 ** -22 * h.abs()
        y[p:q], bound[p:q] = scale * h, abs(scale) * e + 2.0 ** -23 * abs(scale)
    return y, bound


@pytest.mark.parametrize("sizes", [(5, 16, 16, 1), (5, 64, 64, 1), (28, 128, 128, 8), (28, 96, 40, 8), (3, 7), (1, 1), (9, 179, 38, 13),
                                   (12, 164, 47, 24, 7), (28, 64, 64, 64, 64, 8), (2, 3, 3, 3, 3, 3, 3, 3, 1), (28, 192, 192, 8), (30, 300, 20, 4),
                                   (40, 700, 700, 3)])
@pytest.mark.parametrize("lengths", [[1] * 9, [0, 16, 5, 0, 33, 8, 1, 17, 9], [200, 0, 3]])
def test_actions(sizes, lengths):
    members, lead, tail = len(lengths), 1, 2
    theta = theta_for(members, sizes)
    gen = torch.Generator(device="cuda").manual_seed(sum(lengths))
    obs = torch.randn(lead + sum(lengths) + tail, sizes[0], generator=gen, device="cuda")
    edges = [lead]
    for n in lengths:
        edges.append(edges[-1] + n)
    off = torch.tensor(edges, dtype=torch.int32, device="cuda")
    obs[0] = float("nan")
    ys = torch.full((obs.shape[0], sizes[-1] + 3), 5.0, device="cuda")
    out = ys[:, 1:1 + sizes[-1]]
    assert mlp_actions(theta, sizes, obs, off, action_scale=10.0, out=out) is out
    want, bound = actions_exact(theta, sizes, obs, off, 10.0)
    inside = ~want.isnan()
    err = (out.double() - want).abs()
    assert (err[inside] <= bound[inside]).all(), float((err / bound)[inside].max())
    ys[edges[0]:edges[-1], 1:1 + sizes[-1]] = 5.0
    assert (ys == 5).all()
    # the fresh output, 64-bit offsets, strided observations: the same bits
    wide = torch.zeros(obs.shape[0], sizes[0] + 5, device="cuda")
    wide[:, 2:2 + sizes[0]] = obs
    a = mlp_actions(theta, sizes, obs, off, action_scale=10.0)[edges[0]:edges[-1]]
    b = mlp_actions(theta, sizes, wide[:, 2:2 + sizes[0]], off.long(), action_scale=10.0)[edges[0]:edges[-1]]
    assert torch.equal(a, b)


@pytest.mark.parametrize("members,rows,sizes", [(700, 2500, (28, 128, 128, 8)), (1100, 5000, (5, 64, 64, 1)), (2000, 30000, (20, 100, 60, 4)), (300, 9000, (28, 96, 40, 8)),
                                                (3, 4000, (28, 128, 128, 8)), (40, 60, (60, 200, 200, 200, 200, 9)), (64, 64, (28, 512, 300, 8))])
def test_actions_of_populations(members, rows, sizes):
    """Sizes at which other kernels are chosen: a launch per layer, a warp and eight warps an item."""
    theta = theta_for(members, sizes)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    cuts = torch.sort(torch.randint(0, rows + 1, (members - 1,), generator=gen, device="cuda")).values
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cuts, torch.full((1,), rows, device="cuda")]).int()
    obs = torch.randn(rows, sizes[0], generator=gen, device="cuda")
    got = mlp_actions(theta, sizes, obs, off, action_scale=2.0)
    want, bound = actions_exact(theta, sizes, obs, off, 2.0)
    assert ((got.double() - want).abs() <= bound).all(), float(((got.double() - want).abs() / bound).max())
    assert torch.equal(mlp_actions(theta, sizes, obs, off, action_scale=2.0), got)


@pytest.mark.parametrize("groups,rows,n_in,n_out,dtype", [(500, 1500, 128, 130, F32), (500, 1500, 100, 64, F32), (40, 9000, 500, 200, F32), (3, 3, 4000, 70, F32), (20, 2000, 36, 1000, F32),
                                                          (2000, 4000, 64, 40, BF16), (3, 2000, 520, 384, F16), (1, 5000, 128, 128, BF16)])
def test_grouped_populations(groups, rows, n_in, n_out, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + n_in)
    cuts = torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=gen, device="cuda")).values
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cuts, torch.full((1,), rows, device="cuda")])
    x = torch.randn(rows, n_in, generator=gen, device="cuda").to(dtype)
    w = (torch.randn(groups, n_out, n_in, generator=gen, device="cuda") / math.sqrt(n_in)).to(dtype)
    b = torch.randn(groups, n_out, generator=gen, device="cuda").to(dtype)
    check(grouped_linear(x, w, off, b, activation="tanh"), x, w, off, b, "tanh")


def test_actions_layer_by_layer_are_the_same_policy():
    """The products grouped by member, one after the other over the layers of theta, as a user composes them."""
    sizes, lengths = (28, 128, 128, 8), [4, 0, 7, 3, 1]
    theta = theta_for(5, sizes)
    obs = torch.randn(15, 28, device="cuda")
    off = torch.tensor([0, 4, 4, 11, 14, 15], device="cuda")
    h, at = obs, 0
    for n_in, n_out in zip(sizes[:-1], sizes[1:]):
        w = theta[:, at:at + n_out * n_in].unflatten(1, (n_out, n_in))
        b = theta[:, at + n_out * n_in:at + n_out * n_in + n_out]
        at += n_out * n_in + n_out
        h = grouped_linear(h, w, off, b, activation="tanh")
    want, bound = actions_exact(theta, sizes, obs, off, 1.0)
    for got in (h, mlp_actions(theta, sizes, obs, off)):
        assert ((got.double() - want).abs() <= bound).all()


def test_solver_actions_follow_the_population():
    w = W.CFG2
    s = Solver(w)
    off = torch.arange(0, 3 * w.pop_size + 1, 3, device="cuda")
    obs = torch.randn(3 * w.pop_size, 5, device="cuda")
    with pytest.raises(EvoError):
        s.actions(obs, off)                                     # no ask yet
    theta = s.ask()
    got = s.actions(obs, off)
    want, bound = actions_exact(theta, w.layer_sizes, obs, off, w.action_scale)
    assert ((got.double() - want).abs() <= bound).all()
    assert torch.equal(s.actions(obs, off, theta=theta.clone().contiguous()[:, :w.param_dim]) if w.param_dim % 4 == 0 else got, got)
    assert s.sync_status() == 0
    s.close()
    c = Solver(W.CFG3.with_(pop_size=2, batch=8))
    with pytest.raises(EvoError):
        c.actions(obs, off)
    c.close()


def test_actions_refusals():
    sizes = (5, 16, 16, 1)
    theta, obs, off = theta_for(4, sizes), torch.randn(8, 5, device="cuda"), torch.tensor([0, 2, 4, 6, 8], device="cuda")
    mlp_actions(theta, sizes, obs, off)
    for kw in (dict(theta=theta[:, :300]), dict(theta=theta.half()), dict(layer_sizes=(6, 16, 16, 1)), dict(layer_sizes=(5,)), dict(layer_sizes=(5, 0, 1)),
               dict(layer_sizes=(5,) + (4,) * 8 + (1,)), dict(observations=obs[:, :4]), dict(offsets=off[:4]), dict(theta=theta[:, 1:]),
               dict(theta=torch.randn(4, 387, device="cuda")), dict(out=torch.empty(8, 2, device="cuda")), dict(action_scale=float("inf"))):
        args = dict(theta=theta, layer_sizes=sizes, observations=obs, offsets=off)
        args.update(kw)
        with pytest.raises(EvoError):
            mlp_actions(args.pop("theta"), args.pop("layer_sizes"), args.pop("observations"), args.pop("offsets"), **args)


@pytest.mark.parametrize("n_in", [520, 2060, 4100])
def test_long_fp32_sums_are_not_cut_off(n_in):
    """The tensor core cuts 2^-24 of a sum off on average for every 16 numbers that it adds, of a sum that has 2/3 of its size in the mean on its way
    up; in parts of 512 numbers that is at most 32 * 2^-24 * 2/3 = 1.3e-6 (in one sum of 4,100: 1e-5)."""
    x, w, _, off = make(2, [150, 90], n_in, 40, F32)
    want, _ = exact(x, w, off, None)
    got = grouped_linear(x, w, off).double()
    assert float((got - want).norm() / want.norm()) < 1.3e-6
