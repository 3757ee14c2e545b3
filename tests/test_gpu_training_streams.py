"""What a mixture is trained with, captured into graphs and replayed on other inputs, on two streams at once, and twice on the same inputs: the bits of a call by itself, for a
call that takes each of the kernels."""
import pytest
import torch

from paper_2202_05008_b200 import (EvoError, combine_rows, combine_rows_backward, grouped_linear, grouped_linear_backward, muon_step, policy_loss, route_rows,
                                   take_rows)

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _normal(gen, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


def _route(rows, choices, groups):
    def make(gen):
        return [torch.randint(-1, groups, (rows, choices), generator=gen, device="cuda", dtype=torch.int32)]
    return make, lambda m, stream=None: tuple(route_rows(m, groups, stream=stream))


def _place(gen, rows, choices):
    place = torch.randperm(rows * choices, generator=gen, device="cuda").int().view(rows, choices)
    place[torch.rand(rows, choices, generator=gen, device="cuda") < 0.1] = -1
    return place


def _rows(what, rows, choices, cols, dtype):
    def make(gen):
        args = [_normal(gen, rows, cols, dtype=dtype), _normal(gen, rows * choices, cols, dtype=dtype), _place(gen, rows, choices), _normal(gen, rows, choices)]
        return args + [torch.zeros(rows * choices, cols, dtype=dtype, device="cuda")]

    def call(x, y, place, w, out, stream=None):
        # (rows without a place are as they were: a buffer of the call's own, so that two calls at once do not share it)
        room = out.clone() if stream is None else _on(stream, out.clone)
        if what == "take":
            return (take_rows(x, place, w, out=room, stream=stream),)
        if what == "combine":
            return (combine_rows(y, place, w, stream=stream),)
        return combine_rows_backward(x, y, place, w, out=room, stream=stream)
    return make, call


def _on(stream, f):
    with torch.cuda.stream(stream):
        return f()


def _offsets(gen, groups, rows):
    cuts = torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=gen, device="cuda")).values
    return torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cuts, torch.full((1,), rows, device="cuda")]).int()


def _products(groups, rows, n_in, n_out, dtype, act, shared=False):
    def make(gen):
        y = _normal(gen, rows, n_out)
        y = torch.tanh(y) if act == "tanh" else y.relu()
        return [_normal(gen, rows, n_out, dtype=dtype), _normal(gen, rows, n_in, dtype=dtype), _normal(gen, 1 if shared else groups, n_out, n_in, dtype=dtype) * n_in ** -0.5,
                _offsets(gen, groups, rows), y.to(dtype)]

    def call(dy, x, w, o, y, stream=None):
        return grouped_linear_backward(dy, x, w.expand(groups, -1, -1) if shared else w, o, y, activation=act, shared_bias=shared, stream=stream)
    return make, call


def _policy(rows, n, dtype):
    def make(gen):
        return [_normal(gen, rows, n, dtype=dtype), torch.randint(-1, n, (rows,), generator=gen, device="cuda"), _normal(gen, rows) - 3, _normal(gen, rows),
                _normal(gen, rows) - 3]
    return make, lambda x, a, old, adv, ref, stream=None: tuple(policy_loss(x, a, old, adv, ref_logp=ref, kl=0.1, stream=stream))


CALLS = [
    _route(50, 1, 9), _route(900, 3, 200), _route(9000, 2, 70), _route(40000, 2, 300), _route(900, 3, 5000), _route(70000, 1, 100000),
    _rows("take", 300, 2, 64, F32), _rows("take", 300, 2, 61, BF16), _rows("take", 300, 2, 333, F16), _rows("combine", 300, 1, 64, F32), _rows("combine", 300, 2, 512, BF16),
    _rows("combine", 300, 5, 512, F16), _rows("combine", 300, 3, 7, F32), _rows("combine", 300, 3, 1001, BF16), _rows("backward", 300, 1, 64, F32),
    _rows("backward", 300, 2, 512, BF16), _rows("backward", 300, 7, 2048, F16), _rows("backward", 300, 3, 9, F32), _rows("backward", 300, 3, 1001, F16),
    _products(50, 120, 128, 64, F32, "tanh"), _products(700, 1500, 128, 160, F32, "none"), _products(700, 1500, 61, 160, BF16, "tanh"), _products(6, 700, 130, 100, F32, "tanh"),
    _products(6, 700, 136, 104, BF16, "none"), _products(6, 700, 136, 104, F16, "tanh"), _products(6, 700, 131, 101, F16, "relu"), _products(2, 5000, 40, 30, F32, "relu"),
    _products(2, 5000, 40, 24, BF16, "tanh", True), _products(3, 9000, 264, 300, BF16, "none"), _products(3, 40, 2000, 500, F16, "relu"), _products(1, 30000, 130, 70, F16, "tanh"),
    _policy(500, 12, F32), _policy(70, 50, BF16), _policy(70, 100, F16), _policy(9000, 200, BF16), _policy(70, 900, F32), _policy(70, 2000, BF16), _policy(20, 6000, F32),
    _policy(400, 9000, BF16), _policy(6, 70001, F16), _policy(3, 200000, BF16),
]


@pytest.mark.parametrize("which", range(len(CALLS)))
def test_a_captured_call_replays_on_what_its_inputs_hold_by_then(which):
    make, call = CALLS[which]
    gen = torch.Generator(device="cuda").manual_seed(which)
    first, second = make(gen), make(gen)
    want = [[x.clone() for x in call(*args)] for args in (first, second)]
    live, graph = [x.clone() for x in first], torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(*live)
    for args, results in ((second, want[1]), (first, want[0]), (second, want[1])):
        for x, y in zip(live, args):
            x.copy_(y)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(out, results))
    assert all(torch.equal(x, y) for x, y in zip(live, second))          # inputs are left as they were


@pytest.mark.parametrize("which", range(len(CALLS)))
def test_calls_on_two_streams_at_once(which):
    gen = torch.Generator(device="cuda").manual_seed(100 + which)
    for calls in ((CALLS[which], CALLS[which]), (CALLS[which], CALLS[(which + 13) % len(CALLS)])):
        inputs = [make(gen) for make, _ in calls]
        want = [[x.clone() for x in call(*args)] for (_, call), args in zip(calls, inputs)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        got = [[] for _ in calls]
        for _ in range(6):
            for k, (_, call) in enumerate(calls):
                got[k].append(call(*inputs[k], stream=streams[k]))
        torch.cuda.synchronize()
        for k in range(2):
            for results in got[k]:
                assert all(torch.equal(x, y) for x, y in zip(results, want[k]))


def test_graphs_that_share_a_memory_pool():
    """Workspaces of two captured calls may lie at the same place; replayed one after the other, either keeps its results' bits."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    pool, made = torch.cuda.graph_pool_handle(), []
    for make, call in (CALLS[22], CALLS[30], CALLS[3], CALLS[34]):
        args = make(gen)
        want = [x.clone() for x in call(*args)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            out = call(*args)
        made.append((graph, out, want, args))                    # (the inputs have to live as long as the graph)
    for graph, out, want, _ in made + made[::-1]:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_a_stream_of_no_other_device_and_a_gradient_that_would_be_lost():
    x = torch.zeros(4, 8, device="cuda").requires_grad_()
    with pytest.raises(EvoError):
        take_rows(x, torch.zeros(4, dtype=torch.int32, device="cuda"))
    with torch.no_grad():
        take_rows(x, torch.arange(4, dtype=torch.int32, device="cuda"))


def _mixture(x, members, gates, theta, sizes, actions, old, adv):
    """(loss, gradient of theta, of the gates, of x) by the library's calls: experts of two layers."""
    n_in, hidden, n = sizes
    w1, b1, w2, b2 = _layers(theta, sizes)
    groups = theta.shape[0]
    routes = route_rows(members, groups)
    xs = take_rows(x, routes.place)
    h = grouped_linear(xs, w1, routes.offsets, b1, activation="tanh")
    ys = grouped_linear(h, w2, routes.offsets, b2)
    loss, logp, d_logits = policy_loss(combine_rows(ys, routes.place, gates), actions, old, adv, clip=(0.2, 0.2))
    gradient = torch.zeros_like(theta)
    g1, gb1, g2, gb2 = _layers(gradient, sizes)
    d_ys, d_gates = combine_rows_backward(d_logits, ys, routes.place, gates)
    d_h, _, _ = grouped_linear_backward(d_ys, h, w2, routes.offsets, out=(None, g2, gb2))
    d_xs, _, _ = grouped_linear_backward(d_h, xs, w1, routes.offsets, h, activation="tanh", out=(None, g1, gb1))
    return loss, gradient, d_gates, combine_rows(d_xs, routes.place)


def _layers(theta, sizes):
    n_in, hidden, n = sizes
    at = [0, n_in * hidden, n_in * hidden + hidden, n_in * hidden + hidden + hidden * n, n_in * hidden + hidden + hidden * n + n]
    return (theta[:, at[0]:at[1]].unflatten(1, (hidden, n_in)), theta[:, at[1]:at[2]], theta[:, at[2]:at[3]].unflatten(1, (n, hidden)), theta[:, at[3]:at[4]])


@pytest.mark.parametrize("rows,choices,groups,sizes", [(60, 2, 5, (6, 10, 4)), (300, 1, 40, (28, 64, 8)), (2000, 3, 6, (40, 136, 72))])
def test_a_training_step_of_a_mixture(rows, choices, groups, sizes):
    """The whole chain against torch's own gradients in 64 bits, then a Muon step along it."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    n_in, hidden, n = sizes
    dim = (n_in + 1) * hidden + (hidden + 1) * n
    theta = _normal(gen, groups, (dim + 31) // 32 * 32) * 0.3
    x, gates = _normal(gen, rows, n_in), torch.softmax(_normal(gen, rows, choices), 1)
    members = torch.randint(-1, groups, (rows, choices), generator=gen, device="cuda")
    actions, adv = torch.randint(0, n, (rows,), generator=gen, device="cuda"), _normal(gen, rows)
    old = torch.full((rows,), -3.0, device="cuda")                  # (ratios are e^(logp + 3): a few lie near a border by chance, none on it)
    loss, d_theta, d_gates, d_x = _mixture(x, members, gates, theta, sizes, actions, old, adv)

    t, g, z = theta.double().requires_grad_(), gates.double().requires_grad_(), x.double().requires_grad_()
    w1, b1, w2, b2 = _layers(t, sizes)
    logits = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    for j in range(choices):
        m = members[:, j].clamp_min(0)
        y = torch.bmm(w2[m], torch.tanh(torch.bmm(w1[m], z[:, :, None])[:, :, 0] + b1[m])[:, :, None])[:, :, 0] + b2[m]
        logits = logits + torch.where((members[:, j] >= 0)[:, None], g[:, j, None] * y, torch.zeros_like(y))
    logp = torch.log_softmax(logits, 1).gather(1, actions[:, None])[:, 0]
    ratio = torch.exp(logp - old.double())
    border = torch.minimum((ratio - 0.8).abs(), (ratio - 1.2).abs()).min()
    assert border > 1e-6                                            # fp32 decides as fp64 does
    want = -torch.minimum(ratio * adv.double(), ratio.clamp(0.8, 1.2) * adv.double()).mean()
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 1e-5
    for got, exact in ((d_theta, t.grad), (d_gates, g.grad), (d_x, z.grad)):
        # four layers of products in fp32 with 21 bits: 1e-5 of the largest leaves ten times that
        assert (got.double() - exact).abs().max() <= 1e-5 * exact.abs().max() + 1e-9
    center = theta[0, :dim].clone()
    matrices = [(0, hidden, n_in), (n_in * hidden + hidden, n, hidden)]
    after = muon_step(center, torch.zeros_like(center), torch.zeros_like(center), -d_theta[0, :dim].contiguous(), matrices, 1, lr=0.02)
    assert all(v.isfinite().all() for v in after) and not torch.equal(after[0], center)
