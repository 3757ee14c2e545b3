"""The matrix operators captured into graphs and replayed on other inputs, and on two streams at once: the bits of a call by itself, for a call
that takes each of their kernels."""
import pytest
import torch

from paper_2202_05008_b200 import grouped_linear, mlp_actions, muon_step, orthogonalize, workloads as W

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _normal(gen, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


def _orthogonalize(batch, rows, cols, dtype):
    def make(gen):
        return [_normal(gen, batch, rows, cols, dtype=dtype)]
    return make, lambda x, stream=None: (orthogonalize(x, stream=stream),)


def _muon(*sizes):
    matrices, at = [], 2
    for rows, cols in sizes:
        matrices.append((at, rows, cols))
        at += rows * cols + rows

    def make(gen):
        return [_normal(gen, at), _normal(gen, at) * 1e-3, _normal(gen, at).square(), _normal(gen, at) * 1e-2]
    return make, lambda c, m, v, g, stream=None: muon_step(c, m, v, g, matrices, 3, lr=0.02, stream=stream)


def _offsets(gen, groups, rows):
    cuts = torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=gen, device="cuda")).values
    return torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cuts, torch.full((1,), rows, device="cuda")]).int()


def _grouped(groups, rows, n_in, n_out, dtype):
    def make(gen):
        return [_normal(gen, rows, n_in, dtype=dtype), _normal(gen, groups, n_out, n_in, dtype=dtype) * n_in ** -0.5, _offsets(gen, groups, rows), _normal(gen, groups, n_out, dtype=dtype)]
    return make, lambda x, w, o, b, stream=None: (grouped_linear(x, w, o, b, activation="tanh", stream=stream),)


def _actions(members, rows, sizes):
    dim = (W.mlp_param_count(sizes) + 31) // 32 * 32

    def make(gen):
        return [_normal(gen, members, dim) * 0.2, _normal(gen, rows, sizes[0]), _offsets(gen, members, rows)]
    return make, lambda t, x, o, stream=None: (mlp_actions(t, sizes, x, o, action_scale=3.0, stream=stream),)


CALLS = [
    _orthogonalize(3, 12, 700, F32), _orthogonalize(2, 20, 160, BF16), _orthogonalize(2, 24, 2000, F32), _orthogonalize(4, 64, 60, F16), _orthogonalize(2, 100, 500, F32),
    _orthogonalize(2, 200, 300, F32), _orthogonalize(1, 700, 260, BF16),
    _muon((28, 128), (128, 128), (8, 128)), _muon((300, 200), (20, 400), (5, 300), (64, 700)),
    _grouped(50, 120, 128, 64, F32), _grouped(50, 120, 127, 64, F32), _grouped(6, 700, 130, 100, F32), _grouped(3, 4, 1000, 70, F32), _grouped(50, 120, 128, 64, BF16),
    _grouped(6, 700, 136, 100, BF16), _grouped(6, 700, 131, 100, F16), _grouped(3, 300, 9000, 40, F16), _grouped(3, 3, 9000, 40, BF16),
    _actions(20, 70, (5, 16, 16, 1)), _actions(700, 2500, (28, 128, 128, 8)), _actions(5, 400, (28, 600, 64, 3)), _actions(300, 3000, (28, 100, 60, 8)),
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
    pairs = [(CALLS[which], CALLS[which]), (CALLS[which], CALLS[(which + 7) % len(CALLS)])]
    for calls in pairs:
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
