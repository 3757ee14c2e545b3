"""Solvers with the Muon optimiser against the oracle's ranks and gradient and the step's formulas in 64 bits (teacher-forced per
generation: both start from the GPU's state)."""
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import rel_err
from paper_2202_05008_b200 import EvoError, Solver, muon_step, train, workloads as W
from test_gpu_orthogonalize import muon_exact

pytestmark = pytest.mark.gpu
F32 = lambda x: float(np.float32(x))
MLP = ((0, 128, 28), (3712, 128, 128), (20224, 8, 128))
NONE = W.Workload("muon", 64, 21256, seed=9, lr=0.02, policy_kind=W.POLICY_MLP, layer_sizes=(28, 128, 128, 8), optimizer=W.OPT_MUON)
WIDE = W.Workload("muon_wide", 16, 200 * 301 + 3 * 201, seed=10, lr=0.02, policy_kind=W.POLICY_MLP, layer_sizes=(300, 200, 3), optimizer=W.OPT_MUON)
WIDE_MATRICES = ((0, 200, 300), (200 * 301, 3, 200))


def _fitness(w, gen):
    return torch.tensor(W.synthetic_fitness(w.seed, gen, w.pop_size), device="cuda")


def _lstm(h):
    out, at = [], 0
    for _ in range(2):
        out += [(at, 4 * h, 12), (at + 48 * h, 4 * h, h)]
        at += 48 * h + 4 * h * h + 4 * h
    return tuple(out + [(at, 12, h)])


CASES = [
    (NONE, MLP), (WIDE, WIDE_MATRICES), (WIDE.with_(muon_momentum=0.8, muon_weight_decay=0.1, muon_steps=3, muon_plain_momentum=True), WIDE_MATRICES),
    (W.CFG1.with_(optimizer=W.OPT_MUON), ((0, 16, 5), (96, 16, 16), (368, 1, 16))),
    (W.CFG3.with_(optimizer=W.OPT_MUON, batch=8), ((0, 8, 25), (208, 16, 200), (3424, 10, 256))),
    (W.SEQ2SEQ.with_(optimizer=W.OPT_MUON, pop_size=32, batch=8), _lstm(128)),
    (W.SEQ2SEQ.with_(optimizer=W.OPT_MUON, pop_size=32, batch=8, layer_sizes=(64,), param_dim=W.seq2seq_param_count(64)), _lstm(64)),
]


@pytest.mark.parametrize("w,matrices", CASES, ids=lambda x: x.name if isinstance(x, W.Workload) else "")
@pytest.mark.parametrize("noise_mode", [W.NOISE_STORED, W.NOISE_REGENERATED])
def test_tell_takes_the_step(w, matrices, noise_mode):
    s = Solver(w, noise_mode=noise_mode)
    for gen in range(3):
        c0, (m0, v0) = s.center().clone(), (x.clone() for x in s.moments())
        s.ask()
        f = _fitness(w, gen)
        s.tell(f)
        assert s.sync_status() == 0 and s.counters() == (gen + 1, gen + 1)
        _, eps_o = oracle.ask(w.seed, gen, w.pop_size, w.param_dim, np.zeros(w.param_dim, np.float32), w.sigma)
        _, u_o, _ = oracle.centered_rank(f.cpu().numpy())
        assert rel_err(s.gradient().cpu().numpy(), oracle.gradient(u_o, eps_o, F32(w.sigma))) < 1e-5
        mu, steps = w.muon_momentum or 0.95, w.muon_steps or 5
        # the step itself, from the gradient that the solver has, by the operator (same bits) and by the formulas
        kw = dict(lr=F32(w.lr), momentum=F32(mu), nesterov=not w.muon_plain_momentum, weight_decay=F32(w.muon_weight_decay), ns_steps=steps,
                  beta1=F32(0.9), beta2=F32(0.999), adam_eps=F32(1e-8))
        want = muon_step(c0, m0, v0, s.gradient().clone(), matrices, gen + 1, **kw)
        got = (s.center(),) + tuple(s.moments())
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        if steps == 5:
            exact = muon_exact(c0, m0, v0, s.gradient(), matrices, gen + 1, F32(w.lr), F32(mu), not w.muon_plain_momentum, F32(w.muon_weight_decay),
                               F32(0.9), F32(0.999), F32(1e-8))
            # a full-rank matrix' step: 64 x 2^-22 (and the null space's 3.4445^5 2^-22 against |O| >= 0.7 of one direction)
            for at, r, c in matrices:
                part = slice(at, at + r * c)
                move = exact[0][part] - c0[part].double()
                assert float((got[0][part].double() - exact[0][part]).norm()) <= 2.0 ** -22 * (64 + 700) * float(move.norm()) + 2.0 ** -23 * float(c0[part].norm())
    full = s._view_f32(s.center().data_ptr(), 1, s.ldD)[0]
    assert (full[w.param_dim:] == 0).all()
    s.close()


@pytest.mark.parametrize("w", [NONE, WIDE], ids=lambda w: w.name)
def test_nan_fitness_skips_the_step(w):
    s = Solver(w)
    s.ask(); s.tell(_fitness(w, 0))
    before = [s.center().clone()] + [x.clone() for x in s.moments()]
    s.ask()
    f = _fitness(w, 1)
    f[3] = float("nan")
    s.tell(f)
    assert s.sync_status() == 5 and s.counters() == (2, 1)
    assert all(torch.equal(x, y) for x, y in zip([s.center()] + list(s.moments()), before))
    s.ask(); s.tell(_fitness(w, 2))
    assert s.sync_status() == 0 and not torch.equal(s.center(), before[0]) and s.counters() == (3, 2)
    s.close()


@pytest.mark.parametrize("w", [NONE, WIDE], ids=lambda w: w.name)
def test_begin_and_end_a_resumed_solver_and_adapted_sigma_take_the_same_step(w):
    w = w.with_(sigma_mode=W.SIGMA_PGPE)
    a, b = Solver(w), Solver(w)
    for gen in range(2):
        f = _fitness(w, gen)
        a.ask(); a.tell(f)
        b.ask(); b.tell_begin(f); b.tell_end()
        assert torch.equal(a.center(), b.center()) and torch.equal(a.sigma(), b.sigma())
        assert all(torch.equal(x, y) for x, y in zip(a.moments(), b.moments()))
    c = Solver(w)
    m, v = a.moments()
    c.set_state(a.center().clone(), m.clone(), v.clone(), *a.counters())
    c.set_sigma(a.sigma().clone())
    f = _fitness(w, 2)
    a.ask(); a.tell(f)
    c.ask(); c.tell(f)
    assert torch.equal(a.center(), c.center()) and a.sync_status() == 0 and c.sync_status() == 0
    for s in (a, b, c):
        s.close()


def test_a_captured_generation_replays():
    w = W.CFG2.with_(pop_size=32, horizon=20, optimizer=W.OPT_MUON)
    plain = Solver(w)
    for _ in range(3):
        plain.ask()
        fit = plain.rollout()
        plain.tell(fit)
    assert plain.sync_status() == 0
    s = Solver(w, stream=torch.cuda.Stream())
    fitness = torch.empty(w.pop_size, device="cuda")
    torch.cuda.synchronize()
    s.ask(); s.rollout(fitness=fitness); s.tell(fitness)        # the first one outside the graph
    s.stream.synchronize()
    graph = s.capture_generation(fitness)
    with torch.cuda.stream(s.stream):
        graph.replay(); graph.replay()
    assert s.sync_status() == 0 and s.counters() == (3, 3)
    assert torch.equal(s.center(), plain.center())
    del graph
    s.close(); plain.close()


@pytest.mark.parametrize("w", [NONE, WIDE], ids=lambda w: w.name)
def test_the_checked_build_finds_every_guard_untouched(w):
    s, t = Solver(w, debug=True), Solver(w)
    for gen in range(2):
        for x in (s, t):
            x.ask(); x.tell(_fitness(w, gen))
        assert s.debug_check() == (-1, 0, 0)
    assert torch.equal(s.center(), t.center()) and s.sync_status() == 0
    s.close(); t.close()


def test_training_runs_with_every_policy():
    for w in (W.CFG1.with_(optimizer=W.OPT_MUON), W.CFG3.with_(optimizer=W.OPT_MUON, pop_size=4, batch=16)):
        s, history = train.run(w, 2)
        assert len(history) == 2 and all(math.isfinite(x) for pair in history for x in pair)
        assert bool(s.center().isfinite().all()) and float(s.center().abs().max()) > 0
        s.close()


def test_configurations_without_matrices_are_refused():
    for w, code in ((NONE.with_(policy_kind=W.POLICY_NONE), 7), (NONE.with_(layer_sizes=(28, 128, 127, 8)), 1), (NONE.with_(layer_sizes=()), 1),
                    (W.PAINT.with_(optimizer=W.OPT_MUON), 7), (NONE.with_(muon_momentum=1.0), 1), (NONE.with_(muon_steps=65), 1),
                    (NONE.with_(muon_weight_decay=-0.1), 1), (NONE.with_(optimizer=3), 1)):
        with pytest.raises(EvoError) as e:
            Solver(w)
        assert e.value.code == code, w
