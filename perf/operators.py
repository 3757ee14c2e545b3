"""Performance cases of the matrix operators: orthogonalised updates, the Muon step of a parameter vector, matrix products
grouped by population member, and an MLP policy's actions for ragged rows.

With ``own`` false every case runs in plain torch operations (32-bit arithmetic, rounded once at the end); with ``own`` true it
makes the calls that a user of the library makes.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NS = (3.4445, -4.7750, 2.0315)      # the odd quintic whose iteration moves singular values towards 1
NS_STEPS = 5
NS_EPS = 1e-7
LR, MU, DECAY = 0.02, 0.95, 0.01
BETA1, BETA2, ADAM_EPS = 0.9, 0.999, 1e-8
STEP = 7                            # the step's number, for Adam's bias corrections


def _orthogonalize(batch, rows, cols, type_, **kw):
    return dict({"op": "orthogonalize", "batch": batch, "rows": rows, "cols": cols, "type": type_}, **kw)


def _muon(sizes, **kw):
    return dict({"op": "muon", "sizes": "-".join(map(str, sizes))}, **kw)


def _grouped(groups, rows, n_in, n_out, type_, spread, tanh, **kw):
    return dict({"op": "grouped", "groups": groups, "rows": rows, "in": n_in, "out": n_out, "type": type_, "spread": spread,
                 "tanh": tanh}, **kw)


def _actions(members, rows, sizes, spread, **kw):
    return dict({"op": "actions", "members": members, "rows": rows, "sizes": "-".join(map(str, sizes)), "spread": spread}, **kw)


def listed():
    return [
        # the hidden layer of the ordinary control policy: latency only
        _orthogonalize(1, 64, 64, "f32", name="orthogonalize_small"),
        # the gates of the recurrent policy's two cells: taller than wide
        _orthogonalize(2, 512, 128, "f32", name="orthogonalize_gates"),
        # one wide layer of a large network
        _orthogonalize(1, 2048, 2048, "f32", name="orthogonalize_large"),
        # a stack of layers kept in 16 bits, no size a multiple of a tile
        _orthogonalize(5, 1000, 2500, "bf16", name="orthogonalize_stack_bf16"),
        # the update of the large control policy's centre
        _muon((28, 128, 128, 8), name="muon_policy"),
        # the update of a network of a few million weights
        _muon((784, 1536, 1536, 1000), name="muon_network"),
        # one layer of every member of the large population, a few live episodes each: bound by the weights' way from memory
        _grouped(4096, 16384, 128, 128, "f32", 0.3, True, name="grouped_population"),
        # wide layers and many rows: bound by arithmetic; some groups get far more rows than others
        _grouped(32, 8192, 1024, 4096, "bf16", 0.4, False, name="grouped_wide_bf16"),
        # single rows: about one for each group
        _grouped(64, 64, 2048, 2048, "bf16", 0.0, False, name="grouped_single_rows_bf16"),
        # odd sizes in the other 16-bit type
        _grouped(12, 3001, 1000, 1501, "f16", 0.6, True, name="grouped_odd_f16"),
        # the smallest policy and population, one row each
        _actions(16, 16, (5, 16, 16, 1), 0.0, name="actions_small"),
        # the large population, some members' episodes ended
        _actions(4096, 16384, (28, 128, 128, 8), 0.3, name="actions_large"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["orthogonalize", "muon", "grouped", "actions"])
    if op == "orthogonalize":
        rows, cols = _log_int(rng, 2, 2600), _log_int(rng, 2, 2600)
        most = int(9e10 / (15.0 * min(rows, cols) ** 2 * max(rows, cols) + 1e8 * 1.0))
        return _orthogonalize(min(_log_int(rng, 1, 24), max(1, most)), rows, cols, rng.choice(["f32", "f32", "bf16", "f16"]))
    if op == "muon":
        top = rng.choice([96, 200, 500, 1000])
        return _muon([_log_int(rng, 4, top) for _ in range(rng.randint(2, 6))])
    spread = round(rng.uniform(0.0, 0.5), 2)
    if op == "grouped":
        type_ = rng.choice(["f32", "bf16", "f16"])
        n_in, n_out = _log_int(rng, 4, 4096), _log_int(rng, 1, 4096)
        groups = min(_log_int(rng, 1, 4096), max(1, int(1.2e8 / (n_in * n_out))))
        rows = min(_log_int(rng, 1, 20000), max(1, int((3e10 if type_ != "f32" else 6e9) / (n_in * n_out))))
        return _grouped(groups, rows, n_in, n_out, type_, spread, rng.random() < 0.5)
    widths = [_log_int(rng, 2, 64)] + [_log_int(rng, 8, 200) for _ in range(rng.randint(0, 4))] + [_log_int(rng, 1, 16)]
    members = _log_int(rng, 2, 4000)
    return _actions(members, min(max(1, int(members * _log_int(rng, 1, 40) * rng.uniform(0.5, 1.5))), 40000), widths, spread)


def _sizes(case):
    return [int(x) for x in case["sizes"].split("-")]


def _layout(sizes):
    """Per layer: offset of W [out][in], out, in, offset of the bias; and the number of parameters."""
    at, layers = 0, []
    for n_in, n_out in zip(sizes[:-1], sizes[1:]):
        layers.append((at, n_out, n_in, at + n_out * n_in))
        at += n_out * n_in + n_out
    return layers, at


def _offsets(groups, rows, spread, gen):
    """Ragged group sizes: shares drawn log-normally (spread 0: even), the remainders by chance; whole numbers that sum to `rows`."""
    share = torch.exp(torch.randn(groups, generator=gen, device="cuda", dtype=torch.float64) * spread * 2.0)
    edge = torch.cumsum(share, 0) * (rows / share.sum())
    phase = torch.rand(1, generator=gen, device="cuda", dtype=torch.float64)
    ends = torch.floor(edge + phase).clamp(0, rows).to(torch.int32)
    ends[-1] = rows
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), ends])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 17)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    op = case["op"]
    if op == "orthogonalize":
        b, r, c = case["batch"], case["rows"], case["cols"]
        low = min(r, c, 8)          # an estimated gradient: noise of full rank over a few strong directions
        g = normal(b, r, c) + 3.0 * torch.bmm(normal(b, r, low), normal(b, low, c)) / math.sqrt(low)
        return {"case": case, "x": (g * 0.01).to(TYPES[case["type"]])}
    if op == "muon":
        layers, dim = _layout(_sizes(case))
        return {"case": case, "center": normal(dim) * 0.1, "m": normal(dim) * 1e-3, "v": normal(dim).square() * 1e-6,
                "g": normal(dim) * 3e-3, "matrices": [(at, n_out, n_in) for at, n_out, n_in, _ in layers]}
    if op == "grouped":
        groups, n_in, n_out, t = case["groups"], case["in"], case["out"], TYPES[case["type"]]
        offsets = _offsets(groups, case["rows"], case["spread"], gen)
        pitch = -(-(n_out * n_in + n_out) // 32) * 32          # a layer inside the members' parameter rows
        theta = (normal(groups, pitch) / math.sqrt(n_in)).to(t)
        return {"case": case, "x": normal(case["rows"], n_in).to(t), "offsets": offsets,
                "weight": theta[:, :n_out * n_in].unflatten(1, (n_out, n_in)), "bias": theta[:, n_out * n_in:n_out * n_in + n_out],
                "longest": int((offsets[1:] - offsets[:-1]).max())}
    sizes = _sizes(case)
    layers, dim = _layout(sizes)
    members = case["members"]
    offsets = _offsets(members, case["rows"], case["spread"], gen)
    theta = normal(members, -(-dim // 32) * 32)
    for at, n_out, n_in, bias in layers:
        theta[:, at:bias] /= math.sqrt(n_in)
        theta[:, bias:bias + n_out] *= 0.1
    return {"case": case, "theta": theta, "sizes": sizes, "observations": normal(case["rows"], sizes[0]), "offsets": offsets,
            "longest": int((offsets[1:] - offsets[:-1]).max())}


def _plain_newton_schulz(g):
    """Of a batch of fp32 matrices."""
    a, b, c = NS
    x = g / (torch.linalg.vector_norm(g, dim=(-2, -1), keepdim=True) + NS_EPS)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-2, -1)
    for _ in range(NS_STEPS):
        s = torch.bmm(x, x.transpose(-2, -1))
        x = a * x + torch.bmm(b * s + c * torch.bmm(s, s), x)
    return x.transpose(-2, -1) if tall else x


def _plain_grouped(x, weight, bias, offsets, longest, tanh, scale=1.0):
    """Rows padded to the longest group, one batched product, rows back in their places."""
    groups = weight.shape[0]
    row = torch.arange(x.shape[0], device=x.device)
    group = torch.searchsorted(offsets[1:], row.to(offsets.dtype), right=True)
    place = group * longest + row - offsets[group]
    padded = torch.zeros(groups * longest, x.shape[1], device=x.device)
    padded[place] = x.float()
    y = torch.bmm(padded.view(groups, longest, -1), weight.float().transpose(1, 2)) + bias.float()[:, None, :]
    y = y.reshape(groups * longest, -1)[place]
    return scale * torch.tanh(y) if tanh else y


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2202_05008_b200 as evo
        if op == "orthogonalize":
            return evo.orthogonalize(state["x"], steps=NS_STEPS, coefficients=NS, eps=NS_EPS)
        if op == "muon":
            center, m, v = evo.muon_step(state["center"], state["m"], state["v"], state["g"], state["matrices"], STEP, lr=LR,
                                         momentum=MU, weight_decay=DECAY, ns_steps=NS_STEPS, beta1=BETA1, beta2=BETA2,
                                         adam_eps=ADAM_EPS)
            return {"center": center, "m": m, "v": v}
        if op == "grouped":
            return evo.grouped_linear(state["x"], state["weight"], state["offsets"], state["bias"],
                                      activation="tanh" if case["tanh"] else "none")
        return evo.mlp_actions(state["theta"], state["sizes"], state["observations"], state["offsets"], action_scale=10.0)
    if op == "orthogonalize":
        x = state["x"]
        return _plain_newton_schulz(x.float()).to(x.dtype)
    if op == "muon":
        g = state["g"]
        m = MU * state["m"] + (1 - MU) * g
        u = (1 - MU) * g + MU * m
        center = state["center"] * (1 - LR * DECAY)
        adam_m = BETA1 * state["m"] + (1 - BETA1) * g
        v = BETA2 * state["v"] + (1 - BETA2) * g * g
        by_adam = center + LR * (adam_m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + ADAM_EPS)
        new_m, new_v, new_c = adam_m, v, by_adam
        for at, r, c in state["matrices"]:
            part = slice(at, at + r * c)
            o = _plain_newton_schulz(u[part].view(1, r, c)).reshape(-1)
            new_c[part] = center[part] + LR * 0.2 * math.sqrt(max(r, c)) * o
            new_m[part] = m[part]
            new_v[part] = state["v"][part]
        return {"center": new_c, "m": new_m, "v": new_v}
    if op == "grouped":
        x = state["x"]
        return _plain_grouped(x, state["weight"], state["bias"], state["offsets"], state["longest"], case["tanh"]).to(x.dtype)
    h, theta = state["observations"], state["theta"]
    layers, _ = _layout(state["sizes"])
    for i, (at, n_out, n_in, bias) in enumerate(layers):
        last = i + 1 == len(layers)
        h = _plain_grouped(h, theta[:, at:bias].unflatten(1, (n_out, n_in)), theta[:, bias:bias + n_out], state["offsets"],
                           state["longest"], True, 10.0 if last else 1.0)
    return h


def _exact_newton_schulz(g):
    """Of one fp64 matrix: the odd polynomial by products on the right, x (a + b x'x + c (x'x)^2), on the shorter side."""
    a, b, c = NS
    x = g / (math.sqrt(float((g * g).sum())) + NS_EPS)
    flip = x.shape[0] < x.shape[1]
    x = x.t().contiguous() if flip else x
    eye = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
    for _ in range(NS_STEPS):
        s = x.t() @ x
        x = x @ (a * eye + s @ (b * eye + c * s))
    return x.t() if flip else x


def _exact_layer(x, weight, bias, offsets):
    out = torch.zeros(x.shape[0], weight.shape[1], dtype=torch.float64, device=x.device)
    edges = offsets.tolist()
    for g, (first, last) in enumerate(zip(edges[:-1], edges[1:])):
        if last > first:
            out[first:last] = x[first:last] @ weight[g].double().t() + bias[g].double()
    return out


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "orthogonalize":
        return torch.stack([_exact_newton_schulz(g.double()) for g in state["x"]])
    if op == "muon":
        center, m, v, g = (state[k].double() for k in ("center", "m", "v", "g"))
        new_c, new_m, new_v = center.clone(), torch.empty_like(m), torch.empty_like(v)
        new_c *= 1 - LR * DECAY
        matrix = torch.zeros(g.numel(), dtype=torch.bool, device=g.device)
        for at, r, c in state["matrices"]:
            matrix[at:at + r * c] = True
            mm = MU * m[at:at + r * c] + (1 - MU) * g[at:at + r * c]
            u = MU * mm + (1 - MU) * g[at:at + r * c]
            new_m[at:at + r * c] = mm
            new_v[at:at + r * c] = v[at:at + r * c]
            new_c[at:at + r * c] += LR * 0.2 * math.sqrt(max(r, c)) * _exact_newton_schulz(u.view(r, c)).reshape(-1)
        rest = ~matrix
        new_m[rest] = BETA1 * m[rest] + (1 - BETA1) * g[rest]
        new_v[rest] = BETA2 * v[rest] + (1 - BETA2) * g[rest] ** 2
        new_c[rest] += LR * (new_m[rest] / (1 - BETA1 ** STEP)) / (torch.sqrt(new_v[rest] / (1 - BETA2 ** STEP)) + ADAM_EPS)
        return {"center": new_c, "m": new_m, "v": new_v}
    if op == "grouped":
        y = _exact_layer(state["x"].double(), state["weight"], state["bias"], state["offsets"])
        return torch.tanh(y) if case["tanh"] else y
    h = state["observations"].double()
    layers, _ = _layout(state["sizes"])
    for at, n_out, n_in, bias in layers:
        h = torch.tanh(_exact_layer(h, state["theta"][:, at:bias].unflatten(1, (n_out, n_in)), state["theta"][:, bias:bias + n_out],
                                    state["offsets"]))
    return 10.0 * h


def _newton_schulz_flops(rows, cols):
    m, n = min(rows, cols), max(rows, cols)
    return NS_STEPS * (m * m * n + m ** 3 + 2.0 * m * m * n)     # the two symmetric products by half


def work(case):
    op = case["op"]
    if op == "orthogonalize":
        size = 4 if case["type"] == "f32" else 2
        n = case["batch"] * case["rows"] * case["cols"]
        return {"bytes": 2.0 * size * n, "flops": case["batch"] * _newton_schulz_flops(case["rows"], case["cols"])}
    if op == "muon":
        layers, dim = _layout(_sizes(case))
        return {"bytes": 28.0 * dim, "flops": sum(_newton_schulz_flops(r, c) for _, r, c, _ in layers)}
    # the weights of groups that have rows, at least: as many as there are rows
    if op == "grouped":
        size = 4 if case["type"] == "f32" else 2
        used = min(case["groups"], case["rows"])
        return {"bytes": float(size) * (used * (case["in"] * case["out"] + case["out"]) + case["rows"] * (case["in"] + case["out"])),
                "flops": 2.0 * case["rows"] * case["in"] * case["out"]}
    sizes = _sizes(case)
    layers, dim = _layout(sizes)
    return {"bytes": 4.0 * (min(case["members"], case["rows"]) * dim + case["rows"] * (sizes[0] + sizes[-1])),
            "flops": 2.0 * case["rows"] * sum(r * c for _, r, c, _ in layers)}
