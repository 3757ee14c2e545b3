"""Performance cases of the operators that a mixture of members (or experts) is trained with: rows sorted by member and back, the
gradient of that and of the products grouped by member, and the clipped policy loss with its gradient.

With ``own`` false every case runs in plain torch operations (32-bit arithmetic, rounded once at the end); with ``own`` true it
makes the calls that a user of the library makes.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CLIP = (0.2, 0.28)      # how far a ratio may fall below and rise above 1
KL = 0.04
SCALE = 1.0


def _size(case):
    return 4 if case["type"] == "f32" else 2


def _rows(op, rows, choices, groups, cols, type_, dropped, **kw):
    return dict({"op": op, "rows": rows, "choices": choices, "groups": groups, "cols": cols, "type": type_, "dropped": dropped}, **kw)


def _products(groups, rows, n_in, n_out, type_, spread, activation, **kw):
    return dict({"op": "products_gradient", "groups": groups, "rows": rows, "in": n_in, "out": n_out, "type": type_, "spread": spread,
                 "activation": activation}, **kw)


def _policy(rows, actions, type_, masked, **kw):
    return dict({"op": "policy", "rows": rows, "actions": actions, "type": type_, "masked": masked}, **kw)


def listed():
    return [
        # one step of a small population whose observations arrive in any order: latency only
        _rows("sort", 64, 1, 16, 28, "f32", 0.1, name="sort_small"),
        # a batch of long rows for several experts each: bound by the rows' way to and from memory
        _rows("sort", 32768, 4, 64, 2048, "bf16", 0.02, name="sort_large_bf16"),
        # actions of two members for every observation, back in the observations' order
        _rows("combine", 64, 2, 16, 8, "f32", 0.1, name="combine_small"),
        # the way back of a large batch, two experts a row
        _rows("combine", 40000, 2, 64, 2048, "bf16", 0.02, name="combine_large_bf16"),
        # rows of odd length in the other 16-bit type, three experts each
        _rows("combine_gradient", 5003, 3, 24, 1001, "f16", 0.05, name="combine_gradient_odd_f16"),
        # eight experts a row
        _rows("combine_gradient", 16384, 8, 64, 1024, "bf16", 0.02, name="combine_gradient_large_bf16"),
        # a small mixture's hidden layer: latency only
        _products(8, 60, 64, 64, "f32", 0.2, "tanh", name="products_gradient_small"),
        # one layer of every member of the large population, a few rows each: bound by the weights and their gradients
        _products(4096, 16384, 128, 128, "f32", 0.3, "tanh", name="products_gradient_population"),
        # wide experts and many rows, some experts with far more of them than others
        _products(32, 8192, 1024, 4096, "bf16", 0.4, "none", name="products_gradient_wide_bf16"),
        # odd sizes in the other 16-bit type
        _products(12, 3001, 1000, 1501, "f16", 0.6, "relu", name="products_gradient_odd_f16"),
        # the answers of the addition task: twelve symbols
        _policy(1024, 12, "f32", False, name="policy_small"),
        # sequences over a large vocabulary, some symbols forbidden
        _policy(8192, 32000, "bf16", True, name="policy_large_bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sort", "combine", "combine_gradient", "products_gradient", "products_gradient", "policy"])
    type_ = rng.choice(["f32", "bf16", "f16"])
    size = 4 if type_ == "f32" else 2
    if op == "products_gradient":
        n_in, n_out = _log_int(rng, 4, 4096), _log_int(rng, 1, 4096)
        groups = min(_log_int(rng, 1, 4096), max(1, int(2.6e8 / size / (n_in * n_out))))
        rows = min(_log_int(rng, 1, 20000), max(1, int((3e10 if type_ != "f32" else 6e9) / (n_in * n_out))))
        return _products(groups, rows, n_in, n_out, type_, round(rng.uniform(0.0, 0.5), 2), rng.choice(["none", "tanh", "relu"]))
    if op == "policy":
        actions = _log_int(rng, 2, 130000)
        return _policy(min(_log_int(rng, 1, 65536), max(1, int(5e8 / size / actions))), actions, type_, rng.random() < 0.4)
    cols, choices, groups = _log_int(rng, 1, 4096), rng.randint(1, 8), _log_int(rng, 1, 4096)
    most = int(6e8 / (size * cols * (choices + 1) + 16 * choices)) if op != "combine_gradient" else int(5e8 / (size * cols * (2 * choices + 1) + 16 * choices))
    return _rows(op, min(_log_int(rng, 1, 65536), max(1, most)), choices, groups, cols, type_, round(rng.choice([0.0, rng.uniform(0.0, 0.5)]), 2))


def _offsets(groups, rows, spread, gen):
    """Ragged group sizes: shares drawn log-normally (spread 0: even), the remainders by chance; whole numbers that sum to `rows`."""
    share = torch.exp(torch.randn(groups, generator=gen, device="cuda", dtype=torch.float64) * spread * 2.0)
    edge = torch.cumsum(share, 0) * (rows / share.sum())
    phase = torch.rand(1, generator=gen, device="cuda", dtype=torch.float64)
    ends = torch.floor(edge + phase).clamp(0, rows).to(torch.int32)
    ends[-1] = rows
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), ends])


def _order(members, groups):
    """(offsets, source, place) of the stable order by member; pairs without a member have no place."""
    flat = members.reshape(-1).long()
    n = flat.numel()
    live = (flat >= 0) & (flat < groups)
    key = torch.where(live, flat, torch.full_like(flat, groups))
    order = torch.argsort(key, stable=True)
    offsets = torch.searchsorted(key[order], torch.arange(groups + 1, device=flat.device)).to(torch.int32)
    at = torch.arange(n, device=flat.device)
    place = torch.empty_like(flat)
    place[order] = at
    return (offsets, torch.where(at < offsets[-1], order, torch.full_like(order, -1)).to(torch.int32),
            torch.where(live, place, torch.full_like(place, -1)).to(torch.int32).view(members.shape))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    op, t, rows = case["op"], TYPES[case["type"]], case["rows"]
    if op == "products_gradient":
        groups, n_in, n_out = case["groups"], case["in"], case["out"]
        offsets = _offsets(groups, rows, case["spread"], gen)
        pitch = -(-(n_out * n_in + n_out) // 32) * 32          # a layer inside the members' parameter rows, and its gradient in rows like them
        theta = (normal(groups, pitch) / math.sqrt(n_in)).to(t)
        y = normal(rows, n_out)
        y = {"none": y, "tanh": torch.tanh(y), "relu": y.clamp_min(0.0)}[case["activation"]].to(t)
        return {"case": case, "x": normal(rows, n_in).to(t), "dy": (normal(rows, n_out) * 0.1).to(t), "y": y, "offsets": offsets,
                "weight": theta[:, :n_out * n_in].unflatten(1, (n_out, n_in)), "longest": int((offsets[1:] - offsets[:-1]).max())}
    if op == "policy":
        n = case["actions"]
        logits = torch.empty(rows, n, dtype=t, device="cuda")
        actions = torch.empty(rows, dtype=torch.int64, device="cuda")
        logp = torch.empty(rows, dtype=torch.float64, device="cuda")
        step = max(1, (1 << 26) // n)
        for a in range(0, rows, step):
            x = (2.0 * normal(min(step, rows - a), n)).to(t)
            chosen = (x.float() - torch.log(-torch.log(uniform(*x.shape).clamp(1e-30, 1.0 - 6e-8)))).argmax(1)
            if case["masked"]:
                x[(uniform(*x.shape) < 0.3).scatter_(1, chosen[:, None], False)] = -math.inf
            logits[a:a + step], actions[a:a + step] = x, chosen
            logp[a:a + step] = (x.double() - torch.logsumexp(x.double(), 1, keepdim=True)).gather(1, chosen[:, None])[:, 0]
        old = logp + 0.2 * normal(rows)
        # a ratio that lies on a border to the last bit is on either side of it by rounding alone: such rows are moved off it
        for border in (math.log(1.0 - CLIP[0]), math.log(1.0 + CLIP[1])):
            old = torch.where((logp - old - border).abs() < 1e-4, old + 4e-4, old)
        live = uniform(rows) >= 0.1                                 # the others are padding
        live[0] = True
        return {"case": case, "logits": logits, "actions": torch.where(live, actions, torch.full_like(actions, -1)), "old": old.float(),
                "ref": (logp + 0.3 * normal(rows)).float(), "advantage": normal(rows), "weights": live.float() / live.sum()}
    members = torch.randint(0, case["groups"], (rows, case["choices"]), generator=gen, device="cuda", dtype=torch.int32)
    members[uniform(rows, case["choices"]) < case["dropped"]] = -1
    n, cols = members.numel(), case["cols"]
    if op == "sort":
        return {"case": case, "members": members, "x": normal(rows, cols).to(t), "out": torch.zeros(n, cols, dtype=t, device="cuda")}
    _, _, place = _order(members, case["groups"])
    weights = torch.softmax(normal(rows, case["choices"]), 1)
    state = {"case": case, "place": place, "weights": weights, "y": normal(n, cols).to(t)}
    if op == "combine_gradient":
        state.update(d_out=normal(rows, cols).to(t), dy=torch.zeros(n, cols, dtype=t, device="cuda"))
    return state


def _plain_grouped(x, weight, offsets, longest, other=None):
    """Rows padded to the longest group and one batched product: of rows with weights, or (`other`) of rows with rows."""
    groups = offsets.numel() - 1
    row = torch.arange(x.shape[0], device=x.device)
    group = torch.searchsorted(offsets[1:], row.to(offsets.dtype), right=True)
    place = group * longest + row - offsets[group]

    def padded(rows):
        p = torch.zeros(groups * longest, rows.shape[1], device=rows.device)
        p[place] = rows
        return p.view(groups, longest, -1)
    if other is None:
        return torch.bmm(padded(x), weight).view(groups * longest, -1)[place]
    return torch.bmm(padded(x).transpose(1, 2), padded(other))


def _policy_rows(logits, actions, old, ref, advantage, weights):
    """(loss of every row times its weight, log probability of its action, gradient of its logits) in the inputs' precision."""
    live = (actions >= 0) & (weights != 0)
    a = actions.clamp_min(0)[:, None]
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    logp = (logits.gather(1, a) - top - torch.log(total))[:, 0]
    ratio = torch.exp(logp - old)
    inside = torch.where(advantage >= 0, ratio <= 1.0 + CLIP[1], ratio >= 1.0 - CLIP[0])
    surrogate = torch.minimum(ratio * advantage, ratio.clamp(1.0 - CLIP[0], 1.0 + CLIP[1]) * advantage)
    d = ref - logp
    loss = weights * (-surrogate + KL * (torch.exp(d) - d - 1.0))
    slope = weights * (torch.where(inside, -ratio * advantage, torch.zeros_like(ratio)) + KL * (1.0 - torch.exp(d)))
    zero = torch.zeros_like(logp)
    slope = torch.where(live, slope, zero)          # (a padded row's first action may be a forbidden one: 0 times infinity)
    gradient = e.div_(total).mul_(-slope[:, None])
    gradient.scatter_add_(1, a, slope[:, None])
    return torch.where(live, loss, zero), torch.where(live, logp, zero), gradient


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2202_05008_b200 as evo
        if op == "sort":
            routes = evo.route_rows(state["members"], case["groups"])
            rows = evo.take_rows(state["x"], routes.place, out=state["out"])
            return {"offsets": routes.offsets, "source": routes.source, "place": routes.place, "rows": rows}
        if op == "combine":
            return evo.combine_rows(state["y"], state["place"], state["weights"])
        if op == "combine_gradient":
            dy, dw = evo.combine_rows_backward(state["d_out"], state["y"], state["place"], state["weights"], out=state["dy"])
            return {"dy": dy, "dweights": dw}
        if op == "products_gradient":
            dx, dweight, dbias = evo.grouped_linear_backward(state["dy"], state["x"], state["weight"], state["offsets"],
                                                             state["y"], activation=case["activation"], scale=SCALE)
            return {"dx": dx, "dweight": dweight, "dbias": dbias}
        loss, logp, gradient = evo.policy_loss(state["logits"], state["actions"], state["old"], state["advantage"],
                                               ref_logp=state["ref"], weights=state["weights"], clip=CLIP, kl=KL)
        return {"loss": loss, "logp": logp, "gradient": gradient}
    if op == "sort":
        offsets, source, place = _order(state["members"], case["groups"])
        rows = torch.zeros_like(state["out"])
        live = place.reshape(-1) >= 0
        rows[place.reshape(-1)[live].long()] = state["x"].repeat_interleave(case["choices"], 0)[live]
        return {"offsets": offsets, "source": source, "place": place, "rows": rows}
    if op == "combine":
        y, place = state["y"], state["place"].long()
        total = torch.zeros(case["rows"], case["cols"], device=y.device)
        for j in range(case["choices"]):
            w = torch.where(place[:, j] >= 0, state["weights"][:, j], 0.0)
            total += w[:, None] * y[place[:, j].clamp_min(0)].float()
        return total.to(y.dtype)
    if op == "combine_gradient":
        y, place, d_out = state["y"], state["place"].long(), state["d_out"].float()
        dy, dw = torch.zeros_like(y), torch.zeros_like(state["weights"])
        for j in range(case["choices"]):
            live = place[:, j] >= 0
            at = place[live, j]
            dy[at] = (state["weights"][live, j, None] * d_out[live]).to(y.dtype)
            dw[live, j] = (d_out[live] * y[at].float()).sum(1)
        return {"dy": dy, "dweights": dw}
    if op == "products_gradient":
        x, offsets, y = state["x"], state["offsets"], state["y"].float()
        dz = state["dy"].float()
        if case["activation"] == "tanh":
            dz = dz * ((1.0 - y) * (1.0 + y))
        elif case["activation"] == "relu":
            dz = torch.where(y > 0, dz, torch.zeros_like(dz))
        dx = _plain_grouped(dz, state["weight"].float(), offsets, state["longest"])
        dweight = _plain_grouped(dz, None, offsets, state["longest"], x.float())
        dbias = _plain_grouped(dz, None, offsets, state["longest"], torch.ones(x.shape[0], 1, device=x.device))[:, :, 0]
        return {"dx": dx.to(x.dtype), "dweight": dweight.to(x.dtype), "dbias": dbias.to(x.dtype)}
    loss, logp, gradient = _policy_rows(state["logits"].float(), state["actions"], state["old"], state["ref"], state["advantage"], state["weights"])
    return {"loss": loss.sum(dtype=torch.float64).float(), "logp": logp, "gradient": gradient.to(state["logits"].dtype)}


def _exact_policy(state):
    """Row blocks, by the log-sum-exp and the derivative written out."""
    logits, rows, n = state["logits"], state["case"]["rows"], state["case"]["actions"]
    loss = torch.zeros((), dtype=torch.float64, device=logits.device)
    logp = torch.zeros(rows, dtype=torch.float64, device=logits.device)
    gradient = torch.zeros(rows, n, dtype=torch.float64, device=logits.device)
    step = max(1, (1 << 25) // n)
    for first in range(0, rows, step):
        part = slice(first, min(rows, first + step))
        index = torch.nonzero((state["actions"][part] >= 0) & (state["weights"][part] != 0))[:, 0]
        if index.numel() == 0:
            continue
        pick = {k: state[k][part][index].double() for k in ("old", "ref", "advantage", "weights")}
        chosen = state["actions"][part][index]
        x = logits[part][index].double()
        lp = x - torch.logsumexp(x, 1, keepdim=True)
        mine = lp[torch.arange(index.numel(), device=x.device), chosen]
        ratio, adv = torch.exp(mine - pick["old"]), pick["advantage"]
        low, high = 1.0 - CLIP[0], 1.0 + CLIP[1]
        bounded = torch.where(ratio < low, torch.full_like(ratio, low), torch.where(ratio > high, torch.full_like(ratio, high), ratio))
        clipped = bounded * adv < ratio * adv
        gap = pick["ref"] - mine
        loss += (pick["weights"] * (KL * (torch.expm1(gap) - gap) - torch.where(clipped, bounded, ratio) * adv)).sum()
        slope = pick["weights"] * (-KL * torch.expm1(gap) - torch.where(clipped, torch.zeros_like(ratio), ratio * adv))
        g = -slope[:, None] * torch.exp(lp)
        g[torch.arange(index.numel(), device=x.device), chosen] += slope
        gradient[first + index] = g
        logp[first + index] = mine
    return {"loss": loss, "logp": logp, "gradient": gradient}


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "policy":
        return _exact_policy(state)
    if op == "products_gradient":
        x, dy, y, weight = (state[k].double() for k in ("x", "dy", "y", "weight"))
        slope = {"none": torch.ones_like(y), "tanh": 1.0 - y * y, "relu": (y > 0).double()}[case["activation"]]
        dz = dy * slope
        dx = torch.zeros_like(x)
        dweight, dbias = torch.zeros_like(weight), torch.zeros(weight.shape[:2], dtype=torch.float64, device=x.device)
        edges = state["offsets"].tolist()
        for g, (first, last) in enumerate(zip(edges[:-1], edges[1:])):
            if last > first:
                dx[first:last] = dz[first:last] @ weight[g]
                dweight[g] = dz[first:last].t() @ x[first:last]
                dbias[g] = dz[first:last].sum(0)
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    rows, choices = case["rows"], case["choices"]
    if op == "sort":
        flat = state["members"].reshape(-1).long()
        pair = torch.nonzero(flat >= 0)[:, 0]
        source = pair[torch.argsort(flat[pair] * flat.numel() + pair)]
        counts = torch.bincount(flat[pair], minlength=case["groups"])
        place = torch.full_like(flat, -1)
        place[source] = torch.arange(source.numel(), device=flat.device)
        behind = torch.full((flat.numel() - source.numel(),), -1, dtype=torch.int64, device=flat.device)
        sorted_rows = torch.zeros(flat.numel(), case["cols"], dtype=torch.float64, device=flat.device)
        sorted_rows[:source.numel()] = state["x"][source // choices].double()
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=flat.device), torch.cumsum(counts, 0)])
        return {"offsets": offsets.to(torch.int32), "source": torch.cat([source, behind]).to(torch.int32),
                "place": place.view(rows, choices).to(torch.int32), "rows": sorted_rows}
    place = state["place"].reshape(-1).long()
    pair = torch.nonzero(place >= 0)[:, 0]
    row, at, weight = pair // choices, place[pair], state["weights"].reshape(-1)[pair].double()
    if op == "combine":
        total = torch.zeros(rows, case["cols"], dtype=torch.float64, device=place.device)
        return total.index_add_(0, row, weight[:, None] * state["y"][at].double())
    dy = torch.zeros(state["dy"].shape, dtype=torch.float64, device=place.device)
    dw = torch.zeros(rows * choices, dtype=torch.float64, device=place.device)
    step = max(1, (1 << 26) // case["cols"])
    for first in range(0, pair.numel(), step):
        part = slice(first, first + step)
        d_out = state["d_out"][row[part]].double()
        dy[at[part]] = weight[part, None] * d_out
        dw[pair[part]] = (d_out * state["y"][at[part]].double()).sum(1)
    return {"dy": dy, "dweights": dw.view(rows, choices)}


def work(case):
    op, rows, size = case["op"], case["rows"], float(_size(case))
    if op == "products_gradient":
        # the weights of groups that have rows, at least as many as there are rows; the gradient of all
        n_in, n_out = case["in"], case["out"]
        outputs = 1 if case["activation"] == "none" else 2
        return {"bytes": size * (min(case["groups"], rows) * n_in * n_out + case["groups"] * (n_in * n_out + n_out) + rows * (2 * n_in + outputs * n_out)),
                "flops": 4.0 * rows * n_in * n_out}
    if op == "policy":
        # padded rows are not read
        return {"bytes": size * rows * case["actions"] * 1.9 + 28.0 * rows, "flops": 6.0 * rows * case["actions"]}
    pairs, cols = rows * case["choices"], case["cols"]
    live = pairs * (1.0 - case["dropped"])
    if op == "sort":
        return {"bytes": size * cols * (rows + live) + 12.0 * pairs + 4.0 * case["groups"], "flops": 0.0}
    if op == "combine":
        return {"bytes": size * cols * (rows + live) + 8.0 * pairs, "flops": 2.0 * live * cols}
    return {"bytes": size * cols * (rows + 2 * live) + 12.0 * pairs, "flops": 3.0 * live * cols}
