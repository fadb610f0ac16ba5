"""The timed cases of the operators on embedding tables: rows taken out of the tables and gradients brought back into
them (training), scores of single queries against a table held in 4 bits, and what a caller knows applied to such scores
(answering).

Sizes are those of the repository's own workloads (2,000 to 1,000,000 entities, 8 to 1,345 relations, 32 to 200 dimensions)
and of the model sizes they stand in for (up to 512 dimensions).  Ids come as columns of an n x 3 array of triples.  Where
`own` is false, the same results come from elementary torch operations in float32.
"""
import math

import torch

own = False

GROUP = 32                                              # dimensions that share a scale in a 4-bit table
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)       # magnitudes of a 4-bit value; its top bit is the sign
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


# ---- cases ----
def _lookup(n, N, R, d, dtype, out, sb=1.0, pad=0, zipf=False):
    return {"op": "lookup", "n": n, "N": N, "R": R, "d": d, "dtype": dtype, "out": out, "sb": sb, "pad": pad, "zipf": zipf}


def _grad(n, N, d, dtype, out, both=False, pad=0, zipf=False):
    return {"op": "grad", "n": n, "N": N, "d": d, "dtype": dtype, "out": out, "both": both, "pad": pad, "zipf": zipf}


def _scores(n, N, d, dtype, out):
    return {"op": "scores", "n": n, "N": N, "d": d, "dtype": dtype, "out": out}


def _adjust(n, N, dtype, known, seen, masks, bias):
    return {"op": "adjust", "n": n, "N": N, "dtype": dtype, "known": known, "seen": seen, "masks": masks, "bias": bias}


def listed():
    cases = {
        # one query (h, r, ?): its connector row h + r from two tables
        "lookup_one": _lookup(1, 15_000, 1_345, 100, "f32", "f32"),
        # head queries t - r for every triple of a training epoch over a million entities, hubs among them, in bfloat16
        "lookup_epoch": _lookup(1_000_000, 1_000_000, 1_000, 128, "bf16", "bf16", sb=-1.0, zipf=True),
        # gradients of a small training batch into a small table; the batch's last rows are padding
        "grad_batch": _grad(128, 2_000, 32, "f32", "f32", pad=5),
        # an ordinary step: the heads' gradients, then the tails' added to them; hub entities occur thousands of times
        "grad_entities": _grad(32_771, 15_000, 100, "f32", "f32", both=True, zipf=True),
        # the relations' side of a large step: few rows, each a sum over thousands of triples
        "grad_relations": _grad(250_000, 18, 100, "f32", "f32"),
        # an epoch's gradients into a million entities, gradients in bfloat16, sums in float32
        "grad_epoch": _grad(1_000_000, 1_000_000, 128, "bf16", "f32", zipf=True),
        # one query against every entity of a mid-size graph
        "scores_one": _scores(1, 15_000, 100, "f32", "f32"),
        # a few queries against a million entities, the table streams from memory
        "scores_few": _scores(4, 1_000_000, 128, "bf16", "f32"),
        # a ranking batch
        "scores_batch": _scores(128, 100_000, 200, "f32", "f32"),
        # one answer: bias, the relation's allowed entities, known answers, penalties for entities named before
        "adjust_one": _adjust(1, 15_000, "f32", 40, 64, 1_345, True),
        # filtered ranking: the known answers of every query leave the scores, in place
        "adjust_known": _adjust(512, 40_000, "f32", 60, 0, 0, False),
        # all of it for a batch
        "adjust_batch": _adjust(256, 100_000, "bf16", 120, 500, 200, True),
    }
    return [{"name": name, **c} for name, c in cases.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(op):
    return max(sum(work(c).values()) for c in listed() if c["op"] == op)


def draw(rng):
    while True:
        op = rng.choice(["lookup", "grad", "grad", "scores", "scores", "adjust", "adjust"])
        d = rng.choice([32, 64, 100, 128, 200, 256, 512]) if rng.random() < 0.5 else _log_uniform(rng, 16, 512)
        dtype, out = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
        N = _log_uniform(rng, 500, 1_000_000)
        if op == "lookup":
            n = _log_uniform(rng, 1, 1_000_000)
            c = _lookup(n, N, rng.choice([0, _log_uniform(rng, 4, 1_500)]), d, dtype, out, sb=rng.choice([1.0, -1.0, 0.5]),
                        pad=rng.choice([0, n // 10]), zipf=rng.random() < 0.5)
        elif op == "grad":
            n = _log_uniform(rng, 1, 1_000_000)
            N = rng.choice([N, N, _log_uniform(rng, 4, 1_500)])
            c = _grad(n, N, d, dtype, out, both=rng.random() < 0.3, pad=rng.choice([0, n // 10]), zipf=rng.random() < 0.5)
        elif op == "scores":
            c = _scores(rng.choice([1, _log_uniform(rng, 1, 200)]), N, d, dtype, out)
        else:
            n = _log_uniform(rng, 1, 600)
            c = _adjust(n, N, dtype, rng.choice([0, _log_uniform(rng, 1, 2_000)]), rng.choice([0, _log_uniform(rng, 1, 2_000)]),
                        rng.choice([0, _log_uniform(rng, 1, 1_500)]), rng.random() < 0.5)
            if not (c["known"] or c["seen"] or c["masks"] or c["bias"]):
                continue
        if sum(work(c).values()) <= _most(op):
            return c


# ---- inputs ----
def _ids(c, g, n, N):
    """n ids below N; hubs by Zipf's law where the case asks for it; the last `pad` name no row."""
    if c["zipf"]:
        rank = torch.pow(float(N), torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).long().clamp_(max=N) - 1
        ids = torch.randperm(N, generator=g, device="cuda")[rank]
    else:
        ids = torch.randint(0, N, (n,), generator=g, device="cuda")
    if c["pad"]:
        ids[n - c["pad"]:] = -1
    return ids


def _normal(g, shape, dtype="f32"):
    return torch.randn(shape, generator=g, device="cuda").to(_TYPES[dtype])


def _lists(g, n, N, mean):
    """A list of entities for every row: offsets and ids; lengths from none to twice the mean."""
    length = torch.randint(0, 2 * mean + 1, (n,), generator=g, device="cuda")
    length[0] = mean
    offsets = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.cumsum(length, 0)
    ids = torch.randint(0, N, (int(offsets[-1]),), generator=g, device="cuda", dtype=torch.int32)
    return offsets, ids


def _quantise(W):
    """4-bit codes and scales of a table, as the packed table of the library holds them: over every GROUP dimensions the scale is
    the largest magnitude over 6, in bfloat16; a code is the nearest level, the even one of two that are as near."""
    N, d = W.shape
    groups = (d + GROUP - 1) // GROUP
    w = torch.zeros((N, groups * GROUP), dtype=torch.float32, device=W.device)
    w[:, :d] = W
    w = w.view(N, groups, GROUP)
    scale = (w.abs().amax(2) / 6.0).to(torch.bfloat16)
    s, a = scale.double()[..., None], w.abs().double()
    code = torch.zeros(w.shape, dtype=torch.uint8, device=W.device)
    for k in range(7):
        middle = 0.5 * (LEVELS[k] + LEVELS[k + 1]) * s
        code += ((a >= middle) if k % 2 else (a > middle)) & (s > 0)
    code += 8 * (w < 0).to(torch.uint8)
    return code.view(N, groups * GROUP), scale


def _inputs(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "lookup":
        given = {"E": _normal(g, (c["N"], c["d"]), c["dtype"])}
        given["triples"] = torch.zeros((c["n"], 3), dtype=torch.int32, device="cuda")
        given["triples"][:, 0] = _ids(c, g, c["n"], c["N"])
        if c["R"]:
            given["Rv"] = _normal(g, (c["R"], c["d"]), c["dtype"])
            given["triples"][:, 1] = torch.randint(0, c["R"], (c["n"],), generator=g, device="cuda")
    elif c["op"] == "grad":
        given = {"triples": torch.zeros((c["n"], 3), dtype=torch.int32, device="cuda")}
        given["triples"][:, 0] = _ids(c, g, c["n"], c["N"])
        given["triples"][:, 2] = _ids(c, g, c["n"], c["N"])
        given["G"] = _normal(g, (c["n"], c["d"]), c["dtype"])
    elif c["op"] == "scores":
        given = {"W": _normal(g, (c["N"], c["d"]), "bf16"), "x": _normal(g, (c["n"], c["d"]), c["dtype"])}
    else:
        n, N = c["n"], c["N"]
        given = {"scores": (-10.0 + 3.0 * torch.randn((n, N), generator=g, device="cuda")).to(_TYPES[c["dtype"]])}
        if c["bias"]:
            given["bias"] = _normal(g, (N,))
        if c["masks"]:
            given["allowed"] = torch.randint(-2**31, 2**31, (c["masks"], (N + 31) // 32), generator=g, device="cuda").to(torch.int32)
            given["relation"] = torch.randint(0, c["masks"], (n,), generator=g, device="cuda", dtype=torch.int32)
        if c["known"]:
            given["known"] = _lists(g, n, N, c["known"])
        if c["seen"]:
            # entities named before: hubs come up again and again
            given["seen"] = _lists(g, n, max(1, N // 50), c["seen"])
    return given


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["op"] == "scores":
        # a program keeps the packed table, not the table it was made from
        W = state.pop("W")
        if own:
            import paper_2307_12059_amd as kgc
            packer = kgc.Embed(dtype="bf16")
            state["table"] = packer.pack4(W)
            packer.close()
        else:
            code, scale = _quantise(W)
            state["levels"] = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda")
            t = state["levels"][code.long()].view(case["N"], -1, GROUP) * scale.float()[..., None]
            state["sq"] = (t.double() ** 2).sum((1, 2)).float()
            state["code"], state["scale"] = code[:, 0::2] | (code[:, 1::2] << 4), scale
    if own:
        import paper_2307_12059_amd as kgc
        state["embed"] = kgc.Embed(dtype=case["dtype"])
    return state


# ---- the plain form ----
def _rows(table, ids):
    got = table[ids.long().clamp(min=0)].float()
    return torch.where((ids >= 0)[:, None], got, torch.zeros((), device=got.device))


def _scatter(G, ids, N, sign):
    total = torch.zeros((N + 1, G.shape[1]), dtype=torch.float32, device=G.device)
    ids = ids.long()
    return total.index_add_(0, torch.where(ids >= 0, ids, N), G.float() * sign)[:N]


def _plain(state):
    c = state["case"]
    if c["op"] == "lookup":
        out = _rows(state["E"], state["triples"][:, 0])
        if c["R"]:
            out = out + c["sb"] * _rows(state["Rv"], state["triples"][:, 1])
        return out.to(_TYPES[c["out"]])
    if c["op"] == "grad":
        out = _scatter(state["G"], state["triples"][:, 0], c["N"], 1.0).to(_TYPES[c["out"]])
        if c["both"]:
            out = (out.float() + _scatter(state["G"], state["triples"][:, 2], c["N"], -1.0)).to(_TYPES[c["out"]])
        return out
    if c["op"] == "scores":
        code = torch.stack((state["code"] & 15, state["code"] >> 4), 2).view(c["N"], -1, GROUP)
        t = (state["levels"][code.long()] * state["scale"].float()[..., None]).view(c["N"], -1)[:, :c["d"]]
        return (2.0 * (state["x"].float() @ t.t()) - state["sq"]).to(_TYPES[c["out"]])
    scores, n, N = state["scores"], c["n"], c["N"]
    lists = {}
    for k in ("known", "seen"):
        if k in state:
            offsets, ids = state[k]
            row = torch.repeat_interleave(torch.arange(n, device="cuda"), offsets[1:] - offsets[:-1], output_size=ids.shape[0])
            lists[k] = row, ids.long()
    if not (c["bias"] or c["masks"] or c["seen"]):
        scores[lists["known"]] = -math.inf
        return scores
    x = scores.float()
    if c["bias"]:
        x = x + state["bias"]
    if c["seen"]:
        count = torch.zeros((n, N), device="cuda").index_put_(lists["seen"], torch.ones((), device="cuda"), accumulate=True)
        x = torch.where(count > 0, torch.where(x > 0, x / 1.25, x * 1.25) - (0.5 + 0.25 * count), x)
    if c["masks"]:
        words = state["allowed"][state["relation"].long()]
        bits = (words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bits.view(n, -1)[:, :N] != 0, x, -math.inf)
    if c["known"]:
        x[lists["known"]] = -math.inf
    return x.to(scores.dtype)


def run(state):
    if not own:
        return _plain(state)
    c, e = state["case"], state["embed"]
    if c["op"] == "lookup":
        t = state["triples"]
        if c["R"]:
            return e.lookup(state["E"], t[:, 0], state["Rv"], t[:, 1], sb=c["sb"], out_dtype=_TYPES[c["out"]])
        return e.lookup(state["E"], t[:, 0], out_dtype=_TYPES[c["out"]])
    if c["op"] == "grad":
        t = state["triples"]
        out = e.lookup_grad(state["G"], t[:, 0], N=c["N"], out_dtype=_TYPES[c["out"]])
        if c["both"]:
            e.lookup_grad(state["G"], t[:, 2], out=out, scale=-1.0, accumulate=True)
        return out
    if c["op"] == "scores":
        return e.scores4(state["table"], state["x"], alpha=2.0, beta=-1.0, c=state["table"].sq, out_dtype=_TYPES[c["out"]])
    listed_only = not (c["bias"] or c["masks"] or c["seen"])
    return e.adjust(state["scores"], bias=state.get("bias"), allowed=state.get("allowed"), mask_row=state.get("relation"),
                    known=state.get("known"), seen=state.get("seen"), repeat=1.25 if c["seen"] else 1.0,
                    presence=0.5 if c["seen"] else 0.0, frequency=0.25 if c["seen"] else 0.0,
                    out=state["scores"] if listed_only else None)


# ---- what a pass cannot do without ----
def _distinct(c, n, N):
    """How many different rows n ids name, about."""
    if c["zipf"]:                                       # row k is named with the chance ln(1 + 1/k) / ln N
        total, k = 0.0, 1.0
        while k < N:
            top = min(float(N), 1.25 * k + 1.0)
            p = math.log(top / k) / math.log(N) / (top - k)
            total += (top - k) * -math.expm1(-n * p)
            k = top
        return max(1.0, total)
    return max(1.0, -N * math.expm1(n * math.log1p(-1.0 / N)))


def work(case):
    c = case
    if c["op"] == "lookup":
        n, row = c["n"], c["d"]
        tables = _distinct(c, n, c["N"]) + (-c["R"] * math.expm1(n * math.log1p(-1.0 / c["R"])) if c["R"] else 0.0)
        return {"bytes": tables * row * _SIZE[c["dtype"]] + n * row * _SIZE[c["out"]] + n * (8.0 if c["R"] else 4.0),
                "flops": (2.0 if c["R"] else 0.0) * n * row}
    if c["op"] == "grad":
        calls = 2 if c["both"] else 1
        need = c["n"] * (c["d"] * _SIZE[c["dtype"]] + 4.0 * calls) + float(c["N"]) * c["d"] * _SIZE[c["out"]]
        return {"bytes": need, "flops": 1.0 * calls * c["n"] * c["d"]}
    if c["op"] == "scores":
        groups = (c["d"] + GROUP - 1) // GROUP
        table = c["N"] * (c["d"] / 2.0 + 2.0 * groups + 4.0)
        return {"bytes": table + c["n"] * (c["d"] * _SIZE[c["dtype"]] + c["N"] * float(_SIZE[c["out"]])), "flops": 2.0 * c["n"] * c["N"] * c["d"]}
    named = 4.0 * c["n"] * (c["known"] + c["seen"]) + 8.0 * c["n"]
    if not (c["bias"] or c["masks"] or c["seen"]):
        return {"bytes": named + c["n"] * c["known"] * float(_SIZE[c["dtype"]]), "flops": 0.0}
    masks = min(c["n"], c["masks"]) * c["N"] / 8.0
    return {"bytes": 2.0 * c["n"] * c["N"] * _SIZE[c["dtype"]] + masks + (4.0 * c["N"] if c["bias"] else 0.0) + named,
            "flops": (1.0 if c["bias"] else 0.0) * c["n"] * c["N"] + 4.0 * c["n"] * c["seen"]}


# ---- the definitions in 64 bits ----
def _table64(W):
    """What a 4-bit table of W stands for: the nearest level times the scale, entity by entity."""
    N, d = W.shape
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=W.device)
    out = torch.empty((N, d), dtype=torch.float64, device=W.device)
    for k in range(0, d, GROUP):
        w = W[:, k:k + GROUP].double()
        s = (w.abs().max(dim=1, keepdim=True).values.float() / 6.0).to(torch.bfloat16).double()
        away = (w.abs().unsqueeze(2) - levels * s.unsqueeze(2)).abs()
        near = away == away.min(dim=2, keepdim=True).values                 # one level, or the two of a tie
        even = near & (torch.arange(8, device=W.device) % 2 == 0)
        pick = torch.where(even.any(2), even.byte().argmax(2), near.byte().argmax(2))
        out[:, k:k + GROUP] = torch.sign(w) * levels[pick] * s
    return out


def exact(case, seed):
    c, state = case, _inputs(case, seed)
    if c["op"] == "lookup":
        def row(table, ids):
            padded = torch.cat((table.double(), torch.zeros((1, c["d"]), dtype=torch.float64, device="cuda")))
            return padded[torch.where(ids < 0, table.shape[0], ids.long())]
        out = row(state["E"], state["triples"][:, 0])
        return out + c["sb"] * row(state["Rv"], state["triples"][:, 1]) if c["R"] else out
    if c["op"] == "grad":
        out = torch.zeros((c["N"], c["d"]), dtype=torch.float64, device="cuda")
        for column, sign in ((0, 1.0), (2, -1.0)) if c["both"] else ((0, 1.0),):
            ids = state["triples"][:, column].long()
            used = torch.nonzero(ids >= 0)[:, 0]
            out.index_put_((ids[used],), sign * state["G"][used].double(), accumulate=True)
        return out
    if c["op"] == "scores":
        t = torch.cat([_table64(part) for part in state["W"].split(50_000)])
        return torch.cat([2.0 * state["x"].double() @ part.t() - (part * part).sum(1) for part in t.split(100_000)], dim=1)
    x = state["scores"].double()
    inf = torch.tensor(-math.inf, dtype=torch.float64, device="cuda")
    if c["bias"]:
        x += state["bias"].double()
    for k in ("seen", "known"):
        if k not in state:
            continue
        offsets, ids = state[k]
        at = torch.bucketize(torch.arange(ids.shape[0], device="cuda"), offsets[1:], right=True) * c["N"] + ids.long()
        flat = x.view(-1)
        if k == "known":
            flat[at] = inf
        else:
            at, times = torch.unique(at, return_counts=True)
            v = flat[at]
            flat[at] = torch.where(v > 0, v / 1.25, v * 1.25) - 0.5 - 0.25 * times.double()
    if c["masks"]:
        words = state["allowed"].long() & 0xFFFFFFFF
        for k in range(0, c["n"], 16):
            word = words[state["relation"][k:k + 16].long()]
            entity = torch.arange(c["N"], device="cuda")
            keep = (word[:, entity // 32] >> (entity % 32)) & 1
            x[k:k + 16] = torch.where(keep == 1, x[k:k + 16], inf)
    return x
