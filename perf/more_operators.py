"""What lies around the products of a routed layer, as cases that can be timed and checked: the choice of experts, the rows' way to
their experts and back, and the root-mean-square norm in front, with its gradients and its output in 8 bits.

    route         scores -> experts, weights, places, offsets (groot_route): softmax or sigmoid, a bias that counts for the choice
                  only, sets of neighbouring experts of which the best stay open, the top k, weights renormalised or not
    route_train   the same and the gradient of the scores (groot_route_backward)
    rows          rows copied to their experts' places (groot_routed_rows), in 8 bits with their scales too
    sum           out = addend + sum of weight x row at its place (groot_routed_sum): the experts' answers come back
    routed_train  both and their gradients: four calls (groot_routed_sum_backward, and groot_routed_sum for the rows' gradient)
    norm          h = x + residual, y = h / rms(h) x gain (groot_rms_norm), in the type, in 8 bits with a scale for each row, or both
    norm_train    the same with its gradients (groot_rms_norm_backward)

"padded": the last eighth of the batch holds no tokens: their scores are -inf, they have no experts and places of -1.
8-bit outputs are returned as the codes: every operation that leads to them is rounded by itself, so they are defined to the bit.
"""
import math

import torch

own = False

_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}
EPS = 1e-6
INF = float("inf")


def _lib():
    import paper_2511_18297_amd as G                       # only where `own` is true: a tree without the operators runs their plain forms
    return G


def _route_case(name, op, type, n, experts, k, gate, bias=False, sets=1, open_sets=1, set_best=1, renormalise=True, factor=1.0, padded=False):
    return dict(name=name, op=op, type=type, n=n, experts=experts, k=k, gate=gate, bias=bias, sets=sets, open_sets=open_sets,
                set_best=set_best, renormalise=renormalise, factor=factor, padded=padded)


def listed():
    return [
        # one token that is decoded, scores from a product in fp32
        _route_case("route_1_f32", "route", "f32", 1, 64, 4, "softmax"),
        # a decoding batch: many small experts, balanced by a bias, chosen within four of eight sets
        _route_case("route_decode_bf16", "route", "bf16", 128, 256, 8, "sigmoid", bias=True, sets=8, open_sets=4, set_best=2, factor=2.5),
        # prefill of long prompts
        _route_case("route_prefill_f32", "route", "f32", 65536, 128, 8, "softmax"),
        # a training batch, padded, weights as the softmax gives them
        _route_case("route_train_bf16", "route_train", "bf16", 16384, 64, 6, "softmax", sets=8, open_sets=3, renormalise=False, padded=True),
        # a decoding batch in 8 bits on its way to its experts
        dict(name="rows_decode_i8", op="rows", type="i8", n=128, K=2048, experts=32, k=4, padded=False),
        # the experts' answers to a prefill, weighted and added to the residual stream
        dict(name="sum_prefill_bf16", op="sum", type="bf16", n=8192, K=4096, experts=8, k=2, padded=False),
        # training step around the experts of a routed layer, padded batch
        dict(name="routed_train_bf16", op="routed_train", type="bf16", n=8192, K=2048, experts=16, k=4, padded=True),
        # odd sizes: hardly a row begins on 16 bytes
        dict(name="routed_train_odd_f16", op="routed_train", type="f16", n=3001, K=1001, experts=7, k=3, padded=True),
        # one token that is decoded
        dict(name="norm_1_bf16", op="norm", type="bf16", n=1, K=4096, residual=True, out="type"),
        # prefill of a served model: the norm's rows go to products in 8 bits
        dict(name="norm_serve_f16", op="norm", type="f16", n=8192, K=4096, residual=True, out="8bit"),
        # training step of a large model, the residual stream's gradient comes in beside the norm's
        dict(name="norm_train_bf16", op="norm_train", type="bf16", n=16384, K=4096, residual=True),
        # training step of a graph network's hidden features: a 512-bit multiplier x 4 at the hidden width
        dict(name="norm_train_nodes_f32_64", op="norm_train", type="f32", n=8374272, K=64, residual=False),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["route", "route", "route_train", "rows", "sum", "routed_train", "norm", "norm", "norm_train"])
    type = rng.choice(["f32", "bf16", "bf16", "f16"])
    padded = rng.random() < 0.3
    if op in ("route", "route_train"):
        experts = rng.choice([_log(rng, 2, 512), rng.choice([8, 16, 32, 64, 128, 160, 256])])
        k = min(experts, _log(rng, 1, 12))
        sets = rng.choice([s for s in (1, 1, 2, 4, 8) if experts % s == 0])
        set_best = rng.choice([1, min(2, experts // sets)])
        open_sets = rng.randint(min(sets, -(-k * sets // experts)), sets)
        n = _log(rng, 1, min(65536, (1 << 23) // experts))
        return dict(op=op, type=type, n=n, experts=experts, k=k, gate=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, sets=sets,
                    open_sets=open_sets, set_best=set_best, renormalise=rng.random() < 0.6, factor=rng.choice([1.0, 1.0, 2.5]), padded=padded)
    K = _log(rng, 32, 8192)
    if rng.random() < 0.7:                                  # widths are mostly whole multiples of 64
        K = -(-K // 64) * 64
    if op in ("norm", "norm_train"):
        n = _log(rng, 1, min(1 << 20, (1 << 25) // K))
        residual = rng.random() < 0.6
        if op == "norm":
            return dict(op=op, type=type, n=n, K=K, residual=residual, out=rng.choice(["type", "8bit", "both"]))
        return dict(op=op, type=type, n=n, K=K, residual=residual)
    experts = _log(rng, 2, 256)
    k = min(experts, _log(rng, 1, 10))
    if op == "rows" and rng.random() < 0.5:
        type = "i8"
    return dict(op=op, type=type, n=_log(rng, 1, (1 << 25) // (K * k)), K=K, experts=experts, k=k, padded=padded)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _tokens(case):
    """rows of the batch that hold a token"""
    return case["n"] - case["n"] // 8 if case["padded"] else case["n"]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, type=torch.float32):
        return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0, scale, generator=g).to(type)
    op, n, T = case["op"], case["n"], _TYPE[case["type"]]
    s = dict(case)
    if op in ("norm", "norm_train"):
        K = case["K"]
        s["out_type"], s["out_8bit"] = case.get("out") != "8bit", case.get("out") in ("8bit", "both")
        s["X"] = normal(n, K, type=T)
        s["residual"] = (normal(n, K) * torch.exp(normal(K, scale=0.5))).to(T) if case["residual"] else None   # a stream whose channels differ in size
        s["gain"] = (1 + normal(K, scale=0.1)).to(T)
        if op == "norm_train":
            s["dY"], s["dH"] = normal(n, K, scale=0.1, type=T), normal(n, K, scale=0.1, type=T) if case["residual"] else None
        return s
    E, k = case["experts"], case["k"]
    # what the experts' weights make of a token, experts liked by more tokens than others
    scores = normal(n, E, scale=1.5) + normal(E, scale=0.5)
    scores[_tokens(case):] = -INF
    if op in ("route", "route_train"):
        s["scores"] = scores.to(T)
        s["bias"] = normal(E, scale=0.05) if case["bias"] else None
        if op == "route_train":
            s["dweights"] = normal(n, k, scale=0.1)
        return s
    K = case["K"]
    taken, experts = torch.topk(scores, k)
    s["weights"] = torch.where(taken > -INF, torch.softmax(taken, 1), torch.zeros_like(taken))
    s["places"] = _places(torch.where(taken > -INF, experts, torch.full_like(experts, -1)))
    if op == "rows":
        if case["type"] == "i8":
            s["X"] = torch.clamp(torch.round(normal(n, K, scale=35.0)), -127, 127).to(T)
            s["scale"] = torch.exp(normal(n, scale=0.3)) / 127
        else:
            s["X"] = normal(n, K, type=T)
        return s
    s["Y"] = normal(n * k, K, type=T)                        # the experts' answers
    s["addend"] = normal(n, K, type=T)
    if op == "routed_train":
        s["X"] = normal(n, K, type=T)
        s["dout"], s["dR"] = normal(n, K, scale=0.1, type=T), normal(n * k, K, scale=0.1, type=T)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, n, T = s["op"], s["n"], _TYPE[s["type"]]
    like = lambda *shape, type=T: torch.zeros(shape, dtype=type, device="cuda")  # noqa: E731
    if op in ("route", "route_train"):
        k, E = s["k"], s["experts"]
        s["out"] = dict(chosen=like(n, k, type=torch.int32), weights=like(n, k, type=torch.float32), places=like(n, k, type=torch.int32),
                        offsets=like(E + 1, type=torch.int64))
        if op == "route_train":
            s["out"]["dscores"] = like(n, E)
        return s
    K = s["K"]
    if op in ("norm", "norm_train"):
        s["out"] = {"H": like(n, K)} if s["residual"] is not None else {}
        if op == "norm_train":
            s["out"].update(Y=like(n, K), rstd=like(n, type=torch.float32), dX=like(n, K), dgain=like(K))
            return s
        if s["out_type"]:
            s["out"]["Y"] = like(n, K)
        if s["out_8bit"]:
            s["out"].update(Q=like(n, K, type=torch.int8), q_scale=like(n, type=torch.float32))
        return s
    k = s["k"]
    s["out"] = {}
    if op in ("rows", "routed_train"):                       # rows behind the last place stay zeros
        s["out"]["R"] = like(n * k, K)
        if s["type"] == "i8":
            s["out"]["r_scale"] = like(n * k, type=torch.float32)
    if op in ("sum", "routed_train"):
        s["out"]["out"] = like(n, K)
    if op == "routed_train":
        s["out"].update(dY=like(n * k, K), dweights=like(n, k, type=torch.float32), dX=like(n, K))
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass, plain
# ---------------------------------------------------------------------------------------------------------------
def _places(experts):
    """Where (row, slot) comes when all are put in the order of their experts, rows in their own order; -1 without an expert."""
    flat = experts.reshape(-1).long()
    order = torch.sort(torch.where(flat < 0, torch.full_like(flat, 1 << 30), flat), stable=True).indices
    places = torch.empty_like(flat)
    places[order] = torch.arange(flat.numel(), device=flat.device)
    return torch.where(flat < 0, torch.full_like(flat, -1), places).reshape(experts.shape).int()


def _route_plain(s):
    """The choice in 64 bits: whole numbers come of values that can lie next to each other."""
    x, k, E, S = s["scores"].double(), s["k"], s["experts"], s["sets"]
    n, softmax = x.shape[0], s["gate"] == "softmax"
    broken = torch.isnan(x).any(1, keepdim=True) | ((x == INF).any(1, keepdim=True) & softmax)
    if softmax:
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - torch.where(top == -INF, torch.zeros_like(top), top))
        p = e / e.sum(1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-x))
    c = x if s["bias"] is None and s["set_best"] == 1 else p if s["bias"] is None else p + s["bias"].double()
    closed = (x == -INF) | ~(c > -INF) | broken
    c = torch.where(closed, torch.full_like(c, -INF), c)
    if s["open_sets"] < S:
        best = torch.sort(c.reshape(n, S, E // S), dim=2, descending=True).values[:, :, :s["set_best"]]
        value = torch.where(best > -INF, best, torch.zeros_like(best)).sum(2)
        value = torch.where(best[:, :, 0] > -INF, value, torch.full_like(value, -INF))
        order = torch.sort(value, dim=1, descending=True, stable=True).indices
        open_ = torch.zeros((n, S), dtype=torch.bool, device=x.device).scatter_(1, order[:, :s["open_sets"]], True)
        c = torch.where(open_.repeat_interleave(E // S, 1), c, torch.full_like(c, -INF))
    c, chosen = torch.sort(c, dim=1, descending=True, stable=True)
    c, chosen = c[:, :k], chosen[:, :k]
    taken = c > -INF
    if s["renormalise"]:
        u = torch.gather(x, 1, chosen)
        u = u if softmax else torch.clamp(u, max=0) - torch.log1p(torch.exp(-u.abs()))
        u = torch.where(taken, u, torch.full_like(u, -INF))
        q = torch.exp(u - torch.where(taken[:, :1], u.amax(1, keepdim=True), torch.zeros_like(u[:, :1])))
        w = q / q.sum(1, keepdim=True)
    else:
        w = torch.gather(p, 1, chosen)
    w = torch.where(taken, s["factor"] * w, torch.zeros_like(w))
    w = torch.where(broken, torch.full_like(w, float("nan")), w)
    chosen = torch.where(taken, chosen, torch.full_like(chosen, -1))
    counts = torch.zeros(E + 1, dtype=torch.int64, device=x.device).scatter_add_(0, chosen.reshape(-1) + 1, torch.ones_like(chosen.reshape(-1)))
    counts[0] = 0
    r = dict(chosen=chosen.int(), weights=w.float(), places=_places(chosen), offsets=torch.cumsum(counts, 0))
    if s["op"] == "route":
        return r
    dw = s["dweights"]
    d = torch.zeros((n, E), device=x.device).scatter_add_(1, chosen.clamp(min=0), torch.where(taken, dw, torch.zeros_like(dw)))
    if s["renormalise"]:
        q = torch.zeros((n, E), device=x.device).scatter_add_(1, chosen.clamp(min=0), torch.where(taken, w, torch.zeros_like(w)).float())
        ds = q * (d - torch.where(taken, dw * w.float(), torch.zeros_like(dw)).sum(1, keepdim=True) / s["factor"])
        ds = ds if softmax else ds * (1 / (1 + torch.exp(x))).float()
    elif softmax:
        ds = s["factor"] * p.float() * (d - (p.float() * d).sum(1, keepdim=True))
    else:
        ds = s["factor"] * d * (p * (1 / (1 + torch.exp(x)))).float()
    ds = torch.where((x == -INF) & ~broken, torch.zeros_like(ds), ds)
    r["dscores"] = ds.to(s["scores"].dtype)
    return r


def _rows_plain(s, out):
    places = s["places"].reshape(-1).long()
    held = places >= 0
    row = torch.arange(s["n"], device=places.device).repeat_interleave(s["k"])
    out["R"][places[held]] = s["X"][row[held]]
    if s["type"] == "i8":
        out["r_scale"][places[held]] = s["scale"][row[held]]


def _weighted(R, places, weights):
    """sum over the slots of weight x row at its place, in 32 bits; a slot without a place reads as a row of zeros"""
    n, k = places.shape
    rows = torch.where((places >= 0).reshape(-1, 1), R[places.reshape(-1).clamp(min=0).long()].float(), torch.zeros((), device=R.device))
    return (rows.reshape(n, k, -1) * weights[:, :, None]).sum(1)


def _routed_plain(s):
    out, T = s["out"], _TYPE[s["type"]]
    if s["op"] in ("rows", "routed_train"):
        _rows_plain(s, out)
    if s["op"] in ("sum", "routed_train"):
        out["out"].copy_(s["addend"].float() + _weighted(s["Y"], s["places"], s["weights"]))
    if s["op"] == "routed_train":
        n, k, K = s["n"], s["k"], s["K"]
        places, d = s["places"].reshape(-1).long(), s["dout"].float()
        held = places >= 0
        out["dY"][places[held]] = (s["weights"][:, :, None] * d[:, None, :]).reshape(n * k, K)[held].to(T)
        rows = torch.where(held[:, None], s["Y"][places.clamp(min=0)].float(), torch.zeros((), device=d.device))
        out["dweights"].copy_((rows.reshape(n, k, K) * d[:, None, :]).sum(2))
        out["dX"].copy_(_weighted(s["dR"], s["places"], torch.ones_like(s["weights"])))
    return out


def _norm_plain(s):
    """Every operation in 32 bits and rounded by itself, but the long sum: that and the root are in 64 bits, and rounded once."""
    T, K = _TYPE[s["type"]], s["K"]
    h = s["X"].float() if s["residual"] is None else (s["X"].float() + s["residual"].float()).to(T).float()
    g = s["gain"].float()
    rstd = (1 / torch.sqrt(h.double().square().sum(1, keepdim=True) / K + EPS)).float()
    y = (h * rstd) * g
    r = {} if s["residual"] is None else {"H": h.to(T)}
    if s["op"] == "norm":
        if s["out_type"]:
            r["Y"] = y.to(T)
        if s["out_8bit"]:
            scale = y.abs().amax(1, keepdim=True) * torch.tensor(1 / 127, dtype=torch.float32, device=y.device)
            r["Q"] = torch.where(scale > 0, torch.round(y / scale), torch.zeros_like(y)).to(torch.int8)
            r["q_scale"] = scale[:, 0]
        return r
    r.update(Y=y.to(T), rstd=rstd[:, 0])
    dy = s["dY"].float()
    a = dy * g
    dh = rstd * (a - h * (rstd * rstd * ((a * h).sum(1, keepdim=True) / K)))
    if s["dH"] is not None:
        dh = dh + s["dH"].float()
    r["dX"] = dh.to(T)
    r["dgain"] = (dy * (h * rstd)).sum(0).to(T)
    return r


# ---------------------------------------------------------------------------------------------------------------
# one pass through the framework
# ---------------------------------------------------------------------------------------------------------------
def _route_own(s):
    G, o = _lib(), s["out"]
    if "work" not in s:
        s["work"] = torch.empty(max(G.groot_route_workspace(s["n"], s["experts"], s["k"]), 16), dtype=torch.uint8, device="cuda")
    gate = G.GROOT_SOFTMAX if s["gate"] == "softmax" else G.GROOT_SIGMOID
    G.groot_route(s["scores"], s["bias"], o["chosen"], o["weights"], o["places"], o["offsets"], s["work"], gate=gate, sets=s["sets"],
                  open_sets=s["open_sets"], set_best=s["set_best"], renormalise=s["renormalise"], factor=s["factor"])
    if s["op"] == "route_train":
        G.groot_route_backward(s["scores"], o["chosen"], s["dweights"], o["dscores"], gate=gate, renormalise=s["renormalise"], factor=s["factor"])
    return o


def _routed_own(s):
    G, o, op = _lib(), s["out"], s["op"]
    if op == "rows":
        G.groot_routed_rows(s["X"], s["places"], o["R"], s.get("scale"), o.get("r_scale"))
        return o
    if op == "routed_train":
        G.groot_routed_rows(s["X"], s["places"], o["R"])
    G.groot_routed_sum(s["Y"], s["places"], s["weights"], s["addend"], o["out"])
    if op == "routed_train":
        G.groot_routed_sum_backward(s["dout"], s["Y"], s["places"], s["weights"], o["dY"], o["dweights"])
        G.groot_routed_sum(s["dR"], s["places"], None, None, o["dX"])
    return o


def _norm_own(s):
    G, o = _lib(), s["out"]
    if s["op"] == "norm":
        G.groot_rms_norm(s["X"], s["residual"], s["gain"], EPS, o.get("Y"), H=o.get("H"), Q=o.get("Q"), q_scale=o.get("q_scale"))
        return o
    if "work" not in s:
        need = G.groot_rms_norm_backward_workspace(s["n"], s["K"], s["X"].dtype)
        s["work"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    G.groot_rms_norm(s["X"], s["residual"], s["gain"], EPS, o["Y"], H=o.get("H"), rstd=o["rstd"])
    G.groot_rms_norm_backward(o.get("H", s["X"]), o["rstd"], s["gain"], s["dY"], o["dX"], o["dgain"], s["work"], dH=s["dH"])
    return o


def run(s):
    if s["op"] in ("route", "route_train"):
        return _route_own(s) if own else _route_plain(s)
    if s["op"] in ("norm", "norm_train"):
        return _norm_own(s) if own else _norm_plain(s)
    return _routed_own(s) if own else _routed_plain(s)


def work(case):
    """Every input once, every output once; of the routed rows those that a token has."""
    n, b = case["n"], _BYTES[case["type"]]
    if case["op"] in ("norm", "norm_train"):
        K = case["K"]
        bytes, flops = b * n * K * (3 if case["residual"] else 1) + b * K, 5 * n * K
        if case["op"] == "norm":
            kind = case["out"]
            return {"bytes": bytes + (b * n * K if kind != "8bit" else 0) + (n * K + 4 * n if kind != "type" else 0), "flops": flops}
        # Y out, dY (and dH) in, dX out, the gain's gradient; the rows themselves are read once
        return {"bytes": bytes + b * n * K * (4 if case["residual"] else 3) + 4 * n + b * K, "flops": 15 * n * K}
    k, E = case["k"], case["experts"]
    if case["op"] in ("route", "route_train"):
        bytes = b * n * E + 12 * n * k + 8 * (E + 1) + (4 * E if case["bias"] else 0)
        train = case["op"] == "route_train"
        return {"bytes": bytes + (b * n * E + 4 * n * k if train else 0), "flops": n * E * (8 if train else 4)}
    K, m = case["K"], _tokens(case)
    rows = b * m * K + b * m * k * K + 4 * n * k + (4 * m * (k + 1) if case["type"] == "i8" else 0)
    back = b * m * k * K + 2 * b * n * K + 8 * n * k
    if case["op"] == "rows":
        return {"bytes": rows, "flops": m * k * K}
    if case["op"] == "sum":
        return {"bytes": back, "flops": 2 * m * k * K}
    # and the answers' and weights' gradients, and the rows' gradient; places, weights and answers are read once
    return {"bytes": rows + back - 4 * n * k + b * n * K + b * m * k * K + 4 * n * k + b * m * k * K + b * n * K, "flops": 6 * m * k * K}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] in ("route", "route_train"):
        return _route_exact(s)
    return _norm_exact(s) if case["op"] in ("norm", "norm_train") else _routed_exact(s)


def _route_exact(s):
    x, n, E, k, S = s["scores"].double(), s["n"], s["experts"], s["k"], s["sets"]
    softmax, f = s["gate"] == "softmax", s["factor"]
    lp = x - torch.logsumexp(x, 1, keepdim=True) if softmax else torch.nn.functional.logsigmoid(x)
    p = torch.exp(lp)
    none = torch.isinf(x).all(1)                             # rows without a token
    c = p + (s["bias"].double() if s["bias"] is not None else 0)
    c = torch.where(torch.isinf(x), torch.full_like(c, -INF), c)
    if s["bias"] is None and s["set_best"] == 1:
        c = x.clone()
    if s["open_sets"] < S:
        sets = c.reshape(n, S, E // S)
        value = torch.topk(sets, s["set_best"], 2).values.sum(2)
        left = value.clone()
        keep = torch.zeros_like(value, dtype=torch.bool)
        for _ in range(s["open_sets"]):
            at = (left == left.amax(1, keepdim=True)).int().argmax(1, keepdim=True)
            keep.scatter_(1, at, True)
            left.scatter_(1, at, -INF)
        c = torch.where(keep[:, :, None], sets, torch.full_like(sets, -INF)).reshape(n, E)
    chosen = []
    for _ in range(k):
        at = (c == c.amax(1, keepdim=True)).int().argmax(1, keepdim=True)
        chosen.append(at)
        c = c.scatter(1, at, -INF)
    chosen = torch.cat(chosen, 1)
    l = torch.gather(lp, 1, chosen)
    w = f * (torch.softmax(l, 1) if s["renormalise"] else torch.exp(l))
    w[none] = 0
    r = dict(chosen=None, weights=w, places=None, offsets=None)
    if s["op"] == "route":
        return r
    dw = s["dweights"].double()
    ds = torch.zeros_like(x)
    if s["renormalise"]:
        dl = w * (dw - (w * dw).sum(1, keepdim=True) / f)    # gradient at the logarithms of the chosen probabilities
    else:
        dl = w * dw
    ds.scatter_(1, chosen, dl)
    if softmax:
        ds = ds - p * ds.sum(1, keepdim=True)
    else:
        ds = ds * torch.exp(torch.nn.functional.logsigmoid(-x))
    ds[none] = 0
    return dict(r, dscores=ds)


def _routed_exact(s):
    places, n, k, K = s["places"].long(), s["n"], s["k"], s["K"]
    r = {}
    if s["op"] in ("rows", "routed_train"):
        i, slot = torch.nonzero(places >= 0, as_tuple=True)
        r["R"] = None
        if s["type"] == "i8":                                # the rows' codes are whole numbers
            r["r_scale"] = torch.zeros(n * k, dtype=torch.float64, device="cuda").index_put_((places[i, slot],), s["scale"].double()[i])
        else:
            r["R"] = torch.zeros((n * k, K), dtype=torch.float64, device="cuda").index_put_((places[i, slot],), s["X"].double()[i])
    if s["op"] == "rows":
        return r
    out = s["addend"].double()
    dout = s["dout"].double() if s["op"] == "routed_train" else None
    dY = torch.zeros((n * k, K), dtype=torch.float64, device="cuda") if dout is not None else None
    dX, dweights = torch.zeros_like(out), torch.zeros((n, k), dtype=torch.float64, device="cuda")
    for slot in range(k):
        at = places[:, slot]
        i = torch.nonzero(at >= 0)[:, 0]
        at, w = at[i], s["weights"][i, slot].double()
        rows = s["Y"][at].double()
        out[i] += w[:, None] * rows
        if dout is not None:
            dY[at] = w[:, None] * dout[i]
            dweights[i, slot] = (rows * dout[i]).sum(1)
            dX[i] += s["dR"][at].double()
    r["out"] = out
    return r if dout is None else dict(r, dY=dY, dweights=dweights, dX=dX)


def _norm_exact(s):
    K, T = s["K"], s["X"].dtype
    h = s["X"].double()
    if s["residual"] is not None:
        h = (h + s["residual"].double()).to(T).double()      # the stream as it is held
    size = torch.linalg.vector_norm(h, dim=1, keepdim=True) / math.sqrt(K)
    inverse = 1 / torch.sqrt(size * size + EPS)
    unit, g = h * inverse, s["gain"].double()
    r = {} if s["residual"] is None else {"H": h}
    if s["op"] == "norm":
        if s["out_type"]:
            r["Y"] = unit * g
        if s["out_8bit"]:
            r.update(Q=None, q_scale=(unit * g).abs().amax(1) / 127)
        return r
    dy = s["dY"].double()
    r.update(Y=unit * g, rstd=inverse[:, 0], dgain=(dy * unit).sum(0))
    v = dy * g
    dh = (v - unit * (v * unit).mean(1, keepdim=True)) * inverse
    return dict(r, dX=dh if s["dH"] is None else dh + s["dH"].double())
