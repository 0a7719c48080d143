"""Performance cases of the operators that the feed-forward half of a decode step uses.

Three kinds of case (the field ``kind``):

* ``act``      nmm_gemv_nt_act, y = act(x . Wt^T + bias) + residual with Wt [N, K], or with Wt [2 N, K] the gated
               form act(gate) * up
* ``route``    nmm_moe_route, the experts of each token (softmax or sigmoid scores, a bias for balance, groups, top-k,
               weights) and the order in which the experts' products take the (token, expert) pairs
* ``experts``  nmm_moe_experts, the gated products of the chosen experts and their weighted sum

With ``own`` false every case is computed in its plain form, elementary torch operations in 32 bits (the router's scores
in 64, so that neighbours are told apart).
"""
import math

import torch

own = False

HIDDEN, INNER = 7168, 2048              # a layer's width and an expert's
MAX_WEIGHT = 16384 * 7168               # elements of the largest dense weight
MAX_PRODUCTS = 2048 * HIDDEN * INNER    # (pairs of the largest call) x a third of an expert's elements
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def listed():
    return [
        # the smallest call: a 512 x 512 product of one token, all launch latency
        {"name": "act_512", "kind": "act", "M": 1, "K": 512, "N": 512, "fp16": False, "act": "gelu", "gated": False,
         "bias": True, "residual": False},
        # the gate and up products of an expert that every token takes, one token
        {"name": "act_gated_1", "kind": "act", "M": 1, "K": HIDDEN, "N": INNER, "fp16": False, "act": "silu",
         "gated": True, "bias": False, "residual": False},
        # no size a multiple of a tile, everything in the epilogue, fp16
        {"name": "act_ragged_5", "kind": "act", "M": 5, "K": 4099, "N": 5003, "fp16": True, "act": "gelu_tanh",
         "gated": False, "bias": True, "residual": True},
        # the output projection of a batch of 32 onto the residual stream, the largest weight of a layer
        {"name": "act_w_o_32", "kind": "act", "M": 32, "K": 16384, "N": HIDDEN, "fp16": False, "act": "none",
         "gated": False, "bias": False, "residual": True},
        # the same expert's gate and up products for a prefill chunk
        {"name": "act_gated_256", "kind": "act", "M": 256, "K": HIDDEN, "N": INNER, "fp16": False, "act": "silu",
         "gated": True, "bias": False, "residual": False},
        # one token's experts among 256 in 8 groups, all launch latency
        {"name": "route_1", "kind": "route", "T": 1, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "group_top": 2, "renormalize": True, "scale": 2.5, "mask": False, "bf16": False},
        # a padded decode batch
        {"name": "route_64_masked", "kind": "route", "T": 64, "E": 256, "k": 8, "score": "sigmoid", "bias": True,
         "groups": 8, "top_groups": 4, "group_top": 2, "renormalize": True, "scale": 2.5, "mask": True, "bf16": False},
        # a prefill chunk, softmax over 60 experts, no groups
        {"name": "route_32767", "kind": "route", "T": 32767, "E": 60, "k": 6, "score": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_top": 1, "renormalize": False, "scale": 1.0, "mask": False, "bf16": False},
        # one token, 8 of 64 experts: the bytes of eight experts
        {"name": "experts_1", "kind": "experts", "T": 1, "E": 64, "first": 0, "local": 64, "k": 8, "hidden": HIDDEN,
         "inner": INNER, "fp16": False, "act": "silu", "residual": True},
        # a decode batch: every expert has a few rows
        {"name": "experts_64", "kind": "experts", "T": 64, "E": 64, "first": 0, "local": 64, "k": 8, "hidden": HIDDEN,
         "inner": INNER, "fp16": False, "act": "silu", "residual": True},
        # small experts of odd sizes, fp16, half of them on this GPU
        {"name": "experts_ragged_37", "kind": "experts", "T": 37, "E": 12, "first": 5, "local": 6, "k": 3, "hidden": 1037,
         "inner": 331, "fp16": True, "act": "gelu", "residual": False},
        # a prefill chunk on a GPU that holds a quarter of the experts, about 128 rows each
        {"name": "experts_1024_shard", "kind": "experts", "T": 1024, "E": 64, "first": 16, "local": 16, "k": 8,
         "hidden": HIDDEN, "inner": INNER, "fp16": False, "act": "silu", "residual": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size between lo and hi over its logarithm: half of them any number, half a multiple of 64."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.5 else max(lo, v // 64 * 64)


def draw(rng):
    kind = rng.choice(["act", "act", "route", "experts", "experts"])
    if kind == "act":
        M = 1 if rng.random() < 0.2 else _log(rng, 1, 256)
        gated = rng.random() < 0.5
        most = (MAX_WEIGHT if M <= 32 else HIDDEN * 2 * INNER) // (2 if gated else 1)
        K = _size(rng, 512, 16384)
        N = _size(rng, 256, min(16384, most // K))
        return {"kind": kind, "M": M, "K": K, "N": N, "fp16": rng.random() < 0.3, "act": rng.choice(ACTS),
                "gated": gated, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5}
    if kind == "route":
        groups = rng.choice([1, 1, 4, 8])
        E = groups * _log(rng, 2 if groups > 1 else 8, 256 // groups)
        top_groups = rng.randint(max(1, groups // 2), groups)
        k = rng.randint(1, min(8, top_groups * (E // groups)))
        return {"kind": kind, "T": _log(rng, 1, 2 ** 21 // E), "E": E, "k": k,
                "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "groups": groups,
                "top_groups": top_groups, "group_top": rng.choice([1, 2]) if groups > 1 else 1,
                "renormalize": rng.random() < 0.5, "scale": rng.choice([1.0, 2.5]), "mask": rng.random() < 0.3,
                "bf16": rng.random() < 0.3}
    E = _log(rng, 8, 64)
    local = E if rng.random() < 0.5 else rng.randint(max(1, E // 8), E)
    k = rng.randint(1, min(8, E))
    hidden, inner = _size(rng, 512, HIDDEN), _size(rng, 128, INNER)
    T = _log(rng, 1, max(1, min(1024, MAX_PRODUCTS * E // (k * local * hidden * inner))))
    return {"kind": kind, "T": T, "E": E, "first": rng.randint(0, E - local), "local": local, "k": k, "hidden": hidden,
            "inner": inner, "fp16": rng.random() < 0.3, "act": rng.choice(["silu", "gelu", "relu"]),
            "residual": rng.random() < 0.5}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 71)


def _normal(g, shape, dtype=torch.float32, sigma=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=g)


def _up8(n):
    return (n + 7) // 8 * 8


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    kind = case["kind"]
    dt = torch.float16 if case.get("fp16") else torch.bfloat16
    if kind == "act":
        M, K, N = case["M"], case["K"], case["N"]
        rows = 2 * N if case["gated"] else N
        s["x"] = _normal(g, (M, _up8(K)), dt)
        s["Wt"] = _normal(g, (rows, _up8(K)), dt, K ** -0.5)
        s["bias"] = _normal(g, (rows,), dt, 0.5) if case["bias"] else None
        s["residual"] = _normal(g, (M, N), dt) if case["residual"] else None
        s["y"] = torch.zeros((M, N), dtype=dt, device="cuda")
        return s
    T, E, k = case["T"], case["E"], case["k"]
    if kind == "route":
        s["logits"] = _normal(g, (T, E), torch.bfloat16 if case["bf16"] else torch.float32, 1.5)
        s["bias"] = _normal(g, (E,), sigma=0.1 if case["score"] == "sigmoid" else 0.3 / E) if case["bias"] else None
        s["mask"] = (torch.rand((T,), generator=g, device="cuda") < 0.8).to(torch.uint8) if case["mask"] else None
        s["out"] = (torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda"),
                    torch.zeros((E + 1,), dtype=torch.int32, device="cuda"),
                    torch.zeros((T * k,), dtype=torch.int32, device="cuda"))
        return s
    hidden, inner, local = case["hidden"], case["inner"], case["local"]
    # experts of uneven popularity
    score = _normal(g, (T, E)) + 0.3 * _normal(g, (E,))
    top, chosen = torch.sort(score, dim=1, descending=True, stable=True)
    s["chosen"] = chosen[:, :k].to(torch.int32).contiguous()
    w = torch.sigmoid(top[:, :k])
    s["weights"] = (w / w.sum(1, keepdim=True) * 2.5).contiguous()
    flat = s["chosen"].reshape(-1).long()
    s["pairs"] = torch.sort(flat, stable=True)[1].to(torch.int32)
    s["offsets"] = torch.zeros((E + 1,), dtype=torch.int32, device="cuda")
    s["offsets"][1:] = torch.cumsum(torch.bincount(flat, minlength=E), 0)
    s["x"] = _normal(g, (T, _up8(hidden)), dt)
    s["w1"] = _normal(g, (local, 2 * inner, _up8(hidden)), dt, hidden ** -0.5)
    s["w2"] = _normal(g, (local, hidden, _up8(inner)), dt, inner ** -0.5)
    s["residual"] = _normal(g, (T, hidden), dt) if case["residual"] else None
    s["y"] = torch.zeros((T, hidden), dtype=dt, device="cuda")
    return s


def _activation(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_plain(s):
    case = s["case"]
    K, N = case["K"], case["N"]
    z = s["x"][:, :K].float() @ s["Wt"][:, :K].float().T
    if case["bias"]:
        z = z + s["bias"].float()
    y = _activation(z[:, :N], case["act"])
    if case["gated"]:
        y = y * z[:, N:]
    if case["residual"]:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _route_plain(s):
    case = s["case"]
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    logits = s["logits"].double()
    if case["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-logits))
    else:
        score = torch.exp(logits - logits.amax(1, keepdim=True))
        score = score / score.sum(1, keepdim=True)
    choice = score + s["bias"].double() if case["bias"] else score
    if G > 1:
        best = torch.sort(choice.view(T, G, E // G), dim=2, descending=True)[0]
        group = best[:, :, :min(case["group_top"], E // G)].sum(2)
        kept = torch.sort(group, dim=1, descending=True, stable=True)[1][:, :case["top_groups"]]
        open_ = torch.zeros((T, G), dtype=torch.bool, device=logits.device).scatter_(1, kept, True)
        choice = torch.where(open_.repeat_interleave(E // G, 1), choice, -math.inf)
    chosen = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :k]
    w = torch.gather(score, 1, chosen)
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    w = (w * case["scale"]).float()
    flat = chosen.reshape(-1)
    if case["mask"]:
        live = s["mask"].bool()[:, None]
        chosen, w = torch.where(live, chosen, -1), torch.where(live, w, 0.0)
        flat = torch.where(live, chosen, E).reshape(-1)           # behind the last expert
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.zeros((E + 1,), dtype=torch.int32, device=logits.device)
    offsets[1:] = torch.cumsum(counts, 0)
    pairs = torch.sort(flat, stable=True)[1]
    # places behind the last pair are left as they were
    pairs = torch.where(torch.arange(T * k, device=pairs.device) < offsets[E], pairs, 0)
    return chosen.to(torch.int32), w, offsets, pairs.to(torch.int32)


def _experts_plain(s):
    case = s["case"]
    T, k, first, local = case["T"], case["k"], case["first"], case["local"]
    hidden, inner = case["hidden"], case["inner"]
    x, dt = s["x"][:, :hidden].float(), s["x"].dtype
    e = s["chosen"].reshape(-1).long() - first
    here = (e >= 0) & (e < local)
    if T * k <= local:
        # few pairs: each with its expert's weights
        at = e.clamp(0, local - 1)
        xp = x.repeat_interleave(k, 0)
        z = (s["w1"][at][:, :, :hidden].float() @ xp[:, :, None])[:, :, 0]
        h = _activation(z[:, :inner], case["act"]) * z[:, inner:]
        part = (s["w2"][at][:, :, :inner].float() @ h[:, :, None])[:, :, 0]
    else:
        # each expert's rows side by side, as many as the busiest has
        offsets = s["offsets"].long()
        most = max(1, int((offsets[first + 1:first + local + 1] - offsets[first:first + local]).max()))
        place = torch.empty_like(e)
        place[s["pairs"].long()] = torch.arange(T * k, device=e.device)
        place = place - offsets[(e + first).clamp(0, case["E"] - 1)]
        slot = torch.where(here, e * most + place, local * most)
        rows = torch.zeros((local * most + 1, hidden), device=x.device)
        rows[slot] = x.repeat_interleave(k, 0)
        rows = rows[:-1].view(local, most, hidden).transpose(1, 2).contiguous()
        z = s["w1"][:, :, :hidden].float() @ rows
        h = _activation(z[:, :inner], case["act"]) * z[:, inner:]
        part = (s["w2"][:, :, :inner].float() @ h.contiguous()).transpose(1, 2).reshape(local * most, hidden)
        part = part[slot.clamp(max=local * most - 1)]
    w = torch.where(here, s["weights"].reshape(-1), 0.0)
    y = (part * w[:, None]).view(T, k, hidden).sum(1)
    if case["residual"]:
        y = y + s["residual"].float()
    return y.to(dt)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2609_16009_amd as nmm

        if kind == "route":
            score = nmm.NMM_SCORE_SIGMOID if case["score"] == "sigmoid" else nmm.NMM_SCORE_SOFTMAX
            return nmm.nmm_moe_route(s["logits"], *s["out"], score=score, bias=s["bias"], groups=case["groups"],
                                     top_groups=case["top_groups"], group_top=case["group_top"],
                                     renormalize=case["renormalize"], scale=case["scale"], mask=s["mask"])
        act = {"none": nmm.NMM_ACT_NONE, "relu": nmm.NMM_ACT_RELU, "silu": nmm.NMM_ACT_SILU, "gelu": nmm.NMM_ACT_GELU,
               "gelu_tanh": nmm.NMM_ACT_GELU_TANH}[case["act"]]
        if kind == "act":
            return nmm.nmm_gemv_nt_act(s["x"], s["Wt"], s["y"], K=case["K"], act=act, gated=case["gated"],
                                       bias=s["bias"], residual=s["residual"])
        return nmm.nmm_moe_experts(s["x"], s["w1"], s["w2"], s["chosen"], s["weights"], s["offsets"], s["pairs"], s["y"],
                                   hidden=case["hidden"], inner=case["inner"], first=case["first"], act=act,
                                   residual=s["residual"])
    return {"act": _act_plain, "route": _route_plain, "experts": _experts_plain}[kind](s)


def work(case):
    kind = case["kind"]
    if kind == "act":
        M, K, N = case["M"], case["K"], case["N"]
        rows = 2 * N if case["gated"] else N
        return {"bytes": 2 * (rows * K + M * K + M * N * (2 if case["residual"] else 1) + (rows if case["bias"] else 0)),
                "flops": 2 * M * rows * K}
    T, E, k = case["T"], case["E"], case["k"]
    if kind == "route":
        return {"bytes": T * E * (2 if case["bf16"] else 4) + (4 * E if case["bias"] else 0) + (T if case["mask"] else 0) +
                12 * T * k + 4 * (E + 1), "flops": 10 * T * E}
    hidden, inner, local = case["hidden"], case["inner"], case["local"]
    active = local * (1 - (1 - k / E) ** T)            # experts that have a pair, all of them equally popular
    pairs = T * k * local / E
    return {"bytes": active * 6 * hidden * inner + T * hidden * (6 if case["residual"] else 4) + 20 * T * k + 4 * (E + 1),
            "flops": 6 * pairs * hidden * inner}


def _act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / 2 ** 0.5)
    if act == "gelu_tanh":
        # (1 + tanh(u)) / 2 is the logistic function of 2 u
        return z * torch.sigmoid((8 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
    return torch.maximum(z, torch.zeros_like(z)) if act == "relu" else z


def _route_exact(s):
    case = s["case"]
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    l = s["logits"].double()
    score = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.softmax(l, 1)
    c = score.clone()
    if case["bias"]:
        c += s["bias"].double()[None]
    index = torch.arange(E, device="cuda")
    if G > 1:
        rest = c.clone().view(T, G, -1)
        total = torch.zeros((T, G), dtype=torch.float64, device="cuda")
        for _ in range(min(case["group_top"], E // G)):
            v, i = rest.max(2)
            total += v
            rest.scatter_(2, i[..., None], -math.inf)
        # a group stays if fewer than top_groups come before it
        a, b = total[:, :, None], total[:, None, :]
        before = (b > a) | ((b == a) & torch.ones((G, G), dtype=torch.bool, device="cuda").tril(-1))
        c[(before.sum(2) >= case["top_groups"]).repeat_interleave(E // G, 1)] = -math.inf
    chosen = torch.empty((T, k), dtype=torch.long, device="cuda")
    for i in range(k):
        top = c.amax(1, keepdim=True)
        chosen[:, i] = torch.where(c == top, index, E).amin(1)
        c.scatter_(1, chosen[:, i:i + 1], -math.inf)
    w = score[torch.arange(T, device="cuda")[:, None], chosen]
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    w = w * case["scale"]
    if case["mask"]:
        chosen[s["mask"] == 0] = -1
        w[s["mask"] == 0] = 0
    offsets = (chosen.view(1, -1) < torch.arange(E + 1, device="cuda")[:, None]).sum(1) - (chosen < 0).sum()
    pairs = torch.zeros(T * k, dtype=torch.long, device="cuda")
    at = 0
    for e in range(E):
        mine = torch.nonzero(chosen.view(-1) == e)[:, 0]
        pairs[at:at + len(mine)] = mine
        at += len(mine)
    return chosen, w, offsets, pairs


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "route":
        return _route_exact(s)
    if kind == "act":
        K, N = case["K"], case["N"]
        x, y = s["x"].double()[:, :K], torch.empty((case["M"], N), dtype=torch.float64, device="cuda")
        for n in range(0, N, 1024):
            rows = slice(n, min(N, n + 1024))

            def product(first):
                at = slice(first + rows.start, first + rows.stop)
                z = (s["Wt"][at, :K].double() @ x.T.contiguous()).T
                return z + s["bias"][at].double() if case["bias"] else z

            v = _act64(product(0), case["act"])
            y[:, rows] = v * product(N) if case["gated"] else v
        return y + s["residual"].double() if case["residual"] else y
    T, hidden, inner = case["T"], case["hidden"], case["inner"]
    y = s["residual"].double() if case["residual"] else torch.zeros((T, hidden), dtype=torch.float64, device="cuda")
    x = s["x"].double()[:, :hidden]
    for e in range(case["local"]):
        t, i = torch.nonzero(s["chosen"] == case["first"] + e, as_tuple=True)
        if len(t) == 0:
            continue
        z = s["w1"][e, :, :hidden].double() @ x[t].T.contiguous()
        h = _act64(z[:inner], case["act"]) * z[inner:]
        out = (s["w2"][e, :, :inner].double() @ h).T * s["weights"][t, i].double()[:, None]
        y.index_add_(0, t, out)
    return y
