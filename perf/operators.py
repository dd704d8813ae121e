"""Operators of a placement policy, as cases whose time is measured.

A search over placements keeps logits over the resources for every op (a
policy), draws the placements of a batch of scenarios from them, replays them,
and learns from the iteration times: draw (``sample``), log-probability of
every scenario's placement (``logp``), its weighted gradient (``grad``), and
distillation from a table of another policy's best resources (``distill``).
``prepare`` makes what such a search holds before the call, ``run`` makes one
call, or computes the same in elementary torch operations where ``own`` is
false; ``exact`` computes it in 64 bits from the definition.

Scenario s belongs to policy s // run (``run`` scenarios each, the last policy
fewer where the count is ragged).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
_INF = float("inf")


def listed():
    return [
        # one scenario of the smallest graph (data-parallel MLP): a step of a search that replays one placement at a time
        {"name": "sample one", "op": "sample", "n_pol": 1, "ops": 42, "res": 3, "run": 1, "scen": 1, "type": "fp32", "cut": "none"},
        # every scenario of the random layered graph's sweep drawn from one policy
        {"name": "sample sweep", "op": "sample", "n_pol": 1, "ops": 20000, "res": 64, "run": 16384, "scen": 16384, "type": "fp32", "cut": "none"},
        # BERT-large on 16 workers: 12 policies with exploration settings of their own, 4096 scenarios each
        {"name": "sample settings", "op": "sample", "n_pol": 12, "ops": 6624, "res": 48, "run": 4096, "scen": 49152, "type": "bf16", "cut": "each"},
        # logits from a network that saw the scenario: every scenario has its own, cut to the best eight and 90 %
        {"name": "sample conditional", "op": "sample", "n_pol": 1024, "ops": 6624, "res": 48, "run": 1, "scen": 1024, "type": "bf16", "cut": "one"},
        # ResNet-50 on 17 resources (an odd row length), an odd number of scenarios
        {"name": "sample odd", "op": "sample", "n_pol": 1, "ops": 4574, "res": 17, "run": 1001, "scen": 1001, "type": "fp16", "cut": "minp"},
        # how probable each placement of the sweep is under the policy now (importance weights)
        {"name": "logp sweep", "op": "logp", "n_pol": 1, "ops": 20000, "res": 64, "run": 16384, "scen": 16384, "type": "fp32"},
        {"name": "logp conditional", "op": "logp", "n_pol": 1024, "ops": 6624, "res": 48, "run": 1, "scen": 1024, "type": "bf16"},
        # the policy gradient of the sweep, and of a network's logits
        {"name": "grad sweep", "op": "grad", "n_pol": 1, "ops": 20000, "res": 64, "run": 16384, "scen": 16384, "type": "fp32"},
        {"name": "grad conditional", "op": "grad", "n_pol": 1024, "ops": 6624, "res": 48, "run": 1, "scen": 1024, "type": "bf16"},
        # a policy of the smallest graph started from a table of the two best resources per op
        {"name": "distill one", "op": "distill", "n_pol": 1, "ops": 42, "res": 3, "top": 2, "type": "fp32"},
        # the twelve BERT policies from the eight best resources per op
        {"name": "distill settings", "op": "distill", "n_pol": 12, "ops": 6624, "res": 48, "top": 8, "type": "bf16"},
        # near the largest resource count (1024), not a multiple of a vector of lanes
        {"name": "distill wide", "op": "distill", "n_pol": 16, "ops": 20000, "res": 1001, "top": 32, "type": "fp32"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "logp", "grad", "distill"])
    case = {"op": op, "type": rng.choice(["fp32", "bf16", "fp16"]), "res": _log_int(rng, 2, 1024)}
    if op == "distill":
        case["top"] = _log_int(rng, 1, min(64, case["res"]))
        case["n_pol"] = _log_int(rng, 1, 64)
        case["ops"] = _log_int(rng, 1, max(1, min(20000, 320_000_000 // (case["res"] * case["n_pol"]))))
        return case
    if rng.random() < 0.4:  # a policy per scenario, or per few of them
        case["n_pol"], case["run"] = _log_int(rng, 1, 1024), rng.choice([1, 1, 1, 2, 5, 16])
    else:  # policies that many scenarios share
        case["n_pol"], case["run"] = rng.choice([1, 1, 1, 2, 3, 12]), _log_int(rng, 1, 16384)
    case["scen"] = case["n_pol"] * case["run"] - (rng.randint(0, case["run"] - 1) if rng.random() < 0.5 else 0)
    most = min(320_000_000 // (case["res"] * case["n_pol"]), 320_000_000 // case["scen"])
    case["ops"] = _log_int(rng, 1, max(1, min(20000, most)))
    if op == "sample":
        case["cut"] = rng.choice(["none", "one", "minp", "each"])
    return case


def _settings(case, gen):
    """float32 [n_pol, 4] on the host: temperature, top_k, top_p, min_p of each policy."""
    P, R = case["n_pol"], case["res"]
    row = {"none": (1.0, 0.0, 1.0, 0.0), "one": (0.75, float(min(8, R)), 0.9, 0.0), "minp": (1.25, 0.0, 1.0, 0.05)}
    if case.get("cut", "none") != "each":
        return torch.tensor(row[case.get("cut", "none")], dtype=torch.float32).expand(P, 4)
    x = torch.rand((P, 4), generator=gen)
    return torch.stack([0.5 + x[:, 0], torch.floor(1 + x[:, 1] * R), 0.5 + 0.5 * x[:, 2], 0.1 * x[:, 3]], 1)


def _inputs(case, seed):
    """What the case's operator reads, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.Generator().manual_seed(seed)
    P, N, R = case["n_pol"], case["ops"], case["res"]
    dev = "cuda"
    # trained logits: spread over a few units; half of the ops may only run on the first half of the resources
    allowed = torch.where(torch.rand(N, generator=g, device=dev) < 0.5, R // 2 + 1, R)
    x = torch.randn((P, N, R), generator=g, device=dev).mul_(1.5)
    x.masked_fill_(torch.arange(R, device=dev) >= allowed[:, None], -_INF)
    s = {"op": case["op"], "logits": x.to(_TYPES[case["type"]]), "run": case.get("run", 1), "knobs": _settings(case, h).cuda()}
    s["cut"] = case.get("cut", "none")
    if case["op"] == "distill":
        K = case["top"]
        t = torch.randn((P, N, R), generator=g, device=dev).masked_fill_(torch.arange(R, device=dev) >= allowed[:, None], -_INF)
        t, i = torch.topk(t, K, dim=-1)
        s["top_logits"] = (2 * t).to(_TYPES[case["type"]])
        s["top_res"] = torch.where(torch.isinf(t), 65535, i).to(torch.uint16)  # ops with fewer choices than K: padded
        s["weight"] = torch.rand((P, N), generator=g, device=dev)
        return s
    S = case["scen"]
    u = torch.rand((N, S), generator=g, device=dev)
    if case["op"] == "sample":
        s["u"] = u
        return s
    # choices of a trained policy: some resources far more often than others, another order for every op
    shift = torch.randint(0, R, (N, 1), generator=g, device=dev)
    a = u.square_().mul_(allowed[:, None]).to(torch.int32)
    s["place"] = a.add_(shift).remainder_(allowed[:, None]).to(torch.uint16)
    if case["op"] == "grad":
        s["weight"] = torch.randn(S, generator=g, device=dev)  # standardised advantages
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2002_06790_amd as mlsim
        k = s["knobs"]
        if s["cut"] == "each":
            s["policy"] = mlsim.Policy(s["logits"], block=s["run"], temperature=k[:, 0], top_k=k[:, 1], top_p=k[:, 2], min_p=k[:, 3])
        else:
            t, k, p, m = k[0].tolist()
            s["policy"] = mlsim.Policy(s["logits"], block=s["run"], temperature=t, top_k=int(k), top_p=p, min_p=m)
    return s


def _by_policy(x, P, run):
    """[N, S] -> [P, N, run]: the scenarios of each policy, zeros behind the last."""
    N, S = x.shape
    if S < P * run:
        x = torch.cat([x, x.new_zeros((N, P * run - S))], 1)
    return x.view(N, P, run).transpose(0, 1)


def _sample(s):
    k = s["knobs"].double()
    T, top_k, top_p, min_p = (k[:, i, None, None] for i in range(4))
    x = s["logits"].double()
    P, N, R = x.shape
    w = torch.exp((x - x.amax(-1, keepdim=True)) / T)
    if s["cut"] != "none":
        ws, order = torch.sort(x, dim=-1, descending=True, stable=True)
        ws = torch.gather(w, -1, order)
        at = torch.arange(R, device=x.device)
        keep = (at < top_k) | (top_k < 1)
        m = ws * keep
        c = torch.cumsum(m, -1)
        before = torch.cat([torch.zeros_like(c[..., :1]), c[..., :-1]], -1)
        keep = keep & ((before < top_p * c[..., -1:]) | (top_p >= 1)) & (ws >= min_p) | (at == 0)
        w = torch.zeros_like(w).scatter_(-1, order, ws * keep)
    c = torch.cumsum(w, -1)
    u = s["u"]
    target = _by_policy(u.double(), P, s["run"]) * c[..., -1:]
    got = torch.searchsorted(c, target.contiguous(), right=True)
    place = got.transpose(0, 1).reshape(N, -1)[:, :u.shape[1]]
    return place.to(torch.int16)  # uint16 by its bits


def _log_pi(s):
    """float32 [P, N, R] log-probabilities, and the temperatures [P, 1, 1]."""
    T = s["knobs"][:, 0, None, None]
    x = s["logits"].float()
    d = (x - x.amax(-1, keepdim=True)) / T
    return d - torch.log(torch.exp(d).sum(-1, keepdim=True)), T


def _logp(s):
    lp, _ = _log_pi(s)
    N, S = s["place"].shape
    P = lp.shape[0]
    got = torch.gather(lp, -1, _by_policy(s["place"].to(torch.int64), P, s["run"]))
    return got.sum(1, dtype=torch.float64).reshape(-1)[:S].float()


def _grad(s):
    lp, T = _log_pi(s)
    P = lp.shape[0]
    a = _by_policy(s["place"].to(torch.int64), P, s["run"])
    w = _by_policy(s["weight"][None, :], P, s["run"])
    h = torch.zeros_like(lp).scatter_add_(-1, a, w.expand_as(a))
    return ((h - h.sum(-1, keepdim=True) * torch.exp(lp)) / T).to(s["logits"].dtype)


def _distill(s):
    lp, T = _log_pi(s)
    R = lp.shape[-1]
    i = s["top_res"].to(torch.int64)
    t = torch.where(i < R, s["top_logits"].float(), -_INF) / T
    t = torch.exp(t - t.amax(-1, keepdim=True))
    t = t / t.sum(-1, keepdim=True)
    q = torch.zeros_like(lp[..., :1]).expand(*lp.shape[:-1], R + 1).contiguous().scatter_add_(-1, i.clamp_(max=R), t)[..., :R]
    loss = torch.where(q > 0, q * (torch.log(q) - lp), 0.0).sum(-1)
    grad = s["weight"][..., None] * (torch.exp(lp) - q) / T
    return {"loss": loss, "grad": grad.to(s["logits"].dtype)}


def run(state):
    s = state
    op = s["op"]
    if not own:
        return {"sample": _sample, "logp": _logp, "grad": _grad, "distill": _distill}[op](s)
    policy = s["policy"]
    if op == "sample":
        return policy.sample(s["u"]).view(torch.int16)
    if op == "logp":
        return policy.logp(s["place"])
    if op == "grad":
        return policy.grad(s["place"], s["weight"])
    loss, grad = policy.distill(s["top_res"], s["top_logits"], weight=s["weight"])
    return {"loss": loss, "grad": grad}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "sample" and case["ops"] * max(case["scen"], case["n_pol"]) * case["res"] > 20_000_000:
        return None  # counted pair by pair below
    x = s["logits"].double()
    P, N, R = x.shape
    T = s["knobs"][:, 0].double().view(P, 1, 1)
    if case["op"] == "sample":
        return _sample_exact(s, x, T)
    z = x / T
    lse = torch.logsumexp(z, -1, keepdim=True)
    pi = torch.exp(z - lse)
    if case["op"] == "distill":
        i = s["top_res"].to(torch.int64)
        y = s["top_logits"].double() / T
        y = torch.softmax(y.masked_fill(i >= R, -_INF), -1)
        picked = torch.gather(z, -1, i.clamp(max=R - 1))
        loss = torch.xlogy(y, y).sum(-1) - torch.where(i < R, y * (picked - lse), 0.0).sum(-1)
        pi.scatter_add_(-1, i.clamp(max=R - 1), -y)  # padded entries have y = 0
        return {"loss": loss, "grad": pi.mul_(s["weight"].double()[..., None] / T)}
    place, run_ = s["place"], s["run"]
    S = place.shape[1]
    if case["op"] == "logp":
        total = torch.empty(S, dtype=torch.float64, device=x.device)
        for p in range(P):
            part = slice(p * run_, min(S, (p + 1) * run_))
            total[part] = torch.gather(z[p] - lse[p], 1, place[:, part].to(torch.int64)).sum(0)
        return total
    w = s["weight"].double()
    if run_ == 1:
        g = pi.mul_(-w[:, None, None])
        a = place.to(torch.int64).T[..., None]
        return g.scatter_add_(-1, a, w[:, None, None].expand_as(a)).div_(T)
    g = torch.empty_like(pi)
    for p in range(P):
        part = slice(p * run_, min(S, (p + 1) * run_))
        a = place[:, part].to(torch.int64)
        g[p] = torch.zeros_like(pi[p]).scatter_add_(1, a, w[part].expand_as(a)) - w[part].sum() * pi[p]
    return g / T


def _sample_exact(s, x, T):
    """Every resource's place in its row's order by comparing all pairs, then the count of borders that u has passed."""
    P, N, R = x.shape
    _, top_k, top_p, min_p = (s["knobs"][:, i].double().view(P, 1, 1) for i in range(4))
    top_k = torch.where(top_k < 1, R, top_k)
    w = torch.exp((x - x.amax(-1, keepdim=True)) / T)
    i = torch.arange(R, device=x.device)
    kept = torch.empty_like(x, dtype=torch.bool)
    for p in range(P):
        for v in range(0, N, 256):
            y, wy = x[p, v:v + 256], w[p, v:v + 256]
            ahead = (y[:, None, :] > y[:, :, None]) | ((y[:, None, :] == y[:, :, None]) & (i[None, None, :] < i[None, :, None]))
            rank = ahead.sum(-1)
            in_k = rank < top_k[p]
            wk = wy * in_k
            before = (ahead * wk[:, None, :]).sum(-1)
            ok = in_k & ((before < top_p[p] * wk.sum(-1, keepdim=True)) | (top_p[p] >= 1)) & (wy >= min_p[p])
            kept[p, v:v + 256] = ok | (rank == 0)
    c = torch.cumsum(w * kept, -1)
    u = s["u"].double()
    S = u.shape[1]
    place = torch.empty((N, S), dtype=torch.int16, device=x.device)
    for p in range(P):
        part = slice(p * s["run"], min(S, (p + 1) * s["run"]))
        for v in range(0, N, 256):
            passed = c[p, v:v + 256, None, :] <= u[v:v + 256, part, None] * c[p, v:v + 256, None, -1:]
            place[v:v + 256, part] = passed.sum(-1).to(torch.int16)
    return place


def work(case):
    P, N, R, e = case["n_pol"], case["ops"], case["res"], _BYTES[case["type"]]
    rows = P * N * R
    if case["op"] == "distill":
        return {"bytes": 2 * rows * e + P * N * (case["top"] * (2 + e) + 8), "flops": 8 * rows + 8 * P * N * case["top"]}
    S = case["scen"]
    if case["op"] == "sample":
        return {"bytes": rows * e + N * S * 6, "flops": 4 * rows + N * S * math.ceil(math.log2(R + 1))}
    if case["op"] == "logp":
        return {"bytes": rows * e + N * S * 2 + S * 4, "flops": 4 * rows + N * S}
    return {"bytes": 2 * rows * e + N * S * 2 + S * 4, "flops": 7 * rows + N * S}
