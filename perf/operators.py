"""Operators of language models trained by agents: embedding lookup in the agents' state rows and its gradient,
distillation from a teacher's top logits (loss and gradient), and a row's top logits.

`run` computes them in plain torch operations (`own` false) or through the library's entry points (`own` true).
Sizes: the agent counts are those of the repository's workloads; widths and vocabularies are generic."""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the next token of six agents that answer one token at a time: latency
        dict(name="embed_token", kind="embed", n=6, T=1, V=32000, h=1024, off=0, tail=0, type="bf16", pad=0.0),
        # an ordinary training batch of 31 agents
        dict(name="embed_batch", kind="embed", n=31, T=2048, V=32000, h=512, off=0, tail=0, type="bf16", pad=0.0),
        # rows of odd length behind other parameters, ragged sequences
        dict(name="embed_odd", kind="embed", n=5, T=1037, V=50021, h=515, off=7, tail=4, type="f16", pad=0.2),
        # a short sequence over a small vocabulary: latency and launches
        dict(name="grad_short", kind="embed_grad", n=6, T=33, V=1000, h=64, off=0, tail=0, type="f32", pad=0.0, micro=1),
        # the ordinary training batch's gradient, written as whole gradient rows
        dict(name="grad_batch", kind="embed_grad", n=31, T=2048, V=32000, h=512, off=0, tail=0, type="bf16", pad=0.0, micro=1),
        # long padded sequences over a large vocabulary in two microbatches, the second added to the first
        dict(name="grad_micro", kind="embed_grad", n=6, T=16384, V=128000, h=1024, off=0, tail=0, type="f32", pad=0.3, micro=2),
        # a few positions over a small vocabulary, soft and hard targets: latency
        dict(name="distill_short", kind="distill", n=6, T=4, V=8192, K=16, type="f32", temperature=2.0, hard=0.3, pad=0.0, peers=True, grad=True, tail=0),
        # the loss alone, as an evaluation takes it, over rows of odd length with padded positions
        dict(name="distill_loss", kind="distill", n=13, T=100, V=50021, K=100, type="f16", temperature=1.0, hard=0.0, pad=0.25, peers=False, grad=False, tail=0),
        # an ordinary training batch against the peers' top logits, soft and hard targets
        dict(name="distill_batch", kind="distill", n=31, T=256, V=32000, K=64, type="bf16", temperature=2.0, hard=0.5, pad=0.0, peers=True, grad=True, tail=0),
        # the largest: a large batch over a large vocabulary
        dict(name="distill_large", kind="distill", n=31, T=512, V=128000, K=64, type="bf16", temperature=1.0, hard=0.0, pad=0.1, peers=False, grad=True, tail=0),
        # the top logits of one position for each of six agents: few long rows
        dict(name="top_token", kind="top", n=6, T=1, V=128000, K=64, type="f32", tail=0),
        # a batch of positions, as agents send them to their peers; bf16 logits tie often
        dict(name="top_batch", kind="top", n=31, T=256, V=32000, K=64, type="bf16", tail=0),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "distill", "distill", "distill", "top", "top"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    n = int(_log(rng, 1, 101))
    pad = rng.choice([0.0, 0.0, 0.3])
    tail = rng.choice([0, 0, 1, 8])
    if kind in ("embed", "embed_grad"):
        h = int(_log(rng, 16, 2049))
        if rng.random() < 0.6:
            h = -(-h // 16) * 16
        V = int(_log(rng, 64, min(130000, 7e8 / (n * h))))
        T = int(_log(rng, 1, max(2, min(16385, 2e8 / (n * h)))))
        case = dict(kind=kind, n=n, T=T, V=V, h=h, off=rng.choice([0, 0, 5, 64]), tail=tail, type=dtype, pad=pad)
        return dict(case, micro=rng.choice([1, 1, 2])) if kind == "embed_grad" else case
    V = int(_log(rng, 300, 160000))
    if rng.random() < 0.5:
        V = -(-V // 64) * 64
    K = int(_log(rng, 1, 257))
    T = int(_log(rng, 1, max(2, min(1025, 8e8 / (n * V)))))
    case = dict(kind=kind, n=n, T=T, V=V, K=K, type=dtype, tail=tail)
    if kind == "top":
        return case
    return dict(case, temperature=rng.choice([1.0, 1.0, 2.0, 4.0]), hard=rng.choice([0.0, 0.0, 0.3]), pad=pad, peers=rng.random() < 0.5,
                grad=rng.random() < 0.75)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _tokens(case, g):
    """Token numbers whose frequency falls as one over the rank, and -1 behind the end of each agent's sequence."""
    n, T, V = case["n"], case["T"], case["V"]
    u = torch.rand(n, T, generator=g, device="cuda", dtype=torch.float64)
    t = torch.exp(u * math.log(V)).long().sub_(1).clamp_(0, V - 1).int()
    t[:, T - int(case["pad"] * T):] = -1
    return t


def _logits(case, g):
    """(n T, V) logits in rows of V + tail."""
    rows, V = case["n"] * case["T"], case["V"]
    out = torch.empty(rows, V + case["tail"], device="cuda", dtype=TYPES[case["type"]])
    return out.normal_(0.0, 2.0, generator=g)[:, :V]


def prepare(case, seed):
    g, n, T, V = _generator(seed), case["n"], case["T"], case["V"]
    state = {"case": case}
    if case["kind"] in ("embed", "embed_grad"):
        h = case["h"]
        # the agents' tables (or their gradients) begin `off` floats into rows of the state
        rows = torch.empty(n, case["off"] + V * h + case["tail"], device="cuda")
        if case["kind"] == "embed":
            rows.normal_(0.0, 0.02, generator=g)
            state["tokens"] = _tokens(case, g)
            state["out"] = torch.empty(n, T, h, device="cuda", dtype=TYPES[case["type"]])
        else:
            state["tokens"] = [_tokens(case, g) for _ in range(case["micro"])]
            state["G"] = [torch.empty(n, T, h, device="cuda", dtype=TYPES[case["type"]]).normal_(0.0, 1.0, generator=g) for _ in range(case["micro"])]
        state["E"] = rows[:, case["off"]:case["off"] + V * h]
        return state
    state["logits"] = _logits(case, g)
    K, R = case["K"], n * T
    if case["kind"] == "top":
        state["top"] = torch.empty(R, K, device="cuda")
        state["ids"] = torch.empty(R, K, device="cuda", dtype=torch.int32)
        return state
    # the teacher's entries: distinct places, values from the largest down; the student leans the teacher's way
    place = torch.randint(1, V // K + 1, (R, K), generator=g, device="cuda").cumsum(1) - 1
    order = torch.rand(R, K, generator=g, device="cuda").argsort(1)
    state["ids"] = place.gather(1, order).int().contiguous()
    state["top"] = torch.randn(R, K, generator=g, device="cuda").mul_(2.0).add_(8.0).sort(1, descending=True)[0].contiguous()
    peer = torch.randperm(n, generator=g, device="cuda")
    state["peer"] = peer.int() if case["peers"] else None
    at = (state["ids"].view(n, T, K)[peer] if case["peers"] else state["ids"]).reshape(R, K).long()
    values = (state["top"].view(n, T, K)[peer] if case["peers"] else state["top"]).reshape(R, K)
    state["logits"].scatter_add_(1, at, (0.5 * values).to(state["logits"].dtype))
    state["labels"] = torch.randint(0, V, (n, T), generator=g, device="cuda").int() if case["hard"] else None
    # the mean over the batch; with fp16 logits the loss scaled by the number of rows, as such gradients need
    w = torch.full((n, T), 1.0 if case["type"] == "f16" else 1.0 / R, device="cuda")
    w[:, T - int(case["pad"] * T):] = 0.0
    state["weight"] = w
    state["loss"] = torch.empty(n, T, device="cuda")
    state["grad"] = torch.empty(R, V, device="cuda", dtype=state["logits"].dtype) if case["grad"] else None
    return state


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _embed(c, E, tokens):
    n, V, h = c["n"], c["V"], c["h"]
    t = tokens.long()
    inside = (t >= 0) & (t < V)
    agent = torch.arange(n, device="cuda")[:, None]
    rows = E.unflatten(1, (V, h))[agent, t.clamp(0, V - 1)] * math.sqrt(h)
    return torch.where(inside[..., None], rows, torch.zeros((), device="cuda")).to(TYPES[c["type"]])


def _add_rows(c, E, tokens, G):
    n, V, h = c["n"], c["V"], c["h"]
    t = tokens.long()
    inside = (t >= 0) & (t < V)
    row = (t + V * torch.arange(n, device="cuda")[:, None])[inside]
    rows = E.view(n * V, h) if E.is_contiguous() else E.reshape(n * V, h)
    rows.index_add_(0, row, G[inside].float() * math.sqrt(h))
    return E if E.is_contiguous() else E.copy_(rows.view(n, V * h))


def _shares(x):
    """softmax and log softmax over the last dimension"""
    x = x - x.max(-1, keepdim=True)[0]
    e = torch.exp(x)
    total = e.sum(-1, keepdim=True)
    return e / total, x - torch.log(total)


def _distill(c, st):
    n, T, K, V, tau, a = c["n"], c["T"], c["K"], c["V"], c["temperature"], c["hard"]
    ids, top = st["ids"].view(n, T, K), st["top"].view(n, T, K)
    if st["peer"] is not None:
        ids, top = ids[st["peer"].long()], top[st["peer"].long()]
    ids, top, w = ids.reshape(n * T, K).long(), top.reshape(n * T, K), st["weight"].view(-1, 1)
    s = st["logits"].float()
    p, logp = _shares(top / tau)
    q, logq = _shares(s / tau)
    loss = (1 - a) * tau * tau * (p * (logp - logq.gather(1, ids))).sum(1, keepdim=True)
    grad = None
    if c["grad"]:
        grad = (q.scatter_add_(1, ids, -p)).mul_((1 - a) * tau)
    if a:
        label = st["labels"].view(-1, 1).long()
        r, logr = _shares(s)
        loss = loss - a * logr.gather(1, label)
        if c["grad"]:
            grad = grad + a * r.scatter_add_(1, label, torch.full_like(label, -1.0, dtype=torch.float32))
    loss = (w * loss).view(n, T)
    return (loss, (grad * w).to(st["logits"].dtype)) if c["grad"] else loss


def _top(c, st):
    V, K = c["V"], c["K"]
    bits = (st["logits"].float() + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    both = key * 2 ** 32 + (V - 1 - torch.arange(V, device="cuda"))          # the lowest place wins a tie
    at = torch.topk(both, K, dim=1)[1]
    return st["logits"].gather(1, at).float(), at.int()


def _workspace(st, size):
    if "workspace" not in st:                  # made once, as a program keeps it beside its buffers
        st["workspace"] = torch.empty(size, device="cuda", dtype=torch.uint8) if size else None
    return st["workspace"]


def run(state):
    c, kind = state["case"], state["case"]["kind"]
    if own:
        import paper_2306_00256_amd as P
        n, T, V = c["n"], c["T"], c["V"]
        if kind == "embed":
            P.ceca_embed(state["E"], n, V, c["h"], state["tokens"], state["out"], scale=math.sqrt(c["h"]))
            return state["out"]
        if kind == "embed_grad":
            ws = state["workspace"] if "workspace" in state else _workspace(state, P.ceca_embed_grad_workspace_bytes(n, T, V, c["h"]))
            for i in range(c["micro"]):
                P.ceca_embed_grad(state["G"][i], n, V, c["h"], state["tokens"][i], state["E"], scale=math.sqrt(c["h"]), accumulate=i > 0, workspace=ws)
            return state["E"]
        if kind == "distill":
            if "spec" not in state:
                state["spec"] = P.make_distill(state["logits"], n, T, V, top=state["top"], ids=state["ids"], peer=state["peer"], labels=state["labels"],
                                               weight=state["weight"], temperature=c["temperature"], hard=c["hard"])
            ws = state["workspace"] if "workspace" in state else _workspace(state, P.ceca_distill_workspace_bytes(state["spec"]))
            P.ceca_distill(state["spec"], loss=state["loss"], grad=state["grad"], workspace=ws)
            return (state["loss"], state["grad"]) if c["grad"] else state["loss"]
        ws = state["workspace"] if "workspace" in state else _workspace(state, P.ceca_top_logits_workspace_bytes(state["logits"], n * T, V, c["K"]))
        P.ceca_top_logits(state["logits"], n * T, V, c["K"], state["top"], state["ids"], workspace=ws)
        return state["top"], state["ids"]
    if kind == "embed":
        return _embed(c, state["E"], state["tokens"])
    if kind == "embed_grad":
        E = state["E"].zero_()
        for tokens, G in zip(state["tokens"], state["G"]):
            _add_rows(c, E, tokens, G)
        return E
    return _distill(c, state) if kind == "distill" else _top(c, state)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------

def _exact_distill(c, st):
    n, T, K, V, tau, a = c["n"], c["T"], c["K"], c["V"], c["temperature"], c["hard"]
    loss = torch.zeros(n, T, device="cuda", dtype=torch.float64)
    grad = torch.zeros(n, T, V, device="cuda", dtype=torch.float64) if c["grad"] else None
    for i in range(n):
        j = int(st["peer"][i]) if st["peer"] is not None else i
        s = st["logits"][i * T:(i + 1) * T].double()
        u, at = st["top"].view(n, T, K)[j].double(), st["ids"].view(n, T, K)[j].long()
        w = st["weight"][i].double()
        teacher = torch.exp(u / tau - torch.logsumexp(u / tau, 1)[:, None])
        Z = torch.logsumexp(s / tau, 1)
        cross = -(teacher * (torch.gather(s, 1, at) / tau - Z[:, None])).sum(1)
        entropy = -(teacher * torch.log(teacher)).sum(1)
        L = (1 - a) * tau ** 2 * (cross - entropy)
        if a:
            label = st["labels"][i].long()
            Z1 = torch.logsumexp(s, 1)
            L = L + a * (Z1 - torch.gather(s, 1, label[:, None])[:, 0])
        loss[i] = w * L
        if grad is not None:
            d = (1 - a) * tau * torch.exp(s / tau - Z[:, None])
            d.scatter_add_(1, at, -(1 - a) * tau * teacher)
            if a:
                d += a * torch.exp(s - Z1[:, None])
                d[torch.arange(T, device="cuda"), label] -= a
            grad[i] = w[:, None] * d
    return loss if grad is None else (loss, grad.view(n * T, V))


def exact(case, seed):
    st, n, T, V = prepare(case, seed), case["n"], case["T"], case["V"]
    if case["kind"] == "embed":
        out = torch.zeros(n, T, case["h"], device="cuda", dtype=torch.float64)
        for i in range(n):
            real = (st["tokens"][i] >= 0).nonzero()[:, 0]
            table = st["E"][i].view(V, case["h"])
            out[i, real] = table.index_select(0, st["tokens"][i][real].long()).double() * case["h"] ** 0.5
        return out
    if case["kind"] == "embed_grad":
        E = torch.zeros(n, V, case["h"], device="cuda", dtype=torch.float64)
        for tokens, G in zip(st["tokens"], st["G"]):
            for i in range(n):
                real = (tokens[i] >= 0).nonzero()[:, 0]
                E[i].index_add_(0, tokens[i][real].long(), G[i, real].double(), alpha=case["h"] ** 0.5)
        return E.view(n, V * case["h"])
    if case["kind"] == "distill":
        return _exact_distill(case, st)
    K, top, ids = case["K"], [], []
    for some in st["logits"].split(256):
        values, at = torch.sort(some.double(), dim=1, descending=True, stable=True)
        top.append(values[:, :K].clone())
        ids.append(at[:, :K].int())
    return torch.cat(top), torch.cat(ids)


def _distinct(case):
    """The expected number of distinct tokens of one agent's sequence."""
    V, T = case["V"], case["T"] - int(case["pad"] * case["T"])
    v = torch.arange(1, V + 1, dtype=torch.float64)
    share = torch.log((v + 1) / v) / math.log(V)
    share[V - 1] = 0.0
    return float((1 - (1 - share).pow(T)).sum())


def work(case):
    n, T, V, size = case["n"], case["T"], case["V"], SIZE[case["type"]]
    real = n * (T - int(case.get("pad", 0.0) * T))
    if case["kind"] == "embed":
        h = case["h"]
        return {"bytes": 4 * n * T + n * _distinct(case) * h * 4 + n * T * h * size, "flops": real * h}
    if case["kind"] == "embed_grad":
        h, m = case["h"], case["micro"]
        return {"bytes": m * (4 * n * T + real * h * size) + n * V * h * 4 + (m - 1) * n * _distinct(case) * h * 8, "flops": m * 2 * real * h}
    R = n * T
    if case["kind"] == "distill":
        K = case["K"]
        terms = 2 if case["hard"] and case["temperature"] != 1 else 1
        passes = 2 if case["grad"] else 1
        return {"bytes": real * V * size + (R * V * size if case["grad"] else 0) + R * (8 * K + 12), "flops": real * V * (1 + 3 * terms * passes)}
    return {"bytes": R * V * size + 8 * R * case["K"], "flops": R * V}
