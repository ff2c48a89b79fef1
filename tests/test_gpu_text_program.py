"""GPU: the language-model operators together, as agents that train one another use them -- embeddings looked up in the
state rows, the peers' top logits as teachers, the loss's gradient back into the agents' gradient rows, DSGD-CECA steps -- against the
same program in fp64, and the ways in which programs make such calls: captured graphs, side streams, autograd."""
import numpy as np
import pytest

from oracle import ceca as OC
from oracle import schedule as OS
from oracle import text as OT
from gpu_util import make_state, rel_err, split_state
from text_util import tokens_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2306_00256_amd as P
    assert torch.cuda.is_available()
    P.lib()
    return torch, P


def _bytes(torch, size):
    return torch.empty(size, dtype=torch.uint8, device="cuda") if size else None


def _z(P, S, n, r, port):
    rd, _ = P.ceca_schedule(n, r, port)
    return S[n:] if rd.exchange_y else S[:n]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("n,port", [(6, 1), (5, 2)])
def test_agents_that_teach_each_other(env, n, port, tied):
    """logits = (scale E[token]) W^T with E and W (tied: W = E) in every agent's row; agent i learns from agent peer(i)'s top logits
    and from labels.  Four iterations against fp64; 1e-4 as for the other training runs."""
    torch, P = env
    from paper_2306_00256_amd import binding as Bn
    V, h, T, K, tau, hard, lr, scale = 40, 8, 12, 5, 2.0, 0.25, 0.3, float(np.sqrt(np.float32(8)))
    d = V * h if tied else 2 * V * h
    rng = np.random.default_rng(n)
    x0 = (0.5 * rng.standard_normal((n, d))).astype(np.float32)
    tokens = tokens_of(rng, n, T, V, pad=0.15)
    labels = rng.integers(0, V, (n, T)).astype(np.int32)
    weight = np.where((tokens >= 0) & (tokens < V), 1.0 / T, 0.0).astype(np.float32)
    rounds = max(OS.num_rounds(n), 1)
    peers = [OS.peers(n, r, port) for r in range(rounds)]

    def grad64(z, k):
        peer = peers[k % rounds]
        E = z[:, :V * h].reshape(n, V, h)
        W = E if tied else z[:, V * h:].reshape(n, V, h)
        H = OT.embed(E, tokens, scale)
        logits = np.einsum("nth,nvh->ntv", H, W)
        top, ids = OT.top_logits(logits.reshape(n * T, V), K)
        _, g, _ = OT.distill(logits, top.reshape(n, T, K), ids.reshape(n, T, K), tau, hard, labels, weight, peer)
        dW = np.einsum("ntv,nth->nvh", g, H)
        dH = np.einsum("ntv,nvh->nth", g, W)
        if tied:
            return OT.embed_grad(dH, tokens, V, scale, old=dW)[0].reshape(n, d)
        dE = OT.embed_grad(dH, tokens, V, scale)[0]
        return np.concatenate([dE.reshape(n, V * h), dW.reshape(n, V * h)], axis=1)

    iters = 4
    want_x, want_y = OC.run(x0, port, lr, grad64, iters, store32=True)

    S = make_state(torch, x0)
    R = S if port == 1 else torch.empty_like(S)
    td, ld, wd = (torch.from_numpy(a).cuda() for a in (tokens, labels, weight))
    H, dH = torch.empty(n, T, h, device="cuda"), torch.empty(n, T, h, device="cuda")
    top, ids = torch.empty(n, T, K, device="cuda"), torch.empty(n, T, K, dtype=torch.int32, device="cuda")
    e, loss = torch.empty(n, d, device="cuda"), torch.empty(n, T, device="cuda")
    ws = _bytes(torch, P.ceca_embed_grad_workspace_bytes(n, T, V, h))
    for k in range(iters):
        r = k % rounds
        z = _z(P, S, n, r, port)
        E = z[:, :V * h]
        W = (E if tied else z[:, V * h:]).view(n, V, h)
        P.ceca_embed(E, n, V, h, td, H, scale=scale)
        logits = torch.bmm(H, W.transpose(1, 2).contiguous())
        P.ceca_top_logits(logits, n * T, V, K, top, ids, workspace=_bytes(torch, P.ceca_top_logits_workspace_bytes(logits, n * T, V, K)))
        spec = P.make_distill(logits, n, T, V, top=top, ids=ids, peer=torch.tensor(peers[r], dtype=torch.int32, device="cuda"), labels=ld, weight=wd,
                              temperature=tau, hard=hard)
        P.ceca_distill(spec, loss=loss, grad=logits, workspace=_bytes(torch, P.ceca_distill_workspace_bytes(spec)))        # over the logits
        torch.bmm(logits, W.contiguous(), out=dH)
        dW = torch.bmm(logits.transpose(1, 2).contiguous(), H)
        (e if tied else e[:, V * h:]).copy_(dW.view(n, V * h))
        P.ceca_embed_grad(dH, n, V, h, td, e[:, :V * h], scale=scale, accumulate=tied, workspace=ws)
        P.dsgd_ceca_step(S, R, n, d, Bn.make_gradient_loss(e), None, lr, r, port)
        S, R = R, S
    gx, gy = split_state(S, n, d)
    assert max(rel_err(gx, want_x)) <= 1e-4 and max(rel_err(gy, want_y)) <= 1e-4


class _Bigram:
    """Agents whose logits are rows of a V x V table in their state rows: every kernel of an iteration is the library's."""

    def __init__(self, torch, P, n, V, T, K, seed, dtype):
        from paper_2306_00256_amd import binding as Bn
        rng = np.random.default_rng(seed)
        self.torch, self.P, self.Bn = torch, P, Bn
        self.n, self.V, self.T, self.K = n, V, T, K
        self.tokens = torch.from_numpy(tokens_of(rng, n, T, V)).cuda()
        self.labels = torch.from_numpy(rng.integers(0, V, (n, T)).astype(np.int32)).cuda()
        self.S = make_state(torch, rng.standard_normal((n, V * V)).astype(np.float32))
        self.R = torch.zeros_like(self.S)
        self.logits = torch.empty(n, T, V, device="cuda", dtype=dtype)
        self.top, self.ids = torch.empty(n, T, K, device="cuda"), torch.empty(n, T, K, dtype=torch.int32, device="cuda")
        self.loss, self.e = torch.empty(n, T, device="cuda"), torch.empty(n, V * V, device="cuda")
        self.peer = torch.tensor(OS.peers(n, 0, 2), dtype=torch.int32, device="cuda")
        self.spec = P.make_distill(self.logits, n, T, V, top=self.top, ids=self.ids, peer=self.peer, labels=self.labels, temperature=2.0, hard=0.5)
        self.ws = _bytes(torch, P.ceca_embed_grad_workspace_bytes(n, T, V, V))
        self.wd = _bytes(torch, P.ceca_distill_workspace_bytes(self.spec))
        self.wt = _bytes(torch, P.ceca_top_logits_workspace_bytes(self.logits, n * T, V, K))

    def step(self, stream=None):
        P, n, V = self.P, self.n, self.V
        P.ceca_embed(_z(P, self.S, n, 0, 2), n, V, V, self.tokens, self.logits, stream=stream)
        P.ceca_top_logits(self.logits, n * self.T, V, self.K, self.top, self.ids, workspace=self.wt, stream=stream)
        P.ceca_distill(self.spec, loss=self.loss, grad=self.logits, workspace=self.wd, stream=stream)
        P.ceca_embed_grad(self.logits, n, V, V, self.tokens, self.e, workspace=self.ws, stream=stream)
        P.dsgd_ceca_step(self.S, self.R, n, V * V, self.Bn.make_gradient_loss(self.e), None, 0.1, 0, 2, stream=stream)

    def results(self):
        return [t.clone() for t in (self.top, self.ids, self.loss, self.logits, self.e, self.R)]


def _same(torch, a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


# T: one position, no sort, one workgroup's sort, several workgroups' (V = 20: one pass of digits; the chunks of a token many)
@pytest.mark.parametrize("n,V,T,K", [(5, 64, 1, 8), (5, 50, 200, 20), (3, 37, 1500, 5), (2, 20, 17000, 3), (2, 20, 6000, 3), (2, 33000, 2, 64)])
def test_a_captured_step_replays(env, n, V, T, K):
    torch, P = env
    if V > 1000:                          # a part of it: rows that are split over workgroups (V x V floats would be too many)
        return _captured_long_rows(torch, P, n, V, T, K)
    prog = _Bigram(torch, P, n, V, T, K, V + T, torch.float32 if V % 2 else torch.bfloat16)
    prog.step()
    torch.cuda.synchronize()
    want = prog.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        prog.step(stream=torch.cuda.current_stream())
    for k in range(4):
        for t in (prog.top, prog.ids, prog.loss, prog.logits, prog.e, prog.R):
            t.fill_(k)
        if prog.ws is not None:
            prog.ws.fill_(0x33 + k)
        graph.replay()
        torch.cuda.synchronize()
        assert _same(torch, prog.results(), want), k
        prog.step()                       # the program's own calls in between
        torch.cuda.synchronize()
        assert _same(torch, prog.results(), want), k


def _captured_long_rows(torch, P, n, V, T, K):
    logits = torch.randn(n, T, V, device="cuda")
    top, ids = torch.empty(n * T, K, device="cuda"), torch.empty(n * T, K, dtype=torch.int32, device="cuda")
    wt = _bytes(torch, P.ceca_top_logits_workspace_bytes(logits, n * T, V, K))
    spec = P.make_distill(logits, n, T, V, top=top, ids=ids, temperature=0.5)
    wd = _bytes(torch, P.ceca_distill_workspace_bytes(spec))
    assert wt is not None and wd is not None
    loss, grad = torch.empty(n, T, device="cuda"), torch.empty_like(logits)

    def calls():
        P.ceca_top_logits(logits, n * T, V, K, top, ids, workspace=wt)
        P.ceca_distill(spec, loss=loss, grad=grad, workspace=wd)

    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (top, ids, loss, grad)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(4):
        for t in (top, ids, loss, grad):
            t.fill_(k)
        wt.fill_(0x11 * k)
        wd.fill_(0x11 * k)
        graph.replay()
        torch.cuda.synchronize()
        assert _same(torch, (top, ids, loss, grad), want), k
        calls()
        torch.cuda.synchronize()
        assert _same(torch, (top, ids, loss, grad), want), k


def test_two_streams_at_once(env):
    """Two programs with buffers and workspaces of their own, interleaved call by call on two streams: the results of each alone."""
    torch, P = env
    progs = [_Bigram(torch, P, 5, 60, 700, 9, seed, torch.float16) for seed in (1, 2)]
    want = []
    for p in progs:
        p.step()
        torch.cuda.synchronize()
        want.append(p.results())
    streams = [torch.cuda.Stream() for _ in progs]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, st in zip(progs, streams):
            p.step(stream=st)
    torch.cuda.synchronize()
    for p, w in zip(progs, want):
        assert _same(torch, p.results(), w)


def test_loss_first_and_weights_later(env):
    """As an autograd function calls it: the loss alone, then the gradient alone with the factors handed back; against torch's own
    derivative of the same formula in fp64 (the fp32 kernel's bound of the distillation tests at these sizes: (4 * 30 + 90) half
    steps = 1.3e-5 of a share, shares up to 1 here)."""
    torch, P = env
    n, T, V, K = 2, 7, 300, 6
    g = torch.Generator().manual_seed(4)
    logits = (2 * torch.randn(n, T, V, generator=g)).cuda()
    top = torch.randn(n, T, K, generator=g).cuda()
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(n * T)]).view(n, T, K).int().cuda()

    class Distillation(torch.autograd.Function):
        @staticmethod
        def forward(ctx, s):
            ctx.save_for_backward(s)
            loss = torch.empty(n, T, device="cuda")
            P.ceca_distill(P.make_distill(s, n, T, V, top=top, ids=ids, temperature=2.0), loss=loss)
            return loss

        @staticmethod
        def backward(ctx, w):
            (s,) = ctx.saved_tensors
            grad = torch.empty_like(s)
            P.ceca_distill(P.make_distill(s, n, T, V, top=top, ids=ids, weight=w.contiguous(), temperature=2.0), grad=grad)
            return grad

    s = logits.clone().requires_grad_(True)
    factor = torch.rand(n, T, generator=g).cuda()
    (factor * Distillation.apply(s)).sum().backward()
    t = logits.double().requires_grad_(True)
    p = torch.softmax(top.double() / 2, -1)
    loss = 4 * (p * (p.log() - torch.log_softmax(t / 2, -1).gather(-1, ids.long()))).sum(-1)
    (factor.double() * loss).sum().backward()
    assert (s.grad.double() - t.grad).abs().max().item() <= 2 * 1.3e-5


def test_more_rows_than_a_launch_has_workgroups(env):
    """2^22 + 77 short rows, the same 1000 over and over: every row its results, the same as the first 1000's."""
    torch, P = env
    R, V, K, period = (1 << 22) + 77, 5, 2, 1000
    src = torch.randn(period, V, device="cuda")
    at = torch.arange(R, device="cuda") % period
    logits = src[at].contiguous()
    top, ids = torch.zeros(R, K, device="cuda"), torch.zeros(R, K, dtype=torch.int32, device="cuda")
    P.ceca_top_logits(logits, R, V, K, top, ids)
    spec = P.make_distill(logits, 1, R, V, top=top, ids=ids)
    loss = torch.zeros(1, R, device="cuda")
    P.ceca_distill(spec, loss=loss, grad=logits)
    for t in (top, ids, loss.view(R, 1), logits):
        assert torch.equal(t, t[:period][at])
    want = torch.sort(src, dim=1, descending=True)
    assert torch.equal(top[:period], want[0][:, :K]) and torch.equal(ids[:period].long(), want[1][:, :K])
    # lookup and gradient: more positions, more agents and more rows than one launch's workgroups
    n, T, V, h = (1 << 22) + 5, 1, 3, 2
    E = torch.arange(n * V * h, device="cuda", dtype=torch.float32).view(n, V * h) % 8191
    tokens = (torch.arange(n, device="cuda") % 4 - 1).int().view(n, 1)
    out = torch.full((n, T, h), -1.0, device="cuda")
    P.ceca_embed(E, n, V, h, tokens, out)
    rows = E.view(n, V, h)[torch.arange(n, device="cuda"), tokens[:, 0].clamp(min=0).long()] * (tokens >= 0)
    assert torch.equal(out[:, 0], rows)
    P.ceca_embed_grad(out, n, V, h, tokens, E)
    hit = torch.zeros(n, V, device="cuda").scatter_(1, tokens.clamp(min=0).long(), (tokens >= 0).float())
    assert torch.equal(E.view(n, V, h), hit[..., None] * out)
