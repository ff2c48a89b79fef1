"""GPU parity of the language-model operators at sizes that reach every kernel they launch (tests/text_forms.py), against the fp64 oracle.

Tolerances are those of the operators' other tests.  Lookup: one product and one rounding.  Gradient: (terms + 2) half fp32 steps of the sum
of absolute values.  Distillation: shares off by delta = (4 X + V / 64 + 64) half steps of themselves, X the largest difference
from a row's maximum over the temperature, 110 at most (beyond, an fp32 exponential is zero).  Top logits: exact."""
import numpy as np
import pytest

from oracle import text as OT
import text_forms as F
from text_util import HALF_LEAST, HALF_STEP, stored, tokens_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2306_00256_amd as P
    assert torch.cuda.is_available()
    P.lib()
    return torch, P


def _bytes(torch, size):
    return torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") if size else None


@pytest.mark.parametrize("dtype,n,T,h", F.LOOKUPS)
def test_lookup(env, dtype, n, T, h):
    torch, P = env
    rng = np.random.default_rng(h + T)
    V, scale = 61, 1.7
    x = (0.5 * rng.standard_normal((n, V, h))).astype(np.float32)
    tokens = tokens_of(rng, n, T, V)
    out = torch.full((n, T, h), 7.0, device="cuda", dtype=getattr(torch, dtype))
    P.ceca_embed(torch.from_numpy(x).cuda(), n, V, h, torch.from_numpy(tokens).cuda(), out, scale=scale)
    want = OT.embed(x, tokens, float(np.float32(scale)))
    got = out.double().cpu().numpy()
    assert (np.abs(got - want) <= np.abs(want) * (HALF_STEP[dtype] + 2.0 ** -24 * (1 + HALF_STEP[dtype])) + HALF_LEAST[dtype]).all()


def _tables(torch, n, V, h, apart, pitch):
    """n tables of V rows of h floats: `pitch` floats behind every row, `apart` in front of and behind every table; all 5."""
    lde = V * (h + pitch) + apart
    flat = torch.full((n * lde + apart,), 5.0, device="cuda")
    return flat, flat[apart:].as_strided((n, V, h), (lde, h + pitch, 1), apart)


@pytest.mark.parametrize("dtype,n,T,V,h,accumulate,apart,pitch", F.GRADIENTS)
def test_gradient(env, dtype, n, T, V, h, accumulate, apart, pitch):
    torch, P = env
    rng = np.random.default_rng(V + h + T)
    tokens = tokens_of(rng, n, T, V)
    G, g64 = stored(torch, rng.standard_normal((n * T, h)), dtype)
    G[torch.from_numpy(~((tokens >= 0) & (tokens < V)).reshape(-1)).cuda()] = float("nan")        # padding is not looked at
    old = rng.standard_normal((n, V, h)).astype(np.float32) if accumulate else None
    scale = -0.75
    td = torch.from_numpy(tokens).cuda()
    ws = _bytes(torch, P.ceca_embed_grad_workspace_bytes(n, T, V, h))
    runs = []
    for fill in (0x5A, 0xC3):                              # the same bits, whatever workspace and tables held
        flat, E = _tables(torch, n, V, h, apart, pitch)
        E.copy_(torch.from_numpy(old).cuda() if accumulate else torch.tensor(float("nan")))
        if ws is not None:
            ws.fill_(fill)
        P.ceca_embed_grad(G, n, V, h, td, E if pitch else E.as_strided((n, V * h), (E.stride(0), 1)), scale=scale, accumulate=accumulate, workspace=ws)
        runs.append((flat, E))
    (flat, E), (flat2, _) = runs
    assert torch.equal(flat, flat2)
    want, size, terms = OT.embed_grad(g64.reshape(n, T, h), tokens, V, scale, old=old)
    assert (np.abs(E.double().cpu().numpy() - want) <= (terms[..., None] + 2) * 2.0 ** -24 * size).all()
    assert (E.cpu().numpy()[terms == 0] == (old[terms == 0] if accumulate else 0)).all()
    E.fill_(5.0)
    assert (flat == 5).all()                               # what lies between rows and tables


def test_gradient_of_sorted_positions_beyond_32_bits(env):
    """Tables of more than 2^31 floats whose positions are sorted (zeros on their own, walk, join), and gradient rows past 2^32 elements.
    Whole numbers below 1000 of up to 300 terms: sums below 2^24 are exact."""
    torch, P = env
    n, V, h, T = 1, 1100, 2_000_000, 300
    tokens = torch.full((1, T), 1099, dtype=torch.int32)
    tokens[0, ::3], tokens[0, 1], tokens[0, 4], tokens[0, 7] = 1, 1098, 0, -1
    G = (torch.arange(h, device="cuda") % 249 + torch.arange(T, device="cuda")[:, None] % 7).to(torch.float16)
    E = torch.full((n, V * h), float("nan"), device="cuda")
    ws = _bytes(torch, P.ceca_embed_grad_workspace_bytes(n, T, V, h))
    P.ceca_embed_grad(G, n, V, h, tokens.cuda(), E, workspace=ws)
    rows = E.view(V, h)
    named = {v: (tokens[0] == v).nonzero()[:, 0].cuda() for v in (0, 1, 1098, 1099)}
    for v, at in named.items():
        want = torch.zeros(h, device="cuda")
        for t in at.tolist():
            want += G[t].float()
        assert torch.equal(rows[v], want), v
    assert not rows[2:1098].any()
    # added once more: twice the sums
    P.ceca_embed_grad(G, n, V, h, tokens.cuda(), E, accumulate=True, workspace=ws)
    for v, at in named.items():
        want = torch.zeros(h, device="cuda")
        for t in at.tolist():
            want += G[t].float()
        assert torch.equal(rows[v], 2 * want), v
    del E, rows, G, ws
    torch.cuda.empty_cache()
    pitch, T, h, V = 4_000_000, 1100, 8, 50
    flat = torch.empty((T - 1) * pitch + h, dtype=torch.bfloat16, device="cuda")
    G = flat.as_strided((T, h), (pitch, 1))
    src = (torch.arange(T * h, device="cuda").view(T, h) % 101).bfloat16()
    G.copy_(src)
    tokens = (torch.arange(T, device="cuda") % V).int().view(1, T)
    e, want = torch.empty(1, V * h, device="cuda"), torch.empty(1, V * h, device="cuda")
    ws = _bytes(torch, P.ceca_embed_grad_workspace_bytes(1, T, V, h))
    P.ceca_embed_grad(G, 1, V, h, tokens, e, workspace=ws)
    P.ceca_embed_grad(src, 1, V, h, tokens, want, workspace=ws)
    exact = torch.zeros(V, h, device="cuda").index_add_(0, tokens[0].long(), src.float())
    assert torch.equal(e, want) and torch.equal(e.view(V, h), exact)


PERIOD = 13


def _rows(rng, V, K, dtype):
    """PERIOD rows with all that may be among them: ordinary ones, padding, no entries, no label, everything masked, NaN, masks, an id that
    comes several times, the lowest value."""
    x = (3.0 * rng.standard_normal((PERIOD, V))).astype(np.float32)
    top = (2.0 * rng.standard_normal((PERIOD, K)) + 5.0).astype(np.float32)
    ids = rng.integers(0, V, (PERIOD, K)).astype(np.int32)
    labels = rng.integers(0, V, PERIOD).astype(np.int32)
    weight = rng.uniform(0.5, 1.5, PERIOD).astype(np.float32)
    weight[2], x[2] = 0.0, np.nan
    labels[3] = -1
    ids[4] = -1
    x[6] = -np.inf
    x[7, V - 1] = -np.inf
    x[8, V // 2] = np.nan
    x[9, 1::2] = -np.inf
    ids[9] = ids[9] // 2 * 2
    labels[9] = labels[9] // 2 * 2
    ids[11] = [5, 5, V - 1, 5, V - 1, 8, 8, 5][:K]
    labels[11] = 5
    x[12, ::3] = {"float32": -3e38, "bfloat16": -3e38, "float16": -65504.0}[dtype]
    ids[12], labels[12] = ids[12] % (V // 3) * 3 + 1, 1
    return x, top, ids, labels, weight


@pytest.mark.parametrize("hard", [0.0, 0.5])
@pytest.mark.parametrize("dtype,rows,V", F.DISTILLATIONS)
def test_distillation(env, dtype, rows, V, hard):
    torch, P = env
    K, tau = 8, 2.0
    x, top, ids, labels, weight = _rows(np.random.default_rng(V), V, K, dtype)
    dev, x64 = stored(torch, x, dtype)
    want_loss, want, size = np.zeros(PERIOD), np.zeros((PERIOD, V)), np.zeros(PERIOD)
    taken = np.zeros((PERIOD, V))
    X = 0.0
    for r in range(PERIOD):
        want_loss[r], want[r], size[r] = OT.distill_row(x64[r], top[r], ids[r], tau, hard, int(labels[r]), float(weight[r]))
        np.add.at(taken[r], ids[r][ids[r] >= 0], (1 - hard) * tau * weight[r])
        if labels[r] >= 0:
            taken[r, labels[r]] += hard * weight[r]
        f = x64[r][np.isfinite(x64[r])]
        X = max(X, f.max() - f.min() if f.size else 0.0, float(top[r].max() - top[r].min()))
    delta = (4 * min(X, 110.0) + V / 64 + 64) * 2.0 ** -24
    with np.errstate(invalid="ignore"):
        bound = delta * (np.abs(want) + 2 * taken) + 2.0 ** -125 * tau * weight[:, None]
        bound = bound + HALF_STEP[dtype] * (np.abs(want) + bound) + HALF_LEAST[dtype]
    at = torch.arange(rows) % PERIOD
    pick = lambda a: torch.from_numpy(np.ascontiguousarray(a))[at].cuda()  # noqa: E731
    logits = dev[at.cuda()]
    spec = P.make_distill(logits, 1, rows, V, top=pick(top), ids=pick(ids), labels=pick(labels) if hard else None, weight=pick(weight), temperature=tau, hard=hard)
    ws = _bytes(torch, P.ceca_distill_workspace_bytes(spec))
    loss, alone = torch.full((2, rows), 9.0, device="cuda")
    grad = torch.full_like(logits, 9.0)
    P.ceca_distill(spec, loss=loss, grad=grad, workspace=ws)
    P.ceca_distill(spec, loss=alone, workspace=ws)
    for got in (loss, alone):
        got = got.double().cpu().numpy()
        w, s = want_loss[at], size[at]
        with np.errstate(invalid="ignore"):
            assert ((got == w) | (np.isnan(got) & np.isnan(w)) | (np.abs(got - w) <= delta * s)).all()
    want_d, bound_d = torch.from_numpy(want).cuda(), torch.from_numpy(bound).cuda()
    for r0 in range(0, rows, PERIOD):
        g = grad[r0:r0 + PERIOD].double()
        w, b = want_d[:len(g)], bound_d[:len(g)]
        assert ((torch.isnan(g) & torch.isnan(w)) | ((g - w).abs() <= b)).all(), r0
    whole = torch.int32 if dtype == "float32" else torch.int16
    P.ceca_distill(spec, grad=logits, workspace=ws)        # over the logits: the same bits
    assert torch.equal(torch.nan_to_num(logits).view(whole), torch.nan_to_num(grad).view(whole)) and torch.equal(torch.isnan(logits), torch.isnan(grad))


@pytest.mark.parametrize("dtype,rows,V,K", F.TOPS)
def test_top_logits(env, dtype, rows, V, K):
    torch, P = env
    rng = np.random.default_rng(V + K)
    R = min(rows, PERIOD)
    x = 3.0 * rng.standard_normal((R, V))
    x[0] = np.linspace(4.0, -4.0, V)
    if R > 5:
        x[1, 9:] = -np.inf
        x[2] = rng.integers(0, 3, V)
        x[3, V // 3] = np.nan
        x[4] = 0.25
    dev, x64 = stored(torch, x, dtype)
    at = torch.arange(rows) % R
    logits = dev[at.cuda()]
    top, ids = torch.full((rows, K), 4.5, device="cuda"), torch.full((rows, K), -9, dtype=torch.int32, device="cuda")
    P.ceca_top_logits(logits, rows, V, K, top, ids, workspace=_bytes(torch, P.ceca_top_logits_workspace_bytes(logits, rows, V, K)))
    values, places = OT.top_logits(x64, K)
    assert np.array_equal(ids.cpu().numpy(), places[at])
    assert np.array_equal(top.double().cpu().numpy(), values[at], equal_nan=True)
