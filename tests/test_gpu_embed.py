"""GPU parity: embedding lookup in the agents' rows and its gradient, against the fp64 oracle.

Tolerances.  Lookup: one fp32 product (half an fp32 step) and one rounding to the output's type.  Gradient: a row's sum of c terms in
any order takes at most c - 1 fp32 additions, one multiplication by the scale and, where it is added to what is there, one
addition: (c + 2) half steps of the sum of the terms' absolute values (and of the old value)."""
import numpy as np
import pytest

from oracle import text as OT
from text_util import HALF_LEAST, HALF_STEP, TYPES, rows_in, stored, tokens_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2306_00256_amd as P
    assert torch.cuda.is_available()
    P.lib()
    return torch, P


# (n, T, V, h, extra floats in front of a table, behind it, extra pitch of out)
SHAPES = [(1, 1, 1, 1, 0, 0, 0), (1, 1, 50, 64, 0, 0, 0), (6, 1, 1000, 256, 0, 0, 0), (3, 17, 40, 1, 1, 0, 0), (2, 9, 33, 2, 0, 3, 1), (5, 33, 20, 3, 2, 1, 0),
          (2, 5, 7, 4, 0, 0, 0), (2, 64, 100, 5, 3, 0, 2), (31, 65, 300, 64, 0, 0, 0), (4, 100, 77, 127, 0, 1, 0), (3, 50, 60, 129, 1, 0, 1),
          (2, 130, 500, 255, 0, 0, 0), (2, 31, 90, 257, 0, 0, 3), (1, 257, 1000, 515, 7, 4, 1), (7, 40, 64, 512, 0, 64, 0), (1, 33, 30, 1024, 0, 0, 0),
          (2, 20, 20, 1500, 0, 0, 4), (1, 9, 11, 2051, 0, 0, 0)]


def _table(torch, rng, n, V, h, off, tail):
    E, flat = rows_in(torch, n, V * h, off + V * h + tail, "float32", offset=off)
    x = (0.5 * rng.standard_normal((n, V, h))).astype(np.float32)
    E.copy_(torch.from_numpy(x.reshape(n, V * h)).cuda())
    return E, flat, x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,T,V,h,off,tail,extra", SHAPES)
def test_lookup(env, n, T, V, h, off, tail, extra, dtype):
    torch, P = env
    rng = np.random.default_rng(h + T)
    E, _, x = _table(torch, rng, n, V, h, off, tail)
    tokens = tokens_of(rng, n, T, V)
    out, flat = rows_in(torch, n * T, h, h + extra, dtype, offset=extra, fill=7.0)
    scale = 1.7
    P.ceca_embed(E, n, V, h, torch.from_numpy(tokens).cuda(), out, scale=scale)
    want = OT.embed(x, tokens, float(np.float32(scale))).reshape(n * T, h)
    got = out.double().cpu().numpy()
    assert (np.abs(got - want) <= np.abs(want) * (HALF_STEP[dtype] + 2.0 ** -24 * (1 + HALF_STEP[dtype])) + HALF_LEAST[dtype]).all()
    pad = ~((tokens >= 0) & (tokens < V)).reshape(-1)
    assert (got[pad] == 0).all()
    if extra:                                              # what lies between the rows
        assert (flat[extra:].view(n * T, h + extra)[:, h:] == 7).all() and (flat[:extra] == 7).all()


def _gradient(env, n, T, V, h, off, tail, extra, dtype, tokens, accumulate, seed=0):
    torch, P = env
    rng = np.random.default_rng(seed + h + T)
    E, flat, old = _table(torch, rng, n, V, h, off, tail)
    keep = flat.clone()
    if not accumulate:
        E.fill_(float("nan"))
    G, gflat = rows_in(torch, n * T, h, h + extra, dtype, offset=extra)
    g, g64 = stored(torch, rng.standard_normal((n * T, h)), dtype)
    G.copy_(g)
    pad = ~((tokens >= 0) & (tokens < V)).reshape(-1)
    G[torch.from_numpy(pad).cuda()] = float("nan")        # rows of padding are not looked at
    scale = -0.75                                          # exact in fp32
    need = P.ceca_embed_grad_workspace_bytes(n, T, V, h)
    ws = torch.full((need,), 0x5A, dtype=torch.uint8, device="cuda") if need else None
    td = torch.from_numpy(tokens).cuda()
    P.ceca_embed_grad(G, n, V, h, td, E, scale=scale, accumulate=accumulate, workspace=ws)
    got = E.double().cpu().numpy().reshape(n, V, h)
    want, size, terms = OT.embed_grad(g64.reshape(n, T, h), tokens, V, scale, old=old if accumulate else None)
    assert (np.abs(got - want) <= (terms[..., None] + 2) * 2.0 ** -24 * size).all()
    assert (got[terms == 0] == (old[terms == 0] if accumulate else 0)).all()
    if off or tail:                                        # other parameters around the tables
        around = torch.ones_like(flat, dtype=torch.bool)
        around[off:].view(n, off + V * h + tail)[:, :V * h] = False
        assert torch.equal(torch.isnan(flat[around]), torch.isnan(keep[around]))
    # the same call gives the same bits, whatever the workspace held
    again = flat.clone()[off:].view(n, off + V * h + tail)[:, :V * h]
    if accumulate:
        again.copy_(torch.from_numpy(old.reshape(n, V * h)).cuda())
    if ws is not None:
        ws.fill_(0xC3)
    P.ceca_embed_grad(G, n, V, h, td, again, scale=scale, accumulate=accumulate, workspace=ws)
    assert torch.equal(again, E)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,T,V,h,off,tail,extra", SHAPES)
def test_gradient(env, n, T, V, h, off, tail, extra, dtype, accumulate):
    tokens = tokens_of(np.random.default_rng(T), n, T, V)
    _gradient(env, n, T, V, h, off, tail, extra, dtype, tokens, accumulate)


# lengths around the powers of two at which a sort's tiles and a walk's chunks end, vocabularies of one and two rows, and of more
# rows than there are positions
@pytest.mark.parametrize("n,T,V,h", [(1, 31, 5, 8), (2, 32, 1, 8), (2, 33, 2, 8), (1, 63, 70000, 4), (3, 127, 9, 20), (1, 128, 257, 16), (2, 129, 300, 64), (1, 511, 13, 68),
                                     (1, 1023, 100, 12), (2, 1025, 40000, 8), (1, 2049, 600, 36), (5, 4097, 1000, 16), (1, 8191, 3000, 8), (2, 8193, 131072, 4), (1, 16385, 131073, 4),
                                     (1, 20000, 300000, 4), (2, 40000, 50, 8), (1, 70000, 300, 4), (1, 2100, 2_100_000, 2),
                                     (3, 256, 90, 300), (20, 257, 90, 8), (4, 1024, 33, 8), (5, 1024, 33, 260), (3, 4096, 1000, 8)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_at_the_ends_of_tiles(env, n, T, V, h, accumulate):
    tokens = tokens_of(np.random.default_rng(T + 1), n, T, V)
    _gradient(env, n, T, V, h, 0, 0, 0, "float32", tokens, accumulate)


@pytest.mark.parametrize("kind", ["one", "none", "last", "ascending", "halves", "one_agent"])
@pytest.mark.parametrize("n,T,V,h", [(3, 1000, 50, 36), (2, 9000, 9001, 8)])
def test_gradient_of_uneven_tokens(env, kind, n, T, V, h):
    """All positions at one token, none at any, all at the last one; every token once; two halves; one agent without any."""
    tokens = np.full((n, T), 7, dtype=np.int32)
    if kind == "none":
        tokens[:] = -5
    if kind == "last":
        tokens[:] = V - 1
    if kind == "ascending":
        tokens[:] = np.arange(T) % V
    if kind == "halves":
        tokens[:, ::2] = V - 1
    if kind == "one_agent":
        tokens[1] = np.iinfo(np.int32).min
        tokens[2 % n] = np.iinfo(np.int32).max
    _gradient(env, n, T, V, h, 0, 0, 0, "bfloat16", tokens, False)
    _gradient(env, n, T, V, h, 1, 2, 0, "float32", tokens, True)


def test_no_positions(env):
    torch, P = env
    n, V, h = 3, 10, 6
    E = torch.full((n, V * h), 3.0, device="cuda")
    none = torch.empty((n, 0), dtype=torch.int32, device="cuda")
    rows = torch.empty((n, 0, h), device="cuda")
    ws = torch.empty(max(P.ceca_embed_grad_workspace_bytes(n, 0, V, h), 1), dtype=torch.uint8, device="cuda")
    P.ceca_embed(E, n, V, h, none, rows)
    P.ceca_embed_grad(rows, n, V, h, none, E, accumulate=True, workspace=ws)
    assert (E == 3).all()
    P.ceca_embed_grad(rows, n, V, h, none, E, workspace=ws)
    assert (E == 0).all()


def test_tables_with_a_pitch(env):
    """Tables of the shape (n, V, h) whose rows have a pitch of their own: what lies between the rows stays."""
    torch, P = env
    n, V, h, T = 2, 9, 6, 21
    rng = np.random.default_rng(2)
    whole = torch.full((n, V + 1, h + 3), 5.0, device="cuda")
    E = whole[:, :V, :h]
    x = rng.standard_normal((n, V, h)).astype(np.float32)
    E.copy_(torch.from_numpy(x).cuda())
    tokens = tokens_of(rng, n, T, V)
    td = torch.from_numpy(tokens).cuda()
    out = torch.empty(n, T, h, device="cuda")
    P.ceca_embed(E, n, V, h, td, out)
    assert np.array_equal(out.cpu().numpy(), OT.embed(x, tokens, 1.0).astype(np.float32))
    ws = torch.empty(max(P.ceca_embed_grad_workspace_bytes(n, T, V, h), 1), dtype=torch.uint8, device="cuda")
    P.ceca_embed_grad(out, n, V, h, td, E, workspace=ws)
    want, size, terms = OT.embed_grad(out.double().cpu().numpy(), tokens, V, 1.0)
    assert (np.abs(E.double().cpu().numpy() - want) <= (terms[..., None] + 2) * 2.0 ** -24 * size).all()
    assert (whole[:, V:] == 5).all() and (whole[:, :, h:] == 5).all()


def test_offsets_beyond_32_bits(env):
    """A table of more than 2^31 floats, and gradient rows whose pitch takes them past 2^32 bytes."""
    torch, P = env
    n, V, h, T = 1, 1100, 2_000_000, 3
    E = torch.zeros(n, V * h, device="cuda")
    E.view(V, h)[1099] = torch.arange(h, device="cuda") % 1000
    tokens = torch.tensor([[1099, 0, 1099]], dtype=torch.int32, device="cuda")
    out = torch.empty(1, T, h, device="cuda", dtype=torch.bfloat16)
    P.ceca_embed(E, n, V, h, tokens, out)
    want = E.view(V, h)[1099].bfloat16()
    assert torch.equal(out[0, 0], want) and torch.equal(out[0, 2], want) and not out[0, 1].any()
    ws = torch.empty(max(P.ceca_embed_grad_workspace_bytes(n, T, V, h), 1), dtype=torch.uint8, device="cuda")
    E.fill_(1.0)
    P.ceca_embed_grad(out, n, V, h, tokens, E, workspace=ws)
    assert torch.equal(E.view(V, h)[1099], 2 * want.float())
    assert not E[0, :1099 * h].any()
    del E
    pitch = 1_500_000_000
    flat = torch.empty(2 * pitch + 8, dtype=torch.bfloat16, device="cuda")
    G = flat.as_strided((3, 8), (pitch, 1))
    G.copy_(torch.arange(24, device="cuda").view(3, 8))
    e = torch.empty(1, 4 * 8, device="cuda")
    toks = torch.tensor([[3, 1, 3]], dtype=torch.int32, device="cuda")
    ws = torch.empty(max(P.ceca_embed_grad_workspace_bytes(1, 3, 4, 8), 1), dtype=torch.uint8, device="cuda")
    P.ceca_embed_grad(G, 1, 4, 8, toks, e, workspace=ws)
    assert torch.equal(e.view(4, 8)[3], (G[0] + G[2]).float()) and torch.equal(e.view(4, 8)[1], G[1].float()) and not e.view(4, 8)[::2].any()
