"""GPU parity: distillation from a teacher's top logits (loss and gradient) against the fp64 oracle.

Tolerances.  With X the largest |s - max s| / min(temperature, 1), of the entries too, or 110 where it is more (there an fp32
exponential is zero; shares below 2^-126 may be): an exponent's argument is off by at most 4 half fp32 steps of its size (difference, product with 1 / temperature and its rounding, product with log2 e), the
exponential by 4 more; a sum over V terms by as many half steps as one thread adds terms, at most V / 64, and 32 for the tree
over threads.  So every share has the relative error delta = (4 X + V / 64 + 64) half steps at most (64 > 4 + 32, the
quotient and the weights' products), and so does each term of the loss relative to the term's size plus its share.  A
gradient is the difference of two such shares and is then rounded once to its type."""
import numpy as np
import pytest

from oracle import text as OT
from text_util import HALF_LEAST, HALF_STEP, TYPES, rows_in, stored

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2306_00256_amd as P
    assert torch.cuda.is_available()
    P.lib()
    return torch, P


def _range(x):
    f = x[np.isfinite(x)]
    return float(f.max() - f.min()) if f.size else 0.0


def _case(n, T, V, K, seed, spread=3.0):
    rng = np.random.default_rng(seed)
    logits = (spread * rng.standard_normal((n, T, V))).astype(np.float32)
    top = (2.0 * rng.standard_normal((n, T, K)) + 5.0).astype(np.float32)
    ids = rng.integers(0, V, (n, T, K)).astype(np.int32)
    ids[rng.uniform(size=ids.shape) < 0.05] = -1
    ids[rng.uniform(size=ids.shape) < 0.02] = V
    top[rng.uniform(size=ids.shape) < 0.05] = -np.inf
    labels = rng.integers(-1, V + 1, (n, T)).astype(np.int32)
    weight = rng.uniform(0.5, 1.5, (n, T)).astype(np.float32)
    weight[rng.uniform(size=(n, T)) < 0.15] = 0.0
    return logits, top, ids, labels, weight


def _workspace(torch, P, spec):
    need = P.ceca_distill_workspace_bytes(spec)
    return torch.full((need,), 0x5A, dtype=torch.uint8, device="cuda") if need else None


def _check(env, dtype, logits, top, ids, labels, weight, peer, temperature, hard, extra=0, offset=0, in_place=True):
    torch, P = env
    n, T, V = logits.shape
    K = 0 if top is None else top.shape[2]
    rows, _ = rows_in(torch, n * T, V, V + extra, dtype, offset=offset)
    dev, l64 = stored(torch, logits.reshape(n * T, V), dtype)
    rows.copy_(dev)
    put = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    spec = P.make_distill(rows, n, T, V, top=put(top), ids=put(ids), peer=put(peer), labels=put(labels), weight=put(weight), temperature=temperature,
                          hard=hard)
    loss = torch.full((n, T), float("nan"), device="cuda")
    grad, gflat = rows_in(torch, n * T, V, V + extra, dtype, offset=offset, fill=9.0)
    ws = _workspace(torch, P, spec)
    P.ceca_distill(spec, loss=loss, grad=grad, workspace=ws)
    temperature, hard = float(np.float32(temperature)), float(np.float32(hard))
    want_loss, want_grad, size = OT.distill(l64.reshape(n, T, V), top, ids, temperature, hard, labels, weight, peer)
    X = max([_range(r) for r in l64] + ([_range(r) for r in top.reshape(n * T, K).astype(np.float64)] if K else []))
    delta = (4 * min(X / min(temperature, 1.0), 110.0) + V / 64 + 64) * 2.0 ** -24
    got = loss.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        same = (got == want_loss) | (np.isnan(got) & np.isnan(want_loss))
        assert (same | (np.abs(got - want_loss) <= delta * size)).all()
    w = np.ones((n, T)) if weight is None else np.abs(weight.astype(np.float64))
    # the shares that make up a gradient: q and r (at most the gradient's absolute value plus the entries' and the label's), p
    taken = np.zeros((n, T, V))
    for i in range(n):
        j = i if peer is None else min(max(int(peer[i]), 0), n - 1)
        for t in range(T):
            for k in range(K):
                if 0 <= ids[j, t, k] < V:
                    taken[i, t, ids[j, t, k]] = (1 - hard) * temperature * w[i, t]
            if labels is not None and 0 <= labels[i, t] < V:
                taken[i, t, labels[i, t]] += hard * w[i, t]
    g = grad.double().cpu().numpy().reshape(n, T, V)
    with np.errstate(invalid="ignore"):
        bound = delta * (np.abs(want_grad) + 2 * taken) + 2.0 ** -125 * max(temperature, 1.0) * w[..., None]
        bound = bound + HALF_STEP[dtype] * (np.abs(want_grad) + bound) + HALF_LEAST[dtype]
        assert ((np.isnan(g) & np.isnan(want_grad)) | (np.abs(g - want_grad) <= bound)).all()
    if extra or offset:
        assert (gflat[:offset] == 9).all() and (gflat[offset:].view(n * T, V + extra)[:, V:] == 9).all()
    # the loss alone (which may add up in another order) keeps to the same bound; the gradient alone, and over the logits, has the same
    # bits
    loss2 = torch.full_like(loss, float("nan"))
    P.ceca_distill(spec, loss=loss2, workspace=ws)
    alone = loss2.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        same = (alone == want_loss) | (np.isnan(alone) & np.isnan(want_loss))
        assert (same | (np.abs(alone - want_loss) <= delta * size)).all()
    whole = torch.int32 if dtype == "float32" else torch.int16
    bits = grad.contiguous().view(whole)
    grad2 = torch.empty_like(grad).fill_(9.0)
    P.ceca_distill(spec, grad=grad2, workspace=ws)
    assert torch.equal(grad2.contiguous().view(whole), bits) if not torch.isnan(grad).any() else torch.equal(torch.isnan(grad2), torch.isnan(grad))
    if in_place:
        P.ceca_distill(spec, loss=loss2, grad=rows, workspace=ws)
        assert torch.equal(loss.view(torch.int32), loss2.view(torch.int32))
        assert torch.equal(rows.contiguous().view(whole), bits) if not torch.isnan(grad).any() else torch.equal(torch.isnan(rows), torch.isnan(grad))
    return got, g


SHAPES = [(1, 1, 1, 1), (1, 2, 2, 1), (2, 3, 3, 5), (3, 5, 7, 2), (2, 4, 64, 16), (5, 7, 65, 64), (3, 11, 255, 256), (2, 9, 256, 30), (2, 5, 257, 100), (6, 4, 1000, 16),
          (2, 3, 1023, 64), (2, 3, 1025, 7), (31, 2, 2048, 64), (2, 3, 4095, 64), (2, 2, 5003, 256), (1, 3, 8192, 100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,T,V,K", SHAPES)
def test_distillation(env, n, T, V, K, dtype):
    logits, top, ids, labels, weight = _case(n, T, V, K, V + K)
    peer = np.random.default_rng(n).permutation(n).astype(np.int32)
    _check(env, dtype, logits, top, ids, labels, weight, peer, 2.0, 0.3)
    _check(env, dtype, logits, top, ids, None, None, None, 1.0, 0.0, extra=1, offset=1)


@pytest.mark.parametrize("temperature,hard", [(1.0, 0.3), (4.0, 0.0), (0.5, 0.9), (3.0, 1.0), (1000.0, 0.5), (0.01, 0.0)])
@pytest.mark.parametrize("dtype", TYPES)
def test_temperatures_and_shares(env, temperature, hard, dtype):
    logits, top, ids, labels, weight = _case(3, 4, 777, 20, 5)
    _check(env, dtype, logits, top, ids, labels, weight, None, temperature, hard, extra=3)


# rows of more columns than a workgroup's registers hold, few rows and many
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,T,V", [(1, 1, 16384), (1, 2, 16385), (2, 1, 32768), (1, 2, 32771), (1, 1, 65536), (1, 2, 65537), (1, 1, 131072), (1, 1, 131075), (1, 2, 200001), (3, 1, 300000)])
def test_long_rows(env, n, T, V, dtype):
    logits, top, ids, labels, weight = _case(n, T, V, 64, V)
    weight[:] = 0.75
    _check(env, dtype, logits, top, ids, labels, weight, None, 2.0, 0.25)
    _check(env, dtype, logits, top, ids, None, None, None, 1.0, 0.0, extra=5, offset=3)


@pytest.mark.parametrize("rows", [300, 1500])
def test_many_rows(env, rows):
    """More rows than workgroups are on the device at once."""
    logits, top, ids, labels, weight = _case(rows, 1, 700, 9, rows)
    _check(env, "bfloat16", logits, top, ids, labels, weight, None, 2.0, 0.5)


# many rows that take a whole compute unit's registers (a workgroup loops over them), rows of padding among them, and longer ones
@pytest.mark.parametrize("dtype,rows,V", [("float32", 530, 32777), ("bfloat16", 530, 65545), ("float16", 300, 70001), ("bfloat16", 257, 131080), ("float32", 260, 65541)])
@pytest.mark.parametrize("hard", [0.0, 0.5])
def test_many_long_rows(env, dtype, rows, V, hard):
    logits, top, ids, labels, weight = _case(rows, 1, V, 8, rows)
    labels[::7] = -1
    ids[::5] = -1
    _check(env, dtype, logits, top, ids, labels, weight, None, 2.0, hard)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [300, 70000])
def test_cross_entropy_alone(env, dtype, V):
    logits, _, _, labels, weight = _case(2, 3, V, 1, 3)
    _check(env, dtype, logits, None, None, labels, weight, None, 2.0, 1.0)
    _check(env, dtype, logits, None, None, labels, weight, None, 1.0, 0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 3001, 70001])
@pytest.mark.parametrize("hard,temperature", [(0.0, 1.0), (0.4, 2.0)])
def test_masks_and_what_is_not_finite(env, dtype, V, hard, temperature):
    """Row by row: some logits -inf, all of them, all but one, the type's lowest value at some and at all places, NaN, +inf, a
    masked entry, a masked label, no entry, entries of -inf, an entry many times, an entry far below the others, padding of NaN."""
    torch, _ = env
    lowest = float(torch.finfo(getattr(torch, dtype)).min)
    T, K = 14, 8
    logits, top, ids, labels, weight = _case(1, T, V, K, 11)
    weight[:] = 1.0
    labels[:] = 3
    ids[0] = np.arange(K) + 5
    top[0] = np.linspace(8, 1, K)
    x = logits[0]
    x[0, 20::2] = -np.inf
    x[1] = -np.inf
    x[2] = -np.inf
    x[2, 6] = 1.5
    x[3, 20::2] = lowest
    x[4] = lowest
    x[5, 17] = np.nan
    x[6, 18] = np.inf
    x[7, 5] = -np.inf
    x[8, 3] = -np.inf
    ids[0, 9] = [-1, V, -7, V + 5, 2 ** 31 - 1, -2 ** 31, -1, -1]
    top[0, 10] = -np.inf
    ids[0, 11] = 9
    top[0, 12, 1:] = -3e38
    x[13] = np.nan
    weight[0, 13] = 0.0
    loss, grad = _check(env, dtype, logits, top, ids, labels if hard else None, weight, None, temperature, hard)
    assert loss[0, 1] == 0 and not grad[0, 1].any()
    assert np.isnan(loss[0, 5]) and np.isnan(loss[0, 6]) and np.isposinf(loss[0, 7]) and np.isfinite(grad[0, 7]).all()
    assert loss[0, 13] == 0 and not grad[0, 13].any()
    if not hard:
        assert loss[0, 9] == 0 and not grad[0, 9].any() and loss[0, 10] == 0 and not grad[0, 10].any()


def test_what_is_not_finite_among_the_entries(env):
    torch, P = env
    V, K = 500, 4
    logits, top, ids, _, _ = _case(1, 3, V, K, 1)
    ids[0] = np.arange(K)
    top[0, 0, 2], top[0, 1, 1] = np.nan, np.inf
    put = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    spec = P.make_distill(put(logits), 1, 3, V, top=put(top), ids=put(ids))
    loss, grad = torch.empty(1, 3, device="cuda"), torch.empty(3, V, device="cuda")
    P.ceca_distill(spec, loss=loss, grad=grad, workspace=_workspace(torch, P, spec))
    assert torch.isnan(loss).tolist() == [[True, True, False]]
    assert torch.isnan(grad[0, :K]).any() and torch.isfinite(grad[:, K:]).all() and torch.isfinite(grad[2]).all()


def test_gradient_against_differences_of_the_oracle(env):
    """Central differences of the fp64 loss at steps of 1e-4: off by 1e-8 / 6 times the third derivative (below 1 here), far
    below the kernel's own error."""
    torch, P = env
    V, K = 37, 5
    logits, top, ids, labels, weight = _case(1, 2, V, K, 21, spread=1.0)
    weight[:] = 0.8
    put = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    spec = P.make_distill(put(logits), 1, 2, V, top=put(top), ids=put(ids), labels=put(labels), weight=put(weight), temperature=1.5, hard=0.25)
    grad = torch.empty(2, V, device="cuda")
    P.ceca_distill(spec, grad=grad, workspace=_workspace(torch, P, spec))
    g = grad.double().cpu().numpy()
    for t in range(2):
        for v in range(V):
            step = np.zeros(V)
            step[v] = 1e-4
            up, down = (OT.distill_row(logits[0, t].astype(np.float64) + d, top[0, t], ids[0, t], 1.5, 0.25, int(labels[0, t]), float(weight[0, t]))[0] for d in (step, -step))
            assert abs((up - down) / 2e-4 - g[t, v]) <= 2e-6


def test_no_rows(env):
    torch, P = env
    spec = P.make_distill(torch.empty(2, 0, 9, device="cuda"), 2, 0, 9, top=torch.empty(2, 0, 3, device="cuda"),
                          ids=torch.empty(2, 0, 3, dtype=torch.int32, device="cuda"))
    P.ceca_distill(spec, loss=torch.empty(2, 0, device="cuda"), workspace=_workspace(torch, P, spec))


def test_offsets_beyond_32_bits(env):
    """Logits past 2^32 elements: the last rows of a tensor of 9 GB, gradient in place."""
    torch, P = env
    rows, V, pitch = 3, 1000, 2_200_000_000
    flat = torch.empty(2 * pitch + V, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((rows, V), (pitch, 1))
    src = torch.randn(rows, V, device="cuda").bfloat16()
    x.copy_(src)
    top, ids = torch.randn(rows, 4, device="cuda"), torch.randint(0, V, (rows, 4), device="cuda", dtype=torch.int32)
    losses, grads = [], []
    for t in (x, src):
        spec = P.make_distill(t, 1, rows, V, top=top, ids=ids)
        loss = torch.empty(1, rows, device="cuda")
        P.ceca_distill(spec, loss=loss, grad=t, workspace=_workspace(torch, P, spec))
        losses.append(loss)
        grads.append(t.contiguous())
    assert torch.equal(losses[0], losses[1]) and torch.equal(grads[0], grads[1])
