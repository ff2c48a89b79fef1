"""GPU parity: a teacher's small shares and a student's lowest logits in the distillation's loss and gradient.

Tolerances.  A share is exp(x) / sum with x = (u - largest) / temperature: the argument takes four roundings at most (difference,
1 / temperature, its product with log2 e, the product), which the exponential turns into 4 |x| half fp32 steps of the share; the
exponential's own error, the sum over at most 16 entries, the quotient, three factors and the sum over a place that several
entries name are 32 more at most.  Where the student's logit lies 200 below its largest, its own share is below 2^-126 and the gradient is
the teacher's share times its factors, rounded once to its type."""
import numpy as np
import pytest

from oracle import text as OT
from text_util import HALF_STEP

pytestmark = pytest.mark.gpu

BELOW = [0.0, 20.0, 30.0, 38.0, 43.0, 60.0, 80.0, 45.0, 45.0, 50.0, 1.0]       # nats; the last places: one of three entries, one alone


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2306_00256_amd as P
    assert torch.cuda.is_available()
    P.lib()
    return torch, P


def _call(env, logits, top, ids, temperature, loss=True, grad=True):
    """(loss, gradient) of one sequence whose rows all hold the same entries."""
    torch, P = env
    R, V = logits.shape
    at, u = (torch.from_numpy(np.tile(a, (R, 1))).cuda() for a in (ids, top))
    spec = P.make_distill(logits, 1, R, V, top=u, ids=at, temperature=temperature)
    need = P.ceca_distill_workspace_bytes(spec)
    out_l = torch.full((R,), 7.0, device="cuda") if loss else None
    out_g = torch.full((R, V), 7.0, device="cuda", dtype=logits.dtype) if grad else None
    P.ceca_distill(spec, loss=out_l, grad=out_g, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    return out_l, out_g


# rows of one wavefront, of four, split over workgroups, read twice by one workgroup, of a workgroup that loops over rows
SIZES = [("float32", 3, 40), ("bfloat16", 3, 40), ("float32", 3, 3001), ("bfloat16", 90, 3001), ("float32", 2, 70001), ("bfloat16", 2, 70001), ("float32", 260, 65541), ("bfloat16", 260, 131081),
         ("bfloat16", 258, 70001)]


@pytest.mark.parametrize("temperature", [1.0, 2.0])
@pytest.mark.parametrize("dtype,R,V", SIZES)
def test_small_shares_keep_their_bits(env, dtype, R, V, temperature):
    torch, _ = env
    ids = np.array([3, 9, 4, 31, 12, 7, 20, 25, 25, 25, 16], dtype=np.int32)
    top = (5.0 - temperature * np.array(BELOW)).astype(np.float32)
    x = np.random.default_rng(V).uniform(-2, 2, V).astype(np.float32)
    x[ids] = -200.0 * temperature
    x[3], x[16] = 1.5, -0.5
    row = torch.from_numpy(x).to(getattr(torch, dtype))
    _, grad = _call(env, row.cuda().repeat(R, 1), top, ids, temperature)
    _, want, _ = OT.distill_row(row.double().numpy(), top, ids, temperature, 0.0, None, 1.0)
    places = np.array([9, 4, 31, 12, 7, 20, 25])
    below = np.array([20.0, 30.0, 38.0, 43.0, 60.0, 80.0, 50.0])
    got = grad[:, torch.from_numpy(places).cuda()].double().cpu().numpy()
    bound = (4 * below + 32) * 2.0 ** -24
    bound = np.abs(want[places]) * (bound + HALF_STEP[dtype] * (1 + bound))
    assert (np.abs(got - want[places]) <= bound).all()


def test_places_that_many_entries_name(env):
    """256 entries at three places, small and large shares mixed: each place's sum, and the same bits in any order of the entries at
    a place (those of the first two entries of one place exchanged)."""
    torch, _ = env
    V, K = 500, 256
    rng = np.random.default_rng(8)
    ids = rng.choice([17, 18, 400], K).astype(np.int32)
    top = -rng.integers(0, 60, K).astype(np.float32)
    top[ids == 400] -= 40.0                                 # a place of small shares alone
    top[0], ids[0] = 0.0, 17
    x = rng.uniform(-2, 2, V).astype(np.float32)
    x[[17, 18, 400]] = -200.0
    _, grad = _call(env, torch.from_numpy(x).cuda().repeat(2, 1), top, ids, 1.0)
    _, want, _ = OT.distill_row(x.astype(np.float64), top, ids, 1.0, 0.0, None, 1.0)
    # as above with up to 256 additions in either sum; shares 100 nats below
    for v in (17, 18, 400):
        assert (np.abs(grad[:, v].double().cpu().numpy() - want[v]) <= (4 * 100 + 2 * 256 + 32) * 2.0 ** -24 * abs(want[v])).all()
    # (the row's own sum is that of all entries in the order in which they lie: it stays the same where two of one wavefront's lanes that
    # are one apart are exchanged)
    first = next(k for k in range(2, K, 2) if ids[k] == ids[k + 1])
    top[[first, first + 1]] = top[[first + 1, first]]
    _, again = _call(env, torch.from_numpy(x).cuda().repeat(2, 1), top, ids, 1.0)
    assert torch.equal(again, grad)


@pytest.mark.parametrize("dtype,R,V", SIZES[:6])
def test_lowest_logits_at_entries_below_temperature_one(env, dtype, R, V):
    """The type's lowest finite value is an ordinary logit: at temperature 0.5 an entry's loss there, 0.25 p * 6.8e38, is a number of
    fp32 (and a large one: all other terms together are below half a step of it).  Its error is that of p and of some products:
    64 half steps."""
    torch, _ = env
    lowest = float(torch.finfo(getattr(torch, dtype)).min)
    ids, top = np.array([3, 9, 30], dtype=np.int32), np.array([2.0, 1.25, 0.5], dtype=np.float32)
    x = np.random.default_rng(V).uniform(-2, 2, V).astype(np.float32)
    x[9] = lowest
    row = torch.from_numpy(x).to(getattr(torch, dtype))
    want, want_grad, _ = OT.distill_row(row.double().numpy(), top, ids, 0.5, 0.0, None, 1.0)
    assert 1e36 < want < 1e38
    for grad in (True, False):
        loss, _ = _call(env, row.cuda().repeat(R, 1), top, ids, 0.5, grad=grad)
        assert (np.abs(loss.double().cpu().numpy() - want) <= 64 * 2.0 ** -24 * want).all()
    _, g = _call(env, row.cuda().repeat(R, 1), top, ids, 0.5)
    assert (np.abs(g[:, 9].double().cpu().numpy() - want_grad[9]) <= (64 * 2.0 ** -24 + HALF_STEP[dtype]) * abs(want_grad[9]) * 1.01).all()


@pytest.mark.parametrize("dtype,R,V", SIZES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_every_entry_of_a_row_with_one_that_is_not_finite(env, dtype, R, V, value):
    """NaN at the places of all of the row's entries and in its loss, numbers everywhere else."""
    torch, _ = env
    ids, top = np.array([3, 9, 30, 9], dtype=np.int32), np.array([2.0, 1.0, value, 0.5], dtype=np.float32)
    logits = torch.randn(R, V, device="cuda").to(getattr(torch, dtype))
    loss, grad = _call(env, logits, top, ids, 1.0)
    there = torch.zeros(V, dtype=torch.bool, device="cuda")
    there[[3, 9, 30]] = True
    assert torch.isnan(loss).all()
    assert torch.isnan(grad[:, there]).all() and torch.isfinite(grad[:, ~there]).all()
