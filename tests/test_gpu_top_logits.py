"""GPU parity: a row's top logits, exactly (values and places), against the oracle's full sort."""
import numpy as np
import pytest

from oracle import text as OT
from text_util import TYPES, rows_in, stored

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2306_00256_amd as P
    assert torch.cuda.is_available()
    P.lib()
    return torch, P


def _check(env, x, K, dtype, extra=0, offset=0):
    torch, P = env
    R, V = x.shape
    rows, _ = rows_in(torch, R, V, V + extra, dtype, offset=offset)
    dev, x64 = stored(torch, x, dtype)
    rows.copy_(dev)
    top = torch.full((R, K), 4.5, device="cuda")
    ids = torch.full((R, K), -9, dtype=torch.int32, device="cuda")
    need = P.ceca_top_logits_workspace_bytes(rows, R, V, K)
    ws = torch.full((need,), 0x5A, dtype=torch.uint8, device="cuda") if need else None
    P.ceca_top_logits(rows, R, V, K, top, ids, workspace=ws)
    values, places = OT.top_logits(x64, K)
    assert np.array_equal(ids.cpu().numpy(), places)
    assert np.array_equal(top.double().cpu().numpy(), values, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,V,K", [(1, 1, 1), (3, 1, 5), (2, 7, 7), (4, 63, 64), (5, 64, 64), (2, 65, 64), (3, 255, 256), (2, 256, 256), (6, 257, 256), (3, 1000, 1), (2, 1023, 64),
                                   (2, 1025, 100), (3, 4097, 256), (2, 8192, 64), (2, 16385, 33), (1, 32769, 64), (3, 65537, 256), (1, 131073, 64), (2, 200003, 20)])
def test_top_logits(env, R, V, K, dtype):
    rng = np.random.default_rng(V + K)
    x = 3.0 * rng.standard_normal((R, V))
    _check(env, x, K, dtype)
    _check(env, x, min(K, 17), dtype, extra=3, offset=1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_whose_parts_merge_in_two_steps(env, dtype):
    """More parts than one workgroup merges at K = 256: random logits, and logits that fall so that one part has all of the largest."""
    V = 600_001
    x = 3.0 * np.random.default_rng(1).standard_normal((2, V))
    x[1] = np.linspace(4.0, -4.0, V)
    _check(env, x, 256, dtype)


@pytest.mark.parametrize("rows", [300, 2000])
def test_many_rows(env, rows):
    _check(env, np.random.default_rng(rows).standard_normal((rows, 300)), 11, "bfloat16")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(1300, 200), (2500, 64), (3500, 256), (8100, 256)])
def test_many_rows_of_some_columns(env, V, K, dtype):
    """2100 rows, 21 of them again and again, some equal everywhere or masked."""
    torch, P = env
    x = 3.0 * np.random.default_rng(V).standard_normal((21, V))
    x[3] = 1.0
    x[5, 10:] = -np.inf
    x[6, ::3] = 2.0
    x[8, 5] = np.nan
    dev, x64 = stored(torch, x, dtype)
    rows = dev.repeat(100, 1)
    top, ids = torch.full((2100, K), 4.5, device="cuda"), torch.full((2100, K), -9, dtype=torch.int32, device="cuda")
    P.ceca_top_logits(rows, 2100, V, K, top, ids)
    values, places = OT.top_logits(x64, K)
    assert np.array_equal(ids.cpu().numpy(), np.tile(places, (100, 1)))
    assert np.array_equal(top.double().cpu().numpy(), np.tile(values, (100, 1)), equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [100, 5000, 70001])
@pytest.mark.parametrize("K", [1, 64, 256])
def test_ties_order_and_masks(env, V, K, dtype):
    """Rows that are equal everywhere, of few values, ascending, descending, masked but for a few, masked altogether, at the
    type's lowest value, with NaN, infinities and both zeros; the largest all in one thread's share."""
    torch, _ = env
    rng = np.random.default_rng(K)
    lowest = float(torch.finfo(getattr(torch, dtype)).min)
    x = np.zeros((13, V))
    x[1] = rng.integers(0, 3, V)
    x[2] = np.linspace(-5, 5, V)
    x[3] = np.linspace(5, -5, V)
    x[4] = -np.inf
    x[4, [V // 3, V - 1, 0]] = [1.0, 1.0, -2.0]
    x[5] = -np.inf
    x[6] = lowest
    x[6, V // 2:] = -np.inf
    x[7] = rng.standard_normal(V)
    x[7, ::7] = np.nan
    x[7, 3] = np.inf
    x[8] = np.where(rng.integers(0, 2, V) > 0, 0.0, -0.0)
    x[9] = rng.standard_normal(V) - 10.0
    x[9, ::64] = 1.0
    x[10] = -np.abs(rng.standard_normal(V))
    x[10, :300] = 2.0
    x[11] = 1e-30 * rng.standard_normal(V)
    x[12] = np.nan
    _check(env, x, K, dtype)


def test_no_rows(env):
    torch, P = env
    P.ceca_top_logits(torch.empty(0, 5, device="cuda"), 0, 5, 2, torch.empty(0, 2, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"))


def test_offsets_beyond_32_bits(env):
    torch, P = env
    V, pitch = 2000, 2_200_000_000
    flat = torch.empty(2 * pitch + V, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((3, V), (pitch, 1))
    src = torch.randn(3, V, device="cuda").bfloat16()
    x.copy_(src)
    out = []
    for t in (x, src):
        top, ids = torch.empty(3, 9, device="cuda"), torch.empty(3, 9, dtype=torch.int32, device="cuda")
        need = P.ceca_top_logits_workspace_bytes(t, 3, V, 9)
        P.ceca_top_logits(t, 3, V, 9, top, ids, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
        out.append((top, ids))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
