"""CPU-only checks of the language-model operators' entry points: every refusal fires before anything touches a device, and
does so through the C ABI and through the binding."""
import ctypes

import pytest
import torch

import paper_2306_00256_amd as P
from paper_2306_00256_amd import binding as B


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(P.library_path()):
        from paper_2306_00256_amd import build
        build.build_library(verbose=False)
    return P.lib()


# stand-ins for device addresses, far apart; nothing reads them
A, Bp, Cp, D, W = (1 << 32) * 256, (1 << 33) * 256, (1 << 34) * 256, (1 << 35) * 256, (1 << 36) * 256


def test_struct_size_matches_header():
    assert ctypes.sizeof(B.Distill) == 32 + 7 * 8


def _embed(L, E=A, lde=60, ldr=6, n=2, V=10, h=6, tokens=Bp, T=3, out=Cp, type=0, ldo=6):
    return L.ceca_embed(E, lde, ldr, n, V, h, tokens, T, 1.0, out, type, ldo, None)


def _embed_grad(L, G=Cp, type=0, ldg=6, tokens=Bp, T=3, E=A, lde=60, ldr=6, n=2, V=10, h=6, ws=W, wbytes=1 << 30):
    return L.ceca_embed_grad(G, type, ldg, tokens, T, 1.0, 0, E, lde, ldr, n, V, h, ws, wbytes, None)


BAD_TABLES = [dict(E=None), dict(tokens=None), dict(n=0), dict(V=0), dict(h=0), dict(T=-1), dict(n=1 << 20, T=1 << 12), dict(type=3), dict(type=-1), dict(ldr=5),
              dict(ldr=1 << 31, lde=1 << 40), dict(lde=59), dict(E=A + 2), dict(tokens=Bp + 1), dict(n=1 << 20, lde=1 << 30)]


@pytest.mark.parametrize("bad", BAD_TABLES + [dict(out=None), dict(ldo=5), dict(out=Cp + 2), dict(out=Cp + 1, type=1), dict(out=A), dict(out=A + 4 * 119), dict(out=Bp + 4),
                                             dict(T=1 << 20, out=A - 64), dict(ldo=1 << 60)])
def test_lookup_refusals(L, bad):
    assert _embed(L, **bad) == B.CECA_EINVAL and L.ceca_last_error()


@pytest.mark.parametrize("bad", BAD_TABLES + [dict(G=None), dict(ldg=5), dict(G=Cp + 2), dict(G=A + 8), dict(E=Bp)])
def test_gradient_refusals(L, bad):
    assert _embed_grad(L, **bad) == B.CECA_EINVAL and L.ceca_last_error()


def test_gradient_workspace(L):
    for sizes in [(0, 10, 6, 3), (2, 0, 6, 3), (2, 10, 0, 3), (2, 10, 6, -1), (1 << 20, 10, 6, 1 << 12)]:
        assert L.ceca_embed_grad_workspace_bytes(*sizes) == B.CECA_EINVAL
    need = L.ceca_embed_grad_workspace_bytes(2, 10, 6, 1 << 16)
    assert need >= 0
    if need:
        for ws, have in [(None, 1 << 30), (W, need - 1), (W + 128, need)]:
            assert _embed_grad(L, T=1 << 16, ws=ws, wbytes=have) == B.CECA_EWORKSPACE
    # the largest sizes neither overflow nor go wrong
    assert L.ceca_embed_grad_workspace_bytes(1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1) >= 0 or L.ceca_last_error()


def _spec(**kw):
    base = dict(n=2, T=3, V=100, K=4, type=1, temperature=1.0, hard=0.0, logits=A, ld=100, top=Bp, ids=Bp + 4096, peer=None, labels=None, weight=None)
    return B.Distill(**(base | kw))


BAD_SPECS = [dict(n=0), dict(T=-1), dict(V=0), dict(n=1 << 20, T=1 << 12), dict(type=3), dict(K=-1), dict(K=257), dict(temperature=0.0), dict(temperature=-1.0),
             dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-4), dict(hard=-0.1), dict(hard=1.1), dict(hard=float("nan")), dict(ld=99), dict(K=0), dict(logits=None),
             dict(top=None), dict(ids=None), dict(hard=0.5), dict(logits=A + 1), dict(top=Bp + 2), dict(ids=Bp + 1), dict(peer=Bp + 3), dict(hard=0.5, labels=Bp + 1), dict(weight=Bp + 2)]


@pytest.mark.parametrize("bad", BAD_SPECS)
def test_distillation_refusals(L, bad):
    spec = _spec(**bad)
    assert L.ceca_distill_workspace_bytes(ctypes.byref(spec)) == B.CECA_EINVAL
    assert L.ceca_distill(ctypes.byref(spec), Cp, D, 100, W, 1 << 30, None) == B.CECA_EINVAL and L.ceca_last_error()


@pytest.mark.parametrize("loss,grad,ldg", [(None, None, 0), (Cp, D, 99), (Cp + 2, D, 100), (Cp, D + 1, 100), (Cp, A, 101), (Cp, A + 100, 100), (Cp, Bp, 100), (A + 8, D, 100),
                                           (Bp + 4, D, 100), (D + 4, D, 100), (Cp, A - 2, 100), (Cp, D, 1 << 60)])
def test_distillation_output_refusals(L, loss, grad, ldg):
    spec = _spec()
    assert L.ceca_distill(ctypes.byref(spec), loss, grad, ldg, W, 1 << 30, None) == B.CECA_EINVAL and L.ceca_last_error()


def test_distillation_outputs_apart_from_every_input(L):
    for name in ("peer", "labels", "weight"):
        spec = _spec(hard=0.5, labels=W, **({name: Cp} if name != "labels" else {}))
        if name == "labels":
            spec.labels = Cp
        assert L.ceca_distill(ctypes.byref(spec), Cp, D, 100, W + (1 << 20), 1 << 30, None) == B.CECA_EINVAL, name
    assert L.ceca_distill(None, Cp, D, 100, W, 0, None) == B.CECA_EINVAL
    assert L.ceca_distill_workspace_bytes(None) == B.CECA_EINVAL


def _top(L, logits=A, type=1, ld=100, rows=3, V=100, K=5, top=Bp, ids=Cp, ws=W, wbytes=1 << 30):
    return L.ceca_top_logits(logits, type, ld, rows, V, K, top, ids, ws, wbytes, None)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(top=None), dict(ids=None), dict(type=5), dict(ld=99), dict(rows=-1), dict(V=0), dict(K=0), dict(K=257), dict(logits=A + 1), dict(top=Bp + 2),
                                 dict(ids=Cp + 1), dict(top=A), dict(ids=A + 200), dict(ids=Bp + 4), dict(ld=1 << 60)])
def test_top_logits_refusals(L, bad):
    assert _top(L, **bad) == B.CECA_EINVAL and L.ceca_last_error()


def test_nothing_to_do(L):
    assert _embed(L, T=0, tokens=None, out=None) == B.CECA_OK
    assert _top(L, rows=0, logits=None, top=None, ids=None) == B.CECA_OK
    spec = _spec(T=0, logits=None, top=None, ids=None)
    assert L.ceca_distill(ctypes.byref(spec), None, None, 0, None, 0, None) == B.CECA_OK


def test_binding_refuses_types_shapes_and_devices(L):
    n, T, V, h, K = 2, 3, 10, 4, 2
    E, tok, out = torch.zeros(n, V * h), torch.zeros(n, T, dtype=torch.int32), torch.zeros(n, T, h)
    logits, top, ids = torch.zeros(n, T, V), torch.zeros(n, T, K), torch.zeros(n, T, K, dtype=torch.int32)
    make = lambda **kw: P.make_distill(**(dict(logits=logits, n=n, T=T, V=V, top=top, ids=ids) | kw))  # noqa: E731
    spec = make()
    calls = [
        lambda: P.ceca_embed(E, n, V, h, tok, out),                                     # host memory
        lambda: P.ceca_embed(E.double(), n, V, h, tok, out),
        lambda: P.ceca_embed(E[:, :-1], n, V, h, tok, out),
        lambda: P.ceca_embed(E, n, V, h, tok.long(), out),
        lambda: P.ceca_embed(E, n, V, h, tok.reshape(-1)[:5], out),
        lambda: P.ceca_embed(E, n, V, h, tok.t(), out),
        lambda: P.ceca_embed(E, n, V, h, tok, out[:, :, :3]),
        lambda: P.ceca_embed(E, n, V, h, tok, out.double()),
        lambda: P.ceca_embed(E, n, V, h, tok, torch.zeros(n, 2 * T, h)[:, :T]),         # rows not at one pitch
        lambda: P.ceca_embed(E, n, V, h, tok, torch.zeros(n, T, 2 * h)[:, :, ::2]),
        lambda: P.ceca_embed(E, 0, V, h, tok, out),
        lambda: P.ceca_embed_grad(out, n, V, h, tok, E),
        lambda: P.ceca_embed_grad(out.half().int(), n, V, h, tok, E),
        lambda: P.ceca_distill(spec, loss=torch.zeros(n, T)),                           # host memory
        lambda: P.ceca_distill(spec, loss=torch.zeros(n, T + 1)),
        lambda: P.ceca_distill(spec, loss=torch.zeros(n, T).double()),
        lambda: P.ceca_distill(spec, grad=logits.half()),
        lambda: P.ceca_distill(spec, grad=logits[:, :, :-1]),
        lambda: make(ids=None), lambda: make(ids=ids.long()), lambda: make(top=top.half()), lambda: make(top=top[:, :, :1]), lambda: make(peer=torch.zeros(n)),
        lambda: make(labels=torch.zeros(n, T, dtype=torch.int64)), lambda: make(weight=torch.zeros(n)), lambda: make(logits=logits.double()), lambda: make(logits=logits[:, :, 1:]),
        lambda: make(n=0), lambda: make(V=0),
        lambda: P.ceca_top_logits(logits, n * T, V, K, top, ids),                       # host memory
        lambda: P.ceca_top_logits(logits, n * T, V, K, top, ids.long()),
        lambda: P.ceca_top_logits(logits, n * T, V, K + 1, top, ids),
        lambda: P.ceca_top_logits(logits.int(), n * T, V, K, top, ids),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(P.CecaError) as e:
            call()
        assert e.value.code == B.CECA_EINVAL, k
    # pitches of views
    assert make(logits=torch.zeros(n, T, V + 3)[:, :, :V]).ld == V + 3
    assert make(logits=torch.zeros(n * T, V)).ld == V
