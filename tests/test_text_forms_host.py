"""CPU: over the sizes that the language-model operators take, every kernel they launch is launched by a size of tests/text_forms.py, which
the GPU tests run.  A rule that moves without its sizes fails here."""
import math
import random

import pytest

import paper_2306_00256_amd as P
from paper_2306_00256_amd import binding as B
import text_forms as F


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not os.path.exists(P.library_path()):
        from paper_2306_00256_amd import build
        build.build_library(verbose=False)
    P.lib()


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def _sweep(draw, keys):
    rng = random.Random(5)
    found = {}
    for _ in range(6000):
        case = draw(rng)
        for key in keys(case):
            found.setdefault(key, case)
    return found


def _covered(found, cases, keys):
    have = set().union(*(keys(c) for c in cases))
    assert not {k: found[k] for k in found if k not in have}


def test_lookups():
    _covered(_sweep(lambda r: (r.choice(list(F.CODE)), _log(r, 1, 100), _log(r, 1, 20000), _log(r, 1, 3000)), F.lookup_keys), F.LOOKUPS, F.lookup_keys)


def test_gradients():
    draw = lambda r: (r.choice(list(F.CODE)), _log(r, 1, 60), _log(r, 1, 200000), _log(r, 1, 200000), _log(r, 1, 3000), r.random() < 0.5, r.choice([0, 0, 1]), r.choice([0, 0, 1]))  # noqa: E731
    _covered(_sweep(draw, F.gradient_keys), F.GRADIENTS, F.gradient_keys)


def test_distillations():
    _covered(_sweep(lambda r: (r.choice(list(F.CODE)), _log(r, 1, 3000), _log(r, 1, 400000)), F.distillation_keys), F.DISTILLATIONS, F.distillation_keys)


def test_tops():
    _covered(_sweep(lambda r: (r.choice(list(F.CODE)), _log(r, 1, 5000), _log(r, 1, 2000000), _log(r, 1, 256)), F.top_keys), F.TOPS, F.top_keys)


@pytest.mark.parametrize("bad", [dict(call=-1), dict(call=4), dict(flags=-1), dict(flags=16), dict(type=3), dict(n=0), dict(T=-1), dict(V=0), dict(width=0), dict(n=1 << 20, T=1 << 12)])
def test_refusals(bad):
    with pytest.raises(P.CecaError) as e:
        P.ceca_describe_text_launch(**(dict(call=B.TEXT_TOP, type=0, n=2, T=3, V=10, width=4, flags=0) | bad))
    assert e.value.code == B.CECA_EINVAL


def test_a_null_result_is_refused():
    assert P.lib().ceca_describe_text_launch(0, 0, 1, 1, 1, 1, 0, None) == B.CECA_EINVAL
