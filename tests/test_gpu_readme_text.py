"""The language-model example printed in README.md runs as written, behind the first one's imports, and its gradient is the oracle's."""
import os
import re

import numpy as np
import pytest

from oracle import text as OT

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_readme_language_model_example_runs():
    import torch
    import paper_2306_00256_amd as P
    from paper_2306_00256_amd import binding as B
    torch.manual_seed(0)
    code = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), flags=re.S)[1]
    scope = {"torch": torch, "P": P, "B": B}
    exec(compile(code, "README.md", "exec"), scope)
    torch.cuda.synchronize()
    S, e, loss, n, T, V = (scope[k] for k in ("S", "e", "loss", "n", "T", "V"))
    assert torch.isfinite(S).all() and torch.isfinite(loss).all()
    # the last iteration's gradient rows from its logits' gradient: sums of c terms of bf16, (c + 2) half fp32 steps
    want, size, terms = OT.embed_grad(scope["logits"].double().cpu().numpy(), scope["tokens"].cpu().numpy(), V, 1.0)
    got = e.double().cpu().numpy().reshape(n, V, V)
    assert (np.abs(got - want) <= (terms[..., None] + 2) * 2.0 ** -24 * size).all()
