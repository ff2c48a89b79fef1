"""In the language-model example printed in README.md an agent's teacher is its peer's model for the agent's own tokens."""
import os
import re

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_readme_teachers_see_the_students_tokens():
    import torch
    import paper_2306_00256_amd as P
    from paper_2306_00256_amd import binding as B
    torch.manual_seed(1)
    code = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), flags=re.S)[1]
    # one iteration, so that the entries are those of the tables the run begins with
    scope = {"torch": torch, "P": P, "B": B}
    exec(compile(code.replace("range(20)", "range(1)"), "README.md", "exec"), scope)
    torch.cuda.synchronize()
    n, V, T, K, peer = (scope[k] for k in ("n", "V", "T", "K", "peer"))
    z = scope["R"][:n].view(n, V, V)                       # S and R are exchanged at the end of an iteration; x = y at the beginning
    for i in range(n):
        own = z[peer[i]][scope["tokens"][i].long()].bfloat16().float()          # the peer's logits for agent i's tokens
        want = torch.sort(own, dim=1, descending=True)[0][:, :K]
        assert torch.equal(scope["top"].view(n, T, K)[peer[i]], want)
