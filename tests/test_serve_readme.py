"""The decoding step as the documents show it, in a batch with a request that is idle in the step."""
import os
import re
import textwrap

import numpy as np
import pytest

import serve_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def shown(where):
    from paper_2002_12798_b200 import ops

    if where == "README":
        blocks = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), re.S)
        return next(b for b in blocks if "pages_extend" in b)
    lines = ops.__doc__.splitlines()
    return textwrap.dedent("\n".join(line for line in lines if line.startswith("    ")))


@pytest.mark.parametrize("where", ["README", "docstring"])
def test_the_step_in_the_documents(where):
    from paper_2002_12798_b200 import ops

    torch.manual_seed(0)
    code = shown(where)
    assert "attend" in code
    n, q_heads, kv_heads, dim, page_size = 5, 8, 2, 128, 16
    one = dict(dtype=torch.int32, device="cuda")
    x = torch.randn(n, q_heads + 2 * kv_heads, dim, device="cuda", dtype=torch.bfloat16)
    pages = [torch.randn(64, page_size, kv_heads, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    held = torch.tensor([40, 17, 0, 5, 30], **one)
    table = torch.full((n, 8), -1, **one)
    for r, length in enumerate(held.tolist()):
        table[r, : -(-length // page_size)] = torch.arange(8 * r, 8 * r - (-length // page_size), **one)
    new = torch.tensor([1, 0, 0, 1, 1], **one)  # one idle with tokens, one that has not begun
    names = dict(torch=torch, ops=ops, max_requests=n, q_heads=q_heads, kv_heads=kv_heads, k_pages=pages[0], v_pages=pages[1], new_lens=new, seq_lens=held,
                 block_table=table, free_pages=torch.arange(40, 64, **one), free_count=torch.tensor([24], **one), page_size=page_size, max_tokens=n,
                 q=x[:, :q_heads], k=x[:, q_heads : q_heads + kv_heads], v=x[:, q_heads + kv_heads :], done=torch.zeros(n, dtype=torch.bool, device="cuda"),
                 positions=torch.zeros(3, n, **one))
    if where == "docstring":
        names.update(rope=ops.RopePlan(dim), cache=ops.PagedCache(*pages), attention=ops.AttendPlan(n, q_heads, kv_heads, dim))
    exec(code, names)
    step, out = names["step"], names["out"].float().cpu().double().numpy()
    assert step.requests.tolist() == [0, 3, 4, -1, -1] and step.seq_lens.tolist() == [41, 17, 0, 6, 31]
    rope = names["rope"]
    turned = rope.rotate([x[:, :q_heads]], torch.stack([step.positions] * rope.n_axes))[0].float().cpu().double().numpy()
    k, v = (p.float().cpu().double().numpy() for p in pages)
    table, lens = table.cpu().numpy(), step.seq_lens.cpu().numpy()
    for token, r in enumerate([0, 3, 4]):
        want, _, size, mass = ref.attend(turned[token : token + 1], k, v, table[r : r + 1], lens[r : r + 1], dim**-0.5)
        bound, _ = ref.attend_bound(want, size, mass, dim, "bf16")
        assert (np.abs(out[r] - want[0]) <= bound[0]).all(), r
    assert not out[2].any()
