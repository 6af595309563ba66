"""sc_attention_weigh reads q again once o is written: an o that shares memory with q is
refused, before anything is written."""
import pytest
import torch

import paper_2609_22283_amd as sc

from memory_cases import MemCache, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_o_over_q_is_refused(dtype):
    case = MemCache(dtype, 2, 128, 64, 1, [(c, 0) for c in range(3)], seed=121)
    plan = sc.sc_plan_condition(case.cache, [(1, 0), (2, 0)], 24)
    rows, row = 48, 2 * 128
    buf = torch.zeros(4 * rows * row, dtype=case.tdt, device="cuda")
    at = 2 * rows * row - rows * row // 2  # q lies in the middle
    q = buf[at:at + rows * row].view(rows, 2, 128)
    q.copy_(case.queries(rows))
    w = case.weights()
    nb = sc.sc_attention_weigh_workspace_bytes(plan, case.cache)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    kept, before = buf.clone(), w.clone()
    for off in (0, 8, -8, rows * row - 8, 8 - rows * row):
        o = buf[at + off:at + off + rows * row]
        with pytest.raises(sc.ScError) as e:
            sc.sc_attention_weigh(plan, case.cache, 0, q, o, 0.1, w, ws, nb)
        assert e.value.code == sc.SC_EINVAL, off
    torch.cuda.synchronize()
    assert torch.equal(buf, kept) and torch.equal(w, before)
    want, sums = case.attend(q, [[(1, 0)], [(2, 0)]], 0.1)
    for off in (rows * row, -rows * row):  # side by side
        o = buf[at + off:at + off + rows * row].view(rows, 2, 128)
        w.copy_(before)
        sc.sc_attention_weigh(plan, case.cache, 0, q, o, 0.1, w, ws, nb)
        torch.cuda.synchronize()
        close(dtype, o, want, "o")
        exp = case.weights_after(before, sums)
        assert torch.allclose(w.double(), exp, rtol=1e-4, atol=1e-5)
