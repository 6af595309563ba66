"""sc_rope_rotate takes tensors of one GPU: host memory is refused before anything is launched."""
import pytest
import torch

import paper_2609_22283_amd as sc


def _refused(rope, x, y, pos, **kw):
    with pytest.raises(sc.ScError) as e:
        sc.sc_rope_rotate(rope, x, y, pos, **kw)
    assert e.value.code == sc.SC_EINVAL


def _tensors(device, dtype=torch.bfloat16):
    return (torch.ones(3, 2, 8, dtype=dtype, device=device), torch.full((3, 2, 8), 7.0, dtype=dtype, device=device),
            torch.zeros(3, 3, dtype=torch.int32, device=device))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_host_tensors(dtype):
    """CPU only"""
    rope = sc.binding.Rope(sc.binding.sc_rope_desc(1, 1, 8, 0, 0, 16, 10000.0), 1 << 20)
    for device in ("cpu", "meta"):
        x, y, pos = _tensors(device, dtype)
        for out in (x, y):
            _refused(rope, x, out, pos)
            _refused(rope, x, out, pos, stream=0)
    x, y, pos = _tensors("cpu", dtype)
    sc.sc_rope_rotate(rope, x[:0], y[:0], pos[:0])  # of no rows nothing is read


@pytest.mark.gpu
def test_one_of_them_on_the_host():
    table = torch.empty(sc.sc_rope_table_bytes(1, 1, (8, 0, 0), 16), dtype=torch.uint8, device="cuda")
    rope = sc.sc_rope_table_build(table, 1, 1, (8, 0, 0), 16)
    x, y, pos = _tensors("cuda")
    hx, hy, hpos = _tensors("cpu")
    for bad in ((hx, y, pos), (x, hy, pos), (x, y, hpos), (hx, hx, pos), (x, x, hpos), (hx, hy, hpos)):
        _refused(rope, *bad)
        _refused(rope, *bad, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool((y == 7.0).all()) and bool((x == 1.0).all())
    sc.sc_rope_rotate(rope, x, y, pos)
    torch.cuda.synchronize()
    assert torch.equal(y, x)
