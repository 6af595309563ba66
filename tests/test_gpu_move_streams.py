"""A pool that a cache leaves behind on one stream and that was allocated on another."""
import pytest
import torch

import paper_2609_22283_amd as sc
from synth import TAG_K, normal

from fp4_cases import D, bf16_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("given", [True, False])
def test_a_side_streams_pool_moved_on_the_default_stream(given):
    heads, tpp, n = 2, 64, 40
    args = (1, heads, D, tpp, 1, n, sc.SC_DTYPE_FP4)
    size = sc.sc_cache_pool_bytes(*args)
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = sc.sc_cache_create(torch.empty(size, dtype=torch.uint8, device="cuda"), *args)
    torch.cuda.synchronize()
    kd, _ = bf16_dev(normal((tpp, heads, D), (8, TAG_K)))
    for i in range(n):
        c.append(0, (i, 0), kd, kd)
    want, to, left = c.pool.clone(), torch.zeros(size, dtype=torch.uint8, device="cuda"), c.pool.data_ptr()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    c.move(to, n, **({"stream": torch.cuda.default_stream()} if given else {}))
    with torch.cuda.stream(side):
        other = torch.zeros(size, dtype=torch.uint8, device="cuda")
    assert other.data_ptr() != left
    torch.cuda.synchronize()
    assert torch.equal(to, want) and not bool(other.any())
