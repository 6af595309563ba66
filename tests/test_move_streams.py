"""Which streams the pool that a cache leaves behind is recorded on (CPU only: nothing is cached, so that
nothing is launched, and the pools and streams are stand-ins)."""
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd import binding


class Pool:
    """As much of a torch tensor as a cache looks at."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, at):
        self.at, self.recorded = at, []

    def data_ptr(self):
        return self.at

    def record_stream(self, stream):
        self.recorded.append(stream)


@pytest.fixture
def streams(monkeypatch):
    monkeypatch.setattr(binding, "_default_streams", {}, raising=False)
    monkeypatch.setattr(binding._torch.cuda, "default_stream", lambda device: ("default", device))
    monkeypatch.setattr(binding._torch.cuda, "ExternalStream", lambda raw, device: (raw, device))


def _cache(pool):
    return sc.sc_cache_create(pool, 1, 1, 128, 32, 1, 4, sc.SC_DTYPE_FP4)


@pytest.mark.parametrize("raw,stream", [(0, ("default", "cuda:0")), (4711, (4711, "cuda:0"))])
@pytest.mark.parametrize("given", [True, False])
def test_the_old_pool_is_recorded_on_the_moves_stream(streams, monkeypatch, raw, stream, given):
    """The default stream too: a pool of a side stream would go back to that one's memory at once."""
    a, b = Pool(1 << 20), Pool(1 << 30)
    c = _cache(a)
    f = c.fork()
    if not given:
        monkeypatch.setattr(binding, "_stream", lambda s: raw)
    f.move(b, 6, stream=raw if given else None)
    assert a.recorded == [stream] and not b.recorded and c.pool is f.pool is b and c.desc.n_slots == 6
    c.move(a, 4, stream=raw)
    assert b.recorded == [stream] and a.recorded == [stream] and f.pool is a and f.desc.n_slots == 4


def test_a_move_that_fails_keeps_the_pool(streams):
    a = Pool(1 << 20)
    c = _cache(a)
    with pytest.raises(sc.ScError):
        c.move(Pool((1 << 20) + 16), 4)
    assert c.pool is a and not a.recorded and c.desc.n_slots == 4


def test_handles_know_their_pool_if_it_cannot_be_recorded(streams):
    """The pages have gone to the new pool by then."""
    a, b = Pool(1 << 20), Pool(1 << 30)
    a.record_stream = None
    c = _cache(a)
    with pytest.raises(TypeError):
        c.move(b, 6, stream=7)
    assert c.pool is b and c.desc.n_slots == 6
