"""What the binding and the library refuse, and how they cut their work, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    return binding


def test_memory_that_is_lent_is_contiguous_and_on_the_device(b):
    class OnDevice:      # (the questions that the binding asks of a tensor)
        is_cuda = True

        def __init__(self, t):
            self.t = t

        def __getattr__(self, name):
            return getattr(self.t, name)
    host = torch.empty(6)
    assert b._lent(None, "x") == (None, 0)
    assert b._lent(OnDevice(host), "x") == (host.data_ptr(), 24)
    with pytest.raises(TypeError):
        b._lent(host, "x")
    for t in (host[::2], host[:1].expand(6), host.reshape(2, 3).t()):
        with pytest.raises(ValueError):
            b._lent(OnDevice(t), "x")


def test_a_cache_of_the_host_is_refused(b):
    for device in ("cpu", torch.device("cpu"), "meta"):
        with pytest.raises(TypeError):
            b.KvCache(4, 2, 64, 16, device=device)
