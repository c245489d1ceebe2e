import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built libm3")


@pytest.fixture(scope="session")
def oracle_lib():
    import oracle
    oracle.build(force=False)
    return oracle


class FakeStream:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def two_streams(monkeypatch):
    """The binding on host tensors with a recorded library and two streams that are
    none: `log` holds what is done, and on which of them."""
    import torch

    from paper_2603_15569_amd import m3
    here, side = FakeStream(1), FakeStream(2)
    current, log = [here], []

    class On:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            current.append(self.s)

        def __exit__(self, *_):
            current.pop()

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_bytes"):
                    return 4096
                log.append((name, args[-1], current[-1].cuda_stream))
                return m3.M3_OK
            return call

    def allocates(name):
        plain = getattr(torch, name)

        def alloc(*args, **kw):
            log.append((name, current[-1].cuda_stream, current[-1].cuda_stream))
            return plain(*args, **kw)
        monkeypatch.setattr(torch, name, alloc)
    for name in ("empty", "zeros", "empty_like"):
        allocates(name)
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: current[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", FakeStream)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("kept for", s.cuda_stream, t.data_ptr())))
    lib = Library()
    monkeypatch.setattr(m3, "lib", lambda: lib)
    monkeypatch.setattr(m3, "_raw_stream", None)
    monkeypatch.setattr(m3, "_on_gpu", lambda x: None)
    caches = (m3._glr_dims, m3._glr_call, m3._ffn_dims)
    for c in caches:
        c.cache_clear()
    yield here, side, log
    for c in caches:      # (checks of host tensors that were let pass)
        c.cache_clear()
