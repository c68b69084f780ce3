"""Calls while another device than the cache's is current: refused before anything is launched, with each entry point.
The library and the tensors' checks are stood in for, so no GPU is needed."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2601_21758_amd import kv  # noqa: E402


@pytest.fixture
def cache(monkeypatch):
    """A cache on device 1 while device 0 is current; whatever reaches the library is a failure."""
    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_bytes"):
                    return 256
                raise AssertionError(f"{name} was called")
            return call

    monkeypatch.setattr(kv.L, "lib", Library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(kv, "_stream", lambda stream=None: 0 if stream is None else stream.cuda_stream)
    monkeypatch.setattr(kv, "_new", lambda stream, *a, dtype, device: torch.empty(*a, dtype=dtype))
    monkeypatch.setattr(kv, "_need", lambda t, dtype, name: t)
    c = kv.PagedCache.__new__(kv.PagedCache)
    c.device, c.dtype, c.used_on, c.page_size = torch.device("cuda", 1), torch.float16, None, 16
    c.c = types.SimpleNamespace(kv_heads=2, head_dim=64)
    c._c, c._ws_bytes, c._reorder_bytes, c.sizes = 0, 256, {}, ()
    c._ids = lambda t, name, n=None: 0
    c.data = c.refs = c.table = c.length = torch.zeros(1)
    return c


def calls(c, stream):
    one, two = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    sizes = dict(total_q=1, max_q=1, q_heads=2, stream=stream)
    return {"extend": lambda: c.extend(one, one, stream=stream), "fork": lambda: c.fork(one, one, one, stream=stream),
            "release": lambda: c.release(one, stream=stream), "copy": lambda: c.copy(one, one, stream=stream),
            "read": lambda: c.read(0, one, two, total=1, stream=stream),
            "reorder": lambda: c.reorder(one, one, stream=stream),
            "prefix_plan": lambda: kv.prefix_plan(c, one, two, None, None, **sizes),
            "window_plan": lambda: kv.window_plan(c, one, two, 5, 1, **sizes)}


@pytest.mark.parametrize("name", ["extend", "fork", "release", "copy", "read", "reorder", "prefix_plan", "window_plan"])
def test_another_device(cache, name):
    with pytest.raises(ValueError, match="another device than the call's stream"):
        calls(cache, None)[name]()
    other = types.SimpleNamespace(cuda_stream=7, device=torch.device("cuda", 0))
    with pytest.raises(ValueError, match="another device than the call's stream"):
        calls(cache, other)[name]()
