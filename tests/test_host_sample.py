"""Sampling's C ABI and its binding without a GPU: every declared symbol is exported and bound, and what the host can see to be wrong is refused
before anything is launched."""
import ctypes as C
import os
import re

import pytest

torch = pytest.importorskip("torch")

import paper_2605_17415_amd as pkg  # noqa: E402
from paper_2605_17415_amd import sample  # noqa: E402
from test_host_kv_streams import side, world  # noqa: E402,F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE, ODD = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 2)


@pytest.fixture(scope="module")
def lib():
    return sample._library()


def logits(**changes):
    return sample._Logits(**{**dict(data=HERE, row_stride=1000, rows=3, vocabulary=1000, type=1), **changes})


def how(**changes):
    return sample._Sampling(**{**dict(temperature_all=1.0, top_p_all=1.0), **changes})


def call(lib, x=None, s=None, u=HERE, tokens=HERE, logprobs=None, work=HERE, size=1 << 40):
    return lib.ivftq_sample_tokens(C.byref(x or logits()), u, C.byref(s or how()), tokens, logprobs, work, size, None)


def test_every_declared_symbol_is_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ivftq_sample.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(ivftq_[a-z_0-9]+)\s*\(", text)))
    assert declared == sorted(pkg.declared_sample_symbols())
    for name in declared:
        assert hasattr(lib, name)


@pytest.mark.parametrize("change,status", [(dict(type=3), 1), (dict(type=-1), 1), (dict(vocabulary=0), 6), (dict(vocabulary=(1 << 20) + 1, row_stride=1 << 21), 6),
                                           (dict(rows=-1), 1), (dict(rows=1 << 22), 1), (dict(row_stride=999), 1), (dict(row_stride=-1000), 1), (dict(data=None), 1),
                                           (dict(data=C.c_void_p((1 << 20) + 1)), 1), (dict(data=ODD, type=2), 1)])
def test_logits_that_are_refused(lib, change, status):
    assert call(lib, logits(**change)) == status
    assert lib.ivftq_sample_workspace(C.byref(logits(**change)), None) == -1


@pytest.mark.parametrize("change", [dict(temperature_all=-0.5), dict(temperature_all=float("nan")), dict(top_k_all=-1), dict(top_p_all=-0.1), dict(top_p_all=1.5),
                                    dict(top_p_all=float("nan")), dict(min_p_all=-0.1), dict(min_p_all=1.1), dict(min_p_all=float("nan")), dict(temperature=ODD),
                                    dict(top_k=ODD), dict(top_p=ODD), dict(min_p=ODD)])
def test_settings_that_are_refused(lib, change):
    assert call(lib, s=how(**change)) == 1


def test_the_rest(lib):
    assert call(lib, u=None) == call(lib, tokens=None) == call(lib, u=ODD) == call(lib, tokens=ODD) == call(lib, logprobs=ODD) == 1
    assert call(lib, logits(rows=0, data=None), u=None, tokens=None) == 0
    assert lib.ivftq_sample_tokens(None, HERE, C.byref(how()), HERE, None, HERE, 1 << 40, None) == 1
    assert lib.ivftq_sample_tokens(C.byref(logits()), HERE, None, HERE, None, HERE, 1 << 40, None) == 1
    assert lib.ivftq_sample_workspace(C.byref(logits()), None) == 0
    large = logits(vocabulary=70_000, row_stride=70_000)
    need = lib.ivftq_sample_workspace(C.byref(large), None)
    assert need > 0 and need % 256 == 0
    assert call(lib, large, size=need - 1) == call(lib, large, work=None) == call(lib, large, work=C.c_void_p((1 << 20) + 16)) == 1
    # many rows are taken a slice at a time
    assert lib.ivftq_sample_workspace(C.byref(logits(vocabulary=70_000, row_stride=70_000, rows=5000)), None) < 1 << 27
    # what any settings need is enough for each
    for v in (1000, 20_000, 40_000, 70_000):
        for rows in (1, 255, 256):
            x = logits(vocabulary=v, row_stride=v, rows=rows)
            most = lib.ivftq_sample_workspace(C.byref(x), None)
            assert all(0 <= lib.ivftq_sample_workspace(C.byref(x), C.byref(how(**s))) <= most
                       for s in (dict(), dict(top_k=HERE), dict(temperature=HERE), dict(top_k_all=50), dict(top_k_all=5000), dict(top_p_all=0.5), dict(temperature_all=0.0)))


@pytest.fixture
def told(world, monkeypatch):  # noqa: F811
    """The library that notes what it is called with, for sampling too."""
    from paper_2605_17415_amd import kv
    monkeypatch.setattr(sample, "_library", lambda: kv._library())
    return world


def test_memory_streams_and_devices(told):
    for device in (0, 1):
        x, u = told.tensor(3, 50, dtype=torch.float16, device=device), told.tensor(3, dtype=torch.float32, device=device)
        s = side(device)
        told.launched.clear(), told.allocated.clear(), told.recorded.clear()
        pkg.sample_tokens(x, u, stream=s)
        assert [y[1:] for y in told.launched] == [(device, 77)] and told.recorded == ["caller"]
        assert told.allocated and all(y == (device, s) for y in told.allocated)
        pkg.sample_tokens(x, u)
        assert told.launched[-1][1:] == (device, 1000 + device) and (told.device, told.stream) == (0, "caller")
        with pytest.raises(ValueError):
            pkg.sample_tokens(x, u, stream=side(1 - device))


def test_tensors_that_are_refused(told):
    t = told.tensor
    x, u = t(3, 50, dtype=torch.float32), t(3, dtype=torch.float32)
    for bad in (t(3, 50, dtype=torch.int32), t(3, 50, dtype=torch.float64)):
        with pytest.raises(TypeError):
            pkg.sample_tokens(bad, u)
    for bad in (t(50, dtype=torch.float32), t(3, 100, dtype=torch.float32)[:, ::2]):
        with pytest.raises(ValueError):
            pkg.sample_tokens(bad, u)
    for bad in (t(4, dtype=torch.float32), t(3, dtype=torch.float16), t(3, 1, dtype=torch.float32)):
        with pytest.raises(ValueError):
            pkg.sample_tokens(x, bad)
        with pytest.raises(ValueError):
            pkg.sample_tokens(x, u, logprobs=bad)
        for name in ("temperature", "top_p", "min_p"):
            with pytest.raises(ValueError):
                pkg.sample_tokens(x, u, **{name: bad})
    for bad in (t(3, dtype=torch.float32), t(2), t(3, dtype=torch.int64)):
        with pytest.raises(ValueError):
            pkg.sample_tokens(x, u, top_k=bad)
        with pytest.raises((TypeError, ValueError)):
            pkg.sample_tokens(x, u, out=bad)
    with pytest.raises(TypeError):
        pkg.sample_tokens(torch.zeros(3, 50), u)
    assert not told.launched
    x.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        pkg.sample_tokens(x, u)
    with torch.no_grad():
        pkg.sample_tokens(x, u)
    assert len(told.launched) == 1
