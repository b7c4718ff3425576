"""Which stream and which device the key-value cache's calls take memory for and launch on, without a GPU: tensors that say they are on a
device, streams and devices that only note that they are current, a library that notes what it is called with."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")

import paper_2605_17415_amd as pkg  # noqa: E402
from paper_2605_17415_amd import kv  # noqa: E402


class World:
    """What is current, what was allocated where, what was launched where."""

    def __init__(self):
        self.device, self.stream = 0, "caller"
        self.allocated, self.recorded, self.launched = [], [], []

    @contextlib.contextmanager
    def using(self, **what):
        was = self.device, self.stream
        self.device, self.stream = what.get("device", self.device), what.get("stream", self.stream)
        yield
        self.device, self.stream = was


@pytest.fixture
def world(monkeypatch):
    w = World()

    class OnDevice(torch.Tensor):
        where = torch.device("cuda", 0)
        is_cuda = True

        @property
        def device(self):
            return self.where

        @classmethod
        def __torch_function__(cls, func, kinds, args=(), kwargs=None):
            out = super().__torch_function__(func, kinds, args, kwargs or {})
            if func in (torch.Tensor.new_empty, torch.empty_like):
                out.where = args[0].where
                w.allocated.append((out.where.index, w.stream))
            return out

        def record_stream(self, stream):
            w.recorded.append(stream)

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("workspace"):
                    return 256
                w.launched.append((name, w.device, args[-1]))
                return 0
            return call

    monkeypatch.setattr(kv, "_library", lambda: Library())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: w.using(stream=s, device=s.device.index))
    monkeypatch.setattr(torch.cuda, "device", lambda d: w.using(device=torch.device(d).index))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: w.stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: w.device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: w.device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: w.stream if isinstance(w.stream, int) else (1000 + d), raising=False)

    def tensor(*shape, dtype=torch.int32, device=0):
        t = torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)
        t.where = torch.device("cuda", device)
        return t

    w.tensor = tensor
    return w


def side(device=0):
    return types.SimpleNamespace(cuda_stream=77, device=torch.device("cuda", device))


def calls(w, device=0):
    """Every call, and how many tensors it gives back."""
    def t(*shape, dtype=torch.int32):
        return w.tensor(*shape, dtype=dtype, device=device)
    pool, q = t(4, 2, 2, 16, 64, dtype=torch.float16), t(3, 2, 64, dtype=torch.float16)
    table, lengths, refs, ids, pools = t(3, 4), t(3), t(4), t(3), t(1, 4, 16, dtype=torch.uint8)
    return {
        "append": (lambda **s: pkg.kv_append(pool, q, q, table, lengths, **s), 0),
        "read": (lambda **s: pkg.kv_read(pool, table, lengths, q, q, **s), 0),
        "attend": (lambda **s: pkg.kv_attend(q, pool, table, lengths, **s), 1),
        "reserve": (lambda **s: pkg.kv_reserve(table, lengths, refs, ids, 16, **s), 1),
        "fork": (lambda **s: pkg.kv_fork(pools, table, lengths, refs, ids, ids, 16, **s), 1),
        "free": (lambda **s: pkg.kv_free(table, lengths, refs, ids, **s), 0),
        "trim": (lambda **s: pkg.kv_trim(table, lengths, refs, 16, 8, **s), 0),
        "compact": (lambda **s: pkg.kv_compact(pools, table, refs, **s), 1),
        "copy": (lambda **s: pkg.kv_copy(pools, ids, ids, **s), 0),
    }


ALL = ("append", "read", "attend", "reserve", "fork", "free", "trim", "compact", "copy")


@pytest.mark.parametrize("name", ALL)
def test_memory_is_taken_for_the_stream_that_uses_it(world, name):
    """Memory from another stream's share of the caching allocator may still be in use by that stream: no record_stream changes that."""
    call, results = calls(world)[name]
    s = side()
    call(stream=s)
    assert [x[2] for x in world.launched] == [77]
    assert all(stream is s for _, stream in world.allocated), world.allocated
    assert len(world.allocated) >= results
    # what is given back is read by the caller's stream: its memory is not handed on before that stream has passed the reads
    assert world.recorded == ["caller"] * results
    assert world.stream == "caller"


@pytest.mark.parametrize("name", ALL)
def test_without_a_stream_the_current_one_is_used(world, name):
    call, _ = calls(world)[name]
    call()
    assert [x[2] for x in world.launched] == [1000]
    assert all(x == (0, "caller") for x in world.allocated) and not world.recorded


@pytest.mark.parametrize("name", ALL)
def test_a_cache_on_another_device_than_the_current_one(world, name):
    """The library launches on the current device: it is the cache's for the length of the call."""
    call, _ = calls(world, device=1)[name]
    call()
    assert [x[1:] for x in world.launched] == [(1, 1001)]
    assert all(x[0] == 1 for x in world.allocated)
    assert world.device == 0
    world.launched.clear()
    call(stream=side(1))
    assert [x[1:] for x in world.launched] == [(1, 77)]
    assert (world.device, world.stream) == (0, "caller")


@pytest.mark.parametrize("name", ALL)
def test_a_stream_of_another_device_is_refused(world, name):
    call, _ = calls(world)[name]
    with pytest.raises(ValueError):
        call(stream=side(1))
    assert not world.launched


@pytest.mark.parametrize("which", ("k", "v", "q", "out", "pool"))
def test_a_gradient_that_would_be_lost_is_refused(world, which):
    """There is no backward pass: what asks for one is refused, unless gradients are off."""
    pool, table, lengths = world.tensor(4, 2, 2, 16, 64, dtype=torch.float16), world.tensor(3, 4), world.tensor(3)
    q, k, v, out = (world.tensor(3, 2, 64, dtype=torch.float16) for _ in range(4))
    {"k": k, "v": v, "q": q, "out": out, "pool": pool}[which].requires_grad_()

    def call():
        if which in "kv":
            pkg.kv_append(pool, k, v, table, lengths)
        else:
            pkg.kv_attend(q, pool, table, lengths, out=out)

    with pytest.raises(ValueError, match="gradient"):
        call()
    assert not world.launched
    with torch.no_grad():
        call()
    assert len(world.launched) == 1
