"""The key-value cache's calls on a stream that is not the current one, while the current one is busy: results as on the current stream."""
import numpy as np
import pytest

import kv_reference as ref
import test_gpu_kv_pages as plain

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def starts_of(news):
    return torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)


def queries(seed, rows, heads, d, dtype):
    return (torch.randn(rows, heads, d, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype).to(DEV)


def busy():
    """Some milliseconds of work on the current stream."""
    x = torch.ones(4096, 4096, device=DEV, dtype=torch.bfloat16)
    for _ in range(20):
        x = x @ x
    return x


@pytest.mark.parametrize("form,kind", [("bf16", "bf16"), ("code4", "f16")])
@pytest.mark.parametrize("new", (1, 70))
def test_two_calls_of_one_size_on_two_streams(form, kind, new):
    """The same workspace size twice, the first call waiting behind other work of its stream when the second one is made."""
    pkg = _pkg()
    lens, news = [2500, 900], [new, new]
    c = ref.Cache(31, form, 2, 64, 16, lens)
    t, codec = c.device()
    q = [queries(40 + i, 2 * new, 4, 64, ref.TYPES[kind]) for i in range(2)]
    starts, side = starts_of(news), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):                                      # the second time memory is there to be handed out again
        keep = busy()
        one = pkg.kv_attend(q[0], t["pool"], t["table"], t["lengths"], starts=starts, max_new=new, **codec)
        two = pkg.kv_attend(q[1], t["pool"], t["table"], t["lengths"], starts=starts, max_new=new, stream=side, **codec)
        torch.cuda.synchronize()
        del keep
        ref.check_attention(c, q[0].cpu(), one, news)
        ref.check_attention(c, q[1].cpu(), two, news)


@pytest.mark.parametrize("form,kind", [("f16", "f16"), ("code4", "bf16")])
@pytest.mark.parametrize("new", (1, 70))
def test_rows_and_attention_on_a_side_stream(form, kind, new):
    pkg = _pkg()
    lens, news = [300, 75], [new, new]
    c = ref.Cache(32, form, 2, 64, 16, lens)
    t, codec = c.device()
    q, k, v = (queries(50 + i, 2 * new, 4 if i == 0 else 2, 64, ref.TYPES[kind]) for i in range(3))
    other, back = t["pool"].clone(), [torch.full_like(k, 7) for _ in range(4)]
    lse, starts, side = torch.full(q.shape[:2], 5.0, device=DEV), starts_of(news), torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy()
    pkg.kv_append(t["pool"], k, v, t["table"], t["lengths"], starts=starts, stream=side, **codec)
    pkg.kv_read(t["pool"], t["table"], t["lengths"], back[0], back[1], starts=starts, stream=side, **codec)
    out = pkg.kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, max_new=new, lse=lse, stream=side, **codec)
    side.synchronize()
    c.take(t["pool"].cpu())
    ref.check_attention(c, q.cpu(), out, news, lse=lse)
    del keep
    pkg.kv_append(other, k, v, t["table"], t["lengths"], starts=starts, **codec)
    pkg.kv_read(other, t["table"], t["lengths"], back[2], back[3], starts=starts, **codec)
    torch.cuda.synchronize()
    assert torch.equal(other, t["pool"]) and torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])


def test_pages_on_a_side_stream():
    pkg = _pkg()
    s, p = plain.Both(12, 20, 60, 16), plain.Plain(12, 20, 60, 16)
    ints = {n: s.ints(x) for n, x in dict(first=[0, 1, 16, 17, 80, -3, 7, 0, 0, 0, 0, 0], parents=[3, 4, 1], children=[0, 7, 8], ended=[4, 3], more=[1] * 12,
                                          src=[0, 1], dst=[50, 51]).items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = busy()
    state = (s.table, s.lengths, s.refs)
    one = pkg.kv_reserve(*state, ints["first"], page=16, stream=side)
    done = pkg.kv_fork(s.pools, *state, ints["parents"], ints["children"], page=16, stream=side)
    two = pkg.kv_reserve(*state, ints["more"], page=16, stream=side)
    pkg.kv_free(*state, ints["ended"], stream=side)
    pkg.kv_trim(*state, page=16, window=20, sinks=1, stream=side)
    used = pkg.kv_compact(s.pools, s.table, s.refs, stream=side)
    pkg.kv_copy(s.pools, ints["src"], ints["dst"], stream=side)
    side.synchronize()
    assert np.array_equal(one.cpu().numpy(), p.reserve(ints["first"].tolist()))
    assert done.tolist() == p.fork([3, 4, 1], [0, 7, 8])
    assert np.array_equal(two.cpu().numpy(), p.reserve([1] * 12))
    p.free([4, 3])
    p.trim(20, 1)
    assert used.tolist() == [p.compact()]
    p.pools[:, 50], p.pools[:, 51] = p.pools[:, 0], p.pools[:, 1]
    for a, b in ((s.table, p.table), (s.lengths, p.lengths), (s.refs, p.refs), (s.pools, p.pools)):
        assert np.array_equal(a.cpu().numpy(), b)
    del keep
