"""Arguments that are left out, and calls that the arguments alone show to be wrong."""
import numpy as np
import pytest

import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def queries(seed, rows, heads, d, dtype):
    return (torch.randn(rows, heads, d, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype).to(DEV)


@pytest.mark.parametrize("form", ("f16", "code4"))
@pytest.mark.parametrize("news", ([3, 0, 2], [70, 0, 33]))
def test_every_row_has_a_result_where_max_new_is_not_given(form, news):
    lens = [200, 30, 75]
    c = ref.Cache(51, form, 2, 64, 16, lens)
    t, codec = c.device()
    q = queries(51, sum(news), 4, 64, torch.float16)
    starts = torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)
    out = torch.full_like(q, float("nan"))
    assert _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, out=out, **codec) is out
    torch.cuda.synchronize()
    ref.check_attention(c, q.cpu(), out, news)


def test_every_row_has_a_result_where_max_new_is_not_given_to_the_object():
    cache = _pkg().KVCache(1, 2, 64, pages=20, sequences=2, tokens=100, page=16, dtype=torch.float16, device=DEV)
    news = [9, 5]
    cache.reserve(torch.tensor(news, dtype=torch.int32, device=DEV))
    q, k, v = queries(1, 14, 4, 64, torch.float16), queries(2, 14, 2, 64, torch.float16), queries(3, 14, 2, 64, torch.float16)
    starts = torch.tensor([0, 9, 14], dtype=torch.int32, device=DEV)
    cache.append(0, k, v, starts)
    out = torch.full_like(q, float("nan"))
    cache.attend(0, q, starts, out=out)
    want = cache.attend(0, q, starts, max_new=9)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_no_rows_and_no_max_new():
    c = ref.Cache(52, "f16", 2, 64, 16, [20])
    t, _ = c.device()
    none = torch.empty(0, 4, 64, dtype=torch.float16, device=DEV)
    out = _pkg().kv_attend(none, t["pool"], t["table"], t["lengths"], starts=torch.zeros(2, dtype=torch.int32, device=DEV))
    assert out.shape == none.shape


@pytest.mark.parametrize("missing", (-1, 60))
def test_a_fork_of_a_missing_last_page_shows_nothing(missing):
    """The parent's last page is none of the pool: the child's is none either, and no page is taken (its content would be someone's)."""
    pkg = _pkg()
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    table, lengths, refs = torch.full((4, 3), -1, dtype=torch.int32, device=DEV), ints(20, 20, 0, 0), ints(1, 1, 1, 0, 0, 0)
    table[0, 0], table[0, 1] = 0, missing
    table[1, 0], table[1, 1] = 1, 2
    pools = torch.randn(1, 6, 2, 2, 16, 64, device=DEV).half()
    before = pools.clone()
    done = pkg.kv_fork(pools, table, lengths, refs, ints(0, 1), ints(2, 3), page=16)
    torch.cuda.synchronize()
    assert done.tolist() == [1, 1] and lengths.tolist() == [20] * 4
    assert table[2].tolist() == [0, -1, -1] and table[3].tolist() == [1, 3, -1]
    assert refs.tolist() == [2, 2, 1, 1, 0, 0]
    assert torch.equal(pools[:, 3], before[:, 2]) and torch.equal(pools[:, :3], before[:, :3]) and torch.equal(pools[:, 4:], before[:, 4:])


@pytest.mark.parametrize("new", (1, 70))
def test_results_may_take_the_queries_place_over_codes(new):
    """The queries are rotated into the workspace first, nothing reads them afterwards."""
    lens, news = [1300, 90], [new, new]
    c = ref.Cache(53, "code4", 2, 64, 16, lens)
    t, codec = c.device()
    q = queries(53, 2 * new, 4, 64, torch.bfloat16)
    starts = torch.tensor([0, new, 2 * new], dtype=torch.int32, device=DEV)
    want = _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, **codec)
    assert _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, out=q, **codec) is q
    torch.cuda.synchronize()
    assert torch.equal(q, want)
