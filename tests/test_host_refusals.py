"""Arguments of no use to the calls on chosen pages and to sampling: refused with an error that says which, before memory is taken for them."""
import pytest

torch = pytest.importorskip("torch")

import numpy as np  # noqa: E402

import paper_2605_17415_amd as pkg  # noqa: E402
from test_host_kv_streams import world  # noqa: E402,F401
from test_host_sample import told  # noqa: E402,F401


@pytest.mark.parametrize("name", ("temperature", "top_k", "top_p", "min_p"))
def test_settings_that_are_no_numbers(told, name):  # noqa: F811
    x, u = told.tensor(3, 50, dtype=torch.float32), told.tensor(3, dtype=torch.float32)
    for bad in (None, "1", [1.0], 1j, *((50.0, np.float32(2)) if name == "top_k" else ())):
        with pytest.raises(TypeError, match=name):
            pkg.sample_tokens(x, u, **{name: bad})
    for bad in ((1 << 31, -(1 << 40)) if name == "top_k" else (10 ** 400,)):
        with pytest.raises(ValueError, match=name):
            pkg.sample_tokens(x, u, **{name: bad})
    assert not told.launched and not told.allocated
    for good in (1, True, np.int64(1), *(() if name == "top_k" else (1.0, np.float32(0.5), np.float64(0.25)))):
        told.launched.clear()
        pkg.sample_tokens(x, u, **{name: good})
        assert len(told.launched) == 1


@pytest.mark.parametrize("count", (-1, 0, 4097, 1 << 40))
def test_more_pages_than_a_row_is_given_take_no_memory(world, count):  # noqa: F811
    scores, lengths = world.tensor(3, 2, 4, dtype=torch.float32), world.tensor(3)
    with pytest.raises(ValueError, match="count"):
        pkg.kv_select(scores, lengths, 16, count)
    assert not world.allocated and not world.launched


def test_arguments_that_are_no_tensors(world):  # noqa: F811
    t = world.tensor
    pool, q, table, lengths, scores = t(4, 2, 2, 16, 64, dtype=torch.float16), t(3, 2, 64, dtype=torch.float16), t(3, 4), t(3), t(3, 2, 4, dtype=torch.float32)
    for bad in (None, [0, 1, 2], torch.zeros(3, dtype=torch.int32)):
        with pytest.raises(TypeError, match="lengths"):
            pkg.kv_select(scores, bad, 16, 2)
        with pytest.raises(TypeError, match="chosen"):
            pkg.kv_attend_pages(q, pool, table, lengths, bad)
        with pytest.raises(TypeError, match="digests"):
            pkg.kv_digest(pool, bad, table, lengths)
    assert not world.launched
