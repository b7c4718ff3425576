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
