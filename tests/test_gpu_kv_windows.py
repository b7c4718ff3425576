"""Windows without first tokens where a row has just left the first token behind: the window of position p shows p - window + 1 .. p, so
at p = window token 0 is the one token that is outside.  Token 0 takes nearly all of the weight wherever it is seen."""
import math

import numpy as np
import pytest

import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"

FORMS = [("f16", "f16"), ("bf16", "bf16"), ("code4", "bf16"), ("code4", "f16")]


def heavy_beginning(seed, form, d, page, lens, rows, heads, kind):
    """A cache of one head whose sequences begin with a token that all queries look at, and such queries."""
    c = ref.Cache(seed, form, 1, d, page, lens)
    rng = np.random.default_rng(seed)
    u = rng.standard_normal(d)
    u /= np.linalg.norm(u)
    for b, n in enumerate(lens):
        if not n:
            continue
        p = c.table[b, 0]
        if form == "code4":
            c.codes[0, p, 0, 0] = np.abs((c.rotation.astype(np.float64) @ u)[:, None] - c.levels[None].astype(np.float64)).argmin(1)
            c.norms[0, p, 0, 0] = 15.0
        else:
            c.rows16[0, p, 0, 0] = torch.from_numpy(15 * u).to(c.rows16.dtype)
    q = torch.from_numpy(math.sqrt(d) * u + 0.3 * rng.standard_normal((rows, heads, d))).to(ref.TYPES[kind]).to(DEV)
    return c, q


def run(c, q, news, **mask):
    import paper_2605_17415_amd as pkg
    t, codec = c.device()
    lse = torch.full(q.shape[:2], 5.0, device=DEV)
    starts = torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)
    out = pkg.kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, max_new=max(news), lse=lse, **mask, **codec)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("window", (31, 32, 64, 128))
@pytest.mark.parametrize("new", (1, 3))
def test_few_rows_that_leave_the_first_token_behind(form, kind, window, new):
    lens = [window - 1, window, window + 1, window + 2, window + 3, 2 * window]
    news = [new] * len(lens)
    c, q = heavy_beginning(window + new, form, 64, 16, lens, sum(news), 2, kind)
    out, lse = run(c, q, news, window=window)
    ref.check_attention(c, q.cpu(), out, news, lse=lse, window=window)


@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("window", (32, 64, 65, 128, 200))
def test_row_tiles_that_end_where_the_first_token_is_left_behind(form, kind, d, page, window):
    """Rows are 64 tokens of two heads each: sequences whose last row tile ends at p = window and next to it, and one of whose row tiles
    inside does."""
    lens = [window, window + 1, window + 2, window + 1 + 64]
    news = [window, window + 1, window + 2, 128]
    c, q = heavy_beginning(window, form, d, page, lens, sum(news), 2, kind)
    out, lse = run(c, q, news, window=window)
    ref.check_attention(c, q.cpu(), out, news, lse=lse, window=window)
