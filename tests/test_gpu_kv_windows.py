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


@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("window,sinks", [(5999, 0), (3000, 0), (2000, 70)])
def test_row_tiles_in_shares_with_a_window_agree_with_few_rows(form, kind, window, sinks):
    """128 heads leave four workgroups a head, whose shares are then of more than 64 tiles and cut row tiles: every sequence's last rows
    against the kernel of few rows.  Roundings of at most `step` of each weight, independent in the two kernels, move a result of about
    |w|_2 |v| by sqrt(2) step of it in the mean square: five times step; the result's own rounding twice."""
    import paper_2605_17415_amd as pkg
    heads, group, d, page, lens, news, last = 128, 2, 64, 64, [6000, 4100], [200, 130], 3
    need = [-(-n // page) for n in lens]
    g = torch.Generator(device=DEV).manual_seed(window)
    table = torch.full((2, max(need)), -1, dtype=torch.int32, device=DEV)
    order = torch.randperm(sum(need), generator=g, device=DEV).int()
    table[0], table[1, :need[1]] = order[:need[0]], order[need[0]:]
    codec = {}
    if form == "code4":
        pool = torch.randint(0, 256, (sum(need), heads, page * (d + 4)), generator=g, device=DEV, dtype=torch.uint8)
        norms = ((torch.rand(sum(need), heads, 2 * page, generator=g, device=DEV) + 0.5) * math.sqrt(d)).half()
        norms[table[:, 0].long(), :, 0] *= 4
        pool[..., page * d:] = norms.view(torch.uint8)
        codec = {"rotation": torch.from_numpy(pkg.ivftq_haar_rotation(d, 3)).to(DEV), "levels": pkg.ivftq_build_codebook(4, d)[0]}
    else:
        pool = torch.randn(sum(need), heads, 2, page, d, generator=g, device=DEV).to(ref.TYPES[form])
        pool[table[:, 0].long(), :, 0, 0] *= 4
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = (torch.randn(sum(news), heads * group, d, generator=g, device=DEV) * 1.5).to(ref.TYPES[kind])
    rows = torch.cat([torch.arange(e - last, e) for e in np.cumsum(news)]).to(DEV)
    starts, few_starts = (torch.tensor([0] + list(np.cumsum(x)), dtype=torch.int32, device=DEV) for x in (news, [last] * 2))
    logs, few_logs = torch.empty(q.shape[:2], device=DEV), torch.empty(2 * last, heads * group, device=DEV)
    few = pkg.kv_attend(q[rows], pool, table, lengths, starts=few_starts, max_new=last, window=window, sinks=sinks, lse=few_logs, **codec)
    many = pkg.kv_attend(q, pool, table, lengths, starts=starts, max_new=max(news), window=window, sinks=sinks, lse=logs, **codec)
    torch.cuda.synchronize()
    far, size = (many[rows].double() - few.double()).norm(dim=-1), few.double().norm(dim=-1)
    step = 2.0 ** -11 if form == "code4" else ref.HALF[few.dtype]
    assert (far <= (2 * ref.HALF[few.dtype] + 5 * step) * size + 2.0 ** -18 * math.sqrt(d)).all(), float((far / size).max())
    assert (logs[rows] - few_logs).abs().max() <= 1e-4
