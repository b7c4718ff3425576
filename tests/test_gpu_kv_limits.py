"""Calls of more workgroups than one dimension of a grid counts threads for (2^24 of 256 threads)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def test_one_long_prompt_among_very_many_sequences():
    """The row tiles of the longest sequence are counted for every one: 1,026 of 16,384 sequences.  A window of one token shows a row
    its own token, so its result is that token's value."""
    batch, new, group, d, page = 1 << 14, 8208, 16, 64, 16
    news = torch.ones(batch, dtype=torch.int64)
    news[100] = new
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), news.cumsum(0)]).int().to(DEV)
    rows = int(news.sum())
    need = (news + page - 1) // page
    first = need.cumsum(0) - need
    table = torch.full((batch, new // page), -1, dtype=torch.int32)
    table[:, 0] = first.int()
    table[100] = torch.arange(new // page) + first[100]
    pool = torch.randn(int(need.sum()), 1, 2, page, d, device=DEV).bfloat16()
    q = torch.randn(rows, group, d, device=DEV).bfloat16()
    lse = torch.full((rows, group), 5.0, device=DEV)
    out = _pkg().kv_attend(q, pool, table.to(DEV), news.int().to(DEV), starts=starts, max_new=new, window=1, lse=lse)
    torch.cuda.synchronize()
    values = pool[:, 0, 1].reshape(-1, page // 8, d, 8).transpose(2, 3).reshape(-1, page, d)
    keys = pool[:, 0, 0]
    page_of, token_of = torch.empty(rows, dtype=torch.int64), torch.zeros(rows, dtype=torch.int64)
    at = starts.cpu().long()
    page_of[at[:-1]] = first
    inside = torch.arange(new)
    page_of[at[100]: at[101]], token_of[at[100]: at[101]] = first[100] + inside // page, inside % page
    assert torch.equal(out, values[page_of, token_of][:, None].expand_as(out))
    exact = (q.double() * keys[page_of, token_of][:, None].double()).sum(-1) / 8
    assert (lse.double() - exact).abs().max() <= 1e-4


@pytest.mark.parametrize("form", ("bf16", "code4"))
def test_more_pairs_of_sequence_and_head_than_one_dimension_holds(form):
    """130 heads of 2^17 sequences, nearly all of them empty: those give zeros, the others what they give in a call of their own."""
    pkg = _pkg()
    batch, heads, d, page = 1 << 17, 130, 64, 16
    live = torch.tensor([0, 77, batch // 2 + 1, batch - 1])
    codec = {}
    if form == "code4":
        pool = torch.randint(0, 256, (4, heads, page * (d + 4)), device=DEV, dtype=torch.uint8)
        pool[..., page * d:] = (torch.rand(4, heads, 2 * page, device=DEV) + 7).half().view(torch.uint8)
        codec = {"rotation": torch.from_numpy(pkg.ivftq_haar_rotation(d, 3)).to(DEV), "levels": pkg.ivftq_build_codebook(4, d)[0]}
    else:
        pool = torch.randn(4, heads, 2, page, d, device=DEV).bfloat16()
    table, lengths = torch.full((batch, 1), -1, dtype=torch.int32), torch.zeros(batch, dtype=torch.int32)
    table[live, 0], lengths[live] = torch.arange(4, dtype=torch.int32), torch.tensor([3, 16, 1, 9], dtype=torch.int32)
    q = torch.randn(1, heads, d, device=DEV).bfloat16().expand(batch, heads, d)
    out = torch.full((batch, heads, d), 7.0, dtype=torch.bfloat16, device=DEV)
    pkg.kv_attend(q, pool, table.to(DEV), lengths.to(DEV), out=out, **codec)
    few = pkg.kv_attend(q[:4].contiguous(), pool, table[live].to(DEV), lengths[live].to(DEV), **codec)
    torch.cuda.synchronize()
    assert torch.equal(out[live], few) and (few != 0).any()
    out[live] = 0
    assert not out.any()


def test_more_rows_to_free_than_one_dimension_holds():
    n = (1 << 24) + 5
    table, lengths, refs = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([[0], [1], [2]], [5, 6, 7], [1, 1, 1]))
    rows = torch.full((n,), 9, dtype=torch.int32, device=DEV)
    rows[0], rows[-1] = 2, 0
    _pkg().kv_free(table, lengths, refs, rows)
    torch.cuda.synchronize()
    assert table.tolist() == [[-1], [1], [-1]] and lengths.tolist() == [0, 6, 0] and refs.tolist() == [0, 1, 0]
