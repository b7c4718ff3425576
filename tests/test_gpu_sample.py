"""Sampling against its definition: equal tokens, whatever the type, the sizes, the ties and the settings."""
import math

import numpy as np
import pytest

import sample_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def logits(seed, rows, v, kind):
    g = torch.Generator().manual_seed(seed)
    x = 2.2 * torch.randn(rows, v, generator=g)
    x.scatter_add_(1, torch.randint(0, v, (rows, min(v, 40)), generator=g), 3 + 9 * torch.rand(rows, min(v, 40), generator=g) ** 2)
    return x.to(TYPES[kind])


def per_row(v, rows, dtype):
    return torch.as_tensor(np.broadcast_to(np.asarray(v, dtype), (rows,)).copy(), device=DEV)


def check(x, u, out=None, **how):
    """Tokens and logarithms of every row; settings are numbers or lists."""
    rows = x.shape[0]
    u = torch.as_tensor(u, dtype=torch.float32)
    given = {k: per_row(v, rows, np.int32 if k == "top_k" else np.float32) if isinstance(v, (list, np.ndarray)) else v for k, v in how.items()}
    logs = torch.full((rows,), 7.0, device=DEV)
    got = _pkg().sample_tokens(x if x.is_cuda else x.to(DEV), u.to(DEV), out=out, logprobs=logs, **given).cpu().numpy()
    logs, wide = logs.double().cpu().numpy(), x.double().cpu().numpy()
    for r in range(rows):
        one = {k: (v[r] if isinstance(v, (list, np.ndarray)) else v) for k, v in how.items()}
        one = {k: (int(v) if k == "top_k" else np.float32(v)) for k, v in one.items()}
        token, log = ref.sample(wide[r], u[r].item(), **one)
        assert got[r] == token, (r, one, got[r], token)
        # the logarithm is rounded to float32 once
        assert logs[r] == log or abs(logs[r] - log) <= 2.0 ** -23 * abs(log) + 1e-9, (r, one)
    return got


WAYS = [dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=40), dict(top_p=0.9), dict(temperature=0.8, top_k=50, top_p=0.9), dict(min_p=0.05),
        dict(temperature=1.5, top_k=1000, top_p=0.99, min_p=0.001), dict(top_k=1), dict(top_p=0.0), dict(min_p=1.0), dict(temperature=30.0, top_p=0.5)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (1, 2, 63, 1000, 1024, 1025, 5000, 32_001, 32_768, 32_769))
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_settings(kind, v, way):
    rows = 6
    u = np.random.default_rng(v + way).random(rows, np.float32)
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    check(logits(v + way, rows, v, kind), u, **WAYS[way])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,v", [(3, 151_000), (40, 20_003), (1, 1 << 20)])
def test_every_row_its_own_settings(kind, rows, v):
    r = np.random.default_rng(v)
    check(logits(v, rows, v, kind), r.random(rows, np.float32), temperature=r.choice([0.0, 0.5, 1.0, 1.3], rows), top_k=r.choice([0, 1, 7, 300, 5000], rows),
          top_p=r.choice([0.1, 0.8, 0.95, 0.9999, 1.0], rows), min_p=r.choice([0.0, 0.0, 0.01, 0.3], rows))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (4, 1000, 70_000))
def test_ties(kind, v):
    """All alike, and few values: ranks go to the lowest index, also where the mass reaches top_p exactly."""
    u = np.linspace(0, 0.999, 8).astype(np.float32)
    same = torch.full((8, v), -3.25, dtype=TYPES[kind])
    few = torch.randint(0, 3, (8, v), generator=torch.Generator().manual_seed(v)).to(TYPES[kind])
    for x in (same, few):
        for how in (dict(), dict(top_k=3), dict(top_k=v // 2), dict(top_p=0.5), dict(top_p=0.25, top_k=v // 2), dict(min_p=0.5), dict(temperature=0.0), dict(top_p=0.999)):
            check(x, u, **how)


@pytest.mark.parametrize("kind", TYPES)
def test_no_numbers(kind):
    """Masked tokens, no numbers, infinite ones, rows of nothing."""
    x = logits(3, 9, 3000, kind)
    g = torch.Generator().manual_seed(3)
    x[0] = -torch.inf
    x[1] = torch.nan
    x[2, torch.rand(3000, generator=g) < 0.9] = -torch.inf
    x[3, torch.rand(3000, generator=g) < 0.5] = torch.nan
    x[4, 77], x[4, 2011] = torch.inf, torch.inf
    x[5] = -torch.inf
    x[5, 1234] = torch.finfo(x.dtype).min
    x[6] = torch.finfo(x.dtype).min
    x[7, 5] = torch.finfo(x.dtype).max
    x[8] = torch.where(torch.arange(3000) % 2 == 0, 0.0, -0.0)
    u = np.linspace(0.02, 0.98, 9).astype(np.float32)
    for how in (dict(), dict(temperature=0.0), dict(top_k=20), dict(top_k=2500), dict(top_p=0.9), dict(top_k=700, top_p=0.7, min_p=0.1), dict(temperature=1e-30),
                dict(temperature=1e30), dict(temperature=float("inf"))):
        if how.get("temperature") != float("inf"):
            check(x, u, **how)
        else:
            check(x, u, temperature=[float("inf")] * 9)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (3000, 70_000))
def test_temperatures_that_leave_all_weights_alike(kind, v):
    x = logits(v, 4, v, kind)
    x[1, torch.rand(v, generator=torch.Generator().manual_seed(9)) < 0.7] = -torch.inf
    x[2, 3], x[3, 5] = torch.nan, torch.inf
    for temperature in (float("inf"), 1e38, 1e30):
        for how in (dict(), dict(min_p=0.5), dict(min_p=1.0), dict(min_p=1.0, top_k=2000), dict(min_p=1.0, top_p=0.5)):
            check(x, [0.2, 0.99, 0.6, 0.4], temperature=temperature, **how)


def test_settings_out_of_range_in_arrays():
    """They count as the end of the range that they lie behind, no number as no restriction, a temperature that is none as zero."""
    x = logits(4, 6, 4000, "f32")
    u = [0.1, 0.3, 0.5, 0.7, 0.9, 0.99]
    nan = float("nan")
    got = {}
    for name, odd, plain in (("temperature", [-1.0, nan, 0.0, -nan, -1e30, -0.0], [0.0] * 6), ("top_k", [-5, 0, 4000, 1 << 30, -(1 << 31), 9999], [0] * 6),
                             ("top_p", [1.5, nan, 1.0, float("inf"), 2.0, 1.0], [1.0] * 6), ("top_p", [-0.5, 0.0, -1e30, -0.0, -float("inf"), -1.0], [0.0] * 6),
                             ("min_p", [nan, -0.3, 0.0, -1.0, -float("inf"), -0.0], [0.0] * 6), ("min_p", [1.5, 1.0, 2.0, float("inf"), 1e30, 1.0], [1.0] * 6)):
        kind = np.int32 if name == "top_k" else np.float32
        a, b = (_pkg().sample_tokens(x.to(DEV), torch.tensor(u, device=DEV), **{name: per_row(v, 6, kind)}).tolist() for v in (odd, plain))
        assert a == b, name
        got[name] = b
    odd_u = torch.tensor([-1.0, nan, 0.0, 1.0, 7.0, float("inf")], device=DEV)
    near = torch.tensor([0.0, 0.0, 0.0, 1.0, 1.0, 1.0], device=DEV)
    assert torch.equal(_pkg().sample_tokens(x.to(DEV), odd_u), _pkg().sample_tokens(x.to(DEV), near))
    check(x, near.cpu())


@pytest.mark.parametrize("kind", TYPES)
def test_strides(kind):
    """Rows inside wider ones that begin at odd places; results in given places."""
    wide = logits(5, 7, 9000, kind).to(DEV)
    for begin, v in ((1, 4001), (3, 8191), (2, 64)):
        out = torch.full((7,), -9, dtype=torch.int32, device=DEV)
        check(wide[:, begin: begin + v], np.linspace(0, 0.99, 7), out=out, top_p=0.95, top_k=90)
        assert (out >= 0).all()
    assert _pkg().sample_tokens(wide[:0], torch.zeros(0, device=DEV)).shape == (0,)
    one = wide[2:3, 5:2000]
    check(one, [0.4])


def test_shares_are_those_of_the_weights():
    """Over many equally spaced u a token comes up as often as its probability says."""
    x = torch.tensor([[1.0, 0.0, -torch.inf, 2.0, 0.5]])
    n = 4096
    u = (torch.arange(n) + 0.5) / n
    got = _pkg().sample_tokens(x.expand(n, 5).contiguous().to(DEV), u.to(DEV), temperature=0.8).cpu().numpy()
    p = ref.weights(x[0].double().numpy(), 0.8)
    share = np.bincount(got, minlength=5) / n
    assert np.abs(share - p / p.sum()).max() <= 1 / n and (np.diff(got) >= 0).all()


def test_equal_calls_give_equal_tokens():
    x, u = logits(8, 64, 50_000, "bf16").to(DEV), torch.rand(64, device=DEV)
    a, b = (torch.empty(64, device=DEV) for _ in range(2))
    s = _pkg().sample_tokens(x, u, top_p=0.97, logprobs=a)
    t = _pkg().sample_tokens(x, u, top_p=0.97, logprobs=b)
    assert torch.equal(s, t) and torch.equal(a, b) and math.isfinite(float(a.sum()))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (4096, 4097, 9000, 70_001))
def test_long_lists(kind, v):
    """Logits so close together that thousands fall between two ranks that have to be told apart, ranks at the ends of lists, masked tokens."""
    g = torch.Generator().manual_seed(v)
    x = torch.stack([torch.rand(v, generator=g) * 1e-2, 5 + torch.rand(v, generator=g), torch.where(torch.rand(v, generator=g) < 0.01, torch.randn(v, generator=g), -torch.inf),
                     torch.randn(v, generator=g) * 100, torch.cat([torch.full((1,), 30.0), torch.randn(v - 1, generator=g)]), torch.arange(v) * 1e-3]).to(TYPES[kind])
    u = np.linspace(0.01, 0.99, 6).astype(np.float32)
    for how in (dict(top_k=255), dict(top_k=256), dict(top_k=257), dict(top_k=3000), dict(top_k=v - 1), dict(top_p=0.3), dict(top_p=0.99), dict(top_k=2000, top_p=0.6),
                dict(top_k=300, top_p=0.999, min_p=0.2), dict(temperature=100.0, top_p=0.5), dict(temperature=0.01, top_p=0.9, top_k=500), dict(min_p=0.9),
                dict(temperature=1e6, top_k=1000), dict(temperature=1e-6, top_k=v // 2, top_p=0.5)):
        check(x, u, **how)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (64, 65, 3000, 20_000, 100_000))
def test_lists_of_a_wavefront(kind, v):
    """As many ranks as one wavefront has lanes, one less and one more; equal logits at the last one; fewer tokens than ranks."""
    x = logits(v, 5, v, kind)
    x[1] = torch.randn(v, generator=torch.Generator().manual_seed(v)).to(x.dtype).round(decimals=1)
    x[2] = (torch.arange(v, 0, -1) * 0.125).to(x.dtype)
    x[3, torch.arange(v) % 997 != 5] = -torch.inf
    x[4, ::2] = x[4, 1]
    u = np.float32([0.0, 0.3, 0.999, 0.6, 1 - 2.0 ** -24])
    for k in (2, 3, 62, 63, 64, 65, 66):
        for how in (dict(), dict(top_p=0.9), dict(top_p=0.5, temperature=3.0), dict(min_p=0.3), dict(temperature=1e-3), dict(temperature=50.0, top_p=0.99, min_p=0.5)):
            check(x, u, top_k=k, **how)
            check(x, u, top_k=[k] * 5, **how)


def test_more_rows_than_share_a_workspace():
    rows, v = 1100, 66_000
    x = logits(12, rows, v, "bf16")
    r = np.random.default_rng(1)
    check(x, r.random(rows, np.float32), temperature=r.choice([0.0, 0.8, 1.0], rows), top_k=r.choice([0, 20, 600], rows), top_p=r.choice([0.9, 1.0], rows),
          min_p=r.choice([0.0, 0.02], rows))
    u = np.float32(0.4) * np.ones(rows, np.float32)
    check(x, u, top_k=30)
    check(x, u, top_p=0.8)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (9000, 140_000))
def test_large_logits_that_stand_together(kind, v):
    """A vocabulary in the order of its tokens' frequency: the first few groups hold the largest logits."""
    g = torch.Generator().manual_seed(v)
    x = torch.randn(4, v, generator=g) - 3 * torch.log1p(torch.arange(v) / 500.0)
    x[1] = -torch.arange(v) * 1e-3
    x[2, 3000:5000] += 30
    x = x.to(TYPES[kind])
    for how in (dict(top_k=50), dict(top_k=400, top_p=0.9), dict(top_k=1024), dict(top_k=1000, min_p=0.01), dict(top_k=1025), dict(top_p=0.9), dict(min_p=0.3), dict(min_p=1e-9)):
        check(x, np.linspace(0.05, 0.95, 4), **how)


@pytest.mark.parametrize("kind", TYPES)
def test_many_rows_of_middling_vocabularies(kind):
    """One workgroup a row, and several."""
    for rows, v in ((255, 40_000), (256, 40_000), (260, 65_536)):
        r = np.random.default_rng(rows)
        check(logits(v, rows, v, kind), r.random(rows, np.float32), temperature=r.choice([0.0, 0.7, 1.2], rows), top_k=r.choice([0, 30, 1500], rows),
              top_p=r.choice([0.5, 0.95, 1.0], rows), min_p=r.choice([0.0, 0.05], rows))
