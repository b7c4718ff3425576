"""Sampling from long vocabularies whose masked or padded tokens have a finite value, as padded vocabularies and structured output have them: the
same tokens as the definition's, whichever way a row is worked on."""
import numpy as np
import pytest

from test_gpu_sample import TYPES, check, logits

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def masked(kind, v, seed):
    """Rows for each value that masks: a padded end of 267 tokens, all but 3,000 and all but 30 masked, all but every sixth."""
    x = TYPES[kind]
    values = [torch.finfo(x).min, -65504.0] + ([-1e9] if kind != "f16" else [])
    g = torch.Generator().manual_seed(seed)
    rows = []
    for value in values:
        allowed = [torch.arange(v) < v - 267, *(torch.zeros(v, dtype=torch.bool).index_fill_(0, torch.randperm(v, generator=g)[:n], True) for n in (3000, 30)),
                   torch.arange(v) % 6 == 0]
        rows += [torch.where(m, y.float(), value).to(x) for m, y in zip(allowed, logits(seed, len(allowed), v, kind))]
    return torch.stack(rows)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("v", (32_000, 128_000, 151_936))
def test_masked_by_finite_values(kind, v):
    x = masked(kind, v, v)
    u = np.linspace(0.03, 1 - 2.0 ** -24, x.shape[0]).astype(np.float32)
    for temperature in (0.1, 1.0):
        for how in (dict(top_k=50), dict(top_k=400), dict(top_k=1025), dict(top_k=50, top_p=0.9), dict(top_k=20_000, top_p=0.99), dict(top_p=0.9), dict(min_p=0.02), dict()):
            print(f"masked {kind} {v} {temperature} {how}", flush=True)
            check(x, u, temperature=temperature, **how)
