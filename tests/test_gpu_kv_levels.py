"""Codebooks of any scale that the cache accepts: reading back and attention with levels far from those of unit rows."""
import numpy as np
import pytest

import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind", ("f16", "bf16"))
@pytest.mark.parametrize("single", (False, True))
@pytest.mark.parametrize("power", (-6, 7, 14))
def test_levels_of_any_scale_are_read_back(kind, single, power):
    """2^power times the levels of unit rows, of which the largest is 0.34; norms so that the rows are of ordinary length.  Each level is
    good to 2^-22 of the largest, as the rotation's entries are."""
    import paper_2605_17415_amd as pkg
    d, lens = 64, [1, 1, 1, 1] if single else [40, 7]
    c = ref.Cache(41, "code4", 2, d, 16, lens)
    c.levels = (c.levels * np.float32(2.0 ** power)).astype(np.float32)
    c.norms = (c.norms.astype(np.float64) * 2.0 ** -power).astype(np.float16)
    t, codec = c.device()
    k, v = (torch.full((sum(lens), 2, d), 7.0, dtype=ref.TYPES[kind], device=DEV) for _ in range(2))
    starts = None if single else torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=DEV)
    pkg.kv_read(t["pool"], t["table"], t["lengths"], k, v, starts=starts, **codec)
    torch.cuda.synchronize()
    for i, x in enumerate((k, v)):
        want = np.concatenate([np.stack([c.rows(i, b, h, n) for h in range(2)], 1) for b, n in enumerate(lens)])
        size = np.linalg.norm(want, axis=-1, keepdims=True)
        assert (np.abs(x.double().cpu().numpy() - want) <= ref.HALF[x.dtype] * np.abs(want) + 2.0 ** -18 * size + 2.0 ** -25).all()


@pytest.mark.parametrize("new", (1, 70))
@pytest.mark.parametrize("power", (-6, 7, 14))
def test_attention_with_levels_of_any_scale(new, power):
    import paper_2605_17415_amd as pkg
    lens, news = [300, 90], [new, new]
    c = ref.Cache(42, "code4", 1, 64, 16, lens)
    c.levels = (c.levels * np.float32(2.0 ** power)).astype(np.float32)
    c.norms = (c.norms.astype(np.float64) * 2.0 ** -power).astype(np.float16)
    t, codec = c.device()
    q = (torch.randn(2 * new, 2, 64, generator=torch.Generator().manual_seed(1)) * 1.5).bfloat16().to(DEV)
    lse, starts = torch.full(q.shape[:2], 5.0, device=DEV), torch.tensor([0, new, 2 * new], dtype=torch.int32, device=DEV)
    out = pkg.kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, max_new=new, lse=lse, **codec)
    torch.cuda.synchronize()
    ref.check_attention(c, q.cpu(), out, news, lse=lse)
