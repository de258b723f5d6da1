"""Selection of pages whose sums are not finite, or beyond the range of 32 bits."""
import numpy as np
import pytest
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import inputs
from gpu_util import DEV, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,Hkv,D,n_pages", [("f32", 4, 2, 64, 40), ("bf16", 4, 2, 64, 40), ("bf16", 10, 2, 128, 300), ("f32", 6, 1, 128, 300)])
@pytest.mark.parametrize("kind", ["infinite query", "nan query", "large", "large and absent"])
def test_selection_of_sums_that_no_float_holds(dtype, H, Hkv, D, n_pages, kind):
    rng = np.random.default_rng(61)
    sh = inputs.LayerShape(H * D, H, Hkv, D, 10000.0, dtype)
    dt = inputs.torch_dtype(dtype)
    normal = lambda size, std: inputs.round_to_dtype((rng.standard_normal(size) * std).astype(np.float32), dtype)
    large = kind.startswith("large")
    q = normal((1, 2, H, D), 1e19 if large else 1.0)
    a, b = normal((2, n_pages, Hkv, D), 1e19 if large else 1.0)
    bounds = np.stack([np.minimum(a, b), np.maximum(a, b)], axis=2)
    table = rng.permutation(n_pages)[None].astype(np.int32)
    if kind == "infinite query":
        q[0, 0, :, 3], q[0, 1, ::3, 0] = np.inf, -np.inf
    elif kind == "nan query":
        q[0, 0, 1, 5] = np.nan
    elif kind == "large":
        bounds[table[0, n_pages - 6]] = np.nan                  # (before all sums that are merely too large)
    elif kind == "large and absent":
        bounds[:, :, :, :D // 2], bounds[:, :, :, D // 2:] = -1.5e19, 1.5e19
        q[..., :D // 2], q[..., D // 2:] = 1e19, -1e19          # every sum far below the least float, but for
        bounds[table[0, 7]] = 0.0                               # one page, and pages that are not there
        table[0, 10:n_pages - 4] = -1
    page_keys = torch.zeros(n_pages, 16, Hkv, D, dtype=dt, device=DEV)
    bd = torch.from_numpy(bounds).to(device=DEV, dtype=dt)
    cache = qb.page_cache(page_keys, page_keys.clone(), bd, i32(table))
    for keep, first, last in ((3, 0, 0), (12, 1, 1), (min(n_pages - 1, 37), 0, 2)):
        pages = torch.full((1, 2, Hkv, keep), 99, dtype=torch.int32, device=DEV)
        print("scores", dtype, H, Hkv, D, n_pages, kind, keep, flush=True)
        qb.qcf_page_select(qb.make_desc(sh), cache, 1, 2, torch.from_numpy(q).to(device=DEV, dtype=dt), i32([[16 * n_pages - 3, 16 * n_pages]]),
                           keep, first, last, pages)
        torch.cuda.synchronize()
        for i in range(2):
            s = orc.page_scores(q[0, i].astype(np.float64), bounds.astype(np.float64), table[0])
            assert np.array_equal(pages[0, i].cpu().numpy(), orc.page_select(s, keep, first, last)), (i, keep)
