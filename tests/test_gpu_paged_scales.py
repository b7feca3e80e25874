"""The 8-bit write into pages whose scales a caller has set."""
import numpy as np
import pytest
import torch

from test_gpu_paged import CODES, TYPES, pools, run_write

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [1, 9, 600])
@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -127, 2.0 ** -128, 1.5 * 2.0 ** -129, 2.0 ** -149, 1e-39, np.inf])
def test_zeros_into_pages_of_any_scale(device, kind, dtype, rows, scale):
    """Rows of zeros (of both signs) behind rows whose scale is below what a quotient's
    reciprocal holds, or infinite: codes of 0."""
    rng = np.random.default_rng(rows)
    H, page, d, n_pages = 2, 16, 64, 64
    kp, ks = pools(device, rng, n_pages, H, page, d, kind)
    vp, vs = pools(device, rng, n_pages, H, page, d, kind)
    ks[:], vs[:] = scale, scale
    slots = [p * page + 3 + i for p in rng.permutation(n_pages) for i in range(page - 3)][:rows]
    x = torch.zeros(rows, 2, H, d, device=device)
    x[..., ::3] = -0.0
    x[rows // 2, 0, 0] = 1.0  # (one that grows its page's scale)
    x = x.to(TYPES[dtype])
    run_write(device, x[:, 0], x[:, 1], slots, kind, kp, ks, vp, vs)
