"""The serving attention on scores, query rows and value norms far apart, against the
float64 references; tolerance as in test_gpu_serving.py, derived there for a score
of any size.
"""
import numpy as np
import pytest
import torch

from oracle import codec as occ
from test_gpu_serving import Cache, close, run_accum, weight_tol

pytestmark = pytest.mark.gpu


def along(c, which, norms):
    """All rows of a group's K (0) or V (1) become its first row's codewords, with these norms."""
    c.np[2 * which][:] = c.np[2 * which][:, :1]
    h = np.broadcast_to(np.asarray(norms, dtype=np.float64).astype(np.float16), (c.n, c.T))
    c.np[2 * which + 1] = occ.fp16_bits(h.copy())
    for i in (2 * which, 2 * which + 1):
        a = c.np[i].view(np.int16) if c.np[i].dtype == np.uint16 else c.np[i]
        c.dev[i] = torch.from_numpy(a.copy()).to(c.dev[i].device)


def towards(c, g, nats):
    """A query whose scores (scale 1) are `nats` times the key norms of group g."""
    u = c.decoded(g, 1, 0)[0] / occ.from_fp16_bits(c.np[1][g, 0])
    return nats * u / (u @ u)


@pytest.mark.parametrize("nats", [-150.0, -1000.0, 150.0])
@pytest.mark.parametrize("G", [1, 3, 5, 12])
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 1, 16), (128, 4, 256)], ids=str)
def test_accum_scores_far_below_zero(device, d, k, N, G, nats):
    """The last head's scores are all near -150 or -1000 nats: softmax goes by differences."""
    rng = np.random.default_rng(41)
    lens = [1, 40]
    c = Cache(d, k, N, 2, 45, device)
    along(c, 0, 1 + rng.random(45) / 64)
    q = rng.standard_normal((2, G, d))
    for g in range(2):
        q[g, -1] = towards(c, g, nats)
    q = torch.from_numpy(q.astype(np.float32)).to(device)
    before = torch.rand(2, 45, device=device)
    acc = before.clone()
    out = run_accum(c, q, lens, acc, scale=1.0)
    assert bool(acc.isfinite().all())
    qn, out, b, a = (x.double().cpu().numpy() for x in (q, out, before, acc))
    for g, t in enumerate(lens):
        K, V = c.decoded(g, t, 0), c.decoded(g, t, 1)
        w = close(out[g], qn[g], K, V, np.ones((G, t), dtype=bool), 1.0)
        add = w.sum(0)
        # as check_accum, at this scale
        tol = (add * (2 * weight_tol(qn[g], K, 1.0) + 2.0**-24 * G) + 2.0**-24 * np.abs(a[g, :t]))
        assert np.all(np.abs(a[g, :t] - b[g, :t] - add) <= tol)
        assert np.array_equal(a[g, t:], b[g, t:])
