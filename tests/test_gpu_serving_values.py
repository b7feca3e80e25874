"""The serving attention on scores, query rows and value norms far apart, against the
float64 references; tolerance as in test_gpu_serving.py, derived there for a score
of any size.
"""
import numpy as np
import pytest
import torch

from oracle import codec as occ
from oracle import serving as osv
from test_gpu_serving import Cache, close, queries, run_accum, run_tree, weight_tol
from test_gpu_serving_tiles import wide

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


@pytest.mark.parametrize("big", [1e4, 1e7, 1e10, 1e30])
@pytest.mark.parametrize("M,G,large", [(2, 2, False), (3, 4, False), (6, 5, True), (8, 8, True)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 16), (128, 4, 256)], ids=str)
def test_finite_query_rows_are_independent(device, d, k, N, M, G, large, big):
    """One drafted token with queries of any size leaves the others' rows alone, in every row tile."""
    rng = np.random.default_rng(42)
    lens = [150, 9]
    c = Cache(d, k, N, 2, 170, device)
    q, q64 = queries(rng, (2, M, G, d), torch.float32, device)
    masks = np.array([1 << i for i in range(M)], dtype=np.int64)
    q[:, 1] *= big
    q[1, 0] *= 1e-9 / big  # (a mean over the seen tokens)
    q64 = q.double().cpu().numpy()
    out = run_tree(wide(c, 1 << 18) if large else c, q, lens, masks).double().cpu().numpy()
    others = [i for i in range(M) if i != 1]
    for g, L in enumerate(lens):
        close(out[g, others].reshape(-1, d), q64[g, others].reshape(-1, d), c.decoded(g, L + M, 0),
              c.decoded(g, L + M, 1), np.repeat(osv.seen_by_tree(L, masks, M)[others], G, 0))


def test_finite_query_heads_are_independent(device):
    """The same for the heads of a group: those before and behind a huge one."""
    rng = np.random.default_rng(43)
    for G in (5, 8, 12):
        c = Cache(64, 4, 256, 1, 170, device)
        q, _ = queries(rng, (1, G, 64), torch.float32, device)
        q[0, 2] *= 1e12
        acc = torch.zeros(1, 170, device=device)
        out = run_accum(c, q, [165], acc).double().cpu().numpy()
        rows = [i for i in range(G) if i != 2]
        close(out[0, rows], q.double().cpu().numpy()[0, rows], c.decoded(0, 165, 0), c.decoded(0, 165, 1),
              np.ones((G - 1, 165), dtype=bool))
