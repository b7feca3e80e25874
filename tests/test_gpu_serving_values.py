"""The serving attention on scores, query rows and value norms far apart, against the
float64 references; tolerance as in test_gpu_serving.py, derived there for a score
of any size.
"""
import numpy as np
import pytest
import torch

from oracle import codec as occ
from oracle import serving as osv
from test_gpu_serving import Cache, check_tree, close, queries, run_accum, run_tree, weight_tol
from test_gpu_serving_items import Repeated
from test_gpu_serving_tiles import wide

pytestmark = pytest.mark.gpu


def along(c, which, norms):
    """All rows of a group's K (0) or V (1) become its first row's codewords, with these norms."""
    c.np[2 * which][:] = c.np[2 * which][:, :1]
    h = np.broadcast_to(np.asarray(norms, dtype=np.float64).astype(np.float16), c.np[1].shape)
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


@pytest.mark.parametrize("big", [1e5, 1e8, 1e10, 1e14, 1e30])
@pytest.mark.parametrize("M,G,large", [(2, 2, False), (3, 4, False), (6, 5, True), (8, 8, True)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 16), (128, 4, 256)], ids=str)
def test_scores_beyond_the_steps_of_float32(device, d, k, N, M, G, large, big):
    """Finite queries of any size have finite outputs, and weights that sum to 1, in caches of one
    unit per wavefront and of many, where such scores and ordinary ones meet."""
    rng = np.random.default_rng(47)
    n, T = 256, 2500
    c = Repeated(d, k, N, 2, n, T, device)
    lens = rng.integers(T // 2, T - M, n).tolist()
    q, _ = queries(rng, (n, M, G, d), torch.float32, device)
    q[:, 1] *= big
    q[1, 0, 0] *= big
    q64 = q.double().cpu().numpy()
    masks = np.array([1 << i for i in range(M)], dtype=np.int64)
    out = run_tree(c, q, lens, masks)
    assert bool(out.isfinite().all())
    c.check_tree(out, q64, lens, masks, [0, 1, 2, 255])
    if M * G <= 16:
        acc = torch.zeros(n, T, device=device)
        out = run_accum(c, q.reshape(n, M * G, d), lens, acc)
        assert bool(out.isfinite().all()) and bool((acc >= 0).all())
        # every weight to 2^-17 (exponentials, the sum's parts) of itself
        assert bool(((acc.double().sum(1) - M * G).abs() <= 2.0**-16 * M * G).all())
    one = Cache(d, k, N, 2, 170, device)
    out = run_tree(wide(one, 1 << 18) if large else one, q[:2], [150, 9], masks)
    assert bool(out.isfinite().all())


@pytest.mark.parametrize("outlier", [1e3, 3e4, 65504.0])
@pytest.mark.parametrize("M,G", [(2, 2), (3, 4), (6, 5), (8, 8)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 16), (128, 4, 256)], ids=str)
def test_large_value_norms_of_tokens_without_weight(device, d, k, N, M, G, outlier):
    """One token of a large value norm and next to no weight, one that takes most of the
    weight, and a long tail of small equal weights that point one way: the tail's sum stays."""
    rng = np.random.default_rng(44)
    n, T, L = 256, 6000, 5990
    c = Repeated(d, k, N, 1, n, T, device)  # (a workgroup goes over a whole group)
    key, value = np.full(T, 16.0), np.ones(T)
    key[3], value[3] = 0.0, outlier     # 25 nats below the largest score
    key[1030] = 32.0                    # in the same wavefront; the others 12.5 nats below it
    along(c, 0, key)
    along(c, 1, value)
    c.spread(device)
    q = np.broadcast_to(towards(c, 0, 12.5 / 16).astype(np.float32), (n, M, G, d)).copy()
    q *= (1 + rng.random((n, M, G, 1)) / 16).astype(np.float32)
    q = torch.from_numpy(q).to(device)
    masks = np.array([1 << i for i in range(M)], dtype=np.int64)
    out = run_tree(c, q, [L] * n, masks, scale=1.0)
    c.check_tree(out, q.double().cpu().numpy(), [L] * n, masks, [0, 100, 255], 1.0)


@pytest.mark.parametrize("M,G,large", [(2, 2, False), (3, 4, False), (6, 5, True), (8, 8, True)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 16), (128, 4, 256)], ids=str)
def test_large_value_norms_that_a_row_does_not_see(device, d, k, N, M, G, large):
    """A drafted token's value norm has no part in the rows that do not see it, however
    small their own tokens' are."""
    rng = np.random.default_rng(45)
    L = 20
    c = Cache(d, k, N, 1, 40, device)
    for small in (1.0, 1e-3, 3e-6):
        value = small * (1 + rng.random(40))
        value[L + 1] = 65504.0
        h = value.astype(np.float16)
        c.np[3][0] = occ.fp16_bits(h)
        c.dev[3].copy_(torch.from_numpy(c.np[3].view(np.int16)))
        q, q64 = queries(rng, (1, M, G, d), torch.float32, device)
        q, q64 = 3 * q, 3 * q64
        masks = np.array([1 << i for i in range(M)], dtype=np.int64)
        out = run_tree(wide(c, 1 << 18) if large else c, q, [L], masks)
        check_tree(c, q, q64, out, [L], masks)


@pytest.mark.parametrize("M,G,large", [(2, 2, False), (3, 4, False), (6, 5, True), (8, 8, True)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 1, 16), (128, 4, 256)], ids=str)
def test_zero_value_norms_of_the_largest_scores(device, d, k, N, M, G, large):
    """Tokens whose values are zero take most or next to all of the weight; the others' sum,
    up to 2^-70 of it, keeps its bits, and so do the accumulated weights."""
    rng = np.random.default_rng(46)
    T, L = 700, 690
    c = Cache(d, k, N, 1, T, device)
    for nats in (2.0, 20.0, 48.0):
        key, value = np.full(T, 16.0), 1 + rng.random(T)
        key[[5, 300, 301]], value[[5, 300, 301]] = 32.0, 0.0
        along(c, 0, key)
        c.np[3][0] = occ.fp16_bits(value.astype(np.float16))
        c.dev[3].copy_(torch.from_numpy(c.np[3].view(np.int16)))
        q = np.broadcast_to(towards(c, 0, nats / 16).astype(np.float32), (1, M, G, d)).copy()
        q = torch.from_numpy(q).to(device)
        masks = np.array([1 << i for i in range(M)], dtype=np.int64)
        out = run_tree(wide(c, 1 << 18) if large else c, q, [L], masks, scale=1.0)
        check_tree(c, q, q.double().cpu().numpy(), out, [L], masks, 1.0)
        acc = torch.zeros(1, T, device=device)
        run_accum(c, q[:, 0].contiguous(), [L], acc, scale=1.0)
        _, w = osv.attend(q[0, 0].double().cpu().numpy(), c.decoded(0, L, 0), c.decoded(0, L, 1),
                          np.ones((G, L), dtype=bool), 1.0)
        tol = 2 * weight_tol(q[0, 0].double().cpu().numpy(), c.decoded(0, L, 0), 1.0) + 2.0**-24 * (G + 1)
        assert np.all(np.abs(acc[0, :L].double().cpu().numpy() - w.sum(0)) <= tol * w.sum(0))
