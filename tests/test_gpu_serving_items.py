"""Workgroups of the serving attention that go over several items, and over several
units of one, against the float64 references; tolerance as in test_gpu_serving.py.

A call has at most 512 workgroups (256 unless there are at most 8 query rows at
d = 64 and a table code), each with an equal number of runs of 256 tokens.
"""
import numpy as np
import pytest
import torch

from oracle import serving as osv
from test_gpu_serving import Cache, close, queries, random_masks, run_accum, run_tree, weight_tol

pytestmark = pytest.mark.gpu


class Repeated(Cache):
    """n groups that repeat `base` different ones, in turn."""

    def __init__(self, d, k, N, base, n, T, device, **kw):
        super().__init__(d, k, N, base, T, device, **kw)
        self.base, self.n = base, n
        self.spread(device)

    def spread(self, device):
        """The device's groups from the rows in `np`."""
        at = torch.arange(self.n, device=device) % self.base
        self.dev = [torch.from_numpy((a.view(np.int16) if a.dtype == np.uint16 else a).copy()).to(device)[at]
                    for a in self.np]
        self.rows = [[self.decoded(g, self.T, w) for w in (0, 1)] for g in range(self.base)]

    def check_tree(self, out, q64, lens, masks, groups, scale=None):
        M, G = q64.shape[1:3]
        out = out.double().cpu().numpy()
        for g in groups:
            t = lens[g] + M
            K, V = (x[:t] for x in self.rows[g % self.base])
            close(out[g].reshape(M * G, -1), q64[g].reshape(M * G, -1), K, V,
                  np.repeat(osv.seen_by_tree(lens[g], masks, M), G, 0), scale)

    def check_accum(self, out, q64, before, acc, lens, groups, scale=None):
        out, before, acc = (x.double().cpu().numpy() for x in (out, before, acc))
        for g in groups:
            t = lens[g]
            K, V = (x[:t] for x in self.rows[g % self.base])
            w = close(out[g], q64[g], K, V, np.ones((q64.shape[1], t), dtype=bool), scale)
            add = w.sum(0)
            assert np.array_equal(acc[g, t:], before[g, t:])
            tol = (add * (2 * weight_tol(q64[g], K, scale) + 2.0**-24 * q64.shape[1])
                   + 2.0**-24 * np.abs(acc[g, :t]))
            assert np.all(np.abs(acc[g, :t] - before[g, :t] - add) <= tol), g


@pytest.mark.parametrize("M,G", [(1, 5), (3, 4), (1, 12)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 1, 16), (64, 32, 64), (64, 2, 8), (128, 1, 4)], ids=str)
def test_staged_codes_with_several_items_per_workgroup(device, d, k, N, M, G):
    """1200 groups of up to two runs in 256 workgroups, in the outputs and the weights."""
    rng = np.random.default_rng(31)
    n, T = 1200, 320
    c = Repeated(d, k, N, 3, n, T, device)
    lens = rng.integers(0, T - M + 1, n).tolist()
    masks = random_masks(rng, M)
    q, q64 = queries(rng, (n, M, G, d), torch.float32, device)
    c.check_tree(run_tree(c, q, lens, masks), q64, lens, masks, range(n))
    before = torch.rand(n, T, device=device)
    acc = before.clone()
    out = run_accum(c, q[:, 0].contiguous(), lens, acc)
    c.check_accum(out, q64[:, 0], before, acc, lens, range(n))
