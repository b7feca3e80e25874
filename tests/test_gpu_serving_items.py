"""Workgroups of the serving attention that go over several items, and over several
units of one, against the float64 references; tolerance as in test_gpu_serving.py.

A call has at most 512 workgroups (256 unless there are at most 8 query rows at
d = 64 and a table code), each with an equal number of runs of 256 tokens.
"""
import numpy as np
import pytest
import torch

from oracle import codec as occ
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


def along(c, device, key, value):
    """All keys of a group become its first one's codewords; key and value norms by token."""
    c.np[0][:] = c.np[0][:, :1]
    for i, h in ((1, key), (3, value)):
        c.np[i] = occ.fp16_bits(np.broadcast_to(h.astype(np.float16), (c.base, c.T)).copy())
    c.spread(device)


@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("M,G", [(1, 5), (3, 4), (6, 5), (8, 8)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 2, 64), (64, 1, 16), (128, 4, 256)], ids=str)
def test_references_that_move_from_unit_to_unit(device, d, k, N, M, G, falling):
    """Up to 16 units per wavefront, whose scores rise, stay or fall by up to 12 nats from one to
    the next while the value norms go from 1e-6 to 1e4 or back; one to four row tiles, items
    that end inside a workgroup's range and begin in it."""
    rng = np.random.default_rng(32)
    n, T = 256, 4096
    c = Repeated(d, k, N, 2, n, T, device)
    value = 10.0 ** np.linspace(-6, 4, T)
    value[[0, 700]] = 0
    along(c, device, np.linspace(0.5, 64, T), value[::-1] if falling else value)
    slopes = np.linspace(-3, 3, M * G)
    slopes[M * G // 2] = 0
    q = np.zeros((n, M * G, d))
    for g in range(n):
        u = c.rows[g % 2][0][0] / 0.5
        q[g] = rng.permutation(slopes)[:, None] * u / (u @ u)
    q = torch.from_numpy(q.reshape(n, M, G, d).astype(np.float32)).to(device)
    q64 = q.double().cpu().numpy()
    lens = rng.integers(0, T - M + 1, n)
    lens[:8] = [T - M, 0, 257, 256, 255, T - M, T - M - 31, 1]
    lens = lens.tolist()
    masks = random_masks(rng, M)
    groups = list(range(8)) + [100, 101, 255]
    c.check_tree(run_tree(c, q, lens, masks, scale=1.0), q64, lens, masks, groups, 1.0)
    if M == 3:  # (rows of one token; the accumulating form has up to 16)
        q, q64 = q.reshape(n, 12, d), q64.reshape(n, 12, d)
    elif M == 1:
        q, q64 = q[:, 0], q64[:, 0]
    else:
        return
    before = torch.rand(n, T, device=device)
    acc = before.clone()
    out = run_accum(c, q.contiguous(), lens, acc, scale=1.0)
    c.check_accum(out, q64, before, acc, lens, groups, 1.0)
