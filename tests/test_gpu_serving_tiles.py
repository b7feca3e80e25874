"""Attention of drafted tokens over caches of a large capacity, whose rows go in
tiles of 32 (d = 128) or 64 (d = 64), against the float64 references; tolerance as in
test_gpu_serving.py.  The caches are short ones laid out at a large T_stride, with
payload bytes of ones and NaN norms behind them.
"""
import types

import numpy as np
import pytest
import torch

import test_gpu_serving as base
from oracle import codec as occ
from oracle import serving as osv
from test_gpu_serving import Cache, check_tree, close, codebook, queries, random_masks

pytestmark = pytest.mark.gpu


def wide(c, rows=1 << 20):
    """The cache with T_stride = rows / n."""
    dev = []
    for x in c.dev:
        y = torch.full((c.n, rows // c.n) + tuple(x.shape[2:]), 255 if x.dtype == torch.uint8 else 0x7E00,
                       dtype=x.dtype, device=x.device)
        y[:, :c.T] = x
        dev.append(y)
    return types.SimpleNamespace(dev=dev, k=c.k, N=c.N, Rd=c.Rd, Cd=c.Cd)


def run_tree(c, q, lens, masks, **kw):
    return base.run_tree(wide(c), q, lens, masks, **kw)


@pytest.mark.parametrize("M,G", [(8, 8), (6, 5), (40, 8)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 2, 64), (64, 2, 16), (64, 8, 64), (64, 4, 4096),
                                   (64, 4, 512), (64, 8, 1024), (64, 1, 16), (64, 32, 64), (128, 4, 4096),
                                   (128, 4, 256), (128, 16, 64), (128, 8, 256), (128, 1, 16)], ids=str)
@pytest.mark.parametrize("exact", [True, False])
def test_tile_codes(device, d, k, N, M, G, exact):
    rng = np.random.default_rng(M + k)
    lens = [700, 0, 33, 251]
    c = Cache(d, k, N, 4, 760, device, C=codebook(d, k, N, exact=exact))
    q, q64 = queries(rng, (4, M, G, d), torch.bfloat16, device)
    masks = np.stack([random_masks(rng, M) for _ in lens])
    masks[1, 1] = 0  # (no context either: an empty row)
    out = run_tree(c, q, lens, masks)
    assert torch.count_nonzero(out[1, 1]) == 0
    check_tree(c, q, q64, out, lens, masks)


@pytest.mark.parametrize("d", [64, 128])
def test_tile_bad_lengths(device, d):
    rng = np.random.default_rng(3)
    M, G, lens = 9, 7, [-1, 100, 1 << 18, 2**31 - 1]
    c = Cache(d, 4, 256, 4, 160, device)
    q, q64 = queries(rng, (4, M, G, d), torch.float16, device)
    masks = random_masks(rng, M)
    out = run_tree(c, q, lens, masks)
    assert all(bool(out[g].isnan().all()) for g in (0, 2, 3))
    check_tree(c, q, q64, out, lens, masks, groups=[1])


@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 1, 16), (128, 4, 256)], ids=str)
def test_tile_norms_that_are_no_numbers(device, d, k, N):
    """Unseen ones change no bit; a seen one makes the rows that see it no numbers, and
    leaves the others."""
    rng = np.random.default_rng(4)
    M, G, lens = 8, 8, [61, 300]
    c = Cache(d, k, N, 2, 320, device)
    q, q64 = queries(rng, (2, M, G, d), torch.float32, device)
    masks = np.array([1 << i if i != 3 else 1 for i in range(M)], dtype=np.int64)  # 3 is never seen
    a = run_tree(c, q, lens, masks)
    check_tree(c, q, q64, a, lens, masks)
    for x, bits in ((1, 0x7E00), (3, 0x7E00), (3, 0x7C00)):
        c.dev[x][0, 61 + 3] = bits
        assert torch.equal(a, run_tree(c, q, lens, masks))
    for x, bits in ((3, 0x7C00), (3, 0x7E00), (1, 0x7E00)):
        keep = c.dev[x].clone()
        c.dev[x][1, 300 + 1] = bits
        b = run_tree(c, q, lens, masks)
        assert not bool(b[1, 1].isfinite().any()) and torch.equal(a[0], b[0])
        others = [i for i in range(M) if i != 1]
        close(b[1, others].double().cpu().numpy().reshape(-1, d), q64[1, others].reshape(-1, d),
              c.decoded(1, 300 + M, 0), c.decoded(1, 300 + M, 1),
              np.repeat(osv.seen_by_tree(300, masks, M)[others], G, 0))
        c.dev[x].copy_(keep)


@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 2, 64), (64, 1, 16), (128, 4, 256)], ids=str)
def test_tile_value_norms_that_grow(device, d, k, N):
    rng = np.random.default_rng(10)
    M, G = 10, 8
    c = Cache(d, k, N, 1, 700, device)
    h = np.float16(10.0 ** np.linspace(-6, 4, 700))
    h[350] = 0
    c.np[3][0] = occ.fp16_bits(h)
    c.dev[3].copy_(torch.from_numpy(c.np[3].view(np.int16)))
    q, q64 = queries(rng, (1, M, G, d), torch.float32, device)
    masks = random_masks(rng, M)
    for length in (690, 300, 40):
        check_tree(c, q, q64, run_tree(c, q, [length], masks), [length], masks)


@pytest.mark.parametrize("d,k,N", [(64, 8, 16), (128, 4, 256)], ids=str)
def test_tiles_agree_on_long_groups(device, d, k, N):
    """The capacity chooses the tile: large and small ones stand against the reference."""
    rng = np.random.default_rng(12)
    M, G, lens = 64, 2, [5000, 2049, 255]
    c = Cache(d, k, N, 3, 5100, device)
    q, q64 = queries(rng, (3, M, G, d), torch.bfloat16, device)
    masks = random_masks(rng, M)
    check_tree(c, q, q64, run_tree(c, q, lens, masks), lens, masks)
    check_tree(c, q, q64, base.run_tree(c, q, lens, masks), lens, masks)


@pytest.mark.parametrize("M,G", [(2, 3), (3, 5)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_many_records_of_one_group(device, d, M, G):
    """A group of which up to 157 workgroups hold a part each, in the outputs and the weights."""
    rng = np.random.default_rng(13)
    lens = [40000]
    c = Cache(d, 4, 256, 1, 40100, device)
    w = wide(c, 1 << 21)
    q, q64 = queries(rng, (1, M, G, d), torch.float32, device)
    q, q64 = 4 * q, 4 * q64  # (weights far from equal)
    masks = random_masks(rng, M)
    check_tree(c, q, q64, base.run_tree(w, q, lens, masks), lens, masks)
    before = torch.rand(1, 1 << 21, device=device)
    acc = before.clone()
    out = base.run_accum(w, q[:, 0].contiguous(), lens, acc)
    assert torch.equal(acc[:, 40000:], before[:, 40000:])
    base.check_accum(c, q64[:, 0], out, before[:, :c.T], acc[:, :c.T], lens)
