"""Forms of the paged attention that sizes choose: row tiles of one wavefront, parts planned
by a launch of their own, cut items of every type and width.  Tolerance as in
test_gpu_paged.py, derived there."""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from test_gpu_paged import CODES, TYPES, check_attention, host, make_cache, on

pytestmark = pytest.mark.gpu


def run(device, q, cache, lens, starts, kind, causal=True):
    kp, ks, vp, vs, table = cache
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    out = torch.full(q.shape, 7.0, device=device)
    fq.attn_cache8(q, on(device, kp, kind), t(ks), on(device, vp, kind), t(vs), t(table),
                   t(np.asarray(lens, np.int32)), None if starts is None else t(np.asarray(starts, np.int32)),
                   causal=causal, out=out)
    return host(out)


def check_some(out, q, cache, lens, starts, kind, which, causal=True):
    """Sequences `which`, each against the oracle."""
    kp, ks, vp, vs, table = cache
    for g in which:
        b, e = int(starts[g]), int(starts[g + 1])
        check_attention(out[b:e], host(q[b:e]), kp, ks, vp, vs, table[g:g + 1], [int(lens[g])], [0, e - b], causal, kind)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("d,dtype,H,G,n", [(64, "bf16", 12, 4, 64), (64, "fp32", 12, 4, 64), (128, "fp16", 8, 4, 48),
                                           (256, "fp32", 6, 2, 60), (256, "bf16", 6, 2, 60)])
def test_row_tiles_of_one_wavefront(device, d, dtype, H, G, n, kind, causal):
    """More row tiles than fill the card, of items that are not cut, with a bad length, a
    query that is no number, an unknown page and a sequence of no token."""
    rng = np.random.default_rng(d + n)
    rows = rng.integers(20, 41, n)
    lens = rng.integers(41, 300, n).astype(np.int32)
    lens[3], lens[5] = 41, 300
    cache = make_cache(rng, lens, H, 16, d, kind)
    table = cache[4]
    assert table.shape[1] * 16 <= 1024
    starts = np.concatenate([[0], np.cumsum(rows)])
    q = torch.from_numpy(rng.standard_normal((int(starts[-1]) + 2, H * G, d))).to(TYPES[dtype]).to(device)
    # items enough for tiles of one wavefront (three of 32 rows a SIMD at d = 64, two at 128, one at 256)
    assert 2 * H * (len(q) // (32 // G)) >= 256 * 4 * {64: 3, 128: 2, 256: 1}[d]
    lens[7], lens[9] = -1, 0  # (9: fewer tokens than rows if causal, else nothing to see)
    q[starts[11] + 5, 1, 3] = float("nan")
    L = int(lens[13])
    table[13, (L - 1) // 16] = -5  # the last tokens' page
    out = run(device, q, cache, lens, starts, kind, causal)
    assert (out[starts[-1]:] == 7.0).all()
    check_some(out, q, cache, lens, starts, kind, [0, 3, 5, 12, 14, n // 2, n - 1], causal)
    assert np.isnan(out[starts[7]:starts[8]]).all()
    nothing = out[starts[9]:starts[10]]
    assert np.isnan(nothing).all() if causal else (nothing == 0).all()
    bad = np.zeros((int(rows[11]), H * G), bool)
    bad[5, 1] = True
    of11 = out[starts[11]:starts[12]]
    assert np.isnan(of11[bad]).all() and np.isfinite(of11[~bad]).all()
    sees = np.arange(L - rows[13] + 1, L + 1) > (L - 1) // 16 * 16 if causal else np.ones(rows[13], bool)
    of13 = out[starts[13]:starts[14]]
    assert np.isnan(of13[sees]).all() and np.isfinite(of13[~sees]).all()


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("d,dtype,page", [(64, "bf16", 16), (128, "fp16", 64), (256, "fp32", 32)])
@pytest.mark.parametrize("form", ["one", "few", "tiles"])
def test_planned_parts_of_cut_items(device, d, dtype, page, kind, form):
    """More sequences than a workgroup sums up itself, in tables so wide that items are cut,
    and a few sequences that are."""
    rng = np.random.default_rng(d)
    n, G = 600, 2 if form != "tiles" else 1
    rows = {"one": np.ones(n, int), "few": rng.integers(0, 4, n), "tiles": rng.integers(24, 28, n)}[form]
    lens = rng.integers(30, 50, n).astype(np.int32)
    long = [0, 37, n // 2, n - 1]
    lens[long] = [9000, 2049, 6400, 8500]
    rows[long[1:3]] = rows[long[1:3]] if form == "one" else 45
    lens[5] = -1
    cache = make_cache(rng, lens, 1, page, d, kind)
    table = np.full((n, 8192 // page + 200), -1, np.int32)
    table[:, :cache[4].shape[1]] = cache[4][:, :table.shape[1]]
    cache = (*cache[:4], table)
    starts = np.concatenate([[0], np.cumsum(rows)])
    q = torch.from_numpy(rng.standard_normal((int(starts[-1]), G, d))).to(TYPES[dtype]).to(device)
    out = run(device, q, cache, lens, None if form == "one" else starts, kind)
    check_some(out, q, cache, lens, starts, kind, long + [1, 5, 38, 100, 511, 512, 513, n - 2])


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d,G", [(64, 8), (128, 3), (256, 2), (256, 16)])
@pytest.mark.parametrize("rows", [None, 2, 30])
def test_cut_items(device, d, G, dtype, rows, kind):
    """Few long sequences, whose items are cut and joined: every type and width."""
    rng = np.random.default_rng(d + G)
    lens = np.array([4500, 300, 2600], np.int32)
    cache = make_cache(rng, lens, 1, 32, d, kind)
    m = [1, 1, 1] if rows is None else [rows, rows + 3, rows]
    starts = np.concatenate([[0], np.cumsum(m)])
    need = fq.attn_cache8_workspace_bytes(3, int(starts[-1]), 1, G, cache[4].shape[1], 32, d)
    assert need > 0  # (cut)
    q = torch.from_numpy(rng.standard_normal((int(starts[-1]), G, d))).to(TYPES[dtype]).to(device)
    out = run(device, q, cache, lens, None if rows is None else starts, kind)
    check_some(out, q, cache, lens, starts, kind, range(3))
