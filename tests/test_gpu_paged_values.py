"""Attention over the paged 8-bit cache on pages, weights and scores far apart; tolerance
as in test_gpu_paged.py, derived there.
"""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from oracle import paged as opg
from test_gpu_paged import CODES, TYPES, check_attention, host, make_cache, on

pytestmark = pytest.mark.gpu


def attend(device, q, cache, lens, rows, kind, causal=True, scale=0.0):
    """Attention of q (rows of every sequence) over `cache`; rows None: one each, no starts."""
    kp, ks, vp, vs, table = cache
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    starts = np.concatenate([[0], np.cumsum([1] * len(lens) if rows is None else rows)]).astype(np.int32)
    out = fq.attn_cache8(q, on(device, kp, kind), t(ks), on(device, vp, kind), t(vs), t(table),
                         t(np.asarray(lens, np.int32)), None if rows is None else t(starts), causal=causal,
                         scale=scale)
    return host(out), starts


# lens, rows (None: one each), H, G, page, d: whole and cut items, one row and row tiles
FORMS = [([300, 512, 33], None, 2, 8, 16, 64), ([129, 600], [40, 70], 1, 4, 16, 64),
         ([700, 90], [33, 50], 1, 2, 32, 128), ([200], None, 1, 3, 64, 256), ([9000], None, 1, 4, 64, 128),
         ([2600, 40], [30, 40], 1, 4, 16, 64), ([5000, 700], None, 2, 8, 16, 64)]


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("lens,rows,H,G,page,d", FORMS, ids=str)
@pytest.mark.parametrize("exponent", [0, -12, -20, -100])
def test_pages_of_zeros_first(device, kind, lens, rows, H, G, page, d, exponent):
    """Pages of zeros, whose scale is 0, before and between pages of small values."""
    rng = np.random.default_rng(d - exponent)
    cache = kp, ks, vp, vs, table = make_cache(rng, lens, H, page, d, kind)
    for g, t in enumerate(lens):
        for j in range(-(-t // page)):
            vs[table[g, j]] *= np.float32(2.0 ** exponent)
            if (j + 1) * page < t and (j * page < 64 or rng.random() < 0.6):
                vp[table[g, j]], vs[table[g, j]] = 0, 0
    q = torch.randn(len(lens) if rows is None else sum(rows), H * G, d, device=device) * 0.1
    out, starts = attend(device, q, cache, lens, rows, kind)
    check_attention(out, host(q), *cache, lens, starts, True, kind)


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("lens,rows,H,G,page,d", FORMS + [([20, 2, 32, 33], None, 1, 2, 16, 64)], ids=str)
@pytest.mark.parametrize("bits", [10, 20, 40, 100])
def test_token_of_much_weight_and_no_value(device, kind, lens, rows, H, G, page, d, bits):
    """The first token's score is `bits` bits above all others and its values are 0: the
    others keep their bits."""
    rng = np.random.default_rng(d + bits)
    cache = kp, ks, vp, vs, table = make_cache(rng, lens, H, page, d, kind)
    big = opg.to_codes(np.array([96.0]), kind)[0]
    for g in range(len(lens)):
        first = table[g, 0]
        kp[first, :, 0], vp[first, :, 0] = 0, 0
        kp[first, :, 0, 0] = big
        for j in range(-(-lens[g] // page)):
            ks[table[g, j]] = 1.0
            kp[table[g, j], :, (1 if j == 0 else 0):, 0] = 0
    q = torch.randn(len(lens) if rows is None else sum(rows), H * G, d, device=device) * 1e-5
    q[:, :, 0] = bits * float(np.log(2)) / 96
    out, starts = attend(device, q, cache, lens, rows, kind, scale=1.0)
    check_attention(out, host(q), *cache, lens, starts, True, kind, 1.0)


@pytest.mark.parametrize("rows", [None, [40]])
def test_values_of_the_least_weight(device, rows):
    """Values so large, with a weight so small, that they count for as much as the others."""
    rng = np.random.default_rng(3)
    cache = kp, ks, vp, vs, table = make_cache(rng, [128], 1, 16, 64, "int8")
    kp[:], ks[:] = 0, 1.0
    kp[table[0, :8], 0, :, 0] = np.array([100, 0, 50, 0, 100, 50, 100, 100], np.uint8)[:, None]
    for bits in (60, 90, 110, 118):
        # weights 1, 2^-bits, 2^-bits/2; values 2^-60 on the heavy ones
        vs[table[0, :8], 0] = np.exp2([-60.0, bits - 60, bits / 2 - 60, -60, -60, -90, -90, -60])
        q = torch.zeros(1 if rows is None else 40, 2, 64, device=device)
        q[..., 0] = bits * float(np.log(2)) / 100
        out, starts = attend(device, q, cache, [128], rows, "int8", causal=False, scale=1.0)
        check_attention(out, host(q), *cache, [128], starts, False, "int8", 1.0)


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("lens,rows,H,G,page,d", FORMS, ids=str)
@pytest.mark.parametrize("size", [1e4, 1e6, 1e8, 1e10, 1e20, 1e30, 2e37])
def test_scores_of_any_size(device, kind, lens, rows, H, G, page, d, size):
    """Rows stay within the values that they see; where one token's score is above all others
    by more than rounding and 40 nats, they are that token's."""
    rng = np.random.default_rng(d)
    cache = kp, ks, vp, vs, table = make_cache(rng, lens, H, page, d, kind)
    vp &= np.uint8(0x7f)  # (values from 0 up)
    q = torch.randn(len(lens) if rows is None else sum(rows), H * G, d, device=device) * size
    q.clamp_(-3e38, 3e38)
    out, starts = attend(device, q, cache, lens, rows, kind)
    assert np.isfinite(out).all()
    x, alone = host(q), 0
    for g, L in enumerate(lens):
        M = starts[g + 1] - starts[g]
        seen = np.tri(M, L, L - M, dtype=bool)
        for h in range(H):
            K, V = (opg.rows_of(a, b, table[g], L, h, kind) for a, b in ((kp, ks), (vp, vs)))
            for j in range(G):
                y, o = x[starts[g]:starts[g + 1], h * G + j], out[starts[g]:starts[g + 1], h * G + j]
                s = np.where(seen, y @ K.T / np.sqrt(d), -np.inf)
                off = (np.abs(y) @ np.abs(K).T).max(1) / np.sqrt(d) * ((d + 8) * 2.0 ** -24 + 2.0 ** -21)
                for i in range(M):
                    near = s[i] >= (s[i].max() - 2 * off[i] - 40 if size < 1e32 else -1e300)  # (factors are limited)
                    room = 2.0 ** -18 * V[seen[i]].max(0)
                    assert (o[i] >= V[near].min(0) - room).all() and (o[i] <= V[near].max(0) + room).all(), (g, h, j, i)
                    alone += near.sum() == 1
    assert alone > 0 or size < 1e6 or size > 1e32


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("rows", [40, 17])
@pytest.mark.parametrize("page,d", [(16, 64), (32, 128), (16, 256)])
@pytest.mark.parametrize("unknown", [-1, 10 ** 6])
def test_unknown_page_beside_no_numbers(device, kind, rows, page, d, unknown):
    """The pool's first page belongs to no sequence and holds codes that are no numbers: rows
    that do not see an unknown page do not see that one either."""
    rng = np.random.default_rng(5)
    L = 4 * page
    kp, ks, vp, vs, table = make_cache(rng, [L], 1, page, d, kind)
    first = lambda a, x: np.concatenate([np.full_like(a[:1], x), a])
    kp, vp, ks, vs = first(kp, 0x7f), first(vp, 0x7f), first(ks, 1), first(vs, 1)
    vp[0, :, ::2] = 0xff
    table += 1
    table[0, 3] = unknown
    n = min(rows, L)
    q = torch.randn(n, 2, d, device=device)
    out, starts = attend(device, q, (kp, ks, vp, vs, table), [L], [n], kind)
    blind = max(0, n - page)  # rows that see tokens before the unknown page only
    assert np.isnan(out[blind:]).all()
    check_attention(out[:blind], host(q)[:blind], kp, ks, vp, vs, table, [L - page], [0, blind], True, kind)
