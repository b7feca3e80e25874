"""The paged 8-bit cache on the device against `oracle/paged.py`.

Tables, slots, positions, scales and codes are equal.  Rotary positions: sine and
cosine are off by at most 2^-23 (their argument, an eighth of a turn at most, and
their own rounding) and by the rounding of the angle in double; two products and a
sum add 2^-24 each, and the result is rounded by half a step of its type.
Attention: see `check_attention`.
"""
import math

import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from oracle import paged as opg
from oracle import serving as osv

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def host(t):
    return t.detach().cpu().double().numpy()


def raw(t):
    """The bytes of pages."""
    return t.view(torch.uint8).cpu().numpy()


# ------------------------------------------------------------------- rope --
def check_rope(y, x, positions, freqs, layout, scale=1.0, inverse=False):
    half = len(freqs)
    ref = opg.rope(host(x), positions, freqs, layout, scale, inverse)
    size = np.zeros(ref.shape)
    xa = np.abs(host(x))
    a, b = ((slice(0, half), slice(half, 2 * half)) if layout == "half"
            else (slice(0, 2 * half, 2), slice(1, 2 * half, 2)))
    size[..., a] = size[..., b] = xa[..., a] + xa[..., b]
    angle = np.abs(np.asarray(positions, dtype=np.float64))[:, None] * freqs * 2.0 ** -51
    off = np.zeros((len(positions), 1, ref.shape[2]))
    off[:, 0, a] = off[:, 0, b] = angle
    tol = abs(scale) * size * (2.0 ** -21 + off) + torch.finfo(x.dtype).eps / 2 * np.abs(ref)
    tol[..., 2 * half:] = 0
    err = np.abs(host(y) - ref)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,Hq,Hk,d,rot", [(1, 1, 1, 64, 64), (5, 8, 2, 64, 32), (33, 3, 0, 128, 128),
                                           (70, 12, 12, 128, 10), (3, 2, 1, 10, 6), (2, 1, 1, 2, 2),
                                           (2100, 2, 1, 64, 48), (9, 4, 2, 512, 512), (7, 5, 3, 66, 34),
                                           (1500, 9, 4, 30, 22), (40, 1, 1, 500, 10)])
def test_rope(device, layout, dtype, n, Hq, Hk, d, rot):
    g = torch.Generator(device=device).manual_seed(n + d)
    q = torch.randn(n, Hq, d, generator=g, device=device).to(TYPES[dtype])
    k = torch.randn(n, Hk, d, generator=g, device=device).to(TYPES[dtype]) if Hk else None
    pos = torch.randint(-5, 1 << 20, (n,), generator=g, device=device).int()
    freqs = fq.rope_freqs(rot)
    fd = torch.from_numpy(freqs).to(device)
    got = fq.rope(q, k, pos, fd, layout=layout)
    assert got[0].is_contiguous() and (got[1] is None) == (k is None)
    for x, y in zip((q, k), got):
        if x is not None:
            check_rope(y, x, pos.cpu().numpy(), freqs, layout)
    back = fq.rope(q, k, pos, fd, layout=layout, scale=0.5, inverse=True)
    check_rope(back[0], q, pos.cpu().numpy(), freqs, layout, 0.5, True)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_strides_and_in_place(device, layout):
    freqs = fq.rope_freqs(64)
    fd = torch.from_numpy(freqs).to(device)
    for off in (0, 1, 3):
        g = torch.Generator(device=device).manual_seed(off)
        buf = torch.randn(off + 37 * 9 * 64, generator=g, device=device).half()
        rows = buf[off:].view(37, 9, 64)
        q, k, v = rows[:, :5], rows[:, 5:7], rows[:, 7:].clone()
        pos = torch.arange(37, device=device, dtype=torch.int32) * 1000
        want = fq.rope(q.clone(), k.clone(), pos, fd, layout=layout)
        apart = fq.rope(q, k, pos, fd, layout=layout)
        other = torch.empty(5, 37, 64, dtype=torch.float16, device=device).transpose(0, 1)
        fq.rope(q, None, pos, fd, layout=layout, out=(other, None))
        pair = (q, k)
        assert fq.rope(q, k, pos, fd, layout=layout, out=pair)[0] is q
        for x, y, z in zip(want, apart, pair):
            assert torch.equal(x, y) and torch.equal(x, z)
        assert torch.equal(other, want[0]) and torch.equal(rows[:, 7:], v)


def test_rope_far_positions_and_no_rows(device):
    freqs = fq.rope_freqs(64, scaling="ramp", factor=8.0, trained=4096)
    fd = torch.from_numpy(freqs).to(device)
    pos = torch.tensor([0, 1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1], dtype=torch.int32, device=device)
    x = torch.randn(5, 2, 64, device=device)
    check_rope(fq.rope(x, None, pos, fd)[0], x, pos.cpu().numpy().astype(np.int64), freqs, "half")
    assert fq.rope(x[:0], x[:0], pos[:0], fd)[1].shape == (0, 2, 64)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_gradient(device, layout):
    """The inverse turns gradients: against the formula's, and against differences."""
    freqs = fq.rope_freqs(32)
    fd = torch.from_numpy(freqs).to(device)
    x, w = torch.randn(6, 3, 48, device=device), torch.randn(6, 3, 48, device=device)
    pos = torch.randint(0, 5000, (6,), device=device).int()
    p = pos.cpu().numpy()
    grad = fq.rope(w, None, pos, fd, layout=layout, scale=1.25, inverse=True)[0]
    check_rope(grad, w, p, freqs, layout, 1.25, True)
    f = lambda z: (opg.rope(z, p, freqs, layout, 1.25) * host(w)).sum()
    rng, x64 = np.random.default_rng(0), host(x)
    for _ in range(40):
        at = tuple(int(rng.integers(0, n)) for n in x.shape)
        step = np.zeros(x64.shape)
        step[at] = 1e-3  # (f is linear: differences are exact but for 64-bit rounding)
        slope = (f(x64 + step) - f(x64 - step)) / 2e-3
        want = slope if at[2] < 32 else host(w)[at]
        assert abs(host(grad)[at] - want) <= 2.0 ** -20 * 1.25 * 2 * np.abs(host(w)).max() + 1e-9


# ------------------------------------------------------------ page_resize --
def resize_case(rng, n, page, max_pages, top, spare, extra=0, bad=True):
    room = page * max_pages
    lens = rng.integers(0, room + 1, n)
    lens[rng.random(n) < 0.2] = 0
    grow = rng.integers(0, top + 1, n)
    shrink = rng.random(n) < 0.25
    grow[shrink] = -rng.integers(0, lens[shrink] + 1)
    grow = np.where(lens + grow > room, room - lens, grow) if not bad else grow
    if bad and n > 3:
        lens[1], grow[2] = -1, -room - 1
    used = sum(-(-int(t) // page) for t in lens if t > 0)
    n_pages = used + spare
    perm = rng.permutation(n_pages)
    table = np.full((n, max_pages), -1, np.int32)
    at = 0
    for g in range(n):
        m = max(0, -(-int(lens[g]) // page))
        table[g, :m] = perm[at:at + m]
        at += m
    free = np.full(n_pages + 3, -1, np.int32)
    free[:spare] = perm[at:at + spare]
    n_rows = int(grow[grow > 0].sum()) + extra
    return table, lens.astype(np.int32), grow.astype(np.int32), n_pages, free, spare, max(0, n_rows)


def run_resize(device, table, lens, grow, page, n_pages, free, n_free, n_rows, alias=False):
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    want = opg.resize(table, lens, grow, page, n_pages, free, n_free, n_rows)
    td, fd, ld, nd = t(table), t(free), t(lens), t(np.array([n_free], np.int32))
    out = None
    if alias:
        i32 = lambda m: torch.full((m,), 77, dtype=torch.int32, device=device)
        out = (ld, i32(len(lens) + 1), torch.full((n_rows,), 77, device=device), i32(n_rows), nd)
    got = fq.page_resize(td, ld, t(grow), page, n_pages, fd, nd, n_rows, out=out)
    new_lens, starts, slots, positions, left = (x.cpu().numpy() for x in got)
    assert np.array_equal(td.cpu().numpy(), want[0])
    assert np.array_equal(fd.cpu().numpy(), want[1])
    for x, y in zip((new_lens, starts, slots, positions), want[2:6]):
        assert np.array_equal(x, y)
    assert left[0] == want[6]
    return want


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n,page,max_pages,top,spare,extra", [
    (1, 16, 4, 20, 3, 0), (7, 16, 9, 40, 6, 0), (40, 32, 6, 90, 60, 5), (40, 32, 6, 90, 20, 0),
    (300, 16, 8, 3, 40, 0), (3000, 16, 4, 2, 900, 0), (60, 128, 20, 900, 200, 77),
    (2, 1, 300, 200, 250, 0), (1500, 5, 7, 12, 5000, -900)])
def test_page_resize(device, n, page, max_pages, top, spare, extra, seed):
    rng = np.random.default_rng(seed * 1000 + n)
    table, lens, grow, n_pages, free, n_free, n_rows = resize_case(rng, n, page, max_pages, top, spare, extra)
    run_resize(device, table, lens, grow, page, n_pages, free, n_free, n_rows, alias=seed % 2 == 1)


def test_page_resize_edges(device):
    z = lambda *s: np.zeros(s, np.int32)
    run_resize(device, z(0, 4), z(0), z(0), 16, 4, np.arange(4, dtype=np.int32), 4, 3)  # no request
    run_resize(device, z(2, 0), z(2), z(2) + 1, 16, 4, np.arange(4, dtype=np.int32), 4, 2)  # no room
    run_resize(device, z(3, 2), z(3), z(3) + 5, 16, 4, np.arange(4, dtype=np.int32), 0, 15)  # no page
    run_resize(device, z(3, 2), z(3), z(3) + 5, 16, 4, np.arange(4, dtype=np.int32), -7, 15)
    run_resize(device, z(3, 2), z(3), z(3) + 5, 16, 4, np.arange(4, dtype=np.int32), 99, 15)
    run_resize(device, z(3, 2), z(3), z(3) + 5, 16, 4, np.array([9, -3, 2, 1], np.int32), 4, 15)  # bad ids
    run_resize(device, z(3, 2), z(3), np.array([5, -1, 4], np.int32), 16, 4, np.arange(4, dtype=np.int32), 4, 9)
    # requests that need no page are served when there is none
    run_resize(device, z(3, 2), z(3) + 3, np.array([4, 20, 1], np.int32), 16, 4, z(0), 0, 25)
    # pages given back beyond the stack's room are lost
    run_resize(device, np.arange(8, dtype=np.int32).reshape(2, 4), z(2) + 64, z(2) - 64, 16, 8, z(5), 1, 0)


# ----------------------------------------------------------- cache8_write --
def pools(device, rng, n_pages, H, page, d, kind):
    pages = rng.integers(0, 256, (n_pages, H, page, d)).astype(np.uint8)
    if kind == "e4m3":
        pages[(pages & 127) == 127] = 0
    else:
        pages[pages == 128] = 0
    scales = (2.0 ** rng.integers(-8, -2, (n_pages, H))).astype(np.float32)
    return pages, scales


def on(device, pages, kind):
    return torch.from_numpy(pages.copy()).to(device).view(CODES[kind])


def run_write(device, k, v, slots, kind, kp, ks, vp, vs):
    """One call, compared with the oracle's, whose state the arrays then hold."""
    dev = [on(device, kp, kind), torch.from_numpy(ks.copy()).to(device), on(device, vp, kind),
           torch.from_numpy(vs.copy()).to(device)]
    fq.cache8_write(k, v, torch.from_numpy(np.asarray(slots, np.int64)).to(device), *dev)
    opg.write(k.float().cpu().numpy(), slots, kp, ks, kind)
    opg.write(v.float().cpu().numpy(), slots, vp, vs, kind)
    for got, want in ((dev[1], ks), (dev[3], vs)):
        assert np.array_equal(got.cpu().numpy(), want, equal_nan=True)
    assert np.array_equal(raw(dev[0]), kp) and np.array_equal(raw(dev[2]), vp)


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("H,page,d", [(1, 16, 64), (3, 32, 128), (2, 128, 64), (2, 64, 256)])
def test_cache8_write(device, kind, dtype, H, page, d):
    rng = np.random.default_rng(d + page)
    g = torch.Generator(device=device).manual_seed(page)
    kp, ks = pools(device, rng, 12, H, page, d, kind)
    vp, vs = pools(device, rng, 12, H, page, d, kind)
    perm = rng.permutation(12)
    # three sequences: a new one over several pages, one in the middle of a page, one token
    for step in range(4):
        slots = []
        begin, count = (0, 2 * page + 5) if step == 0 else (2 * page + 4 + step, 1)
        slots += [perm[t // page] * page + t % page for t in range(begin, begin + count)]
        begin, count = (7, page + 1) if step == 0 else (page + 7 + step, 1)
        slots += [-1] * (step % 2) + [perm[4 + t // page] * page + t % page for t in range(begin, begin + count)]
        slots += [perm[9] * page + step * 3, 12 * page, -5, perm[10] * page + page - 1]
        x = torch.randn(len(slots), 2, H, d, generator=g, device=device) * 4.0 ** step
        x = x.to(TYPES[dtype])
        run_write(device, x[:, 0], x[:, 1], slots, kind, kp, ks, vp, vs)


@pytest.mark.parametrize("kind", list(CODES))
def test_cache8_write_values(device, kind):
    """Zeros, the least and largest magnitudes, borders of the scale, what is no number."""
    top = 127.0 if kind == "int8" else 448.0
    rng = np.random.default_rng(3)
    kp, ks = pools(device, rng, 6, 1, 16, 64, kind)
    vp, vs = pools(device, rng, 6, 1, 16, 64, kind)
    ks[3] = 0.3  # (not a power of two)
    vs[3] = np.nan
    x = torch.zeros(12, 2, 1, 64, device=device)
    x[1] = 1e-45
    x[2] = 3.4e38
    x[3, 0] = top
    x[3, 1] = math.nextafter(top, math.inf) * (1 + 2.0 ** -23)
    x[4] = torch.linspace(-0.31, 0.29, 64, device=device)
    x[5, 0, 0, 3] = math.inf
    x[5, 1, 0, 9] = math.nan
    x[6] = 1.0
    x[7] = -1e-3
    x[8, 0], x[8, 1] = 2.5, 1e-30
    slots = [0, 1, 2, 17, 3 * 16 + 4, 4 * 16 + 2, 4 * 16 + 3, 4 * 16 + 4, 5 * 16, -1, 0, 16]
    # (the last two name pages a second time: other calls)
    run_write(device, x[:9, 0], x[:9, 1], slots[:9], kind, kp, ks, vp, vs)
    run_write(device, x[9:11, 0], x[9:11, 1], slots[9:11], kind, kp, ks, vp, vs)
    run_write(device, x[6:9, 0], x[6:9, 1], [4 * 16, 4 * 16 + 1, 5 * 16 + 1], kind, kp, ks, vp, vs)


@pytest.mark.parametrize("kind", list(CODES))
def test_cache8_write_token_by_token(device, kind):
    """A page filled one token at a time, its magnitudes growing and shrinking."""
    rng = np.random.default_rng(5)
    kp, ks = pools(device, rng, 2, 2, 32, 64, kind)
    vp, vs = kp.copy(), ks.copy()
    for t in range(32):
        x = torch.from_numpy(rng.standard_normal((1, 2, 2, 64)).astype(np.float32)).to(device)
        x *= 2.0 ** (6 * math.sin(t))
        run_write(device, x[:, 0], x[:, 1], [32 + t], kind, kp, ks, vp, vs)


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("H,page,d,n,dtype", [
    (8, 16, 64, 3000, "bf16"), (16, 16, 128, 2100, "fp16"), (8, 32, 128, 2500, "fp32"),
    (32, 128, 64, 4100, "bf16"), (4, 64, 256, 6000, "fp16"), (8, 64, 64, 1500, "fp32"), (2, 16, 256, 5000, "bf16")])
def test_cache8_write_many_rows(device, kind, H, page, d, n, dtype):
    """Prompts of all lengths, from the middle of a page on, with rows and tokens left out."""
    rng = np.random.default_rng(n + d)
    slots, n_pages = [], 0
    while len(slots) < n:
        begin = int(rng.integers(page)) if rng.random() < 0.7 else 0
        tokens = np.arange(begin, begin + int(rng.integers(1, 5 * page)))
        if rng.random() < 0.3:  # slots of a run need not follow on each other
            tokens = tokens[rng.random(len(tokens)) < 0.8]
        slots += [(n_pages, int(t)) for t in tokens]
        n_pages += 6
        if rng.random() < 0.4:
            slots += [None] * int(rng.integers(1, 4))
    perm = rng.permutation(n_pages)
    slots = [-1 if s is None else int(perm[s[0] + s[1] // page]) * page + s[1] % page for s in slots[:n]]
    kp, ks = pools(device, rng, n_pages, H, page, d, kind)
    vp, vs = pools(device, rng, n_pages, H, page, d, kind)
    g = torch.Generator(device=device).manual_seed(d)
    x = torch.randn(n, 2, H, d, generator=g, device=device) * 2.0 ** torch.randint(
        -6, 6, (n, 1, 1, 1), generator=g, device=device)
    x = x.to(TYPES[dtype])
    run_write(device, x[:, 0], x[:, 1], slots, kind, kp, ks, vp, vs)


# ------------------------------------------------------------ attn_cache8 --
def make_cache(rng, lens, H, page, d, kind, spare=3, spread=0):
    """Pages in no order; what no token owns holds codes and scales that are no numbers."""
    used = [-(-max(0, int(t)) // page) for t in lens]
    n_pages = sum(used) + spare
    perm = rng.permutation(n_pages)
    most = max(1, max(used, default=0)) + 1
    table = np.full((len(lens), most), -7, np.int32)
    kp = np.full((n_pages, H, page, d), 127 if kind == "e4m3" else 100, np.uint8)
    vp, at = kp.copy(), 0
    ks = np.full((n_pages, H), np.nan, np.float32)
    vs = ks.copy()
    for g, t in enumerate(lens):
        table[g, :used[g]] = perm[at:at + used[g]]
        at += used[g]
        for j in range(used[g]):
            p, m = table[g, j], min(page, int(t) - j * page)
            for pages in (kp, vp):
                x = rng.standard_normal((H, m, d)) * (35 if kind == "int8" else 70)
                pages[p, :, :m] = opg.to_codes(x, kind)
            unit = 1 / 35 if kind == "int8" else 1 / 70
            ks[p] = unit * np.exp(0.3 * rng.standard_normal(H))
            vs[p] = unit * np.exp(0.3 * rng.standard_normal(H)) * 2.0 ** rng.integers(-spread, spread + 1)
    return kp, ks, vp, vs, table


def check_attention(out, q, kp, ks, vp, vs, table, lens, starts, causal, kind, scale=None):
    """Element by element.  A score is a sum of d products of exact codes with queries that
    two parts of 11 bits hold (2^-21 of each), in 32 bits, times scales: off by at most
    e = (d + 8) 2^-24 + 2^-21 of the sum of its terms' magnitudes A.  A weight and the sum
    of weights are off by 2 e A, by 2^-19 (exponential, parts of the weight, references) and
    by (t + 8) 2^-24 for the sums over t tokens; so is the result, times sum_t w_t |V_t|."""
    H, d = ks.shape[1], q.shape[2]
    G = q.shape[1] // H
    scale = 1 / math.sqrt(d) if scale is None else scale
    for g in range(len(lens)):
        b, e = int(starts[g]), int(starts[g + 1])
        L, M = int(lens[g]), e - b
        if L < 0 or L > table.shape[1] * kp.shape[2] or (causal and M > L):
            assert np.isnan(out[b:e]).all()
            continue
        seen = np.ones((M, L), bool) if not causal else np.tri(M, L, L - M, dtype=bool)
        for h in range(H):
            K = opg.rows_of(kp, ks, table[g], L, h, kind)
            V = opg.rows_of(vp, vs, table[g], L, h, kind)
            for j in range(G):
                x = q[b:e, h * G + j]
                ref, w = osv.attend(x, K, V, seen, scale)
                A = (np.abs(x) @ np.abs(K).T * abs(scale)).max(initial=0)
                tol = (2 * A * ((d + 8) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -19 + (L + 8) * 2.0 ** -24)
                err = np.abs(out[b:e, h * G + j] - ref)
                lim = tol * (w @ np.abs(V))
                assert (err <= lim).all(), (g, h, j, float((err / np.maximum(lim, 1e-300)).max()))


def run_attention(device, rng, lens, rows, H, G, page, d, kind, dtype, causal, one=False, scale=0.0,
                  q_times=1.0, pad=0, **kw):
    lens = np.asarray(lens, np.int32)
    kp, ks, vp, vs, table = make_cache(rng, np.where(lens > 100000, 0, lens), H, page, d, kind, **kw)
    starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n = int(starts[-1]) + pad
    q = (torch.from_numpy(rng.standard_normal((n, H * G, d))).float() * q_times).to(TYPES[dtype]).to(device)
    t = lambda a: torch.from_numpy(a).to(device)
    out = torch.full((n, H * G, d), 7.0, device=device)
    fq.attn_cache8(q, on(device, kp, kind), t(ks), on(device, vp, kind), t(vs), t(table), t(lens),
                   None if one else t(starts), causal=causal, scale=scale, out=out)
    got = host(out)
    assert (got[n - pad:] == 7.0).all()
    check_attention(got, host(q), kp, ks, vp, vs, table, lens, starts, causal, kind,
                    None if scale <= 0 else scale)
    return got


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("H,G,page,d", [(1, 1, 16, 64), (2, 8, 16, 64), (2, 3, 32, 128), (1, 16, 64, 128),
                                        (1, 5, 128, 256), (3, 2, 16, 256), (1, 16, 32, 256)])
def test_attn_one_row(device, kind, dtype, H, G, page, d):
    rng = np.random.default_rng(d + G)
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300, 1000, -1, 10 ** 9]
    run_attention(device, rng, lens, [1] * len(lens), H, G, page, d, kind, dtype, False, one=True)
    run_attention(device, rng, lens[3:9], [1] * 6, H, G, page, d, kind, dtype, True, one=True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("H,G,page,d,dtype", [(1, 1, 16, 64, "fp16"), (2, 4, 32, 128, "bf16"),
                                              (1, 8, 64, 64, "bf16"), (1, 7, 16, 128, "fp32"),
                                              (2, 16, 128, 64, "bf16"), (1, 2, 16, 256, "fp16")])
def test_attn_chunks(device, causal, kind, H, G, page, d, dtype):
    rng = np.random.default_rng(G + d)
    rows = [5, 0, 1, 40, 17, 100, 3, 2]
    lens = [5, 9, 40, 333, 17, 150, 2, 0]  # (the last two: fewer tokens than rows)
    run_attention(device, rng, lens, rows, H, G, page, d, kind, dtype, causal, pad=3)


@pytest.mark.parametrize("kind", list(CODES))
@pytest.mark.parametrize("n,length,rows,H,G,page,d,causal", [
    (1, 20000, 1, 1, 8, 16, 64, True), (3, 9000, 1, 2, 4, 64, 128, True),
    (1, 700, 600, 1, 8, 32, 64, True), (2, 1500, 130, 2, 1, 16, 64, False),
    (1, 1029, 260, 1, 4, 32, 128, True), (40, 200, 1, 4, 8, 16, 64, True)])
def test_attn_long(device, kind, n, length, rows, H, G, page, d, causal):
    rng = np.random.default_rng(length)
    lens = [length - 37 * g for g in range(n)]
    run_attention(device, rng, lens, [rows] * n, H, G, page, d, kind, "bf16", causal)


@pytest.mark.parametrize("kind", list(CODES))
def test_attn_scales_far_apart(device, kind):
    """Pages of values whose scales differ by 2^60: small ones keep their bits where they weigh."""
    rng = np.random.default_rng(8)
    run_attention(device, rng, [700, 90], [1, 20], 2, 4, 16, 64, kind, "fp32", True, spread=30)


@pytest.mark.parametrize("q_times,scale", [(1e-30, 0.0), (1e4, 0.0), (30.0, 0.5), (1e-3, 40.0)])
def test_attn_queries_of_any_size(device, q_times, scale):
    rng = np.random.default_rng(9)
    run_attention(device, rng, [200, 31], [1, 20], 1, 4, 16, 64, "e4m3", "fp32", True, scale=scale,
                  q_times=q_times)


def test_attn_scales_farther_apart(device):
    """A page of the largest scale whose weight is so small that it counts for as much as the others."""
    rng = np.random.default_rng(14)
    kp, ks, vp, vs, table = make_cache(rng, [64], 1, 16, 64, "int8")
    kp[:] = 0
    kp[table[0, :4], 0, :, 0] = np.array([10, 60, 35, 0], np.uint8)[:, None]  # scores, up to factors
    ks[:], vs[:] = 1.0, 1.0
    vs[table[0, :4], 0] = 2.0 ** np.array([40, -60, -10, 30])
    for step in (0.5, 1.0, 1.5, 2.0):  # 2^(50 step / ln 2) between the first two pages' weights
        q = torch.zeros(1, 1, 64, device=device)
        q[0, 0, 0] = step * math.log(2)
        t = lambda a: torch.from_numpy(a).to(device)
        out = fq.attn_cache8(q, on(device, kp, "int8"), t(ks), on(device, vp, "int8"), t(vs), t(table),
                             t(np.array([64], np.int32)), scale=1.0)
        check_attention(host(out), host(q), kp, ks, vp, vs, table, [64], [0, 1], True, "int8", 1.0)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_attn_queries_that_are_no_numbers(device, rows, dtype):
    """A row of queries with a NaN or an infinity is NaN, and no other row is."""
    rng = np.random.default_rng(15)
    lens = np.array([100, 77], np.int32)
    kp, ks, vp, vs, table = make_cache(rng, lens, 1, 16, 64, "e4m3")
    q = torch.randn(2 * rows, 3, 64, device=device).to(TYPES[dtype])
    q[rows - 1, 1, 5], q[rows, 2, 63] = math.inf, math.nan
    t = lambda a: torch.from_numpy(a).to(device)
    starts = t(np.array([0, rows, 2 * rows], np.int32))
    out = host(fq.attn_cache8(q, on(device, kp, "e4m3"), t(ks), on(device, vp, "e4m3"), t(vs), t(table), t(lens),
                              starts))
    bad = np.zeros((2 * rows, 3), bool)
    bad[rows - 1, 1] = bad[rows, 2] = True
    assert np.isnan(out[bad]).all() and np.isfinite(out[~bad]).all()


def test_attn_without_pages(device):
    """Tables of no page: rows that see nothing are zero, causal rows of no token NaN."""
    rng = np.random.default_rng(16)
    kp, ks, vp, vs, _ = make_cache(rng, [16], 1, 16, 64, "int8")
    t = lambda a: torch.from_numpy(a).to(device)
    args = (on(device, kp, "int8"), t(ks), on(device, vp, "int8"), t(vs),
            torch.zeros(3, 0, dtype=torch.int32, device=device), torch.zeros(3, dtype=torch.int32, device=device))
    starts = t(np.array([0, 2, 2, 50], np.int32))
    q = torch.randn(50, 2, 64, device=device)
    for s in (starts, None):
        rows = q if s is not None else q[:3].contiguous()
        assert (fq.attn_cache8(rows, *args, s, causal=False) == 0).all()
        assert torch.isnan(fq.attn_cache8(rows, *args, s)).all()


def test_attn_table_wider_than_its_sequences(device):
    """Room for 65536 tokens, none of the sequences longer than 700: as in a narrow table."""
    rng = np.random.default_rng(17)
    lens = np.array([700, 3, 0, 512, 64, 333], np.int32)
    for rows in (1, 30):
        kp, ks, vp, vs, table = make_cache(rng, lens, 2, 16, 64, "int8")
        wide = np.full((6, 4096), -1, np.int32)
        wide[:, :table.shape[1]] = table
        q = torch.randn(6 * rows, 8, 64, device=device)
        t = lambda a: torch.from_numpy(a).to(device)
        out = fq.attn_cache8(q, on(device, kp, "int8"), t(ks), on(device, vp, "int8"), t(vs), t(wide), t(lens),
                             t(np.arange(0, 6 * rows + 1, rows, dtype=np.int32)), causal=False)
        check_attention(host(out), host(q), kp, ks, vp, vs, wide, lens, np.arange(0, 6 * rows + 1, rows), False,
                        "int8")


@pytest.mark.parametrize("n,H", [(700, 2), (3000, 1)])
def test_attn_many_sequences(device, n, H):
    """More sequences than threads, a few long among short ones, in one call and in room for more."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 40, n).astype(np.int32)
    lens[[5, n // 2, n - 1]] = 2500
    run_attention(device, rng, lens, [1] * n, H, 2, 16, 64, "int8", "bf16", False, one=True)
    rows = rng.integers(0, 3, n)
    rows[n // 2] = 70
    run_attention(device, rng, lens, rows, H, 2, 16, 64, "int8", "bf16", False)


def test_attn_finite_for_the_largest(device):
    rng = np.random.default_rng(10)
    kp, ks, vp, vs, table = make_cache(rng, [100], 1, 16, 64, "int8")
    t = lambda a: torch.from_numpy(a).to(device)
    q = torch.full((1, 1, 64), 3e38, device=device)
    for times in (1.0, 1e30):
        out = fq.attn_cache8(q, on(device, kp, "int8"), t(ks * np.float32(times)), on(device, vp, "int8"), t(vs),
                             t(table), t(np.array([100], np.int32)))
        V = opg.rows_of(vp, vs, table[0], 100, 0, "int8")
        assert torch.isfinite(out).all() and np.abs(host(out)).max() <= np.abs(V).max() * (1 + 2.0 ** -18)


@pytest.mark.parametrize("kind", list(CODES))
def test_attn_bad_pages_and_lost_scales(device, kind):
    """Unknown pages and scales that are no numbers: NaN where they are seen, nowhere else."""
    rng = np.random.default_rng(11)
    lens, rows = np.array([100, 100, 64, 64], np.int32), [70, 1, 40, 40]
    starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    kp, ks, vp, vs, table = make_cache(rng, lens, 1, 16, 64, kind)
    table[1, 2] = kp.shape[0]
    table[0, 6] = -1
    ks[table[2, 3]] = np.nan
    vs[table[3, 3]] = np.nan
    q = torch.randn(151, 2, 64, device=device)
    t = lambda a: torch.from_numpy(a).to(device)
    out = host(fq.attn_cache8(q, on(device, kp, kind), t(ks), on(device, vp, kind), t(vs), t(table), t(lens),
                              t(starts)))
    assert np.isfinite(out[:66]).all() and np.isnan(out[66:70]).all()  # tokens 96 .. 99 on page 6
    assert np.isnan(out[70]).all()
    assert np.isfinite(out[71:95]).all() and np.isnan(out[95:111]).all()
    assert np.isfinite(out[111:135]).all() and np.isnan(out[135:151]).all()


def test_attn_bad_starts(device):
    rng = np.random.default_rng(12)
    lens = np.array([50, 50, 50], np.int32)
    kp, ks, vp, vs, table = make_cache(rng, lens, 1, 16, 64, "int8")
    t = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(device)
    f = lambda a: torch.from_numpy(a).to(device)
    q = torch.randn(12, 1, 64, device=device)
    args = (q, on(device, kp, "int8"), f(ks), on(device, vp, "int8"), f(vs), t(table), t(lens))
    want = fq.attn_cache8(*args, t([0, 4, 8, 12]))
    for starts, whole in (([0, 4, 8, 13], [0, 1]), ([-1, 4, 8, 12], [1, 2]), ([0, 4, 2, 1], [0])):  # (no row has two sequences)
        out = torch.full((12, 1, 64), 7.0, device=device)
        fq.attn_cache8(*args, t(starts), out=out)
        for g in whole:
            assert torch.equal(out[4 * g:4 * g + 4], want[4 * g:4 * g + 4])
    assert torch.equal(fq.attn_cache8(*args, t([0, 4, 8, 12])), want)


def test_attn_layouts_streams_and_workspace(device):
    """Rows at any element, another stream, a workspace used again: the same bits."""
    rng = np.random.default_rng(13)
    lens = [300, 77, 500]
    kp, ks, vp, vs, table = make_cache(rng, lens, 2, 16, 64, "e4m3")
    t = lambda a: torch.from_numpy(np.asarray(a)).to(device)
    pools_ = (on(device, kp, "e4m3"), t(ks), on(device, vp, "e4m3"), t(vs))
    tab, ln, st = t(table), t(np.array(lens, np.int32)), t(np.array([0, 30, 31, 60], np.int32))
    q = torch.randn(60, 8, 64, device=device).bfloat16()
    want = fq.attn_cache8(q, *pools_, tab, ln, st)
    buf = torch.empty(60 * 8 * 64 + 5, dtype=torch.bfloat16, device=device)
    res = torch.empty(60 * 8 * 64 + 5, device=device)
    for off in (1, 3, 5):
        qo, oo = buf[off:off + q.numel()].view_as(q), res[off:off + q.numel()].view_as(want)
        qo.copy_(q)
        assert torch.equal(fq.attn_cache8(qo, *pools_, tab, ln, st, out=oo), want)
    need = fq.attn_cache8_workspace_bytes(3, 60, 2, 4, table.shape[1], 16, 64)
    ws = torch.full((max(1, need),), 255, dtype=torch.uint8, device=device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            got = fq.attn_cache8(q, *pools_, tab, ln, st, workspace=ws)
    side.synchronize()
    assert torch.equal(got, want)


def test_pools_beyond_32_bits(device):
    """Pages whose bytes lie 5 GB into their pool."""
    H, page, d, n_pages = 8, 128, 128, 40000  # 5.2 GB each
    kp, vp = (torch.empty((n_pages, H, page, d), dtype=torch.int8, device=device) for _ in range(2))
    ks, vs = (torch.empty((n_pages, H), device=device) for _ in range(2))
    ids = [n_pages - 1, 0, n_pages - 2]
    slots = torch.cat([torch.arange(page, device=device) + p * page for p in ids])[:300]
    x = torch.randn(300, 2, H, d, device=device)
    fq.cache8_write(x[:, 0], x[:, 1], slots, kp, ks, vp, vs)
    small = [np.zeros((3, H, page, d), np.uint8), np.zeros((3, H), np.float32),
             np.zeros((3, H, page, d), np.uint8), np.zeros((3, H), np.float32)]
    near = np.arange(300)
    opg.write(x[:, 0].cpu().numpy(), near, small[0], small[1], "int8")
    opg.write(x[:, 1].cpu().numpy(), near, small[2], small[3], "int8")
    for i, p in enumerate(ids):
        m = min(page, 300 - i * page)
        assert np.array_equal(raw(kp[p])[:, :m], small[0][i][:, :m])
        assert np.array_equal(vs[p].cpu().numpy(), small[3][i])
    q = torch.randn(5, H, d, device=device)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=device)
    out = fq.attn_cache8(q, kp, ks, vp, vs, i32([ids]), i32([300]), i32([0, 5]))
    check_attention(host(out), host(q), *small, np.array([[0, 1, 2]]), [300], [0, 5], True, "int8")


# ------------------------------------------------------- as they are used --
@pytest.mark.parametrize("kind", list(CODES))
def test_serving_loop(device, kind):
    """Prompts, then single tokens, with a request that ends and one that begins."""
    H, G, d, page, n_pages, n = 2, 4, 64, 16, 40, 5
    rng = np.random.default_rng(21)
    freqs = fq.rope_freqs(d)
    fd = torch.from_numpy(freqs).to(device)
    kp, ks = pools(device, rng, n_pages, H, page, d, kind)
    vp, vs = kp.copy(), ks.copy()
    dev = [on(device, kp, kind), torch.from_numpy(ks).to(device), on(device, vp, kind),
           torch.from_numpy(vs).to(device)]
    table, free = np.full((n, 12), -1, np.int32), rng.permutation(n_pages).astype(np.int32)
    tab, fr = torch.from_numpy(table).to(device), torch.from_numpy(free).to(device)
    lens, left = np.zeros(n, np.int32), n_pages
    ln, lf = torch.from_numpy(lens).to(device), torch.tensor([left], dtype=torch.int32, device=device)
    steps = [[30, 0, 17, 64, 5], [1, 20, 1, 1, 1], [1, 1, 1, -65, 1], [1, 1, 1, 9, 1], [1, 1, 1, 1, 11]]
    for grow in steps:
        rows = sum(max(0, x) for x in grow)
        gr = torch.tensor(grow, dtype=torch.int32, device=device)
        ln, starts, slots, positions, lf = fq.page_resize(tab, ln, gr, page, n_pages, fr, lf, rows)
        table, free, lens, st, sl, po, left = opg.resize(table, lens, np.array(grow, np.int32), page, n_pages,
                                                         free, left, rows)
        assert np.array_equal(slots.cpu().numpy(), sl) and np.array_equal(ln.cpu().numpy(), lens)
        qkv = torch.randn(rows, H * G + 2 * H, d, device=device).bfloat16()
        q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        q, k = fq.rope(q, k, positions, fd)
        check_rope(k, qkv[:, H * G:H * G + H], po, freqs, "half")
        fq.cache8_write(k, v, slots, *dev)
        opg.write(k.float().cpu().numpy(), sl, kp, ks, kind)
        opg.write(v.float().cpu().numpy(), sl, vp, vs, kind)
        assert np.array_equal(raw(dev[0]), kp) and np.array_equal(dev[3].cpu().numpy(), vs)
        out = fq.attn_cache8(q, *dev, tab, ln, starts)
        check_attention(host(out), host(q), kp, ks, vp, vs, table, lens, st, True, kind)


def test_slots_address_coded_rows(device):
    """Slots as rows of a flat coded cache: `encode` into them, `decode` out of them."""
    d, k, N, page, n_pages = 64, 4, 256, 16, 9
    rng = np.random.default_rng(22)
    R = torch.from_numpy(fq.build_rotation(d, 2)).to(device)
    C = torch.from_numpy((rng.standard_normal((N, k)) / 8).astype(np.float16).astype(np.float32)).to(device)
    P = fq.payload_bytes(d, k, N)
    payload = torch.zeros(n_pages * page, P, dtype=torch.uint8, device=device)
    norms = torch.zeros(n_pages * page, dtype=torch.int16, device=device)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=device)
    tab = torch.full((2, 6), -1, dtype=torch.int32, device=device)
    _, _, slots, positions, _ = fq.page_resize(tab, i32([0, 0]), i32([37, 50]), page, n_pages,
                                               i32(rng.permutation(n_pages)), i32([n_pages]), 87)
    x = torch.randn(87, 1, d, device=device)
    fd = torch.from_numpy(fq.rope_freqs(d)).to(device)
    keys = fq.rope(x, None, positions, fd)[0][:, 0]
    pay, nrm = fq.encode(keys, k, N, R, C)
    payload[slots], norms[slots] = pay, nrm
    assert torch.equal(fq.decode(payload, norms, d, k, N, R, C, token_ids=slots),
                       fq.decode(pay, nrm, d, k, N, R, C))


def test_captured_step(device):
    """One decode step in a graph, replayed over new inputs, between eager calls of its own."""
    H, G, d, page, n_pages, n = 1, 8, 64, 16, 30, 3
    rng = np.random.default_rng(23)
    kp, ks = pools(device, rng, n_pages, H, page, d, "e4m3")

    def state():
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=device)
        s = [on(device, kp, "e4m3"), torch.from_numpy(ks.copy()).to(device), on(device, kp, "e4m3"),
             torch.from_numpy(ks.copy()).to(device)]
        table = torch.full((n, 10), -1, dtype=torch.int32, device=device)
        for g in range(n):
            table[g, :4] = torch.arange(4 * g, 4 * g + 4)
        free = torch.arange(12, 30, device=device, dtype=torch.int32)
        return s, table, i32([50, 63, 64]), free, i32([18])

    ws = [torch.empty(max(1, m), dtype=torch.uint8, device=device) for m in
          (fq.page_resize_workspace_bytes(n), fq.attn_cache8_workspace_bytes(n, n, H, G, 10, page, d))]
    fd = torch.from_numpy(fq.rope_freqs(d)).to(device)
    qkv = torch.randn(n, H * G + 2 * H, d, device=device).bfloat16()
    grow = torch.ones(n, dtype=torch.int32, device=device)

    def step(s, table, lens, free, left, outs, o):
        fq.page_resize(table, lens, grow, page, n_pages, free, left, n, out=(lens,) + outs + (left,),
                       workspace=ws[0])
        q, k = fq.rope(qkv[:, :H * G], qkv[:, H * G:H * G + H], outs[2], fd)
        fq.cache8_write(k, qkv[:, H * G + H:], outs[1], *s)
        fq.attn_cache8(q, *s, table, lens, workspace=ws[1], out=o)

    def outputs():
        return (torch.zeros(n + 1, dtype=torch.int32, device=device), torch.zeros(n, dtype=torch.int64, device=device),
                torch.zeros(n, dtype=torch.int32, device=device))

    eager, captured = state(), state()
    eo, co = outputs(), outputs()
    out_e, out_c = (torch.zeros(n, H * G, d, device=device) for _ in range(2))
    warm = state()
    step(*warm, outputs(), out_c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured, co, out_c)
    for i in range(6):
        qkv.copy_(torch.randn(n, H * G + 2 * H, d, device=device) * (1 + i))
        step(*eager, eo, out_e)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out_e, out_c) and torch.equal(eager[1], captured[1])
        assert torch.equal(eager[2], captured[2]) and torch.equal(raw_t(eager[0][0]), raw_t(captured[0][0]))
        assert torch.equal(eager[0][1], captured[0][1])


@pytest.mark.parametrize("rows", [1, 40])
def test_captured_long_items(device, rows):
    """Items cut into parts, their lengths changing between replays, with eager calls between."""
    rng = np.random.default_rng(24)
    lens = np.array([6000, 300, 2900], np.int32)
    kp, ks, vp, vs, table = make_cache(rng, lens, 2, 16, 64, "e4m3")
    t = lambda a: torch.from_numpy(a).to(device)
    pools_ = (on(device, kp, "e4m3"), t(ks), on(device, vp, "e4m3"), t(vs))
    tab, ln, st = t(table), t(lens), t(np.arange(0, 3 * rows + 1, rows, dtype=np.int32))
    q = torch.randn(3 * rows, 8, 64, device=device)
    ws = torch.empty(fq.attn_cache8_workspace_bytes(3, 3 * rows, 2, 4, table.shape[1], 16, 64), dtype=torch.uint8,
                     device=device)
    assert ws.numel() > 0
    out, want = torch.zeros(3 * rows, 8, 64, device=device), torch.zeros(3 * rows, 8, 64, device=device)
    call = lambda o, w: fq.attn_cache8(q, *pools_, tab, ln, st, workspace=w, out=o)
    call(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for now in ([6000, 300, 2900], [50, 300, 2900], [6000, 40, 41], [5999, -1, 2049], [6000, 300, 2900]):
        ln.copy_(torch.tensor(now, dtype=torch.int32))
        q.normal_()
        call(want, None)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int32), want.view(torch.int32))


def raw_t(t):
    return t.view(torch.uint8)
