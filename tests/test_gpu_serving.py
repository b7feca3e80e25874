"""The serving operators on the device against float64 references.

Attention tolerance, derived: a score is a rotated query (sums of d products)
times a codeword row (a sum of d products), both in float32, whose rounding
errors move it by about sqrt(d) 2^-24 |q| |K| scale each; twice that is allowed.
Weights, their 22-bit parts, exponentials and sums add 2^-18.  An output row may
be off by that much relative to sum_t p_t |V_t|, a token's weight relative to
the weight.  (d = 64, |q| |K| scale = 16: 2e-5.)
"""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from oracle import codec as occ
from oracle import serving as osv

from _fixtures import oracle_rotation

pytestmark = pytest.mark.gpu

# every kind of code: table rows of 4 dims, pairs of blocks, one and two
# dimensions per index, large codebooks, blocks above 16 dims, d = 128
CODES = [(64, 4, 256), (64, 8, 16), (64, 2, 64), (64, 2, 16), (64, 8, 64), (64, 1, 16), (64, 1, 2),
         (64, 2, 256), (64, 2, 8), (64, 4, 2), (64, 4, 512), (64, 8, 1024), (64, 16, 4096),
         (64, 32, 1024), (64, 64, 256), (64, 4, 16384), (128, 4, 4096), (128, 4, 256),
         (128, 8, 256), (128, 16, 64), (128, 1, 16), (128, 2, 64), (128, 16, 16384), (128, 2, 16),
         (128, 16, 256), (128, 4, 64), (64, 4, 64), (64, 8, 2048), (64, 16, 4), (64, 32, 2)]


def codebook(d, k, N, seed=7, exact=True):
    x = np.random.default_rng(seed + 31 * k + N).standard_normal((N, d))
    c = (x / np.linalg.norm(x, axis=1, keepdims=True))[:, :k].astype(np.float32)
    return c.astype(np.float16).astype(np.float32) if exact else c


class Cache:
    """Random rows of n groups (numpy, and on the device), and their decoded form."""

    def __init__(self, d, k, N, n, T, device, seed=0, C=None, norm=8.0):
        rng = np.random.default_rng(seed)
        self.d, self.k, self.N, self.n, self.T = d, k, N, n, T
        self.C = codebook(d, k, N) if C is None else C
        self.R = oracle_rotation(d)
        self.np, self.dev = [], []
        for _ in range(2):
            idx = rng.integers(0, N, (n * T, d // k))
            self.np.append(occ.pack(idx, N).reshape(n, T, -1))
            h = (np.abs(rng.standard_normal((n, T)) * 0.4 + 1) * norm).astype(np.float16)
            self.np.append(occ.fp16_bits(h).copy())
        for a in self.np:
            a = a.view(np.int16) if a.dtype == np.uint16 else a
            self.dev.append(torch.from_numpy(a.copy()).to(device))
        self.Rd = torch.from_numpy(np.array(self.R)).to(device)
        self.Cd = torch.from_numpy(np.array(self.C)).to(device)

    def decoded(self, g, t, which):
        pay, nrm = self.np[2 * which][g, :t], self.np[2 * which + 1][g, :t]
        if t == 0:
            return np.zeros((0, self.d))
        return occ.decode(occ.unpack(pay, self.d // self.k, self.N), occ.from_fp16_bits(nrm),
                          self.R, self.C)


def queries(rng, shape, dtype, device):
    q = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype)
    return q.to(device), q.double().numpy()


def random_masks(rng, M):
    return fq.tree_masks([int(rng.integers(-1, i)) if i else -1 for i in range(M)])


def close(o, q, K, V, seen, scale=None):
    """o [r, d] against the reference, in the module's tolerance; returns the reference weights."""
    ref, w = osv.attend(q, K, V, seen, scale)
    d = q.shape[1]
    sc = 1 / np.sqrt(d) if scale is None else scale
    vabs = w @ np.linalg.norm(V, axis=1) if len(V) else np.zeros(len(q))
    for r in range(len(q)):
        kmax = np.linalg.norm(K[seen[r]], axis=1).max() if seen[r].any() else 0.0
        tol = 2 * np.sqrt(d) * 2.0**-24 * np.linalg.norm(q[r]) * kmax * sc + 2.0**-18
        err = np.linalg.norm(o[r] - ref[r])
        assert err <= tol * vabs[r], (r, err, tol * vabs[r])
    return w


def weight_tol(q, K, scale=None):
    d = q.shape[1]
    sc = 1 / np.sqrt(d) if scale is None else scale
    kmax = np.linalg.norm(K, axis=1).max() if len(K) else 0.0
    return 2 * np.sqrt(d) * 2.0**-24 * np.linalg.norm(q, axis=1).max() * kmax * sc + 2.0**-18


def run_tree(c, q, lens, masks, **kw):
    dev = q.device
    return fq.attn_tree(q, *c.dev, torch.tensor(lens, dtype=torch.int32, device=dev),
                        torch.from_numpy(np.array(masks)).to(dev), c.k, c.N, c.Rd, c.Cd, **kw)


def check_tree(c, q, q64, out, lens, masks, scale=None, groups=None):
    M, G = q64.shape[1:3]
    out = out.double().cpu().numpy()
    for g in range(c.n) if groups is None else groups:
        t = lens[g] + M
        seen = np.repeat(osv.seen_by_tree(lens[g], masks[g] if masks.ndim == 2 else masks, M), G, 0)
        close(out[g].reshape(M * G, -1), q64[g].reshape(M * G, -1), c.decoded(g, t, 0),
              c.decoded(g, t, 1), seen, scale)


# -------------------------------------------------------------------- tree --
@pytest.mark.parametrize("d,k,N", CODES, ids=str)
def test_tree_codes(device, d, k, N):
    rng = np.random.default_rng(k * N)
    M, G, lens = 5, 3, [70, 0, 131]
    c = Cache(d, k, N, 3, 140, device)
    q, q64 = queries(rng, (3, M, G, d), torch.bfloat16, device)
    masks = np.stack([random_masks(rng, M) for _ in range(3)])
    check_tree(c, q, q64, run_tree(c, q, lens, masks), lens, masks)


@pytest.mark.parametrize("M,G,lens,dtype,shared", [
    (1, 1, [0], torch.float32, True),
    (1, 8, [1, 31, 32, 33], torch.float16, True),
    (2, 16, [63, 64, 65, 300], torch.bfloat16, False),
    (7, 5, [5, 1000], torch.float32, False),
    (26, 8, [517, 0, 33], torch.bfloat16, False),
    (64, 1, [17, 190], torch.float16, True),
    (64, 16, [90, 3], torch.bfloat16, False),
    (17, 12, [2500], torch.float32, True),
], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 1, 16), (128, 4, 256)], ids=str)
def test_tree_shapes(device, d, k, N, M, G, lens, dtype, shared):
    rng = np.random.default_rng(M * G)
    n = len(lens)
    c = Cache(d, k, N, n, max(lens) + M + 3, device, seed=M)
    q, q64 = queries(rng, (n, M, G, d), dtype, device)
    masks = random_masks(rng, M) if shared else np.stack([random_masks(rng, M) for _ in lens])
    check_tree(c, q, q64, run_tree(c, q, lens, masks), lens, masks)


@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 1, 16)], ids=str)
def test_tree_masks_that_leave_rows_empty(device, d, k, N):
    """No context and an empty mask: zeros; with a context, the context alone;
    bits from M on are ignored; a token may be masked from itself."""
    rng = np.random.default_rng(5)
    M, G, lens = 6, 2, [0, 40]
    c = Cache(d, k, N, 2, 64, device)
    q, q64 = queries(rng, (2, M, G, d), torch.float32, device)
    masks = np.array([0, 1, -1 << 6, 0b101010, 0b111111, -1], dtype=np.int64)
    out = run_tree(c, q, lens, masks)
    assert torch.count_nonzero(out[0, 0]) == 0 and torch.count_nonzero(out[0, 2]) == 0
    check_tree(c, q, q64, out, lens, masks)


@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 16), (128, 4, 4096)], ids=str)
def test_tree_ignores_what_it_does_not_see(device, d, k, N):
    """Infinite and NaN norms behind the drafted tokens and in drafted tokens that no
    mask names change no bit of the output."""
    rng = np.random.default_rng(6)
    M, G, lens = 5, 4, [37, 60]
    c = Cache(d, k, N, 2, 100, device)
    q, _ = queries(rng, (2, M, G, d), torch.bfloat16, device)
    masks = np.array([0b1, 0b1, 0b10001, 0b1, 0b10001], dtype=np.int64)  # 1, 2, 3 are never seen
    a = run_tree(c, q, lens, masks)
    used = (d // k * (N.bit_length() - 1) - 1) % 8 + 1  # bits of a row's last byte
    for g, L in enumerate(lens):
        for x in (1, 3):
            for row, bits in ((L + 1, 0x7E00), (L + 2, 0x7C00), (L + 3, -1024)):  # NaN, inf, -inf
                c.dev[x][g, row] = bits
            c.dev[x][g, L + M:] = 0x7E00
        for x in (0, 2):
            c.dev[x][g, L + M:] = 255
            c.dev[x][g, L + M:, -1] = (1 << used) - 1
    assert torch.equal(a, run_tree(c, q, lens, masks)) and bool(a.isfinite().all())


def test_tree_bad_lengths(device):
    rng = np.random.default_rng(8)
    M, G, lens = 4, 3, [10, -1, 61, 60, 2**31 - 1, -2**31]
    c = Cache(64, 4, 256, 6, 64, device)
    q, q64 = queries(rng, (6, M, G, 64), torch.float32, device)
    masks = random_masks(rng, M)
    out = run_tree(c, q, lens, masks)
    for g in (1, 2, 4, 5):
        assert bool(out[g].isnan().all())
    check_tree(c, q, q64, out, lens, masks, groups=(0, 3))
    small = Cache(64, 4, 256, 1, 3, device)  # fewer rows than drafted tokens
    assert bool(run_tree(small, q[:1], [0], masks).isnan().all())


@pytest.mark.parametrize("scale", [0.3, 0.01])
@pytest.mark.parametrize("size,norm", [(1.0, 3e-4), (1e-3, 2000.0), (300.0, 0.05), (1.0, 900.0)], ids=str)
@pytest.mark.parametrize("k,N", [(4, 256), (1, 16), (8, 16)], ids=str)
def test_tree_ranges(device, k, N, size, norm, scale):
    """Codebooks that binary16 does not hold, with small and large entries, and
    value norms from 1e-4 to 2000."""
    rng = np.random.default_rng(9)
    M, G, lens = 3, 2, [200, 77]
    C = codebook(64, k, N, exact=False) * np.float32(size)
    c = Cache(64, k, N, 2, 256, device, C=C, norm=norm)
    q, q64 = queries(rng, (2, M, G, 64), torch.float32, device)
    s = scale / (size * norm)
    masks = random_masks(rng, M)
    check_tree(c, q, q64, run_tree(c, q, lens, masks, scale=s), lens, masks, np.float64(np.float32(s)))


@pytest.mark.parametrize("M,G", [(1, 5), (3, 4), (5, 5), (19, 7)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 2, 64), (64, 1, 16), (128, 4, 256), (128, 4, 4096),
                                   (128, 1, 4)], ids=str)
def test_codebooks_that_binary16_does_not_hold(device, d, k, N, M, G):
    """The residual rows' products, for every number of query rows, in the outputs and the weights."""
    rng = np.random.default_rng(21)
    lens = [130, 31]
    c = Cache(d, k, N, 2, 160, device, C=codebook(d, k, N, exact=False))
    q, q64 = queries(rng, (2, M, G, d), torch.float32, device)
    masks = random_masks(rng, M)
    check_tree(c, q, q64, run_tree(c, q, lens, masks), lens, masks)
    before = torch.rand(2, 160, device=device)
    acc = before.clone()
    check_accum(c, q64[:, 0], run_accum(c, q[:, 0].contiguous(), lens, acc), before, acc, lens)


@pytest.mark.parametrize("M,G", [(2, 2), (4, 4), (6, 4), (10, 8)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_tree_norms_that_are_no_numbers_where_they_are_seen(device, d, M, G):
    """A drafted token with an infinite or NaN value norm makes the rows that see it no
    numbers, and leaves those that do not; so does a key norm.  Another group is untouched."""
    rng = np.random.default_rng(22)
    lens = [61, 61]
    c = Cache(d, 4, 256, 2, 80, device)
    q, q64 = queries(rng, (2, M, G, d), torch.float32, device)
    masks = np.array([1 << i for i in range(M)], dtype=np.int64)
    a = run_tree(c, q, lens, masks)
    for x, bits in ((3, 0x7C00), (3, 0x7E00), (1, 0x7E00)):
        keep = c.dev[x].clone()
        c.dev[x][1, 61 + 1] = bits
        b = run_tree(c, q, lens, masks)
        assert not bool(b[1, 1].isfinite().any())
        others = [i for i in range(M) if i != 1]
        close(b[1, others].double().cpu().numpy().reshape(-1, d), q64[1, others].reshape(-1, d),
              c.decoded(1, 61 + M, 0), c.decoded(1, 61 + M, 1),
              np.repeat(osv.seen_by_tree(61, masks, M)[others], G, 0))
        assert torch.equal(a[0], b[0])
        c.dev[x][1, 30] = bits  # in the context: every row of the group sees it
        b = run_tree(c, q, lens, masks)
        assert not bool(b[1].isfinite().any()) and torch.equal(a[0], b[0])
        c.dev[x].copy_(keep)


@pytest.mark.parametrize("M,G", [(2, 2), (4, 4), (6, 4), (10, 8)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 2, 64), (64, 1, 16), (128, 4, 256)], ids=str)
def test_tree_value_norms_that_grow(device, d, k, N, M, G):
    """Value norms that rise by powers of ten along the cache, and a zero row among them."""
    rng = np.random.default_rng(10)
    c = Cache(d, k, N, 1, 700, device)
    h = np.float16(10.0 ** np.linspace(-6, 4, 700))
    h[350] = 0
    c.np[3][0] = occ.fp16_bits(h)
    c.dev[3].copy_(torch.from_numpy(c.np[3].view(np.int16)))
    q, q64 = queries(rng, (1, M, G, d), torch.float32, device)
    masks = random_masks(rng, M)
    for length in (690, 300, 40):
        check_tree(c, q, q64, run_tree(c, q, [length], masks), [length], masks)


def test_tree_query_rows_are_independent(device):
    """A NaN or infinite query row makes its own output NaN and no other; a zero row is the mean."""
    rng = np.random.default_rng(11)
    M, G, lens = 3, 4, [150]
    c = Cache(64, 4, 256, 1, 200, device)
    q, q64 = queries(rng, (1, M, G, 64), torch.float32, device)
    masks = random_masks(rng, M)
    a = run_tree(c, q, lens, masks)
    b = q.clone()
    b[0, 1, 2, 5], b[0, 2, 0, 7], b[0, 0, 1] = float("nan"), float("inf"), 0.0
    o = run_tree(c, b, lens, masks)
    assert bool(o[0, 1, 2].isnan().all()) and bool(o[0, 2, 0].isnan().all())
    same = torch.ones(M, G, dtype=torch.bool)
    same[1, 2] = same[2, 0] = same[0, 1] = False
    assert torch.equal(a[0][same.to(device)], o[0][same.to(device)])
    q64[0, 0, 1] = 0
    seen = osv.seen_by_tree(150, masks, M)[:1]
    close(o[0, 0, 1:2].double().cpu().numpy(), q64[0, 0, 1:2], c.decoded(0, 153, 0),
          c.decoded(0, 153, 1), seen)


def test_tree_of_one_is_decode_attention(device):
    rng = np.random.default_rng(12)
    c = Cache(64, 4, 256, 4, 500, device)
    q, q64 = queries(rng, (4, 8, 64), torch.bfloat16, device)
    a = fq.attn_decode(q, *c.dev, 444, 4, 256, c.Rd, c.Cd).double().cpu().numpy()
    b = run_tree(c, q[:, None], [443] * 4, np.ones(1, dtype=np.int64))[:, 0].double().cpu().numpy()
    for g in range(4):
        K, V = c.decoded(g, 444, 0), c.decoded(g, 444, 1)
        for o in (a, b):
            close(o[g], q64[g], K, V, np.ones((8, 444), dtype=bool))


# ------------------------------------------------------------------- accum --
def run_accum(c, q, lens, acc, **kw):
    return fq.attn_decode_accum(q, *c.dev, torch.tensor(lens, dtype=torch.int32, device=q.device),
                                acc, c.k, c.N, c.Rd, c.Cd, **kw)


def check_accum(c, q64, out, before, acc, lens, groups=None):
    out, before, acc = (x.double().cpu().numpy() for x in (out, before, acc))
    for g in range(c.n) if groups is None else groups:
        t = lens[g]
        K, V = c.decoded(g, t, 0), c.decoded(g, t, 1)
        w = close(out[g], q64[g], K, V, np.ones((q64.shape[1], t), dtype=bool))
        add = w.sum(0)
        assert np.array_equal(acc[g, t:], before[g, t:])
        # the sum over G heads and the addition round once each, to half a step
        tol = add * (2 * weight_tol(q64[g], K) + 2.0**-24 * q64.shape[1]) + 2.0**-24 * np.abs(acc[g, :t])
        assert np.all(np.abs(acc[g, :t] - before[g, :t] - add) <= tol)


@pytest.mark.parametrize("d,k,N", CODES, ids=str)
def test_accum_codes(device, d, k, N):
    rng = np.random.default_rng(k * N + 1)
    lens = [129, 0, 64, 1]
    c = Cache(d, k, N, 4, 133, device)
    q, q64 = queries(rng, (4, 3, d), torch.float16, device)
    before = torch.rand(4, 133, device=device)
    acc = before.clone()
    check_accum(c, q64, run_accum(c, q, lens, acc), before, acc, lens)


@pytest.mark.parametrize("G,lens,dtype", [(1, [1], torch.float32), (8, [31, 32, 33, 2047], torch.bfloat16),
                                          (16, [700, 5], torch.float16), (5, [255, 256, 257], torch.float32)],
                         ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 2, 64), (64, 1, 16), (128, 4, 256)], ids=str)
def test_accum_shapes(device, d, k, N, G, lens, dtype):
    rng = np.random.default_rng(G)
    n = len(lens)
    c = Cache(d, k, N, n, max(lens) + 1, device, seed=G)
    q, q64 = queries(rng, (n, G, d), dtype, device)
    before = torch.rand(n, c.T, device=device)
    before[:, -1] = float("nan")  # behind the last token
    acc = before.clone()
    out = run_accum(c, q, lens, acc)
    before[:, -1], acc_end = 0, acc[:, -1].clone()
    assert bool(acc_end.isnan().all())
    acc[:, -1] = 0
    check_accum(c, q64, out, before, acc, lens)


def test_accum_bad_lengths_and_repeats(device):
    rng = np.random.default_rng(13)
    lens = [30, -1, 65, 64]
    c = Cache(64, 4, 256, 4, 64, device)
    q, q64 = queries(rng, (4, 2, 64), torch.float32, device)
    before = torch.rand(4, 64, device=device)
    acc = before.clone()
    out = run_accum(c, q, lens, acc)
    assert bool(out[1:3].isnan().all()) and torch.equal(acc[1:3], before[1:3])
    check_accum(c, q64, out, before, acc, lens, groups=(0, 3))
    again = before.clone()
    assert torch.equal(run_accum(c, q, lens, again)[[0, 3]], out[[0, 3]]) and torch.equal(again, acc)
    # every step adds one weight per head in all
    total = (acc - before)[[0, 3]].double().sum(1).cpu().numpy()
    assert np.all(np.abs(total - 2) <= 2 * 2.0**-18 + 64 * 2.0**-24)


# ------------------------------------------------------------------ accept --
def accept_ref(c, lens, M, path, n_acc):
    rows, new = [a.copy() for a in c.np], []
    for g in range(c.n):
        L, n = lens[g], n_acc[g]
        if not (0 <= L <= c.T - M and 0 <= n <= min(path.shape[1], M)
                and all(0 <= p < M for p in path[g, :max(n, 0)])):
            new.append(-1)
            continue
        for a, old in zip(rows, c.np):
            a[g, L:L + n] = old[g, [L + p for p in path[g, :n]]]
        new.append(L + n)
    return rows, new


@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 2), (64, 4, 512), (128, 1, 16384),
                                   (64, 64, 2), (64, 32, 16384)], ids=str)
@pytest.mark.parametrize("in_place", [False, True])
def test_accept(device, d, k, N, in_place):
    rng = np.random.default_rng(14)
    M, A = 9, 6
    lens = [20, 0, 55, 56, -1, 3, 4, 5, 6, 7]
    n = len(lens)
    c = Cache(d, k, N, n, 64, device)
    path = np.sort(rng.permuted(np.tile(np.arange(M), (n, 1)), axis=1)[:, :A], axis=1)
    path[5] = [8, 8, 0, 1, 0, 3]          # any order, repeats
    path[6, 4:] = 99                      # behind the accepted ones: not looked at
    path[7, 2], path[8, 0] = 9, -1        # bad entries
    n_acc = np.array([6, 3, 6, 2, 1, 6, 4, 4, 1, 7])
    rows, new = accept_ref(c, lens, M, path, n_acc)
    ld = torch.tensor(lens, dtype=torch.int32, device=device)
    got = fq.accept_draft(*c.dev, ld, M, torch.from_numpy(path).int().to(device),
                          torch.from_numpy(n_acc).int().to(device), ld if in_place else None)
    assert (got.data_ptr() == ld.data_ptr()) == in_place
    assert got.tolist() == new and new[3] == new[4] == new[7] == new[8] == new[9] == -1
    for a, b in zip(rows, c.dev):
        assert np.array_equal(a, b.cpu().numpy().view(a.dtype))


def test_accept_whole_tree(device):
    c = Cache(64, 2, 64, 3, 100, device)
    path = np.stack([np.arange(64)[::-1], np.arange(64), np.full(64, 63)])
    rows, new = accept_ref(c, [36, 0, 10], 64, path, [64, 64, 64])
    got = fq.accept_draft(*c.dev, torch.tensor([36, 0, 10], dtype=torch.int32, device=device), 64,
                          torch.from_numpy(path.copy()).int().to(device),
                          torch.full((3,), 64, dtype=torch.int32, device=device))
    assert got.tolist() == new == [100, 64, 74]
    for a, b in zip(rows, c.dev):
        assert np.array_equal(a, b.cpu().numpy().view(a.dtype))


# ------------------------------------------------------------------- evict --
def check_evict(c, acc, lens, keep, recent, got, T_out, before=None):
    kept = [osv.kept(acc[g], lens[g], keep, recent) if 0 <= lens[g] <= c.T else None
            for g in range(c.n)]
    assert got[5].tolist() == [-1 if x is None else len(x) for x in kept]
    index = got[6].cpu().numpy()
    for g, x in enumerate(kept):
        x = x or []
        assert index[g].tolist() == x + [-1] * (keep - len(x)), g
        for i, a in enumerate(c.np + [acc]):
            o = got[i].cpu().numpy().view(a.dtype)[g]
            assert o.shape[0] == T_out and np.array_equal(o[:len(x)], a[g, x], equal_nan=a.dtype.kind == "f")
            if before is not None:
                assert np.array_equal(o[len(x):], before[i].cpu().numpy().view(a.dtype)[g, len(x):])


def evict_out(c, keep, T_out, device):
    P = c.np[0].shape[2]
    mk = lambda dt, *s: torch.full(s, 77, dtype=dt, device=device)
    return (mk(torch.uint8, c.n, T_out, P), mk(torch.int16, c.n, T_out), mk(torch.uint8, c.n, T_out, P),
            mk(torch.int16, c.n, T_out), mk(torch.float32, c.n, T_out), mk(torch.int32, c.n),
            mk(torch.int32, c.n, keep))


def accumulators(rng, shape):
    acc = np.exp(rng.standard_normal(shape) * 1.5).astype(np.float32)
    acc[rng.random(shape) < 0.1] = 0.0
    acc[rng.random(shape) < 0.05] = -0.0
    acc[rng.random(shape) < 0.3] = np.float32(0.75)  # many equals
    return acc


@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 1, 2), (64, 4, 512), (128, 1, 16384),
                                   (64, 64, 2)], ids=str)
@pytest.mark.parametrize("keep,recent,extra", [(40, 7, 5), (1, 0, 0), (1, 1, 0), (64, 64, 0), (100, 3, 1),
                                               (300, 10, 0)], ids=str)
def test_evict(device, d, k, N, keep, recent, extra):
    rng = np.random.default_rng(keep)
    lens = [200, 0, 1, keep, keep + 1, 199, -1, 201]
    lens = [min(x, 201) for x in lens]
    c = Cache(d, k, N, 8, 200, device)
    acc = accumulators(rng, (8, 200))
    out = evict_out(c, keep, keep + extra, device)
    before = [o.clone() for o in out]
    got = fq.evict(*c.dev, torch.from_numpy(acc).to(device),
                   torch.tensor(lens, dtype=torch.int32, device=device), keep, recent, out=out)
    assert got is out or all(a is b for a, b in zip(got, out))
    check_evict(c, acc, lens, keep, recent, got, keep + extra, before)


@pytest.mark.parametrize("T,keep,recent", [(5000, 2500, 64), (5000, 4999, 0), (5000, 1, 0), (70001, 33000, 1)], ids=str)
@pytest.mark.parametrize("law", ["tail", "same", "nan", "signs"])
def test_evict_long(device, T, keep, recent, law):
    """Lengths above one pass of a workgroup; all equal, NaN, infinite and negative accumulators."""
    rng = np.random.default_rng(T)
    lens = [T, T - 3]
    c = Cache(64, 8, 16, 2, T, device)
    acc = accumulators(rng, (2, T))
    if law == "same":
        acc[:] = 1.5
    elif law == "nan":
        acc[rng.random(acc.shape) < 0.5] = np.nan
        acc[rng.random(acc.shape) < 0.1] = -np.inf
    elif law == "signs":
        acc = (rng.standard_normal((2, T)) * 10.0 ** rng.integers(-40, 38, (2, T))).astype(np.float32)
        acc[:, ::97] = np.inf
    got = fq.evict(*c.dev, torch.from_numpy(acc).to(device),
                   torch.tensor(lens, dtype=torch.int32, device=device), keep, recent)
    check_evict(c, acc, lens, keep, recent, got, keep)


@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (7000, 7000), (7000, 0), (45000, 100)], ids=str)
def test_evict_sliced_lengths(device, keep, recent):
    """A cache of many rows whose groups are empty, short, bad, or end inside a slice."""
    rng = np.random.default_rng(23)
    T = 50000
    lens = [0, 1, keep, min(keep + 1, T), 8192, 8193, 40960, T, -1, T + 1]
    c = Cache(64, 64, 2, len(lens), T, device)
    acc = accumulators(rng, (len(lens), T))
    acc[:, 8190:8195] = 1e9  # equals across a slice's end
    out = evict_out(c, keep, keep, device)
    before = [o.clone() for o in out]
    got = fq.evict(*c.dev, torch.from_numpy(acc).to(device),
                   torch.tensor(lens, dtype=torch.int32, device=device), keep, recent, out=out)
    check_evict(c, acc, lens, keep, recent, got, keep, before)


def test_evict_refuses_overlap(device):
    c = Cache(64, 8, 16, 1, 64, device)
    acc = torch.zeros(1, 64, device=device)
    lens = torch.tensor([64], dtype=torch.int32, device=device)
    out = list(evict_out(c, 32, 32, device))
    out[4] = acc[:, 32:]
    with pytest.raises(ValueError, match="acc_out overlaps acc"):
        fq.evict(*c.dev, acc, lens, 32, 4, out=out)
    out[4], out[5] = torch.zeros(1, 32, device=device), lens
    with pytest.raises(ValueError, match="new_lens overlaps lens"):
        fq.evict(*c.dev, acc, lens, 32, 4, out=out)


# ---------------------------------------------------------------- together --
def serving_step(c, bufs, q_tree, masks, path, n_acc, q, acc, lens, keep, recent, out):
    """Verification, acceptance, one accumulating decode step and eviction, as a serving loop runs them."""
    o1 = fq.attn_tree(q_tree, *bufs, lens, masks, c.k, c.N, c.Rd, c.Cd)
    new = fq.accept_draft(*bufs, lens, q_tree.shape[1], path, n_acc)
    o2 = fq.attn_decode_accum(q, *bufs, new, acc, c.k, c.N, c.Rd, c.Cd)
    ev = fq.evict(*bufs, acc, new, keep, recent, out=out)
    o3 = fq.attn_tree(q[:, None], *ev[:4], ev[5] - 1, torch.ones(1, dtype=torch.int64, device=q.device),
                      c.k, c.N, c.Rd, c.Cd)
    return o1, new, o2, ev, o3


def step_inputs(c, rng, M, G, A, device):
    q_tree, qt64 = queries(rng, (c.n, M, G, c.d), torch.bfloat16, device)
    q, q64 = queries(rng, (c.n, G, c.d), torch.bfloat16, device)
    path = torch.arange(A, device=device).int().mul(2).expand(c.n, A).contiguous()
    return q_tree, qt64, q, q64, path


def test_serving_step(device):
    """The operators in sequence, on drafted rows that the encoder wrote, against the references."""
    rng = np.random.default_rng(15)
    d, k, N, n, T, M, G, A = 64, 4, 256, 5, 260, 8, 4, 3
    lens = [200, 0, 31, 252, 100]
    c = Cache(d, k, N, n, T, device)
    x = torch.from_numpy(rng.standard_normal((2, n * M, d)).astype(np.float32)).to(device)
    for i in range(2):  # the drafted tokens' K and V rows are encoded into place
        pay, nrm = fq.encode(x[i], k, N, c.Rd, c.Cd)
        for g, L in enumerate(lens):
            for j, a in ((2 * i, pay), (2 * i + 1, nrm)):
                c.dev[j][g, L:L + M] = a[g * M:(g + 1) * M]
                c.np[j][g, L:L + M] = a[g * M:(g + 1) * M].cpu().numpy().view(c.np[j].dtype)
    q_tree, qt64, q, q64, path = step_inputs(c, rng, M, G, A, device)
    masks = fq.tree_masks([-1, 0, 0, 1, 2, 3, 4, 5])
    n_acc = [3, 2, 0, 3, 1]
    acc = torch.rand(n, T, device=device)
    before, keep, recent = acc.clone(), 64, 8
    o1, new, o2, ev, o3 = serving_step(
        c, c.dev, q_tree, torch.from_numpy(masks).to(device), path,
        torch.tensor(n_acc, dtype=torch.int32, device=device), q, acc,
        torch.tensor(lens, dtype=torch.int32, device=device), keep, recent, None)
    check_tree(c, q_tree, qt64, o1, lens, masks)
    c.np, want = accept_ref(c, lens, M, path.cpu().numpy(), n_acc)
    assert new.tolist() == want
    check_accum(c, q64, o2, before, acc, want)
    check_evict(c, acc.cpu().numpy(), want, keep, recent, ev, keep)
    for g, L in enumerate(ev[5].tolist()):
        if L == 0:
            assert bool(o3[g].isnan().all())  # length -1: nothing before the drafted token
            continue
        at = ev[6][g, :L].cpu().numpy()
        K, V = c.decoded(g, T, 0)[at], c.decoded(g, T, 1)[at]
        close(o3[g, 0].double().cpu().numpy(), q64[g], K, V, np.ones((G, L), dtype=bool))


def test_captured_step_follows_the_lengths(device):
    """One captured step, replayed on other lengths, counts and queries, with eager
    work between the replays, gives what the eager calls give."""
    rng = np.random.default_rng(16)
    n, T, M, G, A = 6, 400, 8, 4, 4
    c = Cache(64, 8, 16, n, T, device)
    masks = torch.from_numpy(fq.tree_masks([-1, 0, 1, 1, 0, 4, 4, 6])).to(device)
    stat = dict(lens=torch.zeros(n, dtype=torch.int32, device=device),
                n_acc=torch.zeros(n, dtype=torch.int32, device=device),
                acc=torch.zeros(n, T, device=device))
    q_tree, _, q, _, path = step_inputs(c, rng, M, G, A, device)
    bufs = [x.clone() for x in c.dev]
    out = evict_out(c, 50, 50, device)
    args = (masks, path, stat["n_acc"], q, stat["acc"], stat["lens"], 50, 5, out)
    serving_step(c, bufs, q_tree, *args)  # (the first calls load the kernels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = serving_step(c, bufs, q_tree, *args)
    for r in range(4):
        lens = rng.integers(0, T - M + 1, n)
        stat["lens"].copy_(torch.from_numpy(lens))
        stat["n_acc"].copy_(torch.from_numpy(rng.integers(0, A + 1, n)))
        stat["acc"].copy_(torch.rand(n, T, device=device))
        q_tree.normal_()
        q.normal_()
        for b, x in zip(bufs, c.dev):
            b.copy_(x)
        for o in out:
            o.fill_(0)
        acc0 = stat["acc"].clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*captured[:3], *captured[3], captured[4], stat["acc"], *bufs)]
        stat["acc"].copy_(acc0)
        for b, x in zip(bufs, c.dev):
            b.copy_(x)
        out2 = [torch.zeros_like(o) for o in out]
        e = serving_step(c, bufs, q_tree, *args[:-1], out2)
        want = (*e[:3], *e[3], e[4], stat["acc"], *bufs)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.nan_to_num(nan=7.0) if a.is_floating_point() else a,
                               b.nan_to_num(nan=7.0) if b.is_floating_point() else b)


def test_two_streams_at_once(device):
    rng = np.random.default_rng(17)
    cs = [Cache(64, 4, 256, 3, 600, device, seed=s) for s in (1, 2)]
    ins = [queries(rng, (3, 9, 4, 64), torch.float16, device)[0] for _ in cs]
    masks = random_masks(rng, 9)
    alone = [run_tree(c, q, [500, 20, 591], masks) for c, q in zip(cs, ins)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(run_tree(cs[i], ins[i], [500, 20, 591], masks))
    torch.cuda.synchronize()
    for a, outs in zip(alone, got):
        assert all(torch.equal(a, o) for o in outs)


def test_offsets_beyond_32_bits(device):
    """Two groups 2^27 rows apart: the second one's rows start past 2^32 bits and bytes."""
    rng = np.random.default_rng(18)
    d, k, N, T, L, M, G = 64, 2, 64, 1 << 27, 75, 3, 2
    small = Cache(d, k, N, 2, L + M + 1, device)
    P = small.np[0].shape[2]
    pay = torch.empty(2, T, P, dtype=torch.uint8, device=device)
    nrm = torch.empty(2, T, dtype=torch.int16, device=device)
    assert T * P > 1 << 31
    cache = [pay, nrm, pay, nrm]
    small.np[2:], small.dev[2:] = small.np[:2], small.dev[:2]
    for a, b in zip(cache[:2], small.dev[:2]):
        a[:, :b.shape[1]] = b
    lens = torch.tensor([L, L], dtype=torch.int32, device=device)
    q, q64 = queries(rng, (2, M, G, d), torch.float32, device)
    masks = random_masks(rng, M)
    out = fq.attn_tree(q, *cache, lens, torch.from_numpy(masks).to(device), k, N, small.Rd, small.Cd)
    check_tree(small, q, q64, out, [L, L], masks)
    acc = torch.zeros(2, T, device=device)
    o = fq.attn_decode_accum(q[:, 0].contiguous(), *cache, lens, acc, k, N, small.Rd, small.Cd)
    check_accum(small, q64[:, 0], o, torch.zeros(2, small.T), acc[:, :small.T], [L, L])
    ev = fq.evict(*cache, acc, lens, 30, 4)
    check_evict(small, acc[:, :small.T].cpu().numpy(), [L, L], 30, 4, ev, 30)
    path = torch.tensor([[0, 2]] * 2, dtype=torch.int32, device=device)
    two = torch.tensor([2, 2], dtype=torch.int32, device=device)
    assert fq.accept_draft(pay, nrm, pay.clone(), nrm.clone(), lens, M, path, two).tolist() == [L + 2] * 2
    rows, _ = accept_ref(small, [L, L], M, path.cpu().numpy(), [2, 2])
    assert np.array_equal(pay[:, :small.T].cpu().numpy(), rows[0])


@pytest.mark.parametrize("n", [0, 700])
def test_many_and_no_groups(device, n):
    rng = np.random.default_rng(19)
    c = Cache(64, 8, 16, n, 33, device) if n else None
    if not n:
        e = lambda dt, *s: torch.empty(s, dtype=dt, device=device)
        R, C = torch.zeros(64, 64, device=device), torch.zeros(16, 8, device=device)
        cache = (e(torch.uint8, 0, 9, 4), e(torch.int16, 0, 9), e(torch.uint8, 0, 9, 4), e(torch.int16, 0, 9))
        lens = e(torch.int32, 0)
        assert fq.attn_tree(e(torch.float32, 0, 2, 2, 64), *cache, lens, e(torch.int64, 2), 8, 16, R, C).numel() == 0
        assert fq.attn_decode_accum(e(torch.float32, 0, 2, 64), *cache, lens, e(torch.float32, 0, 9), 8, 16, R,
                                    C).numel() == 0
        assert fq.accept_draft(*cache, lens, 2, e(torch.int32, 0, 2), lens).numel() == 0
        assert fq.evict(*cache, e(torch.float32, 0, 9), lens, 4, 1)[6].numel() == 0
        return
    lens = rng.integers(0, 31, n).tolist()
    q, q64 = queries(rng, (n, 3, 2, 64), torch.float32, device)
    masks = random_masks(rng, 3)
    check_tree(c, q, q64, run_tree(c, q, lens, masks), lens, masks)
    before = torch.rand(n, 33, device=device)
    acc = before.clone()
    check_accum(c, q64[:, 0], run_accum(c, q[:, 0].contiguous(), lens, acc), before, acc, lens)


def test_tensors_of_another_stream_and_kept_workspace(device):
    """Inputs made on another stream that the call's stream waits for; one workspace for calls in a row."""
    rng = np.random.default_rng(20)
    c = Cache(128, 8, 256, 2, 300, device)
    q, q64 = queries(rng, (2, 4, 4, 128), torch.bfloat16, device)
    masks = random_masks(rng, 4)
    ws = torch.empty(fq.attn_tree_workspace_bytes(2, 4, 4, 128, 8, 256) + 8, dtype=torch.uint8, device=device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = run_tree(c, q, [290, 3], masks, workspace=ws)
        b = run_tree(c, q, [100, 296], masks, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    check_tree(c, q, q64, a, [290, 3], masks)
    check_tree(c, q, q64, b, [100, 296], masks)


def test_cache_without_rows(device):
    """T_stride = 0: a length of 0 is an empty group, any other is bad."""
    e = lambda dt, *s: torch.empty(s, dtype=dt, device=device)
    cache = (e(torch.uint8, 2, 0, 4), e(torch.int16, 2, 0), e(torch.uint8, 2, 0, 4), e(torch.int16, 2, 0))
    R, C = torch.eye(64, device=device), torch.rand(16, 8, device=device)
    lens = torch.tensor([0, 1], dtype=torch.int32, device=device)
    q = torch.randn(2, 3, 64, device=device)
    o = fq.attn_decode_accum(q, *cache, lens, e(torch.float32, 2, 0), 8, 16, R, C)
    assert torch.count_nonzero(o[0]) == 0 and bool(o[1].isnan().all())
    o = fq.attn_tree(q[:, None], *cache, lens, torch.ones(1, dtype=torch.int64, device=device), 8, 16, R, C)
    assert bool(o.isnan().all())
    assert fq.evict(*cache, e(torch.float32, 2, 0), lens, 4, 1)[5].tolist() == [0, -1]


@pytest.mark.parametrize("k,N", [(8, 16), (1, 16)], ids=str)
def test_mostly_empty_groups(device, k, N):
    """Thousands of groups of which a few hold tokens, in runs of empty and bad ones."""
    rng = np.random.default_rng(24)
    n, T = 5000, 300
    lens = np.where(rng.random(n) < 0.5, 0, -1)
    some = [0, 1, 63, 64, 65, 2047, 4095, 4999]
    lens[some] = [299, 1, 300, 17, 256, 257, 32, 33]
    c = Cache(64, k, N, 1, T, device)
    cache = [x.expand(n, *x.shape[1:]).contiguous() for x in c.dev]
    c.np, c.n = [np.broadcast_to(a, (n, *a.shape[1:])) for a in c.np], n
    c.dev = cache
    q, q64 = queries(rng, (n, 2, 64), torch.float32, device)
    before = torch.zeros(n, T, device=device)
    acc = before.clone()
    out = run_accum(c, q, lens.tolist(), acc)
    check_accum(c, q64, out, before, acc, lens, groups=some)
    none = torch.from_numpy(lens == 0).to(device)
    bad = torch.from_numpy(lens < 0).to(device)
    assert torch.count_nonzero(out[none]) == 0 and bool(out[bad].isnan().all())
    assert torch.count_nonzero(acc[none | bad]) == 0
