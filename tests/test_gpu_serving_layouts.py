"""The serving operators on tensors that begin at any element, and at the largest number
of groups: the results of aligned tensors, bit by bit, and of the references."""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from test_gpu_serving import Cache, close, queries, random_masks

pytestmark = pytest.mark.gpu


def shifted(t):
    """The same values, beginning one element into an allocation."""
    y = torch.zeros(t.numel() + 1, dtype=t.dtype, device=t.device)[1:]
    y.copy_(t.flatten())
    return y.view(t.shape)


@pytest.mark.parametrize("M,G,dtype", [(2, 3, torch.float16), (3, 4, torch.bfloat16), (6, 6, torch.float32)], ids=str)
@pytest.mark.parametrize("d,k,N", [(64, 4, 256), (64, 8, 16), (64, 2, 64), (64, 1, 16), (64, 16, 4), (128, 4, 4096),
                                   (128, 16, 64)], ids=str)
def test_tensors_at_any_element(device, d, k, N, M, G, dtype):
    rng = np.random.default_rng(61)
    n, T, L = 3, 101, 90
    c = Cache(d, k, N, n, T, device)
    q, _ = queries(rng, (n, M, G, d), dtype, device)
    masks = torch.from_numpy(random_masks(rng, M)).to(device)
    lens = torch.tensor([L, 3, T - M], dtype=torch.int32, device=device)
    path = torch.tensor([[1, 0]] * n, dtype=torch.int32, device=device)
    n_acc = torch.tensor([2, 1, 0], dtype=torch.int32, device=device)
    acc0 = torch.rand(n, T, device=device)
    P = c.dev[0].shape[2]

    def step(s):
        cache, acc = [s(x.clone()) for x in c.dev], s(acc0.clone())
        R, C = s(c.Rd), s(c.Cd)
        e = lambda dt, *z: s(torch.zeros(z, dtype=dt, device=device))
        o1 = fq.attn_tree(s(q), *cache, s(lens), s(masks), k, N, R, C, out=e(torch.float32, n, M, G, d))
        new = fq.accept_draft(*cache, s(lens), M, s(path), s(n_acc), new_lens=e(torch.int32, n))
        o2 = fq.attn_decode_accum(s(q[:, 0].contiguous()), *cache, new, acc, k, N, R, C)
        out = (e(torch.uint8, n, 40, P), e(torch.int16, n, 40), e(torch.uint8, n, 40, P), e(torch.int16, n, 40),
               e(torch.float32, n, 40), e(torch.int32, n), e(torch.int32, n, 40))
        return [o1, new, o2, acc, *cache, *fq.evict(*cache, acc, new, 40, 5, out=out)]

    for a, b in zip(step(lambda t: t), step(shifted)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("k,N", [(8, 16), (32, 2)], ids=str)
def test_most_groups(device, k, N):
    rng = np.random.default_rng(62)
    n, T, M, G = 65535, 5, 2, 2
    c = Cache(64, k, N, 5, T, device)
    cache = [x[torch.arange(n, device=device) % 5] for x in c.dev]
    rows = [[c.decoded(g, T, w) for w in (0, 1)] for g in range(5)]
    lens = torch.arange(n, dtype=torch.int32, device=device) % 7 - 1  # -1, 0 .. 5
    q, q64 = queries(rng, (n, M, G, 64), torch.float16, device)
    masks = torch.from_numpy(fq.tree_masks([-1, 0])).to(device)
    out = fq.attn_tree(q, *cache, lens, masks, k, N, c.Rd, c.Cd).double().cpu().numpy()
    acc = torch.zeros(n, T, device=device)
    o2 = fq.attn_decode_accum(q[:, 0].contiguous(), *cache, lens, acc, k, N, c.Rd, c.Cd).double().cpu().numpy()
    ls = lens.tolist()
    for g in [*range(14), 32767, 32768, *range(n - 14, n)]:
        L = ls[g]
        K, V = rows[g % 5]
        if 0 <= L <= T - M:
            seen = np.repeat(np.array([[1] * L + [1, 0], [1] * L + [1, 1]], dtype=bool), G, 0)
            close(out[g].reshape(M * G, 64), q64[g].reshape(M * G, 64), K[:L + M], V[:L + M], seen)
        else:
            assert np.isnan(out[g]).all()
        if L < 0:
            assert np.isnan(o2[g]).all()
        else:
            close(o2[g], q64[g, 0], K[:L], V[:L], np.ones((G, L), dtype=bool))
    # weights sum to one per head, each to 2^-17 of itself
    some = lens > 0
    assert bool(((acc[some].double().sum(1) - G).abs() <= G * 2.0**-16).all())
    assert torch.count_nonzero(acc[~some]) == 0
    got = fq.evict(*cache, acc, lens, 3, 1)
    assert got[5].tolist() == [x if x <= 3 else 3 for x in ls]
    new = fq.accept_draft(*cache, lens, M, torch.zeros(n, 1, dtype=torch.int32, device=device),
                          torch.ones(n, dtype=torch.int32, device=device))
    assert new.tolist() == [x + 1 if 0 <= x <= T - M else -1 for x in ls]
