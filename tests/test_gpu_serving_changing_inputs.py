"""Lengths and accumulators that another stream writes while a call runs: which of the
values a call takes is open, but it takes one, and stays inside its tensors."""
import numpy as np
import pytest
import torch

from test_gpu_serving import Cache, close, queries

import paper_2605_11478_amd as fq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [4, 12])
@pytest.mark.parametrize("k,N", [(4, 256), (1, 16)], ids=str)
def test_lengths_written_meanwhile(device, k, N, G):
    """Every group has the outputs of one of the two lengths, or of none, with a workspace that
    holds no numbers before the call."""
    rng = np.random.default_rng(51)
    n, L = 400, 37
    c = Cache(64, k, N, 1, 40, device)
    cache = [x.expand(n, *x.shape[1:]).contiguous() for x in c.dev]
    q, q64 = queries(rng, (1, G, 64), torch.float32, device)
    q = q.expand(n, G, 64).contiguous()
    lens = torch.zeros(n, dtype=torch.int32, device=device)
    acc = torch.zeros(n, 40, device=device)
    ws = torch.empty(fq.attn_decode_accum_workspace_bytes(n, G, 64, k, N), dtype=torch.uint8, device=device)
    outs, side = [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(12):
        ws.fill_(255)
        with torch.cuda.stream(side):
            for i in range(12):
                lens.fill_(L if i % 2 else -1)
        for _ in range(3):
            outs.append(fq.attn_decode_accum(q, *cache, lens, acc, k, N, c.Rd, c.Cd, workspace=ws))
    torch.cuda.synchronize()
    want = fq.attn_decode_accum(q, *cache, torch.full_like(lens, L), torch.zeros_like(acc), k, N, c.Rd, c.Cd)
    close(want[0].double().cpu().numpy(), q64[0], c.decoded(0, L, 0), c.decoded(0, L, 1), np.ones((G, L), dtype=bool))
    ref = want[0].double()
    for o in outs:
        bad = o.isnan().flatten(1).all(1)
        assert not bool(o[~bad].isnan().any())
        err = (o[~bad].double() - ref).abs()
        # (a group's range may be cut elsewhere: two float32 results of one row)
        assert err.numel() == 0 or bool((err <= 2.0**-16 * ref.norm(dim=-1, keepdim=True)).all())
    assert bool(acc.isfinite().all()) and torch.count_nonzero(acc[:, L:]) == 0


def test_evict_inputs_written_meanwhile(device):
    """A cache in slices whose accumulators and lengths change between the passes, and index
    places that hold large numbers before the call: rows come from the old cache or stay."""
    rng = np.random.default_rng(52)
    n, T, keep = 4, 40000, 9000
    c = Cache(64, 8, 16, n, T, device)
    laws = [torch.from_numpy(rng.random((n, T)).astype(np.float32) * s).to(device) for s in (1, -1, 1e-20)]
    acc = laws[0].clone()
    lens = torch.full((n,), T, dtype=torch.int32, device=device)
    out = [torch.zeros(n, keep, *x.shape[2:], dtype=x.dtype, device=device) for x in c.dev]
    out += [torch.zeros(n, keep, device=device), lens.clone(), torch.zeros(n, keep, dtype=torch.int32, device=device)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for r in range(8):
        out[6].fill_(2**31 - 1 - r)
        for o in out[:5]:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for i in range(16):
                acc.copy_(laws[i % 3])
                lens.fill_((T, keep + 1, -1, T + 1)[i % 4])
        fq.evict(*c.dev, acc, lens, keep, 100, out=out)
        torch.cuda.synchronize()
        index = out[6].long()
        live = (index >= 0) & (index < T)
        assert bool(((index == -1) | live | (index == 2**31 - 1 - r)).all())
        at = index.clamp(0, T - 1)
        for x, o in zip(c.dev, out):
            rows = x.gather(1, at[:, :, None].expand(-1, -1, x.shape[2]) if x.dim() == 3 else at)
            keepers = live[:, :, None] if x.dim() == 3 else live
            assert torch.equal(torch.where(keepers, rows, torch.zeros_like(rows)), o)
