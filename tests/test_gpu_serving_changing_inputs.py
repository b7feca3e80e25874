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
