"""Requests that no page was left for, and what they hold."""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from oracle import paged as opg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
def test_refused_requests_keep_what_they_hold(device, captured):
    """With new lengths in a tensor of their own, a request that was refused grows when pages
    are free again, and gives its own back: no page is lost."""
    page, n_pages, n = 16, 10, 4
    table, lens = np.full((n, 8), -1, np.int32), np.zeros(n, np.int32)
    free, left = np.arange(n_pages, dtype=np.int32), n_pages
    # 10 pages; the third step asks for more than there are, the fourth frees some, the last all
    steps = [[40, 30, 20, 16], [9, 3, 1, 0], [60, 0, 40, 16], [1, -33, 30, 1], [0, 0, 20, 16], None]
    most = 200
    t = lambda a, ty=torch.int32: torch.tensor(np.asarray(a), dtype=ty, device=device)
    td, ld, fd, nd, gd = t(table), t(lens), t(free), t([left]), t(np.zeros(n))
    out = (t(np.zeros(n)), t(np.zeros(n + 1)), t(np.zeros(most), torch.int64), t(np.zeros(most)), nd)
    ws = torch.empty(max(1, fq.page_resize_workspace_bytes(n)), dtype=torch.uint8, device=device)

    def step():
        fq.page_resize(td, ld, gd, page, n_pages, fd, nd, most, out=out, workspace=ws)
        ld.copy_(torch.where(out[0] < 0, ld, out[0]))

    run = step
    if captured:
        step()  # (nothing grows yet)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    refused = 0
    for grow in steps:
        grow = (-lens if grow is None else np.array(grow)).astype(np.int32)
        gd.copy_(torch.from_numpy(grow))
        run()
        torch.cuda.synchronize()
        table, free, new, starts, slots, positions, left = opg.resize(table, lens, grow, page, n_pages, free, left,
                                                                      most)
        assert np.array_equal(out[0].cpu().numpy(), new) and np.array_equal(out[2].cpu().numpy(), slots)
        refused += int((new < 0).sum())
        lens = np.where(new < 0, lens, new).astype(np.int32)
        assert np.array_equal(ld.cpu().numpy(), lens) and int(nd) == left
        held = [int(p) for g in range(n) for p in td.cpu().numpy()[g, :-(-int(lens[g]) // page)]]
        assert sorted(held + fd.cpu().numpy()[:left].tolist()) == list(range(n_pages))
    assert refused > 0 and left == n_pages
