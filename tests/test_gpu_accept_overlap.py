"""New lengths in memory that the acceptance reads for other groups are refused."""
import pytest
import torch

import paper_2605_11478_amd as fq

pytestmark = pytest.mark.gpu


def test_refusal_of_new_lengths_in_the_inputs(device):
    n, T, P = 6, 20, 4
    z = lambda dt, *s: torch.zeros(s, dtype=dt, device=device)
    cache = [z(torch.uint8, n, T, P), z(torch.int16, n, T), z(torch.uint8, n, T, P), z(torch.int16, n, T)]
    buf = torch.full((n + 1,), 7, dtype=torch.int32, device=device)
    path, n_acc = z(torch.int32, n, 2), torch.ones(n, dtype=torch.int32, device=device)
    with pytest.raises(ValueError, match="new_lens overlaps lens"):
        fq.accept_draft(*cache, buf[:n], 3, path, n_acc, new_lens=buf[1:])
    with pytest.raises(ValueError, match="new_lens overlaps path"):
        fq.accept_draft(*cache, buf[:n], 3, path, n_acc, new_lens=path.flatten()[:n])
    assert buf.tolist() == [7] * (n + 1) and path.count_nonzero() == 0
    got = fq.accept_draft(*cache, buf[:n], 3, path, n_acc, new_lens=buf[:n])
    assert got.tolist() == [8] * n and buf[n] == 7
    assert fq.accept_draft(*cache, buf[:n], 3, path, n_acc, new_lens=n_acc).tolist() == [9] * n
