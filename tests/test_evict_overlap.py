"""Outputs of the eviction that share memory with each other are refused."""
import pytest
import torch

import paper_2605_11478_amd as fq

ADDRESSES = dict(kpo=4096, kno=4352, vpo=4608, vno=4864, acco=5120, new=5376, index=5632)


@pytest.mark.parametrize("a,b", [("kpo", "vpo"), ("kno", "vno"), ("new", "index"), ("kpo", "index"),
                                 ("acco", "vno")])
def test_status_of_shared_output_addresses(a, b):
    to = dict(ADDRESSES)
    to[b] = to[a]
    args = dict(kp=256, kn=512, vp=768, vn=832, acc=1024, lens=1280, n=2, T=32, P=4, keep=8, recent=2,
                T_out=8, **to, ws=8192, wsb=1 << 40)
    assert fq.lib().fibq_evict(*args.values(), None) == fq.FIBQ_EINVAL


@pytest.mark.gpu
def test_refusal_of_shared_outputs(device):
    n, T, P, keep = 2, 64, 4, 16
    z = lambda dt, *s: torch.zeros(s, dtype=dt, device=device)
    cache = [z(torch.uint8, n, T, P), z(torch.int16, n, T), z(torch.uint8, n, T, P), z(torch.int16, n, T)]
    acc, lens = torch.rand(n, T, device=device), torch.full((n,), T, dtype=torch.int32, device=device)
    norms = z(torch.int16, 3 * n * keep)

    def outs(**kw):
        o = dict(kp=z(torch.uint8, n, keep, P), kn=z(torch.int16, n, keep), vp=z(torch.uint8, n, keep, P),
                 vn=z(torch.int16, n, keep), acc=z(torch.float32, n, keep), lens=z(torch.int32, n),
                 index=z(torch.int32, n, keep))
        return tuple({**o, **kw}.values())

    half = norms[n * keep // 2:][:n * keep].view(n, keep)
    first = norms[:n * keep].view(n, keep)
    one = z(torch.uint8, n, keep, P)
    for kw, match in ((dict(kp=one, vp=one), "v_payload_out overlaps k_payload_out"),
                      (dict(kn=first, vn=half), "v_norms_out overlaps k_norms_out")):
        with pytest.raises(ValueError, match=match):
            fq.evict(*cache, acc, lens, keep, 4, out=outs(**kw))
    # parts of one tensor that do not overlap are fine
    second = norms[n * keep:2 * n * keep].view(n, keep)
    got = fq.evict(*cache, acc, lens, keep, 4, out=outs(kn=first, vn=second))
    assert got[5].tolist() == [keep] * n
