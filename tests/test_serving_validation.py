"""The serving operators on the CPU: ancestor masks, and the refusals of the
binding and of the C ABI, none of which reaches a kernel."""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq
from oracle import serving as osv

d, k, N, P = 64, 8, 16, 4
QUERIES = {"fibq_payload_bytes", "fibq_strerror", "fibq_attn_tree_workspace_bytes",
           "fibq_attn_decode_accum_workspace_bytes", "fibq_evict_workspace_bytes"}


class _NoLaunch:
    def __init__(self, real):
        self._real = real

    def __getattr__(self, name):
        if name in QUERIES:
            return getattr(self._real, name)
        raise AssertionError(f"{name} was called: the binding let a bad argument through")


@pytest.fixture
def nolaunch(monkeypatch):
    monkeypatch.setattr(fq, "_lib", _NoLaunch(fq.lib()))


def _cache(n=2, T=32):
    pay, nrm = torch.zeros((n, T, P), dtype=torch.uint8), torch.zeros((n, T), dtype=torch.int16)
    return [pay, nrm, pay.clone(), nrm.clone()]


def _rc():
    return torch.zeros((d, d)), torch.zeros((N, k))


def _err(fn, match, exc=ValueError):
    with pytest.raises(exc, match=match):
        fn()


def test_tree_masks():
    assert fq.tree_masks([-1]).tolist() == [1]
    assert fq.tree_masks([-1, 0, 0, 2, -1]).tolist() == [1, 3, 5, 13, 16]
    chain = fq.tree_masks(np.arange(64) - 1)
    assert chain.dtype == np.int64 and chain[62] == 2 ** 63 - 1 and chain[63] == -1
    seen = osv.seen_by_tree(3, chain, 64)
    assert np.array_equal(seen[:, 3:], np.tri(64, dtype=bool)) and seen[:, :3].all()
    for bad in ([0], [-1, 1], [-2], [-1, 5], [], np.arange(65) - 1):
        with pytest.raises(fq.FibqError):
            fq.tree_masks(bad)
    _err(lambda: fq.tree_masks([[-1]]), "one-dimensional")


def test_attn_tree_rejects(nolaunch):
    R, C = _rc()
    cache, lens, masks = _cache(), torch.zeros(2, dtype=torch.int32), torch.ones(3, dtype=torch.int64)
    q = torch.zeros((2, 3, 4, d))

    def call(q=q, cache=cache, lens=lens, masks=masks, R=R, C=C, **kw):
        return fq.attn_tree(q, *cache, lens, masks, k, N, R, C, **kw)

    _err(call, "must be a device tensor")
    _err(lambda: call(q=q[0]), "q must have shape")
    _err(lambda: call(q=q.double()), "q must have dtype")
    _err(lambda: call(q=q.transpose(1, 2)), "q must be contiguous")
    _err(lambda: call(q=q[:1]), "lens must have shape")
    _err(lambda: call(cache=[c[:, :, :3] if c.dim() == 3 else c for c in cache]), "k_payload must have shape")
    _err(lambda: call(cache=cache[:3] + [cache[3][:, :31]]), "v_norms must have shape")
    _err(lambda: call(lens=lens.long()), "lens must have dtype")
    _err(lambda: call(lens=torch.zeros(3, dtype=torch.int32)), "lens must have shape")
    _err(lambda: call(masks=masks.int()), "masks must have dtype")
    _err(lambda: call(masks=masks[:2]), "masks must have shape")
    _err(lambda: call(masks=masks.expand(2, 3)), "masks must be contiguous")
    _err(lambda: call(masks=[1, 1, 1]), "masks must be a torch tensor", TypeError)
    _err(lambda: call(R=R.double()), "R must have dtype")
    _err(lambda: call(C=C[:8]), "C must have shape")
    _err(lambda: call(out=torch.zeros((2, 3, 4, 32))), "out must have shape")
    _err(lambda: call(workspace=torch.zeros(4)), "workspace must have dtype")


def test_attn_decode_accum_rejects(nolaunch):
    R, C = _rc()
    cache, lens = _cache(), torch.zeros(2, dtype=torch.int32)
    q, acc = torch.zeros((2, 4, d)), torch.zeros((2, 32))

    def call(q=q, lens=lens, acc=acc, **kw):
        return fq.attn_decode_accum(q, *cache, lens, acc, k, N, R, C, **kw)

    _err(call, "must be a device tensor")
    _err(lambda: call(q=q[None]), "q must have shape")
    _err(lambda: call(acc=acc.half()), "acc must have dtype")
    _err(lambda: call(acc=acc[:, :31]), "acc must have shape")
    _err(lambda: call(acc=acc.t().contiguous().t()), "acc must be contiguous")
    _err(lambda: call(lens=lens[:1]), "lens must have shape")
    _err(lambda: call(out=torch.zeros((2, 4, d), dtype=torch.float16)), "out must have dtype")


def test_accept_draft_rejects(nolaunch):
    cache, lens = _cache(), torch.zeros(2, dtype=torch.int32)
    path, n = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    _err(lambda: fq.accept_draft(*cache, lens, 4, path, n), "must be a device tensor")
    _err(lambda: fq.accept_draft(*cache, lens, 4, path.long(), n), "path must have dtype")
    _err(lambda: fq.accept_draft(*cache, lens, 4, path[:1], n), "path must have shape")
    _err(lambda: fq.accept_draft(*cache, lens, 4, path, n[:1]), "n_acc must have shape")
    _err(lambda: fq.accept_draft(*cache, lens, 4, path, n, lens.long()), "new_lens must have dtype")


def test_evict_rejects(nolaunch):
    cache, lens, acc = _cache(), torch.zeros(2, dtype=torch.int32), torch.zeros((2, 32))
    _err(lambda: fq.evict(*cache, acc, lens, 8, 2), "must be a device tensor")
    _err(lambda: fq.evict(*cache, acc, lens, 0, 0), "keep = 0")
    _err(lambda: fq.evict(*cache, acc.double(), lens, 8, 2), "acc must have dtype")
    small = _cache(2, 4) + [torch.zeros((2, 4)), lens.clone(), torch.zeros((2, 8), dtype=torch.int32)]
    _err(lambda: fq.evict(*cache, acc, lens, 9, 2, out=small), "index must have shape")
    _err(lambda: fq.evict(*cache, acc, lens, 8, 2, out=small[:6]), "seven tensors")
    small[2] = small[2][:, :3]
    _err(lambda: fq.evict(*cache, acc, lens, 8, 2, out=small), "v_payload must have shape")


def _tree(**kw):
    """Status of fibq_attn_tree for addresses that no valid call would reach."""
    a = dict(q=256, q_dtype=0, kp=256, kn=256, vp=256, vn=256, lens=256, masks=256, ms=0, n=2, M=3,
             G=4, T=32, d=d, k=k, b=0.5, N=N, R=256, C=256, scale=0.0, out=256, ws=256, wsb=1 << 40)
    a.update(kw)
    return fq.lib().fibq_attn_tree(*a.values(), None)


def _accum(**kw):
    a = dict(q=256, q_dtype=0, kp=256, kn=256, vp=256, vn=256, lens=256, acc=256, n=2, G=4, T=32,
             d=d, k=k, b=0.5, N=N, R=256, C=256, scale=0.0, out=256, ws=256, wsb=1 << 40)
    a.update(kw)
    return fq.lib().fibq_attn_decode_accum(*a.values(), None)


COMMON = [dict(q=None), dict(q_dtype=3), dict(kp=None), dict(vn=None), dict(lens=None), dict(n=-1),
          dict(n=65536), dict(G=0), dict(G=17), dict(T=-1), dict(T=1 << 30), dict(d=63),
          dict(b=0.25), dict(N=15), dict(R=None), dict(C=None), dict(out=None),
          dict(scale=float("nan")), dict(scale=float("inf"))]


@pytest.mark.parametrize("kw", COMMON + [dict(M=0), dict(M=65), dict(ms=2), dict(ms=-3),
                                         dict(masks=None)], ids=str)
def test_attn_tree_status(kw):
    assert _tree(**kw) == fq.FIBQ_EINVAL


@pytest.mark.parametrize("kw", COMMON + [dict(acc=None)], ids=str)
def test_attn_decode_accum_status(kw):
    assert _accum(**kw) == fq.FIBQ_EINVAL


@pytest.mark.parametrize("call", [_tree, _accum])
def test_attention_unsupported_empty_and_workspace(call):
    assert call(d=192, k=8, b=0.5) == fq.FIBQ_EUNSUPPORTED
    assert call(n=0, q=None, kp=None) == fq.FIBQ_OK
    need = (fq.attn_tree_workspace_bytes(2, 3, 4, d, k, N) if call is _tree
            else fq.attn_decode_accum_workspace_bytes(2, 4, d, k, N))
    if need:
        assert call(ws=None) == fq.FIBQ_EWORKSPACE
        assert call(wsb=need - 1) == fq.FIBQ_EWORKSPACE
        assert call(ws=256 + 16) == fq.FIBQ_EWORKSPACE


def test_workspace_queries_of_invalid_problems():
    assert fq.attn_tree_workspace_bytes(2, 0, 4, d, k, N) == 0
    assert fq.attn_tree_workspace_bytes(2, 65, 4, d, k, N) == 0
    assert fq.attn_tree_workspace_bytes(-1, 3, 4, d, k, N) == 0
    assert fq.attn_decode_accum_workspace_bytes(2, 17, d, k, N) == 0
    assert fq.attn_decode_accum_workspace_bytes(2, 4, 96, k, N) == 0
    assert fq.evict_workspace_bytes(-1, 4) == 0


@pytest.mark.parametrize("kw", [dict(n=-1), dict(n=65536), dict(T=1 << 30), dict(P=0), dict(P=257),
                                dict(M=0), dict(M=65), dict(A=0), dict(A=65), dict(path=None),
                                dict(n_acc=None), dict(new=None), dict(kp=None)], ids=str)
def test_accept_draft_status(kw):
    a = dict(kp=256, kn=256, vp=256, vn=256, lens=256, n=2, T=32, P=P, M=4, path=256, A=3,
             n_acc=256, new=256)
    assert fq.lib().fibq_accept_draft(*{**a, **kw}.values(), None) == fq.FIBQ_EINVAL


@pytest.mark.parametrize("kw", [dict(n=-1), dict(n=65536), dict(T=-1), dict(P=0), dict(keep=0),
                                dict(keep=1 << 30), dict(recent=-1), dict(recent=9),
                                dict(T_out=7), dict(kp=None), dict(acc=None), dict(lens=None),
                                dict(kpo=None), dict(index=None), dict(kpo=256), dict(new=1280),
                                dict(acco=1024)], ids=str)
def test_evict_status(kw):
    a = dict(kp=256, kn=512, vp=768, vn=768 + 64, acc=1024, lens=1280, n=2, T=32, P=P, keep=8,
             recent=2, T_out=8, kpo=4096, kno=4352, vpo=4608, vno=4864, acco=5120, new=5376,
             index=5632, ws=8192, wsb=1 << 40)
    assert fq.lib().fibq_evict(*{**a, **kw}.values(), None) == fq.FIBQ_EINVAL


def test_no_groups_is_a_no_op():
    L = fq.lib()
    null = [None] * 5
    assert L.fibq_accept_draft(*null, 0, 32, P, 4, None, 3, None, None, None) == fq.FIBQ_OK
    assert L.fibq_evict(*null, None, 0, 32, P, 8, 2, 8, *null, None, None, None, 0, None) == fq.FIBQ_OK
