"""The paged 8-bit cache on the CPU: frequencies of rotary positions, and the refusals
of the binding and of the C ABI, none of which reaches a kernel."""
import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq

QUERIES = {"fibq_strerror", "fibq_page_resize_workspace_bytes", "fibq_attn_cache8_workspace_bytes"}


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


def _err(fn, match, exc=ValueError):
    with pytest.raises(exc, match=match):
        fn()


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_rope_freqs():
    f = fq.rope_freqs(8)
    assert f.dtype == np.float64 and np.allclose(f, [1, 1e-1, 1e-2, 1e-3], rtol=1e-15)
    assert np.array_equal(fq.rope_freqs(8, scaling="linear", factor=4.0), f / 4)
    b = fq.rope_freqs(8, scaling="base", factor=4.0)  # the fastest stays, the slowest is 4 times slower
    assert b[0] == 1 and abs(b[3] * 4 / f[3] - 1) < 1e-12 and (np.diff(b / f) < 0).all()
    r = fq.rope_freqs(8, scaling="ramp", factor=4.0, trained=2000, low=1.0, high=32.0)
    # 318, 31.8, 3.18 and 0.318 turns over the trained positions
    w = np.clip((2000 * f / (2 * np.pi) - 1) / 31, 0, 1)
    assert r[0] == f[0] and r[3] == f[3] / 4 and np.allclose(r, f * (w + (1 - w) / 4), rtol=1e-15)
    for kw in (dict(rot=7), dict(rot=0), dict(rot=8, base=0.0), dict(rot=8, factor=-1.0),
               dict(rot=8, scaling="other"), dict(rot=8, scaling="ramp"), dict(rot=2, scaling="base"),
               dict(rot=8, scaling="ramp", trained=9, low=2.0, high=2.0)):
        with pytest.raises(ValueError):
            fq.rope_freqs(**kw)


def test_rope_rejects(nolaunch):
    q, k, pos = torch.zeros(5, 4, 16), torch.zeros(5, 2, 16), _i32(5)
    f = torch.zeros(4, dtype=torch.float64)

    def call(q=q, k=k, pos=pos, f=f, **kw):
        return fq.rope(q, k, pos, f, **kw)

    _err(call, "must be a device tensor")
    _err(lambda: call(layout="other"), "layout must be")
    _err(lambda: call(q=q[0]), "q must have shape")
    _err(lambda: call(q=q.double()), "q must have dtype")
    _err(lambda: call(q=q.transpose(1, 2)[:, :, :2]), "contiguous heads")
    _err(lambda: call(k=k.half()), "k must have dtype")
    _err(lambda: call(k=k[:4]), "k must have shape")
    _err(lambda: call(k=torch.zeros(5, 2, 18)), "k must have shape")
    _err(lambda: call(pos=pos.long()), "positions must have dtype")
    _err(lambda: call(pos=pos[:4]), "positions must have shape")
    _err(lambda: call(f=f.float()), "freqs must have dtype")
    _err(lambda: call(out=(q,)), "out must hold")
    _err(lambda: call(out=(q, None)), "out must hold")
    _err(lambda: call(out=(q, k.half())), "k out must have dtype")
    _err(lambda: call(out=(q[:, :1].expand(5, 4, 16), k)), "twice")


def test_rope_overlaps():
    """Which rows share memory."""
    buf = torch.zeros(5, 10, 16)
    q, k = buf[:, :4], buf[:, 4:6]
    assert fq._apart(q, k) and fq._apart(k, q) and fq._apart(buf[:, 9:], q)
    assert not fq._apart(q, buf[:, 3:5]) and not fq._apart(q, q) and not fq._apart(k, buf)
    assert fq._apart(buf[:2], buf[2:]) and not fq._apart(buf[:3, :4], buf[2:, :4])
    assert not fq._apart(buf.transpose(0, 1)[:5], buf[:, :4])


def _resize(**kw):
    a = dict(table=_i32(3, 4), lens=_i32(3), grow=_i32(3), page=16, n_pages=9, free=_i32(9),
             n_free=_i32(1), n_rows=7)
    out, ws = kw.pop("out", None), kw.pop("workspace", None)
    return fq.page_resize(*{**a, **kw}.values(), out=out, workspace=ws)


def test_page_resize_rejects(nolaunch):
    _err(_resize, "must be a device tensor")
    _err(lambda: _resize(table=_i32(3)), "table must have shape")
    _err(lambda: _resize(lens=_i32(2)), "lens must have shape")
    _err(lambda: _resize(grow=_i32(3).long()), "grow must have dtype")
    _err(lambda: _resize(free=_i32(9, 1)), "free must have shape")
    _err(lambda: _resize(n_free=_i32(2)), "n_free must have shape")
    _err(lambda: _resize(n_rows=-1), "n_rows = -1")
    _err(lambda: _resize(out=(_i32(3),)), "five tensors")
    _err(lambda: _resize(out=(_i32(3), _i32(4), _i32(7), _i32(7), _i32(1))), "slots must have dtype")
    _err(lambda: _resize(workspace=torch.zeros(4, dtype=torch.uint8)), "workspace holds 4")


def _pools(dtype=torch.int8, n_pages=9, H=2, page=16, d=64):
    return [torch.zeros((n_pages, H, page, d), dtype=dtype), torch.zeros(n_pages, H),
            torch.zeros((n_pages, H, page, d), dtype=dtype), torch.zeros(n_pages, H)]


def test_cache8_write_rejects(nolaunch):
    k, slots = torch.zeros(5, 2, 64), torch.zeros(5, dtype=torch.int64)
    call = lambda k=k, v=k, slots=slots, p=None: fq.cache8_write(k, v, slots, *(p or _pools()))
    _err(call, "must be a device tensor")
    _err(lambda: call(k=k.double()), "k must have dtype")
    _err(lambda: call(v=k.half()), "v must have dtype")
    _err(lambda: call(k=k[:, :1]), "k must have shape")
    _err(lambda: call(v=k[:4]), "v must have shape")
    _err(lambda: call(slots=slots.int()), "slots must have dtype")
    _err(lambda: call(slots=slots[:4]), "slots must have shape")
    _err(lambda: call(p=_pools(torch.uint8)), "k_pages must have dtype")
    bad = _pools()
    _err(lambda: call(p=bad[:2] + [bad[2][:8], bad[3]]), "v_pages must have shape")
    _err(lambda: call(p=bad[:1] + [bad[1].double()] + bad[2:]), "k_scales must have dtype")
    _err(lambda: call(p=[bad[0].transpose(1, 2).contiguous().transpose(1, 2)] + bad[1:]),
         "k_pages must be contiguous")


def test_attn_cache8_rejects(nolaunch):
    q = torch.zeros(3, 8, 64)

    def call(q=q, p=None, table=_i32(3, 4), lens=_i32(3), **kw):
        return fq.attn_cache8(q, *(p or _pools()), table, lens, **kw)

    _err(call, "must be a device tensor")
    _err(lambda: call(q=torch.zeros(3, 8, 32)), "q must have shape")
    _err(lambda: call(q=torch.zeros(3, 7, 64)), "7 heads")
    _err(lambda: call(q=q.transpose(0, 1)), "q must be contiguous")
    _err(lambda: call(q=torch.zeros(4, 8, 64)), "starts must be given")
    _err(lambda: call(starts=_i32(3)), "starts must have shape")
    _err(lambda: call(table=_i32(3, 4).long()), "table must have dtype")
    _err(lambda: call(lens=_i32(2)), "lens must have shape")
    _err(lambda: call(out=torch.zeros(3, 8, 64).half()), "out must have dtype")
    _err(lambda: call(workspace=torch.zeros(4)), "workspace must have dtype")


def _status(name, defaults, kw):
    return getattr(fq.lib(), name)(*{**defaults, **kw}.values(), None)


ROPE = dict(q=256, k=512, dtype=0, n=2, Hq=4, Hk=2, d=16, qr=64, qh=16, kr=32, kh=16, pos=1024,
            freqs=2048, rot=8, layout=0, scale=1.0, inverse=0, qo=4096, ko=8192, qor=64, qoh=16, kor=32,
            koh=16)


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(dtype=3), dict(n=-1), dict(n=1 << 31),
                                dict(Hq=0), dict(Hk=-1), dict(Hq=2000, Hk=49), dict(d=15), dict(d=514),
                                dict(rot=0), dict(rot=18), dict(rot=7), dict(layout=2), dict(pos=None),
                                dict(freqs=None), dict(qo=None), dict(ko=None), dict(qr=-1),
                                dict(qor=63), dict(koh=15, kor=16), dict(scale=float("nan")),
                                dict(qo=512), dict(ko=4096), dict(ko=256), dict(qo=256, qor=128)], ids=str)
def test_rope_status(kw):
    assert _status("fibq_rope", ROPE, kw) == fq.FIBQ_EINVAL


@pytest.mark.parametrize("kw", [dict(n=(1 << 24) + 1, qoh=15, qor=1 << 39),
                                dict(n=(1 << 24) + 1, koh=15, kor=1 << 39)], ids=str)
def test_rope_status_far_strides(kw):
    """An output that holds elements twice, whose extent is more than 64 bits take."""
    assert _status("fibq_rope", ROPE, kw) == fq.FIBQ_EINVAL


def test_rope_status_most_rows():
    """More workgroups than a grid holds are no valid problem."""
    for n in ((1 << 25) + 1, (1 << 26) + 1, 1 << 30):
        assert _status("fibq_rope", ROPE, dict(n=n)) == fq.FIBQ_EINVAL


RESIZE = dict(table=256, lens=512, grow=768, n=2, mp=4, page=16, n_pages=9, free=1024, cap=9, n_free=1280,
              n_rows=3, new_lens=4096, starts=4352, slots=4608, pos=4864, new_free=5120, ws=8192, wsb=1 << 20)


@pytest.mark.parametrize("kw", [dict(table=None), dict(lens=None), dict(grow=None), dict(n=-1), dict(n=65536),
                                dict(mp=-1), dict(mp=1 << 30), dict(page=0), dict(page=65537), dict(n_pages=-1),
                                dict(free=None), dict(cap=-1), dict(n_free=None), dict(n_rows=-1),
                                dict(n_rows=1 << 31), dict(new_lens=None), dict(starts=None), dict(slots=None),
                                dict(pos=None), dict(new_free=None), dict(new_lens=768), dict(starts=512),
                                dict(new_free=1024), dict(pos=4608)], ids=str)
def test_page_resize_status(kw):
    assert _status("fibq_page_resize", RESIZE, kw) == fq.FIBQ_EINVAL


WRITE = dict(k=256, v=512, dtype=0, n=3, kr=128, kh=64, vr=128, vh=64, slots=768, H=2, d=64, page=16, n_pages=9,
             codes=0, kp=4096, ks=5120, vp=8192, vs=6144)


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(dtype=3), dict(n=-1), dict(n=1 << 31), dict(H=0),
                                dict(H=1025), dict(d=0), dict(page=15), dict(page=256), dict(n_pages=0),
                                dict(n_pages=1 << 31), dict(codes=2), dict(kp=None), dict(ks=None), dict(vp=None),
                                dict(vs=None), dict(slots=None), dict(kr=-1), dict(vh=-1), dict(kp=4104),
                                dict(vp=4096), dict(vs=5120), dict(n=1 << 24)], ids=str)
def test_cache8_write_status(kw):
    assert _status("fibq_cache8_write", WRITE, kw) == fq.FIBQ_EINVAL


ATTN = dict(q=256, dtype=0, kp=4096, ks=512, vp=8192, vs=768, codes=1, table=1024, lens=1280, starts=1536, n=2,
            rows=3, H=2, G=4, mp=4, page=16, n_pages=9, d=64, causal=1, scale=0.0, out=2048, ws=256 * 99,
            wsb=1 << 40)


@pytest.mark.parametrize("kw", [dict(q=None), dict(dtype=3), dict(kp=None), dict(ks=None), dict(vp=None),
                                dict(vs=None), dict(codes=2), dict(table=None), dict(lens=None), dict(starts=None),
                                dict(n=-1), dict(n=65536), dict(rows=-1), dict(rows=1 << 31), dict(H=0),
                                dict(H=1025), dict(G=0), dict(G=17), dict(mp=-1), dict(mp=1 << 27), dict(page=8),
                                dict(n_pages=0), dict(d=0), dict(scale=float("inf")), dict(out=None),
                                dict(kp=4100), dict(rows=1 << 23)], ids=str)
def test_attn_cache8_status(kw):
    assert _status("fibq_attn_cache8", ATTN, kw) == fq.FIBQ_EINVAL


def test_unsupported_empty_and_workspace():
    assert _status("fibq_attn_cache8", ATTN, dict(d=96)) == fq.FIBQ_EUNSUPPORTED
    assert _status("fibq_cache8_write", WRITE, dict(d=96)) == fq.FIBQ_EUNSUPPORTED
    assert _status("fibq_attn_cache8", ATTN, dict(n=0, q=None, kp=None)) == fq.FIBQ_OK
    assert _status("fibq_attn_cache8", ATTN, dict(rows=0, q=None, kp=None)) == fq.FIBQ_OK
    assert _status("fibq_cache8_write", WRITE, dict(n=0, k=None)) == fq.FIBQ_OK
    assert _status("fibq_rope", ROPE, dict(n=0, q=None)) == fq.FIBQ_OK
    for name, a, need in (("fibq_attn_cache8", ATTN, fq.attn_cache8_workspace_bytes(2, 3, 2, 4, 4, 16, 64)),
                          ("fibq_page_resize", RESIZE, fq.page_resize_workspace_bytes(2))):
        if need:
            for kw in (dict(ws=None), dict(wsb=need - 1), dict(ws=8192 + 16)):
                assert _status(name, a, kw) == fq.FIBQ_EWORKSPACE
    for bad in ((-1, 3, 2, 4, 4, 16, 64), (2, 3, 2, 17, 4, 16, 64), (2, 3, 2, 4, 4, 24, 64), (2, 3, 2, 4, 4, 16, 80)):
        assert fq.attn_cache8_workspace_bytes(*bad) == 0
    assert fq.page_resize_workspace_bytes(65536) == 0 and fq.page_resize_workspace_bytes(-1) == 0
