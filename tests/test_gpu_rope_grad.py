"""Gradients through `rope` as torch records them.  They are the inverse turn of the
results' gradients, which test_gpu_paged.py holds against the formula and differences:
equal bit for bit, or summed up by torch where a leaf is used twice."""
import pytest
import torch

import paper_2605_11478_amd as fq

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def inputs(device, dtype, n=37, heads=9, d=64, rot=48):
    x = torch.randn(n, heads, d, device=device).to(TYPES[dtype])
    positions = torch.randint(0, 100000, (n,), device=device).int()
    return x, positions, torch.from_numpy(fq.rope_freqs(rot)).to(device)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("inverse", [False, True])
def test_gradients_of_parts_of_one_leaf(device, dtype, layout, inverse):
    x, positions, freqs = inputs(device, dtype)
    plain = fq.rope(x[:, :6], x[:, 6:8], positions, freqs, layout, 1.5, inverse)
    leaf = x.clone().requires_grad_()
    q, k = fq.rope(leaf[:, :6], leaf[:, 6:8], positions, freqs, layout, 1.5, inverse)
    assert q.requires_grad and k.requires_grad
    assert torch.equal(q, plain[0]) and torch.equal(k, plain[1])
    w = torch.randn_like(x)
    want = torch.zeros_like(x)
    want[:, :6], want[:, 6:8] = fq.rope(w[:, :6], w[:, 6:8], positions, freqs, layout, 1.5, not inverse)
    got, = torch.autograd.grad([q, k], leaf, [w[:, :6], w[:, 6:8]], retain_graph=True)
    assert torch.equal(got, want)
    # gradients without dense heads: expanded, transposed
    one = torch.ones((), dtype=x.dtype, device=device)
    got, = torch.autograd.grad(q, leaf, one.expand(q.shape), retain_graph=True)
    assert torch.equal(got[:, :6], fq.rope(one.expand(q.shape).contiguous(), None, positions, freqs, layout, 1.5,
                                           not inverse)[0]) and (got[:, 6:] == 0).all()
    turned = w[:, 6:8].transpose(1, 2).contiguous().transpose(1, 2)
    got, = torch.autograd.grad(k, leaf, turned)
    assert torch.equal(got[:, 6:8], want[:, 6:8]) and (got[:, :6] == 0).all()


def test_gradients_of_one_of_both(device):
    x, positions, freqs = inputs(device, "fp32")
    q, k = x[:, :6].clone(), x[:, 6:8].clone()
    w = torch.randn_like(q)
    for a, b in ((q.requires_grad_(), None), (q, k)):
        y, z = fq.rope(a, b, positions, freqs)
        assert y.requires_grad and (z is None or not z.requires_grad)
        assert torch.equal(torch.autograd.grad(y, q, w)[0], fq.rope(w, None, positions, freqs, inverse=True)[0])
    y, z = fq.rope(q.detach(), k.requires_grad_(), positions, freqs)
    assert z.requires_grad and not y.requires_grad
    z.sum().backward()
    assert torch.equal(k.grad, fq.rope(torch.ones_like(z), None, positions, freqs, inverse=True)[0])


def test_second_gradients(device):
    x, positions, freqs = inputs(device, "fp32")
    x.requires_grad_()
    w = torch.randn_like(x).requires_grad_()
    y, _ = fq.rope(x, None, positions, freqs)
    g, = torch.autograd.grad(y, x, w, create_graph=True)
    v = torch.randn_like(x)
    assert torch.equal(torch.autograd.grad(g, w, v)[0], fq.rope(v, None, positions, freqs)[0])


def test_refusals_and_unrecorded_calls(device):
    x, positions, freqs = inputs(device, "fp32")
    leaf = x.clone().requires_grad_()
    out = torch.empty_like(x)
    for pair in ((out, None), (leaf, None)):
        with pytest.raises(ValueError, match="out takes no part"):
            fq.rope(leaf, None, positions, freqs, out=pair)
    with pytest.raises(ValueError, match="out takes no part"):
        fq.rope(x, None, positions, freqs, out=(leaf, None))
    with pytest.raises(ValueError, match="freqs must not"):
        fq.rope(x, None, positions, freqs.clone().requires_grad_())
    assert torch.equal(leaf, x)
    want = fq.rope(x, None, positions, freqs)[0]
    with torch.no_grad():
        fq.rope(leaf, None, positions, freqs, out=(out, None))
        assert torch.equal(out, want) and not fq.rope(leaf, None, positions, freqs)[0].requires_grad
    y, _ = fq.rope(leaf, None, positions, freqs)
    positions.add_(1)  # what the backward pass needs was written
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_no_rows(device):
    x, positions, freqs = inputs(device, "bf16", n=0)
    x.requires_grad_()
    y, _ = fq.rope(x, None, positions, freqs)
    y.sum().backward()
    assert x.grad.shape == x.shape
