"""Tensors that are more than their memory says are refused, on a
planning-only context: forward tangents, the negative bit, and zeros that have
no memory."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2607_18582_amd import Mure, MureError


@pytest.fixture()
def mure():
    m = Mure(device=-1)
    yield m
    m.close()


def negative(*shape):
    """The imaginary part of a conjugate: a float32 view with the negative bit."""
    t = torch.zeros(*shape, 1, dtype=torch.complex64).conj().imag[..., 0]
    assert t.is_neg()
    return t


def zeros(*shape):
    return torch._efficientzerotensor(shape)


def test_forward_tangents(mure):
    seqs = mure.sequences([4, 3])
    x, taps = torch.ones(7, 8), torch.ones(8, 4)
    with fwd.dual_level():
        for a, b in ((fwd.make_dual(x, torch.ones(7, 8)), taps), (x, fwd.make_dual(taps, torch.ones(8, 4)))):
            with pytest.raises(ValueError, match="tangent"):
                seqs.conv(a, b)
            with fwd._set_fwd_grad_enabled(False), pytest.raises(MureError, match="planning-only"):
                seqs.conv(a, b)
        with pytest.raises(MureError, match="planning-only"):
            seqs.conv(x, taps)
        dual = fwd.make_dual(x, x)
        with pytest.raises(ValueError, match="tangent"):
            mure.block_norm(dual, before="rms")
        with pytest.raises(ValueError, match="tangent"):
            seqs.scan(x, dual, torch.ones(8, 2), torch.ones(7, 2), torch.ones(7, 2))
        with pytest.raises(ValueError, match="tangent"):
            seqs.conv(x, taps, out=dual)


@pytest.mark.parametrize("make,word", [(negative, "negative bit"), (zeros, "no memory")])
def test_views_that_are_not_their_memory(mure, make, word):
    seqs = mure.sequences([4, 3])
    x, taps, A, b = torch.ones(7, 8), torch.ones(8, 4), torch.ones(8, 2), torch.ones(7, 2)
    v = make(8)
    for call in (lambda: seqs.conv(make(7, 8), taps), lambda: seqs.conv(x, make(8, 4)), lambda: seqs.conv(x, taps, v),
                 lambda: seqs.conv(x, taps, out=make(7, 8)), lambda: seqs.conv(x, taps, state=make(2, 3, 8)),
                 lambda: seqs.scan(x, x, make(8, 2), b, b), lambda: seqs.scan(x, x, A, make(7, 2), b),
                 lambda: seqs.scan(x, x, A, b, b, skip=v), lambda: mure.block_norm(x, make(7, 8)),
                 lambda: mure.block_norm(x, x, scale=v)):
        with pytest.raises(ValueError, match=word):
            call()
    with pytest.raises(MureError, match="planning-only"):
        seqs.conv(negative(7, 8).resolve_neg(), taps)
