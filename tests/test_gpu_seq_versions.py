"""A tensor that receives results counts as changed: autograd sees that what it
saved of it is gone."""
import pytest
import torch

from paper_2607_18582_amd import Mure, MureError

pytestmark = pytest.mark.gpu


def test_results_raise_the_version():
    m = Mure(device=0)
    seqs = m.sequences([4, 3])
    rows = lambda *s: torch.ones(*s, device="cuda")  # noqa: E731
    x, taps, A, b = rows(7, 8), rows(8, 4), -rows(8, 2), rows(7, 2)
    calls = {"conv out": (rows(7, 8), lambda t: seqs.conv(x, taps, out=t)),
             "conv state": (rows(2, 3, 8), lambda t: seqs.conv(x, taps, state=t, state_out=t)),
             "scan out": (rows(7, 8), lambda t: seqs.scan(x, x, A, b, b, out=t)),
             "scan state": (rows(2, 8, 2), lambda t: seqs.scan(x, x, A, b, b, state=t, state_out=t)),
             "norm out": (rows(7, 8), lambda t: m.block_norm(x, before="rms", out=t)),
             "norm residual": (rows(7, 8), lambda t: m.block_norm(x, t, residual_out=t))}
    inputs = [x, taps, A, b]
    for name, (t, call) in calls.items():
        before = t._version
        call(t)
        assert t._version == before + 1, name
        call(t)
        assert t._version == before + 2, name
    assert all(v._version == 0 for v in inputs)
    # what autograd has saved of it
    w = rows(7, 8).requires_grad_()
    t = rows(7, 8)
    loss = (w * t).sum()
    seqs.conv(x, taps, out=t)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    # not by a call that is refused
    before = x._version
    with pytest.raises(MureError, match="overlaps"):
        seqs.conv(x, taps, out=x)
    assert x._version == before
    # tensors of inference mode have none
    with torch.inference_mode():
        t = rows(7, 8)
    expected, _ = seqs.conv(x, taps)
    seqs.conv(x, taps, out=t)
    with torch.inference_mode():
        seqs.conv(x, taps, out=t)
    torch.cuda.synchronize()
    assert torch.equal(t, expected)
    m.close()
