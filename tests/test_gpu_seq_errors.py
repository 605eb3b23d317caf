"""An error that another call of the thread has left in the HIP runtime is not
taken for the failure of a launch."""
import ctypes as C

import pytest
import torch

from paper_2607_18582_amd import Mure

pytestmark = pytest.mark.gpu

HIP_ERROR_OUT_OF_MEMORY = 2


def runtime():
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64" in line)
    return C.CDLL(path)


def test_errors_of_other_calls():
    m = Mure(device=0)
    g = torch.Generator().manual_seed(0)
    rows = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    length, D, N = 600, 24, 16
    x, taps, dt, b, c, A = rows(length, D), rows(D, 4), rows(length, D), rows(length, N), rows(length, N), -rows(D, N).abs()
    seqs = m.sequences([length])
    calls = [lambda: seqs.conv(x, taps), lambda: seqs.scan(x, dt, A, b, c), lambda: m.block_norm(x, before="rms")]
    expected = [call()[0] for call in calls]
    torch.cuda.synchronize()
    hip = runtime()
    for call, e in zip(calls, expected):
        p = C.c_void_p()
        assert hip.hipMalloc(C.byref(p), C.c_size_t(1 << 60)) == HIP_ERROR_OUT_OF_MEMORY
        try:
            got = call()[0]
        finally:
            hip.hipGetLastError()
        torch.cuda.synchronize()
        assert torch.equal(got, e)
    seqs.close()
    m.close()
