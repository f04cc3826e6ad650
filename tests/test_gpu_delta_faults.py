"""Bounded waits of the delta rule's kernels that run out: the kernels return, the failure is reported, the next call is right.
The failure is a signal that is not given (one chunk is never loaded) under a small limit of polls; nothing faults or hangs."""
import pytest
import torch

from test_gpu_delta import BF16, DEV, F32, hd, make  # noqa: F401

pytestmark = pytest.mark.gpu

HS_ERR_COPY_TIMEOUT = 6


@pytest.fixture
def hs():
    from paper_2311_06281_b200 import heinsen_scan
    yield heinsen_scan
    heinsen_scan.debug_config(0, -1)


# shape, type, silent chunk, lengths: both kinds of pass, the first, a middle and the last, partly filled chunk
CASES = [((2, 300, 2, 2, 2, 2, 64, 64), BF16, 0, None), ((2, 300, 2, 2, 2, 2, 128, 64), F32, 2, None), ((1, 300, 1, 1, 1, 1, 256, 64), BF16, 9, None),
         ((5, 200, 16, 16, 16, 16, 64, 128), BF16, 1, None), ((5, 200, 16, 16, 16, 16, 128, 128), BF16, 3, (200, 10, 195, 200, 0))]


@pytest.mark.parametrize("shape,dtype,silent,lengths", CASES, ids=str)
def test_a_wait_that_runs_out_is_reported(hd, hs, shape, dtype, silent, lengths):  # noqa: F811
    ins = make(*shape, dtype, "token", True)
    ends = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    ws = hd.workspace(*ins[:5])
    want = hd.delta_attention(*ins, lengths=ends, workspace=ws)
    hs.check(ws)
    for _ in range(2):
        hs.debug_config(20000, silent)
        hd.delta_attention(*ins, lengths=ends, workspace=ws)
        with pytest.raises(hs.HeinsenScanError) as e:
            hs.check(ws)
        assert e.value.status == HS_ERR_COPY_TIMEOUT
        with pytest.raises(hs.HeinsenScanError):
            hd.check(DEV)
        hs.debug_config(0, -1)
        got = hd.delta_attention(*ins, lengths=ends, workspace=ws)
        hs.check(ws)
        hd.check(DEV)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("shape,dtype,silent,lengths", CASES, ids=str)
def test_gradients_are_right_again_after_a_wait_that_ran_out(hd, hs, shape, dtype, silent, lengths):  # noqa: F811
    ins = [x.requires_grad_() for x in make(*shape, dtype, "token", True)]
    ends = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    d_o = torch.randn(*shape[:3], shape[7], device=DEV).to(dtype)

    def gradients(silence):
        o, s = hd.delta_attention(*ins, lengths=ends)
        if silence:
            hs.debug_config(20000, silent)
        got = torch.autograd.grad([o, s], ins, [d_o, torch.ones_like(s)])
        torch.cuda.synchronize()
        hs.debug_config(0, -1)
        return got
    want = gradients(False)
    hd.check(DEV)
    gradients(True)
    with pytest.raises(hs.HeinsenScanError):
        hd.check(DEV)
    assert all(torch.equal(a, b) for a, b in zip(gradients(False), want))
    hd.check(DEV)
