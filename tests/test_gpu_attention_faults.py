"""Bounded waits of the tensor-core passes that run out: the kernels return, the failure is reported, the next call is right.
The failure is a signal that is not given (the decays of one chunk are never announced) under a small limit of polls; nothing
faults or hangs."""
import pytest
import torch

from test_gpu_attention import BF16, DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu

HS_ERR_COPY_TIMEOUT = 6


@pytest.fixture
def hs():
    from paper_2311_06281_b200 import heinsen_scan
    yield heinsen_scan
    heinsen_scan.debug_config(0, -1)


# (b, t, h), the silent chunk, lengths: whole and cut sequences, the first, a middle and the last, partly filled chunk
CASES = [((2, 1000, 60), 3, None), ((1, 1500, 2), 2, None), ((1, 1500, 2), 11, None), ((3, 520, 40), 0, None),
         ((2, 700, 50), 4, (600, 530)), ((1, 100, 1), 0, None)]


@pytest.mark.parametrize("shape,silent,lengths", CASES, ids=str)
def test_a_wait_that_runs_out_is_reported_in_the_workspace(ha, hs, shape, silent, lengths):  # noqa: F811
    q, k, v, log_a, s0 = make(*shape, *[shape[2]] * 3, 128, 64, BF16, state=True)
    ends = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    ws = ha.workspace(q, k, v, log_a)
    want = ha.decay_attention(q, k, v, log_a, s0, lengths=ends, workspace=ws)
    hs.check(ws)
    for _ in range(2):
        hs.debug_config(20000, silent)
        ha.decay_attention(q, k, v, log_a, s0, lengths=ends, workspace=ws)
        with pytest.raises(hs.HeinsenScanError) as e:
            hs.check(ws)
        assert e.value.status == HS_ERR_COPY_TIMEOUT
        hs.debug_config(0, -1)
        got = ha.decay_attention(q, k, v, log_a, s0, lengths=ends, workspace=ws)
        hs.check(ws)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("shape,silent,lengths", CASES, ids=str)
def test_gradients_are_right_again_after_a_wait_that_ran_out(ha, hs, shape, silent, lengths):  # noqa: F811
    ins = [x.requires_grad_() for x in make(*shape, *[shape[2]] * 3, 128, 64, BF16, state=True)]
    ends = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    d_o = torch.randn(*shape, 64, device=DEV).to(BF16)

    def gradients(silence):
        o, s = ha.decay_attention(*ins, lengths=ends)
        if silence:
            hs.debug_config(20000, silent)
        got = torch.autograd.grad([o, s], ins, [d_o, torch.ones_like(s)])
        torch.cuda.synchronize()
        hs.debug_config(0, -1)
        return got
    want = gradients(False)
    gradients(True)
    assert all(torch.equal(a, b) for a, b in zip(gradients(False), want))


def test_a_call_on_the_cuda_cores_does_not_report_an_earlier_failure(ha, hs):  # noqa: F811
    q, k, v, log_a, s0 = make(1, 700, 2, 2, 2, 2, 64, 64, BF16, state=True)
    ws = torch.empty(max(ha.workspace(*x, log_a).numel() for x in ((q, k, v), (q.float(), k.float(), v.float()))),
                     dtype=torch.uint8, device=DEV)
    for other in ([q.float(), k.float(), v.float(), log_a, s0], [x[:, :5].float() for x in (q, k, v, log_a)]):
        hs.debug_config(20000, 1)
        ha.decay_attention(q, k, v, log_a, s0, workspace=ws)
        with pytest.raises(hs.HeinsenScanError):
            hs.check(ws)
        hs.debug_config(0, -1)
        ha.decay_attention(*other, workspace=ws)  # float32: another kernel, the same workspace
        hs.check(ws)


@pytest.mark.parametrize("backward", [False, True])
def test_failures_without_a_kept_workspace_are_found(ha, hs, backward):  # noqa: F811
    ins = [x.requires_grad_(backward) for x in make(1, 1500, 2, 2, 2, 2, 128, 128, BF16, state=True)]
    try:
        ha.check(DEV)
    except hs.HeinsenScanError:
        pass  # what the tests before have left
    ha.check(DEV)

    def call(silence):
        if silence and not backward:
            hs.debug_config(20000, 5)
        o, s = ha.decay_attention(*ins)
        if backward:
            if silence:
                hs.debug_config(20000, 5)
            torch.autograd.grad(o.float().sum(), ins)
        hs.debug_config(0, -1)
    for _ in range(2):
        call(True)
        with pytest.raises(hs.HeinsenScanError) as e:
            ha.check(DEV)
        assert e.value.status == HS_ERR_COPY_TIMEOUT
        ha.check(DEV)  # told once
        call(False)
        ha.check(torch.device(DEV))
