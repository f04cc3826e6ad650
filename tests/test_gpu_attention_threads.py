"""decay_attention called from several host threads at once, each on a stream of its own."""
import threading

import pytest
import torch

from test_gpu_attention import DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu


def test_threads_with_different_widths_do_not_disturb_each_other(ha):  # noqa: F811
    """The shared memory that a kernel may ask for belongs to the kernel, not to a call: calls of one width must not take it
    away from those of another between their own request and launch."""
    widths, rounds = (256, 16, 128, 40), 150
    calls = []
    for d in widths:
        ins = [x.requires_grad_() for x in make(1, 40, 2, 2, 2, 2, d, d, F32, state=True, seed=d)]
        d_o = torch.randn(1, 40, 2, d, device=DEV)

        def call(ins=ins, d_o=d_o):
            o, s = ha.decay_attention(*ins)
            return (o, s, *torch.autograd.grad([o], ins, [d_o]))
        calls.append((call, [x.detach().clone() for x in call()]))
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(len(widths))

    def work(call, want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(rounds):
                    got = call()
                    if not all(torch.equal(a, b) for a, b in zip(got, want)):
                        raise AssertionError("another result")
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed[0]


def test_calls_of_the_library_from_many_threads_are_all_accepted(ha):  # noqa: F811
    """The same closer to the library: nothing but its calls, which run beside each other between the interpreter's turns."""
    forward, failed, start = ha._call().forward, [], threading.Barrier(8)

    def work(d):
        try:
            q, k, v, log_a, s0 = make(1, 20, 2, 2, 2, 2, d, d, F32, state=True, seed=d)
            want, _ = ha.decay_attention(q, k, v, log_a, s0)
            ws, o, s = ha.workspace(q, k, v, log_a), torch.empty_like(want), torch.empty_like(s0)
            p = ha._problem(q, k, v, log_a, s0, d ** -0.5, None)
            stream = torch.cuda.Stream()
            args = p.packed, ha._ROWS.pack(*ha._rows(o, "o")), s.data_ptr(), ws.data_ptr(), ws.numel(), stream.cuda_stream
            torch.cuda.synchronize()
            start.wait()
            refused = sum(forward(*args) != 0 for _ in range(4000))
            stream.synchronize()
            assert refused == 0, f"{refused} of 4000 calls of width {d} were refused"
            assert torch.equal(o, want)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(d,)) for d in (256, 40, 256, 48, 256, 64, 200, 72)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
