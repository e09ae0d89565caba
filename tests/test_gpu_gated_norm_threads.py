"""Gradients of wide rows from two host threads at once, each on a stream of its own."""
import threading

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_two_widths_from_two_threads(stream):
    """Rows of more than 4096 channels take shared memory by their width, from one kernel for all of them.  What one thread's call sets up for its width must
    not take away what another's is about to launch with: the binding lets go of the GIL around the call."""
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(1)
    dtype = torch.bfloat16 if stream == "bf16" else torch.float32
    calls, want, failed = [], [], []
    for D in (4608, 8192):
        r, (b, dh) = torch.randn((3, D), generator=gen, device="cuda").to(dtype), (torch.randn((3, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
        w = torch.randn(D, generator=gen, device="cuda").bfloat16()
        calls.append(lambda r=r, b=b, dh=dh, w=w: trdq.trdq_gated_norm_backward(r, b, dh, weight=w))
        want.append(calls[-1]())
    torch.cuda.synchronize()
    start = threading.Barrier(2)

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(20):
                    got = [calls[i]() for _ in range(200)]
                    assert all(torch.equal(g[k], want[i][k]) for g in got[::20] for k in g if g[k] is not None)
        except BaseException as e:   # noqa: BLE001 (a thread's failure is the test's)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if failed:
        raise failed[0]
