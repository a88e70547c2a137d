"""The residual's calls from several threads at once: widths whose vectors take different amounts of shared memory in one kernel."""
import threading

import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("widths,M", [((6144, 7168), 16), ((4608, 8192), 2000)])
def test_two_widths_of_one_kernel(widths, M):
    import torch
    out = {}

    def work(C, calls, key):
        torch.cuda.set_device(0)
        x = torch.linspace(-3, 5, M * C, device="cuda").view(M, C).half()
        h, stream = torch.empty(2, M, C, dtype=torch.float16, device="cuda"), torch.cuda.Stream()
        torch.cuda.synchronize()
        try:
            for i in range(calls):
                B.lq_residual_norm(B.lq_residual(M, C, x.data_ptr(), None, h[min(i, 1)].data_ptr(), norm=B.NORM_LAYER), stream.cuda_stream)
            stream.synchronize()
            out[key] = h[0].clone()
            assert calls == 1 or torch.equal(h[0], h[1])
        except Exception as e:                             # (told to the test's own thread)
            out[key] = e

    for C in widths:
        work(C, 1, ("alone", C))
    threads = [threading.Thread(target=work, args=(C, 4000, C)) for C in widths for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for C in widths:
        assert not isinstance(out[C], Exception), out[C]
        assert torch.equal(out[C], out["alone", C])
