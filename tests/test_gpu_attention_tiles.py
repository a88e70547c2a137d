"""The tiles of many rows at every width of a head that they have an instance for, and at widths that these are padded from."""
import pytest

from paper_2604_18117_b200 import binding as B

from .test_gpu_kvcache import filled, run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [8, 16, 40, 56, 64, 72, 80, 88, 96, 104, 112, 120, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
def test_widths(D, window, sinks):
    """Prompts in one batch with rows of the other form, all seen and causal."""
    lens, ns = [300, 40, 513, 0, 700, 129], [300, 1, 200, 0, 260, 129]
    c = filled(D, 2, lens, 32 if D % 16 else 96)
    run_attention(c, ns, lens, 4, True, window, sinks, behind=2)
    if not window:
        run_attention(c, ns, lens, 4, False)
    c.close()


@pytest.mark.parametrize("D", [8, 40, 64, 72, 80, 88, 96, 104, 112, 128])
@pytest.mark.parametrize("ns,lens", [([1500, 900], [1500, 3000]), ([300, 40], [4500, 4000])], ids=["prompts", "shared"])
def test_copies_come_behind_the_loads_of_what_they_replace(D, ns, lens):
    """Call after call the same bits, and those of 64 bits: a record that came into its place before the one there had been read would show."""
    import torch
    c = filled(D, 2, lens, 64)
    run_attention(c, ns, lens, 2)
    q = torch.randn(sum(ns), 16, D, dtype=torch.float16, device="cuda")
    out = torch.empty(2, sum(ns), 16, D, dtype=torch.float16, device="cuda")
    b = c.batch(ns, c.len)
    for i in range(150):
        a = B.lq_attn(q.data_ptr(), q.stride()[:2], out[min(i, 1)].data_ptr(), out.stride()[1:3], 16, 0.1)
        B.lq_cache_attention(c.h, 0, b, a, torch.cuda.current_stream().cuda_stream)
        assert i == 0 or torch.equal(out[0], out[1]), i
    c.close()
