"""Sequences of as many tokens as there are numbers, most of them on one page: written at their end, read back there, attended to."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu

HIGH = 2 ** 31 - 1


@pytest.mark.parametrize("length", [HIGH, HIGH - 30, HIGH - 31])
@pytest.mark.parametrize("rows", [1, 200])
def test_the_longest_sequences(length, rows):
    """Two tokens of all outweigh the rest by e^100: one of the first and one of the last."""
    import torch
    D, page = 8, 65536
    c = B.lq_kvcache_create(1, 3, page, 1, D)
    table = torch.zeros(32768, dtype=torch.int32, device="cuda")
    table[0], table[-1] = 2, 1
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    values = np.random.default_rng(1).integers(-127, 128, (2, D)).astype(np.float16)
    new = 300
    k, v = (torch.zeros(new, D, dtype=torch.float16, device="cuda") for _ in "kv")
    q = torch.zeros(rows, D, dtype=torch.float16, device="cuda")
    q[:, 0] = 1
    for at, end, value in ((7, new, values[0]), (new - 1 - rows, length, values[1])):
        k.zero_()
        v.zero_()
        k[at, 0] = 100
        v[at] = torch.from_numpy(value).cuda()
        n = ints(end)
        B.lq_kvcache_append(c, 0, B.lq_kvbatch(1, new, n.data_ptr(), table.data_ptr(), 32768), B.lq_kvrows(k.data_ptr(), (0, D, D), v.data_ptr(), (0, D, D)), B.OUT_F16, st)
        torch.cuda.synchronize()
    b = B.lq_kvbatch(1, rows, n.data_ptr(), table.data_ptr(), 32768)
    out = torch.full((2, new, D), 7.0, device="cuda")
    begin = ints(length - new)
    B.lq_kvcache_read(c, 0, b, begin.data_ptr(), new, B.lq_kvrows(out[0].data_ptr(), (0, D, D), out[1].data_ptr(), (0, D, D)), B.OUT_F32, st)
    assert torch.equal(out[0], k.float()) and torch.equal(out[1], v.float())
    # (halves of whole numbers up to 127: exact)
    for causal, window, sinks, want in ((False, 0, 0, values.mean(0)), (True, 0, 0, values.mean(0)), (True, 250, HIGH, values.mean(0)), (True, 250, 0, values[1]),
                                        (True, HIGH, HIGH, values.mean(0)), (True, 250, 7, values[1]), (True, 250, 8, values.mean(0))):
        got = torch.full((rows, D), 7.0, dtype=torch.float16, device="cuda")
        B.lq_cache_attention(c, 0, b, B.lq_attn(q.data_ptr(), (D, D), got.data_ptr(), (D, D), 1, 1.0, causal, window, sinks), st)
        assert (got.cpu().numpy() == want).all(), (causal, window, sinks, got[0], want)
    assert B.lq_get_device_status(0) == (0, 0)
    B.lq_kvcache_free(c)
