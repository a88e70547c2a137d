"""Batches at the ends of what they may be: the most sequences, the most query heads to a head, lengths that shrink."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

from .test_gpu_kvcache import Cache, filled, run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ragged", [False, True])
def test_the_most_sequences(ragged):
    """65535 of them, of one or two tokens; the first token sees itself alone, so its output is its value."""
    import torch
    S, D = 65535, 16
    c = B.lq_kvcache_create(1, S, 32, 1, D)
    ns = torch.tensor([(1 if not ragged else (s * 7) % 3) for s in range(S)], dtype=torch.int32)
    start = torch.cat([torch.zeros(1, dtype=torch.int32), ns.cumsum(0, dtype=torch.int32)])
    rows = int(start[-1])
    pages = torch.randperm(S, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    nd, sd = ns.cuda(), start.cuda()
    b = B.lq_kvbatch(S, rows, nd.data_ptr(), pages.data_ptr(), 1, sd.data_ptr() if ragged else None)
    k = torch.zeros(rows, D, dtype=torch.float16, device="cuda")
    v = torch.randint(-127, 128, (rows, D), device="cuda").half()
    v[:, 0] = 127                                          # (steps of one: whole numbers are held as they are)
    st = torch.cuda.current_stream().cuda_stream
    B.lq_kvcache_append(c, 0, b, B.lq_kvrows(k.data_ptr(), (0, D, D), v.data_ptr(), (0, D, D)), B.OUT_F16, st)
    out = torch.full((rows + 1, D), 7.0, dtype=torch.float16, device="cuda")
    B.lq_cache_attention(c, 0, b, B.lq_attn(k.data_ptr(), (D, D), out.data_ptr(), (D, D), 1, 1.0), st)
    second = torch.zeros(rows, dtype=torch.bool)
    second[start[:-1][ns == 2].long() + 1] = True
    want = torch.where(second.cuda()[:, None], (v + v.roll(1, 0)) / 2, v)       # equal weights; halves of whole numbers up to 254 are exact
    assert torch.equal(out[:rows], want) and (out[rows:] == 7).all()
    assert B.lq_get_device_status(0) == (0, 0)
    B.lq_kvcache_free(c)


@pytest.mark.parametrize("D,hq,hk", [(64, 4096, 1), (16, 4096, 4096), (192, 512, 2)])
def test_the_most_heads(D, hq, hk):
    c = filled(D, hk, [40, 3], 32)
    run_attention(c, [1, 1], [40, 3], hq, uniform=True)
    run_attention(c, [2, 1], [40, 3], hq, behind=1)
    c.close()


@pytest.mark.parametrize("D", [64, 256])
def test_tokens_that_are_taken_back(D):
    """Lengths that shrink, to within a block and beyond one, and what is then written in their place."""
    c = Cache(D, 2, [200, 150], 64)
    c.append([100, 90])
    for back, ns in (([3, 0], [1, 2]), ([40, 33], [70, 5]), ([1, 64], [1, 1])):
        c.len = [n - x for n, x in zip(c.len, back)]
        c.append(ns)
        c.check()
        run_attention(c, ns, c.len, 4)
    c.close()


@pytest.mark.parametrize("D,hq,hk", [(128, 8, 2), (72, 4, 4), (256, 4, 2)])
def test_a_captured_batch_takes_the_forms_that_its_arrays_ask_for(D, hq, hk):
    """One graph; first rows, lengths and pages change between its replays, so that prompts become single tokens, sequences empty, and the other way round."""
    import torch

    from .test_gpu_kvcache import attend
    lens = [900, 700, 333, 64]
    c = filled(D, hk, lens, 64)
    rows = 420
    q = torch.randn(rows, hq, D, dtype=torch.float16, device="cuda")
    out = torch.zeros_like(q)
    sd, ld, pd = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (5, 4, 4 * c.stride))
    b = B.lq_kvbatch(4, rows, ld.data_ptr(), pd.data_ptr(), c.stride, sd.data_ptr())
    a = B.lq_attn(q.data_ptr(), q.stride()[:2], out.data_ptr(), out.stride()[:2], hq, 0.1)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        B.lq_cache_attention(c.h, 0, b, a, side.cuda_stream)
    x = q.double().cpu().numpy()
    for order, ns, ts in (((0, 1, 2, 3), (300, 1, 60, 5), lens), ((3, 2, 1, 0), (1, 1, 1, 1), (9, 300, 700, 900)), ((1, 0, 3, 2), (0, 400, 0, 1), (0, 900, 64, 1)),
                          ((2, 2, 2, 2), (7, 70, 33, 310), (7, 333, 33, 310)), ((0, 1, 2, 3), (0, 0, 0, 0), lens), ((0, 1, 2, 3), (300, 1, 60, 5), lens)):
        ts = [t if order == (0, 1, 2, 3) or t <= lens[s] else lens[s] for s, t in zip(order, ts)]
        sd.copy_(torch.tensor([0, *np.cumsum(ns)], dtype=torch.int32))
        ld.copy_(torch.tensor(ts, dtype=torch.int32))
        pd.copy_(torch.from_numpy(c.pages[list(order)].reshape(-1)))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got, at = out.double().cpu().numpy(), 0
        for s, n, t in zip(order, ns, ts):
            want, err = attend(x[at:at + n], c.held[0][s][:t], c.held[1][s][:t], 0.1, t - n, True, 0, 0)
            assert (np.abs(got[at:at + n] - want) <= err).all(), (order, s)
            at += n
        assert (got[at:] == 7).all()
    del graph
    c.close()


def test_without_launches_that_overlap():
    """The same bits where no kernel starts before the one ahead of it has ended."""
    import torch
    lens, ns = [1500, 900, 40], [300, 1, 40]
    c = filled(128, 2, lens, 64)
    q = torch.randn(sum(ns), 8, 128, dtype=torch.float16, device="cuda")
    out = torch.zeros(2, *q.shape, dtype=torch.float16, device="cuda")
    for i in range(2):
        B.lq_set_option("overlap", 1 - i)
        try:
            B.lq_cache_attention(c.h, 0, c.batch(ns, lens), B.lq_attn(q.data_ptr(), q.stride()[:2], out[i].data_ptr(), q.stride()[:2], 8, 0.1),
                                 torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
        finally:
            B.lq_set_option("overlap", 1)
    assert torch.equal(out[0], out[1])
    c.check()
    c.close()
