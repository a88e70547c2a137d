"""The arrays of a batch: what they may hold, and where they may lie."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

from .test_gpu_kvcache import Cache, attend, filled, write

pytestmark = pytest.mark.gpu

LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("many", [1, 60])
def test_first_rows_that_are_none(many):
    """Ends far below their starts, starts below zero, ends behind the call's rows: nothing but the call's rows is touched, and what the last sequence has for
    itself is right."""
    import torch
    lens = [40, 10 * many, 100, 500]
    c = filled(64, 2, lens, 32)
    rows = 8 * many + 3
    starts = [[5 * many, LOW, 6 * many, 6 * many, 8 * many], [LOW, LOW, LOW + 1, 6 * many, 8 * many], [HIGH, -1, 6 * many, 6 * many, 8 * many],
              [HIGH, LOW, HIGH, 6 * many, 8 * many]]
    for start in starts:
        x = torch.randn(rows, 4, 64, dtype=torch.float16, device="cuda")
        out = torch.full((rows + 64, 4, 64), 7.0, dtype=torch.float16, device="cuda")
        sd, ld = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (start, lens))
        b = B.lq_kvbatch(4, rows, ld.data_ptr(), c.pages_d.data_ptr(), c.stride, sd.data_ptr())
        st = torch.cuda.current_stream().cuda_stream
        B.lq_cache_attention(c.h, 0, b, B.lq_attn(x.data_ptr(), (256, 64), out.data_ptr(), (256, 64), 4, 0.1), st)
        torch.cuda.synchronize()
        assert (out[rows:] == 7).all()
        clamp = lambda v: min(max(v, 0), rows)
        if any(clamp(a) < clamp(e) and clamp(e) > 6 * many for a, e in zip(start[:3], start[1:4])):
            continue                                       # (another one has its rows too)
        want, err = attend(x[6 * many:8 * many].double().cpu().numpy(), c.held[0][3][:500], c.held[1][3][:500], 0.1, 500 - 2 * many, True, 0, 0)
        assert (np.abs(out[6 * many:8 * many].double().cpu().numpy() - want) <= err).all()
        # the same to write: its last tokens, as they are there already
        keys = torch.zeros(rows, 2, 2, 64, device="cuda")
        for side in range(2):
            keys[6 * many:8 * many, side] = torch.from_numpy(c.held[side][3][500 - 2 * many:500]).float()
        B.lq_kvcache_append(c.h, 0, b, B.lq_kvrows(keys.data_ptr(), (0, 256, 64), keys[:, 1].data_ptr(), (0, 256, 64)), B.OUT_F32, st)
        torch.cuda.synchronize()
    B.lq_get_device_status(0)                              # (some of them do not fit their lengths)
    B.lq_kvcache_free(c.h)


@pytest.mark.parametrize("rows", [HIGH, HIGH - 30, HIGH - 31, HIGH - 32])
def test_as_many_rows_as_there_are_numbers(rows):
    """Calls of up to 2^31 - 1 rows, of which the first sequence begins far behind."""
    import torch
    c = Cache(16, 1, [60, 90], 32)
    c.append([20, 3])
    ns = [10, 39]
    first = rows - sum(ns)
    x = c.values(2 * sum(ns)).astype(np.float16)
    buf = torch.from_numpy(x).cuda().view(sum(ns), 2, 16)
    c.len = [a + n for a, n in zip(c.len, ns)]
    sd, ld = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([first, first + ns[0], rows], c.len))
    b = B.lq_kvbatch(2, rows, ld.data_ptr(), c.pages_d.data_ptr(), c.stride, sd.data_ptr())
    k, v = (buf[:, i].data_ptr() - first * 64 for i in range(2))                # (where row 0 would lie)
    B.lq_kvcache_append(c.h, 0, b, B.lq_kvrows(k, (0, 32, 16), v, (0, 32, 16)), B.OUT_F16, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for side in range(2):
        at = 0
        for s, n in enumerate(ns):
            write(c.held[side][s], c.exps[side][s], x.reshape(sum(ns), 2, 1, 16)[at:at + n, side].astype(np.float64), c.len[s] - n)
            at += n
    c.check()
    c.close()


def code(f, *a):
    try:
        f(*a)
    except B.LqError as e:
        return e.code
    return 0


def test_outputs_lie_on_no_array():
    """An array of the batch, whole or its last entry, inside an output, in a gap of it and right behind it."""
    import torch
    c = B.lq_kvcache_create(1, 8, 32, 1, 64)
    S = 4
    buf = torch.zeros(4096, dtype=torch.float16, device="cuda")
    other = torch.zeros(64, dtype=torch.int32, device="cuda")
    q = torch.zeros(S * 64, dtype=torch.float16, device="cuda")
    apart = {"length": other.data_ptr(), "pages": other.data_ptr() + 64, "start": other.data_ptr() + 128, "begin": other.data_ptr() + 192}
    size = {"length": S, "pages": 2 * S, "start": S + 1, "begin": S}
    out = buf.data_ptr() + 1024                            # rows of 64 halves, 192 apart: 128 bytes in 384
    end = out + 3 * 384 + 128
    for name in size:
        n = 4 * size[name]
        for at, want in ((out, 1), (out + 384 + 124, 1), (out - n + 4, 1), (end - 4, 1), (out + 128, 0), (out + 384 - n, 0), (out - n, 0), (end, 0)):
            a = {**apart, name: at}
            b = B.lq_kvbatch(S, S, a["length"], a["pages"], 2, a["start"])
            o = B.lq_kvrows(out, (192, 64, 64), None, (0, 0, 0)), B.lq_kvrows(None, (0, 0, 0), out, (192, 64, 64))
            if name != "begin":
                assert code(B.lq_cache_attention, c, 0, b, B.lq_attn(q.data_ptr(), (64, 64), out, (192, 64), 1, 0.1)) == want, (name, at - out)
            for r in o:
                if name != "start":                          # (which reading does not use)
                    assert code(B.lq_kvcache_read, c, 0, b, a["begin"], 1, r) == want, (name, at - out)
                else:
                    assert code(B.lq_kvcache_read, c, 0, b, a["begin"], 1, r) == 0
    torch.cuda.synchronize()
    B.lq_get_device_status(0)                              # (the arrays' zeros are lengths below their rows)
    assert (buf == 0).all()
    B.lq_kvcache_free(c)


def test_reading_wants_no_rows():
    """Rows of none, first rows of none or anywhere: the same is read.  Rows that the sequences cannot share alike are refused here too."""
    import torch
    lens = [40, 10, 77]
    c = filled(64, 2, lens, 32)
    ld, wild = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.tensor([HIGH, LOW, -3, 5], dtype=torch.int32, device="cuda")
    out = torch.zeros(3, 3, 77, 2, 64, device="cuda")
    for i, (rows, start) in enumerate(((0, None), (6, None), (1000, wild.data_ptr()))):
        r = B.lq_kvrows(out[i].data_ptr(), (77 * 128, 128, 64), None, (0, 0, 0))
        B.lq_kvcache_read(c.h, 0, B.lq_kvbatch(3, rows, ld.data_ptr(), c.pages_d.data_ptr(), c.stride, start), None, 77, r, B.OUT_F32)
    torch.cuda.synchronize()
    for got in out.double().cpu().numpy():
        for s, n in enumerate(lens):
            assert np.array_equal(got[s, :n], c.held[0][s][:n]) and (got[s, n:] == 0).all()
    assert code(B.lq_kvcache_read, c.h, 0, B.lq_kvbatch(3, 4, ld.data_ptr(), c.pages_d.data_ptr(), c.stride), None, 77, r, B.OUT_F32) == 1
    c.close()


def test_calls_of_more_thread_blocks_than_a_launch_has():
    c = B.lq_kvcache_create(1, 1, 32, 4096, 8)
    fake, far = 1 << 40, 1 << 50                           # (refused before anything is read)
    rows = lambda seq: B.lq_kvrows(far, (seq, 4096 * 8, 8), None, (0, 0, 0))
    b = lambda n, s=1, stride=1: B.lq_kvbatch(s, n, fake, fake + (1 << 20), stride)
    both = B.lq_kvrows(far, (0, 0, 8), far, (0, 0, 8))
    assert code(B.lq_kvcache_append, c, 0, b(1 << 24), both) == 2 and code(B.lq_kvcache_append, c, 0, b(HIGH), both) == 2
    assert code(B.lq_kvcache_read, c, 0, b(0, 1, 1 << 20), None, 1 << 24, rows(0)) == 2
    assert code(B.lq_kvcache_read, c, 0, b(0, 65535, 8), None, 256, rows(256 * 4096 * 8)) == 2
    B.lq_kvcache_free(c)
