"""Low-rank adapters of many requests beside a projection, against the formula in 64 bits."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu


class Set:
    """Adapters on the GPU (scales and ranks of their own) with the same factors on the host."""

    def __init__(self, rng, K, N, max_rank, ranks, scales=None, slots=None):
        import torch
        self.K, self.N, self.ranks = K, N, list(ranks)
        self.scales = [1.0 + 0.25 * i for i in range(len(ranks))] if scales is None else scales
        self.h = B.lq_adapters_create(K, N, max_rank, slots or len(ranks), 0)
        self.A = [(rng.standard_normal((K, r)) * 0.2 / np.sqrt(K)).astype(np.float16) for r in ranks]
        self.B = [(rng.standard_normal((r, N)) * 0.3).astype(np.float16) for r in ranks]
        st = torch.cuda.current_stream().cuda_stream
        for s, r in enumerate(ranks):
            self.put(s, self.A[s], self.B[s], self.scales[s], st)
        torch.cuda.synchronize()

    def put(self, slot, A, Bf, scale, stream):
        import torch
        self.A[slot], self.B[slot], self.scales[slot], self.ranks[slot] = A, Bf, scale, A.shape[1]
        self.kept = [torch.from_numpy(A).cuda(), torch.from_numpy(Bf).cuda()]
        B.lq_adapters_set(self.h, slot, A.shape[1], self.kept[0].data_ptr(), self.kept[1].data_ptr(), scale, stream)
        torch.cuda.synchronize()

    def free(self):
        B.lq_adapters_free(self.h)


def reference(S, X, Y0, ids, f32):
    """Y in 64 bits and how far an element may be from it.  Steps of the path, each with its roundings: sums over K on the tensor core (an addition may
    cut 2^-23 of the partial sum; ceil(K / 16) of them and 24 more where warps and blocks are joined), two halves of the intermediate (2^-22 of the row's
    largest), sums over the rank (two products a 16), the scale and the last sum in fp32, one rounding to the output's type."""
    X64, Y = X.astype(np.float64), Y0.astype(np.float64)
    err = np.zeros_like(Y)
    for a, r in enumerate(S.ranks):
        rows = np.nonzero(ids == a)[0]
        if r == 0 or rows.size == 0:
            continue
        A, Bf, s = S.A[a].astype(np.float64), S.B[a].astype(np.float64), float(np.float32(S.scales[a]))
        T = X64[rows] @ A
        dT = (np.ceil(S.K / 16) + 24) * 2.0 ** -23 * (np.abs(X64[rows]) @ np.abs(A)) + 2.0 ** -22 * np.abs(T).max(1, keepdims=True)
        Y[rows] += s * (T @ Bf)
        err[rows] = abs(s) * (dT @ np.abs(Bf) + (2 * np.ceil(r / 16) + 4) * 2.0 ** -23 * (np.abs(T) @ np.abs(Bf)))
    err += 2.0 ** -23 * np.abs(Y)
    return Y, err + ((np.abs(Y) + err) * 2.0 ** -24 if f32 else (np.abs(Y) + err) * 2.0 ** -11 + 2.0 ** -25)


def forward(S, ids, X, Y0, f32, in_place=False, slots=None, M_max=None, rowmap=None):
    import torch
    M = X.shape[0]
    m = rowmap or B.lq_rowmap_create(M_max or M, slots or len(S.ranks), 0)
    st = torch.cuda.current_stream().cuda_stream
    i, x, y0 = torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(X).cuda(), torch.from_numpy(Y0).cuda()
    room = torch.full((M + 3, S.N), 7.0, dtype=y0.dtype, device="cuda")       # rows behind the last one are left alone
    if in_place:
        room[:M] = y0
        y0 = room
    B.lq_rowmap_set(m, i.data_ptr(), M, st)
    B.lq_adapters_forward(S.h, m, x.data_ptr(), y0.data_ptr(), room.data_ptr(), B.OUT_F32 if f32 else B.OUT_F16, st)
    torch.cuda.synchronize()
    if rowmap is None:
        B.lq_rowmap_free(m)
    out = room.cpu().numpy()
    assert (out[M:] == 7).all()
    assert B.lq_get_device_status(0)[0] == 0
    return out[:M]


def inputs(rng, M, K, N, f32):
    X = rng.standard_normal((M, K)).astype(np.float32)
    X[:, rng.permutation(K)[:8]] *= 20
    return X.astype(np.float16), rng.standard_normal((M, N)).astype(np.float32 if f32 else np.float16)


@pytest.mark.parametrize("M,K,N,ranks,runs,f32", [
    (1, 8, 8, [1], 1, True),
    (1, 1152, 1152, [16, 16], 1, False),
    (2, 40, 24, [3], 0, True),
    (15, 1160, 2312, [24, 7, 1], 0, True),
    (16, 256, 32, [128, 64], 1, False),
    (17, 264, 40, [128, 100], 0, True),
    (33, 8192, 64, [96, 33], 0, False),
    (64, 512, 1000, [32] * 64, 0, False),
    (127, 1152, 136, [16], 1, True),
    (129, 640, 8192, [13, 48], 3, False),
    (300, 72, 520, [64, 17, 128], 2, True),
    (1000, 1152, 1152, [32, 8, 32], 5, False),
    (1365, 1160, 2312, [24, 12, 18, 1], 0, True),
    (2500, 96, 72, [32] * 40, 0, False),
    (4096, 2240, 256, [128, 64], 4, True),
    (5000, 136, 344, [16, 1], 7, False),
    (700, 576, 520, [64, 48, 20, 64], 20, False),          # many-row form: neighbours of less than half a tile
    (261, 1152, 200, [96, 128, 70], 0, True),              # rows of three adapters in any order
    (900, 64, 8, [128] * 30, 60, False),                   # tiles of few rows, one step each
    (40000, 72, 136, [40, 40], 3, False),                  # several tiles to a CTA, runs that end inside them
])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_against_64_bits(M, K, N, ranks, runs, f32, in_place):
    rng = np.random.default_rng(M * 7 + K)
    S = Set(rng, K, N, max(ranks), ranks)
    X, Y0 = inputs(rng, M, K, N, f32)
    ids = np.arange(M) * runs // M % len(ranks) if runs else rng.permutation(np.arange(M) % len(ranks))
    if M > 10 and M % 2:                                   # some rows without an adapter
        ids[rng.random(M) < 0.2] = -1
        ids[rng.random(M) < 0.05] = len(ranks) + 3         # outside the slots: none either
    Y = forward(S, ids, X, Y0, f32, in_place)
    S.free()
    ref, bound = reference(S, X, Y0, ids, f32)
    none = (ids < 0) | (ids >= len(ranks))
    assert np.array_equal(Y[none], Y0[none])               # to the bit
    over = np.abs(Y - ref) - bound
    assert over.max() <= 0, (over.max(), np.unravel_index(over.argmax(), Y.shape))


def test_every_element_is_where_it_belongs():
    """Factors with one entry each pick a single input for a single output: no permutation of either inner order may show."""
    import torch
    K, N, r = 264, 200, 40
    rng = np.random.default_rng(5)
    S = Set(rng, K, N, r, [r], scales=[2.0])
    X = rng.integers(-30, 30, (70, K)).astype(np.float16)
    Y0 = np.zeros((70, N), np.float32)
    for k, j, n in [(0, 0, 0), (263, 39, 199), (31, 8, 33), (32, 31, 7), (100, 32, 64), (7, 17, 95)]:
        A, Bf = np.zeros((K, r), np.float16), np.zeros((r, N), np.float16)
        A[k, j], Bf[j, n] = 1, 1
        S.put(0, A, Bf, 2.0, torch.cuda.current_stream().cuda_stream)
        Y = forward(S, np.zeros(70, int), X, Y0, True)
        want = np.zeros_like(Y0)
        want[:, n] = 2 * X[:, k]
        assert np.array_equal(Y, want), (k, j, n)
    S.free()


def test_wide_magnitudes_neither_overflow_nor_vanish():
    """An intermediate beyond the halves' range, and one far below it: the row's power of two carries both."""
    import torch
    rng = np.random.default_rng(11)
    K, N = 1024, 64
    for f in (1.0, 2.0 ** -20):
        S = Set(rng, K, N, 16, [16], scales=[2.0 ** -8])
        S.put(0, (rng.standard_normal((K, 16)) * 40 * f).astype(np.float16), S.B[0], 2.0 ** -8, torch.cuda.current_stream().cuda_stream)
        X = (rng.standard_normal((40, K)) * 200).astype(np.float16)
        X[7] = np.clip(X[7].astype(np.float32) * 100, -60000, 60000)      # rows side by side, each with its own scale
        X[8] = 0
        Y0 = np.zeros((40, N), np.float32)
        Y = forward(S, np.zeros(40, int), X, Y0, True)
        ref, bound = reference(S, X, Y0, np.zeros(40, int), True)
        assert np.abs(X.astype(np.float64) @ S.A[0].astype(np.float64)).max() > 65504 * f
        assert (np.abs(Y - ref) <= bound).all() and not Y[8].any()
        S.free()


def test_a_slot_is_replaced_and_emptied_in_stream_order():
    import torch
    rng = np.random.default_rng(2)
    K, N, M = 128, 96, 50
    S = Set(rng, K, N, 32, [32, 8], slots=5)
    X, Y0 = inputs(rng, M, K, N, True)
    ids = np.arange(M) % 4                                 # slots 2 and 3 have never been filled
    first = forward(S, ids, X, Y0, True, slots=5)
    assert np.array_equal(first[ids >= 2], Y0[ids >= 2])
    A, Bf = (rng.standard_normal((K, 20)) * 0.1).astype(np.float16), rng.standard_normal((20, N)).astype(np.float16)
    S.put(1, A, Bf, -0.5, torch.cuda.current_stream().cuda_stream)      # a lower and then a higher rank than before
    again = forward(S, ids, X, Y0, True, slots=5)
    ref, bound = reference(S, X, Y0, ids, True)
    assert np.array_equal(again[ids != 1], first[ids != 1]) and (np.abs(again - ref) <= bound).all()
    B.lq_adapters_set(S.h, 0, 0, None, None, 1.0, torch.cuda.current_stream().cuda_stream)
    S.ranks[0] = 0
    last = forward(S, ids, X, Y0, True, slots=5)
    assert np.array_equal(last[ids != 1], Y0[ids != 1]) and np.array_equal(last[ids == 1], again[ids == 1])
    S.free()


@pytest.mark.parametrize("M", [150, 1500, 3000])
@pytest.mark.parametrize("in_place", [False, True])
def test_empty_slots_are_no_adapters(M, in_place):
    """Slots that hold nothing, between others: their rows keep Y0, also where whole tiles are theirs."""
    rng = np.random.default_rng(M)
    S = Set(rng, 200, 264, 64, [40, 64], slots=6)
    X, Y0 = inputs(rng, M, 200, 264, False)
    ids = (np.arange(M) * 11 // M) % 6
    Y = forward(S, ids, X, Y0, False, in_place, slots=6)
    ref, bound = reference(S, X, Y0, ids, False)
    assert np.array_equal(Y[ids >= 2], Y0[ids >= 2]) and (np.abs(Y - ref) <= bound).all()
    S.free()


def test_the_most_slots_and_rows_of_each():
    rng = np.random.default_rng(21)
    S = Set(rng, 64, 40, 8, [8] * 5, slots=1023)
    for M in (1023, 5000):
        X, Y0 = inputs(rng, M, 64, 40, True)
        ids = rng.permutation(np.arange(M) % 1023)         # a row or a few for every slot, five of which hold something
        Y = forward(S, ids, X, Y0, True, slots=1023)
        ref, bound = reference(S, X, Y0, ids, True)
        assert np.array_equal(Y[ids >= 5], Y0[ids >= 5]) and (np.abs(Y - ref) <= bound).all()
    S.free()


def test_equal_calls_give_equal_bits_and_a_map_is_used_again():
    rng = np.random.default_rng(3)
    S = Set(rng, 1152, 576, 32, [32, 16, 8])
    m = B.lq_rowmap_create(3000, 3, 0)
    got = []
    for M in (3000, 70, 1, 2000, 70, 3000):
        r = np.random.default_rng(M)
        X, Y0 = inputs(r, M, 1152, 576, False)
        ids = r.integers(-1, 3, M)
        Y = forward(S, ids, X, Y0, False, rowmap=m)
        ref, bound = reference(S, X, Y0, ids, False)
        assert (np.abs(Y - ref) <= bound).all(), M
        got.append(Y)
    assert np.array_equal(got[0], got[5]) and np.array_equal(got[1], got[4])
    B.lq_rowmap_free(m)
    S.free()


def test_captured_calls_follow_the_array_that_they_read():
    """A graph that sorts and adds: each replay goes by what the row array and the inputs hold by then."""
    import torch
    rng = np.random.default_rng(4)
    K, N, M = 640, 320, 600
    S = Set(rng, K, N, 32, [32, 16, 24])
    m = B.lq_rowmap_create(M, 3, 0)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    x, y0, y = (torch.zeros(M, c, dtype=torch.float16, device="cuda") for c in (K, N, N))
    side = torch.cuda.Stream()

    def call(st):
        B.lq_rowmap_set(m, ids.data_ptr(), M, st)
        B.lq_adapters_forward(S.h, m, x.data_ptr(), y0.data_ptr(), y.data_ptr(), B.OUT_F16, st)

    side.wait_stream(torch.cuda.current_stream())
    call(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(torch.cuda.current_stream().cuda_stream)
    for seed in range(3):
        r = np.random.default_rng(seed)
        X, Y0 = inputs(r, M, K, N, False)
        i = r.integers(-1, 3, M) if seed else np.zeros(M, int)
        ids.copy_(torch.from_numpy(i.astype(np.int32)))
        x.copy_(torch.from_numpy(X))
        y0.copy_(torch.from_numpy(Y0))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ref, bound = reference(S, X, Y0, i, False)
        assert (np.abs(y.cpu().numpy() - ref) <= bound).all(), seed
    del graph
    B.lq_rowmap_free(m)
    S.free()


def test_a_nan_in_one_row_stays_there():
    rng = np.random.default_rng(6)
    S = Set(rng, 320, 160, 16, [16])
    for M in (20, 700):
        X, Y0 = inputs(rng, M, 320, 160, True)
        ids = np.zeros(M, int)
        ids[3] = -1
        X[5, 100] = np.nan
        X[3] = np.inf                                      # no adapter: never looked at
        Y = forward(S, ids, X, Y0, True)
        bad = ~np.isfinite(Y).all(1)
        assert bad[5] and bad.sum() == 1
    S.free()


def test_refusals():
    import torch
    S = Set(np.random.default_rng(1), 64, 64, 20, [8, 8])
    m, big = B.lq_rowmap_create(10, 2, 0), B.lq_rowmap_create(10, 3, 0)
    x = torch.zeros(64, 64, dtype=torch.float16, device="cuda")
    i = torch.zeros(16, dtype=torch.int32, device="cuda")
    P = x.data_ptr()

    def code(f, *a):
        with pytest.raises(B.LqError) as e:
            f(*a)
        return e.value.code

    assert code(B.lq_adapters_forward, S.h, m, P, P, P, B.OUT_F16, 0) == 1            # the map holds no rows yet
    assert code(B.lq_rowmap_set, m, i.data_ptr(), 11, 0) == 1                         # more rows than it was made for
    assert code(B.lq_rowmap_set, m, i.data_ptr(), 0, 0) == 1
    assert code(B.lq_rowmap_set, m, i.data_ptr() + 2, 4, 0) == 1
    assert code(B.lq_rowmap_set, m, None, 4, 0) == 1
    for r in (m, big):
        B.lq_rowmap_set(r, i.data_ptr(), 4, 0)
    assert code(B.lq_adapters_forward, S.h, big, P, P, P, B.OUT_F16, 0) == 1          # a map of more slots than the set has
    assert code(B.lq_adapters_forward, S.h, m, P, P, P, 2, 0) == 1
    for bad in ((P + 8, P, P), (P, P + 2, P), (P, P, P + 4), (None, P, P), (P, None, P), (P, P, None)):
        assert code(B.lq_adapters_forward, S.h, m, *bad, B.OUT_F16, 0) == 1
    assert code(B.lq_adapters_set, S.h, 2, 8, P, P, 1.0, 0) == 1                      # no such slot
    assert code(B.lq_adapters_set, S.h, -1, 8, P, P, 1.0, 0) == 1
    assert code(B.lq_adapters_set, S.h, 0, -1, P, P, 1.0, 0) == 1
    assert code(B.lq_adapters_set, S.h, 0, 21, P, P, 1.0, 0) == 2                     # above max_rank
    assert code(B.lq_adapters_set, S.h, 0, 8, None, P, 1.0, 0) == 1
    assert code(B.lq_adapters_set, S.h, 0, 8, P, P, float("nan"), 0) == 6
    torch.cuda.synchronize()
    for r in (m, big):
        B.lq_rowmap_free(r)
    S.free()


@pytest.mark.parametrize("M,other", [(40, 100), (2000, 2500)])
def test_a_map_that_a_replayed_graph_has_set_is_not_another_forwards(M, other):
    """The rows of a map are those of the call that ran last on the device; a forward of another number writes nothing and says so."""
    import torch
    rng = np.random.default_rng(7)
    K, N = 64, 64
    S = Set(rng, K, N, 16, [16, 8])
    m = B.lq_rowmap_create(other, 2, 0)
    ids = torch.arange(other, dtype=torch.int32, device="cuda") % 2
    X, Y0 = inputs(rng, other, K, N, False)
    x, y0, y = torch.from_numpy(X).cuda(), torch.from_numpy(Y0).cuda(), torch.full((other, N), 5.0, dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    forward_ = lambda: B.lq_adapters_forward(S.h, m, x.data_ptr(), y0.data_ptr(), y.data_ptr(), B.OUT_F16, side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):             # captured, not run: the map has no rows yet
        B.lq_rowmap_set(m, ids.data_ptr(), other, torch.cuda.current_stream().cuda_stream)
    for replay in (False, True):
        if replay:
            B.lq_rowmap_set(m, ids.data_ptr(), M, side.cuda_stream)
            side.synchronize()
            graph.replay()
            torch.cuda.synchronize()
        forward_()
        torch.cuda.synchronize()
        assert (y == 5).all() and B.lq_get_device_status(0)[0] == 1 and B.lq_get_device_status(0)[0] == 0
    B.lq_rowmap_set(m, ids.data_ptr(), M, side.cuda_stream)
    forward_()
    torch.cuda.synchronize()
    ref, bound = reference(S, X[:M], Y0[:M], np.arange(M) % 2, False)
    assert (np.abs(y.cpu().numpy()[:M] - ref) <= bound).all() and (y[M:] == 5).all() and B.lq_get_device_status(0)[0] == 0
    del graph
    B.lq_rowmap_free(m)
    S.free()


def test_outputs_that_share_memory_with_inputs_are_refused():
    import torch
    S = Set(np.random.default_rng(8), 64, 64, 8, [8])
    m = B.lq_rowmap_create(32, 1, 0)
    B.lq_rowmap_set(m, torch.zeros(32, dtype=torch.int32, device="cuda").data_ptr(), 32, 0)
    torch.cuda.synchronize()
    t = torch.zeros(3 * 32 * 64, dtype=torch.float16, device="cuda")
    at = lambda row: t.data_ptr() + row * 128
    st = torch.cuda.current_stream().cuda_stream
    for x, y0, y in ((0, 32, 33), (0, 33, 32), (0, 32, 63), (0, 32, 0), (0, 64, 31), (32, 64, 1)):
        with pytest.raises(B.LqError) as e:
            B.lq_adapters_forward(S.h, m, at(x), at(y0), at(y), B.OUT_F16, st)
        assert e.value.code == 1, (x, y0, y)
    B.lq_adapters_forward(S.h, m, at(0), at(32), at(64), B.OUT_F16, st)
    B.lq_adapters_forward(S.h, m, at(0), at(32), at(32), B.OUT_F16, st)
    B.lq_adapters_forward(S.h, m, at(0), at(0), at(32), B.OUT_F16, st)
    torch.cuda.synchronize()
    B.lq_rowmap_free(m)
    S.free()


@pytest.mark.parametrize("rank,max_rank", [(8, 8), (30, 128)])
def test_outputs_behind_four_billion_elements(rank, max_rank):
    """Rows whose elements lie behind 2^32 of them, neighbours and scattered, in place."""
    import torch
    rng = np.random.default_rng(9)
    K, N, M = 8, 8192, (1 << 19) + 777
    S = Set(rng, K, N, max_rank, [rank, rank])
    X = rng.standard_normal((M, K)).astype(np.float16)
    for scattered in (False, True):
        ids = np.arange(M) % 3 if scattered else np.arange(M) // 200000
        look = np.r_[0:5, 199998:200003, 400000 - 3:400003, (1 << 19) - 4:(1 << 19) + 4, M - 300:M]
        y = torch.empty(M, N, dtype=torch.float16, device="cuda").fill_(0.5)
        x, i = torch.from_numpy(X).cuda(), torch.from_numpy(ids.astype(np.int32)).cuda()
        m = B.lq_rowmap_create(M, 2, 0)
        st = torch.cuda.current_stream().cuda_stream
        B.lq_rowmap_set(m, i.data_ptr(), M, st)
        B.lq_adapters_forward(S.h, m, x.data_ptr(), y.data_ptr(), y.data_ptr(), B.OUT_F16, st)
        torch.cuda.synchronize()
        ref, bound = reference(S, X[look], np.full((look.size, N), 0.5, np.float16), ids[look], False)
        got = y[torch.from_numpy(look).cuda()].cpu().numpy()
        assert (np.abs(got - ref) <= bound).all()
        assert bool((y[i == 2] == 0.5).all()) and bool((y[i < 2] != 0.5).any(1).all())
        del y
        B.lq_rowmap_free(m)
    assert B.lq_get_device_status(0)[0] == 0
    S.free()


def test_a_thousand_slots_of_which_few_are_used():
    rng = np.random.default_rng(10)
    S = Set(rng, 128, 136, 16, [16, 8, 5], slots=1023)
    for M in (1, 130, 1537, 9000):
        X, Y0 = inputs(rng, M, 128, 136, False)
        ids = rng.integers(-1, 3, M)
        Y = forward(S, ids, X, Y0, False, slots=1023)
        ref, bound = reference(S, X, Y0, ids, False)
        assert (np.abs(Y - ref) <= bound).all(), M
    S.free()


@pytest.mark.parametrize("M,K,max_rank,used", [(1600, 2048, 16, 300), (1700, 1160, 128, 200), (700, 320, 64, 400), (5000, 640, 40, 600)])
@pytest.mark.parametrize("none", [False, True])
def test_more_tiles_than_are_at_work_at_once(M, K, max_rank, used, none):
    rng = np.random.default_rng(M)
    N = 72
    S = Set(rng, K, N, max_rank, [int(r) for r in rng.integers(0, max_rank + 1, used)], slots=used)
    X, Y0 = inputs(rng, M, K, N, True)
    ids = rng.integers(-1 if none else 0, used, M)
    Y = forward(S, ids, X, Y0, True)
    ref, bound = reference(S, X, Y0, ids, True)
    assert (np.abs(Y - ref) <= bound).all()
    S.free()


@pytest.mark.parametrize("M,K,N,rank,f32", [(8192, 512, 2240, 128, False), (16384, 512, 2304, 100, False), (4096, 64, 4000, 128, True), (8192, 128, 2304, 32, False),
                                            (1400, 1160, 2312, 24, True)])
def test_pass_after_pass_gives_the_same_bits(M, K, N, rank, f32):
    """Many passes back to back: what a copy ahead, or a store behind, overwrites too early differs from pass to pass."""
    import torch
    rng = np.random.default_rng(12)
    S = Set(rng, K, N, rank, [rank] * 3)
    X, Y0 = inputs(rng, M, K, N, f32)
    ids = np.arange(M) * 4 // M - 1
    m = B.lq_rowmap_create(M, 3, 0)
    st = torch.cuda.current_stream().cuda_stream
    i, x, y0 = torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(X).cuda(), torch.from_numpy(Y0).cuda()
    ys = [torch.empty_like(y0) for _ in range(2)]
    B.lq_rowmap_set(m, i.data_ptr(), M, st)
    for turn in range(30):
        for _ in range(3):
            for y in ys if turn else ys[:1]:
                B.lq_adapters_forward(S.h, m, x.data_ptr(), y0.data_ptr(), y.data_ptr(), B.OUT_F32 if f32 else B.OUT_F16, st)
        if turn == 0:
            first = ys[0].clone()
        else:
            assert all(torch.equal(first, y) for y in ys), turn
    look = rng.permutation(M)[:700]
    ref, bound = reference(S, X[look], Y0[look], ids[look], f32)
    assert (np.abs(first.cpu().numpy()[look] - ref) <= bound).all()
    B.lq_rowmap_free(m)
    S.free()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rank", [65, 96, 128])
def test_few_rows_of_wide_factors(rank, f32):
    """From one row on these have tiles of 128 rows, up to 16 rows fetched four at a time."""
    rng = np.random.default_rng(rank)
    for K, N in ((8, 8), (200, 136), (2048, 320)):
        S = Set(rng, K, N, rank, [rank, 1, 0, rank // 2])
        for M in (1, 2, 4, 5, 15, 16, 17, 33, 129):
            X, Y0 = inputs(rng, M, K, N, f32)
            for ids in (np.zeros(M, int), rng.integers(-1, 5, M), np.full(M, 2), np.arange(M) * 3 // M):
                Y = forward(S, ids, X, Y0, f32, in_place=bool(M & 1))
                ref, bound = reference(S, X, Y0, ids, f32)
                assert (np.abs(Y - ref) <= bound).all(), (K, M)
        S.free()


@pytest.mark.parametrize("M", [20, 1600])
@pytest.mark.parametrize("max_rank", [16, 128])
def test_the_largest_scale_and_sums(M, max_rank):
    """The largest sums of X A that halves make, under the largest scale: right where the result is a float, Y0 where B is zero.  Scales above
    are refused."""
    rng = np.random.default_rng(13)
    K, N = 8192, 40
    top = float(np.nextafter(np.float32(2.0 ** 96), np.float32(0)))
    S = Set(rng, K, N, max_rank, [8], scales=[top])
    A, Bf = np.full((K, 8), 65504, np.float16), np.zeros((8, N), np.float16)
    Bf[0, 8:16], Bf[0, 16:24] = 2.0 ** -24, -2.0 ** -24
    S.put(0, A, Bf, top, 0)
    X = np.where(np.arange(M)[:, None] % 2 == 0, 65504, rng.integers(0, 2, (M, K))).astype(np.float16)
    Y0 = rng.standard_normal((M, N)).astype(np.float32)
    Y = forward(S, np.zeros(M, int), X, Y0, True)
    ref, bound = reference(S, X, Y0, np.zeros(M, int), True)
    assert np.array_equal(Y[:, :8], Y0[:, :8]) and np.array_equal(Y[:, 24:], Y0[:, 24:])
    assert np.abs(ref).max() > 2.0 ** 116 and (np.abs(Y - ref) <= bound).all()
    for scale in (2.0 ** 96, -2.0 ** 96, 3e38):
        with pytest.raises(B.LqError) as e:
            S.put(0, A, Bf, scale, 0)
        assert e.value.code == 2
    B.lq_adapters_set(S.h, 0, 0, None, None, 3e38, 0)       # an empty slot has none
    S.ranks[0] = 0
    assert np.array_equal(forward(S, np.zeros(M, int), X, Y0, True), Y0)
    S.free()


@pytest.mark.parametrize("M,K,N,rank,f32", [(1600, 64, 512, 32, False), (2100, 72, 640, 128, True), (4096, 512, 2304, 128, False), (8192, 1152, 1152, 32, True),
                                            (700, 256, 512, 24, False)])
def test_many_rows_follow_what_changes_from_pass_to_pass(M, K, N, rank, f32):
    """Map, factors, X and Y0 are other ones in each pass, written by the kernels right before, of which each lets the next one start early; nothing
    waits on the host.  Queued, captured and replayed the bits are those of calls that wait for each other."""
    import torch
    rng = np.random.default_rng(M + rank)
    passes, slots, dt = 5, 6, torch.float32 if f32 else torch.float16
    S = Set(rng, K, N, rank, [rank] * slots)
    m = B.lq_rowmap_create(M, slots, 0)
    none = B.lq_rope_create(B.lq_rope_config_default([]), 0)
    code = B.OUT_F32 if f32 else B.OUT_F16
    ids = torch.empty(passes, M, dtype=torch.int32, device="cuda")
    x = torch.empty(passes, M, K, dtype=torch.float16, device="cuda")
    src = torch.empty(passes, M, N, dtype=dt, device="cuda")
    y0, y = torch.empty(M, N, dtype=dt, device="cuda"), torch.empty(passes, M, N, dtype=dt, device="cuda")
    A = [torch.from_numpy((rng.standard_normal((K, rank)) / np.sqrt(K)).astype(np.float16)).cuda() for _ in range(passes)]
    Bf = [torch.from_numpy((rng.standard_normal((rank, N)) * 0.3).astype(np.float16)).cuda() for _ in range(passes)]

    def fill(seed):
        r = np.random.default_rng(seed)
        for k in range(passes):                            # neighbours in one pass, scattered in the next
            i = np.arange(M) * 7 // M - 1 if k % 2 else r.integers(-1, slots, M)
            ids[k].copy_(torch.from_numpy(((i + seed) % (slots + 1) - 1).astype(np.int32)))
            x[k].copy_(torch.from_numpy(r.standard_normal((M, K)).astype(np.float16)))
            src[k].copy_(torch.from_numpy(r.standard_normal((M, N)).astype(np.float16)).to(dt))
        y.fill_(7)
        torch.cuda.synchronize()

    first = [(torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda()) for a, b in zip(S.A, S.B)]

    def run(st, wait):
        # (every run begins with the first factors in all slots)
        calls = [lambda s=s, a=a, b=b: B.lq_adapters_set(S.h, s, rank, a.data_ptr(), b.data_ptr(), S.scales[s], st) for s, (a, b) in enumerate(first)]
        for k in range(passes):
            heads = lambda k=k: B.lq_qk_norm_rope(B.lq_heads(src[k].data_ptr(), (0, N, 64), y0.data_ptr(), (0, N, 64), N // 64), None, 64, 1, M, B.NORM_RMS,
                                                  1e-6, none, None, code, code, st)
            sort = lambda k=k: B.lq_rowmap_set(m, ids[k].data_ptr(), M, st)
            put = lambda k=k: B.lq_adapters_set(S.h, k % slots, rank, A[k].data_ptr(), Bf[k].data_ptr(), 1.0 - k, st)
            calls += [(heads, sort, put), (sort, put, heads), (put, heads, sort)][k % 3]
            calls.append(lambda k=k: B.lq_adapters_forward(S.h, m, x[k].data_ptr(), y0.data_ptr(), y[k].data_ptr(), code, st))
            calls.append(lambda k=k: B.lq_adapters_forward(S.h, m, x[k].data_ptr(), y[k].data_ptr(), y[k].data_ptr(), code, st))
        for c in calls:
            c()
            if wait:
                torch.cuda.synchronize()

    side = torch.cuda.Stream()
    graph = None
    for seed in range(3):
        fill(seed)
        run(side.cuda_stream, True)
        want = y.clone()
        for turn in range(6):
            y.fill_(7)
            torch.cuda.synchronize()
            run(side.cuda_stream, False)
            torch.cuda.synchronize()
            assert torch.equal(y, want), (seed, turn)
        if graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                run(torch.cuda.current_stream().cuda_stream, False)
        for turn in range(6):
            y.fill_(7)
            torch.cuda.synchronize()
            graph.replay()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want), (seed, turn, "replayed")
    # the last pass against the formula, twice the adapters on its Y0
    look = rng.permutation(M)[:300]
    k = passes - 1
    for j in range(passes):
        S.A[j], S.B[j], S.scales[j] = A[j].cpu().numpy(), Bf[j].cpu().numpy(), 1.0 - j
    X, i, Y0 = x[k].cpu().numpy()[look], ids[k].cpu().numpy()[look], y0.cpu().numpy()[look]
    once, bound = reference(S, X, Y0, i, f32)
    ref, more = reference(S, X, once, i, f32)
    assert (np.abs(y[k].cpu().numpy()[look] - ref) <= bound + more).all()
    assert B.lq_get_device_status(0)[0] == 0
    del graph
    B.lq_rowmap_free(m)
    B.lq_rope_free(none)
    S.free()


@pytest.mark.parametrize("K,N,rank,f32", [(64, 512, 32, False), (640, 1152, 128, True)])
def test_two_threads_on_one_stream(K, N, rank, f32):
    """Two threads, each with maps and buffers of its own, one set, one stream: a launch of the other may come between any two of a call's.  The map
    changes from call to call, and between maps of one thread the rows' number too."""
    import threading
    import torch
    rng = np.random.default_rng(14)
    dt, code, passes = torch.float32 if f32 else torch.float16, B.OUT_F32 if f32 else B.OUT_F16, 12
    S = Set(rng, K, N, rank, [rank] * 4)
    none = B.lq_rope_create(B.lq_rope_config_default([]), 0)
    side = torch.cuda.Stream()

    class Work:
        def __init__(self, seed, sizes):
            r = torch.Generator(device="cuda").manual_seed(seed)
            M = max(sizes)
            self.sizes = [sizes[k % len(sizes)] for k in range(passes)]
            self.map = B.lq_rowmap_create(M, 4, 0)
            self.ids = torch.randint(-1, 4, (passes, M), generator=r, device="cuda", dtype=torch.int32)
            self.ids[1::2] = self.ids[1::2].sort(dim=1).values
            self.x = torch.randn(passes, M, K, generator=r, device="cuda").half()
            self.src = torch.randn(passes, M, N, generator=r, device="cuda").to(dt)
            self.y = torch.full((passes, M, N), 7.0, dtype=dt, device="cuda")

        def run(self, wait=False):
            st = side.cuda_stream
            for k, M in enumerate(self.sizes):
                y = self.y[k].data_ptr()
                B.lq_rowmap_set(self.map, self.ids[k].data_ptr(), M, st)
                B.lq_qk_norm_rope(B.lq_heads(self.src[k].data_ptr(), (0, N, 64), y, (0, N, 64), N // 64), None, 64, 1, M, B.NORM_RMS, 1e-6, none, None,
                                  code, code, st)
                B.lq_adapters_forward(S.h, self.map, self.x[k].data_ptr(), y, y, code, st)
                if wait:
                    torch.cuda.synchronize()

    work = [Work(1, (1800, 2500)), Work(2, (3000, 1700, 1600))]
    torch.cuda.synchronize()
    want = []
    for w in work:
        w.run(wait=True)
        want.append(w.y.clone())
    for turn in range(25):
        for w in work:
            w.y.fill_(7)
        torch.cuda.synchronize()
        threads = [threading.Thread(target=w.run) for w in work]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert all(torch.equal(w.y, v) for w, v in zip(work, want)), turn
    assert B.lq_get_device_status(0)[0] == 0
    for w in work:
        B.lq_rowmap_free(w.map)
    B.lq_rope_free(none)
    S.free()
