"""The token embedding and its table's gradient against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as O
from paper_2506_13996_amd import binding as B
from tests import step_util as U

pytestmark = pytest.mark.gpu
IGN = -100


def _tokens(law, N, V, seed=0):
    rng = np.random.default_rng(seed)
    if law == "same":
        t = np.full(N, V - 1)
    elif law == "distinct":
        t = rng.permutation(np.arange(N) % V)
    elif law == "ignored":
        t = np.full(N, IGN)
    elif law == "two":          # long runs of two tokens and single ones between
        t = np.where(rng.random(N) < 0.9, np.where(rng.random(N) < 0.5, 0, V - 1), rng.integers(0, V, N))
    else:
        w = np.arange(1, V + 1) ** -1.1
        t = rng.choice(V, N, p=w / w.sum())
    t = t.astype(np.int32)
    if law in ("zipf", "two") and N > 4:
        t[rng.random(N) < 0.1] = IGN
    return t


def _backward(t, dy, V, scale=1.0, ignore=IGN, flags=0, start=None):
    N, H = dy.shape
    dtype = torch.float32 if flags & B.ALST_FLAG_DW_FP32 else torch.bfloat16
    dE = U.Guarded((V, H), dtype)
    if start is not None:
        dE.t.copy_(start)
    ws = U.guarded_workspace(B.alst_embedding_workspace_bytes(N, H, V))
    B.alst_embedding_backward(torch.from_numpy(t).cuda(), dy.cuda(), scale, ignore, dE=dE.t, workspace=ws.t, flags=flags)
    status = B.alst_last_device_status(ws.t)
    torch.cuda.synchronize()
    assert dE.intact() and ws.intact()
    return dE.t, status


def _check_backward(got, t, dy, V, scale=1.0, ignore=IGN, start=None):
    want, mag, rows = O.embedding_backward(t, U.to64(dy), scale, ignore, V)
    old = U.to64(start) if start is not None else np.zeros_like(want)
    # a row's terms are added one after the other inside a range and range by range: no more additions than rows, + scale, old
    U.check("dE", got, want + old, mag + np.abs(old), rows[:, None] + 2.0)


@pytest.mark.parametrize("N,H,V", [(1, 8, 1), (1, 64, 50), (2, 512, 7), (33, 520, 512), (4097, 72, 513), (700, 1600, 5003)])
@pytest.mark.parametrize("fp32", [False, True])
def test_forward(N, H, V, fp32):
    g = torch.Generator().manual_seed(N + H)
    E, t = U.bf16((V, H), g), _tokens("zipf", N, V)
    y = U.Guarded((N, H), torch.float32 if fp32 else torch.bfloat16)
    status = torch.full((1,), 123, dtype=torch.int32, device="cuda")
    B.alst_embedding_forward(torch.from_numpy(t).cuda(), E.cuda(), 1.7, IGN, y=y.t, device_status_out=status,
                             flags=B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0)
    want = O.embedding_forward(t, U.to64(E), float(np.float32(1.7)), IGN)
    U.check("y", y.t, want, np.abs(want), 1)
    assert y.intact() and int(status) == 123            # written only for a token out of range


def test_forward_reports_tokens_out_of_range_and_gives_them_zeros():
    V, H = 10, 64
    E = torch.ones((V, H), dtype=torch.bfloat16, device="cuda")
    for bad in (V, -1, 2 ** 31 - 1, -2 ** 31):
        t = torch.tensor([3, bad, IGN, 0], dtype=torch.int32, device="cuda")
        y = U.Guarded((4, H), torch.bfloat16)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.alst_embedding_forward(t, E, y=y.t, device_status_out=status)
        assert int(status) == B.ALST_ERR_LABEL_RANGE
        assert y.t[:, 0].tolist() == [1, 0, 0, 1] and y.intact()
    # rows of zeros do not go by the scale
    B.alst_embedding_forward(torch.tensor([3, IGN, 1, IGN], dtype=torch.int32, device="cuda"), E, float("inf"), y=y.t)
    assert y.t[:, 0].tolist() == [float("inf"), 0, float("inf"), 0]
    # an ignore_index inside the vocabulary
    B.alst_embedding_forward(torch.tensor([3, 0, 3, 0], dtype=torch.int32, device="cuda"), E, 1.0, 3, y=y.t)
    assert y.t[:, 0].tolist() == [0, 1, 0, 1]


@pytest.mark.parametrize("N,H,V", [(1, 8, 1), (1, 520, 513), (2, 64, 2), (31, 8, 512), (32, 512, 7), (33, 72, 511), (64, 8, 64),
                                   (65, 1024, 100), (1000, 1600, 5003), (4096, 64, 1000), (4097, 64, 1000), (20000, 136, 3000)])
@pytest.mark.parametrize("law", ["zipf", "same", "distinct", "ignored", "two"])
def test_backward(N, H, V, law):
    g = torch.Generator().manual_seed(N)
    t, dy = _tokens(law, N, V), U.bf16((N, H), g)
    got, status = _backward(t, dy, V, scale=0.5)
    _check_backward(got, t, dy, V, scale=0.5)
    assert status == B.ALST_OK


def _by_lengths(lengths, seed=0):
    """Tokens 1, 3, 5, ... with these numbers of rows, in random order."""
    t = np.repeat(np.arange(len(lengths)) * 2 + 1, lengths).astype(np.int32)
    np.random.default_rng(seed).shuffle(t)
    return t, 2 * len(lengths) + 2


@pytest.mark.parametrize("run,rows", [(8, 2000), (16, 70000), (128, 600000)])
@pytest.mark.parametrize("first", [0, 1, 5])
def test_tokens_whose_rows_end_at_and_beside_the_ranges_of_the_sums(run, rows, first):
    """Sorted rows are added up in ranges of 8 rows in short calls and of 128 in long ones (at 8 columns): tokens that fill a range, end
    or begin with one, lie in two, and go through one, two and many."""
    some = [first, run - first, run, run, 2 * run, run - 1, 1, run + 1, run - 1, 1, 2 * run - 1, 1, 3 * run, run // 2, run, run // 2,
            run // 2, 2 * run, run // 2, run // 2, 4 * run + 3, run - 3, 9 * run + 1, run - 1, 20 * run, 2, run - 2, 1]
    some = [n for n in some if n]
    lengths = some * (rows // sum(some)) + [rows % sum(some) + 1]
    t, V = _by_lengths(lengths)
    assert len(t) in (rows, rows + 1)
    g = torch.Generator().manual_seed(run)
    dy = U.bf16((len(t), 8), g)
    got, _ = _backward(t, dy, V, flags=B.ALST_FLAG_DW_FP32)
    index = torch.from_numpy(t).long()
    want = torch.zeros((V, 8), dtype=torch.float64).index_add_(0, index, dy.double()).numpy()
    mag = torch.zeros((V, 8), dtype=torch.float64).index_add_(0, index, dy.double().abs()).numpy()
    U.check("dE", got, want, mag, np.bincount(t, minlength=V)[:, None] + 2.0)


LONG = [(600001, 8, 70000), (1 << 20, 8, 300), ((1 << 20) + 1, 8, 300)]


@pytest.mark.parametrize("N,H,V,law", [(*s, law) for s in LONG for law in ("zipf", "same", "two")] +
                         [(59000, 4104, 900, law) for law in ("zipf", "same")])
def test_backward_of_long_calls(N, H, V, law):
    """Long ranges, shares of the sort above 4096 rows (from 2^20 rows on), more than 512 columns times 8."""
    t = _tokens(law, N, V, 5)
    dy = U.bf16((N, H), torch.Generator().manual_seed(N))
    got, status = _backward(t, dy, V, flags=B.ALST_FLAG_DW_FP32)
    keep = torch.from_numpy(t != IGN)
    index = torch.from_numpy(t)[keep].long()
    want = torch.zeros((V, H), dtype=torch.float64).index_add_(0, index, dy[keep].double())
    mag = torch.zeros((V, H), dtype=torch.float64).index_add_(0, index, dy[keep].double().abs())
    rows = np.bincount(t[t != IGN], minlength=V)[:, None]
    # 128 rows of a range, the partial sums of a wavefront (an eighth of a token's ranges), eight wavefronts, scale
    U.check("dE", got, U.to64(want), U.to64(mag), np.minimum(rows, 128 + rows / 1024 + 8) + 2.0)
    assert status == B.ALST_OK


@pytest.mark.parametrize("V", [(1 << 18) - 1, 1 << 18, 1 << 20, 1 << 24])
def test_backward_of_large_vocabularies(V):
    """The number of the sort's passes changes at 2^18 tokens and at 2^27."""
    N, H = 5000, 8
    g = torch.Generator().manual_seed(V)
    rng = np.random.default_rng(V)
    t = np.concatenate([rng.integers(0, V, N - 40), np.repeat([0, V - 1], 20)]).astype(np.int32)
    rng.shuffle(t)
    dy = U.bf16((N, H), g)
    got, _ = _backward(t, dy, V)
    want = torch.zeros((V, H), dtype=torch.float64).index_add_(0, torch.from_numpy(t).long(), dy.double())
    mag = torch.zeros((V, H), dtype=torch.float64).index_add_(0, torch.from_numpy(t).long(), dy.double().abs())
    U.check("dE", got, want.numpy(), mag.numpy(), 42)


@pytest.mark.parametrize("fp32_rows", [False, True])
@pytest.mark.parametrize("fp32_sums", [False, True])
@pytest.mark.parametrize("accumulate", [False, True])
def test_backward_types_and_accumulation(fp32_rows, fp32_sums, accumulate):
    N, H, V = 3001, 200, 700
    g = torch.Generator().manual_seed(7)
    t = _tokens("zipf", N, V, 3)
    t[t == 5] = 6                       # a token that does not occur
    dy = torch.randn((N, H), generator=g) if fp32_rows else U.bf16((N, H), g)
    flags = (B.ALST_FLAG_RESIDUAL_FP32 if fp32_rows else 0) | (B.ALST_FLAG_DW_FP32 if fp32_sums else 0)
    start = None
    if accumulate:
        flags |= B.ALST_FLAG_DW_ACCUMULATE
        start = torch.randn((V, H), generator=g).to(torch.float32 if fp32_sums else torch.bfloat16)
        start[5] = float("nan")         # is neither read nor written
    got, _ = _backward(t, dy, V, scale=3.0, flags=flags, start=start)
    if accumulate:
        assert torch.isnan(got[5]).all()
        got[5] = start[5] = 0
    _check_backward(got, t, dy, V, scale=3.0, start=start)


def test_backward_leaves_out_ignored_rows_whatever_they_hold():
    N, H, V = 500, 64, 40
    g = torch.Generator().manual_seed(1)
    rng = np.random.default_rng(1)
    t, dy = rng.integers(0, V, N).astype(np.int32), U.bf16((N, H), g)
    out = rng.random(N) < 0.3
    t[out] = rng.choice([IGN, V, -1, 2 ** 31 - 1, -2 ** 31], out.sum())
    dy[torch.from_numpy(out)] = float("nan")
    dy[torch.from_numpy(out.nonzero()[0][::3])] = float("inf")
    got, status = _backward(t, dy, V)
    assert status == B.ALST_ERR_LABEL_RANGE
    dy[torch.from_numpy(out)] = 0
    _check_backward(got, t, dy, V)
    # an ignore_index inside the vocabulary: that row of dE is zeros
    t = rng.integers(0, V, N).astype(np.int32)
    got, status = _backward(t, dy, V, ignore=4)
    assert status == B.ALST_OK and (got[4] == 0).all()
    _check_backward(got, t, dy, V, ignore=4)


def test_backward_gives_the_same_bits_every_time_and_on_another_stream():
    N, H, V = 9000, 264, 300
    g = torch.Generator().manual_seed(2)
    t, dy = _tokens("zipf", N, V), torch.randn((N, H), generator=g)
    flags = B.ALST_FLAG_RESIDUAL_FP32 | B.ALST_FLAG_DW_FP32
    first, _ = _backward(t, dy, V, flags=flags)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        second, _ = _backward(t, dy, V, flags=flags)
    assert torch.equal(first, second)
    # a workspace of a longer call serves a shorter one
    big = torch.empty(B.alst_embedding_workspace_bytes(2 * N, H, V), dtype=torch.uint8, device="cuda")
    third = torch.empty_like(first)
    B.alst_embedding_backward(torch.from_numpy(t).cuda(), dy.cuda(), dE=third, workspace=big, flags=flags)
    assert torch.equal(first, third)


def test_tokens_at_any_offset_of_a_batch():
    N, H, V = 333, 64, 50
    g = torch.Generator().manual_seed(8)
    batch = torch.from_numpy(np.random.default_rng(8).integers(0, V, (4, N)).astype(np.int32))
    E, dy, d = U.bf16((V, H), g), U.bf16((N, H), g), batch.cuda()
    ws = B.alloc_embedding_workspace(N, H, V)
    for k in range(4):
        y, dE = U.Guarded((N, H), torch.bfloat16), U.Guarded((V, H), torch.bfloat16)
        B.alst_embedding_forward(d[k], E.cuda(), y=y.t)
        B.alst_embedding_backward(d[k], dy.cuda(), dE=dE.t, workspace=ws)
        assert torch.equal(y.t.cpu(), E[batch[k].long()]) and y.intact() and dE.intact()
        _check_backward(dE.t, batch[k].numpy(), dy, V)


def test_captured_calls_follow_their_inputs():
    N, H, V = 700, 72, 90
    g = torch.Generator().manual_seed(4)
    sets = [(_tokens("two" if k else "zipf", N, V, k), U.bf16((N, H), g), U.bf16((V, H), g)) for k in range(3)]
    t, dy, E = (torch.empty_like(torch.as_tensor(x)).cuda() for x in sets[0])
    y, dE = torch.empty((N, H), dtype=torch.bfloat16, device="cuda"), torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    ws = B.alloc_embedding_workspace(N, H, V)

    def step():
        B.alst_embedding_forward(t, E, 2.0, y=y)
        B.alst_embedding_backward(t, dy, 2.0, dE=dE, workspace=ws)

    t.copy_(torch.from_numpy(sets[0][0]))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for ti, dyi, Ei in sets:
        t.copy_(torch.from_numpy(ti)); dy.copy_(dyi); E.copy_(Ei)
        y.fill_(float("nan")); dE.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        gy, gE = y.clone(), dE.clone()
        step()
        assert torch.equal(gy, y) and torch.equal(gE, dE)
        _check_backward(gE, ti, dyi, V, scale=2.0)
