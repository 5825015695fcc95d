"""Embedding lookup and its gradient against plain sums in 64 bits.

Lookup: one fp32 product and one rounding, the same bits as torch's.  Gradient: c terms added in fp32 in any order are off by at most
(c - 1) 2^-24 of the sum of their absolute values, the scale by 2^-24 of that, the result by half a step of its type."""
import numpy as np
import pytest

from paper_2506_22714_amd import binding as lb

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float32: 0.0}     # half a step of numbers below the normal ones
TYPES = [torch.float16, torch.bfloat16, torch.float32]
SCALE = 0.75


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lb.lib()


def ids_of(n, rows, kind, seed=0):
    rng = np.random.default_rng(seed)
    if kind == "uniform":
        ids = rng.integers(0, rows, n)
    elif kind == "hot":                         # a few rows have most of the ids
        ids = (rows * rng.random(n) ** 6).astype(np.int64)
    elif kind == "one":
        ids = np.full(n, rows // 2)
    elif kind == "ends":
        ids = np.where(rng.random(n) < 0.5, 0, rows - 1)
    elif kind == "ordered":
        ids = np.sort(rng.integers(0, rows, n))
    else:
        ids = np.full(n, -1)
    if kind in ("uniform", "hot"):
        ids = np.where(rng.random(n) < 0.1, -1, ids)
    return torch.from_numpy(np.ascontiguousarray(ids)).cuda()


def check_gradient(got, dout, ids, rows, scale=SCALE):
    ids = ids.reshape(-1).long()
    keep = (ids >= 0) & (ids < rows)
    at, order = torch.sort(ids[keep], stable=True)
    d = dout.double()[keep][order] * scale
    count = torch.bincount(at, minlength=rows)
    ends = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), count.cumsum(0)])
    # (differences of running sums, in 64 bits: torch's scattered sums take minutes for ids that are all equal)
    runs = lambda t: torch.cat([torch.zeros(1, t.shape[1], dtype=torch.float64, device="cuda"), t.cumsum(0)])      # noqa: E731
    sums, sizes = runs(d), runs(d.abs())
    ref, size = sums[ends[1:]] - sums[ends[:-1]], sizes[ends[1:]] - sizes[ends[:-1]]
    slack = 2.0 ** -50 * float(sizes[-1].max())
    count = count[:, None].double()
    far = (got.double() - ref).abs() - ((count + 1) * 2.0 ** -24 * size * (1 + 2.0 ** -10) + torch.finfo(dout.dtype).eps / 2 * ref.abs() * (1 + 2.0 ** -8) + SMALLEST[dout.dtype] + slack)
    assert far.max() <= 0, (float(far.max()), int(far.argmax()))
    assert bool((got[count[:, 0] == 0] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,width", [(1, 1, 1), (1, 5, 3), (17, 1 << 17, 128), (63, 10, 64), (300, 1000, 100), (1000, 7, 333), (65, 64, 8), (4099, 5000, 33), (513, 40, 1030)])
def test_lookup(dtype, n, rows, width):
    table = torch.randn(rows, width, device="cuda").to(dtype)
    for itype in (torch.int64, torch.int32):
        ids = ids_of(n, rows, "uniform", seed=n).to(itype)
        got = lb.embedding(table, ids, scale=SCALE)
        want = (SCALE * table[ids.clamp(min=0).long()].float()).to(dtype)
        want[ids < 0] = 0
        assert got.dtype == dtype and torch.equal(got, want)
    assert torch.equal(lb.embedding(table, ids), torch.where((ids < 0)[:, None], torch.zeros_like(want), table[ids.clamp(min=0).long()]))


def test_lookup_of_what_is_no_row_and_special_values():
    table = torch.tensor([[1.0, float("inf")], [float("nan"), -float("inf")], [60000.0, 1e-7]], device="cuda", dtype=torch.float16)
    got = lb.embedding(table, torch.tensor([[-1, 3, 0], [-2, 1, 2]], device="cuda"), scale=2.0)
    want = torch.tensor([[[0, 0], [np.nan, np.nan], [2, np.inf]], [[np.nan, np.nan], [np.nan, -np.inf], [np.inf, 2 * float(table[2, 1])]]])
    np.testing.assert_array_equal(got.float().cpu().numpy(), want.numpy())
    empty = lb.embedding(torch.zeros(0, 4, device="cuda"), torch.tensor([-1, 0], device="cuda"))
    assert bool((empty[0] == 0).all()) and bool(empty[1].isnan().all())
    assert lb.embedding(table, torch.zeros(0, dtype=torch.int64, device="cuda")).shape == (0, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width,ld,offset", [(64, 72, 0), (64, 67, 0), (64, 64, 1), (100, 129, 3), (5, 8, 2)])
def test_strides_alignment_and_what_lies_between_rows(dtype, width, ld, offset):
    rows, n = 50, 333
    def strided(r):
        flat = torch.randn(r * ld + offset, device="cuda").to(dtype)
        return flat, flat[offset:].as_strided((r, width), (ld, 1))
    _, table = strided(rows)
    flat, out = strided(n)
    keep = flat.clone()
    ids = ids_of(n, rows, "hot", seed=3)
    assert lb.embedding(table, ids, SCALE, out=out) is out
    want = (SCALE * table[ids.clamp(min=0)].float()).to(dtype)
    want[ids < 0] = 0
    assert torch.equal(out, want)
    out.copy_(keep[offset:].as_strided((n, width), (ld, 1)))
    assert torch.equal(flat, keep)
    flat, grad = strided(rows)
    keep = flat.clone()
    _, dout = strided(n)
    assert lb.embedding_backward(dout, ids, rows, SCALE, out=grad) is grad
    check_gradient(grad.clone(), dout, ids, rows)
    grad.copy_(keep[offset:].as_strided((rows, width), (ld, 1)))
    assert torch.equal(flat, keep)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["uniform", "hot", "one", "ends", "ordered", "padding"])
@pytest.mark.parametrize("n,rows,width", [(1, 1, 1), (2, 3, 7), (64, 64, 16), (511, 1000, 65), (512, 5, 128), (4097, 300, 100), (9000, 20000, 32), (70001, 257, 64), (30000, 40000, 520)])
def test_gradient(dtype, kind, n, rows, width):
    g = torch.Generator(device="cuda").manual_seed(n + width)
    dout = torch.randn(n, width, generator=g, device="cuda").to(dtype)
    ids = ids_of(n, rows, kind, seed=width)
    got = lb.embedding_backward(dout, ids.int() if n % 2 else ids, rows, scale=SCALE)
    check_gradient(got, dout, ids, rows)
    assert torch.equal(got, lb.embedding_backward(dout, ids, rows, scale=SCALE))       # the same bits every time


@pytest.mark.parametrize("n,rows,width", [(1 << 20, 1 << 20, 16), (300007, 70000, 16), (200000, 16, 16), (1500001, (1 << 24) + 3, 16), (100003, 2049 * 1024, 8), (50001, 2047, 40),
                                          (50001, 2048, 1040), (40000, (1 << 21) - 1, 5), (16385, 3, 600), (20000, 1, 1)])
def test_gradient_of_many_ids(n, rows, width):
    g = torch.Generator(device="cuda").manual_seed(1)
    for kind in ("hot", "one", "ends", "uniform"):
        dout = torch.randn(n, width, generator=g, device="cuda").bfloat16()
        ids = ids_of(n, rows, kind)
        got = lb.embedding_backward(dout, ids, rows, scale=SCALE)
        check_gradient(got, dout, ids, rows)
        assert torch.equal(got, lb.embedding_backward(dout, ids, rows, scale=SCALE))


def test_gradient_of_ids_that_are_no_rows():
    dout = torch.full((6, 3), float("nan"), device="cuda")
    dout[2] = 1.0
    ids = torch.tensor([-1, 9, 2, -5, 1 << 40, 5], device="cuda")
    got = lb.embedding_backward(dout, ids, 5)
    want = torch.zeros(5, 3, device="cuda")
    want[2] = 1
    assert torch.equal(got, want)
    assert bool((lb.embedding_backward(dout[:0], ids[:0], 4) == 0).all())
    assert lb.embedding_backward(dout, ids, 0).shape == (0, 3)


def test_gradient_of_whole_numbers_is_exact():
    """Sums below 2^24 of whole numbers have no error, whatever their order."""
    ids = ids_of(100000, 3000, "hot", seed=5)
    dout = torch.randint(-3, 4, (100000, 40), device="cuda").float()
    got = lb.embedding_backward(dout, ids, 3000)
    keep = ids >= 0
    assert torch.equal(got.double(), torch.zeros(3000, 40, dtype=torch.float64, device="cuda").index_add_(0, ids[keep], dout.double()[keep]))


def test_offsets_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs some 30 GiB")
    rows, width = (1 << 24) + 5, 264                            # 2^32 elements and more
    table = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([rows - 1, 0, 1 << 23, rows - 2, rows - 1], device="cuda")
    table[at] = torch.randn(5, width, device="cuda").bfloat16()
    assert torch.equal(lb.embedding(table, at), table[at])
    dout = torch.randn(5, width, device="cuda").bfloat16()
    table.fill_(1)
    lb.embedding_backward(dout, at, rows, out=table)
    rest = [1, 2, 3]
    assert torch.equal(table[at[rest]], dout[rest])
    assert torch.equal(table[rows - 1], (dout[0].float() + dout[4].float()).bfloat16())
    assert int((table != 0).any(1).sum()) == 4
    del table
    # and rows of dout
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    ids[-1] = 3
    wide = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    wide[-1] = dout[0]
    assert torch.equal(lb.embedding_backward(wide, ids, 5)[3], dout[0])
    del wide
    torch.cuda.empty_cache()


def test_replayed_from_a_graph_and_on_another_stream():
    n, rows, width = 5000, 700, 64
    table = torch.randn(rows, width, device="cuda").half()
    dout = torch.randn(n, width, device="cuda").half()
    ids = ids_of(n, rows, "hot")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = lb.embedding(table, ids), lb.embedding_backward(dout, ids, rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grad = lb.embedding(table, ids), lb.embedding_backward(dout, ids, rows)
    for seed in range(3):
        ids.copy_(ids_of(n, rows, ("hot", "one", "uniform")[seed], seed=seed))
        dout.normal_()
        graph.replay()
        want = lb.embedding(table, ids), lb.embedding_backward(dout, ids, rows)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(grad, want[1])
    assert first[0].shape == (n, width)


def test_refusals_of_the_binding():
    table, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in (lambda: lb.embedding(table, ids.cpu()), lambda: lb.embedding(table, ids.float()), lambda: lb.embedding(table, ids.repeat(2)[::2]),
                 lambda: lb.embedding(table.t(), ids), lambda: lb.embedding(table.double(), ids), lambda: lb.embedding(table[:1].expand(4, 8), ids),
                 lambda: lb.embedding(table, ids, out=torch.zeros(2, 8, device="cuda")), lambda: lb.embedding(table, ids, out=torch.zeros(3, 8, device="cuda").half()),
                 lambda: lb.embedding(table[:, :0], ids), lambda: lb.embedding_backward(table, ids, 5), lambda: lb.embedding_backward(table[:3], ids, 5, out=table)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lb.LibraError):
        lb.libra_embedding_backward_workspace(3, -1, 8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,width", [(5000, 6000, 128), (5000, 6000, 65), (5000, 6000, 3), (40000, 50000, 64), (40000, 50000, 67), (40000, 50000, 5)])
def test_products_with_the_scale_are_formed_in_fp32(dtype, n, rows, width):
    """A row of one id, or of two, is one fp32 product, rounded once more to its type: the same bits as the lookup's, in every way that the
    gradient goes.  (0.7 times one fp16 number in forty is so near the middle of two that rounding the exact product gives another one.)"""
    scale = float(np.float32(0.7))
    g = torch.Generator(device="cuda").manual_seed(width)
    whole = torch.randint(-2047, 2048, (n, width), generator=g, device="cuda").float() / 256           # sums of two are exact in fp32
    dout = whole.to(dtype)
    ids = torch.randperm(rows, generator=g, device="cuda")[:n]
    ids[1::100] = ids[::100]
    sums = torch.zeros(rows, width, device="cuda").index_add_(0, ids, dout.float())
    assert torch.equal(lb.embedding_backward(dout, ids, rows, scale=scale), (sums * scale).to(dtype))
    assert torch.equal(lb.embedding(dout, torch.arange(n, device="cuda"), scale=scale), (dout.float() * scale).to(dtype))


def test_the_widest_row():
    """2^31 - 1 elements: columns are counted to beyond the end of a row."""
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs some 20 GiB")
    table = torch.zeros(1, (1 << 31) - 1, dtype=torch.float16, device="cuda")
    for at in (0, 1 << 30, (1 << 31) - 3000):
        table[0, at:at + 3000].normal_()
    got = lb.embedding(table, torch.tensor([0, -1], device="cuda"))
    assert torch.equal(got[0], table[0]) and not bool(got[1].any())
    del table, got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,rows,width,dtype", [(150001, 20000, 37, torch.float16), (20000, (1 << 22) + 5, 8, torch.bfloat16), (40000, 300, 520, torch.float32)])
def test_the_gradient_of_many_ids_replayed_from_a_graph(n, rows, width, dtype):
    """Other ids in every replay: no count, sum or row of zeros stays from the one before.  More tiles than a block adds up by itself, three
    passes of the sort, rows of several workgroups."""
    dout = torch.randn(n, width, device="cuda").to(dtype)
    ids = ids_of(n, rows, "hot")
    lb.embedding_backward(dout, ids, rows, SCALE)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grad = lb.embedding_backward(dout, ids, rows, SCALE)
    for seed, kind in enumerate(("one", "uniform", "padding", "ends", "hot", "ordered", "one")):
        ids.copy_(ids_of(n, rows, kind, seed=seed))
        dout.normal_()
        graph.replay()
        want = lb.embedding_backward(dout, ids, rows, SCALE)
        torch.cuda.synchronize()
        assert torch.equal(grad, want), kind
        if seed % 3 == 0:
            check_gradient(grad, dout, ids, rows)


def test_two_graphs_and_two_streams_of_many_ids():
    """Workspaces of calls that run at the same time, eager ones and replayed ones."""
    cases = []
    for seed, (n, rows) in enumerate(((200000, 70000), (140000, 3000))):
        ids = ids_of(n, rows, ("hot", "uniform")[seed], seed=seed)
        cases.append((torch.randn(n, 64, device="cuda").half(), ids, rows))
    want = [lb.embedding_backward(*c) for c in cases]
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in cases], []
    for graph, c in zip(graphs, cases):
        with torch.cuda.graph(graph):
            outs.append(lb.embedding_backward(*c))
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(4):
        for o in outs:
            o.fill_(1)
        torch.cuda.synchronize()
        eager = []
        for c, s, graph in zip(cases, streams, graphs):
            with torch.cuda.stream(s):
                eager.append(lb.embedding_backward(*c))
                graph.replay()
                eager.append(lb.embedding_backward(*c))
        torch.cuda.synchronize()
        for k, w in enumerate(want):
            assert torch.equal(outs[k], w) and torch.equal(eager[2 * k], w) and torch.equal(eager[2 * k + 1], w)
