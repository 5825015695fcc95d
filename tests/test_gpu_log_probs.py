"""Log probabilities, entropy, alternatives and their gradient against the definition in 64 bits.

With u = 2^-24: z = scale (x - max) is off by 2 u |z|; exp(z) then by (2 |z| + 2 |z| + 2) u of itself (the error of z, of the product with
log2 e, of the instruction); the sum s of exp(z) by the mean of that, where the mean of |z| is at most log(classes) < 13, and by u for each
addition a term goes through: at most classes / 64 + 16.  That is the relative error of s and the absolute one of log s:
  u_s = u (64 + classes / 64).  log p = z - log s: u_s + 4 u |log p|.  H = log s - sum exp(z) z / s: u_s (1 + H) + 4 u sum p z^2.
A gradient has p from log p, so p (4 |log p| + 80 + classes / 64) u of what it is multiplied with, the errors of log p and H times p e, four
roundings of its parts, and half a step of its type."""
import numpy as np
import pytest

from paper_2506_22714_amd import binding as lb

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF = float("inf")
U = 2.0 ** -24
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -149}
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lb.lib()


def definition(x, targets, top, scale):
    """(log p of all classes, entropy, classes in order, sum p z^2) in 64 bits, on the CPU."""
    z = torch.nan_to_num(x.double().cpu() * scale, nan=float("nan"), posinf=INF, neginf=-INF)
    empty = (z == -INF).all(1)
    logp = torch.log_softmax(z, 1)
    logp[empty] = -INF
    p = logp.exp()
    h = torch.where(empty, torch.zeros(len(z), dtype=torch.float64), -torch.special.xlogy(p, p).sum(1))
    d = z - z.amax(1, keepdim=True)
    square = torch.where(p > 0, p * d * d, torch.zeros_like(p)).sum(1)
    order = torch.sort(x.double().cpu(), dim=1, descending=True, stable=True).indices[:, :top]
    return logp, h, order, square


def close(got, ref, tol, what):
    got, ref = got.double().cpu(), ref.double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    far = torch.where(same, torch.zeros_like(ref), (got - ref).abs() - tol)
    assert not bool(far.isnan().any()) and bool((far <= 0).all()), (what, float(far.max()), int(far.argmax()))


def check(x, targets, top, scale, gradient=True, grads=None, seed=0):
    n, classes = x.shape
    logp, h, order, square = definition(x, targets, top, scale)
    us = U * (64 + classes / 64)
    r = lb.log_probs(x, targets, top=top, scale=scale)
    assert torch.equal(r.top_index.cpu(), order)
    best = logp.gather(1, order)
    finite = lambda t: torch.where(t.isfinite(), t.abs(), torch.zeros_like(t))      # noqa: E731
    close(r.top, best, us + 4 * U * finite(best), "top")
    tol_h = us * (1 + h) + 4 * U * square
    close(r.entropy, h, tol_h, "entropy")
    t = None
    if targets is not None:
        t = targets.cpu().long()
        want = logp.gather(1, t.clamp(0, classes - 1)[:, None])[:, 0]
        want[t == -1] = 0
        want[(t < -1) | (t >= classes)] = float("nan")
        close(r.target, want, us + 4 * U * finite(want), "target")
    else:
        assert r.target is None
    if not gradient:
        return r
    g = torch.Generator(device="cuda").manual_seed(seed)
    d = torch.randn(n, generator=g, device="cuda") if targets is not None else None
    e = torch.randn(n, generator=g, device="cuda")
    a = torch.randn(n, top, generator=g, device="cuda")
    use = (True, True, True) if grads is None else grads
    d, e, a = (v if on else None for v, on in zip((d, e, a), use))
    got = lb.log_probs_backward(x, r, targets, d, e, a, scale=scale)
    assert got.dtype == x.dtype
    zero = torch.zeros(n, dtype=torch.float64)
    dd = zero if d is None else torch.where(t == -1, zero, d.double().cpu())
    ee = zero if e is None else e.double().cpu()
    aa = torch.zeros(n, top, dtype=torch.float64) if a is None else a.double().cpu()
    parts = torch.zeros(n, classes, dtype=torch.float64)
    if t is not None:
        parts.scatter_add_(1, t.clamp(0, classes - 1)[:, None], dd[:, None])
    parts.scatter_add_(1, order, aa)
    p = logp.exp()
    safe = torch.where(p > 0, logp, torch.zeros_like(logp))
    all_, big = (dd + aa.sum(1))[:, None], (dd.abs() + aa.abs().sum(1))[:, None]
    ref = scale * (parts - p * (all_ + ee[:, None] * (safe + h[:, None])))
    ref[(x == -INF).all(1).cpu()] = 0
    tol = p * (big * (top + 2) * U + (all_.abs() + ee.abs()[:, None] * (safe.abs() + h[:, None])) * U * (4 * safe.abs() + 80 + classes / 64)
               + ee.abs()[:, None] * (us + 4 * U * safe.abs() + tol_h[:, None])) + 4 * U * (big + ref.abs() / scale)
    tol = scale * tol + torch.finfo(x.dtype).eps / 2 * ref.abs() * (1 + 2.0 ** -8) + SMALLEST[x.dtype]
    close(got, ref, tol, "gradient")
    return r


def logits(n, classes, dtype, seed=0, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (spread * torch.randn(n, classes, generator=g, device="cuda")).to(dtype)


def targets_of(n, classes, seed=0):
    rng = np.random.default_rng(seed)
    t = rng.integers(0, classes, n)
    t[rng.random(n) < 0.1] = -1
    return torch.from_numpy(t).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,classes", [(1, 1), (3, 2), (5, 7), (130, 8), (64, 33), (257, 40), (33, 64), (9, 65), (31, 128), (70, 300), (17, 512), (6, 1000), (5, 1024), (9, 1025), (4, 2049),
                                       (3, 5000), (300, 4100), (2, 32768), (1, 131072), (2, 100003)])
def test_against_the_definition(dtype, n, classes):
    x = logits(n, classes, dtype, seed=classes)
    for top in sorted({0, 1, min(classes, 5), min(classes, 20), min(classes, 64)}):
        check(x, targets_of(n, classes, seed=top), top, 0.7, seed=top)
    check(x, targets_of(n, classes).int(), min(classes, 2), 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [5, 64, 300, 1024, 3000, 70000])
def test_equal_logits_go_by_class(dtype, classes):
    """Few distinct values: the alternatives are the lowest classes among equals; -0 equals 0."""
    g = torch.Generator(device="cuda").manual_seed(classes)
    x = torch.randint(-2, 3, (7, classes), generator=g, device="cuda").to(dtype)
    x[x == 0] *= torch.where(torch.rand(int((x == 0).sum()), generator=g, device="cuda") < 0.5, -1.0, 1.0).to(dtype)
    x[1] = 0.25
    x[2] = torch.arange(classes, device="cuda").clamp(max=2000).to(dtype)          # in ascending order
    x[3] = -x[2]
    for top in (1, min(classes, 3), min(classes, 33), min(classes, 64)):
        check(x, targets_of(7, classes), top, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [3, 40, 200, 1024, 1500, 40000])
def test_masks(dtype, classes):
    """-Inf, the type's lowest number, rows with one class left and with none."""
    n = 12
    x = logits(n, classes, dtype, seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    x[torch.rand(n, classes, generator=g, device="cuda") < 0.5] = -INF
    x[0] = -INF
    x[1] = -INF
    x[1, classes - 1] = 3.0
    x[2] = torch.finfo(dtype).min
    x[3, : classes // 2] = torch.finfo(dtype).min
    x[4] = -INF
    x[4, 0] = torch.finfo(dtype).min
    x[5, classes // 2:] = -INF
    t = targets_of(n, classes, seed=3)
    t[0] = 0
    for top in (0, 2, min(classes, 20)):
        check(x, t, top, 0.5)


def of_all_kinds(n, classes, dtype, seed):
    """Rows of ordinary logits, equal ones, ascending ones, masked ones (half, all but one, all), of the lowest number, with a NaN and infinities."""
    x = logits(n, classes, dtype, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.arange(n, device="cuda") % 11
    x[kind == 1] = 0.25
    x[kind == 2] = torch.arange(classes, device="cuda").clamp(max=2000).to(dtype) / 64
    x[kind == 3] = torch.randint(-2, 3, (int((kind == 3).sum()), classes), generator=g, device="cuda").to(dtype)
    x[(kind == 4)[:, None] & (torch.rand(n, classes, generator=g, device="cuda") < 0.5)] = -INF
    x[kind == 5] = -INF
    x[(kind == 5), torch.randint(classes, (int((kind == 5).sum()),), generator=g, device="cuda")] = 1.5
    x[kind == 6] = -INF
    x[(kind == 7)[:, None] & (torch.rand(n, classes, generator=g, device="cuda") < 0.9)] = torch.finfo(dtype).min
    x[(kind == 8) & (torch.arange(n, device="cuda") % 2 == 0), classes // 3] = float("nan")
    x[kind == 9, classes // 2:] = -INF
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,classes", [(6, 3), (6, 300), (6, 1500), (1040, 2500), (6, 5000), (6, 90000)])
@pytest.mark.parametrize("e", [1.0, -2.5, 1e6])
def test_masked_classes_have_no_gradient_of_the_entropy(dtype, n, classes, e):
    """However large the entropy's gradient is: p log p is 0 there, not 0 times infinity."""
    x = logits(n, classes, dtype, seed=4, spread=1.0)
    masked = torch.rand(n, classes, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") < 0.4
    masked[:, 0] = False
    x[masked & (torch.arange(n, device="cuda") % 2 == 0)[:, None]] = -INF
    x[masked & (torch.arange(n, device="cuda") % 2 == 1)[:, None]] = torch.finfo(dtype).min
    t = torch.zeros(n, dtype=torch.int64, device="cuda")
    r = lb.log_probs(x, t, top=1)
    g = lb.log_probs_backward(x, r, t, torch.ones(n, device="cuda"), torch.full((n,), e, device="cuda"))
    assert bool((g[masked] == 0).all()) and bool((g.isfinite() | (g.abs() > torch.finfo(dtype).max)).all()) and not bool(g.isnan().any())
    assert bool((g[:, 1:][~masked[:, 1:]] != 0).any()) or classes == 3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,classes,top", [(1023, 2042, 5), (1024, 2042, 0), (1024, 4096, 64), (1031, 4097, 3), (1030, 2053, 1), (1100, 3000, 20), (2053, 8201, 10)])
def test_many_rows(dtype, n, classes, top):
    """As many rows as get a wave each, and one fewer."""
    x = of_all_kinds(n, classes, dtype, seed=classes)
    odd = torch.isnan(x).any(1)
    good = x[~odd]
    check(good, targets_of(len(good), classes), top, 0.7)
    # a NaN stays in its row.  (The other rows at the same addresses: the order of a row's sums goes by its 16-byte pieces.)
    t = targets_of(n, classes, seed=3)
    r, without = lb.log_probs(x, t, top=top, scale=0.7), lb.log_probs(x.nan_to_num(nan=0.0, posinf=INF, neginf=-INF), t, top=top, scale=0.7)
    for got, want in zip(r, without):
        assert got is want is None or torch.equal(got[~odd], want[~odd])
    assert bool(r.entropy[odd].isnan().all()) and bool(r.target[odd & (t != -1)].isnan().all())
    if top:
        assert bool((r.top_index[odd, 0] == classes // 3).all()) and bool(r.top[odd].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ld,offset", [(0, 0), (1, 0), (8, 3)])
def test_sizes_at_which_the_way_changes(dtype, ld, offset):
    for classes in (16, 17, 32, 33, 41, 48, 49, 64, 65, 96, 97, 128, 129, 192, 193, 256, 257, 384, 385, 512, 513, 768, 769, 1017, 1018, 1024, 1025, 1529, 1536, 1537, 2041, 2042):
        n = 23
        held = torch.full((offset + n * (classes + ld),), 7.0, dtype=dtype, device="cuda")
        x = torch.as_strided(held, (n, classes), (classes + ld, 1), offset)
        x.copy_(of_all_kinds(n, classes, dtype, seed=classes).nan_to_num(nan=1.0, posinf=3.0, neginf=-INF))
        for top in (2, min(classes, 40)):
            check(x, targets_of(n, classes, seed=top), top, 1.0)


def test_many_rows_with_space_between_them():
    """The gradient of rows of a wave each leaves what lies between its rows."""
    n, classes, ld = 1500, 2501, 2507
    held = logits(n, ld, torch.bfloat16, seed=5)
    x, t = held[:, 3:3 + classes], targets_of(n, classes)
    out = torch.full((n, ld + 4), 9.0, dtype=torch.bfloat16, device="cuda")
    r = lb.log_probs(x, t, top=3)
    d, e, a = (torch.randn(n, device="cuda"), torch.randn(n, device="cuda"), torch.randn(n, 3, device="cuda"))
    lb.log_probs_backward(x, r, t, d, e, a, out=out[:, 1:1 + classes])
    tight = lb.log_probs_backward(x.contiguous(), r, t, d, e, a)      # (with these sums: theirs would go by other 16-byte pieces)
    check(x, t, 3, 1.0)
    assert torch.equal(out[:, 1:1 + classes], tight)
    assert bool((out[:, :1] == 9).all()) and bool((out[:, 1 + classes:] == 9).all())


@pytest.mark.parametrize("classes", [5, 300, 5000])
def test_nan_and_infinity_spoil_their_row_alone(classes):
    x = logits(6, classes, torch.float32)
    x[1, 2] = float("nan")
    x[3, classes - 1] = INF
    x[4, 1] = INF
    x[4, 3] = float("nan")
    t = torch.tensor([0, 1, -1, 2, 3, 1], device="cuda")
    r = lb.log_probs(x, t, top=3)
    g = lb.log_probs_backward(x, r, t, torch.ones(6, device="cuda"), torch.ones(6, device="cuda"), torch.ones(6, 3, device="cuda"))
    for k in (1, 3, 4):
        assert bool(r.entropy[k].isnan()) and bool(r.top[k].isnan().all()) and bool(g[k].isnan().all())
        assert bool(r.target[k].isnan())
    assert r.top_index[1, 0] == 2 and r.top_index[3, 0] == classes - 1 and r.top_index[4, :2].tolist() == [3, 1]
    keep = [0, 2, 5]
    clean = lb.log_probs(x[keep], t[keep], top=3)
    for got, want in zip(r, clean):
        assert torch.equal(got[keep], want)
    assert bool(g[keep].isfinite().all())


def test_targets_that_are_no_classes():
    x = logits(5, 10, torch.bfloat16)
    t = torch.tensor([-1, 10, -2, 1 << 40, 9], device="cuda")
    r = lb.log_probs(x, t)
    assert r.target[0] == 0 and bool(r.target[1:4].isnan().all()) and bool(r.target[4].isfinite())
    g = lb.log_probs_backward(x, r, t, torch.ones(5, device="cuda"))
    assert bool((g[0] == 0).all()) and bool(g[1:4].isnan().all()) and bool(g[4].isfinite().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [30, 600, 3000, 60000])
def test_large_numbers_and_scales(dtype, classes):
    x = logits(4, classes, dtype, spread=50.0)
    x[1] += 2000
    for scale in (1e-3, 1.0, 7.0):
        check(x, targets_of(4, classes), min(classes, 4), scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes,ld,offset", [(40, 41, 0), (40, 48, 1), (64, 72, 0), (1000, 1003, 1), (3000, 3008, 0), (3000, 3001, 3), (70000, 70001, 1)])
def test_strides_alignment_and_what_lies_between_rows(dtype, classes, ld, offset):
    n = 9
    def strided():
        flat = torch.randn(n * ld + offset, device="cuda").to(dtype)
        return flat, flat[offset:].as_strided((n, classes), (ld, 1))
    _, x = strided()
    t = targets_of(n, classes)
    top = 7
    r = check(x, t, top, 1.0)
    plain = lb.log_probs(x.contiguous(), t, top=top)
    assert torch.equal(plain.top_index, r.top_index)
    flat, out = strided()
    keep = flat.clone()
    d = torch.randn(n, device="cuda")
    want = lb.log_probs_backward(x, r, t, d, d, torch.ones(n, top, device="cuda"))
    assert lb.log_probs_backward(x, r, t, d, d, torch.ones(n, top, device="cuda"), out=out) is out
    close(out, want.cpu(), torch.finfo(dtype).eps * want.double().cpu().abs() + 4 * SMALLEST[dtype] + 1e-9, "out")
    out.copy_(keep[offset:].as_strided((n, classes), (ld, 1)))
    assert torch.equal(flat, keep)


@pytest.mark.parametrize("classes", [40, 900, 9000])
def test_parts_of_the_gradient_alone(classes):
    x, t = logits(6, classes, torch.float32), targets_of(6, classes)
    for grads in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        check(x, t, 3, 0.9, grads=grads)
    check(x, None, 3, 0.9, grads=(False, True, True))


def test_gradient_against_differences():
    from paper_2506_22714_amd import autograd as ag
    g = torch.Generator().manual_seed(0)
    x = torch.stack([torch.linspace(-2, 2, 12)[torch.randperm(12, generator=g)] for _ in range(3)]).cuda()    # further apart than the step
    t = torch.tensor([3, -1, 11], device="cuda")
    w = torch.randn(3, 4, device="cuda")
    def f(v):
        logp, h, top, _ = ag.log_probs(v, t, top=4, scale=0.8)
        return (logp.double() * torch.tensor([1.0, 2.0, -0.5], device="cuda")).sum() + 0.3 * h.double().sum() + (top.double() * w).sum()
    v = x.clone().requires_grad_()
    f(v).backward()
    step = 2.0 ** -5
    for k in range(36):
        d = torch.zeros(36, device="cuda")
        d[k] = step
        d = d.view(3, 12)
        slope = float((f(x + d) - f(x - d)) / (2 * step))
        # 18 fp32 results, each off by 64 u + 4 u 5 at most, times weights of size 1, divided by the step; the third derivative times step^2 / 6
        assert abs(slope - float(v.grad.view(-1)[k])) < 20 * 90 * U / step + 10 * step ** 2 / 6, k


def test_no_rows():
    x = torch.zeros(0, 5, device="cuda")
    r = lb.log_probs(x, torch.zeros(0, dtype=torch.int64, device="cuda"), top=2)
    assert r.top_index.shape == (0, 2)
    assert lb.log_probs_backward(x, r, None, None, torch.zeros(0, device="cuda")).shape == (0, 5)


def test_offsets_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs some 20 GiB")
    n, classes = (1 << 17) + 3, 32768 + 8                       # more than 2^32 logits
    x = torch.zeros(n, classes, dtype=torch.bfloat16, device="cuda")
    last = logits(4, classes, torch.bfloat16)
    x[-4:] = last
    t = torch.zeros(n, dtype=torch.int64, device="cuda")
    t[-4:] = torch.arange(4, device="cuda") + 5
    r, want = lb.log_probs(x, t, top=3), lb.log_probs(last, t[-4:], top=3)
    tol = U * (64 + classes / 64)
    close(r.target[-4:], want.target.cpu(), 2 * tol + 8 * U * want.target.abs().double().cpu(), "target")
    assert torch.equal(r.top_index[-4:], want.top_index)
    assert bool(((r.target[:-4] + float(np.log(classes))).abs() < tol * 12).all())
    d = torch.ones(n, device="cuda")
    g = lb.log_probs_backward(x, r, t, d)
    small = lb.log_probs_backward(last, want, t[-4:], d[-4:])
    close(g[-4:], small.cpu(), torch.finfo(torch.bfloat16).eps * small.double().cpu().abs() + 1e-9, "gradient")
    assert bool((g[:-4, 0] > 0.99).all()) and bool((g[:-4, 1:] < 0).all())
    del x, g
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,classes", [(300, 40), (40, 700), (20, 5000), (2, 90000)])
def test_replayed_from_a_graph_and_on_another_stream(n, classes):
    x, t = logits(n, classes, torch.float16), targets_of(n, classes)
    d = torch.randn(n, device="cuda")
    def both():
        r = lb.log_probs(x, t, top=5)
        return [*r, lb.log_probs_backward(x, r, t, d, d)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for seed in range(3):
        x.copy_(logits(n, classes, torch.float16, seed=seed + 5))
        d.normal_()
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_refusals_of_the_binding():
    x, t = logits(4, 10, torch.float32), torch.zeros(4, dtype=torch.int64, device="cuda")
    r = lb.log_probs(x, t, top=2)
    d = torch.ones(4, device="cuda")
    for call in (lambda: lb.log_probs(x, t[:3]), lambda: lb.log_probs(x, t.float()), lambda: lb.log_probs(x, t.cpu()), lambda: lb.log_probs(x.t()),
                 lambda: lb.log_probs(x[0]), lambda: lb.log_probs_backward(x, r, None, d), lambda: lb.log_probs_backward(x, r, t, d.double()),
                 lambda: lb.log_probs_backward(x, r, t, d[:3]), lambda: lb.log_probs_backward(x, r, t, None, None, d),
                 lambda: lb.log_probs_backward(x[:3], r, t[:3]), lambda: lb.log_probs_backward(x, r, t, d, out=x.half())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lb.log_probs(x, t, top=11), lambda: lb.log_probs(x, t, top=-1), lambda: lb.log_probs(x, t, scale=0.0),
                 lambda: lb.log_probs(logits(2, 100, torch.float32), top=65)):
        with pytest.raises((lb.LibraError, RuntimeError)):
            call()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,classes", [(5000, 3), (5000, 40), (2000, 700), (2000, 2500), (64, 70000)])
def test_products_with_the_scale_are_formed_in_fp32(dtype, n, classes):
    """A masked class has no probability, so the gradient of its log probability is scale * d: an fp32 product, rounded once more."""
    scale = float(np.float32(0.7))
    x = torch.full((n, classes), -INF, device="cuda", dtype=dtype)
    x[:, 1] = 0.0
    t = torch.full((n,), classes - 1, dtype=torch.int64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(classes)
    d = torch.randint(-2047, 2048, (n,), generator=g, device="cuda").float() / 256
    got = lb.log_probs_backward(x, lb.log_probs(x, t, scale=scale), t, d, scale=scale)
    assert torch.equal(got[:, classes - 1], (d * scale).to(dtype))
    # and as one of the alternatives: the most likely class and the lowest masked one
    r = lb.log_probs(x, t, top=2, scale=scale)
    assert r.top_index[:, 1].tolist() == [0] * n
    a = torch.stack([torch.zeros_like(d), d], 1)
    assert torch.equal(lb.log_probs_backward(x, r, None, None, None, a, scale=scale)[:, 0], (d * scale).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("classes", [30, 3000, 60000])
def test_the_largest_scale(dtype, classes):
    """2^127; twice that times log2 e is infinite, and it is refused."""
    x = (logits(4, classes, torch.float32) * 2.0 ** -122).to(dtype)
    check(x, targets_of(4, classes), min(classes, 4), 2.0 ** 127, gradient=False)
    for scale in (1.8e38, 3.4e38):
        with pytest.raises(lb.LibraError):
            lb.log_probs(x, scale=scale)
