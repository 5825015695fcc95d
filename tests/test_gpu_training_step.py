"""A whole training step of a small graph network as a program runs it: rows of a learned table -> an aggregation on the graph -> attention
on the graph -> classes -> loss with an entropy bonus -> gradients -> AdamW, against the same in 64 bits on dense matrices."""
import numpy as np
import pytest

from paper_2506_22714_amd import binding as lb
from paper_2506_22714_amd import workloads as wl

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lb.lib()


def setup(seed=0):
    A = wl.random_pattern(300, 300, 0.05, seed=4, empty_rows=0.1)
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, 120, 300)                    # several nodes share a row of the table
    ids[::50] = -1
    targets = rng.integers(0, 10, 300)
    targets[::7] = -1
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()      # noqa: E731
    table = dev((0.5 * rng.standard_normal((120, 32))).astype(np.float32))
    head = dev((0.3 * rng.standard_normal((32, 10))).astype(np.float32))
    return A, dev(ids), dev(targets), table, head


def loss_of(logp, h, given):
    return -logp.sum() / given - 0.05 * h.mean()


def ours(sm, vals, ids, targets, table, head):
    from paper_2506_22714_amd import autograd as ag
    x = ag.embedding(table, ids, scale=1.5)
    x = ag.spmm(sm, vals, x)
    s = ag.sddmm(sm, torch.ones_like(vals), x, x)
    x = ag.spmm(sm, ag.edge_softmax(sm, s, 0.2), x)
    logp, h, top, classes = ag.log_probs(x @ head, targets, top=3, scale=2.0)
    return loss_of(logp, h, (targets >= 0).sum()), top, classes


def plain(A, vals, ids, targets, table, head):
    dense = torch.zeros(A.M, A.Kc, dtype=torch.float64, device="cuda")
    rows = torch.from_numpy(np.repeat(np.arange(A.M), np.diff(A.rowptr))).cuda()
    cols = torch.from_numpy(A.col.astype(np.int64)).cuda()
    dense = dense.index_put((rows, cols), vals.double())
    there = torch.zeros_like(dense, dtype=torch.bool).index_put((rows, cols), torch.tensor(True, device="cuda"))
    x = torch.where((ids < 0)[:, None], 0.0, 1.5 * table[ids.clamp(min=0)])
    x = dense @ x
    s = torch.where(there, 0.2 * (x @ x.t()), -torch.inf)
    some = there.any(1, keepdim=True)
    alpha = torch.where(there, torch.softmax(torch.where(some, s, 0.0), 1), 0.0)
    x = alpha @ x
    logp = torch.log_softmax(2.0 * (x @ head), 1)
    h = -(logp.exp() * logp).sum(1)
    given = torch.where(targets >= 0, logp.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    return loss_of(given, h, (targets >= 0).sum())


def make(A):
    from paper_2506_22714_amd import autograd as ag
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()      # noqa: E731
    return ag.SparseMatrix(A.M, A.Kc, dev(A.rowptr), dev(A.col), dtype=torch.float32)


def test_gradients_and_update_of_a_whole_step():
    from paper_2506_22714_amd.optim import AdamW
    A, ids, targets, table, head = setup()
    sm = make(A)
    vals = torch.from_numpy(A.val.astype(np.float32)).cuda()
    ps = [torch.nn.Parameter(table.clone()), torch.nn.Parameter(head.clone())]
    qs = [table.double().requires_grad_(), head.double().requires_grad_()]
    opt = AdamW(ps, lr=1e-2, weight_decay=0.1)
    for step in range(3):
        opt.zero_grad()
        loss, _, _ = ours(sm, vals, ids, targets, *ps)
        loss.backward()
        for q, p in zip(qs, ps):
            q.grad = None
            q.data = p.detach().double()
        want = plain(A, vals, ids, targets, *qs)
        want.backward()
        assert abs(float(loss) - float(want)) < 1e-4 * max(1.0, abs(float(want)))
        for p, q in zip(ps, qs):
            # sums of some hundred fp32 terms, five products deep: 2^-24 * 100 * 5 of the gradients' size
            size = float(q.grad.abs().max())
            assert float((p.grad.double() - q.grad).abs().max()) < 2.0 ** -24 * 500 * 4 * size
        before = [p.detach().double() for p in ps]
        grads = [p.grad.double() for p in ps]
        if step == 0:
            states = [[torch.zeros_like(g), torch.zeros_like(g)] for g in grads]
        opt.step()
        for p, b, g, s in zip(ps, before, grads, states):
            s[0] = 0.9 * s[0] + 0.1 * g
            s[1] = 0.999 * s[1] + 0.001 * g * g
            new = b * (1 - 1e-2 * 0.1) - 1e-2 * (s[0] / (1 - 0.9 ** (step + 1))) / ((s[1] / (1 - 0.999 ** (step + 1))).sqrt() + 1e-8)
            # some forty roundings of 2^-24 of steps of 1e-2, the parameter's own; the eps of 1e-8 keeps the quotient steady
            assert float((p.detach().double() - new).abs().max()) < 2.0 ** -24 * (2 * float(new.abs().max()) + 4 * 40 * 1e-2)
    sm.close()


def test_a_whole_step_replayed_from_a_graph():
    """The captured step against the eager one, from the same weights, three times in a row."""
    from paper_2506_22714_amd.optim import AdamW
    A, ids, targets, table, head = setup(1)
    sm = make(A)
    vals = torch.from_numpy(A.val.astype(np.float32)).cuda()
    runs = []
    for captured in (False, True):
        ps = [torch.nn.Parameter(table.clone()), torch.nn.Parameter(head.clone())]
        opt = AdamW(ps, lr=1e-2, state_bits=8, capturable=captured)
        def step():
            opt.zero_grad(set_to_none=True)
            loss, _, _ = ours(sm, vals, ids, targets, *ps)
            loss.backward()
            opt.step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        seen = []
        for _ in range(3):
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            seen.append([p.detach().clone() for p in ps])
        runs.append(seen)
    for eager, replayed in zip(*runs):
        for a, b in zip(eager, replayed):
            # Steps of 1e-2.  Atomic sums of the aggregation differ in their last places between runs: a gradient near zero may turn its
            # sign, and a state's rounding its direction (an eighth of it); few elements meet either
            assert float((a - b).abs().mean()) < 1e-3
    sm.close()


def test_log_probs_without_targets():
    from paper_2506_22714_amd import autograd as ag
    x = torch.randn(5, 9, device="cuda", requires_grad=True)
    logp, h, top, classes = ag.log_probs(x, top=2, scale=1.5)
    assert logp is None
    (h.sum() - top[:, 1].sum()).backward()
    z = x.detach().double().requires_grad_()
    lp = torch.log_softmax(1.5 * z, 1)
    (-(lp.exp() * lp).sum() - lp.gather(1, classes[:, 1:]).sum()).backward()
    assert float((x.grad.double() - z.grad).abs().max()) < 2.0 ** -24 * 400


def test_no_second_derivatives():
    from paper_2506_22714_amd import autograd as ag
    w = torch.randn(5, 4, device="cuda", requires_grad=True)
    ids = torch.tensor([1, 1, -1], device="cuda")
    (g,) = torch.autograd.grad((ag.embedding(w, ids) ** 2).sum(), w, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_broadcast_and_strided_gradients():
    from paper_2506_22714_amd import autograd as ag
    w = torch.randn(6, 8, device="cuda", requires_grad=True)
    ids = torch.tensor([[1, 1], [0, -1], [5, 1]], device="cuda")
    ag.embedding(w, ids, scale=2.0).sum().backward()            # a gradient of one element, expanded
    want = torch.zeros(6, 8, device="cuda")
    want[1], want[0], want[5] = 6.0, 2.0, 2.0
    assert torch.equal(w.grad, want)
    w.grad = None
    u = torch.randn(8, 3, 2, device="cuda")
    (ag.embedding(w, ids).permute(2, 0, 1) * u).sum().backward()
    want = torch.zeros(6, 8, device="cuda", dtype=torch.float64)
    for a in range(3):
        for b in range(2):
            if ids[a, b] >= 0:
                want[ids[a, b]] += u[:, a, b].double()
    assert float((w.grad.double() - want).abs().max()) < 4 * 2.0 ** -24 * 10
    x = torch.randn(4, 9, device="cuda", requires_grad=True)
    logp, h, top, classes = ag.log_probs(x.t()[:, :].contiguous(), torch.tensor([0, 1, 2, 3, 0, 1, 2, 3, -1], device="cuda"), top=2)
    (logp.sum() + h[::2].sum() + top.t()[0].sum()).backward()
    z = x.detach().double().requires_grad_()
    lp = torch.log_softmax(z.t(), 1)
    ref = lp[torch.arange(8), torch.arange(8) % 4].sum() - (lp.exp() * lp).sum(1)[::2].sum() + lp.amax(1).sum()
    ref.backward()
    assert float((x.grad.double() - z.grad).abs().max()) < 2.0 ** -24 * 400
    assert not classes.requires_grad


def test_rows_that_are_not_contiguous():
    from paper_2506_22714_amd import autograd as ag
    w = torch.randn(8, 6, device="cuda")
    ids = torch.tensor([5, 0, -1, 5], device="cuda")
    a, b = w.clone().requires_grad_(), w.clone().requires_grad_()
    u = torch.randn(4, 8, device="cuda")
    (ag.embedding(a.t(), ids) * u).sum().backward()
    (ag.embedding(b.t().contiguous(), ids) * u).sum().backward()
    assert torch.equal(a.grad, b.grad)
    t = torch.tensor([1, 0, -1, 7, 2, 2], device="cuda")
    a, b = w.clone().requires_grad_(), w.clone().requires_grad_()
    for x, of in ((a, a.t()), (b, b.t().contiguous())):
        logp, h, top, _ = ag.log_probs(of, t, top=3)
        (logp.sum() + 2 * h.sum() + top[:, 2].sum()).backward()
    assert torch.equal(a.grad, b.grad)


def test_embedding_gradient_against_differences():
    """The lookup is linear: over steps of a power of two its differences in fp32 are exact but for the roundings of scale * weight."""
    from paper_2506_22714_amd import autograd as ag
    w = torch.randint(-8, 9, (5, 3), device="cuda").float()
    ids = torch.tensor([4, 1, 4, -1, 0, 4], device="cuda")
    u = torch.randint(-4, 5, (6, 3), device="cuda").float()
    f = lambda v: float((ag.embedding(v, ids, scale=0.5) * u).sum())        # noqa: E731
    v = w.clone().requires_grad_()
    (ag.embedding(v, ids, scale=0.5) * u).sum().backward()
    for k in range(15):
        d = torch.zeros(15, device="cuda")
        d[k] = 2.0
        d = d.view(5, 3)
        assert (f(w + d) - f(w - d)) / 4 == float(v.grad.view(-1)[k])


def test_two_streams_at_once():
    """Calls that need a workspace, on two streams, against the same calls one after the other."""
    g = torch.Generator(device="cuda").manual_seed(0)
    cases = []
    for n, rows in ((70000, 5000), (90000, 20000)):
        ids = torch.randint(-1, rows, (n,), generator=g, device="cuda")
        cases.append((torch.randn(n, 64, generator=g, device="cuda").half(), ids, rows, torch.randn(3, 80000 + rows, generator=g, device="cuda"),
                      torch.randint(0, 1000, (3,), generator=g, device="cuda")))
    def call(c):
        return [lb.embedding_backward(c[0], c[1], c[2]), *lb.log_probs(c[3], c[4], top=7)]
    want = [call(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    for _ in range(5):
        for k, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[k].append(call(c))
    torch.cuda.synchronize()
    for w, several in zip(want, got):
        for one in several:
            assert all(torch.equal(a, b) for a, b in zip(w, one))


def test_the_optimizer_agrees_with_torch():
    """Three steps of both; fp32 on both sides, some forty roundings of 2^-24 a step apart, of steps of 1e-2 and weights of size 4."""
    from paper_2506_22714_amd.optim import AdamW
    ps = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in (1000, 77)]
    qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    a, b = AdamW(ps, lr=1e-2, weight_decay=0.1), torch.optim.AdamW(qs, lr=1e-2, weight_decay=0.1)
    for _ in range(3):
        for p, q in zip(ps, qs):
            p.grad = torch.randn_like(p)
            q.grad = p.grad.clone()
        a.step()
        b.step()
    for p, q in zip(ps, qs):
        assert float((p - q).detach().abs().max()) < 3 * 2.0 ** -24 * (40 * 1e-2 + 2 * 5)


def test_results_on_their_inputs_are_refused():
    """In place, shifted by a row or by a column; two halves of one array's columns are apart."""
    held = torch.randn(40, 32, device="cuda")
    x, t = held[:20, :16], torch.zeros(20, dtype=torch.int64, device="cuda")
    r = lb.log_probs(x, t)
    d = torch.ones(20, device="cuda")
    index = torch.arange(20, device="cuda")
    for out in (x, held[1:21, :16], held[:20, 8:24], held[:20, 15:31], held.reshape(80, 16)[:20]):
        for call in (lambda: lb.log_probs_backward(x, r, t, d, out=out), lambda: lb.embedding(x, index, out=out),
                     lambda: lb.embedding_backward(x, index, 20, out=out)):
            with pytest.raises(ValueError, match="overlaps"):
                call()
    for out in (held[:20, 16:], held[20:, 3:19], held[5:25, 16:]):
        before = x.clone()
        assert torch.equal(lb.log_probs_backward(x, r, t, d, out=out), lb.log_probs_backward(before, r, t, d))
        assert torch.equal(lb.embedding(x, index, 2.0, out=out), 2 * before) and torch.equal(lb.embedding_backward(x, index, 20, out=out), before)
        assert torch.equal(x, before)


def test_numbers_that_32_bits_do_not_hold():
    """Refused, not cut to 32 bits.  (Tensors without rows: they take no memory.)"""
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    for width in (1 << 31, (1 << 32) + 8):
        x = torch.empty(0, width, device="cuda")
        with pytest.raises(ValueError, match="elements"):
            lb.embedding(x, none)
        with pytest.raises(ValueError, match="elements"):
            lb.embedding_backward(x, none, 0)
    for top in ((1 << 32) + 1, (1 << 33) + 2, 3 - (1 << 32)):
        for n in (0, 2):
            with pytest.raises(RuntimeError):
                lb.log_probs(torch.zeros(n, 10, device="cuda"), top=top)
